// lnorm.cu -- layer norm of a residual stream with its gradients (entry points
// in tabpack_ops.h).
//
//   s = x + residual (rounded to the stream's type),  m = mean(s),
//   r = 1 / sqrt(mean((s - m)^2) + eps),  h = (s - m) r,  y = h w + b
//   dx = r (t - mean(t) - h mean(t h)) + dsum with t = dy w
//   dw = sum_rows dy h,  db = sum_rows dy
//
// One pass: a row's elements stay in registers between its sums and its
// outputs, so the squares are those of the centred values (no difference of
// two large sums).  The norm is taken of s as it is stored: the statistics
// that are kept for the backward pass are then exactly those of the s that it
// reads, and it needs one round of sums per row instead of two.
//
// A sum of fp32 values is off by some 2^-24 of their size, which where a row is all but
// constant is more than its deviation (389 times 12345.6: h was 0.30 and not 0).  So what
// is summed is the difference from the row's first element q, exact where it is small:
//   u = s - q,  m = q + mean(u),  s - m = u - mean(u)
// whose error is of the size of the row's spread, whatever its mean.
//
// Bound by HBM and by the chain of a row's loads, sums and stores (8192 rows of 2048,
// bf16: forward with a residual 25 us, 0.80 of the measured copy rate, backward
// with dsum 26, 0.77, and 4 for the blocks' sums), by single elements more by the
// latter (2003 rows of 5001, fp32: forward 21 us, 0.56, backward 25, 0.72).  A row's
// two forward sums by one barrier, from the warps' means and centred squares: slower
// by its divisions (28 us); resident blocks with the next row ahead, where rows come
// by 16 bytes: 29.
#include <algorithm>
#include <type_traits>

#include "lanes.cuh"
#include "prod.cuh"

using namespace tp;

namespace {

constexpr int32_t kMaxD = 16384;
constexpr int64_t kMaxRows = (int64_t(1) << 31) - 256;
constexpr int kBwdBlocks = 2 * kSms;

// Warps per row and groups of eight elements per lane, so that few lanes idle.  By
// single elements, whose addresses and predicates take issue slots, a lane has
// eight, and a row more warps (2003 rows of 5001, fp32, backward: sixteen a lane 38
// us).
template <typename F>
void by_row(int d, bool vec, F f) {
  if (vec) {
    if (d > 4096 && d <= 5120) f(Width<10, 2>(), std::integral_constant<int, 8>());
    else if (d > 5120 && d <= 6144) f(Width<12, 2>(), std::integral_constant<int, 8>());
    else by_width(d, [&](auto s) { f(s, std::integral_constant<int, 8>()); });
    return;
  }
  using One = std::integral_constant<int, 1>;
  if (d <= 256) f(Width<1, 1>(), One());
  else if (d <= 512) f(Width<2, 1>(), One());
  else if (d <= 1024) f(Width<4, 1>(), One());
  else if (d <= 2048) f(Width<8, 1>(), One());
  else if (d <= 3584) f(Width<14, 1>(), One());
  else if (d <= 4096) f(Width<16, 1>(), One());
  else if (d <= 5120) f(Width<20, 1>(), One());
  else if (d <= 6144) f(Width<24, 1>(), One());
  else if (d <= 8192) f(Width<32, 1>(), One());
  else f(Width<32, 2>(), One());
}

// Sums of kN values over the kW warps of a row, in a fixed order; red: a set of
// [kN][32] that no one else writes before the next barrier but one.
template <int kW, int kN>
__device__ __forceinline__ void row_sums(float (&v)[kN], float (*red)[32], int warp, int lane, int grp) {
#pragma unroll
  for (int i = 0; i < kN; ++i) v[i] = warp_sum(v[i]);
  if constexpr (kW > 1) {
    if (lane == 0)
#pragma unroll
      for (int i = 0; i < kN; ++i) red[i][warp] = v[i];
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kN; ++i) {
      v[i] = 0.f;
#pragma unroll
      for (int k = 0; k < kW; ++k) v[i] += red[i][grp * kW + k];
    }
  }
}

// The element that a row's others are compared with: its first one, or 0 where that is so large that differences could
// overflow, or no number.
template <typename T>
struct Pivot {
  T x, res;
  __device__ __forceinline__ void load(const T* px, const T* pres, bool there) {
    x = there ? *px : Elem<T>::from_f(0.f);
    if (pres) res = there ? *pres : Elem<T>::from_f(0.f);
  }
  __device__ __forceinline__ float get(bool with_res) const {
    float q = Elem<T>::to_f(x);
    if (with_res) q = Elem<T>::to_f(Elem<T>::from_f(q + Elem<T>::to_f(res)));
    return fabsf(q) < 0x1p120f ? q : 0.f;
  }
};

template <typename T>
struct FwdArgs {
  const T *x, *res;
  const float *w, *b;
  T *sum, *y;
  float2* stats;
  int64_t ldx, ldr, rows;
  int32_t d;
  float eps;
  bool over;   // the sum is written over x or residual
};

// kW warps per row, 8 kV elements per lane.  Rows of sixteen warps ask for the weights late,
// which leaves the registers for a second block an SM (8192 x 8192: bf16 145 us, so
// 107; fp32 195, 166).
template <typename T, int kW, int kV, int kE>
__global__ void __launch_bounds__(threads(kW), kW == 16 && kV == 2 && kE == 8 ? 2 : 0) k_ln_fwd(const FwdArgs<T> g) {
  constexpr bool kLate = kW == 16 && kE == 8 && (kV == 2 || sizeof(T) == 4);
  using L = Lane<T, kW, kV, kE>;
  __shared__ float red[2][1][32];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int grp = warp / kW, wl = threadIdx.x - grp * 32 * kW;
  const int64_t row = (int64_t)blockIdx.x * (threads(kW) / 32 / kW) + grp;
  const bool live = row < g.rows;
  const int d = live ? g.d : 0;   // a row past the last one has no elements
  pdl_trigger();
  pdl_wait();
  L x, res;
  Pivot<T> first;
  Lane<float, kW, kV, kE> w, b;
  x.load(g.x + row * g.ldx, wl, d);
  if (g.res) res.load(g.res + row * g.ldr, wl, d);
  first.load(g.x + row * g.ldx, g.res ? g.res + row * g.ldr : nullptr, live);
  if (!kLate) {
    w.load(g.w, wl, d);
    if (g.b) b.load(g.b, wl, d);
  }
  float v[L::kGroups][kE], a[1] = {0.f};
  const float pivot = first.get(g.res != nullptr);
  if (g.over) __syncthreads();   // every warp has the row's first element
#pragma unroll
  for (int i = 0; i < L::kGroups; ++i) {
    x.get(i, v[i]);
    if (g.res) {
      float r[kE];
      res.get(i, r);
#pragma unroll
      for (int e = 0; e < kE; ++e) v[i][e] = Elem<T>::to_f(Elem<T>::from_f(v[i][e] + r[e]));
    }
    if (g.sum) L::put(g.sum + row * g.d, i, wl, d, v[i]);
#pragma unroll
    for (int e = 0; e < kE; ++e) {
      v[i][e] -= pivot;
      if (L::col(i, wl) < d) a[0] += v[i][e];
    }
  }
  row_sums<kW>(a, red[0], warp, lane, grp);
  const float mean = a[0] / (float)g.d;
  a[0] = 0.f;
#pragma unroll
  for (int i = 0; i < L::kGroups; ++i)
#pragma unroll
    for (int e = 0; e < kE; ++e) {
      v[i][e] -= mean;
      if (L::col(i, wl) < d) a[0] += v[i][e] * v[i][e];
    }
  if (kLate) {
    w.load(g.w, wl, d);
    if (g.b) b.load(g.b, wl, d);
  }
  row_sums<kW>(a, red[1], warp, lane, grp);
  const float r = 1.f / sqrtf(a[0] / (float)g.d + g.eps);
  if (live && wl == 0 && g.stats) g.stats[row] = make_float2(pivot + mean, r);
  if (!g.y) return;
#pragma unroll
  for (int i = 0; i < L::kGroups; ++i) {
    float wt[kE], bt[kE] = {};
    w.get(i, wt);
    if (g.b) b.get(i, bt);
#pragma unroll
    for (int e = 0; e < kE; ++e) v[i][e] = v[i][e] * r * wt[e] + bt[e];
    L::put(g.y + row * g.d, i, wl, d, v[i]);
  }
}

// Many rows by single elements: a block of the row's warps takes rows in turn,
// with the weights in shared memory and the next row asked for before this one is
// worked on.
constexpr int many_threads(int kW) { return kW == 1 ? 128 : 32 * kW; }
constexpr int many_blocks(int kW, int kV) {   // an SM: as many threads as leave the registers for a row and the next one
  const int n = 65536 / 48 / many_threads(kW);
  return n < 1 ? 1 : n < 16 ? n : 16;
}
template <typename T, int kW, int kV, int kE>
__global__ void __launch_bounds__(many_threads(kW), many_blocks(kW, kV)) k_ln_fwd_many(const FwdArgs<T> g) {
  static_assert(kE == 1, "one element at a time");
  using L = Lane<T, kW, kV, kE>;
  constexpr int kRows = many_threads(kW) / 32 / kW, kCols = 32 * kW * kV * 8;
  extern __shared__ __align__(16) float ws[];   // weights, then biases
  __shared__ float red[2][2][1][32];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int grp = warp / kW, wl = threadIdx.x - grp * 32 * kW;
  pdl_trigger();
  pdl_wait();
  const int64_t stride = (int64_t)gridDim.x * kRows;
  int64_t row = (int64_t)blockIdx.x * kRows + grp;
  L x, res;
  Pivot<T> first;
  auto ask = [&](int64_t at) {
    const int d = at < g.rows ? g.d : 0;   // a row past the last one has no elements
    x.load(g.x + at * g.ldx, wl, d);
    if (g.res) res.load(g.res + at * g.ldr, wl, d);
    first.load(g.x + at * g.ldx, g.res ? g.res + at * g.ldr : nullptr, d > 0);
  };
  ask(row);
  for (int c = threadIdx.x; c < kCols; c += many_threads(kW)) {
    ws[c] = c < g.d ? g.w[c] : 0.f;
    ws[kCols + c] = c < g.d && g.b ? g.b[c] : 0.f;
  }
  __syncthreads();
  int turn = 0;
  for (int64_t base = (int64_t)blockIdx.x * kRows; base < g.rows; base += stride, row += stride, turn ^= 1) {
    const int d = row < g.rows ? g.d : 0;
    float v[L::kGroups][kE], a[1] = {0.f};
    const float pivot = first.get(g.res != nullptr);
#pragma unroll
    for (int i = 0; i < L::kGroups; ++i) {
      x.get(i, v[i]);
      if (g.res) {
        float r[kE];
        res.get(i, r);
#pragma unroll
        for (int e = 0; e < kE; ++e) v[i][e] = Elem<T>::to_f(Elem<T>::from_f(v[i][e] + r[e]));
      }
    }
    if (base + stride < g.rows) ask(row + stride);
    if (g.sum)
#pragma unroll
      for (int i = 0; i < L::kGroups; ++i) L::put(g.sum + row * g.d, i, wl, d, v[i]);
#pragma unroll
    for (int i = 0; i < L::kGroups; ++i) {
      v[i][0] -= pivot;
      a[0] += L::col(i, wl) < g.d ? v[i][0] : 0.f;
    }
    // (two sets of sums in turn: the next row's may be written while these are read)
    row_sums<kW>(a, red[turn][0], warp, lane, grp);
    const float mean = a[0] / (float)g.d;
    a[0] = 0.f;
#pragma unroll
    for (int i = 0; i < L::kGroups; ++i) {
      v[i][0] -= mean;
      a[0] += L::col(i, wl) < g.d ? v[i][0] * v[i][0] : 0.f;
    }
    row_sums<kW>(a, red[turn][1], warp, lane, grp);
    const float r = 1.f / sqrtf(a[0] / (float)g.d + g.eps);
    if (d && wl == 0 && g.stats) g.stats[row] = make_float2(pivot + mean, r);
    if (g.y)
#pragma unroll
      for (int i = 0; i < L::kGroups; ++i) {
        const float *w = ws + L::col(i, wl), *b = w + kCols;
        v[i][0] = v[i][0] * r * w[0] + b[0];
        L::put(g.y + row * g.d, i, wl, d, v[i]);
      }
  }
}

template <typename T>
struct BwdArgs {
  const T *dy, *s, *dsum;
  const float* w;
  const float2* stats;
  T* dx;
  float* part;      // [gridDim.x][2 d]
  int64_t lddy, lds, lddsum, rows;
  int32_t d;
};

template <typename T, int kW, int kV, int kE>
__global__ void __launch_bounds__(threads(kW), kW > 8 && !(kW == 14 && kE == 1) ? 1 : 2) k_ln_bwd(const BwdArgs<T> g) {
  using L = Lane<T, kW, kV, kE>;
  constexpr int kRows = threads(kW) / 32 / kW;   // rows at a time
  constexpr int kCols = 32 * kW * kV * 8;
  __shared__ float red[2][2][32];
  __shared__ __align__(16) float join[kRows > 1 ? kRows * kCols : kCols];
  float* ws = join;   // first the weights, at the end the rows' sums
  // of the widest rows the sums stay in shared memory, a thread's side by side with its neighbours' (8192 rows of
  // 16384, where registers do not hold them: bf16 341 us, so 240; fp32 577, 433)
  constexpr bool kShared = kCols == kMaxD;
  __shared__ float4 sums[kShared ? 2 * kCols / 4 : 1];
  auto sum_at = [&](int half, int i, int h) -> float4& { return sums[(half * (kV * 2) + i * (kE / 4) + h) * threads(kW) + threadIdx.x]; };
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int grp = warp / kW, wl = threadIdx.x - grp * 32 * kW;
  pdl_trigger();
  pdl_wait();
  // the next rows are asked for before these are worked on, where there are registers for them
  constexpr bool kAhead = kE == 8 ? kV <= 2 && sizeof(T) == 2 : kV == 1 && kW < 32 && kW != 14;
  const int64_t stride = (int64_t)gridDim.x * kRows;
  int64_t row = (int64_t)blockIdx.x * kRows + grp;
  L s, t, o;
  float2 st;
  auto ask = [&](int64_t at) {
    const int d = at < g.rows ? g.d : 0;   // a row past the last one has no elements
    s.load(g.s + at * g.lds, wl, d);
    t.load(g.dy + at * g.lddy, wl, d);
    if (g.dsum) o.load(g.dsum + at * g.lddsum, wl, d);
    st = d ? g.stats[at] : make_float2(0.f, 0.f);
  };
  // (a few loads in flight: 100 rows of 4096, bf16, 9.5 us without, 7.9; all of them, 7.0, cost 8192 rows 61 instead of 50)
#pragma unroll 4
  for (int c = threadIdx.x; c < kCols; c += threads(kW)) ws[c] = c < g.d ? g.w[c] : 0.f;
  __syncthreads();
  auto weights = [&](int i, float (&v)[kE]) {
    const float* p = ws + L::col(i, wl);
    if constexpr (kE == 8) {
      const float4 a = reinterpret_cast<const float4*>(p)[0], b = reinterpret_cast<const float4*>(p)[1];
      v[0] = a.x, v[1] = a.y, v[2] = a.z, v[3] = a.w, v[4] = b.x, v[5] = b.y, v[6] = b.z, v[7] = b.w;
    } else {
      v[0] = p[0];
    }
  };
  float dw[L::kGroups][kE], db[L::kGroups][kE];
#pragma unroll
  for (int i = 0; i < L::kGroups; ++i)
#pragma unroll
    for (int e = 0; e < kE; ++e) dw[i][e] = db[i][e] = 0.f;
  if constexpr (kShared)
    for (int k = threadIdx.x; k < 2 * kCols / 4; k += threads(kW)) sums[k] = make_float4(0.f, 0.f, 0.f, 0.f);
  if (kAhead) ask(row);
  int turn = 0;
  for (int64_t base = (int64_t)blockIdx.x * kRows; base < g.rows; base += stride, row += stride, turn ^= 1) {
    const int d = row < g.rows ? g.d : 0;
    if (!kAhead) ask(row);
    const L sn = s, tn = t, on = o;   // these rows
    const float mean = st.x, r = st.y;
    if (kAhead && base + stride < g.rows) ask(row + stride);
    float a[2] = {0.f, 0.f};
#pragma unroll
    for (int i = 0; i < L::kGroups; ++i) {
      float sv[kE], tv[kE], wv[kE];
      sn.get(i, sv);
      tn.get(i, tv);
      weights(i, wv);
#pragma unroll
      for (int e = 0; e < kE; ++e) {   // (past the row dy is 0)
        const float q = tv[e] * wv[e];
        a[0] += q;
        a[1] += L::col(i, wl) < d ? q * ((sv[e] - mean) * r) : 0.f;
      }
    }
    // two sets of sums in turn: the next rows' may be written while these are read
    row_sums<kW>(a, red[turn], warp, lane, grp);
    const float m0 = a[0] / (float)g.d, m1 = a[1] / (float)g.d;
    if (d) {
#pragma unroll
      for (int i = 0; i < L::kGroups; ++i) {
        float sv[kE], tv[kE], wv[kE];
        sn.get(i, sv);
        tn.get(i, tv);
        weights(i, wv);
        float hv[kE];
#pragma unroll
        for (int e = 0; e < kE; ++e) hv[e] = (sv[e] - mean) * r;
        if constexpr (kShared && kE == 8) {
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            float4 &a = sum_at(0, i, h), &b = sum_at(1, i, h);
            const float *tq = tv + 4 * h, *hq = hv + 4 * h;
            a = make_float4(a.x + tq[0] * hq[0], a.y + tq[1] * hq[1], a.z + tq[2] * hq[2], a.w + tq[3] * hq[3]);
            b = make_float4(b.x + tq[0], b.y + tq[1], b.z + tq[2], b.w + tq[3]);
          }
        } else if constexpr (kShared) {
          float* one = reinterpret_cast<float*>(sums);
          one[i * threads(kW) + threadIdx.x] += tv[0] * hv[0];
          one[kCols + i * threads(kW) + threadIdx.x] += tv[0];
        } else {
#pragma unroll
          for (int e = 0; e < kE; ++e) dw[i][e] += tv[e] * hv[e], db[i][e] += tv[e];
        }
#pragma unroll
        for (int e = 0; e < kE; ++e) tv[e] = r * (tv[e] * wv[e] - m0 - hv[e] * m1);
        if (g.dsum) {
          on.get(i, sv);
#pragma unroll
          for (int e = 0; e < kE; ++e) tv[e] += sv[e];
        }
        L::put(g.dx + row * g.d, i, wl, d, tv);
      }
    }
  }
  if (g.part == nullptr) return;
#pragma unroll 1
  for (int half = 0; half < 2; ++half) {
    float* part = g.part + ((int64_t)blockIdx.x * 2 + half) * g.d;
    if constexpr (kRows > 1) {
      __syncthreads();   // the last readers of what is there
#pragma unroll
      for (int i = 0; i < L::kGroups; ++i)
#pragma unroll
        for (int e = 0; e < kE; ++e) join[grp * kCols + L::col(i, wl) + e] = half ? db[i][e] : dw[i][e];
      __syncthreads();
      for (int c = threadIdx.x; c < g.d; c += threads(kW)) {
        float a = join[c];
#pragma unroll
        for (int k = 1; k < kRows; ++k) a += join[k * kCols + c];
        part[c] = a;
      }
    } else {
#pragma unroll
      for (int i = 0; i < L::kGroups; ++i) {
        float v[kE];
#pragma unroll
        for (int e = 0; e < kE; ++e) v[e] = half ? db[i][e] : dw[i][e];
        if constexpr (kShared && kE == 8) {
          const float4 a = sum_at(half, i, 0), b = sum_at(half, i, 1);
          v[0] = a.x, v[1] = a.y, v[2] = a.z, v[3] = a.w, v[4] = b.x, v[5] = b.y, v[6] = b.z, v[7] = b.w;
        } else if constexpr (kShared) {
          v[0] = reinterpret_cast<const float*>(sums)[half * kCols + i * threads(kW) + threadIdx.x];
        }
        Lane<float, kW, kV, kE>::put(part, i, wl, g.d, v);   // (kE = 8: d is a multiple of 8)
      }
    }
  }
}

// ------------------------------------------------ rows of odd widths, packed
// Rows that start `off` elements past a multiple of 16 bytes, all matrices' alike (as
// packed rows of an odd width do): a row is taken as one that begins at that multiple.
// Loads are whole groups of eight; what of a row's first and last one is the rows'
// beside it is cleared, and the last row's last group, behind which the matrix ends,
// is read by elements.  A block's rows, a multiple of eight apart, have the same off.
// bf16 only, and only of many rows: 8192 rows of 4097, us, by single elements and so:
// forward 94, 68, backward 111, 71; of 7001: 157, 114 and 213, 110; 2000 rows of
// 4097: 25, 20 and 27, 25, of 2003: 11.1, 11.0 and 12.9, 17.3 (fp32, 8192 of 4097:
// 98, 95 and 94, 105; of 7001: 155, 179 and 229, 193).  Eight columns a lane and twice the
// warps: forward 86.  The first element's part in the forward times: 4 to 6 us of the 8192 rows.
using Half = __nv_bfloat16;
template <int kW>
struct OddLane {
  using L = Lane<Half, kW, 2, 8>;
  L in;
  static __device__ __forceinline__ bool full(int i, int wl, int off, int end) {
    return L::col(i, wl) >= off && L::col(i, wl) + 8 <= end;
  }
  // p: the multiple of 16 bytes; end = off + d, or 0 for no row; last: of the matrix
  __device__ __forceinline__ void load(const Half* p, int wl, int end, bool last) {
    if (!last) {
      in.load(p, wl, end);
      return;
    }
    in.load(p, wl, end & ~7);   // (the groups that end inside the row)
#pragma unroll
    for (int i = 0; i < L::kGroups; ++i)
      if (L::col(i, wl) < end && L::col(i, wl) + 8 > end) {
        uint32_t w[4] = {};
#pragma unroll
        for (int e = 0; e < 8; ++e)
          if (L::col(i, wl) + e < end) w[e >> 1] |= (uint32_t)__bfloat16_as_ushort(p[L::col(i, wl) + e]) << (16 * (e & 1));
        in.u[i][0] = make_uint4(w[0], w[1], w[2], w[3]);
      }
  }
  // nothing of the rows beside it
  __device__ __forceinline__ void clip(int wl, int off, int end) {
#pragma unroll
    for (int i = 0; i < L::kGroups; ++i)
      if (!full(i, wl, off, end)) {
        uint32_t w[4] = {in.u[i][0].x, in.u[i][0].y, in.u[i][0].z, in.u[i][0].w};
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int c = L::col(i, wl) + 2 * e;
          w[e] &= (c >= off && c < end ? 0xFFFFu : 0u) | (c + 1 >= off && c + 1 < end ? 0xFFFF0000u : 0u);
        }
        in.u[i][0] = make_uint4(w[0], w[1], w[2], w[3]);
      }
  }
  static __device__ __forceinline__ void put(Half* p, int i, int wl, int off, int end, const float (&v)[8]) {
    if (full(i, wl, off, end)) {
      L::put(p, i, wl, end, v);
    } else if (L::col(i, wl) < end) {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const int c = L::col(i, wl) + e;
        if (c >= off && c < end) p[c] = Elem<Half>::from_f(v[e]);
      }
    }
  }
};

constexpr int odd_blocks(int kW) { return 20 / kW < 1 ? 1 : 20 / kW; }   // an SM
template <int kW>
__global__ void __launch_bounds__(32 * kW, odd_blocks(kW)) k_ln_fwd_odd(const FwdArgs<Half> g) {
  using O = OddLane<kW>;
  using L = typename O::L;
  constexpr int kCols = 32 * kW * 16;
  extern __shared__ __align__(16) float ws[];   // weights, then biases, `off` places on
  __shared__ float red[2][2][1][32];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, wl = threadIdx.x;
  pdl_trigger();
  pdl_wait();
  int64_t row = blockIdx.x;
  const int off = (int)(((uintptr_t)(g.x + row * g.ldx) & 15) / sizeof(Half)), end = off + g.d;
  O x, res;
  Pivot<Half> first;
  auto ask = [&](int64_t at) {
    const int till = at < g.rows ? end : 0;
    x.load(g.x + at * g.ldx - off, wl, till, at == g.rows - 1);
    if (g.res) res.load(g.res + at * g.ldr - off, wl, till, at == g.rows - 1);
    first.load(g.x + at * g.ldx, g.res ? g.res + at * g.ldr : nullptr, till > 0);
  };
  ask(row);
  for (int c = threadIdx.x; c < kCols; c += 32 * kW) {
    const bool in = c >= off && c < end;
    ws[c] = in ? g.w[c - off] : 0.f;
    ws[kCols + c] = in && g.b ? g.b[c - off] : 0.f;
  }
  __syncthreads();
  int turn = 0;
  for (; row < g.rows; row += gridDim.x, turn ^= 1) {
    float v[L::kGroups][8], a[1] = {0.f};
    const float pivot = first.get(g.res != nullptr);
    x.clip(wl, off, end);
    if (g.res) res.clip(wl, off, end);
#pragma unroll
    for (int i = 0; i < L::kGroups; ++i) {
      x.in.get(i, v[i]);
      if (g.res) {
        float r[8];
        res.in.get(i, r);
#pragma unroll
        for (int e = 0; e < 8; ++e) v[i][e] = Elem<Half>::to_f(Elem<Half>::from_f(v[i][e] + r[e]));
      }
    }
    ask(row + gridDim.x);
    if (g.sum)
#pragma unroll
      for (int i = 0; i < L::kGroups; ++i) O::put(g.sum + row * g.d - off, i, wl, off, end, v[i]);
#pragma unroll
    for (int i = 0; i < L::kGroups; ++i) {
      const bool all = O::full(i, wl, off, end);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const int c = L::col(i, wl) + e;
        v[i][e] -= pivot;
        a[0] += all || (c >= off && c < end) ? v[i][e] : 0.f;
      }
    }
    row_sums<kW>(a, red[turn][0], warp, lane, 0);
    const float mean = a[0] / (float)g.d;
    a[0] = 0.f;
#pragma unroll
    for (int i = 0; i < L::kGroups; ++i) {
      const bool all = O::full(i, wl, off, end);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const int c = L::col(i, wl) + e;
        v[i][e] = all || (c >= off && c < end) ? v[i][e] - mean : 0.f;
        a[0] += v[i][e] * v[i][e];
      }
    }
    row_sums<kW>(a, red[turn][1], warp, lane, 0);
    const float r = 1.f / sqrtf(a[0] / (float)g.d + g.eps);
    if (threadIdx.x == 0 && g.stats) g.stats[row] = make_float2(pivot + mean, r);
    if (g.y)
#pragma unroll
      for (int i = 0; i < L::kGroups; ++i) {
        const float* w = ws + L::col(i, wl);
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const float4 w4 = reinterpret_cast<const float4*>(w)[h], b4 = reinterpret_cast<const float4*>(w + kCols)[h];
          v[i][4 * h] = v[i][4 * h] * r * w4.x + b4.x, v[i][4 * h + 1] = v[i][4 * h + 1] * r * w4.y + b4.y;
          v[i][4 * h + 2] = v[i][4 * h + 2] * r * w4.z + b4.z, v[i][4 * h + 3] = v[i][4 * h + 3] * r * w4.w + b4.w;
        }
        O::put(g.y + row * g.d - off, i, wl, off, end, v[i]);
      }
  }
}

template <int kW>
__global__ void __launch_bounds__(32 * kW, kW > 8 ? 1 : 2) k_ln_bwd_odd(const BwdArgs<Half> g) {
  using O = OddLane<kW>;
  using L = typename O::L;
  constexpr int kCols = 32 * kW * 16;
  extern __shared__ __align__(16) float ws[];   // weights, `off` places on
  __shared__ float red[2][2][32];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, wl = threadIdx.x;
  pdl_trigger();
  pdl_wait();
  int64_t row = blockIdx.x;
  const int off = (int)(((uintptr_t)(g.s + row * g.lds) & 15) / sizeof(Half)), end = off + g.d;
  O s, t, o;
  float2 st;
  auto ask = [&](int64_t at) {
    const int till = at < g.rows ? end : 0;
    const bool last = at == g.rows - 1;
    s.load(g.s + at * g.lds - off, wl, till, last);
    t.load(g.dy + at * g.lddy - off, wl, till, last);
    if (g.dsum) o.load(g.dsum + at * g.lddsum - off, wl, till, last);
    st = till ? g.stats[at] : make_float2(0.f, 0.f);
  };
  ask(row);
  for (int c = threadIdx.x; c < kCols; c += 32 * kW) ws[c] = c >= off && c < end ? g.w[c - off] : 0.f;
  __syncthreads();
  auto weights = [&](int i, float (&v)[8]) {
    const float4 a = reinterpret_cast<const float4*>(ws + L::col(i, wl))[0], b = reinterpret_cast<const float4*>(ws + L::col(i, wl))[1];
    v[0] = a.x, v[1] = a.y, v[2] = a.z, v[3] = a.w, v[4] = b.x, v[5] = b.y, v[6] = b.z, v[7] = b.w;
  };
  float dw[L::kGroups][8], db[L::kGroups][8];
#pragma unroll
  for (int i = 0; i < L::kGroups; ++i)
#pragma unroll
    for (int e = 0; e < 8; ++e) dw[i][e] = db[i][e] = 0.f;
  int turn = 0;
  for (; row < g.rows; row += gridDim.x, turn ^= 1) {
    O sn = s, tn = t;   // this row
    const O on = o;
    sn.clip(wl, off, end);
    tn.clip(wl, off, end);
    const float mean = st.x, r = st.y;
    ask(row + gridDim.x);
    float a[2] = {0.f, 0.f};
#pragma unroll
    for (int i = 0; i < L::kGroups; ++i) {   // (outside the row dy and the weights are 0)
      float sv[8], tv[8], wv[8];
      sn.in.get(i, sv);
      tn.in.get(i, tv);
      weights(i, wv);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float q = tv[e] * wv[e];
        a[0] += q;
        a[1] += q * ((sv[e] - mean) * r);
      }
    }
    row_sums<kW>(a, red[turn], warp, lane, 0);
    const float m0 = a[0] / (float)g.d, m1 = a[1] / (float)g.d;
#pragma unroll
    for (int i = 0; i < L::kGroups; ++i) {
      float sv[8], tv[8], wv[8];
      sn.in.get(i, sv);
      tn.in.get(i, tv);
      weights(i, wv);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float h = (sv[e] - mean) * r;
        dw[i][e] += tv[e] * h;
        db[i][e] += tv[e];
        tv[e] = r * (tv[e] * wv[e] - m0 - h * m1);
      }
      if (g.dsum) {
        on.in.get(i, sv);
#pragma unroll
        for (int e = 0; e < 8; ++e) tv[e] += sv[e];
      }
      O::put(g.dx + row * g.d - off, i, wl, off, end, tv);
    }
  }
  if (g.part == nullptr) return;
  float* part = g.part + (int64_t)blockIdx.x * 2 * g.d - off;
#pragma unroll
  for (int i = 0; i < L::kGroups; ++i)
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const int c = L::col(i, wl) + e;
      if (c >= off && c < end) part[c] = dw[i][e], part[g.d + c] = db[i][e];
    }
}

// dw and db = the blocks' sums: 32 columns a block, a run of blocks for each of
// its 32 warps, whose loads are all in flight at once.
// (Of fewer blocks than warps, a warp a block.)
__global__ void __launch_bounds__(1024) k_ln_dw(const float* part, int n, int d, float* dw, float* db) {
  __shared__ float s[32][33];
  pdl_trigger();
  pdl_wait();
  const int lane = threadIdx.x & 31, k = threadIdx.x >> 5, c = blockIdx.x * 32 + lane;
  float v[(kBwdBlocks + 31) / 32], a = 0.f;
#pragma unroll
  for (int i = 0; i < (kBwdBlocks + 31) / 32; ++i) {
    const int b = k + 32 * i;
    v[i] = c < 2 * d && b < n ? part[(int64_t)b * 2 * d + c] : 0.f;
  }
#pragma unroll
  for (int i = 0; i < (kBwdBlocks + 31) / 32; ++i) a += v[i];
  s[k][lane] = a;
  __syncthreads();
  if (k == 0 && c < 2 * d) {
#pragma unroll 31
    for (int q = 1; q < min(n, 32); ++q) a += s[q][lane];
    if (c >= d) {
      if (db) db[c - d] = a;
    } else if (dw) {
      dw[c] = a;
    }
  }
}

// As many blocks as run at once: two an SM, or one of the largest.  (Blocks that
// take several rows at a time may find none: they leave sums of 0.)
int bwd_blocks(int64_t rows, int d) { return (int)std::min<int64_t>(rows, d > 4096 ? kSms : kBwdBlocks); }

// Rows of the kernels for packed odd widths: wide ones, and enough of them (measured
// beside the kernels).
bool odd_width(int64_t rows, int d, bool back) {
  return d > 1024 && d <= 8192 - 8 && rows >= (back && d <= 4096 ? 4096 : 1024);
}
// Do this matrix's rows lie as those of a packed one do that starts at a multiple of 16 bytes?
bool odd_like(const void* p, int64_t ld, int64_t d) { return ((uintptr_t)p & 15) == 0 && (!p || (ld - d) % 8 == 0); }
template <typename F>
void by_odd(int d, F f) {
  if (d <= 2048 - 8) f(Width<4, 2>());
  else if (d <= 4096 - 8) f(Width<8, 2>());
  else if (d <= 5120 - 8) f(Width<10, 2>());
  else if (d <= 6144 - 8) f(Width<12, 2>());
  else f(Width<16, 2>());
}

template <typename T>
void forward(const FwdArgs<T>& a, cudaStream_t st) {
  const bool vec = a.d % 8 == 0 && aligned16(a.x, a.ldx, sizeof(T)) && aligned16(a.res, a.ldr, sizeof(T)) &&
                   aligned16(a.w, 0, 4) && aligned16(a.b, 0, 4) && aligned16(a.sum, 0, 4) && aligned16(a.y, 0, 4);
  if constexpr (sizeof(T) == 2) {
    if (!vec && odd_width(a.rows, a.d, false) && odd_like(a.x, a.ldx, a.d) && odd_like(a.res, a.ldr, a.d) &&
        odd_like(a.sum, a.d, a.d) && odd_like(a.y, a.d, a.d)) {
      by_odd(a.d, [&](auto s) {
        constexpr int smem = 2 * 32 * s.w * 16 * 4;
        static OncePerDevice once;
        once([] { return cudaFuncSetAttribute(k_ln_fwd_odd<decltype(s)::w>, cudaFuncAttributeMaxDynamicSharedMemorySize, 64 * 1024); });
        const unsigned blocks = (unsigned)std::min<int64_t>(a.rows, odd_blocks(s.w) * kSms) / 8 * 8;
        launch_pdl(k_ln_fwd_odd<s.w>, dim3(blocks), dim3(32 * s.w), smem, st, a);
      });
      return;
    }
  }
  by_row(a.d, vec, [&](auto s, auto e) {
    if constexpr (e.value == 1) {
      constexpr int kRows = many_threads(s.w) / 32 / s.w, smem = 2 * 32 * s.w * s.v * 8 * 4;
      const int64_t blocks = ceil_div(a.rows, kRows), most = many_blocks(s.w, s.v) * kSms;
      if (blocks > most && smem <= 64 * 1024) {
        if (smem + sizeof(float[2][2][1][32]) > 48 * 1024) {   // (with the kernel's static ones)
          static OncePerDevice once;
          once([] {
            return cudaFuncSetAttribute(k_ln_fwd_many<T, decltype(s)::w, decltype(s)::v, 1>,
                                        cudaFuncAttributeMaxDynamicSharedMemorySize, 64 * 1024);
          });
        }
        launch_pdl(k_ln_fwd_many<T, s.w, s.v, 1>, dim3((unsigned)most), dim3(many_threads(s.w)), smem, st, a);
        return;
      }
    }
    const dim3 grid((unsigned)ceil_div(a.rows, threads(s.w) / 32 / s.w)), block(threads(s.w));
    launch_pdl(k_ln_fwd<T, s.w, s.v, e.value>, grid, block, 0, st, a);
  });
}
// Returns the blocks, of at most `blocks`, that leave sums.
template <typename T>
int backward(const BwdArgs<T>& a, int blocks, cudaStream_t st) {
  const bool vec = a.d % 8 == 0 && aligned16(a.dy, a.lddy, sizeof(T)) && aligned16(a.s, a.lds, sizeof(T)) &&
                   aligned16(a.dsum, a.lddsum, sizeof(T)) && aligned16(a.dx, 0, 4);
  if constexpr (sizeof(T) == 2) {
    if (!vec && odd_width(a.rows, a.d, true) && odd_like(a.s, a.lds, a.d) && odd_like(a.dy, a.lddy, a.d) &&
        odd_like(a.dsum, a.lddsum, a.d) && odd_like(a.dx, a.d, a.d)) {
      blocks = blocks / 8 * 8;
      by_odd(a.d, [&](auto s) {
        launch_pdl(k_ln_bwd_odd<s.w>, dim3((unsigned)blocks), dim3(32 * s.w), 32 * s.w * 16 * 4, st, a);
      });
      return blocks;
    }
  }
  by_row(a.d, vec, [&](auto s, auto e) {
    launch_pdl(k_ln_bwd<T, s.w, s.v, e.value>, dim3((unsigned)blocks), dim3(threads(s.w)), 0, st, a);
  });
  return blocks;
}

tp_status check(int64_t rows, int32_t d, int32_t precision) {
  if (rows < 0 || rows > kMaxRows) return ops_fail(TP_EINVAL, "rows %lld out of range", (long long)rows);
  if (d < 1 || d > kMaxD) return ops_fail(TP_EINVAL, "d %d must be in 1..%d", d, kMaxD);
  if (precision != TP_BF16 && precision != TP_FP32) return ops_fail(TP_EINVAL, "unknown precision %d", precision);
  return TP_OK;
}

tp_status done(cudaError_t e, const char* who) {
  if (e == cudaSuccess) return TP_OK;
  cudaGetLastError();   // reported here
  return ops_fail(TP_ECUDA, "%s: %s", who, cudaGetErrorString(e));
}

}  // namespace

extern "C" {

tp_status pack_layer_norm(const void* x, int64_t ldx, const void* residual, int64_t ldr, const float* w, const float* b,
                          int64_t rows, int32_t d, float eps, int32_t precision, void* sum, void* y, float* stats,
                          void* cuda_stream) {
  tp_status s = check(rows, d, precision);
  if (s != TP_OK) return s;
  if (!(eps >= 0.f)) return ops_fail(TP_EINVAL, "eps must not be negative");
  if (ldx < d || (residual && ldr < d)) return ops_fail(TP_EINVAL, "ldx and ldr must not be less than d %d", d);
  if (rows == 0) return TP_OK;
  if (!x || !w || !(sum || y || stats)) return ops_fail(TP_EINVAL, "null argument");
  if ((uintptr_t)stats & 7) return ops_fail(TP_EINVAL, "stats must be 8-byte aligned");
  if ((s = ops_device()) != TP_OK) return s;
  cudaStream_t st = (cudaStream_t)cuda_stream;
  const bool over = sum && (sum == x || sum == residual);
  if (precision == TP_FP32)
    forward(FwdArgs<float>{(const float*)x, (const float*)residual, w, b, (float*)sum, (float*)y, (float2*)stats, ldx, ldr,
                           rows, d, eps, over}, st);
  else
    forward(FwdArgs<__nv_bfloat16>{(const __nv_bfloat16*)x, (const __nv_bfloat16*)residual, w, b, (__nv_bfloat16*)sum,
                                   (__nv_bfloat16*)y, (float2*)stats, ldx, ldr, rows, d, eps, over}, st);
  return done(cudaGetLastError(), "pack_layer_norm");
}

tp_status pack_layer_norm_bytes(int64_t rows, int32_t d, int64_t* backward_bytes) {
  const tp_status s = check(rows, d, TP_BF16);
  if (s != TP_OK) return s;
  if (!backward_bytes) return ops_fail(TP_EINVAL, "null argument");
  *backward_bytes = (int64_t)bwd_blocks(rows, d) * 2 * d * 4;
  return TP_OK;
}

tp_status pack_layer_norm_backward(const void* dy, int64_t lddy, const void* sum, int64_t lds, const float* w,
                                   const float* stats, const void* dsum, int64_t lddsum, int64_t rows, int32_t d,
                                   int32_t precision, void* dx, float* dw, float* db, void* workspace,
                                   int64_t workspace_bytes, void* cuda_stream) {
  tp_status s = check(rows, d, precision);
  if (s != TP_OK) return s;
  if (lddy < d || lds < d || (dsum && lddsum < d))
    return ops_fail(TP_EINVAL, "lddy, lds and lddsum must not be less than d %d", d);
  cudaStream_t st = (cudaStream_t)cuda_stream;
  if (rows == 0) {   // sums over no rows
    if (!dw && !db) return TP_OK;
    if ((s = ops_device()) != TP_OK) return s;
    cudaError_t e = dw ? cudaMemsetAsync(dw, 0, (size_t)d * 4, st) : cudaSuccess;
    if (e == cudaSuccess && db) e = cudaMemsetAsync(db, 0, (size_t)d * 4, st);
    return done(e, "pack_layer_norm_backward");
  }
  if (!dy || !sum || !w || !stats || !dx) return ops_fail(TP_EINVAL, "null argument");
  if ((uintptr_t)stats & 7) return ops_fail(TP_EINVAL, "stats must be 8-byte aligned");
  int blocks = bwd_blocks(rows, d);
  const bool sums = dw || db;
  const int64_t need = sums ? (int64_t)blocks * 2 * d * 4 : 0;
  if (need && (workspace_bytes < need || !workspace || ((uintptr_t)workspace & 255)))
    return ops_fail(TP_EINVAL, "a workspace of %lld bytes, 256-byte aligned, is needed", (long long)need);
  if ((s = ops_device()) != TP_OK) return s;
  float* part = sums ? (float*)workspace : nullptr;
  if (precision == TP_FP32)
    blocks = backward(BwdArgs<float>{(const float*)dy, (const float*)sum, (const float*)dsum, w, (const float2*)stats, (float*)dx,
                            part, lddy, lds, lddsum, rows, d}, blocks, st);
  else
    blocks = backward(BwdArgs<__nv_bfloat16>{(const __nv_bfloat16*)dy, (const __nv_bfloat16*)sum, (const __nv_bfloat16*)dsum, w,
                                    (const float2*)stats, (__nv_bfloat16*)dx, part, lddy, lds, lddsum, rows, d}, blocks, st);
  if (sums)
    launch_pdl(k_ln_dw, dim3((unsigned)ceil_div(2 * d, 32)), dim3(32 * std::min(blocks, 32)), 0, st, (const float*)part, blocks, d, dw, db);
  return done(cudaGetLastError(), "pack_layer_norm_backward");
}

}  // extern "C"
