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
// Bound by HBM and by the chain of a row's loads, sums and stores (8192 rows of 2048,
// bf16: forward with a residual 25 us, 0.80 of the measured copy rate, backward
// with dsum 26, 0.77, and 4 for the blocks' sums), by single elements more by the
// latter (2003 rows of 5001, fp32: forward 25 us, 0.48, backward 28, 0.64).  A row's
// two forward sums by one barrier, from the warps' means and centred squares: slower
// by its divisions (28 us); resident blocks with the next row ahead, where rows come
// by 16 bytes: 29.  Rows of odd widths by 16-byte groups with single elements at their
// ends: 32 and 46 (the ends' branches and selections in every row).
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

template <typename T>
struct FwdArgs {
  const T *x, *res;
  const float *w, *b;
  T *sum, *y;
  float2* stats;
  int64_t ldx, ldr, rows;
  int32_t d;
  float eps;
};

// kW warps per row, 8 kV elements per lane.
template <typename T, int kW, int kV, int kE>
__global__ void __launch_bounds__(threads(kW)) k_ln_fwd(const FwdArgs<T> g) {
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
  Lane<float, kW, kV, kE> w, b;
  x.load(g.x + row * g.ldx, wl, d);
  if (g.res) res.load(g.res + row * g.ldr, wl, d);
  w.load(g.w, wl, d);
  if (g.b) b.load(g.b, wl, d);
  float v[L::kGroups][kE], a[1] = {0.f};
#pragma unroll
  for (int i = 0; i < L::kGroups; ++i) {
    x.get(i, v[i]);
    if (g.res) {
      float r[kE];
      res.get(i, r);
#pragma unroll
      for (int e = 0; e < kE; ++e) v[i][e] = Elem<T>::to_f(Elem<T>::from_f(v[i][e] + r[e]));
    }
#pragma unroll
    for (int e = 0; e < kE; ++e) a[0] += v[i][e];   // (past the row: zeros)
    if (g.sum) L::put(g.sum + row * g.d, i, wl, d, v[i]);
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
  row_sums<kW>(a, red[1], warp, lane, grp);
  const float r = 1.f / sqrtf(a[0] / (float)g.d + g.eps);
  if (live && wl == 0 && g.stats) g.stats[row] = make_float2(mean, r);
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
  auto ask = [&](int64_t at) {
    const int d = at < g.rows ? g.d : 0;   // a row past the last one has no elements
    x.load(g.x + at * g.ldx, wl, d);
    if (g.res) res.load(g.res + at * g.ldr, wl, d);
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
#pragma unroll
    for (int i = 0; i < L::kGroups; ++i) {
      x.get(i, v[i]);
      if (g.res) {
        float r[kE];
        res.get(i, r);
#pragma unroll
        for (int e = 0; e < kE; ++e) v[i][e] = Elem<T>::to_f(Elem<T>::from_f(v[i][e] + r[e]));
      }
#pragma unroll
      for (int e = 0; e < kE; ++e) a[0] += v[i][e];   // (past the row: zeros)
    }
    if (base + stride < g.rows) ask(row + stride);
    if (g.sum)
#pragma unroll
      for (int i = 0; i < L::kGroups; ++i) L::put(g.sum + row * g.d, i, wl, d, v[i]);
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
    if (d && wl == 0 && g.stats) g.stats[row] = make_float2(mean, r);
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
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int grp = warp / kW, wl = threadIdx.x - grp * 32 * kW;
  pdl_trigger();
  pdl_wait();
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
#pragma unroll
        for (int e = 0; e < kE; ++e) {
          const float h = (sv[e] - mean) * r;
          dw[i][e] += tv[e] * h;
          db[i][e] += tv[e];
          tv[e] = r * (tv[e] * wv[e] - m0 - h * m1);
        }
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
        Lane<float, kW, kV, kE>::put(part, i, wl, g.d, v);   // (kE = 8: d is a multiple of 8)
      }
    }
  }
}

// dw and db = the blocks' sums: 32 columns a block, a run of blocks for each of
// its 32 warps, whose loads are all in flight at once.
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
#pragma unroll
    for (int q = 1; q < 32; ++q) a += s[q][lane];
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

template <typename T>
void forward(const FwdArgs<T>& a, cudaStream_t st) {
  const bool vec = a.d % 8 == 0 && aligned16(a.x, a.ldx, sizeof(T)) && aligned16(a.res, a.ldr, sizeof(T)) &&
                   aligned16(a.w, 0, 4) && aligned16(a.b, 0, 4) && aligned16(a.sum, 0, 4) && aligned16(a.y, 0, 4);
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
template <typename T>
void backward(const BwdArgs<T>& a, int blocks, cudaStream_t st) {
  const bool vec = a.d % 8 == 0 && aligned16(a.dy, a.lddy, sizeof(T)) && aligned16(a.s, a.lds, sizeof(T)) &&
                   aligned16(a.dsum, a.lddsum, sizeof(T)) && aligned16(a.dx, 0, 4);
  by_row(a.d, vec, [&](auto s, auto e) {
    launch_pdl(k_ln_bwd<T, s.w, s.v, e.value>, dim3((unsigned)blocks), dim3(threads(s.w)), 0, st, a);
  });
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
  if (precision == TP_FP32)
    forward(FwdArgs<float>{(const float*)x, (const float*)residual, w, b, (float*)sum, (float*)y, (float2*)stats, ldx, ldr,
                           rows, d, eps}, st);
  else
    forward(FwdArgs<__nv_bfloat16>{(const __nv_bfloat16*)x, (const __nv_bfloat16*)residual, w, b, (__nv_bfloat16*)sum,
                                   (__nv_bfloat16*)y, (float2*)stats, ldx, ldr, rows, d, eps}, st);
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
  const int blocks = bwd_blocks(rows, d);
  const bool sums = dw || db;
  const int64_t need = sums ? (int64_t)blocks * 2 * d * 4 : 0;
  if (need && (workspace_bytes < need || !workspace || ((uintptr_t)workspace & 255)))
    return ops_fail(TP_EINVAL, "a workspace of %lld bytes, 256-byte aligned, is needed", (long long)need);
  if ((s = ops_device()) != TP_OK) return s;
  float* part = sums ? (float*)workspace : nullptr;
  if (precision == TP_FP32)
    backward(BwdArgs<float>{(const float*)dy, (const float*)sum, (const float*)dsum, w, (const float2*)stats, (float*)dx,
                            part, lddy, lds, lddsum, rows, d}, blocks, st);
  else
    backward(BwdArgs<__nv_bfloat16>{(const __nv_bfloat16*)dy, (const __nv_bfloat16*)sum, (const __nv_bfloat16*)dsum, w,
                                    (const float2*)stats, (__nv_bfloat16*)dx, part, lddy, lds, lddsum, rows, d}, blocks, st);
  if (sums)
    launch_pdl(k_ln_dw, dim3((unsigned)ceil_div(2 * d, 32)), dim3(1024), 0, st, (const float*)part, blocks, d, dw, db);
  return done(cudaGetLastError(), "pack_layer_norm_backward");
}

}  // extern "C"
