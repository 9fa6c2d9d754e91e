// norm.cu -- RMS norm of a residual stream: forward with the residual's
// addition, output in the stream's type or in 8 bits with a scale per row,
// and its gradients (entry points in tabpack_ops.h).
//
//   s = x + residual,  n = s r w,  r = 1 / sqrt(mean(s^2) + eps)
//   dx = r (t - s r^2 mean(t s)) + dsum with t = dy w;  dw = sum_rows dy s r
//
// One pass: a row's elements stay in registers between the sums and the
// outputs.  Bound by HBM (8192 rows of 2048, forward with a residual: bf16 22 us,
// 0.91 of the measured copy rate, fp32 40 us, 0.98) and, in the backward pass,
// by its two sums per row, which the next row's loads do not quite cover (bf16
// without dsum 23.6 us, 0.63, with it 29 us, 0.68; fp32, which asks for no
// row ahead, 44 and 50 us, 0.67 and 0.80).  Above 8192 columns the backward pass
// has no registers left (1024 rows of 16384, with dsum: bf16 45 us, 0.44; fp32 75
// us, 0.53).
//
// A row takes one to sixteen warps, so that a lane holds at most 16 of its
// elements, 32 above 8192 (forward / backward without dsum, bf16, us, when adding
// up dw took 2.7 more: 8192 rows of 2048, two warps 24 / 31, four 22 / 26.5,
// eight 22 / 31; 16384 of 1024, one warp 23.5 / 40, two 21 / 25, four 25 / 30).
// dw is summed per block over the rows it takes (at most kBwdBlocks blocks), then
// over the blocks, both in a fixed order.
#include <algorithm>

#include "prod.cuh"

using namespace tp;

namespace {

constexpr int32_t kMaxD = 16384;
constexpr int64_t kMaxRows = (int64_t(1) << 31) - 256;
constexpr int kBwdBlocks = 2 * kSms;
constexpr int threads(int warps_per_row) { return warps_per_row > 8 ? 32 * warps_per_row : 256; }

inline bool aligned16(const void* p, int64_t ld, int bytes) {
  return ((uintptr_t)p & 15) == 0 && ((ld * bytes) & 15) == 0;
}

// A lane's elements of a row: kV * 8 of them, as groups of kE = 8 at columns
// (i * lanes + lane) * 8 where every address is a multiple of 16 bytes and d
// of 8, else one by one.  A group is inside the row or past it (zeros): the
// loads are predicated, not branched around, so that all are in flight at
// once (8192 rows of 2048, bf16, forward: 90 us with a branch per group).
// They stay as they were read, so that a row that is asked for ahead costs a
// register per two bf16 elements.
template <typename T, int kW, int kV, int kE>
struct Lane {
  static constexpr int kGroups = kV * 8 / kE, kU = kE == 8 ? (int)sizeof(T) / 2 : 0;
  uint4 u[kGroups][kU ? kU : 1];   // kE = 8
  T one[kGroups];                  // kE = 1
  static __device__ __forceinline__ int col(int i, int wl) { return (i * 32 * kW + wl) * kE; }
  __device__ __forceinline__ void load(const T* p, int wl, int d) {
#pragma unroll
    for (int i = 0; i < kGroups; ++i) {
      const int c = col(i, wl);
      if constexpr (kE == 8) {
#pragma unroll
        for (int h = 0; h < kU; ++h)
          u[i][h] = c < d ? *(reinterpret_cast<const uint4*>(p + c) + h) : make_uint4(0u, 0u, 0u, 0u);
      } else {
        one[i] = c < d ? p[c] : Elem<T>::from_f(0.f);
      }
    }
  }
  __device__ __forceinline__ void get(int i, float (&v)[kE]) const {
    if constexpr (kE == 8) {
#pragma unroll
      for (int h = 0; h < kU; ++h) {
        const uint32_t w[4] = {u[i][h].x, u[i][h].y, u[i][h].z, u[i][h].w};
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          if constexpr (sizeof(T) == 4) {
            v[4 * h + e] = __uint_as_float(w[e]);
          } else {
            v[2 * e] = __uint_as_float(w[e] << 16);
            v[2 * e + 1] = __uint_as_float(w[e] & 0xFFFF0000u);
          }
        }
      }
    } else {
      v[0] = Elem<T>::to_f(one[i]);
    }
  }
  // group i of a row, from fp32
  static __device__ __forceinline__ void put(T* p, int i, int wl, int d, const float (&v)[kE]) {
    if (col(i, wl) >= d) return;
    T* o = p + col(i, wl);
    if constexpr (kE == 1) {
      o[0] = Elem<T>::from_f(v[0]);
    } else if constexpr (sizeof(T) == 4) {
      reinterpret_cast<float4*>(o)[0] = make_float4(v[0], v[1], v[2], v[3]);
      reinterpret_cast<float4*>(o)[1] = make_float4(v[4], v[5], v[6], v[7]);
    } else {
      uint32_t w[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const __nv_bfloat162 b = __floats2bfloat162_rn(v[2 * e], v[2 * e + 1]);
        w[e] = *reinterpret_cast<const uint32_t*>(&b);
      }
      *reinterpret_cast<uint4*>(o) = make_uint4(w[0], w[1], w[2], w[3]);
    }
  }
};

__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}
__device__ __forceinline__ uint32_t warp_max(uint32_t v) { return __reduce_max_sync(0xffffffffu, v); }

template <typename T>
struct FwdArgs {
  const T *x, *res;
  const float* w;
  T *sum, *y;
  int8_t* q;
  float* scale;
  int64_t ldx, ldr, rows;
  int32_t d;
  float eps;
};

// kW warps per row, 8 kV elements per lane.
template <typename T, int kW, int kV, int kE>
__global__ void __launch_bounds__(threads(kW)) k_rms_fwd(const FwdArgs<T> g) {
  using L = Lane<T, kW, kV, kE>;
  __shared__ float red[16];
  __shared__ uint32_t redu[16];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int grp = warp / kW, wl = threadIdx.x - grp * 32 * kW;
  const int64_t row = (int64_t)blockIdx.x * (threads(kW) / 32 / kW) + grp;
  const bool live = row < g.rows;
  const int d = live ? g.d : 0;   // a row past the last one has no elements
  pdl_trigger();
  pdl_wait();
  L x, res;
  Lane<float, kW, kV, kE> w;
  x.load(g.x + row * g.ldx, wl, d);
  if (g.res) res.load(g.res + row * g.ldr, wl, d);
  w.load(g.w, wl, d);
  float v[L::kGroups][kE], ss = 0.f;
#pragma unroll
  for (int i = 0; i < L::kGroups; ++i) {
    x.get(i, v[i]);
    if (g.res) {
      float r[kE];
      res.get(i, r);
#pragma unroll
      for (int e = 0; e < kE; ++e) v[i][e] += r[e];
    }
#pragma unroll
    for (int e = 0; e < kE; ++e) ss += v[i][e] * v[i][e];
    if (g.sum) L::put(g.sum + row * d, i, wl, d, v[i]);
  }
  ss = warp_sum(ss);
  if constexpr (kW > 1) {
    if (lane == 0) red[warp] = ss;
    __syncthreads();
    ss = 0.f;
#pragma unroll
    for (int k = 0; k < kW; ++k) ss += red[grp * kW + k];
  }
  const float r = 1.f / sqrtf(ss / (float)g.d + g.eps);
  uint32_t top = 0;   // the largest |n|, as bits: a NaN is above infinity
#pragma unroll
  for (int i = 0; i < L::kGroups; ++i) {
    float wt[kE];
    w.get(i, wt);
#pragma unroll
    for (int e = 0; e < kE; ++e) {
      v[i][e] = v[i][e] * r * wt[e];
      // (past the row: 0, or NaN where r is infinite, which is kept out)
      if (L::col(i, wl) < d) top = max(top, __float_as_uint(v[i][e]) & 0x7FFFFFFFu);
    }
    if (g.y) L::put(g.y + row * d, i, wl, d, v[i]);
  }
  if (g.q == nullptr) return;
  top = warp_max(top);
  if constexpr (kW > 1) {
    if (lane == 0) redu[warp] = top;
    __syncthreads();
    top = 0;
#pragma unroll
    for (int k = 0; k < kW; ++k) top = max(top, redu[grp * kW + k]);
  }
  const bool finite = top < 0x7F800000u;
  const float scale = finite ? __uint_as_float(top) / 127.f : __uint_as_float(0x7FC00000u);
  if (live && wl == 0) g.scale[row] = scale;
  // n times a rounded reciprocal, rounded to an integer by adding 1.5 2^23 (whose low byte it then is).  Where what is
  // left of n is not clearly less than half a scale (4 values in 10^5), and in rows of scale 0 or next to it or with
  // a NaN, the side of the tie above the integer below is taken from a multiply-add whose sign is exact; an
  // integer off by one because the quotient is next to it leads to the same answer.  (That way for all: 20011 x 1024
  // 30.9 us.)
  const bool some = finite && scale > 0.f, usual = top >= 0x10000000u && finite;
  const float up = usual ? 1.f : 18446744073709551616.f, unit = scale * up;   // (1 / scale might overflow)
  const float inv = some ? 1.f / unit : 0.f, edge = usual ? 0.49998f * scale : 0.f;
  int8_t* q = g.q + row * d;
#pragma unroll
  for (int i = 0; i < L::kGroups; ++i) {
    if (L::col(i, wl) >= d) continue;
    uint32_t b[kE];
    bool near = false;
#pragma unroll
    for (int e = 0; e < kE; ++e) {
      const float m = fmaf(v[i][e], inv, 12582912.f);
      near |= !(fabsf(fmaf(12582912.f - m, scale, v[i][e])) < edge);
      b[e] = __float_as_uint(m) & 0xFFu;
    }
    if (near) {
#pragma unroll
      for (int e = 0; e < kE; ++e) {
        const float n = v[i][e] * up;
        int k = __float2int_rd(n * inv);
        const float over = fmaf(-((float)k + 0.5f), unit, n);
        k += over > 0.f || (over == 0.f && (k & 1));
        // (a scale below the normal numbers may be up to half too small)
        b[e] = some ? (uint32_t)max(-127, min(k, 127)) & 0xFFu : 0u;
      }
    }
    if constexpr (kE == 8)
      *reinterpret_cast<uint2*>(q + L::col(i, wl)) = make_uint2(b[0] | b[1] << 8 | b[2] << 16 | b[3] << 24,
                                                                b[4] | b[5] << 8 | b[6] << 16 | b[7] << 24);
    else
      q[L::col(i, wl)] = (int8_t)b[0];
  }
}

template <typename T>
struct BwdArgs {
  const T *dy, *s, *dsum;
  const float* w;
  T* dx;
  float* part;      // [gridDim.x][d]
  int64_t lddy, lds, lddsum, rows;
  int32_t d;
  float eps;
};

template <typename T, int kW, int kV, int kE>
__global__ void __launch_bounds__(threads(kW), kW > 8 ? 1 : 2) k_rms_bwd(const BwdArgs<T> g) {
  using L = Lane<T, kW, kV, kE>;
  constexpr int kRows = threads(kW) / 32 / kW;   // rows at a time
  constexpr int kCols = 32 * kW * kV * 8;
  __shared__ float red[2][2][16];
  __shared__ __align__(16) float join[kRows > 1 ? kRows * kCols : kCols];
  float* ws = join;   // first the weights, at the end the rows' sums
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int grp = warp / kW, wl = threadIdx.x - grp * 32 * kW;
  pdl_trigger();
  pdl_wait();
  // the weights stay in shared memory: the rows ahead need the registers
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
  float acc[L::kGroups][kE];
#pragma unroll
  for (int i = 0; i < L::kGroups; ++i)
#pragma unroll
    for (int e = 0; e < kE; ++e) acc[i][e] = 0.f;
  // bf16: the next rows are asked for before these are worked on (8192 x 2048: 37 -> 32 us)
  constexpr bool kAhead = sizeof(T) == 2 && kV <= 2 && kE == 8;
  const int64_t stride = (int64_t)gridDim.x * kRows;
  int64_t row = (int64_t)blockIdx.x * kRows + grp;
  L s, t, o;
  auto ask = [&](int64_t at) {
    const int d = at < g.rows ? g.d : 0;   // a row past the last one has no elements
    s.load(g.s + at * g.lds, wl, d);
    t.load(g.dy + at * g.lddy, wl, d);
    if (g.dsum) o.load(g.dsum + at * g.lddsum, wl, d);
  };
  if (kAhead) ask(row);
  int turn = 0;
  for (int64_t base = (int64_t)blockIdx.x * kRows; base < g.rows; base += stride, row += stride, turn ^= 1) {
    const int d = row < g.rows ? g.d : 0;
    if (!kAhead) ask(row);
    const L sn = s, tn = t, on = o;   // these rows
    if (kAhead && base + stride < g.rows) ask(row + stride);
    float ss = 0.f, ts = 0.f;
#pragma unroll
    for (int i = 0; i < L::kGroups; ++i) {
      float sv[kE], tv[kE], wv[kE];
      sn.get(i, sv);
      tn.get(i, tv);
      weights(i, wv);
#pragma unroll
      for (int e = 0; e < kE; ++e) {
        ss += sv[e] * sv[e];
        ts += tv[e] * wv[e] * sv[e];
      }
    }
    ss = warp_sum(ss);
    ts = warp_sum(ts);
    if constexpr (kW > 1) {
      // two sets of sums in turn: the next rows' may be written while these are read
      if (lane == 0) red[turn][0][warp] = ss, red[turn][1][warp] = ts;
      __syncthreads();
      ss = ts = 0.f;
#pragma unroll
      for (int k = 0; k < kW; ++k) ss += red[turn][0][grp * kW + k], ts += red[turn][1][grp * kW + k];
    }
    const float r = 1.f / sqrtf(ss / (float)g.d + g.eps);
    const float f = r * r * (ts / (float)g.d);
    if (d) {
#pragma unroll
      for (int i = 0; i < L::kGroups; ++i) {
        float sv[kE], tv[kE], wv[kE];
        sn.get(i, sv);
        tn.get(i, tv);
        weights(i, wv);
#pragma unroll
        for (int e = 0; e < kE; ++e) {
          acc[i][e] += tv[e] * sv[e] * r;
          tv[e] = r * (tv[e] * wv[e] - sv[e] * f);
        }
        if (g.dsum) {
          on.get(i, sv);
#pragma unroll
          for (int e = 0; e < kE; ++e) tv[e] += sv[e];
        }
        L::put(g.dx + row * d, i, wl, d, tv);
      }
    }
  }
  if (g.part == nullptr) return;
  float* part = g.part + (int64_t)blockIdx.x * g.d;
  if constexpr (kRows > 1) {
    __syncthreads();   // the weights' last readers
#pragma unroll
    for (int i = 0; i < L::kGroups; ++i)
#pragma unroll
      for (int e = 0; e < kE; ++e) join[grp * kCols + L::col(i, wl) + e] = acc[i][e];
    __syncthreads();
    for (int c = threadIdx.x; c < g.d; c += threads(kW)) {
      float a = join[c];
#pragma unroll
      for (int k = 1; k < kRows; ++k) a += join[k * kCols + c];
      part[c] = a;
    }
  } else {
#pragma unroll
    for (int i = 0; i < L::kGroups; ++i) Lane<float, kW, kV, kE>::put(part, i, wl, g.d, acc[i]);
  }
}

// dw = the blocks' sums: 32 columns a block, a run of blocks for each of its 32
// warps, whose loads are all in flight at once (the backward pass of 8192 rows
// of 2048: with eight warps a block 26.3 us, so 23.6).
__global__ void __launch_bounds__(1024) k_rms_dw(const float* part, int n, int d, float* dw) {
  __shared__ float s[32][33];
  pdl_trigger();
  pdl_wait();
  const int lane = threadIdx.x & 31, k = threadIdx.x >> 5, c = blockIdx.x * 32 + lane;
  float v[(kBwdBlocks + 31) / 32], a = 0.f;
#pragma unroll
  for (int i = 0; i < (kBwdBlocks + 31) / 32; ++i) {
    const int b = k + 32 * i;
    v[i] = c < d && b < n ? part[(int64_t)b * d + c] : 0.f;
  }
#pragma unroll
  for (int i = 0; i < (kBwdBlocks + 31) / 32; ++i) a += v[i];
  s[k][lane] = a;
  __syncthreads();
  if (k == 0 && c < d) {
#pragma unroll
    for (int q = 1; q < 32; ++q) a += s[q][lane];
    dw[c] = a;
  }
}

// Warps per row and groups of eight per lane for a row of d elements.
template <int kW, int kV>
struct Width {
  static constexpr int w = kW, v = kV;
};
template <typename F>
void by_width(int d, F f) {
  if (d <= 256) f(Width<1, 1>());
  else if (d <= 512) f(Width<1, 2>());
  else if (d <= 1024) f(Width<2, 2>());
  else if (d <= 2048) f(Width<4, 2>());
  else if (d <= 4096) f(Width<8, 2>());
  else if (d <= 8192) f(Width<16, 2>());
  else f(Width<16, 4>());
}
int rows_per_block(int d) { return d <= 512 ? 8 : d <= 1024 ? 4 : d <= 2048 ? 2 : 1; }
int bwd_blocks(int64_t rows, int d) { return (int)std::min<int64_t>(ceil_div(rows, rows_per_block(d)), kBwdBlocks); }

template <typename T>
void forward(const FwdArgs<T>& a, cudaStream_t st) {
  const bool vec = a.d % 8 == 0 && aligned16(a.x, a.ldx, sizeof(T)) && aligned16(a.res, a.ldr, sizeof(T)) &&
                   aligned16(a.w, 0, 4) && aligned16(a.sum, 0, 4) && aligned16(a.y, 0, 4) && ((uintptr_t)a.q & 7) == 0;
  by_width(a.d, [&](auto s) {
    const dim3 grid((unsigned)ceil_div(a.rows, rows_per_block(a.d))), block(threads(s.w));
    if (vec) launch_pdl(k_rms_fwd<T, s.w, s.v, 8>, grid, block, 0, st, a);
    else launch_pdl(k_rms_fwd<T, s.w, s.v, 1>, grid, block, 0, st, a);
  });
}
template <typename T>
void backward(const BwdArgs<T>& a, cudaStream_t st) {
  const bool vec = a.d % 8 == 0 && aligned16(a.dy, a.lddy, sizeof(T)) && aligned16(a.s, a.lds, sizeof(T)) &&
                   aligned16(a.dsum, a.lddsum, sizeof(T)) && aligned16(a.w, 0, 4) && aligned16(a.dx, 0, 4);
  by_width(a.d, [&](auto s) {
    const dim3 grid((unsigned)bwd_blocks(a.rows, a.d)), block(threads(s.w));
    if (vec) launch_pdl(k_rms_bwd<T, s.w, s.v, 8>, grid, block, 0, st, a);
    else launch_pdl(k_rms_bwd<T, s.w, s.v, 1>, grid, block, 0, st, a);
  });
}

tp_status check(int64_t rows, int32_t d, float eps, int32_t precision) {
  if (rows < 0 || rows > kMaxRows) return ops_fail(TP_EINVAL, "rows %lld out of range", (long long)rows);
  if (d < 1 || d > kMaxD) return ops_fail(TP_EINVAL, "d %d must be in 1..%d", d, kMaxD);
  if (!(eps >= 0.f)) return ops_fail(TP_EINVAL, "eps must not be negative");
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

tp_status pack_rms_norm(const void* x, int64_t ldx, const void* residual, int64_t ldr, const float* w, int64_t rows,
                        int32_t d, float eps, int32_t precision, void* sum, void* y, int8_t* q, float* scale,
                        void* cuda_stream) {
  tp_status s = check(rows, d, eps, precision);
  if (s != TP_OK) return s;
  if (ldx < d || (residual && ldr < d)) return ops_fail(TP_EINVAL, "ldx and ldr must not be less than d %d", d);
  if ((q == nullptr) != (scale == nullptr)) return ops_fail(TP_EINVAL, "q and scale go together");
  if (rows == 0) return TP_OK;
  if (!x || !w || !(sum || y || q)) return ops_fail(TP_EINVAL, "null argument");
  if ((s = ops_device()) != TP_OK) return s;
  cudaStream_t st = (cudaStream_t)cuda_stream;
  if (precision == TP_FP32)
    forward(FwdArgs<float>{(const float*)x, (const float*)residual, w, (float*)sum, (float*)y, q, scale, ldx, ldr, rows, d,
                           eps}, st);
  else
    forward(FwdArgs<__nv_bfloat16>{(const __nv_bfloat16*)x, (const __nv_bfloat16*)residual, w, (__nv_bfloat16*)sum,
                                   (__nv_bfloat16*)y, q, scale, ldx, ldr, rows, d, eps}, st);
  return done(cudaGetLastError(), "pack_rms_norm");
}

tp_status pack_rms_norm_bytes(int64_t rows, int32_t d, int64_t* backward_bytes) {
  const tp_status s = check(rows, d, 0.f, TP_BF16);
  if (s != TP_OK) return s;
  if (!backward_bytes) return ops_fail(TP_EINVAL, "null argument");
  *backward_bytes = (int64_t)bwd_blocks(rows, d) * d * 4;
  return TP_OK;
}

tp_status pack_rms_norm_backward(const void* dy, int64_t lddy, const void* sum, int64_t lds, const float* w,
                                 const void* dsum, int64_t lddsum, int64_t rows, int32_t d, float eps,
                                 int32_t precision, void* dx, float* dw, void* workspace, int64_t workspace_bytes,
                                 void* cuda_stream) {
  tp_status s = check(rows, d, eps, precision);
  if (s != TP_OK) return s;
  if (lddy < d || lds < d || (dsum && lddsum < d))
    return ops_fail(TP_EINVAL, "lddy, lds and lddsum must not be less than d %d", d);
  cudaStream_t st = (cudaStream_t)cuda_stream;
  if (rows == 0) {   // a sum over no rows
    if (!dw) return TP_OK;
    if ((s = ops_device()) != TP_OK) return s;
    return done(cudaMemsetAsync(dw, 0, (size_t)d * 4, st), "pack_rms_norm_backward");
  }
  if (!dy || !sum || !w || !dx) return ops_fail(TP_EINVAL, "null argument");
  const int blocks = bwd_blocks(rows, d);
  const int64_t need = dw ? (int64_t)blocks * d * 4 : 0;
  if (need && (workspace_bytes < need || !workspace || ((uintptr_t)workspace & 255)))
    return ops_fail(TP_EINVAL, "a workspace of %lld bytes, 256-byte aligned, is needed", (long long)need);
  if ((s = ops_device()) != TP_OK) return s;
  float* part = dw ? (float*)workspace : nullptr;
  if (precision == TP_FP32)
    backward(BwdArgs<float>{(const float*)dy, (const float*)sum, (const float*)dsum, w, (float*)dx, part, lddy, lds, lddsum,
                            rows, d, eps}, st);
  else
    backward(BwdArgs<__nv_bfloat16>{(const __nv_bfloat16*)dy, (const __nv_bfloat16*)sum, (const __nv_bfloat16*)dsum, w,
                                    (__nv_bfloat16*)dx, part, lddy, lds, lddsum, rows, d, eps}, st);
  if (dw) launch_pdl(k_rms_dw, dim3((unsigned)ceil_div(d, 32)), dim3(1024), 0, st, (const float*)part, blocks, d, dw);
  return done(cudaGetLastError(), "pack_rms_norm_backward");
}

}  // extern "C"
