// norm.cu -- RMS norm of a residual stream: forward with the residual's
// addition, output in the stream's type or in 8 bits with a scale per row,
// and its gradients (entry points in tabpack_ops.h).
//
//   s = x + residual,  n = s r w,  r = 1 / sqrt(mean(s^2) + eps)
//   dx = r (t - s r^2 mean(t s)) + dsum with t = dy w;  dw = sum_rows dy s r
//
// Bound by HBM: one pass, a row's elements stay in registers between the sums
// and the outputs.  A row takes one to eight warps, so that a lane holds at
// most 32 of its elements (64 above 8192).  dw is summed per block over the
// rows it takes (at most kBwdBlocks blocks), then over the blocks, both in a
// fixed order.
#include <algorithm>

#include "prod.cuh"

using namespace tp;

namespace {

constexpr int kThreads = 256;
constexpr int32_t kMaxD = 16384;
constexpr int64_t kMaxRows = (int64_t(1) << 31) - 256;
constexpr int kBwdBlocks = 2 * kSms;

__device__ __forceinline__ bool aligned16(const void* p, int64_t ld, int bytes) {
  return ((uintptr_t)p & 15) == 0 && ((ld * bytes) & 15) == 0;
}

// Eight elements of a row from column c on (zeros past d).
template <typename T>
__device__ __forceinline__ void load8(const T* p, int c, int d, bool vec, float (&v)[8]) {
  if (vec && c + 8 <= d) {
    if constexpr (sizeof(T) == 4) {
      const float4 a = *reinterpret_cast<const float4*>(p + c), b = *reinterpret_cast<const float4*>(p + c + 4);
      v[0] = a.x, v[1] = a.y, v[2] = a.z, v[3] = a.w, v[4] = b.x, v[5] = b.y, v[6] = b.z, v[7] = b.w;
    } else {
      const uint4 a = *reinterpret_cast<const uint4*>(p + c);
      const uint32_t u[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        v[2 * e] = __uint_as_float(u[e] << 16);
        v[2 * e + 1] = __uint_as_float(u[e] & 0xFFFF0000u);
      }
    }
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = c + e < d ? Elem<T>::to_f(p[c + e]) : 0.f;
  }
}
template <typename T>
__device__ __forceinline__ void store8(T* p, int c, int d, bool vec, const float (&v)[8]) {
  if (vec && c + 8 <= d) {
    if constexpr (sizeof(T) == 4) {
      *reinterpret_cast<float4*>(p + c) = make_float4(v[0], v[1], v[2], v[3]);
      *reinterpret_cast<float4*>(p + c + 4) = make_float4(v[4], v[5], v[6], v[7]);
    } else {
      uint32_t u[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const __nv_bfloat162 b = __floats2bfloat162_rn(v[2 * e], v[2 * e + 1]);
        u[e] = *reinterpret_cast<const uint32_t*>(&b);
      }
      *reinterpret_cast<uint4*>(p + c) = make_uint4(u[0], u[1], u[2], u[3]);
    }
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (c + e < d) p[c + e] = Elem<T>::from_f(v[e]);
  }
}

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

// kW warps per row, kV groups of eight elements per lane.
template <typename T, int kW, int kV>
__global__ void __launch_bounds__(kThreads) k_rms_fwd(const FwdArgs<T> g) {
  __shared__ float red[8];
  __shared__ uint32_t redu[8];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int grp = warp / kW, wl = threadIdx.x - grp * 32 * kW, d = g.d;
  const int64_t row = (int64_t)blockIdx.x * (8 / kW) + grp;
  const bool live = row < g.rows;
  const bool vx = aligned16(g.x, g.ldx, sizeof(T)), vr = aligned16(g.res, g.ldr, sizeof(T));
  const bool vw = aligned16(g.w, 0, 4), vs = aligned16(g.sum, d, sizeof(T)), vy = aligned16(g.y, d, sizeof(T));
  const bool vq = ((uintptr_t)g.q & 7) == 0 && (d & 7) == 0;
  pdl_trigger();
  pdl_wait();
  float v[kV][8];
  float ss = 0.f;
  if (live) {
#pragma unroll
    for (int i = 0; i < kV; ++i) {
      const int c = (i * 32 * kW + wl) * 8;
      load8(g.x + row * g.ldx, c, d, vx, v[i]);
    }
    if (g.res) {
#pragma unroll
      for (int i = 0; i < kV; ++i) {
        const int c = (i * 32 * kW + wl) * 8;
        float r[8];
        load8(g.res + row * g.ldr, c, d, vr, r);
#pragma unroll
        for (int e = 0; e < 8; ++e) v[i][e] += r[e];
      }
    }
    if (g.sum) {
#pragma unroll
      for (int i = 0; i < kV; ++i) store8(g.sum + row * d, (i * 32 * kW + wl) * 8, d, vs, v[i]);
    }
#pragma unroll
    for (int i = 0; i < kV; ++i)
#pragma unroll
      for (int e = 0; e < 8; ++e) ss += v[i][e] * v[i][e];
  }
  ss = warp_sum(ss);
  if constexpr (kW > 1) {
    if (lane == 0) red[warp] = ss;
    __syncthreads();
    ss = 0.f;
#pragma unroll
    for (int k = 0; k < kW; ++k) ss += red[grp * kW + k];
  }
  const float r = 1.f / sqrtf(ss / (float)d + g.eps);
  uint32_t top = 0;   // the largest |n|, as bits: a NaN is above infinity
  if (live) {
#pragma unroll
    for (int i = 0; i < kV; ++i) {
      const int c = (i * 32 * kW + wl) * 8;
      float w[8];
      load8(g.w, c, d, vw, w);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        v[i][e] = v[i][e] * r * w[e];
        if (c + e < d) top = max(top, __float_as_uint(v[i][e]) & 0x7FFFFFFFu);
      }
      if (g.y) store8(g.y + row * d, c, d, vy, v[i]);
    }
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
  if (!live) return;
  const bool finite = top < 0x7F800000u;
  const float scale = finite ? __uint_as_float(top) / 127.f : __uint_as_float(0x7FC00000u);
  if (wl == 0) g.scale[row] = scale;
  const bool some = finite && scale > 0.f;
  int8_t* q = g.q + row * d;
#pragma unroll
  for (int i = 0; i < kV; ++i) {
    const int c = (i * 32 * kW + wl) * 8;
    uint32_t b[8];
#pragma unroll
    for (int e = 0; e < 8; ++e)   // the clamp: a scale that lost bits below the normal numbers
      b[e] = some ? (uint32_t)(uint8_t)(int8_t)max(-127, min(127, __float2int_rn(v[i][e] / scale))) : 0u;
    if (vq && c + 8 <= d)
      *reinterpret_cast<uint2*>(q + c) = make_uint2(b[0] | b[1] << 8 | b[2] << 16 | b[3] << 24,
                                                    b[4] | b[5] << 8 | b[6] << 16 | b[7] << 24);
    else
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (c + e < d) q[c + e] = (int8_t)b[e];
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

template <typename T, int kW, int kV>
__global__ void __launch_bounds__(kThreads) k_rms_bwd(const BwdArgs<T> g) {
  constexpr int kRows = 8 / kW;            // rows at a time
  __shared__ float red[2][2][8];
  __shared__ float join[kRows > 1 ? kRows * 32 * kW * kV * 8 : 1];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int grp = warp / kW, wl = threadIdx.x - grp * 32 * kW, d = g.d;
  const bool vy = aligned16(g.dy, g.lddy, sizeof(T)), vs = aligned16(g.s, g.lds, sizeof(T));
  const bool vd = aligned16(g.dsum, g.lddsum, sizeof(T)), vw = aligned16(g.w, 0, 4), vx = aligned16(g.dx, d, sizeof(T));
  pdl_trigger();
  pdl_wait();
  float acc[kV][8];
#pragma unroll
  for (int i = 0; i < kV; ++i)
#pragma unroll
    for (int e = 0; e < 8; ++e) acc[i][e] = 0.f;
  int turn = 0;
  for (int64_t base = (int64_t)blockIdx.x * kRows; base < g.rows; base += (int64_t)gridDim.x * kRows, turn ^= 1) {
    const int64_t row = base + grp;
    const bool live = row < g.rows;
    float s[kV][8], t[kV][8];
    float ss = 0.f, ts = 0.f;
    if (live) {
#pragma unroll
      for (int i = 0; i < kV; ++i) {
        const int c = (i * 32 * kW + wl) * 8;
        load8(g.s + row * g.lds, c, d, vs, s[i]);
        load8(g.dy + row * g.lddy, c, d, vy, t[i]);
      }
#pragma unroll
      for (int i = 0; i < kV; ++i) {
        float w[8];
        load8(g.w, (i * 32 * kW + wl) * 8, d, vw, w);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          ss += s[i][e] * s[i][e];
          ts += t[i][e] * w[e] * s[i][e];
        }
      }
    }
    ss = warp_sum(ss);
    ts = warp_sum(ts);
    if constexpr (kW > 1) {
      // two sets of sums in turn: the next row's may be written while this row's are read
      if (lane == 0) red[turn][0][warp] = ss, red[turn][1][warp] = ts;
      __syncthreads();
      ss = ts = 0.f;
#pragma unroll
      for (int k = 0; k < kW; ++k) ss += red[turn][0][grp * kW + k], ts += red[turn][1][grp * kW + k];
    }
    if (live) {
      const float r = 1.f / sqrtf(ss / (float)d + g.eps);
      const float f = r * r * (ts / (float)d);
#pragma unroll
      for (int i = 0; i < kV; ++i) {
        const int c = (i * 32 * kW + wl) * 8;
        float w[8], o[8];
        load8(g.w, c, d, vw, w);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          o[e] = r * (t[i][e] * w[e] - s[i][e] * f);
          acc[i][e] += t[i][e] * s[i][e] * r;
        }
        if (g.dsum) {
          load8(g.dsum + row * g.lddsum, c, d, vd, w);
#pragma unroll
          for (int e = 0; e < 8; ++e) o[e] += w[e];
        }
        store8(g.dx + row * d, c, d, vx, o);
      }
    }
  }
  if (g.part == nullptr) return;
  float* part = g.part + (int64_t)blockIdx.x * d;
  if constexpr (kRows > 1) {
    constexpr int kCols = 32 * kW * kV * 8;
#pragma unroll
    for (int i = 0; i < kV; ++i)
#pragma unroll
      for (int e = 0; e < 8; ++e) join[grp * kCols + (i * 32 * kW + wl) * 8 + e] = acc[i][e];
    __syncthreads();
    for (int c = threadIdx.x; c < d; c += kThreads) {
      float a = join[c];
#pragma unroll
      for (int k = 1; k < kRows; ++k) a += join[k * kCols + c];
      part[c] = a;
    }
  } else {
#pragma unroll
    for (int i = 0; i < kV; ++i)
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const int c = (i * 32 * kW + wl) * 8 + e;
        if (c < d) part[c] = acc[i][e];
      }
  }
}

// dw = the blocks' sums: 32 columns a block, eight runs of blocks each.
__global__ void __launch_bounds__(256) k_rms_dw(const float* part, int n, int d, float* dw) {
  __shared__ float s[8][33];
  pdl_trigger();
  pdl_wait();
  const int lane = threadIdx.x & 31, k = threadIdx.x >> 5, c = blockIdx.x * 32 + lane;
  float a = 0.f;
  if (c < d)
#pragma unroll 4
    for (int b = k; b < n; b += 8) a += part[(int64_t)b * d + c];
  s[k][lane] = a;
  __syncthreads();
  if (k == 0 && c < d) {
#pragma unroll
    for (int q = 1; q < 8; ++q) a += s[q][lane];
    dw[c] = a;
  }
}

// Warps per row and groups per lane for a row of d elements.
template <typename F>
void by_width(int d, F f) {
  if (d <= 256) f(std::integral_constant<int, 1>(), std::integral_constant<int, 1>());
  else if (d <= 512) f(std::integral_constant<int, 1>(), std::integral_constant<int, 2>());
  else if (d <= 1024) f(std::integral_constant<int, 1>(), std::integral_constant<int, 4>());
  else if (d <= 2048) f(std::integral_constant<int, 2>(), std::integral_constant<int, 4>());
  else if (d <= 4096) f(std::integral_constant<int, 4>(), std::integral_constant<int, 4>());
  else if (d <= 8192) f(std::integral_constant<int, 8>(), std::integral_constant<int, 4>());
  else f(std::integral_constant<int, 8>(), std::integral_constant<int, 8>());
}
int rows_per_block(int d) { return d <= 1024 ? 8 : d <= 2048 ? 4 : d <= 4096 ? 2 : 1; }
int bwd_blocks(int64_t rows, int d) { return (int)std::min<int64_t>(ceil_div(rows, rows_per_block(d)), kBwdBlocks); }

template <typename T>
void forward(const FwdArgs<T>& a, cudaStream_t st) {
  by_width(a.d, [&](auto w, auto v) {
    launch_pdl(k_rms_fwd<T, w.value, v.value>, dim3((unsigned)ceil_div(a.rows, 8 / w.value)), dim3(kThreads), 0, st, a);
  });
}
template <typename T>
void backward(const BwdArgs<T>& a, cudaStream_t st) {
  by_width(a.d, [&](auto w, auto v) {
    launch_pdl(k_rms_bwd<T, w.value, v.value>, dim3((unsigned)bwd_blocks(a.rows, a.d)), dim3(kThreads), 0, st, a);
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
  if (dw) launch_pdl(k_rms_dw, dim3((unsigned)ceil_div(d, 32)), dim3(256), 0, st, (const float*)part, blocks, d, dw);
  return done(cudaGetLastError(), "pack_rms_norm_backward");
}

}  // extern "C"
