// dropout.cu -- dropout whose mask is computed where it is applied and never
// stored (entry point in tabpack_ops.h).
//
//   y(r, c) = x(r, c) / (1 - p) if word c & 3 of Philox4x32-10 at counter
//   (r, c >> 2, step, site) under key seed is not below floor(p 2^32), else 0;
//   plus residual(r, c)
//
// the rule of a pack's own masks.  The gradient is the same map of dy.
//
// Bound by HBM, and in bf16 nearly as much by the generator: 32 bits an
// element are 20 multiplier pairs for four of them.  Of those, what depends on
// the row alone or on the column alone is computed once for the several that a
// thread takes: the first round and half of the next two.  8192 x 2048, bf16: with
// a residual 20 us (0.75 of the copy rate), without 17 (0.58); without the
// generator 33 for both instead of 37.  Products of 64 bits instead of their two
// halves apart: the same or slower.
#include <algorithm>

#include "lanes.cuh"
#include "prod.cuh"

using namespace tp;

namespace {

constexpr int32_t kMaxD = 1 << 17;
constexpr int64_t kMaxRows = (int64_t(1) << 31) - 256, kMaxElems = int64_t(1) << 40;

template <typename T>
struct Args {
  const T *x, *res;
  T* y;
  int64_t ldx, ldr, rows;
  int32_t d, shift;      // a row takes 2^shift threads of a block
  uint32_t k0, k1, step, site, drop;
  float up;
};

// Round 1 of (row, col, step, site): (x0 ^ col, w1, w2, w3); round 2: (v0, v1, v2 = hi(Ma (x0 ^ col)) ^ x2, v3 = lo(Ma (x0
// ^ col))); round 3: (hi(Mb v2) ^ y0, lo(Mb v2), v3 ^ y2, y3).  What of it a row decides, and what a column.
struct RowPart {
  uint32_t x2, y0, y2, y3;
  __device__ __forceinline__ RowPart(uint32_t row, uint32_t step, uint32_t site, uint32_t k0, uint32_t k1) {
    const uint32_t w1 = kPhiloxMb * step, w2 = __umulhi(kPhiloxMa, row) ^ site ^ k1, w3 = kPhiloxMa * row;
    const uint32_t v0 = __umulhi(kPhiloxMb, w2) ^ w1 ^ (k0 + kPhiloxWa), v1 = kPhiloxMb * w2;
    x2 = w3 ^ (k1 + kPhiloxWb);
    y0 = v1 ^ (k0 + 2u * kPhiloxWa);
    y2 = __umulhi(kPhiloxMa, v0) ^ (k1 + 2u * kPhiloxWb), y3 = kPhiloxMa * v0;
  }
};
struct ColPart {
  uint32_t hi, v3;
  __device__ __forceinline__ ColPart(uint32_t col, uint32_t step, uint32_t k0) {
    const uint32_t c = __umulhi(kPhiloxMb, step) ^ k0 ^ col;
    hi = __umulhi(kPhiloxMa, c), v3 = kPhiloxMa * c;
  }
};
__device__ __forceinline__ U4 draw4(const RowPart& r, const ColPart& c, uint32_t k0, uint32_t k1) {
  const uint32_t v2 = c.hi ^ r.x2;
  return philox_rounds<7>(__umulhi(kPhiloxMb, v2) ^ r.y0, kPhiloxMb * v2, c.v3 ^ r.y2, r.y3, k0 + 3u * kPhiloxWa,
                          k1 + 3u * kPhiloxWb);
}

template <typename T>
__device__ __forceinline__ void drop8(const Args<T>& g, float (&v)[8], const RowPart& r, const ColPart (&c)[2]) {
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const U4 w = draw4(r, c[h], g.k0, g.k1);
    v[4 * h] = w.x >= g.drop ? v[4 * h] * g.up : 0.f;
    v[4 * h + 1] = w.y >= g.drop ? v[4 * h + 1] * g.up : 0.f;
    v[4 * h + 2] = w.z >= g.drop ? v[4 * h + 2] * g.up : 0.f;
    v[4 * h + 3] = w.w >= g.drop ? v[4 * h + 3] * g.up : 0.f;
  }
}

template <typename T>
constexpr int drop_blocks() { return sizeof(T) == 2 ? 6 : 5; }   // an SM
// Eight columns a thread, loads and stores of 16 bytes, the next row asked for
// before this one is worked on.  A block's threads are one row's (kWide: what a row
// decides is then computed by the uniform units, once a warp) or several rows'.
template <typename T, bool kWide>
__global__ void __launch_bounds__(256, drop_blocks<T>()) k_drop8(const Args<T> g) {
  using L = Lane<T, 1, 1, 8>;
  const int tx = kWide ? threadIdx.x : threadIdx.x & ((1 << g.shift) - 1), ty = kWide ? 0 : threadIdx.x >> g.shift;
  const int rows_at_once = kWide ? 1 : 256 >> g.shift;
  const int c = 8 * (blockIdx.x * (1 << g.shift) + tx);
  pdl_trigger();
  const ColPart cols[2] = {ColPart((uint32_t)c >> 2, g.step, g.k0), ColPart(((uint32_t)c >> 2) + 1, g.step, g.k0)};
  pdl_wait();
  if (c >= g.d) return;
  const int64_t step = (int64_t)gridDim.y * rows_at_once;
  int64_t row = (int64_t)blockIdx.y * rows_at_once + ty;
  L x, res;
  auto ask = [&](int64_t r) {
    const int there = r < g.rows ? 8 : 0;
    x.load(g.x + r * g.ldx + c, 0, there);
    if (g.res) res.load(g.res + r * g.ldr + c, 0, there);
  };
  ask(row);
  for (; row < g.rows; row += step) {
    float v[8], w[8];
    x.get(0, v);
    if (g.res) res.get(0, w);
    ask(row + step);
    if (g.drop) drop8(g, v, RowPart((uint32_t)row, g.step, g.site, g.k0, g.k1), cols);
    if (g.res) {
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] += w[e];
    }
    L::put(g.y + row * g.d + c, 0, 0, 8, v);
  }
}

// Any alignment: a warp takes 128 columns of a row, 32 side by side at a time,
// whose words come from the eight lanes that have drawn them.
template <typename T>
__global__ void __launch_bounds__(256) k_drop1(const Args<T> g) {
  const int lane = threadIdx.x & 31, wide = (g.d + 127) >> 7;
  const int64_t total = g.rows * wide;
  pdl_trigger();
  pdl_wait();
  for (int64_t at = (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5); at < total; at += (int64_t)gridDim.x * 8) {
    const int64_t row = total >> 31 ? at / wide : (int64_t)((uint32_t)at / (uint32_t)wide);
    const int c0 = (int)(at - row * wide) * 128;
    T x[4], r[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int c = c0 + 32 * i + lane;
      x[i] = c < g.d ? g.x[row * g.ldx + c] : Elem<T>::from_f(0.f);
      r[i] = c < g.d && g.res ? g.res[row * g.ldr + c] : Elem<T>::from_f(0.f);
    }
    uint32_t keep = 0xFu;
    if (g.drop) {
      const U4 w = draw4(RowPart((uint32_t)row, g.step, g.site, g.k0, g.k1),
                         ColPart(((uint32_t)c0 >> 2) + lane, g.step, g.k0), g.k0, g.k1);
      keep = (uint32_t)(w.x >= g.drop) | (uint32_t)(w.y >= g.drop) << 1 | (uint32_t)(w.z >= g.drop) << 2 |
             (uint32_t)(w.w >= g.drop) << 3;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int c = c0 + 32 * i + lane;
      const uint32_t k = __shfl_sync(0xffffffffu, keep, 8 * i + (lane >> 2)) >> (lane & 3) & 1;
      float v = !g.drop ? Elem<T>::to_f(x[i]) : k ? Elem<T>::to_f(x[i]) * g.up : 0.f;
      if (g.res) v += Elem<T>::to_f(r[i]);
      if (c < g.d) g.y[row * g.d + c] = Elem<T>::from_f(v);
    }
  }
}

template <typename T>
void run(Args<T> a, cudaStream_t st) {
  const bool vec = a.d % 8 == 0 && aligned16(a.x, a.ldx, sizeof(T)) && aligned16(a.res, a.ldr, sizeof(T)) && aligned16(a.y, 0, 4);
  if (vec) {
    a.shift = 0;
    while (a.shift < 8 && (8 << a.shift) < a.d) ++a.shift;
    const bool wide = a.shift >= 5;
    const int64_t across = ceil_div(a.d, 8 << a.shift), at_once = wide ? 1 : 256 >> a.shift;
    // as many blocks as run at once (8192 x 2048, bf16, both passes: 37 us; a block a row 41)
    const int64_t most = std::max<int64_t>(1, drop_blocks<T>() * (wide ? 256 >> a.shift : 1) * kSms / across);
    const dim3 grid((unsigned)across, (unsigned)std::min<int64_t>(std::min<int64_t>(ceil_div(a.rows, at_once), most), 65535));
    if (wide) launch_pdl(k_drop8<T, true>, grid, dim3(1u << a.shift), 0, st, a);
    else launch_pdl(k_drop8<T, false>, grid, dim3(256), 0, st, a);
  } else {
    const int64_t blocks = ceil_div(a.rows * ceil_div(a.d, 128), 8);
    launch_pdl(k_drop1<T>, dim3((unsigned)std::min<int64_t>(blocks, 8 * kSms)), dim3(256), 0, st, a);
  }
}

}  // namespace

extern "C" {

tp_status pack_dropout(const void* x, int64_t ldx, const void* residual, int64_t ldr, int64_t rows, int32_t d, float p,
                       uint64_t seed, uint32_t step, uint32_t site, int32_t precision, void* y, void* cuda_stream) {
  if (rows < 0 || rows > kMaxRows) return ops_fail(TP_EINVAL, "rows %lld out of range", (long long)rows);
  if (d < 1 || d > kMaxD) return ops_fail(TP_EINVAL, "d %d must be in 1..%d", d, kMaxD);
  if (rows * d > kMaxElems) return ops_fail(TP_EINVAL, "more than 2^40 elements in a matrix");
  if (!(p >= 0.f && p < 1.f)) return ops_fail(TP_EINVAL, "p must be in [0, 1)");
  if (precision != TP_BF16 && precision != TP_FP32) return ops_fail(TP_EINVAL, "unknown precision %d", precision);
  if (ldx < d || (residual && ldr < d)) return ops_fail(TP_EINVAL, "ldx and ldr must not be less than d %d", d);
  if (rows == 0) return TP_OK;
  if (!x || !y) return ops_fail(TP_EINVAL, "null argument");
  const tp_status s = ops_device();
  if (s != TP_OK) return s;
  cudaStream_t st = (cudaStream_t)cuda_stream;
  const uint32_t drop = (uint32_t)((double)p * 4294967296.0);   // (a float below 1: at most 2^32 - 256)
  const float up = (float)(1.0 / (1.0 - (double)p));
  if (precision == TP_FP32)
    run(Args<float>{(const float*)x, (const float*)residual, (float*)y, ldx, ldr, rows, d, 0, (uint32_t)seed,
                    (uint32_t)(seed >> 32), step, site, drop, up}, st);
  else
    run(Args<__nv_bfloat16>{(const __nv_bfloat16*)x, (const __nv_bfloat16*)residual, (__nv_bfloat16*)y, ldx, ldr, rows, d, 0,
                            (uint32_t)seed, (uint32_t)(seed >> 32), step, site, drop, up}, st);
  const cudaError_t e = cudaGetLastError();
  return e == cudaSuccess ? TP_OK : ops_fail(TP_ECUDA, "pack_dropout: %s", cudaGetErrorString(e));
}

}  // extern "C"
