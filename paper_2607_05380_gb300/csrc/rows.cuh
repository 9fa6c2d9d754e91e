// rows.cuh -- products of a few rows (rows.cu) and the gated block's activations.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "tabpack_ops.h"
#include "tp_internal.cuh"

namespace tp {

// Do these products take `rows` rows against this many weights, in rows of
// `pitch` bytes (or of several pitches, or'ed)?  Measured against the tcgen05
// products (device time of a call, us, rows / tcgen05):
//   gated block, d = d_out = 512, f = 2048: 64 rows 7.8 / 12.4, 192 rows 15.2 / 14.2
//   d = d_out = 1024, f = 2048: 32 rows 7.9 / 15.3, 128 rows 15.7 / 16.3
//   d = d_out = 2048, f = 4096: 32 rows 18.4 / 25.5, 64 rows 27.3 / 26.1
//   d = d_out = 256, f = 512: 512 rows 7.4 / 10.5, 1024 rows 11.9 / 10.6
//   8-bit product, 2048 -> 4096: 128 rows 13.2 / 20.6, 256 rows 23.6 / 21.3
//   1024 -> 1000: 256 rows 5.0 / 11.0, 768 rows 12.8 / 11.5
// Loads of four bytes (gated 1022, 2046: 64 rows 19.5 / 22.5, 128 rows 26.1 /
// 23.7) or of an element (gated 389, 1001: 32 rows 11.9 / 14.8, 128 rows 17.0 /
// 15.3; 8-bit 2001 -> 1000: 8 rows 8.4 / 12.1, 16 rows 12.0, 28 rows 20.6, 32 rows
// 21.9 / 14.0) pay for less; the limit for elements lets more rows through than
// those figures would (up to 29 of 2001 -> 1000).  Only the weights' pitch counts
// here: rows of x at an odd pitch or address make k_rows load both by elements
// (gated 1024, 2048: 64 rows 25 instead of 10.5).
bool rows_take(int64_t rows, int64_t weights, int64_t pitch, bool q8);
// The same of a 32-bit block, in fp32 multiply-adds (rows / tcgen05):
//   d = d_out = 512, f = 2048: 8 rows 15.8 / 42, 64 rows 32 / 40
//   1024, 2048: 32 rows 31 / 44, 48 rows 50 / 44
//   2048, 4096: one row 27 / 131, 16 rows 72 / 100, 24 rows 106 / 100
//   389, 1001: 64 rows 26 / 40
bool rows_take32(int64_t rows, int64_t weights);

struct RowsGated {
  const void *x, *w_gu;
  int64_t ldx, rows;
  int32_t d, f, act;
  bool f32;
  void* h;                 // [rows, f] in the block's type, pitch ldh
  int64_t ldh;
  void *a, *p, *parts;     // kept for the backward pass (NULL: nothing), pitch ld_keep: act(g), u act'(g) and,
  int64_t ld_keep, part;   // of a 32-bit block, h as bf16 parts `part` elements apart; of a bf16 block 24-bit
  uint8_t *a_lo, *p_lo;    // floats, their lower 8 bits here
};
cudaError_t rows_gated(const RowsGated& q, cudaStream_t st);
cudaError_t rows_plain(const void* x, int64_t ldx, const void* w, int64_t rows, int32_t k, int32_t n, bool f32, void* y,
                       cudaStream_t st);
cudaError_t rows_quant(const int8_t* q, int64_t ldq, const float* sx, const int8_t* w, const float* sw, const float* bias,
                       int64_t rows, int32_t k, int32_t n, bool f32, void* y, cudaStream_t st);

// Four int8 as two pairs of fp16: 1024 + (v + 128) has v + 128 in its low bits.
__device__ __forceinline__ void s8_to_f16(uint32_t v, uint32_t& lo, uint32_t& hi) {
  v ^= 0x80808080u;
  const __half2 bias = __halves2half2(__ushort_as_half(0x6480), __ushort_as_half(0x6480));   // 1152
  uint32_t a = __byte_perm(v, 0x64646464u, 0x4140), b = __byte_perm(v, 0x64646464u, 0x4342);
  __half2 x = __hsub2(*reinterpret_cast<__half2*>(&a), bias), y = __hsub2(*reinterpret_cast<__half2*>(&b), bias);
  lo = *reinterpret_cast<uint32_t*>(&x);
  hi = *reinterpret_cast<uint32_t*>(&y);
}

// Two 32-bit values' first bf16 parts (a's in the lower half): finite ones stay
// finite, where rounding to nearest makes an infinity of what is above bf16's
// largest number (3.39e38); the parts after it hold the rest, and an infinity or
// a NaN again.
__device__ __forceinline__ uint32_t first_parts(float a, float b) {
  uint32_t r;
  asm("cvt.rn.satfinite.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(b), "f"(a));
  return r;
}

// The upper 24 bits of a float, rounded to nearest (ties up), in bits 8..31.
__device__ __forceinline__ uint32_t round_24(float v) {
  const uint32_t u = __float_as_uint(v);
  return (u & 0x7F800000u) == 0x7F800000u ? u | (u & 0xFFu ? 0x100u : 0u) : u + 0x80u;   // (a NaN stays one)
}

// act(g) and act'(g); the exponential and the quotient to 2 ulp where the
// results are rounded to bf16.  The activation is a template parameter: all
// three in one unrolled chunk of 32 did not fit the instruction caches (a
// 20011 x 1024 -> 4096 forward pass, 478 us against 340 us).
template <int kAct, bool kF32>
__device__ __forceinline__ float act_value(float g, float& d) {
  if constexpr (kAct == TP_ACT_RELU) {
    d = g > 0.f ? 1.f : 0.f;
    return g != g ? g : fmaxf(g, 0.f);
  }
  if constexpr (kAct == TP_ACT_SILU) {
    const float s = kF32 ? 1.f / (1.f + expf(-g)) : __fdividef(1.f, 1.f + __expf(-g));
    d = s * (1.f + g * (1.f - s));
    return g * s;
  }
  const float e = kF32 ? expf(-0.5f * g * g) : __expf(-0.5f * g * g);
  float p;   // Phi(g)
  if constexpr (kF32) {
    p = 0.5f * erfcf(-0.70710678118654752f * g);
  } else {
    // Phi(-v) = exp(-v^2 / 2) t (c0 + c1 t + ... + c6 t^6), t = 1 / (1 + 0.365 v), v >= 0: the polynomial was fitted to
    // erfcx(v / sqrt 2) / (2 t) over v <= 14.5 by least squares reweighted towards the least largest relative
    // error, 1.2e-6 in fp32, so that act(g) keeps its digits out to where it vanishes; its exponential is act' 's
    const float t = __fdividef(1.f, fmaf(0.365f, fabsf(g), 1.f));
    float q = fmaf(t, 0.0481844135f, -0.17675133f);
    q = fmaf(t, q, 0.165481776f);
    q = fmaf(t, q, 0.0351994522f);
    q = fmaf(t, q, 0.137966141f);
    q = fmaf(t, q, 0.144241735f);
    q = fmaf(t, q, 0.145678267f);
    q *= t * e;
    p = g < 0.f ? q : 1.f - q;
  }
  d = fmaf(g * 0.39894228040143268f, e, p);
  return g * p;
}

}  // namespace tp
