// rows.cuh -- products of a few rows (rows.cu) and the gated block's activations.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "tabpack_ops.h"
#include "tp_internal.cuh"

namespace tp {

// Up to this many rows the products stream the weights past the rows.
constexpr int kFewRows = 32;

// Can these products take x and w as they lie there (elem: bytes of an element)?
bool rows_fit(int64_t rows, const void* x, int64_t ldx, const void* w, int32_t k, int elem);
cudaError_t rows_gated(const void* x, int64_t ldx, const void* w_gu, int64_t rows, int32_t d, int32_t f, int act, void* h,
                       int64_t ldh, void* a, void* p, cudaStream_t st);
cudaError_t rows_plain(const void* x, int64_t ldx, const void* w, int64_t rows, int32_t k, int32_t n, void* y,
                       cudaStream_t st);
cudaError_t rows_quant(const int8_t* q, int64_t ldq, const float* sx, const int8_t* w, const float* sw, const float* bias,
                       int64_t rows, int32_t k, int32_t n, bool f32, void* y, cudaStream_t st);

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
  const float p = 0.5f * erfcf(-0.70710678118654752f * g);
  d = p + g * 0.39894228040143268f * (kF32 ? expf(-0.5f * g * g) : __expf(-0.5f * g * g));
  return g * p;
}

}  // namespace tp
