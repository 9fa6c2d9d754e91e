// lanes.cuh -- rows of a matrix spread over the lanes of one to sixteen warps,
// for the kernels that keep a row in registers between its sums and its
// outputs (norm.cu, lnorm.cu).
#pragma once

#include <cuda_bf16.h>

#include "tp_internal.cuh"

namespace tp {

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
inline int rows_per_block(int d) { return d <= 512 ? 8 : d <= 1024 ? 4 : d <= 2048 ? 2 : 1; }

}  // namespace tp
