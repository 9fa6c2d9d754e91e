// f8.cu -- products in 8-bit floating point (e4m3) with a scale for each block of
// 128, and the quantisation that makes such operands (entry points in
// tabpack_ops.h).
//
//   scale = max |x| / 448 of a block, q = the e4m3 number nearest to x / scale
//   y[r, c] = sum_b scale[r, b] w_scale[c / 128, b] sum_{k in block b} q[r, k] w[c, k] + bias[c]
//
// The product: a persistent tcgen05 launch (kind::f8f6f4).  A scale block is a K
// block: its 128 bytes a row are one swizzled line of shared memory and four
// MMAs.  Every K block has an accumulator of its own in TMEM, of two to four in
// turn; the epilogue warps read it while the next ones are made, and add it, times
// its row's and its column block's scale, to their fp32 sums in registers.  So the
// scales cost a multiply-add an element and K block beside the MMAs, and the
// tensor cores' own chains are four instructions long.
//
// 8192 x 4096 -> 4096 by CTA pairs of 256 x 256: 130 us, 2.11 PFLOP/s, 1.10 of
// cuBLAS's measured bf16 burst.  MMAs and operands alone take 71 us; handing the
// accumulators over adds 23, reading them 12, the multiply-adds 22, looking at the scales 2.  The same to 2 us:
// halves of 128 columns with barriers and MMA issuers of their own, sixteen epilogue
// warps, 16 or 64 columns a load, the next chunk's load before the multiply-adds,
// CTAs of 128 x 256; scales through shared memory and packed multiply-adds were
// slower (178 and 162 us in all against 154).
//
// Quantisation: bound by issue slots (8192 x 4096, bf16, scales a row: 26 us, 0.57 of
// the copy rate), blocks of 128 rows by 16-byte loads (4096 x 4096: bf16 14.4 us, 0.52; fp32
// 13.8, 0.90).
//
// Waits are bounded as in prod.cu, and set the same error word.
#include <algorithm>
#include <type_traits>

#include <cuda_fp16.h>

#include "lanes.cuh"
#include "prod.cuh"
#include "tc_ptx.cuh"
#include "tc_warp.cuh"

namespace tp {
namespace {

constexpr int kBlock = 128;                // of a scale
constexpr int32_t kMaxDim = 1 << 17;
constexpr int64_t kMaxRows = (int64_t(1) << 31) - 256, kMaxElems = int64_t(1) << 40;

// ----------------------------------------------------------------- quantise
// A block's scale and what its elements are divided by.  Below 2^-64 both sides
// of the quotient are taken 2^64 times, so that no step of it leaves the normal
// numbers.
struct BlockScale {
  float scale, up, unit, inv;
  __device__ __forceinline__ explicit BlockScale(uint32_t top) {
    const float t = __uint_as_float(top);
    const bool finite = top < 0x7F800000u;
    scale = finite ? t / 448.f : __uint_as_float(0x7FC00000u);
    up = t < 5.4e-20f ? 18446744073709551616.f : 1.f;
    unit = scale * up;
    inv = finite && scale > 0.f ? __fdividef(1.f, unit) : 0.f;   // 0: the block's q are 0
  }
};

// Floats whose nearest e4m3 numbers are those of x / scale.  The quotients by a
// reciprocal are right to within three places.  Where that leaves open on which
// side of the border between two e4m3 numbers one lies (20 bits below the last
// one kept; in bf16 data, whose quotients often are borders, one in a few
// hundred), and below 2^-6, where the numbers are 2^-9 apart, the side is that of
// x - border * scale, which a multiply-add gives exactly.
template <int kN>
__device__ __forceinline__ void quotients(float (&x)[kN], const BlockScale& s) {
  if (s.up != 1.f) {
#pragma unroll
    for (int e = 0; e < kN; ++e) x[e] *= s.up;
  }
#pragma unroll
  for (int e = 0; e < kN; ++e) {
    float t = x[e] * s.inv;
    const bool small = fabsf(t) < 0.015625f && t != 0.f;
    // (the 20 bits, moved to the top, within four of the middle)
    if (__float_as_uint(t) * 4096u - (0x7FFFCu << 12) <= (8u << 12) || small) {
      const float border = small ? (floorf(t * 512.f) + 0.5f) * (1.f / 512.f)
                                 : __uint_as_float((__float_as_uint(t) & 0xFFF00000u) | 0x80000u);
      const float r = fmaf(-border, s.unit, x[e]), side = r > 0.f ? 1.f : r < 0.f ? -1.f : 0.f;
      t = fmaf(fabsf(border) * 0x1p-20f, side, border);
    }
    x[e] = t;
  }
  if (s.inv == 0.f)   // zeros, or no numbers (an infinity times 0 is none)
#pragma unroll
    for (int e = 0; e < kN; ++e) x[e] = 0.f;
}
// Two numbers as e4m3 (the first one in the lower byte), to the nearest, ties to even, at most 448.
__device__ __forceinline__ uint32_t e4m3x2(float a, float b) {
  uint16_t r;
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(b), "f"(a));
  return r;
}

template <typename T>
struct QuantArgs {
  const T* x;
  uint8_t* q;
  float* scale;
  int64_t ldx, ldq, rows;
  int32_t k, blocks;      // blocks of 128 columns
  int32_t q16;            // q's rows start at multiples of 16 bytes
};

// Scales per row and block: eight lanes a block, sixteen elements each, so that a
// scale's two divisions are shared by many.
template <typename T>
__global__ void __launch_bounds__(256) k_quant_rows(const QuantArgs<T> g) {
  using L = Lane<T, 1, 1, 8>;
  const int lane = threadIdx.x & 7, b = blockIdx.x * 4 + ((threadIdx.x >> 3) & 3), c = b * kBlock + lane * 16;
  const int64_t step = (int64_t)gridDim.y * 8;
  pdl_trigger();
  pdl_wait();
  const int in = c < g.k ? min(16, g.k - c) : 0;   // 0, 8 or 16 elements
  int64_t row = (int64_t)blockIdx.y * 8 + (threadIdx.x >> 5);
  L x[2];
  auto ask = [&](int64_t r) {
    const bool there = r < g.rows;
    x[0].load(g.x + r * g.ldx + c, 0, there && in > 0 ? 8 : 0);
    x[1].load(g.x + r * g.ldx + c + 8, 0, there && in > 8 ? 8 : 0);
  };
  ask(row);
  for (; row < g.rows; row += step) {
    float v[16];
    const uint4 in4[2] = {x[0].u[0][0], x[1].u[0][0]};   // (of bf16 all eight numbers)
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      float w[8];
      x[h].get(0, w);
#pragma unroll
      for (int e = 0; e < 8; ++e) v[8 * h + e] = w[e];
    }
    ask(row + step);   // the next row's, while this one is worked on
    uint32_t top = 0;
    if constexpr (sizeof(T) == 2) {   // two at a time: bits without their signs are ordered as the numbers are, NaN last
#pragma unroll
      for (int h = 0; h < 2; ++h)
        top = __vmaxu2(top, __vmaxu2(__vmaxu2(in4[h].x & 0x7FFF7FFFu, in4[h].y & 0x7FFF7FFFu),
                                     __vmaxu2(in4[h].z & 0x7FFF7FFFu, in4[h].w & 0x7FFF7FFFu)));
      top = max(top << 16, top & 0xFFFF0000u);
    } else {
#pragma unroll
      for (int e = 0; e < 16; ++e) top = max(top, __float_as_uint(v[e]) & 0x7FFFFFFFu);
    }
#pragma unroll
    for (int o = 4; o > 0; o >>= 1) top = max(top, __shfl_xor_sync(0xffffffffu, top, o));
    const BlockScale s(top);
    if (in && lane == 0) g.scale[row * g.blocks + b] = s.scale;
    quotients(v, s);
    uint32_t w[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) w[e] = e4m3x2(v[4 * e], v[4 * e + 1]) | e4m3x2(v[4 * e + 2], v[4 * e + 3]) << 16;
    uint8_t* q = g.q + row * g.ldq + c;
    if (in == 16 && g.q16) *reinterpret_cast<uint4*>(q) = make_uint4(w[0], w[1], w[2], w[3]);
    else if (in) {
      *reinterpret_cast<uint2*>(q) = make_uint2(w[0], w[1]);
      if (in > 8) *reinterpret_cast<uint2*>(q + 8) = make_uint2(w[2], w[3]);
    }
  }
}

// Any alignment: a warp a block, its lanes side by side.
template <typename T>
__global__ void __launch_bounds__(256) k_quant_rows1(const QuantArgs<T> g) {
  const int lane = threadIdx.x & 31;
  const int64_t total = g.rows * g.blocks;
  pdl_trigger();
  pdl_wait();
  for (int64_t at = (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5); at < total; at += (int64_t)gridDim.x * 8) {
    const int64_t row = at / g.blocks;
    const int c0 = (int)(at - row * g.blocks) * kBlock + lane;
    float v[4];
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      v[i] = c0 + 32 * i < g.k ? Elem<T>::to_f(g.x[row * g.ldx + c0 + 32 * i]) : 0.f;
      top = max(top, __float_as_uint(v[i]) & 0x7FFFFFFFu);
    }
    top = warp_max(top);
    const BlockScale s(top);
    if (lane == 0) g.scale[at] = s.scale;
    quotients(v, s);
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (c0 + 32 * i < g.k) g.q[row * g.ldq + c0 + 32 * i] = (uint8_t)e4m3x2(v[i], 0.f);
  }
}

// Scales per 128 x 128 block: a CTA a block, a warp sixteen rows.
template <typename T>
__global__ void __launch_bounds__(256) k_quant_blocks(const QuantArgs<T> g) {
  __shared__ uint32_t tops[8];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int64_t r0 = (int64_t)blockIdx.y * kBlock + warp * 16;
  const int c0 = blockIdx.x * kBlock + lane;
  pdl_trigger();
  pdl_wait();
  float v[16][4];
  uint32_t top = 0;
#pragma unroll
  for (int r = 0; r < 16; ++r)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      v[r][i] = r0 + r < g.rows && c0 + 32 * i < g.k ? Elem<T>::to_f(g.x[(r0 + r) * g.ldx + c0 + 32 * i]) : 0.f;
      top = max(top, __float_as_uint(v[r][i]) & 0x7FFFFFFFu);
    }
  top = warp_max(top);
  if (lane == 0) tops[warp] = top;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < 8; ++w) top = max(top, tops[w]);
  const BlockScale s(top);
  if (threadIdx.x == 0) g.scale[(int64_t)blockIdx.y * g.blocks + blockIdx.x] = s.scale;
#pragma unroll
  for (int r = 0; r < 16; ++r) {
    quotients(v[r], s);
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (r0 + r < g.rows && c0 + 32 * i < g.k) g.q[(r0 + r) * g.ldq + c0 + 32 * i] = (uint8_t)e4m3x2(v[r][i], 0.f);
  }
}

// The same by 16-byte loads: sixteen lanes a row, eight columns each.
template <typename T>
__global__ void __launch_bounds__(256) k_quant_blocks8(const QuantArgs<T> g) {
  using L = Lane<T, 1, 1, 8>;
  __shared__ uint32_t tops[8];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int64_t r0 = (int64_t)blockIdx.y * kBlock + warp * 16 + (lane >> 4);
  const int c = blockIdx.x * kBlock + (lane & 15) * 8;
  pdl_trigger();
  pdl_wait();
  L x[8];
  uint32_t top = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) x[i].load(g.x + (r0 + 2 * i) * g.ldx + c, 0, c < g.k && r0 + 2 * i < g.rows ? 8 : 0);
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    float v[8];
    x[i].get(0, v);
#pragma unroll
    for (int e = 0; e < 8; ++e) top = max(top, __float_as_uint(v[e]) & 0x7FFFFFFFu);
  }
  top = warp_max(top);
  if (lane == 0) tops[warp] = top;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < 8; ++w) top = max(top, tops[w]);
  const BlockScale s(top);
  if (threadIdx.x == 0) g.scale[(int64_t)blockIdx.y * g.blocks + blockIdx.x] = s.scale;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    float v[8];
    x[i].get(0, v);
    quotients(v, s);
    if (c < g.k && r0 + 2 * i < g.rows)
      *reinterpret_cast<uint2*>(g.q + (r0 + 2 * i) * g.ldq + c) =
          make_uint2(e4m3x2(v[0], v[1]) | e4m3x2(v[2], v[3]) << 16, e4m3x2(v[4], v[5]) | e4m3x2(v[6], v[7]) << 16);
  }
}

template <typename T>
void quantise(const QuantArgs<T>& a, int block_rows, cudaStream_t st) {
  const bool vec = a.k % 8 == 0 && aligned16(a.x, a.ldx, sizeof(T)) && ((uintptr_t)a.q & 7) == 0 && a.ldq % 8 == 0;
  if (block_rows != 1) {
    const dim3 grid((unsigned)a.blocks, (unsigned)ceil_div(a.rows, kBlock));
    if (vec) launch_pdl(k_quant_blocks8<T>, grid, dim3(256), 0, st, a);
    else launch_pdl(k_quant_blocks<T>, grid, dim3(256), 0, st, a);
    return;
  }
  const int64_t total = a.rows * a.blocks, across = ceil_div(a.blocks, 4);
  // (8192 x 4096, bf16: blocks for two turns of the GPU take 0.87 of the time of as many as run at once)
  const dim3 grid((unsigned)across, (unsigned)std::min<int64_t>(ceil_div(a.rows, 8), std::max<int64_t>(1, 12 * kSms / across)));
  if (vec) launch_pdl(k_quant_rows<T>, grid, dim3(256), 0, st, a);
  else launch_pdl(k_quant_rows1<T>, dim3((unsigned)std::min<int64_t>(ceil_div(total, 8), 16 * kSms)), dim3(256), 0, st, a);
}

// ------------------------------------------------------------------ staging
// 16 bytes from `p`, `left` of which lie inside the row; zeros past it.  Elsewhere
// than at a multiple of 16 by words that lie inside [lo, hi), the whole matrix, and
// at its ends by bytes.
template <bool kVec>
__device__ __forceinline__ uint4 bytes16(const uint8_t* p, int left, const uint8_t* lo, const uint8_t* hi) {
  if (left <= 0) return make_uint4(0u, 0u, 0u, 0u);
  if constexpr (kVec) {
    if (left >= 16) return *reinterpret_cast<const uint4*>(p);
  }
  const int shift = (int)((uintptr_t)p & 3);
  const uint8_t* from = p - shift;
  uint32_t w[4];
  if (from >= lo && from + 20 <= hi) {
    uint32_t v[5];
#pragma unroll
    for (int i = 0; i < 5; ++i) v[i] = 4 * i < left + shift ? *reinterpret_cast<const uint32_t*>(from + 4 * i) : 0u;
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = __funnelshift_r(v[i], v[i + 1], 8 * shift);
#pragma unroll
    for (int i = 0; i < 4; ++i) {   // nothing of what lies behind the row
      const int in = left - 4 * i;
      w[i] = in >= 4 ? w[i] : in <= 0 ? 0u : w[i] & (0xffffffffu >> (8 * (4 - in)));
    }
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = 0u;
#pragma unroll
    for (int e = 0; e < 16; ++e)
      if (e < left) w[e >> 2] |= (uint32_t)p[e] << (8 * (e & 3));
  }
  return make_uint4(w[0], w[1], w[2], w[3]);
}

// Rows of k bytes at any address into rows that TMA takes.
struct CopyArgs {
  const uint8_t* src;
  uint8_t* dst;
  int64_t ld, ldp, rows;
  int32_t k;
};
__global__ void __launch_bounds__(256) k_copy_rows(const CopyArgs a, const CopyArgs b) {
  const CopyArgs& g = blockIdx.y ? b : a;
  const int groups = (int)(g.ldp >> 4);
  pdl_trigger();
  pdl_wait();
  const int64_t total = g.rows * groups;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < total; i += (int64_t)gridDim.x * 256) {
    const int64_t row = i / groups;
    const int c = (int)(i - row * groups) * 16;
    *reinterpret_cast<uint4*>(g.dst + row * g.ldp + c) =
        bytes16<false>(g.src + row * g.ld + c, g.k - c, g.src, g.src + (g.rows - 1) * g.ld + g.k);
  }
}

// ------------------------------------------------------------------ product
// A warpgroup of the producer, the MMA issuer and two idle warps, and two of the
// epilogue, which the first one leaves its registers to: 128 (40 + 2 x 232) =
// 384 x 168, what the block is launched with.
constexpr int kEpiWarps = 8, kThreads = 128 + 32 * kEpiWarps;
constexpr int kFewRegs = 40, kManyRegs = 232;
static_assert(128 * kFewRegs + 256 * kManyRegs <= kThreads * 168, "register split");
constexpr int kABytes = 128 * kBlock;
constexpr int kStages = 6, kMaxBufs = 4;
constexpr int kTmemCols = 512;
constexpr int kBufBytes = 32 * 32 * 4;   // per epilogue warp

struct Tail {
  uint64_t full[kStages], empty[kStages], tfull[kMaxBufs], tempty[kMaxBufs], done;
  uint32_t tmem_base;
  int abort;
};

struct F8Args {
  CUtensorMap a, b;
  const uint8_t *q, *w;            // what the maps read
  int64_t ldq, ldw;
  const float *sx, *sw, *bias;
  void* y;
  int* err;
  int32_t M, N, k, kb, tm, tn, f32;   // kb: K blocks; tiles
};

// A K block's sum is multiplied by the product f = a b of its two scales, but where that leaves the normal numbers and
// the result need not (2^-70 2^-75 times up to 2^25; 2^64 2^64 times 0) by the larger one and then by the smaller,
// so that nothing in between leaves them either.
__device__ __forceinline__ bool two_steps(float a, float b, float f) {
  const float m = fabsf(f);
  return (m < 0x1p-126f && a != 0.f && b != 0.f) || m == __int_as_float(0x7F800000);
}
__device__ __forceinline__ float add_scaled(float sum, float a, float b, float acc) {
  const float f = a * b;
  if (!two_steps(a, b, f)) return fmaf(sum, f, acc);
  const bool first = fabsf(a) > fabsf(b);
  return fmaf(sum * (first ? a : b), first ? b : a, acc);
}
__device__ __forceinline__ uint32_t f16_of(uint32_t two) {   // two e4m3 numbers (the lower 16 bits)
  uint32_t r;
  asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(r) : "h"((uint16_t)two));
  return r;
}
__device__ __forceinline__ float2 f32_of(uint32_t two) { return __half22float2(*reinterpret_cast<const __half2*>(&two)); }
// A K block's products of one row of q with kN rows of w, without the tensor cores (each product is exact).
template <int kN, bool kVec>
__device__ __forceinline__ void block_sums(const uint8_t* q, const uint8_t* const (&w)[kN], int kb, int k_all, const uint8_t* q_lo,
                                           const uint8_t* q_hi, const uint8_t* w_lo, const uint8_t* w_hi, float (&sum)[kN]) {
#pragma unroll
  for (int j = 0; j < kN; ++j) sum[j] = 0.f;
#pragma unroll 1
  for (int k = kb * kBlock; k < min((kb + 1) * kBlock, k_all); k += 16) {
    const uint4 a4 = bytes16<kVec>(q + k, k_all - k, q_lo, q_hi);
    const uint32_t a[4] = {a4.x, a4.y, a4.z, a4.w};
    uint4 b4[kN];
#pragma unroll
    for (int j = 0; j < kN; ++j) b4[j] = bytes16<kVec>(w[j] + k, k_all - k, w_lo, w_hi);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float2 x = f32_of(f16_of(a[i >> 1] >> (16 * (i & 1))));
#pragma unroll
      for (int j = 0; j < kN; ++j) {
        const uint32_t b[4] = {b4[j].x, b4[j].y, b4[j].z, b4[j].w};
        const float2 y = f32_of(f16_of(b[i >> 1] >> (16 * (i & 1))));
        sum[j] = fmaf(x.y, y.y, fmaf(x.x, y.x, sum[j]));
      }
    }
  }
}
// Four neighbouring results over K blocks, for the rows that two_steps was true of.  (Four at a time: a warp's 128
// columns of the longest K, 131072, well inside what the other warps wait for it.)
__device__ __forceinline__ void four_sums(const F8Args& g, int row, int col, int kb0, int kb1, float (&acc)[4]) {
  const uint8_t *q = g.q + (int64_t)row * g.ldq, *w[4];
  const float *sx = g.sx + (int64_t)row * g.kb, *sw = g.sw + (int64_t)(min(col, g.N - 1) / kBlock) * g.kb;
  const uint8_t *q_end = g.q + (g.M - 1) * g.ldq + g.k, *w_end = g.w + (g.N - 1) * g.ldw + g.k;
#pragma unroll
  for (int j = 0; j < 4; ++j) w[j] = g.w + (int64_t)min(col + j, g.N - 1) * g.ldw, acc[j] = 0.f;
#pragma unroll 1
  for (int kb = kb0; kb < kb1; ++kb) {
    float sum[4];
    block_sums<4, true>(q, w, kb, g.k, g.q, q_end, g.w, w_end, sum);
#pragma unroll
    for (int j = 0; j < 4; ++j) acc[j] = add_scaled(sum[j], sx[kb], sw[kb], acc[j]);
  }
}

// One K block: four MMAs (K = 32 each, 32 bytes apart) into an accumulator of
// its own; then `bar` and `bar2` (in every CTA of the tile) are told.
#define TP_F8_MMA4(GROUP, COMMIT)                                                                                     \
  "{\n .reg .pred e, p, t;\n .reg .b64 a1, a2, a3, b1, b2, b3;\n elect.sync _|e, 0xffffffff;\n"                        \
  " setp.ne.b32 p, 0, 0;\n setp.eq.b32 t, 0, 0;\n"                                                                    \
  " add.s64 a1, %1, 2;\n add.s64 a2, %1, 4;\n add.s64 a3, %1, 6;\n"                                                   \
  " add.s64 b1, %2, 2;\n add.s64 b2, %2, 4;\n add.s64 b3, %2, 6;\n"                                                   \
  " @e tcgen05.mma.cta_group::" GROUP ".kind::f8f6f4 [%0], %1, %2, %3, p;\n"                                          \
  " @e tcgen05.mma.cta_group::" GROUP ".kind::f8f6f4 [%0], a1, b1, %3, t;\n"                                          \
  " @e tcgen05.mma.cta_group::" GROUP ".kind::f8f6f4 [%0], a2, b2, %3, t;\n"                                          \
  " @e tcgen05.mma.cta_group::" GROUP ".kind::f8f6f4 [%0], a3, b3, %3, t;\n" COMMIT "}\n"
#define TP_F8_COMMIT1                                                                        \
  " @e tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%4];\n"        \
  " @e tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%5];\n"
#define TP_F8_COMMIT2                                                                                                 \
  " @e tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%4], %6;\n"          \
  " @e tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%5], %6;\n"
template <int kCta>
__device__ __forceinline__ void mma_block(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t bar, uint32_t bar2) {
  if constexpr (kCta == 2)
    asm volatile(TP_F8_MMA4("2", TP_F8_COMMIT2)::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(bar), "r"(bar2), "h"((uint16_t)3)
                 : "memory");
  else
    asm volatile(TP_F8_MMA4("1", TP_F8_COMMIT1)::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(bar), "r"(bar2) : "memory");
}

// Eight row blocks at a time walk the columns, so that tiles that run at once share operands in L2.
__device__ __forceinline__ void tile_at(const F8Args& g, int t, int& m, int& n) {
  const int group = t / (8 * g.tn), rows = min(8, g.tm - 8 * group), local = t - group * 8 * g.tn;
  m = 8 * group + local % rows;
  n = local / rows;
}

// A warp's 32 x 32 chunk (lane = row) into rows at any address: a row's 32 columns
// side by side (20011 x 1024 -> 1001: 102 us by each lane's own eight columns).
template <typename T>
__device__ __forceinline__ void emit_rows(float* buf, int lane, const float (&v)[32], T* out, int n, int r0, int m_lim, int c0) {
  __syncwarp();
#pragma unroll
  for (int e = 0; e < 32; ++e) buf[lane * 32 + (e ^ lane)] = v[e];
  __syncwarp();
  if (c0 + lane < n)
#pragma unroll 8
    for (int r = 0; r < 32; ++r)
      if (r0 + r < m_lim) out[(int64_t)(r0 + r) * n + c0 + lane] = Elem<T>::from_f(buf[r * 32 + (lane ^ r)]);
}

// wait_all without a call: the epilogue's registers leave none for one.
__device__ __forceinline__ bool wait_here(uint64_t* bar, uint32_t parity, volatile int* abort_flag, int* err,
                                          uint64_t budget_ns, int site) {
  if (__all_sync(0xffffffffu, mbar_try_wait(bar, parity))) return true;
  const uint64_t t0 = global_ns();
  while (true) {
    if (__all_sync(0xffffffffu, mbar_try_wait(bar, parity))) return true;
    if (__any_sync(0xffffffffu, *abort_flag != 0)) return false;
    if (__any_sync(0xffffffffu, global_ns() - t0 > budget_ns)) {
      *abort_flag = 1;
      atomicCAS(err, 0, site);
      return false;
    }
  }
}

// kN: columns of a tile, kCta * 128 its rows; kSplit: CTAs of a cluster that share
// out a tile's K blocks (kCta = 1).
template <int kCta, int kN, int kSplit>
__global__ void __launch_bounds__(kThreads, 1) k_prod_f8(const __grid_constant__ F8Args g) {
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = (uint8_t*)(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);
  constexpr int kNh = kN / kCta;                        // rows of B that this CTA stages
  constexpr uint32_t kStageBytes = kABytes + kNh * kBlock;
  constexpr int kBufs = kTmemCols / kN < kMaxBufs ? kTmemCols / kN : kMaxBufs;
  constexpr int kCols = kN / 2;                         // of an epilogue warp
  uint8_t* bufs = smem + kStages * kStageBytes;
  Tail* tl = (Tail*)(bufs + kEpiWarps * kBufBytes);
  const int warp = (int)uniform(threadIdx.x >> 5), lane = threadIdx.x & 31;
  const int rank = kCta == 2 ? (int)uniform(cluster_rank()) : 0;
  const bool leader = rank == 0;
  constexpr int kClu = kCta * kSplit;
  const int clu = blockIdx.x / kClu, n_clu = gridDim.x / kClu, n_tiles = g.tm * g.tn;
  const int part = kSplit > 1 ? (int)uniform(cluster_rank()) : 0;
  const int kb_first = g.kb * part / kSplit, kb_end = g.kb * (part + 1) / kSplit;

  if (threadIdx.x == 0) {
    for (int s = 0; s < kStages; ++s) {
      mbar_init(&tl->full[s], 1);
      mbar_init(&tl->empty[s], 1);
    }
    for (int b = 0; b < kBufs; ++b) {
      mbar_init(&tl->tfull[b], 1);
      mbar_init(&tl->tempty[b], kEpiWarps * kCta);
    }
    mbar_init(&tl->done, 1);
    tl->abort = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 1) {
    if constexpr (kCta == 2) {
      asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&tl->tmem_base)),
                   "r"(kTmemCols)
                   : "memory");
      asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
    } else {
      asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&tl->tmem_base)),
                   "r"(kTmemCols)
                   : "memory");
      asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  if (kClu > 1) cluster_sync();    // the peers' barriers and memory exist before anything targets them
  if (warp == 0 && lane < 2) asm volatile("prefetch.tensormap [%0];" ::"l"(lane ? &g.b : &g.a) : "memory");
  pdl_wait();                      // the set-up above overlaps the previous kernel
  fence_proxy_async_global();      // what it wrote by plain stores is read by TMA
  const uint32_t tmem = uniform(tl->tmem_base);
  volatile int* abort_flag = &tl->abort;
  int* err = g.err;

  if (warp < 4) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kFewRegs));
    if (warp == 0) {
      // ---------------------------------------------------------- producer
      uint32_t stage = 0, phase = 0, issued = 0;
      bool ok = true;
      const uint32_t s0 = smem_u32(smem), full0 = smem_u32(&tl->full[0]);
      const uint32_t lead0 = kCta == 2 ? mapa(full0, 0) : full0;   // the barriers that copies complete on
      for (int t = clu; ok && t < n_tiles; t += n_clu) {
        int m, n;
        tile_at(g, t, m, n);
        const int ya = (m * kCta + rank) * 128, yb = n * kN + rank * kNh;
        for (int kb = kb_first; kb < kb_end; ++kb) {
          if (!wait_all(&tl->empty[stage], phase ^ 1u, abort_flag, err, kWaitNs, 61)) {
            ok = false;
            break;
          }
          const uint32_t dst = s0 + stage * kStageBytes, bar = lead0 + 8 * stage;
          if (leader) expect_elect(full0 + 8 * stage, kCta * kStageBytes);
          tma_elect<kCta>(dst, &g.a, bar, kBlock * kb, ya, 0);
          tma_elect<kCta>(dst + kABytes, &g.b, bar, kBlock * kb, yb, 0);
          issued |= 1u << stage;
          if (++stage == kStages) {
            stage = 0;
            phase ^= 1u;
          }
        }
      }
      // every copy has landed before the CTA leaves: a stage's last one is of this
      // turn of the ring below `stage`, of the one before from there on
      if (leader)
        for (int s = 0; s < kStages; ++s)
          if (issued & (1u << s)) {
            int dummy = 0;
            mbar_wait(&tl->full[s], s < (int)stage ? phase : phase ^ 1u, &dummy, err, kWaitNs, 62);
          }
    } else if (warp == 1) {
      if (leader) {
        // --------------------------------------------------------------- MMA
        const uint32_t s0 = smem_u32(smem), empty0 = smem_u32(&tl->empty[0]), tfull0 = smem_u32(&tl->tfull[0]);
        const uint64_t da = smem_desc(s0, 16, 1024), db = smem_desc(s0 + kABytes, 16, 1024);
        // fp32 accumulators, e4m3 operands (format 0), both K-major
        const uint32_t idesc = (1u << 4) | ((uint32_t)(kN >> 3) << 17) | ((uint32_t)(128 * kCta >> 4) << 24);
        uint32_t stage = 0, phase = 0, buf = 0, buf_phase = 0;
        bool ok = true;
        for (int t = clu; ok && t < n_tiles; t += n_clu)
          for (int kb = kb_first; kb < kb_end; ++kb) {
            if (!wait_all(&tl->tempty[buf], buf_phase ^ 1u, abort_flag, err, 2 * kWaitNs, 63) ||
                !wait_all(&tl->full[stage], phase, abort_flag, err, 2 * kWaitNs, 64)) {
              ok = false;
              break;
            }
            tc_fence_after();
            mma_block<kCta>(tmem + buf * kN, da + stage * (kStageBytes >> 4), db + stage * (kStageBytes >> 4), idesc,
                            empty0 + 8 * stage, tfull0 + 8 * buf);
            if (++stage == kStages) {
              stage = 0;
              phase ^= 1u;
            }
            if (++buf == kBufs) {
              buf = 0;
              buf_phase ^= 1u;
            }
          }
        commit_elect<kCta>(smem_u32(&tl->done));   // all MMAs are over before TMEM is freed
        int dummy = 0;
        mbar_wait(&tl->done, 0, &dummy, err, kWaitNs, 65);
      }
    }
    if constexpr (kSplit > 1) {   // the epilogue's two meetings
      __syncwarp();
      cluster_sync();
      cluster_sync();
    }
  } else {
    // ------------------------------------------------------------ epilogue
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kManyRegs));
    const int q = warp & 3, half = (warp - 4) >> 2;
    uint8_t* out_buf = bufs + (warp - 4) * kBufBytes;
    uint32_t buf = 0, buf_phase = 0;
    const uint32_t t0 = tmem + ((uint32_t)(32 * q) << 16) + half * kCols;
    bool ok = true;
    for (int t = clu; ok && t < n_tiles; t += n_clu) {
      int m, n;
      tile_at(g, t, m, n);
      const int r0 = (m * kCta + rank) * 128 + 32 * q, c0 = n * kN + half * kCols;
      const int row = min(r0 + lane, g.M - 1);
      const float* sx = g.sx + (int64_t)row * g.kb;
      const float* sw = g.sw + (int64_t)(min(c0, g.N - 1) / kBlock) * g.kb;
      float acc[kCols];
#pragma unroll
      for (int e = 0; e < kCols; ++e) acc[e] = 0.f;
      float ax = sx[kb_first], aw = sw[kb_first];
      bool apart = false;   // a K block of this row wants two steps
      for (int kb = kb_first; kb < kb_end; ++kb) {
        const float f = ax * aw;
        apart = apart || two_steps(ax, aw, f);
        if (kb + 1 < kb_end) ax = sx[kb + 1], aw = sw[kb + 1];
        if (!wait_here(&tl->tfull[buf], buf_phase, abort_flag, err, 2 * kWaitNs, 66)) {
          ok = false;
          break;
        }
        tc_fence_after();
#pragma unroll
        for (int c = 0; c < kCols; c += 32) {
          uint32_t v[32];
          tmem_ask32(t0 + buf * kN + c, v);
          tmem_wait();
          tmem_got(v);
          if (c + 32 == kCols) {   // the accumulator is read: free for the block but one after this before its last sums
            tc_fence_before();
            __syncwarp();
            if (lane == 0) {
              if constexpr (kCta == 2) mbar_arrive_cluster_relaxed(mapa(smem_u32(&tl->tempty[buf]), 0));
              else mbar_arrive_relaxed(&tl->tempty[buf]);
            }
          }
#pragma unroll
          for (int e = 0; e < 32; ++e) acc[c + e] = fmaf(__uint_as_float(v[e]), f, acc[c + e]);
        }
        if (++buf == kBufs) {
          buf = 0;
          buf_phase ^= 1u;
        }
      }
      // (a branch for it in the loop above, per K block: 8192 x 4096 -> 4096 134 us instead of 121)
      if (ok && __any_sync(0xffffffffu, apart)) {
        float* buf = (float*)out_buf;
#pragma unroll
        for (int c = 0; c < kCols; c += 32) {
          __syncwarp();
#pragma unroll 1
          for (int e = 0; apart && e < 32; e += 4) {
            float v[4];
            four_sums(g, row, c0 + c + e, kb_first, kb_end, v);
#pragma unroll
            for (int j = 0; j < 4; ++j) buf[lane * 32 + ((e + j) ^ lane)] = v[j];
          }
#pragma unroll
          for (int e = 0; e < 32; ++e) acc[c + e] = apart ? buf[lane * 32 + (e ^ lane)] : acc[c + e];
        }
      }
      if constexpr (kSplit > 1) {
        // the others' sums go to the first CTA's ring, which no copy or MMA uses any more, and are added in order
        cluster_sync();
        float* ring = (float*)smem + (warp - 4) * (32 * kCols);
        if (part > 0) {
          const uint32_t to = mapa(smem_u32(ring + (part - 1) * (256 * kCols)), 0);
#pragma unroll
          for (int e = 0; e < kCols; e += 4)
            asm volatile("st.shared::cluster.v4.f32 [%0], {%1, %2, %3, %4};" ::"r"(to + (e * 32 + 4 * lane) * 4), "f"(acc[e]),
                         "f"(acc[e + 1]), "f"(acc[e + 2]), "f"(acc[e + 3])
                         : "memory");
        }
        cluster_sync();
        if (part > 0) break;
#pragma unroll
        for (int p = 0; p < kSplit - 1; ++p)
#pragma unroll
          for (int e = 0; e < kCols; e += 4) {
            const float4 v = *reinterpret_cast<const float4*>(ring + p * (256 * kCols) + e * 32 + 4 * lane);
            acc[e] += v.x, acc[e + 1] += v.y, acc[e + 2] += v.z, acc[e + 3] += v.w;
          }
      }
      if (!ok) break;
      const bool live = r0 + lane < g.M;
#pragma unroll
      for (int c = 0; c < kCols; c += 32) {
        const int col = c0 + c, left = g.N - col;
        if (left <= 0) break;
        const float b = g.bias && col + lane < g.N ? g.bias[col + lane] : 0.f;
        float v[32];
#pragma unroll
        for (int e = 0; e < 32; ++e) v[e] = acc[c + e] + __shfl_sync(0xffffffffu, b, e);
        const int64_t at = (int64_t)(r0 + lane) * g.N + col;
        if (g.f32) {
          if (left >= 32 && ((uintptr_t)g.y & 31) == 0 && (g.N & 7) == 0) put_f32(v, (float*)g.y + at, live, 32);
          else if (vec_ok(g.y, g.N, 4)) emit_f32(out_buf, lane, v, (float*)g.y, g.N, r0, g.M, col, g.N, true);
          else emit_rows((float*)out_buf, lane, v, (float*)g.y, g.N, r0, g.M, col);
        } else {
          uint32_t pk[16];
          pack32(v, pk);
          if (left >= 32 && ((uintptr_t)g.y & 31) == 0 && (g.N & 15) == 0) put_bf16(pk, (__nv_bfloat16*)g.y + at, live, 32);
          else if (vec_ok(g.y, g.N, 2)) emit_bf16(out_buf, lane, pk, (__nv_bfloat16*)g.y, g.N, r0, g.M, col, g.N, true);
          else emit_rows((float*)out_buf, lane, v, (__nv_bfloat16*)g.y, g.N, r0, g.M, col);
        }
      }
    }
  }

  pdl_trigger();   // not earlier: CTAs of the next kernel parked beside a running product slow it down
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  if constexpr (kCta == 2) {
    // the leader's last commit arrives in both CTAs: its arrival here, too, is over before this memory is another's
    if (warp == 1 && !leader) {
      int dummy = 0;
      mbar_wait(&tl->done, 0, &dummy, err, 4 * kWaitNs, 65);
    }
    cluster_sync();
  }
  if (warp == 1) {
    if constexpr (kCta == 2)
      asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(kTmemCols) : "memory");
    else
      asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(kTmemCols) : "memory");
  }
}

template <int kCta, int kN, int kSplit>
cudaError_t launch_f8(F8Args& g, const void* q, int64_t ldq, const void* w, int64_t ldw, int64_t k, cudaStream_t st) {
  constexpr int kClu = kCta * kSplit;
  static_assert(kSplit == 1 || (kSplit - 1) * 256 * (kN / 2) * 4 <= kStages * (kABytes + kN * kBlock), "a ring holds the other parts");
  g.tm = (int32_t)ceil_div(g.M, 128 * kCta), g.tn = (int32_t)ceil_div(g.N, kN);
  if (!tma_map_bytes(&g.a, q, k, g.M, ldq, kBlock, 128) || !tma_map_bytes(&g.b, w, k, g.N, ldw, kBlock, kN / kCta))
    return cudaErrorInvalidValue;
  const int smem = 1024 + kStages * (kABytes + kN / kCta * kBlock) + kEpiWarps * kBufBytes + (int)sizeof(Tail);
  static OncePerDevice once;
  const cudaError_t e = once(
      [] { return cudaFuncSetAttribute(k_prod_f8<kCta, kN, kSplit>, cudaFuncAttributeMaxDynamicSharedMemorySize, 232448); });
  if (e != cudaSuccess) return e;
  cudaLaunchConfig_t cfg = {};
  // a cluster a tile where K is shared out, else as many as run at once
  const int64_t tiles = (int64_t)g.tm * g.tn;
  cfg.gridDim = dim3(kClu * (unsigned)(kSplit > 1 ? tiles : std::min<int64_t>(tiles, kSms / kCta)));
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = kClu;
  attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = kClu > 1 ? 2 : 1;
  return cudaLaunchKernelEx(&cfg, k_prod_f8<kCta, kN, kSplit>, g);
}

tp_status check(int64_t rows, int32_t k, int32_t n, int32_t precision) {
  if (rows < 0 || rows > kMaxRows) return ops_fail(TP_EINVAL, "rows %lld out of range", (long long)rows);
  if (k < 1 || n < 1 || k > kMaxDim || n > kMaxDim)
    return ops_fail(TP_EINVAL, "k %d and n %d must be in 1..%d", k, n, kMaxDim);
  if (rows * (k > n ? k : n) > kMaxElems) return ops_fail(TP_EINVAL, "more than 2^40 elements in a matrix");
  if (precision != TP_BF16 && precision != TP_FP32) return ops_fail(TP_EINVAL, "unknown precision %d", precision);
  return TP_OK;
}

// The tile, by times measured: us a K block, of a tile alone on its SMs and with
// all of them at work (there the pairs' half of the traffic from L2 counts), and
// what a launch and a tile's results take besides.  A K block's time is hardly less for fewer
// columns, because it is the chain from MMA to epilogue and back that it waits for.
struct Shape {
  int rows, cols, split;
  double kb, kb_full, fixed, epi;
};
constexpr Shape kShapes[] = {{256, 256, 1, 0.44, 0.55, 5.0, 3.0}, {128, 128, 1, 0.235, 0.31, 3.2, 1.5},
                             {128, 64, 1, 0.225, 0.31, 2.7, 1.0}, {128, 64, 2, 0.225, 0.31, 4.2, 1.0},
                             {128, 64, 4, 0.225, 0.31, 5.5, 1.0}};
int pick_shape(int64_t rows, int64_t n, int64_t kb) {
  int pick = 0;
  double best = 1e30;
  for (int i = 0; i < 5; ++i) {
    const Shape& s = kShapes[i];
    const int64_t tiles = ceil_div(rows, s.rows) * ceil_div(n, s.cols), at_once = kSms / (s.rows / 128 * s.split);
    if (s.split > 1 && (tiles > at_once || kb < s.split)) continue;
    const double waves = (double)ceil_div(tiles, at_once);
    const double t = s.fixed + waves * (double)ceil_div(kb, s.split) * (tiles > at_once ? s.kb_full : s.kb) + (waves - 1) * s.epi;
    if (t < best) best = t, pick = i;
  }
  return pick;
}
cudaError_t run_product(F8Args& g, const void* q, int64_t ldq, const void* w, int64_t ldw, int64_t k, cudaStream_t st) {
  switch (pick_shape(g.M, g.N, g.kb)) {
    case 0: return launch_f8<2, 256, 1>(g, q, ldq, w, ldw, k, st);
    case 1: return launch_f8<1, 128, 1>(g, q, ldq, w, ldw, k, st);
    case 2: return launch_f8<1, 64, 1>(g, q, ldq, w, ldw, k, st);
    case 3: return launch_f8<1, 64, 2>(g, q, ldq, w, ldw, k, st);
    default: return launch_f8<1, 64, 4>(g, q, ldq, w, ldw, k, st);
  }
}

// ----------------------------------------------------------------- few rows
// A serving call: bound by the weights' bytes, each of which is read once, straight
// into the registers of the warp that multiplies it, as the 16-row operand of
// mma.sync (e4m3 as fp16, exact); the rows of x are its eight columns.  A warp
// takes K blocks in turns; a block's sums are scaled and added in fp32; the warps'
// meet in shared memory, added in order.
struct FewArgs {
  const uint8_t *x, *w;
  const float *sx, *sw, *bias;
  void* y;
  int64_t ldx, ldw;
  int32_t rows, k, n, kb, f32;
};
constexpr int kStride = 20;   // floats between tokens of a partial sum: conflict-free stores
// (One CTA an SM asked for: left to itself the compiler takes two of sixteen warps, and spills.  16 rows of 8192 ->
// 2048: 11.9 us instead of 6.2.)
template <int kNT, int kWarps, bool kVec>
__global__ void __launch_bounds__(32 * kWarps, kNT == 2 && kWarps == 16 ? 1 : 0) k_few_f8(const FewArgs g) {
  __shared__ float red[kWarps][8 * kNT][kStride];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, gid = lane >> 2, t = lane & 3;
  const int n0 = blockIdx.x * 16, m0 = blockIdx.y * 8 * kNT;
  pdl_trigger();
  const uint8_t* wr[2];
#pragma unroll
  for (int h = 0; h < 2; ++h) wr[h] = g.w + (int64_t)min(n0 + gid + 8 * h, g.n - 1) * g.ldw;
  if (warp < g.kb)
#pragma unroll
    for (int h = 0; h < 2; ++h) asm volatile("prefetch.global.L2 [%0];" ::"l"(wr[h] + min(kBlock * warp + 32 * t, g.k - 1)));
  pdl_wait();
  const uint8_t *w_end = g.w + (g.n - 1) * g.ldw + g.k, *x_end = g.x + (g.rows - 1) * g.ldx + g.k;
  float acc[kNT][4];
#pragma unroll
  for (int j = 0; j < kNT; ++j)
#pragma unroll
    for (int e = 0; e < 4; ++e) acc[j][e] = 0.f;
  const float* sw = g.sw + (int64_t)(n0 / kBlock) * g.kb;
  bool apart = false;   // a K block of one of the rows wants two steps
  for (int b = warp; b < g.kb; b += kWarps) {
    // a lane's 32 bytes of a row's 128: two pieces of 16, 64 apart; both operands agree on the order of k
    uint4 wv[2][2], xv[kNT][2];
    float s[kNT][2];
#pragma unroll
    for (int p = 0; p < 2; ++p) {
      const int k = kBlock * b + 64 * p + 16 * t;
#pragma unroll
      for (int h = 0; h < 2; ++h) wv[h][p] = bytes16<kVec>(wr[h] + k, n0 + gid + 8 * h < g.n ? g.k - k : 0, g.w, w_end);
#pragma unroll
      for (int j = 0; j < kNT; ++j) {
        const int m = m0 + 8 * j + gid;
        xv[j][p] = bytes16<kVec>(g.x + (int64_t)min(m, g.rows - 1) * g.ldx + k, m < g.rows ? g.k - k : 0, g.x, x_end);
      }
    }
    const float ws = sw[b];
#pragma unroll
    for (int j = 0; j < kNT; ++j)
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        const int m = m0 + 8 * j + 2 * t + c;
        const float one = m < g.rows ? g.sx[(int64_t)m * g.kb + b] : 0.f;
        s[j][c] = one * ws;
        apart = apart || two_steps(one, ws, s[j][c]);
      }
    float blk[kNT][4];
#pragma unroll
    for (int j = 0; j < kNT; ++j)
#pragma unroll
      for (int e = 0; e < 4; ++e) blk[j][e] = 0.f;
#pragma unroll
    for (int p = 0; p < 2; ++p) {
      uint32_t a[2][8];   // the 16 numbers of each of the lane's rows, as pairs
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const uint32_t v[4] = {wv[h][p].x, wv[h][p].y, wv[h][p].z, wv[h][p].w};
#pragma unroll
        for (int i = 0; i < 4; ++i) a[h][2 * i] = f16_of(v[i]), a[h][2 * i + 1] = f16_of(v[i] >> 16);
      }
#pragma unroll
      for (int j = 0; j < kNT; ++j) {
        const uint32_t v[4] = {xv[j][p].x, xv[j][p].y, xv[j][p].z, xv[j][p].w};
#pragma unroll
        for (int i = 0; i < 4; ++i)
          asm volatile(
              "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, "
              "%3};"
              : "+f"(blk[j][0]), "+f"(blk[j][1]), "+f"(blk[j][2]), "+f"(blk[j][3])
              : "r"(a[0][2 * i]), "r"(a[1][2 * i]), "r"(a[0][2 * i + 1]), "r"(a[1][2 * i + 1]), "r"(f16_of(v[i])),
                "r"(f16_of(v[i] >> 16)));
      }
    }
#pragma unroll
    for (int j = 0; j < kNT; ++j)
#pragma unroll
      for (int e = 0; e < 4; ++e) acc[j][e] = fmaf(blk[j][e], s[j][e & 1], acc[j][e]);
  }
#pragma unroll
  for (int j = 0; j < kNT; ++j) {
    red[warp][8 * j + 2 * t][gid] = acc[j][0];
    red[warp][8 * j + 2 * t + 1][gid] = acc[j][1];
    red[warp][8 * j + 2 * t][gid + 8] = acc[j][2];
    red[warp][8 * j + 2 * t + 1][gid + 8] = acc[j][3];
  }
  if (__any_sync(0xffffffffu, apart)) {
    __syncwarp();
#pragma unroll 1
    for (int i = lane; i < 16 * 8 * kNT; i += 32) {
      const int m = m0 + (i >> 4), n = n0 + (i & 15);
      if (m >= g.rows || n >= g.n) continue;
      const uint8_t *x = g.x + (int64_t)m * g.ldx, *w[1] = {g.w + (int64_t)n * g.ldw};
      float sum[1], v = 0.f;
      bool any = false;
#pragma unroll 1
      for (int b = warp; b < g.kb; b += kWarps) {
        const float ax = g.sx[(int64_t)m * g.kb + b], aw = sw[b];
        block_sums<1, kVec>(x, w, b, g.k, g.x, x_end, g.w, w_end, sum);
        v = add_scaled(sum[0], ax, aw, v);
        any = any || two_steps(ax, aw, ax * aw);
      }
      if (any) red[warp][i >> 4][i & 15] = v;
    }
  }
  __syncthreads();
  for (int i = threadIdx.x; i < 16 * 8 * kNT; i += 32 * kWarps) {
    const int ml = i >> 4, c = i & 15, m = m0 + ml, n = n0 + c;
    if (m >= g.rows || n >= g.n) continue;
    float v = red[0][ml][c];
#pragma unroll
    for (int w = 1; w < kWarps; ++w) v += red[w][ml][c];
    if (g.bias) v += g.bias[n];
    if (g.f32) ((float*)g.y)[(int64_t)m * g.n + n] = v;
    else ((__nv_bfloat16*)g.y)[(int64_t)m * g.n + n] = __float2bfloat16_rn(v);
  }
}
template <int kWarps, bool kVec>
void launch_few(const FewArgs& a, cudaStream_t st) {
  const int nt = a.rows <= 8 ? 1 : a.rows <= 16 ? 2 : 4;
  const dim3 grid((unsigned)ceil_div(a.n, 16), (unsigned)ceil_div(a.rows, 8 * nt)), block(32 * kWarps);
  if (nt == 1) launch_pdl(k_few_f8<1, kWarps, kVec>, grid, block, 0, st, a);
  else if (nt == 2) launch_pdl(k_few_f8<2, kWarps, kVec>, grid, block, 0, st, a);
  else launch_pdl(k_few_f8<4, kWarps, kVec>, grid, block, 0, st, a);
}
// Do these take `rows` rows?  Measured against the best tcgen05 tile (us): 2048 ->
// 4096, 16 rows 4.7 / 7.1, 32 rows 6.7 / 7.2, 48 rows 10.7 / 7.1; 1024 -> 1000, 128
// rows 3.6 / 4.8, 200 rows 6.1 / 4.9; 4096 -> 4096, 16 rows 6.8 / 11, 32 rows 10.3 /
// 8.5; 512 -> 512, 256 rows 2.7 / 4.0.
bool few_take(int64_t rows, int64_t k, int64_t n) {
  if (rows > 256) return false;
  const int64_t work = rows * k * n;
  return rows <= 16 || (rows <= 32 && work <= 270000000) || work <= 140000000;
}

// An operand's rows as TMA takes them, staged where they lie otherwise.
int64_t staged_bytes(int64_t rows, int32_t k) { return round_up(rows * round_up(k, 16), 256); }

tp_status done(cudaError_t e, const char* who) {
  if (e == cudaSuccess) return TP_OK;
  cudaGetLastError();   // reported here
  return ops_fail(TP_ECUDA, "%s: %s", who, cudaGetErrorString(e));
}

}  // namespace
}  // namespace tp

using namespace tp;

extern "C" {

tp_status pack_quantise_f8(const void* x, int64_t ldx, int64_t rows, int32_t k, int32_t block_rows, int32_t precision,
                           void* q, int64_t ldq, float* scale, void* cuda_stream) {
  tp_status s = check(rows, k, 1, precision);
  if (s != TP_OK) return s;
  if (block_rows != 1 && block_rows != kBlock) return ops_fail(TP_EINVAL, "block_rows %d must be 1 or %d", block_rows, kBlock);
  if (ldx < k || ldq < k) return ops_fail(TP_EINVAL, "ldx and ldq must not be less than k %d", k);
  if (block_rows != 1 && rows > int64_t(kBlock) * 65535)
    return ops_fail(TP_EINVAL, "at most %d rows in blocks of %d", kBlock * 65535, kBlock);
  if (rows == 0) return TP_OK;
  if (!x || !q || !scale) return ops_fail(TP_EINVAL, "null argument");
  if ((s = ops_device()) != TP_OK) return s;
  cudaStream_t st = (cudaStream_t)cuda_stream;
  const int32_t blocks = (int32_t)ceil_div(k, kBlock), q16 = aligned16(q, ldq, 1);
  if (precision == TP_FP32)
    quantise(QuantArgs<float>{(const float*)x, (uint8_t*)q, scale, ldx, ldq, rows, k, blocks, q16}, block_rows, st);
  else
    quantise(QuantArgs<__nv_bfloat16>{(const __nv_bfloat16*)x, (uint8_t*)q, scale, ldx, ldq, rows, k, blocks, q16}, block_rows, st);
  return done(cudaGetLastError(), "pack_quantise_f8");
}

tp_status pack_product_f8_bytes(int64_t rows, int32_t k, int32_t n, int32_t aligned, int64_t* workspace) {
  const tp_status s = check(rows, k, n, TP_BF16);
  if (s != TP_OK) return s;
  if (!workspace) return ops_fail(TP_EINVAL, "null argument");
  *workspace = rows == 0 || aligned || few_take(rows, k, n) ? 0 : staged_bytes(rows, k) + staged_bytes(n, k);
  return TP_OK;
}

tp_status pack_product_f8(const void* q, int64_t ldq, const float* scale, const void* w, int64_t ldw, const float* w_scale,
                          const float* bias, int64_t rows, int32_t k, int32_t n, int32_t precision, void* y,
                          void* workspace, int64_t workspace_bytes, void* cuda_stream) {
  tp_status s = check(rows, k, n, precision);
  if (s != TP_OK) return s;
  if (ldq < k || ldw < k) return ops_fail(TP_EINVAL, "ldq and ldw must not be less than k %d", k);
  if (rows == 0) return TP_OK;
  if (!q || !scale || !w || !w_scale || !y) return ops_fail(TP_EINVAL, "null argument");
  if (rows == 1) ldq = round_up(k, 16);   // (one row has no distance to the next)
  if (n == 1) ldw = round_up(k, 16);
  const bool q_ok = aligned16(q, ldq, 1), w_ok = aligned16(w, ldw, 1);
  if (few_take(rows, k, n)) {
    if ((s = ops_device()) != TP_OK) return s;
    const FewArgs a{(const uint8_t*)q, (const uint8_t*)w, scale, w_scale, bias, y, ldq, ldw, (int32_t)rows, k, n,
                    (int32_t)ceil_div(k, kBlock), precision == TP_FP32};
    cudaStream_t st = (cudaStream_t)cuda_stream;
    // sixteen warps where there are K blocks for them and the CTAs are few
    const bool deep = a.kb > 8 && ceil_div(n, 16) * ceil_div(rows, 32) <= 2 * kSms;
    if (q_ok && w_ok) deep ? launch_few<16, true>(a, st) : launch_few<8, true>(a, st);
    else deep ? launch_few<16, false>(a, st) : launch_few<8, false>(a, st);
    return done(cudaGetLastError(), "pack_product_f8");
  }
  const int64_t need = q_ok && w_ok ? 0 : staged_bytes(rows, k) + staged_bytes(n, k);
  if (need && (workspace_bytes < need || !workspace || ((uintptr_t)workspace & 255)))
    return ops_fail(TP_EINVAL, "a workspace of %lld bytes, 256-byte aligned, is needed", (long long)need);
  if ((s = ops_device()) != TP_OK) return s;
  cudaStream_t st = (cudaStream_t)cuda_stream;
  F8Args g{};
  cudaError_t e = prod_err_word(&g.err);
  if (e != cudaSuccess) return done(e, "pack_product_f8");
  if (need) {
    const int64_t ldp = round_up(k, 16);
    uint8_t* qs = (uint8_t*)workspace;
    uint8_t* ws = qs + staged_bytes(rows, k);
    const CopyArgs cq{(const uint8_t*)q, qs, ldq, ldp, rows, k}, cw{(const uint8_t*)w, ws, ldw, ldp, n, k};
    const int64_t blocks = std::min<int64_t>(ceil_div(std::max<int64_t>(rows, n) * (ldp / 16), 256), 8 * kSms);
    launch_pdl(k_copy_rows, dim3((unsigned)blocks, !q_ok && !w_ok ? 2 : 1), dim3(256), 0, st, q_ok ? cw : cq, cw);
    if ((e = cudaGetLastError()) != cudaSuccess) return done(e, "pack_product_f8");
    if (!q_ok) q = qs, ldq = ldp;
    if (!w_ok) w = ws, ldw = ldp;
  }
  g.q = (const uint8_t*)q, g.w = (const uint8_t*)w, g.ldq = ldq, g.ldw = ldw;
  g.sx = scale, g.sw = w_scale, g.bias = bias, g.y = y;
  g.M = (int32_t)rows, g.N = n, g.k = k, g.kb = (int32_t)ceil_div(k, kBlock), g.f32 = precision == TP_FP32;
  e = run_product(g, q, ldq, w, ldw, k, st);
  return done(e, "pack_product_f8");
}

}  // extern "C"
