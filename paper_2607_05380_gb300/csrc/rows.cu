// rows.cu -- the products of a few rows (a serving call): y[m, n] = sum_k
// x[m, k] w[n, k] with one epilogue, for the gated block's two products (bf16)
// and the 8-bit product (int8 as fp16, exact).
//
// Bound by the weights' bytes: each is read once, straight into the registers
// of the warp that multiplies it, as the 16-row operand of mma.sync (the rows
// of x are its 8 columns); tcgen05 would want the weights in shared memory
// and 128 rows of x.  A CTA takes 16 or 32 output columns (the gated block: 16
// pairs) and up to 32 rows of x; its eight or sixteen warps take K in turns of
// 64; their sums meet in shared memory and are added in a fixed order.  The
// order of k inside a turn is free as long as both operands agree on it, so a
// lane's 16 elements are those of two 16-byte loads (one of int8), which the
// four lanes of a row make of whole sectors, with no shuffles.
//
// The weights' first steps are asked for (into L2) before the previous kernel
// of the stream has finished.
//
// Gated block of 1024 and 2048, its 12.6 MB of weights in L2: one row 4.3 us in
// two launches, 32 rows 7.6; 8-bit product 2048 -> 4096, one row 2.9 us.
#include <type_traits>

#include "kernels.cuh"
#include "prod.cuh"
#include "rows.cuh"

namespace tp {
namespace {

constexpr int kStride = 20;   // floats between tokens of a partial sum: conflict-free stores

enum Mode { kGated, kPlain, kQuant };

struct RowArgs {
  const void *x, *w;
  int64_t ldx, up;        // up: elements from a gate row to its up row
  int32_t rows, k, n;
  void* out;              // [rows, ldo]
  int64_t ldo;
  void *a, *p;            // kGated: act(g), u act'(g), pitch ld_keep (NULL: not wanted)
  __nv_bfloat16* parts;   // 32-bit blocks that keep something: h as three bf16 parts, `part` elements apart
  int64_t ld_keep, part;
  uint8_t *a_lo, *p_lo;   // bf16 blocks: the lower 8 of a's and p's 24 bits
  const float *sx, *sw, *bias;
  int32_t f32;            // kQuant: 32-bit output
};

__device__ __forceinline__ void mma_bf16(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, "
      "%3};"
      : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void mma_f16(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, "
      "%3};"
      : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

// 16 bytes, `left` of which lie inside the row, by loads of kLd bytes that the
// address is a multiple of; zeros past the row.
template <int kLd>
__device__ __forceinline__ uint4 bytes16(const char* p, int left) {
  if constexpr (kLd == 16) {
    return left > 0 ? *reinterpret_cast<const uint4*>(p) : make_uint4(0u, 0u, 0u, 0u);
  } else {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if constexpr (kLd == 4) {
        w[i] = 4 * i < left ? *reinterpret_cast<const uint32_t*>(p + 4 * i) : 0u;
      } else if constexpr (kLd == 2) {
        const uint32_t lo = 4 * i < left ? *reinterpret_cast<const uint16_t*>(p + 4 * i) : 0u;
        w[i] = lo | (4 * i + 2 < left ? (uint32_t)*reinterpret_cast<const uint16_t*>(p + 4 * i + 2) << 16 : 0u);
      } else {
        w[i] = 0u;
#pragma unroll
        for (int e = 0; e < 4; ++e)
          w[i] |= 4 * i + e < left ? (uint32_t)*reinterpret_cast<const uint8_t*>(p + 4 * i + e) << (8 * e) : 0u;
      }
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
  }
}
// Lane t's 16 elements of the 64 from element k on; zeros past K.
template <int kMode, int kLd>
__device__ __forceinline__ void load16(const char* row, int k, int t, int K, bool ok, uint4 (&v)[2]) {
  if constexpr (kMode == kQuant) {
    k += 16 * t;
    v[0] = bytes16<kLd>(row + k, ok ? K - k : 0);
  } else {
    k += 8 * t;
    v[0] = bytes16<kLd>(row + (int64_t)k * 2, ok ? 2 * (K - k) : 0);
    v[1] = bytes16<kLd>(row + (int64_t)k * 2 + 64, ok ? 2 * (K - k - 32) : 0);
  }
}
template <int kMode>
__device__ __forceinline__ void pairs(const uint4 (&v)[2], uint32_t (&r)[8]) {
  if constexpr (kMode == kQuant) {
    s8_to_f16(v[0].x, r[0], r[1]);
    s8_to_f16(v[0].y, r[2], r[3]);
    s8_to_f16(v[0].z, r[4], r[5]);
    s8_to_f16(v[0].w, r[6], r[7]);
  } else {
    r[0] = v[0].x, r[1] = v[0].y, r[2] = v[0].z, r[3] = v[0].w;
    r[4] = v[1].x, r[5] = v[1].y, r[6] = v[1].z, r[7] = v[1].w;
  }
}

// kR: 16-row tiles of the weights (kGated: gate and up); kNT: groups of eight
// rows of x; kLd: bytes of a load; kAct: of the gated block.
template <int kMode, int kR, int kNT, int kWarps, int kLd, int kAct>
__global__ void __launch_bounds__(32 * kWarps, 16 / kWarps) k_rows(const RowArgs g) {
  constexpr int kBytes = kMode == kQuant ? 1 : 2, kCols = kMode == kGated ? 16 : 16 * kR;
  constexpr int kTok = kWarps * kR * kNT > 64 ? 16 : 8 * kNT;   // rows whose sums are joined at a time
  __shared__ float red[kWarps][kR][kTok][kStride];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, gid = lane >> 2, t = lane & 3;
  const int n0 = blockIdx.x * kCols, m0 = blockIdx.y * 8 * kNT;
  pdl_trigger();
  const char* w = (const char*)g.w;
  int64_t at[kR][2];                                     // byte offsets of the lane's two rows of each tile
  bool ok[kR][2];
#pragma unroll
  for (int q = 0; q < kR; ++q)
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int r = n0 + gid + 8 * h + (kMode == kGated ? 0 : 16 * q);
      ok[q][h] = r < g.n;
      at[q][h] = ((int64_t)(ok[q][h] ? r : 0) * g.k + (kMode == kGated ? q * g.up : 0)) * kBytes;
    }
  const int blocks = (g.k + 63) >> 6;
#pragma unroll
  for (int s = 0; s < 2; ++s) {
    const int k = 64 * (warp + kWarps * s) + (kMode == kQuant ? 16 : 8) * t;
    if (k < g.k) {
#pragma unroll
      for (int q = 0; q < kR; ++q)
#pragma unroll
        for (int h = 0; h < 2; ++h)
          asm volatile("prefetch.global.L2 [%0];" ::"l"(w + at[q][h] + (int64_t)k * kBytes));
    }
  }
  pdl_wait();
  float acc[kR][kNT][4];
#pragma unroll
  for (int q = 0; q < kR; ++q)
#pragma unroll
    for (int j = 0; j < kNT; ++j)
#pragma unroll
      for (int e = 0; e < 4; ++e) acc[q][j][e] = 0.f;

  // two steps at a time where the registers allow it: their loads are in flight together
  constexpr int kS = kNT <= 2 ? 2 : 1;
  for (int b = warp; b < blocks; b += kS * kWarps) {
    uint4 wv[kS][kR][2][2], xv[kS][kNT][2];
#pragma unroll
    for (int s = 0; s < kS; ++s) {
      const int k = 64 * (b + kWarps * s);
#pragma unroll
      for (int q = 0; q < kR; ++q)
#pragma unroll
        for (int h = 0; h < 2; ++h) load16<kMode, kLd>(w + at[q][h], k, t, g.k, ok[q][h], wv[s][q][h]);
#pragma unroll
      for (int j = 0; j < kNT; ++j) {
        const int m = m0 + 8 * j + gid;
        load16<kMode, kLd>((const char*)g.x + (int64_t)min(m, g.rows - 1) * g.ldx * kBytes, k, t, g.k, m < g.rows, xv[s][j]);
      }
    }
#pragma unroll
    for (int s = 0; s < kS; ++s) {
      uint32_t r[kR][2][8];
#pragma unroll
      for (int q = 0; q < kR; ++q)
#pragma unroll
        for (int h = 0; h < 2; ++h) pairs<kMode>(wv[s][q][h], r[q][h]);
#pragma unroll
      for (int j = 0; j < kNT; ++j) {
        uint32_t x[8];
        pairs<kMode>(xv[s][j], x);
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
          for (int q = 0; q < kR; ++q) {
            const uint32_t a[4] = {r[q][0][2 * i], r[q][1][2 * i], r[q][0][2 * i + 1], r[q][1][2 * i + 1]};
            if constexpr (kMode == kQuant) mma_f16(acc[q][j], a, x[2 * i], x[2 * i + 1]);
            else mma_bf16(acc[q][j], a, x[2 * i], x[2 * i + 1]);
          }
      }
    }
  }
#pragma unroll
  for (int j0 = 0; j0 < kNT; j0 += kTok / 8) {
    if (j0) __syncthreads();
#pragma unroll
    for (int q = 0; q < kR; ++q)
#pragma unroll
      for (int j = 0; j < kTok / 8; ++j) {
        const float(&v)[4] = acc[q][j0 + j];
        red[warp][q][8 * j + 2 * t][gid] = v[0];
        red[warp][q][8 * j + 2 * t + 1][gid] = v[1];
        red[warp][q][8 * j + 2 * t][gid + 8] = v[2];
        red[warp][q][8 * j + 2 * t + 1][gid + 8] = v[3];
      }
    __syncthreads();
    for (int i = threadIdx.x; i < kCols * kTok; i += 32 * kWarps) {
      const int ml = i / kCols, c = i % kCols, m = m0 + 8 * j0 + ml, n = n0 + c;
      if (m >= g.rows || n >= g.n) continue;
      auto sum = [&](int q) {
        float s = red[0][q][ml][c & 15];
#pragma unroll
        for (int v = 1; v < kWarps; ++v) s += red[v][q][ml][c & 15];
        return s;
      };
      const int64_t o = (int64_t)m * g.ldo + n;
      if constexpr (kMode == kGated) {
        float d;
        const float a = act_value<kAct, false>(sum(0), d), u = sum(kR - 1);
        ((__nv_bfloat16*)g.out)[o] = __float2bfloat16_rn(a * u);
        if (g.a) {
          const int64_t at_keep = (int64_t)m * g.ld_keep + n;
          const uint32_t wa = round_24(a), wp = round_24(u * d);
          ((uint16_t*)g.a)[at_keep] = (uint16_t)(wa >> 16);
          ((uint16_t*)g.p)[at_keep] = (uint16_t)(wp >> 16);
          g.a_lo[at_keep] = (uint8_t)(wa >> 8);
          g.p_lo[at_keep] = (uint8_t)(wp >> 8);
        }
      } else {
        float v = sum(c >> 4);
        if constexpr (kMode == kQuant) v = v * g.sx[m] * g.sw[n] + (g.bias ? g.bias[n] : 0.f);
        if (g.f32) ((float*)g.out)[o] = v;
        else ((__nv_bfloat16*)g.out)[o] = __float2bfloat16_rn(v);
      }
    }
  }
}

// ------------------------------------------------------ 32-bit gated blocks
// Few rows of fp32: multiply-adds, bound by the weights' bytes up to eight rows
// a pass.  A warp takes kC weight rows (the gated block: kC / 2 pairs) and
// kM rows of x; its lanes take K in groups of four, kC weight loads for kM
// loads of x (which the block's warps share in L1).  kVec: whole groups
// at multiples of 16 bytes; else element by element, in the same order.
template <int kC, int kM, bool kGate, bool kVec, int kAct>
__global__ void __launch_bounds__(256) k_rows32(const RowArgs g) {
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  constexpr int kN = kGate ? kC / 2 : kC;                 // output columns
  const int n0 = (blockIdx.x * 8 + warp) * kN, m0 = blockIdx.y * kM;
  pdl_trigger();
  pdl_wait();
  if (n0 >= g.n) return;
  const float *x[kM], *w[kC];
#pragma unroll
  for (int m = 0; m < kM; ++m) x[m] = (const float*)g.x + (int64_t)min(m0 + m, g.rows - 1) * g.ldx;
#pragma unroll
  for (int c = 0; c < kC; ++c)
    w[c] = (const float*)g.w + (int64_t)min(n0 + c % kN, g.n - 1) * g.k + (kGate && c >= kN ? g.up : 0);
  float acc[kC * kM];
#pragma unroll
  for (int i = 0; i < kC * kM; ++i) acc[i] = 0.f;
#pragma unroll 2
  for (int k = 4 * lane; k < g.k; k += 128) {
    auto four = [&](const float* p, float (&v)[4]) {
      if constexpr (kVec) {
        const float4 q = *reinterpret_cast<const float4*>(p + k);
        v[0] = q.x, v[1] = q.y, v[2] = q.z, v[3] = q.w;
      } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = k + e < g.k ? p[k + e] : 0.f;
      }
    };
    float wv[kC][4], xv[kM][4];
#pragma unroll
    for (int c = 0; c < kC; ++c) four(w[c], wv[c]);
#pragma unroll
    for (int m = 0; m < kM; ++m) four(x[m], xv[m]);
#pragma unroll
    for (int m = 0; m < kM; ++m)
#pragma unroll
      for (int c = 0; c < kC; ++c)
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[kM * c + m] = fmaf(wv[c][e], xv[m][e], acc[kM * c + m]);
  }
  // the lanes' sums: halving exchanges until every lane holds one of the kC kM
  // values, the lane's high bits its number, then the lanes of a value
  constexpr int kVals = kC * kM, kRep = 32 / kVals;
#pragma unroll
  for (int h = kVals / 2; h >= 1; h >>= 1) {
    const bool up = (lane & (h * kRep)) != 0;
#pragma unroll
    for (int i = 0; i < h; ++i) {
      const float keep = up ? acc[h + i] : acc[i], send = up ? acc[i] : acc[h + i];
      acc[i] = keep + __shfl_xor_sync(0xffffffffu, send, h * kRep);
    }
  }
  float v = acc[0];
#pragma unroll
  for (int r = kRep / 2; r >= 1; r >>= 1) v += __shfl_xor_sync(0xffffffffu, v, r);
  const int at = lane / kRep, c = at / kM, m = m0 + at % kM;
  float u = 0.f;
  if (kGate) u = __shfl_down_sync(0xffffffffu, v, 16);   // the pair's up column: half the values on
  const int n = n0 + c;
  if (c >= kN || m >= g.rows || n >= g.n || lane % kRep != 0) return;
  const int64_t o = (int64_t)m * g.ldo + n;
  if constexpr (kGate) {
    float d;
    const float a = act_value<kAct, true>(v, d);
    float h = a * u;
    ((float*)g.out)[o] = h;
    if (g.a) {
      const int64_t at_keep = (int64_t)m * g.ld_keep + n;
      ((float*)g.a)[at_keep] = a;
      ((float*)g.p)[at_keep] = u * d;
#pragma unroll
      for (int q = 0; q < 3; ++q) {
        const __nv_bfloat16 b = q == 0 ? __ushort_as_bfloat16((uint16_t)first_parts(h, 0.f)) : __float2bfloat16_rn(h);
        g.parts[q * g.part + at_keep] = b;
        h -= __bfloat162float(b);
      }
    }
  } else {
    ((float*)g.out)[o] = v;
  }
}

template <bool kGate, int kAct>
cudaError_t start32(const RowArgs& a, cudaStream_t st) {
  const bool vec = (((uintptr_t)a.x | (uintptr_t)a.w | (uintptr_t)(a.ldx * 4) | (uintptr_t)((int64_t)a.k * 4)) & 15) == 0;
  const dim3 block(256);
  // eight rows of x share four weight rows a warp; one row takes two, for twice the warps (gated block of 512
  // and 2048, four / two, us: one row 9.7 / 8.3, 8 rows 15.8 / 22.8)
  auto go = [&](auto c, auto m, auto v) {
    const int cols = 8 * (kGate ? c.value / 2 : c.value);
    launch_pdl(k_rows32<c.value, m.value, kGate, v.value, kAct>,
               dim3((unsigned)ceil_div(a.n, cols), (unsigned)ceil_div(a.rows, m.value)), block, 0, st, a);
  };
  auto go_v = [&](auto c, auto m) {
    if (vec) go(c, m, std::true_type());
    else go(c, m, std::false_type());
  };
  if (a.rows == 1) go_v(std::integral_constant<int, 2>(), std::integral_constant<int, 1>());
  else go_v(std::integral_constant<int, 4>(), std::integral_constant<int, 8>());
  return cudaGetLastError();
}

template <int kMode, int kR, int kWarps, int kLd, int kAct>
void launch(const RowArgs& a, cudaStream_t st) {
  const dim3 block(32 * kWarps), grid((unsigned)ceil_div(a.n, kMode == kGated ? 16 : 16 * kR), (unsigned)ceil_div(a.rows, 32));
  if (a.rows <= 8) launch_pdl(k_rows<kMode, kR, 1, kWarps, kLd, kAct>, grid, block, 0, st, a);
  else if (a.rows <= 16) launch_pdl(k_rows<kMode, kR, 2, kWarps, kLd, kAct>, grid, block, 0, st, a);
  else launch_pdl(k_rows<kMode, kR, 4, kWarps, kLd, kAct>, grid, block, 0, st, a);
}
template <int kMode, int kAct>
cudaError_t start(const RowArgs& a, cudaStream_t st) {
  constexpr int kBytes = kMode == kQuant ? 1 : 2, kR = kMode == kGated ? 2 : 1;
  const uintptr_t low = (uintptr_t)a.x | (uintptr_t)a.w | (uintptr_t)(a.ldx * kBytes) | (uintptr_t)((int64_t)a.k * kBytes);
  // sixteen warps a CTA where a warp of eight would take its loads in several turns and there is about one CTA
  // per SM, or two of few rows (sixteen / eight, us): 8-bit 2048 -> 4096, one row 3.2 / 3.9, 32 rows 6.4 / 4.9;
  // 2048 -> 2048, 32 rows 4.1 / 4.6, 64 rows 7.0 / 5.1; 1024 -> 4096, 8 rows 3.2 / 3.1; gated block of 512 and
  // 2048, 8 rows 4.6 / 5.8; of 1024 and 2048, 8 rows 5.1 / 6.3, 64 rows 10.9 / 10.2
  const int64_t few = ceil_div(a.n, 16) * ceil_div(a.rows, 32);
  const bool deep = few <= (a.rows <= (kMode == kQuant ? 8 : 32) ? 2 : 1) * kSms && a.k * kBytes > 1024;
  if ((low & 15) == 0) {
    if (deep) {
      launch<kMode, kR, 16, 16, kAct>(a, st);
    } else if constexpr (kMode == kGated) {
      launch<kMode, kR, 8, 16, kAct>(a, st);
    } else {
      // many columns: 32 a CTA, so that x comes from L2 half as often (8-bit, 512 -> 16000, 128 rows 24 -> 20 us;
      // one row 3.1 -> 3.4)
      if (few > 2 * kSms) launch<kMode, 2, 8, 16, kAct>(a, st);
      else launch<kMode, 1, 8, 16, kAct>(a, st);
    }
  } else if ((low & 3) == 0) {
    launch<kMode, kR, 8, 4, kAct>(a, st);
  } else {
    launch<kMode, kR, 8, kBytes, kAct>(a, st);
  }
  return cudaGetLastError();
}

}  // namespace

bool rows_take32(int64_t rows, int64_t weights) { return rows <= 16 || (rows <= 64 && rows * weights <= 220000000); }

bool rows_take(int64_t rows, int64_t weights, int64_t pitch, bool q8) {
  const int64_t work = rows * weights;
  if (pitch % 4 != 0) return rows <= 1024 && work <= (q8 ? 60000000 : 70000000);
  const bool whole = pitch % 16 == 0;
  if (rows <= (q8 && whole ? 128 : 32)) return true;
  return rows <= 1024 && work <= (q8 ? (whole ? 700000000 : 300000000) : (whole ? 540000000 : 250000000));
}

cudaError_t rows_gated(const RowsGated& q, cudaStream_t st) {
  RowArgs r{};
  r.x = q.x, r.w = q.w_gu, r.ldx = q.ldx, r.up = (int64_t)q.f * q.d, r.rows = (int32_t)q.rows, r.k = q.d, r.n = q.f;
  r.out = q.h, r.ldo = q.ldh, r.a = q.a, r.p = q.p, r.parts = (__nv_bfloat16*)q.parts, r.ld_keep = q.ld_keep, r.part = q.part;
  r.a_lo = q.a_lo, r.p_lo = q.p_lo;
  if (q.f32) {
    if (q.act == TP_ACT_RELU) return start32<true, TP_ACT_RELU>(r, st);
    if (q.act == TP_ACT_SILU) return start32<true, TP_ACT_SILU>(r, st);
    return start32<true, TP_ACT_GELU>(r, st);
  }
  if (q.act == TP_ACT_RELU) return start<kGated, TP_ACT_RELU>(r, st);
  if (q.act == TP_ACT_SILU) return start<kGated, TP_ACT_SILU>(r, st);
  return start<kGated, TP_ACT_GELU>(r, st);
}

cudaError_t rows_plain(const void* x, int64_t ldx, const void* w, int64_t rows, int32_t k, int32_t n, bool f32, void* y,
                       cudaStream_t st) {
  RowArgs r{};
  r.x = x, r.w = w, r.ldx = ldx, r.rows = (int32_t)rows, r.k = k, r.n = n, r.out = y, r.ldo = n;
  return f32 ? start32<false, -1>(r, st) : start<kPlain, -1>(r, st);
}

cudaError_t rows_quant(const int8_t* q, int64_t ldq, const float* sx, const int8_t* w, const float* sw, const float* bias,
                       int64_t rows, int32_t k, int32_t n, bool f32, void* y, cudaStream_t st) {
  RowArgs r{};
  r.x = q, r.w = w, r.ldx = ldq, r.rows = (int32_t)rows, r.k = k, r.n = n, r.out = y, r.ldo = n;
  r.sx = sx, r.sw = sw, r.bias = bias, r.f32 = f32;
  return start<kQuant, -1>(r, st);
}

}  // namespace tp
