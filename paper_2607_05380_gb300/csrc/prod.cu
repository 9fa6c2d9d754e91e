// prod.cu -- single products on tcgen05 with fused epilogues (see prod.cuh).
//
// A persistent launch: each CTA (or CTA pair) walks output tiles of 128 (256)
// rows by n_tile columns with stride gridDim.  Warp 0 stages 64-wide K blocks
// of both operands by TMA into a ring in shared memory (128-byte swizzle),
// warp 1 issues tcgen05.mma (K = 16 an instruction) into one of two TMEM
// accumulators, warps 2-9 read the other and run the epilogue.  K-major and
// MN-major operands are read straight from their row-major arrays.
//
// Bound by the tensor cores where all three sizes are large (a CTA pair's
// 256 x 256 tile streams 32 KB per SM and K block), by the operands' bytes
// where a product has few rows.
//
// 32-bit operands enter as three bf16 parts whose sum they are; the six
// products of parts above 2^-24 go into the same accumulator, smallest first,
// so that only the last of them rounds at the sum's own size.  The
// accumulators do not round to nearest: a chain of n instructions ends about
// n 10^-8 of its value off, so a chain takes at most kChainKb K blocks; a
// tile has two, and longer reductions are split.
//
// Reductions are split over CTAs where a launch has too few tiles; the parts'
// sums are then added in a fixed order by k_prod_join.
//
// Every wait is bounded (2 s): a role that gives up sets the error word that
// pack_ops_check reads and an abort flag; the others then stop, copies and
// MMAs in flight are waited for, TMEM is freed and the CTA exits.
#include <cudaTypedefs.h>

#include <algorithm>
#include <atomic>
#include <cstdarg>
#include <cstdio>
#include <mutex>
#include <type_traits>

#include "kernels.cuh"
#include "prod.cuh"
#include "rows.cuh"
#include "tc_ptx.cuh"

namespace tp {

namespace {

constexpr int kEpiWarps = 8, kThreads = 64 + 32 * kEpiWarps;
constexpr int kABytes = 128 * 128;       // 128 rows of a K block
constexpr int kBox = 64 * 128;           // a 64 x 64 MN-major box
constexpr int kMaxStages = 8;
constexpr int kBufBytes = 32 * 32 * 4;   // per epilogue warp
constexpr int kSmemMax = 232448;
constexpr int kTmemCols = 512, kAccCols = 256;
constexpr uint64_t kWaitNs = 2000000000ull;
constexpr int kChainKb = 16;

__device__ int g_prod_err;

struct Tail {
  uint64_t full[kMaxStages], empty[kMaxStages], tfull[2], tempty[2], done;
  uint32_t tmem_base;
  int abort;
};

struct ProdArgs {
  CUtensorMap map[kProdMaps];
  ProdJob job[kProdJobs];
  int32_t n_jobs, n_tiles, fp16, n_tile, chains, stages;
};
static_assert(sizeof(ProdArgs) <= 4096, "kernel parameters");

__device__ __forceinline__ void tma_load_3d(uint32_t dst, const CUtensorMap* map, uint64_t* bar, int x, int y, int z) {
  asm volatile(
      "cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5}], [%2];" ::"r"(
          dst),
      "l"(map), "r"(smem_u32(bar)), "r"(x), "r"(y), "r"(z)
      : "memory");
}
__device__ __forceinline__ void tma_load_3d_pair(uint32_t dst, const CUtensorMap* map, uint32_t bar, int x, int y, int z) {
  asm volatile(
      "cp.async.bulk.tensor.3d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, "
      "%5}], [%2];" ::"r"(dst),
      "l"(map), "r"(bar), "r"(x), "r"(y), "r"(z)
      : "memory");
}

// A tile's place: job, output origin and K blocks.
struct Tile {
  int job, m0, n0, kb0, kbn, split;
};
template <int kCta>
__device__ __forceinline__ Tile tile_at(const ProdArgs& g, int t) {
  Tile r;
  r.job = 0;
  for (int j = 1; j < g.n_jobs; ++j)
    if (t >= g.job[j].tile0) r.job = j;
  const ProdJob& b = g.job[r.job];
  int local = t - b.tile0;
  const int per = b.tm * b.tn;
  r.split = local / per;
  local -= r.split * per;
  // eight row blocks at a time walk the columns, so that a wave's tiles share operands in L2
  const int group = local / (8 * b.tn);
  const int rows = min(8, b.tm - 8 * group);
  local -= group * 8 * b.tn;
  r.m0 = (8 * group + local % rows) * 128 * kCta;
  r.n0 = local / rows;
  r.kb0 = r.split * b.kb_split;
  r.kbn = min(b.kb_split, b.kb - r.kb0);
  return r;
}

__device__ __forceinline__ bool vec_ok(const void* p, int64_t ld, int bytes) {
  return ((uintptr_t)p & 15) == 0 && ((ld * bytes) & 15) == 0;
}

// A warp's 32 x 32 chunk (lane = row) written as row segments through its
// buffer: out rows r0 .. r0 + 31 below m_lim, columns c0 .. c0 + 31 below n_lim.
__device__ __forceinline__ void emit_bf16(uint8_t* buf, int lane, const uint32_t (&pk)[16], __nv_bfloat16* out,
                                          int64_t ld, int r0, int m_lim, int c0, int n_lim, bool vec) {
  __syncwarp();
#pragma unroll
  for (int s = 0; s < 4; ++s)
    *reinterpret_cast<uint4*>(buf + lane * 64 + ((s ^ ((lane >> 1) & 3)) << 4)) =
        make_uint4(pk[4 * s], pk[4 * s + 1], pk[4 * s + 2], pk[4 * s + 3]);
  __syncwarp();
  const int slot = lane & 3, c = c0 + 8 * slot;
#pragma unroll
  for (int it = 0; it < 4; ++it) {
    const int row = 8 * it + (lane >> 2);
    const uint4 v = *reinterpret_cast<const uint4*>(buf + row * 64 + ((slot ^ ((row >> 1) & 3)) << 4));
    if (r0 + row >= m_lim) continue;
    __nv_bfloat16* o = out + (int64_t)(r0 + row) * ld + c;
    if (vec && c + 8 <= n_lim) {
      *reinterpret_cast<uint4*>(o) = v;
    } else {
      const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (c + e < n_lim) reinterpret_cast<uint16_t*>(o)[e] = (uint16_t)(w[e >> 1] >> (16 * (e & 1)));
    }
  }
}
__device__ __forceinline__ void emit_f32(uint8_t* buf, int lane, const float (&v)[32], float* out, int64_t ld, int r0,
                                         int m_lim, int c0, int n_lim, bool vec) {
  __syncwarp();
#pragma unroll
  for (int s = 0; s < 8; ++s)
    *reinterpret_cast<float4*>(buf + lane * 128 + ((s ^ (lane & 7)) << 4)) =
        make_float4(v[4 * s], v[4 * s + 1], v[4 * s + 2], v[4 * s + 3]);
  __syncwarp();
  const int slot = lane & 7, c = c0 + 4 * slot;
#pragma unroll
  for (int it = 0; it < 8; ++it) {
    const int row = 4 * it + (lane >> 3);
    const float4 w = *reinterpret_cast<const float4*>(buf + row * 128 + ((slot ^ (row & 7)) << 4));
    if (r0 + row >= m_lim) continue;
    float* o = out + (int64_t)(r0 + row) * ld + c;
    if (vec && c + 4 <= n_lim) {
      *reinterpret_cast<float4*>(o) = w;
    } else {
      const float e[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
      for (int k = 0; k < 4; ++k)
        if (c + k < n_lim) o[k] = e[k];
    }
  }
}
// fp32 values as one bf16 number each, or as three whose sum they are
// (buffers `part` elements apart).
__device__ __forceinline__ void emit_parts(uint8_t* buf, int lane, float (&v)[32], bool three, __nv_bfloat16* out,
                                           int64_t part, int64_t ld, int r0, int m_lim, int c0, int n_lim, bool vec) {
  uint32_t pk[16];
#pragma unroll 1
  for (int q = 0; q < (three ? 3 : 1); ++q) {
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      pk[e] = pack_bf16x2(v[2 * e], v[2 * e + 1]);
      v[2 * e] -= __uint_as_float(pk[e] << 16);
      v[2 * e + 1] -= __uint_as_float(pk[e] & 0xFFFF0000u);
    }
    emit_bf16(buf, lane, pk, out + q * part, ld, r0, m_lim, c0, n_lim, vec);
  }
}

// 32 values of a row (fp32 or bf16) from column c0 on, zeros past n_lim.
template <bool kF32>
__device__ __forceinline__ void load_row(const void* base, int64_t at, int c0, int n_lim, float (&v)[32]) {
  if constexpr (kF32) {
    const float* p = (const float*)base + at + c0;
#pragma unroll
    for (int s = 0; s < 8; ++s) {
      // the pitch is a multiple of 8 elements: whole groups may be read
      const float4 w = c0 + 4 * s < n_lim ? *reinterpret_cast<const float4*>(p + 4 * s) : make_float4(0.f, 0.f, 0.f, 0.f);
      v[4 * s] = w.x, v[4 * s + 1] = w.y, v[4 * s + 2] = w.z, v[4 * s + 3] = w.w;
    }
  } else {
    const __nv_bfloat16* p = (const __nv_bfloat16*)base + at + c0;
#pragma unroll
    for (int s = 0; s < 4; ++s) {
      const uint4 w = c0 + 8 * s < n_lim ? *reinterpret_cast<const uint4*>(p + 8 * s) : make_uint4(0u, 0u, 0u, 0u);
      const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        v[8 * s + 2 * e] = __uint_as_float(u[e] << 16);
        v[8 * s + 2 * e + 1] = __uint_as_float(u[e] & 0xFFFF0000u);
      }
    }
  }
}

// The epilogue of one 32 x 32 chunk; acc: its accumulator (kEpiGated: the
// gate product), acc2: the up product.
template <int kEpi, int kAct, bool kF32>
__device__ __forceinline__ void epilogue(const ProdArgs& g, const ProdJob& j, uint8_t* buf, int lane, float (&acc)[32],
                                         float (&acc2)[32], int r0, int c0) {
  const int row = r0 + lane;
  if constexpr (kEpi == kEpiGated) {
    const bool keep = j.a != nullptr;
    float da[32];
#pragma unroll
    for (int e = 0; e < 32; ++e) {
      float d;
      const float a = act_value<kAct, kF32>(acc[e], d);
      da[e] = acc2[e] * d;
      acc2[e] *= a;
      acc[e] = a;
    }
    if (keep) {
      if constexpr (kF32) {
        emit_f32(buf, lane, acc, (float*)j.a, j.ldo, r0, j.M, c0, j.N, true);
        emit_f32(buf, lane, da, (float*)j.p, j.ldo, r0, j.M, c0, j.N, true);
      } else {
        emit_parts(buf, lane, acc, false, (__nv_bfloat16*)j.a, 0, j.ldo, r0, j.M, c0, j.N, true);
        emit_parts(buf, lane, da, false, (__nv_bfloat16*)j.p, 0, j.ldo, r0, j.M, c0, j.N, true);
      }
    }
    emit_parts(buf, lane, acc2, kF32, (__nv_bfloat16*)j.out, j.part, j.ldo, r0, j.M, c0, j.N, true);
  } else if constexpr (kEpi == kEpiDgated) {
    float f[32];
    const int64_t at = (int64_t)min(row, j.M - 1) * j.ldo;
    load_row<kF32>(j.p, at, c0, j.N, f);
#pragma unroll
    for (int e = 0; e < 32; ++e) f[e] *= acc[e];
    emit_parts(buf, lane, f, kF32, (__nv_bfloat16*)j.out, j.part, j.ldo, r0, j.M, c0, j.N, true);
    load_row<kF32>(j.a, at, c0, j.N, f);
#pragma unroll
    for (int e = 0; e < 32; ++e) f[e] *= acc[e];
    emit_parts(buf, lane, f, kF32, (__nv_bfloat16*)j.out + j.half, j.part, j.ldo, r0, j.M, c0, j.N, true);
  } else {
    if constexpr (kEpi == kEpiQuant) {
      const float sx = row < j.M ? j.sx[row] : 0.f;
      const int c = c0 + lane;
      const float sw = c < j.N ? j.sw[c] : 0.f, b = c < j.N && j.bias ? j.bias[c] : 0.f;
#pragma unroll
      for (int e = 0; e < 32; ++e)
        acc[e] = acc[e] * sx * __shfl_sync(0xffffffffu, sw, e) + __shfl_sync(0xffffffffu, b, e);
    }
    const bool vec = vec_ok(j.out, j.ldo, kF32 ? 4 : 2);
    if constexpr (kF32) emit_f32(buf, lane, acc, (float*)j.out, j.ldo, r0, j.M, c0, j.N, vec);
    else emit_parts(buf, lane, acc, false, (__nv_bfloat16*)j.out, 0, j.ldo, r0, j.M, c0, j.N, vec);
  }
}

template <int kCta, int kEpi, int kAct, bool kF32>
__global__ void __launch_bounds__(kThreads, 1) k_prod(const __grid_constant__ ProdArgs g) {
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = (uint8_t*)(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);
  const int nh = g.n_tile / kCta;                       // rows of B that this CTA stages
  const uint32_t stage_bytes = kABytes + (uint32_t)nh * 128;
  const int stages = g.stages;
  uint8_t* bufs = smem + stages * stage_bytes;
  Tail* tl = (Tail*)(bufs + kEpiWarps * kBufBytes);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int rank = kCta == 2 ? (int)cluster_rank() : 0;
  const bool leader = rank == 0;
  const int clu = blockIdx.x / kCta, n_clu = gridDim.x / kCta;

  if (threadIdx.x == 0) {
    for (int s = 0; s < stages; ++s) {
      mbar_init(&tl->full[s], 1);
      mbar_init(&tl->empty[s], 1);
    }
    for (int b = 0; b < 2; ++b) {
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
  if (kCta == 2) cluster_sync();   // the peer's barriers exist before any copy or arrival targets them
  pdl_wait();                      // the set-up above overlaps the previous kernel
  const uint32_t tmem = tl->tmem_base;
  volatile int* abort_flag = &tl->abort;
  int* err = &g_prod_err;

  if (warp == 0) {
    // ------------------------------------------------------------ producer
    uint32_t stage = 0, phase = 0, issued = 0, last_parity = 0;
    bool ok = true;
    for (int t = clu; ok && t < g.n_tiles; t += n_clu) {
      const Tile u = tile_at<kCta>(g, t);
      const ProdJob& j = g.job[u.job];
      const int nbA = j.a_mn ? 2 : 1;
      // B: K-major one box of nh rows (kEpiGated in one CTA: gate and up rows apart), MN-major boxes of 64
      constexpr bool kTwoHalves = kEpi == kEpiGated && kCta == 1;
      const int nbB = j.b_mn ? nh >> 6 : (kTwoHalves ? 2 : 1);
      const int qb = lane - nbA;
      const bool is_a = lane < nbA, mine = is_a || qb < nbB;
      const CUtensorMap* map = &g.map[is_a ? j.map_a : j.map_b];
      const bool mn = is_a ? j.a_mn != 0 : j.b_mn != 0;
      int xy, add_seg = 0;
      uint32_t off;
      if (is_a) {
        xy = u.m0 + rank * 128 + 64 * lane;
        off = (uint32_t)lane * kBox;
      } else if (kEpi == kEpiGated) {
        // the tile's columns: n_tile / 2 of the gate, then the same of the up half
        xy = u.n0 * (g.n_tile / 2);
        add_seg = (kCta == 2 ? rank : qb) * j.up;
        off = kABytes + (kCta == 2 ? 0u : (uint32_t)qb * (g.n_tile / 2) * 128);
      } else {
        xy = u.n0 * g.n_tile + rank * nh + 64 * qb;
        off = kABytes + (uint32_t)qb * kBox;
      }
      for (int q = 0; ok && q < j.n_pairs; ++q) {
        const int seg = (is_a ? j.sa[q] : j.sb[q]) + add_seg;
        for (int kb = u.kb0; kb < u.kb0 + u.kbn; ++kb) {
          bool got = true;
          if (lane == 0) {
            got = mbar_wait(&tl->empty[stage], phase ^ 1u, abort_flag, err, kWaitNs, 41);
            if (got && leader) mbar_expect_tx(&tl->full[stage], kCta * stage_bytes);
          }
          if (!__shfl_sync(0xffffffffu, got, 0)) {
            ok = false;
            break;
          }
          if (mine) {
            const uint32_t dst = smem_u32(smem + stage * stage_bytes) + off;
            const int x = mn ? xy : 64 * kb, y = mn ? 64 * kb : xy;
            if constexpr (kCta == 2) tma_load_3d_pair(dst, map, mapa(smem_u32(&tl->full[stage]), 0), x, y, seg);
            else tma_load_3d(dst, map, &tl->full[stage], x, y, seg);
          }
          issued |= 1u << stage;
          last_parity = (last_parity & ~(1u << stage)) | (phase << stage);
          if (++stage == (uint32_t)stages) {
            stage = 0;
            phase ^= 1u;
          }
        }
      }
    }
    if (lane == 0 && leader)   // every copy has landed before the CTA leaves
      for (int s = 0; s < stages; ++s)
        if (issued & (1u << s)) {
          int dummy = 0;
          mbar_wait(&tl->full[s], (last_parity >> s) & 1u, &dummy, err, kWaitNs, 42);
        }
  } else if (warp == 1) {
    if (lane == 0 && leader) {
      // --------------------------------------------------------------- MMA
      const uint32_t s0 = smem_u32(smem);
      const uint64_t dA_k = smem_desc(s0, 16, 1024), dA_mn = smem_desc(s0, kBox, 1024);
      const uint64_t dB_k = smem_desc(s0 + kABytes, 16, 1024), dB_mn = smem_desc(s0 + kABytes, kBox, 1024);
      const uint32_t step = stage_bytes >> 4;
      uint32_t stage = 0, phase = 0, acc = 0, acc_phase = 0;
      bool ok = true;
      for (int t = clu; ok && t < g.n_tiles; t += n_clu) {
        const Tile u = tile_at<kCta>(g, t);
        const ProdJob& j = g.job[u.job];
        if (!mbar_wait(&tl->tempty[acc], acc_phase ^ 1u, abort_flag, err, 2 * kWaitNs, 43)) break;
        tc_fence_after();
        const uint32_t d0 = tmem + acc * kAccCols;
        uint32_t idesc = instr_desc(128 * kCta, g.n_tile, j.a_mn, j.b_mn);
        if (g.fp16) idesc &= ~((1u << 7) | (1u << 10));
        const uint64_t ta = j.a_mn ? dA_mn : dA_k, tb = j.b_mn ? dB_mn : dB_k;
        const uint32_t ka = j.a_mn ? 2048 >> 4 : 32 >> 4, kb_ = j.b_mn ? 2048 >> 4 : 32 >> 4;
        const int split_at = g.chains == 2 ? (u.kbn + 1) >> 1 : u.kbn;   // first K block of the second chain
        for (int q = 0; ok && q < j.n_pairs; ++q) {
          for (int kb = 0; kb < u.kbn; ++kb) {
            if (!mbar_wait(&tl->full[stage], phase, abort_flag, err, 2 * kWaitNs, 44)) {
              ok = false;
              break;
            }
            const uint64_t sa = ta + stage * step, sb = tb + stage * step;
            const uint32_t d = d0 + (kb >= split_at ? kAccCols / 2 : 0);
            const uint32_t first = q > 0 || (kb != 0 && kb != split_at) ? 1u : 0u;
            umma_bf16<kCta>(d, sa, sb, idesc, first);
            umma_bf16<kCta>(d, sa + ka, sb + kb_, idesc, 1u);
            umma_bf16<kCta>(d, sa + 2 * ka, sb + 2 * kb_, idesc, 1u);
            umma_bf16<kCta>(d, sa + 3 * ka, sb + 3 * kb_, idesc, 1u);
            umma_commit<kCta>(&tl->empty[stage]);
            if (++stage == (uint32_t)stages) {
              stage = 0;
              phase ^= 1u;
            }
          }
        }
        if (!ok) break;
        umma_commit<kCta>(&tl->tfull[acc]);
        acc ^= 1u;
        if (acc == 0) acc_phase ^= 1u;
      }
      umma_commit<kCta>(&tl->done);   // all MMAs are over before TMEM is freed
      int dummy = 0;
      mbar_wait(&tl->done, 0, &dummy, err, kWaitNs, 45);
    }
  } else {
    // ------------------------------------------------------------ epilogue
    const int q = warp & 3, half = (warp - 2) >> 2;
    uint8_t* buf = bufs + (warp - 2) * kBufBytes;
    uint32_t acc = 0, acc_phase = 0;
    const int cols = kEpi == kEpiGated ? g.n_tile / 2 : g.n_tile;
    for (int t = clu; t < g.n_tiles; t += n_clu) {
      const Tile u = tile_at<kCta>(g, t);
      const ProdJob& j = g.job[u.job];
      if (!__all_sync(0xffffffffu, mbar_wait(&tl->tfull[acc], acc_phase, abort_flag, err, 2 * kWaitNs, 46))) break;
      tc_fence_after();
      const uint32_t ta = tmem + ((uint32_t)(32 * q) << 16) + acc * kAccCols;
      const int r0 = u.m0 + rank * 128 + 32 * q;
      const bool second = g.chains == 2 && u.kbn > 1;
#pragma unroll 1
      for (int c = 32 * half; c < cols; c += 64) {
        uint32_t v[32];
        float a[32], a2[32];
        tmem_ld32(ta + c, v);
#pragma unroll
        for (int e = 0; e < 32; ++e) a[e] = __uint_as_float(v[e]);
        if (second) {
          tmem_ld32(ta + kAccCols / 2 + c, v);
#pragma unroll
          for (int e = 0; e < 32; ++e) a[e] += __uint_as_float(v[e]);
        }
        if constexpr (kEpi == kEpiGated) {
          tmem_ld32(ta + cols + c, v);
#pragma unroll
          for (int e = 0; e < 32; ++e) a2[e] = __uint_as_float(v[e]);
          if (second) {
            tmem_ld32(ta + kAccCols / 2 + cols + c, v);
#pragma unroll
            for (int e = 0; e < 32; ++e) a2[e] += __uint_as_float(v[e]);
          }
        }
        const int c0 = u.n0 * cols + c;
        if (r0 >= j.M || c0 >= j.N) continue;   // warp-uniform
        if (j.splits > 1)
          emit_f32(buf, lane, a, j.partial + (int64_t)u.split * j.M * j.ldp, j.ldp, r0, j.M, c0, j.N, true);
        else
          epilogue<kEpi, kAct, kF32>(g, j, buf, lane, a, a2, r0, c0);
      }
      tc_fence_before();
      __syncwarp();
      if (lane == 0) {   // the loads above have completed
        if constexpr (kCta == 2) mbar_arrive_cluster_relaxed(mapa(smem_u32(&tl->tempty[acc]), 0));
        else mbar_arrive_relaxed(&tl->tempty[acc]);
      }
      acc ^= 1u;
      if (acc == 0) acc_phase ^= 1u;
    }
  }

  pdl_trigger();   // not earlier: CTAs of the next kernel parked beside a running product slow it down
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  if (kCta == 2) cluster_sync();
  if (warp == 1) {
    if constexpr (kCta == 2)
      asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(kTmemCols) : "memory");
    else
      asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(kTmemCols) : "memory");
  }
}

// ------------------------------------------------- joining split reductions
struct JoinArgs {
  ProdJob job[kProdJobs];
  int32_t n_jobs, epi;
};
// out = the splits' sums added in order (kEpiQuant: scaled); four columns per thread.
template <bool kF32>
__global__ void __launch_bounds__(256) k_prod_join(const __grid_constant__ JoinArgs g) {
  pdl_trigger();
  pdl_wait();
  const ProdJob& j = g.job[blockIdx.y];
  const int groups = (j.N + 3) >> 2;
  const int64_t total = (int64_t)j.M * groups, plane = (int64_t)j.M * j.ldp;
  const bool vec = vec_ok(j.out, j.ldo, kF32 ? 4 : 2);
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < total; i += (int64_t)gridDim.x * 256) {
    const int64_t r = i / groups;
    const int c = (int)(i - r * groups) * 4;
    const float* p = j.partial + r * j.ldp + c;
    float4 s = *reinterpret_cast<const float4*>(p);
#pragma unroll 4
    for (int k = 1; k < j.splits; ++k) {
      const float4 v = *reinterpret_cast<const float4*>(p + k * plane);
      s.x += v.x, s.y += v.y, s.z += v.z, s.w += v.w;
    }
    float e[4] = {s.x, s.y, s.z, s.w};
    if (g.epi == kEpiQuant) {
      const float sx = j.sx[r];
#pragma unroll
      for (int k = 0; k < 4; ++k)
        if (c + k < j.N) e[k] = e[k] * sx * j.sw[c + k] + (j.bias ? j.bias[c + k] : 0.f);
    }
    if constexpr (kF32) {
      float* o = (float*)j.out + r * j.ldo + c;
      if (vec && c + 4 <= j.N) *reinterpret_cast<float4*>(o) = make_float4(e[0], e[1], e[2], e[3]);
      else
        for (int k = 0; k < 4 && c + k < j.N; ++k) o[k] = e[k];
    } else {
      __nv_bfloat16* o = (__nv_bfloat16*)j.out + r * j.ldo + c;
      if (vec && c + 4 <= j.N)
        *reinterpret_cast<uint2*>(o) = make_uint2(pack_bf16x2(e[0], e[1]), pack_bf16x2(e[2], e[3]));
      else
        for (int k = 0; k < 4 && c + k < j.N; ++k) o[k] = __float2bfloat16_rn(e[k]);
    }
  }
}

// ------------------------------------------------------------------ staging
// Eight elements per thread: one pass over the source, 16-byte stores.
__global__ void __launch_bounds__(256) k_stage(const __grid_constant__ StageLaunch g) {
  pdl_trigger();
  pdl_wait();
  const StageJob& j = g.job[blockIdx.y];
  const int groups = (int)(j.ldp >> 3);
  const int64_t total = j.rows * groups;
  const int eb = j.type == kStageF32 ? 4 : j.type == kStageS8 ? 1 : 2;
  const bool vec = ((uintptr_t)j.src & (eb == 1 ? 7 : 15)) == 0 && ((j.ld * eb) & (eb == 1 ? 7 : 15)) == 0;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < total; i += (int64_t)gridDim.x * 256) {
    const int64_t r = i / groups;
    const int c = (int)(i - r * groups) * 8;
    const int64_t seg = r / j.rows_seg, rs = r - seg * j.rows_seg;
    const bool whole = vec && c + 8 <= j.cols;
    if (j.type == kStageF32) {
      const float* p = (const float*)j.src + r * j.ld + c;
      float v[8];
      if (whole) {
        const float4 a = *reinterpret_cast<const float4*>(p), b = *reinterpret_cast<const float4*>(p + 4);
        v[0] = a.x, v[1] = a.y, v[2] = a.z, v[3] = a.w, v[4] = b.x, v[5] = b.y, v[6] = b.z, v[7] = b.w;
      } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = c + e < j.cols ? p[e] : 0.f;
      }
#pragma unroll
      for (int q = 0; q < 3; ++q) {
        uint32_t pk[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          pk[e] = pack_bf16x2(v[2 * e], v[2 * e + 1]);
          v[2 * e] -= __uint_as_float(pk[e] << 16);
          v[2 * e + 1] -= __uint_as_float(pk[e] & 0xFFFF0000u);
        }
        *reinterpret_cast<uint4*>((__nv_bfloat16*)j.dst + ((seg * 3 + q) * j.rows_seg + rs) * j.ldp + c) =
            make_uint4(pk[0], pk[1], pk[2], pk[3]);
      }
    } else {
      uint16_t h[8];
      if (j.type == kStageS8) {
        const int8_t* p = (const int8_t*)j.src + r * j.ld + c;
        int8_t b[8];
        if (whole) {
          const uint2 w = *reinterpret_cast<const uint2*>(p);
#pragma unroll
          for (int e = 0; e < 8; ++e) b[e] = (int8_t)((e < 4 ? w.x : w.y) >> (8 * (e & 3)));
        } else {
#pragma unroll
          for (int e = 0; e < 8; ++e) b[e] = c + e < j.cols ? p[e] : (int8_t)0;
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) h[e] = __half_as_ushort(__short2half_rn((short)b[e]));
      } else {
        const uint16_t* p = (const uint16_t*)j.src + r * j.ld + c;
#pragma unroll
        for (int e = 0; e < 8; ++e) h[e] = c + e < j.cols ? p[e] : (uint16_t)0;
      }
      *reinterpret_cast<uint4*>((uint16_t*)j.dst + (seg * j.rows_seg + rs) * j.ldp + c) =
          make_uint4(h[0] | (uint32_t)h[1] << 16, h[2] | (uint32_t)h[3] << 16, h[4] | (uint32_t)h[5] << 16,
                     h[6] | (uint32_t)h[7] << 16);
    }
  }
}

// ------------------------------------------------------------------- host
PFN_cuTensorMapEncodeTiled_v12000 get_encode() {
  static PFN_cuTensorMapEncodeTiled_v12000 fn = [] {
    void* p = nullptr;
    cudaDriverEntryPointQueryResult q;
    if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &p, 12000, cudaEnableDefault, &q) != cudaSuccess ||
        q != cudaDriverEntryPointSuccess)
      p = nullptr;
    return (PFN_cuTensorMapEncodeTiled_v12000)p;
  }();
  return fn;
}

bool encode(CUtensorMap* m, const ProdOperand& o, bool fp16, int box_rows) {
  auto fn = get_encode();
  if (!fn) return false;
  cuuint64_t dims[3] = {(cuuint64_t)o.cols, (cuuint64_t)o.rows, (cuuint64_t)o.n_seg};
  cuuint64_t strides[2] = {(cuuint64_t)o.ld * 2, (cuuint64_t)(o.n_seg > 1 ? o.seg : o.ld * 8) * 2};
  cuuint32_t box[3] = {64, (cuuint32_t)box_rows, 1};
  cuuint32_t es[3] = {1, 1, 1};
  return fn(m, fp16 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT16 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<void*>(o.base),
            dims, strides, box, es, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
            CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

int stage_count(int cta, int n_tile) {
  const int bytes = kABytes + n_tile / cta * 128;
  return std::min<int>(kMaxStages, (kSmemMax - 1024 - kEpiWarps * kBufBytes - (int)sizeof(Tail)) / bytes);
}

// Nanoseconds of one K block of a tile: the tensor cores' 6.28 (12.56) TFLOP/s
// a CTA (pair), or the staged bytes at about 100 GB/s an SM.
double kblock_ns(int cta, int n_tile) {
  const double mma = 128.0 * cta * n_tile * 64 * 2 / (12560.0 * cta);
  return std::max(mma, (kABytes + n_tile / cta * 128.0) / 100.0);
}

template <int kCta, int kEpi, int kAct, bool kF32>
cudaError_t launch(const ProdArgs& a, int max_clusters, cudaStream_t st) {
  const int stage_bytes = kABytes + a.n_tile / kCta * 128;
  const int smem = a.stages * stage_bytes + kEpiWarps * kBufBytes + (int)sizeof(Tail) + 1024;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(kCta * std::min(a.n_tiles, max_clusters));
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = kCta;
  attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = kCta == 2 ? 2 : 1;
  return cudaLaunchKernelEx(&cfg, k_prod<kCta, kEpi, kAct, kF32>, a);
}

// The kernels that launches choose from: f(kernel's constants).
template <typename F>
cudaError_t with_kernel(int cta, int epi, int act, bool f32, F f) {
  auto cta_of = [&](auto e, auto a, auto t) {
    if (cta == 2) return f(std::integral_constant<int, 2>(), e, a, t);
    return f(std::integral_constant<int, 1>(), e, a, t);
  };
  auto type_of = [&](auto e, auto a) {
    // 32-bit operands take tiles of one CTA only (prod_plan)
    if (f32) {
      if constexpr (e.value != kEpiQuant) return f(std::integral_constant<int, 1>(), e, a, std::true_type());
      else return cta_of(e, a, std::true_type());
    }
    return cta_of(e, a, std::false_type());
  };
  using None = std::integral_constant<int, -1>;
  using Gated = std::integral_constant<int, kEpiGated>;
  if (epi == kEpiPlain) return type_of(std::integral_constant<int, kEpiPlain>(), None());
  if (epi == kEpiDgated) return type_of(std::integral_constant<int, kEpiDgated>(), None());
  if (epi == kEpiQuant) return type_of(std::integral_constant<int, kEpiQuant>(), None());
  if (act == TP_ACT_RELU) return type_of(Gated(), std::integral_constant<int, TP_ACT_RELU>());
  if (act == TP_ACT_SILU) return type_of(Gated(), std::integral_constant<int, TP_ACT_SILU>());
  return type_of(Gated(), std::integral_constant<int, TP_ACT_GELU>());
}

constexpr int kMaxDevices = 64;
struct DeviceState {
  bool ready = false;
  int sms = 0, pairs = 0;
};
DeviceState g_dev[kMaxDevices];
std::mutex g_dev_mu;

// Once per device: shared-memory limits of the kernels, and how many CTA pairs fit.
cudaError_t device_state(DeviceState* out) {
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  if (dev < 0 || dev >= kMaxDevices) return cudaErrorInvalidDevice;
  std::lock_guard<std::mutex> lock(g_dev_mu);
  DeviceState& d = g_dev[dev];
  if (!d.ready) {
    if ((e = cudaDeviceGetAttribute(&d.sms, cudaDevAttrMultiProcessorCount, dev)) != cudaSuccess) return e;
    auto allow = [](auto c, auto k, auto a, auto t) {
      return cudaFuncSetAttribute(k_prod<c.value, k.value, a.value, t.value>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                  kSmemMax);
    };
    for (int v = 0; v < 4 * 3 * 4; ++v) {   // CTAs and type, activation, epilogue
      const int epi = v & 3, act = (v >> 2) % 3, ct = (v >> 2) / 3;
      if ((e = with_kernel(1 + (ct & 1), epi, act, ct >> 1, allow)) != cudaSuccess) return e;
    }
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(2 * d.sms);
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = stage_count(2, 256) * (kABytes + 128 * 128) + kEpiWarps * kBufBytes + (int)sizeof(Tail) + 1024;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = 2;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    if ((e = cudaOccupancyMaxActiveClusters(&d.pairs, (void*)k_prod<2, kEpiPlain, -1, false>, &cfg)) != cudaSuccess) return e;
    d.ready = true;
  }
  *out = d;
  return cudaSuccess;
}

}  // namespace

tp_status ops_fail(tp_status s, const char* fmt, ...) {
  char buf[320];
  va_list ap;
  va_start(ap, fmt);
  vsnprintf(buf, sizeof buf, fmt, ap);
  va_end(ap);
  record_thread_error(buf);
  return s;
}

tp_status ops_device() {
  static std::atomic<bool> found{false};
  if (found.load(std::memory_order_relaxed)) return TP_OK;
  int n = 0;
  const cudaError_t e = cudaGetDeviceCount(&n);
  if (e == cudaSuccess && n > 0) {
    found.store(true, std::memory_order_relaxed);
    return TP_OK;
  }
  cudaGetLastError();
  return ops_fail(TP_ECUDA, "no CUDA device: %s", cudaGetErrorString(e));
}

void prod_pairs(ProdJob& j, bool f32, int halves) {
  static const uint8_t pa[6] = {2, 0, 1, 1, 0, 0}, pb[6] = {0, 2, 1, 0, 1, 0};
  int n = 0;
  for (int q = 0; q < (f32 ? 6 : 1); ++q)
    for (int h = 0; h < halves; ++h, ++n) {
      j.sa[n] = f32 ? h * 3 + pa[q] : h;
      j.sb[n] = f32 ? h * 3 + pb[q] : h;
    }
  j.n_pairs = n;
}

void prod_plan(ProdLaunch& l, int64_t* partial_bytes) {
  struct Shape { int cta, n; };
  // a CTA pair's tile, then narrower ones of one CTA: few rows or columns
  static const Shape shapes[4] = {{2, 256}, {1, 256}, {1, 128}, {1, 64}};
  const bool may_split = l.epi == kEpiPlain || l.epi == kEpiQuant;
  const bool parts = l.f32 && !l.fp16;         // 32-bit operands: two chains in a 128-column tile
  double best = 1e300;
  ProdLaunch pick = l;
  for (const Shape& s : shapes) {
    if (parts && (s.cta != 1 || s.n > 128)) continue;
    const int units = kSms / s.cta, chains = parts ? 2 : 1;
    const int cols = l.epi == kEpiGated ? s.n / 2 : s.n;
    for (int level = 0; level < (may_split ? 6 : 1); ++level) {
      ProdLaunch p = l;
      p.cta = s.cta, p.n_tile = s.n, p.chains = chains, p.n_tiles = 0;
      double work = 0, longest = 0, join = 0;
      bool any = false;
      for (int k = 0; k < l.n_jobs; ++k) {
        ProdJob& j = p.job[k];
        j.kb = (int)ceil_div(j.K, 64);
        j.tm = (int)ceil_div(j.M, 128 * s.cta);
        j.tn = (int)ceil_div(j.N, cols);
        int per = j.kb;
        if (may_split) {
          per = std::max(std::min(j.kb, 4), (int)ceil_div(j.kb, 1 << level));
          if (parts) per = std::min(per, 2 * kChainKb);
        }
        j.splits = (int)ceil_div(j.kb, per);
        j.kb_split = (int)ceil_div(j.kb, j.splits);
        j.splits = (int)ceil_div(j.kb, j.kb_split);
        j.tile0 = p.n_tiles;
        const int64_t tiles = (int64_t)j.tm * j.tn * j.splits;
        p.n_tiles += (int)tiles;
        // a tile's K blocks, and what its epilogue keeps the next tile waiting
        const double t = 300.0 + (double)j.n_pairs * j.kb_split * kblock_ns(s.cta, s.n);
        work += t * tiles;
        longest = std::max(longest, t);
        if (j.splits > 1) {
          any = true;
          join += 2.0 * j.splits * j.M * j.N * 4 / 5000.0;
        }
      }
      const double waves = (double)ceil_div(p.n_tiles, units) * work / p.n_tiles;
      const double est = std::max(std::max(waves, longest), work / units) + join + (any ? 2500.0 : 0.0);
      if (est < best * 0.98) {
        best = est;
        pick = p;
      }
    }
  }
  l = pick;
  int64_t bytes = 0;
  for (int k = 0; k < l.n_jobs; ++k) {
    ProdJob& j = l.job[k];
    j.ldp = round_up(j.N, 4);
    if (j.splits > 1) bytes += round_up((int64_t)j.splits * j.M * j.ldp * 4, 256);
  }
  *partial_bytes = bytes;
}

cudaError_t prod_run(ProdLaunch& l, void* partial, cudaStream_t st, const char** what) {
  DeviceState dev;
  *what = "kernel attributes";
  cudaError_t e = device_state(&dev);
  if (e != cudaSuccess) return e;
  ProdArgs a;
  JoinArgs join;
  join.n_jobs = 0, join.epi = l.epi;
  Carver c(partial);
  a.n_jobs = l.n_jobs, a.n_tiles = l.n_tiles, a.fp16 = l.fp16, a.n_tile = l.n_tile;
  a.chains = l.chains, a.stages = stage_count(l.cta, l.n_tile);
  bool done[kProdMaps] = {};
  int64_t join_work = 0;
  *what = "cuTensorMapEncodeTiled";
  for (int k = 0; k < l.n_jobs; ++k) {
    ProdJob& j = l.job[k];
    if (j.splits > 1) {
      j.partial = (float*)c.take((int64_t)j.splits * j.M * j.ldp * 4);
      join.job[join.n_jobs++] = j;
      join_work = std::max<int64_t>(join_work, (int64_t)j.M * ceil_div(j.N, 4));
    }
    a.job[k] = j;
    // an operand is read with the same boxes by every product of a launch
    const int nh = l.epi == kEpiGated ? l.n_tile / 2 : l.n_tile / l.cta;
    if (!done[j.map_a] && !encode(&a.map[j.map_a], l.op[j.map_a], l.fp16, j.a_mn ? 64 : 128)) return cudaErrorInvalidValue;
    if (!done[j.map_b] && !encode(&a.map[j.map_b], l.op[j.map_b], l.fp16, j.b_mn ? 64 : nh)) return cudaErrorInvalidValue;
    done[j.map_a] = done[j.map_b] = true;
  }
  *what = "product launch";
  const int clusters = l.cta == 2 ? dev.pairs : dev.sms;
  e = with_kernel(l.cta, l.epi, l.act, l.f32, [&](auto c, auto k, auto a_, auto t) {
    return launch<c.value, k.value, a_.value, t.value>(a, clusters, st);
  });
  if (e == cudaSuccess && join.n_jobs) {
    *what = "join launch";
    const dim3 grid((unsigned)std::min<int64_t>(ceil_div(join_work, 256), kSms * 8), join.n_jobs);
    if (l.f32) launch_pdl(k_prod_join<true>, grid, dim3(256), 0, st, join);
    else launch_pdl(k_prod_join<false>, grid, dim3(256), 0, st, join);
    e = cudaGetLastError();
  }
  return e;
}

cudaError_t stage_run(const StageLaunch& s, cudaStream_t st) {
  int64_t most = 0;
  for (int k = 0; k < s.n; ++k) most = std::max<int64_t>(most, s.job[k].rows * (s.job[k].ldp >> 3));
  if (s.n == 0 || most == 0) return cudaSuccess;
  launch_pdl(k_stage, dim3((unsigned)std::min<int64_t>(ceil_div(most, 256), kSms * 8), s.n), dim3(256), 0, st, s);
  return cudaGetLastError();
}

}  // namespace tp

using namespace tp;

extern "C" tp_status pack_ops_check(void* cuda_stream) {
  int v = 0;
  cudaStream_t st = (cudaStream_t)cuda_stream;
  cudaError_t e = cudaMemcpyFromSymbolAsync(&v, g_prod_err, sizeof v, 0, cudaMemcpyDeviceToHost, st);
  if (e == cudaSuccess) e = cudaStreamSynchronize(st);
  if (e == cudaSuccess && v != 0) {
    const int zero = 0;
    e = cudaMemcpyToSymbolAsync(g_prod_err, &zero, sizeof zero, 0, cudaMemcpyHostToDevice, st);
    if (e == cudaSuccess) e = cudaStreamSynchronize(st);
  }
  if (e != cudaSuccess) {
    cudaGetLastError();   // reported here
    return ops_fail(TP_ECUDA, "pack_ops_check: %s", cudaGetErrorString(e));
  }
  if (v != 0) return ops_fail(TP_ETIMEOUT, "a wait of a tensor-core product gave up (site %d)", v);
  return TP_OK;
}
