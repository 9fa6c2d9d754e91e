// tc_warp.cuh -- what the warps of a tcgen05 product do as wholes: copies, MMAs
// and commits by one elected lane, TMEM loads, and a warp's 32 x 32 chunk of
// results on its way to memory.  Shared by prod.cu and f8.cu.
#pragma once

#include "tc_ptx.cuh"

namespace tp {
namespace {

constexpr uint64_t kWaitNs = 2000000000ull;   // of a bounded wait

// The producer and the MMA issuer walk their loops as whole, converged warps
// and leave the single thread to a predicate inside the instruction sequences
// below: the loops' values then live in the uniform registers that TMA and
// tcgen05.mma take their operands from.  (One lane in a branch of its own
// moved every operand there anew: 290 ns a K block whatever the tile's width.)
__device__ __forceinline__ bool wait_all(uint64_t* bar, uint32_t parity, volatile int* abort_flag, int* err,
                                         uint64_t budget_ns, int site) {
  if (__all_sync(0xffffffffu, mbar_try_wait(bar, parity))) return true;
  return __all_sync(0xffffffffu, mbar_wait_slow(bar, parity, abort_flag, err, budget_ns, site));
}
__device__ __forceinline__ void expect_elect(uint32_t bar, uint32_t bytes) {
  asm volatile(
      "{\n .reg .pred e;\n elect.sync _|e, 0xffffffff;\n @e mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;\n}\n" ::"r"(
          bar),
      "r"(bytes)
      : "memory");
}
// kCta 2: the copy completes on barrier `bar` of the pair's leader (a shared::cluster address)
template <int kCta>
__device__ __forceinline__ void tma_elect(uint32_t dst, const CUtensorMap* map, uint32_t bar, int x, int y, int z) {
  if constexpr (kCta == 2)
    asm volatile(
        "{\n .reg .pred e;\n elect.sync _|e, 0xffffffff;\n @e "
        "cp.async.bulk.tensor.3d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, "
        "%5}], [%2];\n}\n" ::"r"(dst),
        "l"(map), "r"(bar), "r"(x), "r"(y), "r"(z)
        : "memory");
  else
    asm volatile(
        "{\n .reg .pred e;\n elect.sync _|e, 0xffffffff;\n @e "
        "cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5}], "
        "[%2];\n}\n" ::"r"(dst),
        "l"(map), "r"(bar), "r"(x), "r"(y), "r"(z)
        : "memory");
}
template <int kCta>
__device__ __forceinline__ void commit_elect(uint32_t bar) {
  if constexpr (kCta == 2)
    asm volatile(
        "{\n .reg .pred e;\n elect.sync _|e, 0xffffffff;\n @e "
        "tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;\n}\n" ::"r"(
            bar),
        "h"((uint16_t)3)
        : "memory");
  else
    asm volatile(
        "{\n .reg .pred e;\n elect.sync _|e, 0xffffffff;\n @e "
        "tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];\n}\n" ::"r"(bar)
        : "memory");
}
__device__ __forceinline__ uint32_t uniform(uint32_t v) { return __shfl_sync(0xffffffffu, v, 0); }

// A warp's 32 lanes x 32 columns of TMEM; the values are there after tmem_wait
// and may be used once tmem_got has tied them to it.
__device__ __forceinline__ void tmem_ask32(uint32_t taddr, uint32_t (&v)[32]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
      "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
      : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7]), "=r"(v[8]),
        "=r"(v[9]), "=r"(v[10]), "=r"(v[11]), "=r"(v[12]), "=r"(v[13]), "=r"(v[14]), "=r"(v[15]), "=r"(v[16]),
        "=r"(v[17]), "=r"(v[18]), "=r"(v[19]), "=r"(v[20]), "=r"(v[21]), "=r"(v[22]), "=r"(v[23]), "=r"(v[24]),
        "=r"(v[25]), "=r"(v[26]), "=r"(v[27]), "=r"(v[28]), "=r"(v[29]), "=r"(v[30]), "=r"(v[31])
      : "r"(taddr));
}
__device__ __forceinline__ void tmem_wait() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void tmem_got(uint32_t (&v)[32]) {
#pragma unroll
  for (int e = 0; e < 32; ++e) asm volatile("" : "+r"(v[e]));
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
// Eight words of a lane's own row: a whole 32-byte sector (address a multiple of 32).
__device__ __forceinline__ void store32(void* p, const uint32_t* w) {
  asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(p), "r"(w[0]), "r"(w[1]), "r"(w[2]),
               "r"(w[3]), "r"(w[4]), "r"(w[5]), "r"(w[6]), "r"(w[7])
               : "memory");
}
__device__ __forceinline__ void load32(const void* p, uint32_t* w) {
  asm volatile("ld.global.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
               : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]), "=r"(w[4]), "=r"(w[5]), "=r"(w[6]), "=r"(w[7])
               : "l"(p)
               : "memory");
}
// A lane's 32 columns of its row straight to memory, in whole sectors: `out`
// is row r's column c0.  Columns from n on are written too where n is not a
// multiple of a sector's elements: rows have room for whole sectors.
__device__ __forceinline__ void put_bf16(const uint32_t (&pk)[16], __nv_bfloat16* out, bool live, int n) {
  if (!live) return;
  store32(out, pk);
  if (n > 16) store32(out + 16, pk + 8);
}
__device__ __forceinline__ void put_f32(const float (&v)[32], float* out, bool live, int n) {
  if (!live) return;
#pragma unroll
  for (int s = 0; s < 4; ++s) {
    uint32_t w[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) w[e] = __float_as_uint(v[8 * s + e]);
    if (n > 8 * s) store32(out + 8 * s, w);
  }
}
__device__ __forceinline__ void pack32(const float (&v)[32], uint32_t (&pk)[16]) {
#pragma unroll
  for (int e = 0; e < 16; ++e) pk[e] = pack_bf16x2(v[2 * e], v[2 * e + 1]);
}
}  // namespace
}  // namespace tp
