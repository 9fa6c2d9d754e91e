// prod.cu -- single products on tcgen05 with fused epilogues (see prod.cuh).
//
// A persistent launch: each CTA (or CTA pair) walks output tiles of 128 (256)
// rows by n_tile columns with stride gridDim.  Warps 0 and 10 stage 64-wide K
// blocks of A and B by TMA into a ring in shared memory (128-byte swizzle; one
// warp for both: 324 ns a K block of a pair's 256 columns, MN-major, against
// 287), warp 1 issues tcgen05.mma (K = 16 an instruction) into one of two TMEM
// accumulators, warps 2-9 read the other and run the epilogue.  K-major and
// MN-major operands are read straight from their row-major arrays.
//
// Bound by the tensor cores where all three sizes are large: a CTA pair's
// 256 x 256 tile streams 32 KB per SM and K block (a gated block of 1024 and
// 4096, 20011 rows, forward, 275 us: 1.83 PFLOP/s, 0.96 of cuBLAS's measured
// 8192^3 burst); by a launch's fill, last epilogues and uneven rounds, 4 to 7
// us, where they are not (2048 rows, 1024 and 2048, 33 us: 0.78 PFLOP/s).
//
// 32-bit operands enter as three bf16 parts whose sum they are; the six
// products of parts above 2^-24 go into the same accumulator, smallest first,
// so that only the last of them rounds at the sum's own size.  The
// accumulators do not round to nearest: a chain of n instructions ends about
// n 10^-8 of its value off, so a chain takes at most kChainKb K blocks; a
// tile has two, and longer reductions are split.
//
// Where the tiles do not come out even over the SMs, the K blocks of the last
// one to two rounds' tiles are shared out evenly instead: a cluster's run of
// them ends inside a tile, whose first part it takes before all else and whose
// fp32 sums it leaves in the workspace, and begins inside another, whose last
// part it takes at the end, adding the sums that the clusters before it have
// left there long since, in order.  A cluster publishes before it waits, and
// waits only on clusters of lower numbers, which are dispatched no later than
// it is, so the waits end whatever else holds SMs.
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

constexpr int kEpiWarps = 8, kThreads = 96 + 32 * kEpiWarps;   // and a producer each for A and B, and the MMA issuer
constexpr int kWarpB = 2 + kEpiWarps;
constexpr int kABytes = 128 * 128;       // 128 rows of a K block
constexpr int kBox = 64 * 128;           // a 64 x 64 MN-major box
constexpr int kMaxStages = 8;
constexpr int kBufBytes = 32 * 32 * 4;   // per epilogue warp
// kEpiDgated of a bf16 block: an epilogue warp's 32 x 32 values of u act'(g) and of act(g) as they come in by TMA,
// the upper 16 bits, then the lower 8
constexpr int kKeptHi = 32 * 32 * 2, kKeptLo = 32 * 32, kKeptBytes = 2 * (kKeptHi + kKeptLo);
constexpr int kMapHi = 2, kMapLo = 3, kMapOut = 4;   // its maps: act(g) and u act'(g), two segments; dg and du
constexpr int kSmemMax = 232448;
constexpr int kTmemCols = 512, kAccCols = 256;
constexpr uint64_t kWaitNs = 2000000000ull;
constexpr int kChainKb = 16;

__device__ int g_prod_err, g_prod_taken;
// Takes the error word, so that none that comes in meanwhile is erased.
__global__ void k_take_err() { g_prod_taken = atomicExch(&g_prod_err, 0); }

// What checks have taken, per device: how often, and the last site.
struct Failures {
  int count = 0, site = 0;
};
// pack_debug_ops_withhold: the next launch that shares out tiles spoils a flag.
std::atomic<bool> g_withhold{false};

struct Tail {
  uint64_t full[kMaxStages], empty[kMaxStages], tfull[2], tempty[2], done;
  uint64_t kept[kEpiWarps][2];   // a warp's two slots: filled
  uint32_t tmem_base;
  int abort;
};

struct ProdArgs {
  CUtensorMap map[kProdMaps];
  ProdJob job[kProdJobs];
  int32_t n_jobs, n_tiles, n_maps, fp16, n_tile, chains, stages;
  int32_t whole, part_kb;   // part_kb: longest reduction between two additions in fp32
  float* slots;             // [2][clusters][CTA][128 n_tile]: published sums; a cluster's own
  int* flags;               // [clusters][CTA][epilogue warp]
  int* zero;                // n_zero words are set to 0: the next launch's flags
  int32_t n_zero;
  int32_t cut[kSms + 1];
};
static_assert(sizeof(ProdArgs) <= 4096, "kernel parameters");

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
// One K block: four MMAs (K = 16 each), whose operands lie ka and kb (of 16
// bytes) apart; the first one adds to the accumulator if `add`.  Then `bar`
// (in every CTA of the tile) is told once they are over.
#define TP_MMA4(GROUP, COMMIT)                                                                                        \
  "{\n .reg .pred e, p, t;\n .reg .b64 a1, a2, a3, b1, b2, b3;\n elect.sync _|e, 0xffffffff;\n"                        \
  " setp.ne.b32 p, %4, 0;\n setp.eq.b32 t, 0, 0;\n"                                                                   \
  " add.s64 a1, %1, %5;\n add.s64 a2, a1, %5;\n add.s64 a3, a2, %5;\n"                                                \
  " add.s64 b1, %2, %6;\n add.s64 b2, b1, %6;\n add.s64 b3, b2, %6;\n"                                                \
  " @e tcgen05.mma.cta_group::" GROUP ".kind::f16 [%0], %1, %2, %3, p;\n"                                             \
  " @e tcgen05.mma.cta_group::" GROUP ".kind::f16 [%0], a1, b1, %3, t;\n"                                             \
  " @e tcgen05.mma.cta_group::" GROUP ".kind::f16 [%0], a2, b2, %3, t;\n"                                             \
  " @e tcgen05.mma.cta_group::" GROUP ".kind::f16 [%0], a3, b3, %3, t;\n" COMMIT "}\n"
#define TP_COMMIT1 " @e tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%7];\n"
#define TP_COMMIT2 \
  " @e tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%7], %8;\n"
template <int kCta>
__device__ __forceinline__ void mma_elect(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t add, uint64_t ka,
                                          uint64_t kb, uint32_t bar) {
  if constexpr (kCta == 2)
    asm volatile(TP_MMA4("2", TP_COMMIT2)::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(add), "l"(ka), "l"(kb), "r"(bar),
                 "h"((uint16_t)3)
                 : "memory");
  else
    asm volatile(TP_MMA4("1", TP_COMMIT1)::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(add), "l"(ka), "l"(kb), "r"(bar)
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

// One accumulation: K blocks kb0 .. kb0 + kbn - 1 of a tile.
struct Item {
  int job, m0, n0, kb0, kbn;
  bool carry_in, carry_out;   // the reduction continues one that this cluster left in its own slot / is continued
  bool publish;               // leaves its sums for the cluster that finishes the tile
  int add0;                   // finishes a tile: adds the sums of clusters add0 .. this one - 1
};
struct Place { int tile, kb; };

// Where the K block numbered pos of the shared-out tiles lies.
__host__ __device__ __forceinline__ Place place_of(const ProdArgs& g, int pos) {
  for (int j = 0; j < g.n_jobs; ++j) {
    const int first = max(g.job[j].tile0, g.whole), end = j + 1 < g.n_jobs ? g.job[j + 1].tile0 : g.n_tiles;
    const int units = max(0, end - first) * g.job[j].kb;
    if (pos < units) return Place{first + pos / g.job[j].kb, pos % g.job[j].kb};
    pos -= units;
  }
  return Place{g.n_tiles, 0};
}

// A cluster's items in the order it takes them; every role walks them alike.
template <int kCta>
struct Walk {
  const ProdArgs& g;
  const int clu, n_clu;
  Place from, to;
  int phase = 0, next_tile = 0;
  int tile = 0, kb = 0, kb_end = 0, kind = 0, add0 = 0;   // the run of K blocks that items are cut from
  bool first = false;

  __host__ __device__ __forceinline__ Walk(const ProdArgs& g_, int c, int n) : g(g_), clu(c), n_clu(n) {
    from = to = Place{g.n_tiles, 0};
    if (g.whole < g.n_tiles) from = place_of(g, g.cut[c]), to = place_of(g, g.cut[c + 1]);
  }
  __host__ __device__ __forceinline__ int job_of(int t) const {
    int j = 0;
    for (int k = 1; k < g.n_jobs; ++k)
      if (t >= g.job[k].tile0) j = k;
    return j;
  }
  // kind 0: a whole tile, 1: published, 2: finishes a tile that others began
  __host__ __device__ __forceinline__ void run(int t, int a, int b, int k) { tile = t, kb = a, kb_end = b, kind = k, first = true; }
  __host__ __device__ __forceinline__ bool next_run() {
    while (phase < 4) {
      if (phase == 0) {
        phase = 1;
        next_tile = clu;
        if (from.tile == to.tile) {
          if (from.kb < to.kb) {
            run(to.tile, from.kb, to.kb, 1);
            return true;
          }
        } else if (to.kb > 0) {
          run(to.tile, 0, to.kb, 1);
          return true;
        }
      } else if (phase == 1) {
        if (next_tile < g.whole) {
          run(next_tile, 0, g.job[job_of(next_tile)].kb, 0);
          next_tile += n_clu;
          return true;
        }
        phase = 2;
        next_tile = from.kb ? from.tile + 1 : from.tile;
      } else if (phase == 2) {
        if (next_tile < to.tile) {
          run(next_tile, 0, g.job[job_of(next_tile)].kb, 0);
          ++next_tile;
          return true;
        }
        phase = 3;
      } else {
        phase = 4;
        if (from.tile < to.tile && from.kb > 0) {
          run(from.tile, from.kb, g.job[job_of(from.tile)].kb, 2);
          add0 = clu;   // back to the cluster that began the tile
          while (add0 > 0) {
            const Place p = place_of(g, g.cut[add0]);
            if (p.tile != tile || p.kb == 0) break;
            --add0;
          }
          return true;
        }
      }
    }
    return false;
  }
  __host__ __device__ __forceinline__ bool next(Item& it) {
    if (kb >= kb_end && !next_run()) return false;
    it.job = job_of(tile);
    const ProdJob& b = g.job[it.job];
    // eight row blocks at a time walk the columns, so that a round's tiles share operands in L2
    int local = tile - b.tile0;
    const int group = local / (8 * b.tn), rows = min(8, b.tm - 8 * group);
    local -= group * 8 * b.tn;
    it.m0 = (8 * group + local % rows) * 128 * kCta;
    it.n0 = local / rows;
    it.kb0 = kb;
    it.kbn = min(kb_end - kb, g.part_kb);
    it.carry_in = !first;
    kb += it.kbn;
    it.carry_out = kb < kb_end;
    it.publish = kind == 1;
    it.add0 = kind == 2 ? add0 : clu;
    first = false;
    return true;
  }
};

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
// fp32 values as one bf16 number each, or as three whose sum they are
// (buffers `part` elements apart), into rows with room for whole sectors.
template <bool kThree>
__device__ __forceinline__ void put_parts(float (&v)[32], __nv_bfloat16* out, int64_t part, bool live, int n) {
  uint32_t pk[16];
  if constexpr (!kThree) {
    pack32(v, pk);
    put_bf16(pk, out, live, n);
  } else {
#pragma unroll
    for (int e = 0; e < 16; ++e) pk[e] = first_parts(v[2 * e], v[2 * e + 1]);
#pragma unroll 1
    for (int q = 0; q < 3; ++q) {
      put_bf16(pk, out + q * part, live, n);
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        v[2 * e] -= __uint_as_float(pk[e] << 16);
        v[2 * e + 1] -= __uint_as_float(pk[e] & 0xFFFF0000u);
      }
      pack32(v, pk);   // (the last time for nothing)
    }
  }
}

// A lane's 32 columns in a slot: groups of four, the lanes' side by side.
__device__ __forceinline__ void put_slot(float* p, int lane, const float (&v)[32]) {
#pragma unroll
  for (int s = 0; s < 8; ++s)
    reinterpret_cast<float4*>(p)[32 * s + lane] = make_float4(v[4 * s], v[4 * s + 1], v[4 * s + 2], v[4 * s + 3]);
}
__device__ __forceinline__ void add_slot(const float* p, int lane, float (&v)[32]) {
#pragma unroll
  for (int s = 0; s < 8; ++s) {
    const float4 w = __ldcg(reinterpret_cast<const float4*>(p) + 32 * s + lane);
    v[4 * s] += w.x, v[4 * s + 1] += w.y, v[4 * s + 2] += w.z, v[4 * s + 3] += w.w;
  }
}

// 24-bit floats: the upper 16 bits of 32 columns as pairs, the next 8 as quads.
// act(g) and u act'(g) are kept so: as bf16 their rounding is a third one (beside
// those of dg, du and the outputs), 2.9e-3 of dx instead of 2.4e-3 (norm-wise;
// rounding the outputs alone 1.7e-3), for a byte more each.
__device__ __forceinline__ void put_24(const float (&v)[32], __nv_bfloat16* hi, uint8_t* lo, bool live, int n) {
  uint32_t u[16], b[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = round_24(v[4 * e + i]);
    u[2 * e] = __byte_perm(w[0], w[1], 0x7632), u[2 * e + 1] = __byte_perm(w[2], w[3], 0x7632);
    b[e] = __byte_perm(__byte_perm(w[0], w[1], 0x0051), __byte_perm(w[2], w[3], 0x0051), 0x5410);
  }
  put_bf16(u, hi, live, n);
  if (live) store32(lo, b);
}

// kEpiDgated of a bf16 block: what the epilogue reads besides the accumulator
// comes in, and what it writes goes out, by TMA through the warp's own shared
// memory, one chunk ahead.  (By loads and stores of the lanes' own rows, a
// 32-byte sector in 32 different lines each, the loads and stores alone took
// 6 us of a pair's 256-column tile: 16384 x 1024 -> 4096, 223 us; 133 us so,
// of which the bytes take 105.)
struct Kept {
  uint8_t* in;                // [2][32 rows][64 B], [2][32 rows][32 B]; first u act'(g), then act(g)
  uint8_t* out;               // [2][32 rows][64 B]: dg, du
  uint64_t* bar;                   // [2] filled
  uint32_t phase = 0, asked = 0;   // a bit a slot
  __device__ __forceinline__ void ask(const ProdArgs& g, int h, int c0, int r0) {
    const uint32_t b = smem_u32(bar + h);
    expect_elect(b, kKeptHi + kKeptLo);
    tma_elect<1>(smem_u32(in) + h * kKeptHi, &g.map[kMapHi], b, c0, r0, 1 - h);
    tma_elect<1>(smem_u32(in) + 2 * kKeptHi + h * kKeptLo, &g.map[kMapLo], b, c0, r0, 1 - h);
    asked |= 1u << h;
  }
  __device__ __forceinline__ bool wait(int h, volatile int* abort_flag, int* err) {
    const bool ok = __all_sync(0xffffffffu, mbar_wait(bar + h, phase >> h & 1, abort_flag, err, kWaitNs, 48));
    if (ok) phase ^= 1u << h, asked &= ~(1u << h);
    return ok;
  }
  // f = what has come in times acc (what the lowest byte holds is below their rounding)
  __device__ __forceinline__ void times(int h, int lane, float (&f)[32], const float (&acc)[32]) const {
    const uint8_t* hi = in + h * kKeptHi + lane * 64;
    const uint8_t* lo = in + 2 * kKeptHi + h * kKeptLo + lane * 32;
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      const uint4 bq = *reinterpret_cast<const uint4*>(lo + ((s ^ ((lane >> 2) & 1)) << 4));
      const uint32_t b[4] = {bq.x, bq.y, bq.z, bq.w};
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        const uint4 uq = *reinterpret_cast<const uint4*>(hi + (((2 * s + t) ^ ((lane >> 1) & 3)) << 4));
        const uint32_t u[4] = {uq.x, uq.y, uq.z, uq.w};
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const uint32_t at = e & 3, hw = 4 + 2 * (e & 1);   // byte of b, first byte of the pair's half
          const int i = 16 * s + 8 * t + e;
          f[i] = __uint_as_float(__byte_perm(b[2 * t + (e >> 2)], u[e >> 1], at | at << 4 | hw << 8 | (hw + 1) << 12)) * acc[i];
        }
      }
    }
  }
  // f on its way out.  After this the slot that f was made from may be filled again: the copy that does so must not
  // overtake loads that have been issued but not served, and here every lane has stored what its loads came back
  // with, before the warp's barrier.  (Neither that barrier alone nor an mbarrier's arrival after the loads waits
  // for them: 4043 x 477 -> 2354, after a forward pass, had 16-byte pieces of the next chunk in one pass of
  // seven.)
  __device__ __forceinline__ void put(const ProdArgs& g, int h, int lane, const float (&f)[32], int c0, int r0) {
    uint32_t pk[16];
    pack32(f, pk);
    if (lane == 0) asm volatile("cp.async.bulk.wait_group.read 1;" ::: "memory");   // the buffer's last store has read it
    __syncwarp();
    uint8_t* to = out + h * kKeptHi + lane * 64;
#pragma unroll
    for (int s = 0; s < 4; ++s)
      *reinterpret_cast<uint4*>(to + ((s ^ ((lane >> 1) & 3)) << 4)) =
          make_uint4(pk[4 * s], pk[4 * s + 1], pk[4 * s + 2], pk[4 * s + 3]);
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    __syncwarp();
    if (lane == 0)
      asm volatile(
          "cp.async.bulk.tensor.3d.global.shared::cta.bulk_group [%0, {%2, %3, %4}], [%1];\n cp.async.bulk.commit_group;" ::"l"(
              &g.map[kMapOut]),
          "r"(smem_u32(out + h * kKeptHi)), "r"(c0), "r"(r0), "r"(h)
          : "memory");
  }
};

// The epilogue of one 32 x 32 chunk; acc: its accumulator (kEpiGated: the
// gate product), acc2: the up product.
template <int kEpi, int kAct, bool kF32>
__device__ __forceinline__ void epilogue(const ProdJob& j, uint8_t* buf, int lane, float (&acc)[32], float (&acc2)[32],
                                         int r0, int c0) {
  const int row = r0 + lane, n = j.N - c0;
  const bool live = row < j.M;
  const int64_t at = (int64_t)row * j.ldo + c0;
  if constexpr (kEpi == kEpiGated) {
    float da[32];
#pragma unroll
    for (int e = 0; e < 32; ++e) {
      float d;
      const float a = act_value<kAct, kF32>(acc[e], d);
      da[e] = acc2[e] * d;
      acc2[e] *= a;
      acc[e] = a;
    }
    if (j.a != nullptr) {
      if constexpr (kF32) {
        put_f32(acc, (float*)j.a + at, live, n);
        put_f32(da, (float*)j.p + at, live, n);
      } else {
        put_24(acc, (__nv_bfloat16*)j.a + at, j.a_lo + at, live, n);
        put_24(da, (__nv_bfloat16*)j.p + at, j.p_lo + at, live, n);
      }
    }
    put_parts<kF32>(acc2, (__nv_bfloat16*)j.out + at, j.part, live, n);
  } else if constexpr (kEpi == kEpiDgated) {   // of a 32-bit block
    float f[32];
    __nv_bfloat16* out = (__nv_bfloat16*)j.out + at;
    const int64_t from = (int64_t)min(row, j.M - 1) * j.ldo + c0;
#pragma unroll 1
    for (int h = 0; h < 2; ++h) {
      const float* src = (const float*)(h ? j.a : j.p) + from;
#pragma unroll
      for (int s = 0; s < 4; ++s) {
        uint32_t w[8] = {};
        if (n > 8 * s) load32(src + 8 * s, w);
#pragma unroll
        for (int e = 0; e < 8; ++e) f[8 * s + e] = __uint_as_float(w[e]) * acc[8 * s + e];
      }
      put_parts<true>(f, out + h * j.half, j.part, live, n);
    }
  } else {
    if constexpr (kEpi == kEpiQuant) {
      const float sx = live ? j.sx[row] : 0.f;
      const int c = c0 + lane;
      const float sw = c < j.N ? j.sw[c] : 0.f, b = c < j.N && j.bias ? j.bias[c] : 0.f;
#pragma unroll
      for (int e = 0; e < 32; ++e)
        acc[e] = acc[e] * sx * __shfl_sync(0xffffffffu, sw, e) + __shfl_sync(0xffffffffu, b, e);
    }
    // whole sectors where the rows lie on them, else through the warp's buffer
    if constexpr (kF32) {
      if (n >= 32 && ((uintptr_t)j.out & 31) == 0 && (j.ldo & 7) == 0) put_f32(acc, (float*)j.out + at, live, n);
      else emit_f32(buf, lane, acc, (float*)j.out, j.ldo, r0, j.M, c0, j.N, vec_ok(j.out, j.ldo, 4));
    } else {
      uint32_t pk[16];
      pack32(acc, pk);
      if (n >= 32 && ((uintptr_t)j.out & 31) == 0 && (j.ldo & 15) == 0) put_bf16(pk, (__nv_bfloat16*)j.out + at, live, n);
      else emit_bf16(buf, lane, pk, (__nv_bfloat16*)j.out, j.ldo, r0, j.M, c0, j.N, vec_ok(j.out, j.ldo, 2));
    }
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
  constexpr bool kStaged = kEpi == kEpiDgated && !kF32;
  uint8_t* kept_in = bufs + kEpiWarps * kBufBytes;
  Tail* tl = (Tail*)(kept_in + (kStaged ? kEpiWarps * kKeptBytes : 0));
  const int warp = (int)uniform(threadIdx.x >> 5), lane = threadIdx.x & 31;
  const int rank = kCta == 2 ? (int)uniform(cluster_rank()) : 0;
  const bool leader = rank == 0;
  const int clu = blockIdx.x / kCta, n_clu = gridDim.x / kCta;

  if (threadIdx.x == 0) {
    for (int s = 0; s < stages; ++s) {
      mbar_init(&tl->full[s], 2);   // one per producer
      mbar_init(&tl->empty[s], 1);
    }
    for (int b = 0; b < 2; ++b) {
      mbar_init(&tl->tfull[b], 1);
      mbar_init(&tl->tempty[b], kEpiWarps * kCta);
    }
    mbar_init(&tl->done, 1);
    if constexpr (kStaged)
      for (int w = 0; w < 2 * kEpiWarps; ++w) mbar_init(&tl->kept[0][w], 1);
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
  if (warp == 0 && lane < kProdMaps && lane < g.n_maps)
    asm volatile("prefetch.tensormap [%0];" ::"l"(&g.map[lane]) : "memory");
  pdl_wait();                      // the set-up above overlaps the previous kernel
  fence_proxy_async_global();      // what it wrote by plain stores is read by TMA
  const uint32_t tmem = uniform(tl->tmem_base);
  volatile int* abort_flag = &tl->abort;
  int* err = &g_prod_err;

  if (warp == 0 || warp == kWarpB) {
    // -------------------------------------------------- producers of A and B
    const bool is_a = warp == 0;
    uint32_t stage = 0, phase = 0, issued = 0;
    bool ok = true;
    const uint32_t s0 = smem_u32(smem), full0 = smem_u32(&tl->full[0]);
    const uint32_t lead0 = kCta == 2 ? mapa(full0, 0) : full0;   // the barriers that copies complete on
    Walk<kCta> walk(g, clu, n_clu);
    Item u;
    while (ok && walk.next(u)) {
      const ProdJob& j = g.job[u.job];
      const CUtensorMap* map = &g.map[is_a ? j.map_a : j.map_b];
      const bool mn = (is_a ? j.a_mn : j.b_mn) != 0;
      // kEpiGated: n_tile / 2 columns of the gate, then the same of the up half (in a pair one each)
      constexpr bool kHalves = kEpi == kEpiGated && kCta == 1;
      const int half_n = g.n_tile / 2, rows = is_a ? 128 : nh;
      const int x0 = is_a ? u.m0 + rank * 128 : kEpi == kEpiGated ? u.n0 * half_n : u.n0 * g.n_tile + rank * nh;
      const uint32_t off = is_a ? 0 : kABytes;
      for (int q = 0; ok && q < j.n_pairs; ++q) {
        const int z = is_a ? j.sa[q] : j.sb[q] + (kEpi == kEpiGated && kCta == 2 ? rank * j.up : 0);
        for (int kb = u.kb0; kb < u.kb0 + u.kbn; ++kb) {
          if (!wait_all(&tl->empty[stage], phase ^ 1u, abort_flag, err, kWaitNs, 41)) {
            ok = false;
            break;
          }
          const uint32_t dst = s0 + stage * stage_bytes + off, bar = lead0 + 8 * stage;
          const int k = 64 * kb;
          if (leader) expect_elect(full0 + 8 * stage, (uint32_t)(kCta * 128) * rows);
          // K-major: one box of all rows (gate and up rows apart); MN-major: boxes of 64
          if (mn) {
            tma_elect<kCta>(dst, map, bar, x0, k, z);
            if (rows > 64) tma_elect<kCta>(dst + kBox, map, bar, x0 + 64, k, z);
            if (rows > 128) {
              tma_elect<kCta>(dst + 2 * kBox, map, bar, x0 + 128, k, z);
              tma_elect<kCta>(dst + 3 * kBox, map, bar, x0 + 192, k, z);
            }
          } else {
            tma_elect<kCta>(dst, map, bar, k, x0, z);
            if (kHalves && !is_a) tma_elect<kCta>(dst + half_n * 128, map, bar, k, x0, z + j.up);
          }
          issued |= 1u << stage;
          if (++stage == (uint32_t)stages) {
            stage = 0;
            phase ^= 1u;
          }
        }
      }
    }
    // every copy has landed before the CTA leaves: a stage's last one is of this
    // turn of the ring below `stage`, of the one before from there on
    if (leader && is_a)
      for (int s = 0; s < stages; ++s)
        if (issued & (1u << s)) {
          int dummy = 0;
          mbar_wait(&tl->full[s], s < (int)stage ? phase : phase ^ 1u, &dummy, err, kWaitNs, 42);
        }
  } else if (warp == 1) {
    if (leader) {
      // --------------------------------------------------------------- MMA
      const uint32_t s0 = smem_u32(smem), empty0 = smem_u32(&tl->empty[0]);
      const uint64_t dA_k = smem_desc(s0, 16, 1024), dA_mn = smem_desc(s0, kBox, 1024);
      const uint64_t dB_k = smem_desc(s0 + kABytes, 16, 1024), dB_mn = smem_desc(s0 + kABytes, kBox, 1024);
      const uint32_t step = stage_bytes >> 4;
      uint32_t stage = 0, phase = 0, acc = 0, acc_phase = 0;
      bool ok = true;
      Walk<kCta> walk(g, clu, n_clu);
      Item u;
      while (ok && walk.next(u)) {
        const ProdJob& j = g.job[u.job];
        if (!wait_all(&tl->tempty[acc], acc_phase ^ 1u, abort_flag, err, 2 * kWaitNs, 43)) break;
        tc_fence_after();
        const uint32_t d0 = tmem + acc * kAccCols;
        uint32_t idesc = instr_desc(128 * kCta, g.n_tile, j.a_mn, j.b_mn);
        if (g.fp16) idesc &= ~((1u << 7) | (1u << 10));
        const uint64_t ta = j.a_mn ? dA_mn : dA_k, tb = j.b_mn ? dB_mn : dB_k;
        const uint64_t ka = j.a_mn ? 2048 >> 4 : 32 >> 4, kb_ = j.b_mn ? 2048 >> 4 : 32 >> 4;
        const int split_at = g.chains == 2 ? (u.kbn + 1) >> 1 : u.kbn;   // first K block of the second chain
        for (int q = 0; ok && q < j.n_pairs; ++q) {
          for (int kb = 0; kb < u.kbn; ++kb) {
            if (!wait_all(&tl->full[stage], phase, abort_flag, err, 2 * kWaitNs, 44)) {
              ok = false;
              break;
            }
            const uint32_t d = d0 + (kb >= split_at ? kAccCols / 2 : 0);
            const uint32_t add = q > 0 || (kb != 0 && kb != split_at) ? 1u : 0u;
            mma_elect<kCta>(d, ta + stage * step, tb + stage * step, idesc, add, ka, kb_, empty0 + 8 * stage);
            if (++stage == (uint32_t)stages) {
              stage = 0;
              phase ^= 1u;
            }
          }
        }
        if (!ok) break;
        commit_elect<kCta>(smem_u32(&tl->tfull[acc]));
        acc ^= 1u;
        if (acc == 0) acc_phase ^= 1u;
      }
      commit_elect<kCta>(smem_u32(&tl->done));   // all MMAs are over before TMEM is freed
      int dummy = 0;
      mbar_wait(&tl->done, 0, &dummy, err, kWaitNs, 45);
    }
  } else {
    // ------------------------------------------------------------ epilogue
    const int q = warp & 3, half = (warp - 2) >> 2;
    uint8_t* buf = bufs + (warp - 2) * kBufBytes;
    uint32_t acc = 0, acc_phase = 0;
    const int cols = kEpi == kEpiGated ? g.n_tile / 2 : g.n_tile;
    // this warp's 32 lanes x n_tile columns in the slots, a chunk of 32 columns after another
    const int64_t slot = (int64_t)128 * g.n_tile, mine = (int64_t)(clu * kCta + rank) * slot + (int64_t)32 * q * g.n_tile;
    float* own = g.slots + (int64_t)n_clu * kCta * slot + mine;
    if (blockIdx.x == 0)
      for (int i = threadIdx.x - 64; i < g.n_zero; i += 32 * kEpiWarps) g.zero[i] = 0;
    Walk<kCta> walk(g, clu, n_clu);
    Item u;
    Kept kept{kept_in + (warp - 2) * kKeptBytes, buf, tl->kept[warp - 2]};
    bool ok = true;
    while (ok && walk.next(u)) {
      const ProdJob& j = g.job[u.job];
      const int r0 = u.m0 + rank * 128 + 32 * q;
      const bool finish = !u.publish && !u.carry_out;
      if constexpr (kStaged)
        if (finish && r0 < j.M && u.n0 * cols + 32 * half < j.N) {
          kept.ask(g, 0, u.n0 * cols + 32 * half, r0);
          kept.ask(g, 1, u.n0 * cols + 32 * half, r0);
        }
      if (!__all_sync(0xffffffffu, mbar_wait(&tl->tfull[acc], acc_phase, abort_flag, err, 2 * kWaitNs, 46))) break;
      tc_fence_after();
      bool there = true;
      if (finish)
        for (int k = u.add0; k < clu; ++k)   // (a cluster without K blocks leaves nothing)
          if (g.cut[k] < g.cut[k + 1])
            there = there && dep_wait(g.flags + (k * kCta + rank) * kEpiWarps + warp - 2, 1, 1, abort_flag, err,
                                      2 * kWaitNs, 47, lane);
      if (!there) break;
      const uint32_t ta = tmem + ((uint32_t)(32 * q) << 16) + acc * kAccCols;
      const bool second = g.chains == 2 && u.kbn > 1;
#pragma unroll 1
      for (int c = 32 * half; c < cols; c += 64) {
        const int c0 = u.n0 * cols + c;
        if (r0 >= j.M || c0 >= j.N) break;   // warp-uniform
        uint32_t v[32], v2[32];
        float a[32], a2[32];
        tmem_ask32(ta + c, v);
        if constexpr (kEpi == kEpiGated) tmem_ask32(ta + cols + c, v2);
        tmem_wait();
        tmem_got(v);
        if constexpr (kEpi == kEpiGated) tmem_got(v2);
#pragma unroll
        for (int e = 0; e < 32; ++e) {
          a[e] = __uint_as_float(v[e]);
          if constexpr (kEpi == kEpiGated) a2[e] = __uint_as_float(v2[e]);
        }
        if (second) {
          tmem_ask32(ta + kAccCols / 2 + c, v);
          if constexpr (kEpi == kEpiGated) tmem_ask32(ta + kAccCols / 2 + cols + c, v2);
          tmem_wait();
          tmem_got(v);
          if constexpr (kEpi == kEpiGated) tmem_got(v2);
#pragma unroll
          for (int e = 0; e < 32; ++e) {
            a[e] += __uint_as_float(v[e]);
            if constexpr (kEpi == kEpiGated) a2[e] += __uint_as_float(v2[e]);
          }
        }
        // sums of the same reduction from before
        if (u.carry_in) {
          add_slot(own + 32 * c, lane, a);
          if constexpr (kEpi == kEpiGated) add_slot(own + 32 * (cols + c), lane, a2);
        }
        if (!finish) {
          float* to = u.carry_out ? own : g.slots + mine;
          put_slot(to + 32 * c, lane, a);
          if constexpr (kEpi == kEpiGated) put_slot(to + 32 * (cols + c), lane, a2);
          continue;
        }
        for (int k = u.add0; k < clu; ++k) {
          if (g.cut[k] == g.cut[k + 1]) continue;
          const float* of = g.slots + mine - (int64_t)(clu - k) * kCta * slot;
          add_slot(of + 32 * c, lane, a);
          if constexpr (kEpi == kEpiGated) add_slot(of + 32 * (cols + c), lane, a2);
        }
        if constexpr (kStaged) {   // dg = dh u act'(g), du = dh act(g)
          const bool more = c + 64 < cols && c0 + 64 < j.N;
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            ok = ok && kept.wait(h, abort_flag, err);
            if (!ok) break;
            kept.times(h, lane, a2, a);
            kept.put(g, h, lane, a2, c0, r0);
            if (more) kept.ask(g, h, c0 + 64, r0);   // (after put)
          }
          if (!ok) break;
        } else {
          epilogue<kEpi, kAct, kF32>(j, buf, lane, a, a2, r0, c0);
        }
      }
      if (!ok) break;
      tc_fence_before();
      __syncwarp();
      if (lane == 0) {   // the loads above have completed
        if constexpr (kCta == 2) mbar_arrive_cluster_relaxed(mapa(smem_u32(&tl->tempty[acc]), 0));
        else mbar_arrive_relaxed(&tl->tempty[acc]);
      }
      if (u.publish && !u.carry_out && lane == 0)   // after the warp's stores (the barrier above)
        red_release_add(g.flags + (clu * kCta + rank) * kEpiWarps + warp - 2, 1);
      acc ^= 1u;
      if (acc == 0) acc_phase ^= 1u;
    }
    if constexpr (kStaged) {   // copies in flight: of a role that gave up, and the stores
      int dummy = 0;
      for (int h = 0; h < 2; ++h)
        if (kept.asked >> h & 1) mbar_wait(kept.bar + h, kept.phase >> h & 1, &dummy, err, kWaitNs, 49);
      if (lane == 0) asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");
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
      mbar_wait(&tl->done, 0, &dummy, err, 4 * kWaitNs, 45);
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

// ------------------------------------------------------------------ staging
// One pass over the source, 16-byte stores; a block takes 256 / 2^shift rows at
// a time, 2^shift threads a row (a division for every group of eight elements
// cost more than moving it).
__device__ __forceinline__ uint4 pack_f16(const int (&v)[8]) {
  uint32_t h[4];
#pragma unroll
  for (int e = 0; e < 4; ++e)
    h[e] = __half_as_ushort(__int2half_rn(v[2 * e])) | (uint32_t)__half_as_ushort(__int2half_rn(v[2 * e + 1])) << 16;
  return make_uint4(h[0], h[1], h[2], h[3]);
}
__global__ void __launch_bounds__(256) k_stage(const __grid_constant__ StageLaunch g) {
  pdl_trigger();
  pdl_wait();
  if (blockIdx.x == 0 && blockIdx.y == 0)
    for (int i = threadIdx.x; i < g.n_zero; i += 256) g.zero[i] = 0;
  const StageJob& j = g.job[blockIdx.y];
  const int width = 1 << j.shift, tx = threadIdx.x & (width - 1), groups = (int)(j.ldp >> 3);
  const int eb = j.type == kStageF32 ? 4 : j.type == kStageS8 ? 1 : 2;
  const bool vec = ((uintptr_t)j.src & (eb == 1 ? 7 : 15)) == 0 && ((j.ld * eb) & (eb == 1 ? 7 : 15)) == 0;
  if (j.type == kStageS8 && j.cols % 16 == 0 && j.ld % 16 == 0 && ((uintptr_t)j.src & 15) == 0) {
    // 16 elements a thread, of four rows at a time (8192 x 2048 -> 4096 in all: 90 us with one load of 8 in flight, 85 so)
    const int sh = max(j.shift - 1, 0), t16 = threadIdx.x & ((1 << sh) - 1);
    const int64_t step = (int64_t)gridDim.x * (256 >> sh);
    for (int64_t r = (int64_t)blockIdx.x * (256 >> sh) + (threadIdx.x >> sh); r < j.rows; r += 4 * step)
      for (int c = 16 * t16; c < j.cols; c += 16 << sh) {
        uint4 w[4];
#pragma unroll
        for (int u = 0; u < 4; ++u)
          if (r + u * step < j.rows) w[u] = *reinterpret_cast<const uint4*>((const int8_t*)j.src + (r + u * step) * j.ld + c);
#pragma unroll
        for (int u = 0; u < 4; ++u) {
          if (r + u * step >= j.rows) break;
          uint4* dst = reinterpret_cast<uint4*>((uint16_t*)j.dst + (r + u * step) * j.ldp + c);
          uint4 h[2];
          s8_to_f16(w[u].x, h[0].x, h[0].y), s8_to_f16(w[u].y, h[0].z, h[0].w);
          s8_to_f16(w[u].z, h[1].x, h[1].y), s8_to_f16(w[u].w, h[1].z, h[1].w);
          dst[0] = h[0], dst[1] = h[1];
        }
      }
    return;
  }
  for (int64_t r = (int64_t)blockIdx.x * (256 >> j.shift) + (threadIdx.x >> j.shift); r < j.rows;
       r += (int64_t)gridDim.x * (256 >> j.shift)) {
    const int64_t seg = r >= j.rows_seg ? 1 : 0, rs = r - seg * j.rows_seg;   // one or two segments
    if (j.type == kStageF32) {
      const float* src = (const float*)j.src + r * j.ld;
      __nv_bfloat16* dst = (__nv_bfloat16*)j.dst + (seg * 3 * j.rows_seg + rs) * j.ldp;
#pragma unroll 2
      for (int q8 = tx; q8 < groups; q8 += width) {
        const int c = 8 * q8;
        float v[8];
        if (vec && c + 8 <= j.cols) {
          const float4 a = *reinterpret_cast<const float4*>(src + c), b = *reinterpret_cast<const float4*>(src + c + 4);
          v[0] = a.x, v[1] = a.y, v[2] = a.z, v[3] = a.w, v[4] = b.x, v[5] = b.y, v[6] = b.z, v[7] = b.w;
        } else {
#pragma unroll
          for (int e = 0; e < 8; ++e) v[e] = c + e < j.cols ? src[c + e] : 0.f;
        }
#pragma unroll
        for (int q = 0; q < 3; ++q) {
          uint32_t pk[4];
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            pk[e] = q == 0 ? first_parts(v[2 * e], v[2 * e + 1]) : pack_bf16x2(v[2 * e], v[2 * e + 1]);
            v[2 * e] -= __uint_as_float(pk[e] << 16);
            v[2 * e + 1] -= __uint_as_float(pk[e] & 0xFFFF0000u);
          }
          *reinterpret_cast<uint4*>(dst + q * j.rows_seg * j.ldp + c) = make_uint4(pk[0], pk[1], pk[2], pk[3]);
        }
      }
    } else {
      uint16_t* dst = (uint16_t*)j.dst + (seg * j.rows_seg + rs) * j.ldp;
      const int8_t* s8 = (const int8_t*)j.src + r * j.ld;
      const uint16_t* s16 = (const uint16_t*)j.src + r * j.ld;
#pragma unroll 4
      for (int q8 = tx; q8 < groups; q8 += width) {
        const int c = 8 * q8;
        uint4 out;
        if (j.type == kStageS8) {
          int v[8];
          if (vec && c + 8 <= j.cols) {
            const uint2 w = *reinterpret_cast<const uint2*>(s8 + c);
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = (int8_t)((e < 4 ? w.x : w.y) >> (8 * (e & 3)));
          } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = c + e < j.cols ? s8[c + e] : 0;
          }
          out = pack_f16(v);
        } else {
          uint32_t h[8];
#pragma unroll
          for (int e = 0; e < 8; ++e) h[e] = c + e < j.cols ? s16[c + e] : 0u;
          out = make_uint4(h[0] | h[1] << 16, h[2] | h[3] << 16, h[4] | h[5] << 16, h[6] | h[7] << 16);
        }
        *reinterpret_cast<uint4*>(dst + c) = out;
      }
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

// [segs][rows][cols] of eb bytes, ld bytes from row to row
bool encode(CUtensorMap* m, CUtensorMapDataType type, const void* base, int64_t cols, int64_t rows, int64_t ld, int64_t seg,
            int n_seg, int box_cols, int box_rows, CUtensorMapSwizzle swizzle) {
  auto fn = get_encode();
  if (!fn) return false;
  cuuint64_t dims[3] = {(cuuint64_t)cols, (cuuint64_t)rows, (cuuint64_t)n_seg};
  cuuint64_t strides[2] = {(cuuint64_t)ld, (cuuint64_t)(n_seg > 1 ? seg : ld * 8)};
  cuuint32_t box[3] = {(cuuint32_t)box_cols, (cuuint32_t)box_rows, 1};
  cuuint32_t es[3] = {1, 1, 1};
  return fn(m, type, 3, const_cast<void*>(base), dims, strides, box, es, CU_TENSOR_MAP_INTERLEAVE_NONE, swizzle,
            CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}
bool encode(CUtensorMap* m, const ProdOperand& o, bool fp16, int box_rows) {
  return encode(m, fp16 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT16 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, o.base, o.cols, o.rows,
                o.ld * 2, o.seg * 2, o.n_seg, 64, box_rows, CU_TENSOR_MAP_SWIZZLE_128B);
}

// Shared memory beside the ring's stages, and how many of them fit.
int smem_rest(bool kept) { return 1024 + kEpiWarps * (kBufBytes + (kept ? kKeptBytes : 0)) + (int)sizeof(Tail); }
int stage_count(int cta, int n_tile, bool kept) {
  const int bytes = kABytes + n_tile / cta * 128;
  return std::min<int>(kMaxStages, (kSmemMax - smem_rest(kept)) / bytes);
}

// A tile's shape and its times in ns, measured (bf16, operands in L2): a K
// block, what a launch of one tile per cluster takes besides (the epilogue
// among it), and the epilogue alone, which the next tile's K blocks hide.
struct Shape {
  int cta, n;
  double kb, fixed, epi;
};
constexpr Shape kShapes[] = {{2, 256, 287, 7000, 2800}, {2, 128, 195, 5600, 1400}, {1, 256, 320, 5900, 2800},
                             {1, 128, 213, 4400, 1400}, {1, 64, 180, 3900, 700}};

template <int kCta, int kEpi, int kAct, bool kF32>
cudaError_t launch(const ProdArgs& a, int clusters, cudaStream_t st) {
  const int stage_bytes = kABytes + a.n_tile / kCta * 128;
  const int smem = a.stages * stage_bytes + smem_rest(kEpi == kEpiDgated && !kF32);
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(kCta * clusters);
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
    if (f32) return cta_of(e, a, std::true_type());
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
Failures g_failures[kMaxDevices];
std::mutex g_failures_mu;

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
    cfg.dynamicSmemBytes = stage_count(2, 256, false) * (kABytes + 128 * 128) + smem_rest(false);
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

namespace {

// Time of a whole tile among others, ns: its K blocks or, where that is longer,
// its epilogue.
double tile_ns(const ProdJob& j, const Shape& s) { return std::max(j.n_pairs * j.kb * s.kb, s.epi); }

// Shares out the tiles from p.whole on: runs of K blocks that end all clusters
// at about the same time.
void share_out(ProdLaunch& p, const Shape& s) {
  const int C = p.clusters;
  double load[kSms] = {}, total = 0;
  for (int k = 0; k < p.n_jobs; ++k) {
    const ProdJob& j = p.job[k];
    const int first = j.tile0, end = first + j.tm * j.tn;
    const double t = tile_ns(j, s);
    for (int c = 0; c < C; ++c) {   // whole tiles first .. min(end, whole) - 1 with number c modulo C
      const int last = std::min(end, p.whole);
      if (last > first) load[c] += t * ((last - 1 - c + C) / C - (first - 1 - c + C) / C);
    }
    total += t * std::max(0, end - std::max(first, p.whole));
  }
  // the level to which `total` fills up the clusters
  double level = total;
  for (int c = 0; c < C; ++c) level += load[c];
  level /= C;
  for (int round = 0; round < 3; ++round) {
    double room = total;
    int n = 0;
    for (int c = 0; c < C; ++c)
      if (load[c] < level) room += load[c], ++n;
    level = room / n;
  }
  // cut the tiles' K blocks at the clusters' shares; a cut less than two K
  // blocks from a tile's edge moves to the edge
  int job = 0, tile = p.whole, pos = 0;
  double want = 0, done = 0;   // time up to tile's first K block
  auto step = [&] {
    while (job + 1 < p.n_jobs && tile >= p.job[job + 1].tile0) ++job;
  };
  step();
  p.cut[0] = 0;
  for (int c = 0; c < C; ++c) {
    want += std::max(0.0, level - load[c]);
    while (tile < p.n_tiles) {
      const ProdJob& j = p.job[job];
      const double t = tile_ns(j, s);
      if (c + 1 < C && done + t > want) break;
      done += t;
      pos += j.kb;
      ++tile;
      step();
    }
    int in = 0;
    if (tile < p.n_tiles) {
      const ProdJob& j = p.job[job];
      in = (int)((want - done) / tile_ns(j, s) * j.kb);
      if (in < 2) in = 0;
      else if (j.kb - in < 2) in = j.kb;
    }
    p.cut[c + 1] = std::max(p.cut[c], pos + in);
  }
}

}  // namespace

void prod_plan(ProdLaunch& l) {
  // whole tiles: the longest first; dealt out round robin, the last round's short ones then go to the clusters
  // with least.  Shared out: the longest last, among those that are cut.
  auto order = [&](bool longest_first) {
    std::stable_sort(l.job, l.job + l.n_jobs, [=](const ProdJob& a, const ProdJob& b) {
      const int64_t x = (int64_t)a.n_pairs * ceil_div(a.K, 64), y = (int64_t)b.n_pairs * ceil_div(b.K, 64);
      return longest_first ? x > y : x < y;
    });
  };
  order(true);
  const bool parts = l.f32 && !l.fp16;         // 32-bit operands: two chains in a 128-column tile
  double best = 1e300;
  const Shape* pick = nullptr;
  int pick_whole = 0, pick_clusters = 0;
  auto lay = [&](ProdLaunch& p, const Shape& s) {
    p.cta = s.cta, p.n_tile = s.n, p.chains = parts ? 2 : 1, p.n_tiles = 0;
    for (int k = 0; k < p.n_jobs; ++k) {
      ProdJob& j = p.job[k];
      j.kb = (int)ceil_div(j.K, 64);
      j.tm = (int)ceil_div(j.M, 128 * s.cta);
      j.tn = (int)ceil_div(j.N, p.epi == kEpiGated ? s.n / 2 : s.n);
      j.tile0 = p.n_tiles;
      p.n_tiles += j.tm * j.tn;
    }
  };
  for (const Shape& s : kShapes) {
    if (parts && s.n > 128) continue;
    lay(l, s);
    const int C = kSms / s.cta;
    double work = 0, longest = 0, blocks = 0;
    for (int k = 0; k < l.n_jobs; ++k) {
      const ProdJob& j = l.job[k];
      const double tiles = (double)j.tm * j.tn, t = tile_ns(j, s) + 100.0;
      work += t * tiles;
      blocks += tiles * j.n_pairs * j.kb;
      longest = std::max(longest, t);
    }
    // every tile whole
    const double rounds = (double)ceil_div(l.n_tiles, C);
    const double even = s.fixed + std::max(longest, rounds * work / l.n_tiles) + (l.n_jobs > 1 ? 0.5 * longest : 0.0);
    if (even < best) best = even, pick = &s, pick_whole = l.n_tiles, pick_clusters = C;
    // the last one to two rounds shared out: runs of at least four K blocks, at most sixteen clusters a tile.
    // (Of many rounds the last ones' tiles, cut, no longer share operands in L2 with their neighbours: 16384 rows,
    // 1024 -> 4096, backward, 680 us against 595 us whole.  Where one tile alone takes longer than a cluster's
    // share, cutting it gains more than that: 80 rows, 2048 -> 4096, backward, 47 us against 62 us.  32-bit
    // products gain less from it than their two chains' additions cost: 120 rows, 1024 -> 2048, 68 us against 61 us.)
    const int whole = std::max(0, l.n_tiles / C - 1) * C;
    const int clusters = (int)std::min<double>(std::min<double>(C, std::max(1.0, blocks / 4)), 16.0 * work / longest);
    const double share = work / clusters, adds = std::max(1.0, longest / share);
    const double shared = s.fixed + share + 6000.0 + (1.0 + adds) * s.epi;
    if (clusters > 1 && (clusters == C || whole == 0) && shared < (l.n_tiles <= 3 * C || (longest > share && !parts) ? 0.93 : 0.8) * best)
      best = shared, pick = &s, pick_whole = whole, pick_clusters = clusters;
  }
  lay(l, *pick);
  if (pick_whole < l.n_tiles) {
    order(false);
    lay(l, *pick);
  }
  l.whole = pick_whole;
  l.clusters = std::min(pick_clusters, l.whole == l.n_tiles ? l.n_tiles : pick_clusters);
  const int64_t slot = (int64_t)l.clusters * l.cta * 128 * l.n_tile * 4;
  l.slot_bytes = l.flag_bytes = 0;
  if (l.whole < l.n_tiles) {
    share_out(l, *pick);
    l.slot_bytes = slot;
    l.flag_bytes = (int64_t)l.clusters * l.cta * kEpiWarps * 4;
  }
  if (parts)
    for (int k = 0; k < l.n_jobs; ++k)
      if (l.job[k].kb > 2 * kChainKb) l.slot_bytes = 2 * slot;
}

namespace {
// The flags of the first cluster that leaves sums for another one, once: set so low that its announcement does not
// raise them to what the other waits for.
cudaError_t withhold_one(const ProdArgs& a, int cta, int clusters, cudaStream_t st) {
  for (int c = 0; c < clusters; ++c) {
    Walk<1> walk(a, c, clusters);
    Item it;
    while (walk.next(it))
      if (it.publish)
        return g_withhold.exchange(false) ? cudaMemsetAsync(a.flags + c * cta * kEpiWarps, 0x80, cta * kEpiWarps * 4, st)
                                          : cudaSuccess;
  }
  return cudaSuccess;
}

// Runs a planned launch; slots: at least slot_bytes, flags: flag_bytes of zeros (256-byte aligned); zero: n_zero
// words that it clears.
cudaError_t prod_run(ProdLaunch& l, void* slots, int* flags, int* zero, int n_zero, cudaStream_t st, const char** what) {
  DeviceState dev;
  *what = "kernel attributes";
  cudaError_t e = device_state(&dev);
  if (e != cudaSuccess) return e;
  const int fit = l.cta == 2 ? dev.pairs : dev.sms;
  if (fit < l.clusters) {   // not a whole GB300: only whole tiles can be taken by fewer clusters
    *what = "the product is planned for 152 SMs";
    if (l.whole < l.n_tiles) return cudaErrorInvalidConfiguration;
  }
  const int clusters = std::min(fit, l.clusters);
  ProdArgs a;
  a.n_jobs = l.n_jobs, a.n_tiles = l.n_tiles, a.n_maps = 0, a.fp16 = l.fp16, a.n_tile = l.n_tile;
  const bool kept = l.epi == kEpiDgated && !l.f32;
  a.chains = l.chains, a.stages = stage_count(l.cta, l.n_tile, kept);
  a.whole = l.whole, a.part_kb = l.f32 && !l.fp16 ? 2 * kChainKb : 1 << 30;
  a.slots = (float*)slots, a.flags = flags, a.zero = zero, a.n_zero = n_zero;
  for (int c = 0; c <= kSms; ++c) a.cut[c] = c <= l.clusters && l.whole < l.n_tiles ? l.cut[c] : 0;
  bool done[kProdMaps] = {};
  *what = "cuTensorMapEncodeTiled";
  for (int k = 0; k < l.n_jobs; ++k) {
    ProdJob& j = l.job[k];
    a.job[k] = j;
    // an operand is read with the same boxes by every product of a launch
    const int nh = l.epi == kEpiGated ? l.n_tile / 2 : l.n_tile / l.cta;
    if (!done[j.map_a] && !encode(&a.map[j.map_a], l.op[j.map_a], l.fp16, j.a_mn ? 64 : 128)) return cudaErrorInvalidValue;
    if (!done[j.map_b] && !encode(&a.map[j.map_b], l.op[j.map_b], l.fp16, j.b_mn ? 64 : nh)) return cudaErrorInvalidValue;
    done[j.map_a] = done[j.map_b] = true;
    a.n_maps = std::max(a.n_maps, std::max(j.map_a, j.map_b) + 1);
  }
  if (kept) {
    const ProdJob& j = l.job[0];   // (one product; its columns fill whole sectors of a row)
    const int64_t hi = (const char*)j.p - (const char*)j.a, lo = j.p_lo - j.a_lo;
    if (!encode(&a.map[kMapHi], CU_TENSOR_MAP_DATA_TYPE_UINT16, j.a, j.ldo, j.M, j.ldo * 2, hi, 2, 32, 32, CU_TENSOR_MAP_SWIZZLE_64B) ||
        !encode(&a.map[kMapLo], CU_TENSOR_MAP_DATA_TYPE_UINT8, j.a_lo, j.ldo, j.M, j.ldo, lo, 2, 32, 32, CU_TENSOR_MAP_SWIZZLE_32B) ||
        !encode(&a.map[kMapOut], CU_TENSOR_MAP_DATA_TYPE_UINT16, j.out, j.ldo, j.M, j.ldo * 2, j.half * 2, 2, 32, 32,
                CU_TENSOR_MAP_SWIZZLE_64B))
      return cudaErrorInvalidValue;
    a.n_maps = kMapOut + 1;
  }
  *what = "spoiling a flag";
  if (l.whole < l.n_tiles && g_withhold.load(std::memory_order_relaxed) &&
      (e = withhold_one(a, l.cta, clusters, st)) != cudaSuccess)
    return e;
  *what = "product launch";
  return with_kernel(l.cta, l.epi, l.act, l.f32, [&](auto c, auto k, auto a_, auto t) {
    return launch<c.value, k.value, a_.value, t.value>(a, clusters, st);
  });
}

void sizes(const ProdLaunch* l, int n, int64_t& slots, int64_t& flags) {
  slots = flags = 0;
  for (int k = 0; k < n; ++k) slots = std::max(slots, round_up(l[k].slot_bytes, 256)), flags += l[k].flag_bytes;
}
}  // namespace

int64_t prod_bytes(const ProdLaunch* l, int n) {
  int64_t slots, flags;
  sizes(l, n, slots, flags);
  return slots + round_up(flags, 256);
}

cudaError_t prod_run_all(StageLaunch& stage, ProdLaunch* l, int n, void* workspace, cudaStream_t st, const char** what) {
  int64_t slots, flags;
  sizes(l, n, slots, flags);
  int* at = (int*)((char*)workspace + slots);
  cudaError_t e = cudaSuccess;
  // flags are cleared by the staging launch or, where there is none, the first product's apart, the others' by the
  // product before them (a memset of its own keeps the next launch's set-up from overlapping: 3 us)
  const bool staged = stage.n > 0;
  stage.zero = at, stage.n_zero = (int)(flags / 4);
  if (staged) {
    *what = "staging launch";
    e = stage_run(stage, st);
  } else if (l[0].flag_bytes) {
    *what = "clearing flags";
    e = cudaMemsetAsync(at, 0, l[0].flag_bytes, st);
  }
  for (int k = 0; e == cudaSuccess && k < n; ++k) {
    int* next = at + l[k].flag_bytes / 4;
    e = prod_run(l[k], workspace, at, next, staged || k + 1 == n ? 0 : (int)(l[k + 1].flag_bytes / 4), st, what);
    at = next;
  }
  return e;
}

cudaError_t stage_run(StageLaunch& s, cudaStream_t st) {
  int64_t most = 0;
  for (int k = 0; k < s.n; ++k) {
    StageJob& j = s.job[k];
    j.shift = 0;
    while (j.shift < 8 && (1 << j.shift) < j.ldp >> 3) ++j.shift;
    most = std::max<int64_t>(most, ceil_div(j.rows, 256 >> j.shift));
  }
  if (most == 0) return cudaSuccess;
  launch_pdl(k_stage, dim3((unsigned)std::min<int64_t>(most, kSms * 8), s.n), dim3(256), 0, st, s);
  return cudaGetLastError();
}

}  // namespace tp

using namespace tp;

extern "C" tp_status pack_ops_check(void* cuda_stream) {
  // what this thread's last check of a stream saw, once something has given up; of more streams than that the
  // oldest entry goes, and its stream is told again
  struct Seen {
    int dev, count;
    void* stream;
  };
  constexpr int kSeen = 64;
  thread_local Seen seen[kSeen];
  thread_local int n_seen = 0;
  int v = 0, dev = 0;
  cudaStream_t st = (cudaStream_t)cuda_stream;
  auto read = [&](const int& from) {
    cudaError_t e = cudaMemcpyFromSymbolAsync(&v, from, sizeof v, 0, cudaMemcpyDeviceToHost, st);
    return e == cudaSuccess ? cudaStreamSynchronize(st) : e;
  };
  cudaError_t e = cudaGetDevice(&dev);
  if (e == cudaSuccess && (dev < 0 || dev >= kMaxDevices)) e = cudaErrorInvalidDevice;
  if (e == cudaSuccess) e = read(g_prod_err);
  Failures f;
  if (e == cudaSuccess) {
    // whoever takes the word counts it before another check looks at the count
    std::lock_guard<std::mutex> lock(g_failures_mu);
    if (v != 0) {
      k_take_err<<<1, 1, 0, st>>>();
      e = cudaGetLastError();
      if (e == cudaSuccess) e = read(g_prod_taken);
      if (e == cudaSuccess && v != 0) ++g_failures[dev].count, g_failures[dev].site = v;
    }
    f = g_failures[dev];
  }
  if (e != cudaSuccess) {
    cudaGetLastError();   // reported here
    return ops_fail(TP_ECUDA, "pack_ops_check: %s", cudaGetErrorString(e));
  }
  if (f.count == 0) return TP_OK;
  int k = 0;
  while (k < std::min(n_seen, kSeen) && !(seen[k].dev == dev && seen[k].stream == cuda_stream)) ++k;
  if (k == std::min(n_seen, kSeen)) k = n_seen++ % kSeen, seen[k] = Seen{dev, 0, cuda_stream};
  if (f.count == seen[k].count) return TP_OK;
  seen[k].count = f.count;
  return ops_fail(TP_ETIMEOUT, "a wait of a tensor-core product gave up (site %d)", f.site);
}

extern "C" tp_status pack_debug_ops_withhold(void) {
  g_withhold.store(true);
  return TP_OK;
}
