// prod.cuh -- single products on the 5th-generation tensor cores (prod.cu),
// shared by the student operators: the gated block (gated.cu) and the 8-bit
// product (quant.cu).
//
// A launch computes up to kProdJobs products C[r, c] = sum_k A(r, k) B(c, k)
// of 16-bit operands with one kind of epilogue.  An operand is a row-major
// matrix, or several of the same shape at equal distances ("segments"): the
// gate and up halves of a gated block's weights, and the three bf16 parts of
// a 32-bit operand.  A product runs over a list of segment pairs; each adds
// its own reduction to the same accumulator.
#pragma once

#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <atomic>

#include "tabpack_ops.h"
#include "tp_internal.cuh"

namespace tp {

constexpr int kProdJobs = 4, kProdMaps = 8, kProdPairs = 12;
constexpr int kSms = 152;          // the GB300's SMs; launches are planned for them

// A 16-bit matrix [rows, cols] with pitch ld (elements), n_seg times, seg elements apart.
struct ProdOperand {
  const void* base;
  int64_t ld, rows, cols, seg;
  int n_seg;
};

// Fused epilogues.
//   kEpiPlain  out = acc (bf16 or fp32)
//   kEpiGated  the tile holds a column block of the gate product and the same
//              block of the up product: h = act(g) u (as bf16 parts) and, for
//              a backward pass, act(g) and u act'(g)
//   kEpiDgated acc = dh: dg = dh u act'(g) and du = dh act(g), as bf16 parts
//   kEpiQuant  out = acc sx[r] sw[c] + b[c] (bf16 or fp32)
enum ProdEpi : int32_t { kEpiPlain = 0, kEpiGated = 1, kEpiDgated = 2, kEpiQuant = 3 };

struct ProdJob {
  // the product (set by the caller)
  int32_t M, N, K;                 // N: output columns (kEpiGated: of each half)
  int32_t map_a, map_b;            // operands, by their place in ProdLaunch::op
  int32_t a_mn, b_mn;              // 0: rows of the operand run over k's other index (K-major), 1: over k
  int32_t n_pairs;
  uint8_t sa[kProdPairs], sb[kProdPairs];   // segments of A and B
  int32_t up;                      // kEpiGated: segments from the gate half of B to the up half
  void* out;                       // kEpiGated: h; kEpiDgated: [dg; du]
  int64_t ldo;
  int64_t part;                    // elements between the bf16 parts of out
  int64_t half;                    // kEpiDgated: elements from dg to du
  void *a, *p;                     // kEpiGated / kEpiDgated: act(g), u act'(g) (NULL: not wanted): fp32, or of a
  uint8_t *a_lo, *p_lo;            // bf16 block the upper 16 bits of a 24-bit float, its lower 8 here
  const float *sx, *sw, *bias;     // kEpiQuant
  // the plan (set by prod_plan): K blocks, tiles, the first one's number
  int32_t kb, tm, tn, tile0;
};

struct ProdLaunch {
  int32_t epi, act, fp16, f32;     // f32: 32-bit outputs; operands of three parts and short accumulator chains
  int32_t n_jobs, n_ops;
  ProdOperand op[kProdMaps];
  ProdJob job[kProdJobs];
  // the plan: CTAs per tile, its columns, accumulator chains, tiles; clusters
  // (tile slots that run at once), and how the tiles are shared out: tiles
  // below whole go round robin, one cluster each; the others' K blocks, one
  // tile after another, are cut at cut[1], cut[2], ... into one run a cluster
  int32_t cta, n_tile, chains, n_tiles, clusters, whole;
  int32_t cut[kSms + 1];
  int64_t slot_bytes, flag_bytes;  // workspace for cut tiles' sums and their flags
};

// 32-bit mode: the six products of two parts that are above 2^-24, smallest
// first; halves: 1, or 2 for a reduction that runs over both halves of a
// gated block (segment = half * 3 + part).
void prod_pairs(ProdJob& j, bool f32, int halves);

// Chooses tiles and shares them out.
void prod_plan(ProdLaunch& l);
// Copies operands into a layout that TMA takes: rows of `cols` elements to
// rows of pitch ldp (a multiple of 8), in segments of rows_seg rows; fp32
// elements become three bf16 parts (segments s * 3 .. s * 3 + 2 of segment s),
// 8-bit integers fp16, bf16 stays.
enum StageType : int32_t { kStageBf16 = 0, kStageF32 = 1, kStageS8 = 2 };
struct StageJob {
  const void* src;
  void* dst;
  int64_t ld, rows, rows_seg, ldp;   // rows: rows_seg, or twice that
  int32_t cols, type, shift;         // shift: set by stage_run
};
constexpr int kStageJobs = 4;
struct StageLaunch {
  StageJob job[kStageJobs];
  int32_t n, n_zero;
  int* zero;                // n_zero words are set to 0 beside the copies
};
cudaError_t stage_run(StageLaunch& s, cudaStream_t st);

// Runs the staging copies (none: n = 0) and then n planned launches one after
// another in a workspace of prod_bytes.
int64_t prod_bytes(const ProdLaunch* l, int n);
cudaError_t prod_run_all(StageLaunch& stage, ProdLaunch* l, int n, void* workspace, cudaStream_t st, const char** what);

// Is a 16-bit operand fit for TMA as it lies there?
inline bool tma_ready(const void* p, int64_t ld) { return ((uintptr_t)p & 15) == 0 && ld % 8 == 0; }

// The device's word that a bounded wait of a product which gives up sets, and pack_ops_check reads.
cudaError_t prod_err_word(int** word);
// A TMA map of [rows][cols] bytes, ld from row to row, 128-byte swizzle; base and ld are multiples of 16.
bool tma_map_bytes(CUtensorMap* m, const void* base, int64_t cols, int64_t rows, int64_t ld, int box_cols, int box_rows);

// Runs f (a cudaError_t of no arguments: a kernel's attributes) once per device
// that succeeds; a failure is tried again by the next call.
struct OncePerDevice {
  std::atomic<uint64_t> done{0};
  template <typename F>
  cudaError_t operator()(F f) {
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    const uint64_t bit = dev < 64 ? uint64_t(1) << dev : 0;
    if (done.load(std::memory_order_relaxed) & bit) return cudaSuccess;
    if ((e = f()) == cudaSuccess) done.fetch_or(bit, std::memory_order_relaxed);
    return e;
  }
};

// Error reporting of the entry points without a handle.
tp_status ops_fail(tp_status s, const char* fmt, ...);
// Is a CUDA device there that the library runs on (an error status if not)?
tp_status ops_device();

// Consecutive pieces of a caller's workspace, 256 bytes aligned.
struct Carver {
  char* base;
  int64_t used = 0;
  explicit Carver(void* p) : base((char*)p) {}
  void* take(int64_t bytes) {
    void* p = base ? base + used : nullptr;
    used += round_up(bytes, 256);
    return p;
  }
};

}  // namespace tp
