// gated.cu -- the gated feed-forward block, forward and backward (entry points
// in tabpack_ops.h, products in prod.cu).
//
//   g = x Wg^T, u = x Wu^T, h = act(g) u, y = h Wd^T            (two launches)
//   dh = dy Wd, dg = dh u act'(g), du = dh act(g)               (one launch)
//   dx = [dg du] Wgu, dWgu = [dg du]^T x, dWd = dy^T h          (one launch)
//
// Both projections are one product: a tile holds a block of gate columns and
// the same block of up columns, so that the epilogue has both factors of h in
// registers and neither g nor u is written.  For the backward pass it keeps
// act(g) and u act'(g), the two numbers that dh is multiplied by, instead of g
// and u, to 24 bits: no exponential in the backward epilogue, and no rounding
// that shows.  Roundings to bf16 (of bf16 blocks): h, dg and du, because the
// tensor cores take them so; every sum is fp32.  32-bit blocks
// keep fp32 and multiply in three bf16 parts each (see prod.cu).
//
// Forward and backward of 2048 rows, d = d_out = 1024, f = 2048, bf16: 85 us,
// of which the operations at the measured tensor rate take 40; of 16384 rows,
// f = 4096: 831 us, 1.49 PFLOP/s (power cap; 788 at best); fp32, of 2000 rows,
// d = d_out = 1024, f = 2048: 392 us, of which the six products take 237.
#include <algorithm>

#include "prod.cuh"
#include "rows.cuh"

using namespace tp;

namespace {

struct Geo {
  int64_t rows;
  int32_t d, f, d_out;
  bool f32;
  int parts;                     // bf16 parts of an operand
  int64_t ldf;                   // pitch of h, act(g), u act'(g) and their gradients: whole 32-byte sectors
  Geo(int64_t r, int32_t d_, int32_t f_, int32_t o, int32_t prec)
      : rows(r), d(d_), f(f_), d_out(o), f32(prec == TP_FP32), parts(f32 ? 3 : 1), ldf(round_up(f_, 32)) {}
};

// What a forward pass keeps: h as bf16 parts, act(g) and u act'(g) as fp32 or,
// of a bf16 block, as 24-bit floats; pitch ldf.
struct Saved {
  void *h, *a, *p;
  uint8_t *a_lo, *p_lo;
  int64_t h_bytes, bytes;
  Saved(const Geo& g, void* base) {
    Carver c(base);
    h = c.take(g.parts * g.rows * g.ldf * 2);
    h_bytes = c.used;
    a = c.take(g.rows * g.ldf * (g.f32 ? 4 : 2));
    p = c.take(g.rows * g.ldf * (g.f32 ? 4 : 2));
    a_lo = (uint8_t*)c.take(g.f32 ? 0 : g.rows * g.ldf);
    p_lo = (uint8_t*)c.take(g.f32 ? 0 : g.rows * g.ldf);
    bytes = c.used;
  }
};

bool by_rows(const Geo& g) {
  const int64_t weights = (int64_t)g.f * (2 * (int64_t)g.d + g.d_out);
  return g.f32 ? rows_take32(g.rows, weights) : rows_take(g.rows, weights, 2 * ((int64_t)g.d | g.f), false);
}

constexpr int32_t kMaxDim = 1 << 17;
constexpr int64_t kMaxRows = (int64_t(1) << 31) - 256, kMaxElems = int64_t(1) << 40;   // (tiles are numbered in 32 bits)

tp_status check(int64_t rows, int32_t d, int32_t f, int32_t d_out, int32_t precision) {
  if (rows < 0 || rows > kMaxRows) return ops_fail(TP_EINVAL, "rows %lld out of range", (long long)rows);
  if (d < 1 || f < 1 || d_out < 1 || d > kMaxDim || f > kMaxDim || d_out > kMaxDim)
    return ops_fail(TP_EINVAL, "d %d, f %d and d_out %d must be in 1..%d", d, f, d_out, kMaxDim);
  if (rows * std::max(d, std::max(f, d_out)) > kMaxElems) return ops_fail(TP_EINVAL, "more than 2^40 elements in a matrix");
  if (precision != TP_BF16 && precision != TP_FP32) return ops_fail(TP_EINVAL, "unknown precision %d", precision);
  return TP_OK;
}

// An input matrix as an operand: as it lies there where it is bf16 and TMA
// takes it, else a copy (in parts) in the workspace.  halves: segments that
// its rows fall into (the gate and up halves).  Without a pointer (sizes are
// being asked for) a matrix counts as one that has to be copied.
struct Stager {
  const Geo& g;
  Carver& ws;
  StageLaunch launch;
  Stager(const Geo& g_, Carver& w) : g(g_), ws(w) { launch.n = 0; }
  ProdOperand operand(const void* src, int64_t ld, int64_t rows, int32_t cols, int halves) {
    const int64_t seg_rows = rows / halves;
    ProdOperand o{src, ld, seg_rows, cols, seg_rows * ld, halves};
    if (src != nullptr && !g.f32 && tma_ready(src, ld)) return o;
    o.ld = round_up(cols, 8);
    o.seg = seg_rows * o.ld;
    o.n_seg = halves * g.parts;
    o.base = ws.take(rows * g.parts * o.ld * 2);
    launch.job[launch.n++] =
        StageJob{src, const_cast<void*>(o.base), ld, rows, seg_rows, o.ld, cols, g.f32 ? kStageF32 : kStageBf16};
    return o;
  }
};

struct Plans {
  ProdLaunch l[2];
};

void job(ProdLaunch& l, int64_t M, int64_t N, int64_t K, int ma, int mb, bool a_mn, bool b_mn, int halves, void* out,
         int64_t ldo) {
  ProdJob& j = l.job[l.n_jobs++];
  j = ProdJob{};
  j.M = (int32_t)M, j.N = (int32_t)N, j.K = (int32_t)K;
  j.map_a = ma, j.map_b = mb, j.a_mn = a_mn, j.b_mn = b_mn;
  j.out = out, j.ldo = ldo;
  prod_pairs(j, l.f32, halves);
}

void start(ProdLaunch& l, const Geo& g, int epi, int act) {
  l = ProdLaunch{};
  l.epi = epi, l.act = act, l.f32 = g.f32;
}

int64_t plan(Plans& p) {
  for (ProdLaunch& l : p.l) prod_plan(l);
  return prod_bytes(p.l, 2);
}

void plan_forward(Plans& p, const Geo& g, int act, const ProdOperand& x, const ProdOperand& wgu, const ProdOperand& wd,
                  const Saved& s, bool keep, void* y) {
  start(p.l[0], g, kEpiGated, act);
  p.l[0].op[0] = x, p.l[0].op[1] = wgu;
  job(p.l[0], g.rows, g.f, g.d, 0, 1, false, false, 1, s.h, g.ldf);
  ProdJob& j = p.l[0].job[0];
  j.up = g.parts, j.part = g.rows * g.ldf;
  j.a = keep ? s.a : nullptr, j.p = keep ? s.p : nullptr, j.a_lo = s.a_lo, j.p_lo = s.p_lo;
  start(p.l[1], g, kEpiPlain, 0);
  p.l[1].op[0] = ProdOperand{s.h, g.ldf, g.rows, g.f, g.rows * g.ldf, g.parts}, p.l[1].op[1] = wd;
  job(p.l[1], g.rows, g.d_out, g.f, 0, 1, false, false, 1, y, g.d_out);
}

void plan_backward(Plans& p, const Geo& g, const ProdOperand& dy, const ProdOperand& x, const ProdOperand& wgu,
                   const ProdOperand& wd, const Saved& s, void* dgu, void* dx, void* dwgu, void* dwd) {
  const int64_t plane = g.rows * g.ldf;
  const ProdOperand h{s.h, g.ldf, g.rows, g.f, plane, g.parts};
  const ProdOperand d2{dgu, g.ldf, g.rows, g.f, plane, 2 * g.parts};
  start(p.l[0], g, kEpiDgated, 0);
  p.l[0].op[0] = dy, p.l[0].op[1] = wd;
  job(p.l[0], g.rows, g.f, g.d_out, 0, 1, false, true, 1, dgu, g.ldf);
  ProdJob& j = p.l[0].job[0];
  j.part = plane, j.half = g.parts * plane, j.a = s.a, j.p = s.p;
  j.a_lo = s.a_lo, j.p_lo = s.p_lo;

  ProdLaunch& l = p.l[1];
  start(l, g, kEpiPlain, 0);
  const int64_t e = g.f32 ? 4 : 2;
  // an operand that two products read along different dimensions has two maps
  l.op[0] = d2, l.op[1] = wgu, l.op[2] = d2, l.op[3] = x, l.op[4] = dy, l.op[5] = h;
  job(l, g.rows, g.d, g.f, 0, 1, false, true, 2, dx, g.d);
  job(l, g.f, g.d, g.rows, 2, 3, true, true, 1, dwgu, g.d);
  job(l, g.f, g.d, g.rows, 2, 3, true, true, 1, dwgu ? (char*)dwgu + (int64_t)g.f * g.d * e : nullptr, g.d);
  for (int q = 0; q < l.job[2].n_pairs; ++q) l.job[2].sa[q] += g.parts;   // du
  job(l, g.d_out, g.f, g.rows, 4, 5, true, true, 1, dwd, g.f);
}

tp_status run(Plans& p, Stager& st, Carver& c, int64_t workspace_bytes, cudaStream_t stream, const char* who) {
  const int64_t need = c.used + plan(p);
  if (workspace_bytes < need) return ops_fail(TP_EINVAL, "%s: a workspace of %lld bytes is needed", who, (long long)need);
  const tp_status s = ops_device();
  if (s != TP_OK) return s;
  void* products = c.take(0);
  const char* what = "";
  const cudaError_t e = prod_run_all(st.launch, p.l, 2, products, stream, &what);
  if (e == cudaSuccess) return TP_OK;
  cudaGetLastError();   // reported here
  return ops_fail(TP_ECUDA, "%s: %s: %s", who, what, cudaGetErrorString(e));
}

}  // namespace

extern "C" {

tp_status pack_gated_bytes(int64_t rows, int32_t d, int32_t f, int32_t d_out, int32_t precision, int64_t* saved,
                           int64_t* forward, int64_t* backward) {
  const tp_status s = check(rows, d, f, d_out, precision);
  if (s != TP_OK) return s;
  const Geo g(rows, d, f, d_out, precision);
  const Saved sv(g, nullptr);
  if (saved) *saved = sv.bytes;
  if (forward) {
    Carver c(nullptr);
    c.take(sv.h_bytes);   // h, where it is not kept
    Stager st(g, c);
    const ProdOperand x = st.operand(nullptr, d, rows, d, 1), wgu = st.operand(nullptr, d, 2 * (int64_t)f, d, 2);
    const ProdOperand wd = st.operand(nullptr, f, d_out, f, 1);
    Plans p;
    plan_forward(p, g, 0, x, wgu, wd, sv, false, nullptr);
    *forward = rows == 0 ? 0 : by_rows(g) ? sv.h_bytes : c.used + plan(p);
  }
  if (backward) {
    Carver c(nullptr);
    c.take(2 * g.parts * rows * g.ldf * 2);
    Stager st(g, c);
    const ProdOperand dy = st.operand(nullptr, d_out, rows, d_out, 1), x = st.operand(nullptr, d, rows, d, 1);
    const ProdOperand wgu = st.operand(nullptr, d, 2 * (int64_t)f, d, 2), wd = st.operand(nullptr, f, d_out, f, 1);
    Plans p;
    plan_backward(p, g, dy, x, wgu, wd, sv, nullptr, nullptr, nullptr, nullptr);
    *backward = rows ? c.used + plan(p) : 0;
  }
  return TP_OK;
}

tp_status pack_gated_forward(const void* x, int64_t ldx, const void* w_gate_up, const void* w_down, int64_t rows,
                             int32_t d, int32_t f, int32_t d_out, int32_t act, int32_t precision, void* y, void* saved,
                             void* workspace, int64_t workspace_bytes, void* cuda_stream) {
  tp_status s = check(rows, d, f, d_out, precision);
  if (s != TP_OK) return s;
  if (act < TP_ACT_RELU || act > TP_ACT_GELU) return ops_fail(TP_EINVAL, "unknown activation %d", act);
  if (ldx < d) return ops_fail(TP_EINVAL, "ldx %lld is less than d %d", (long long)ldx, d);
  if (rows == 0) return TP_OK;
  if (!x || !w_gate_up || !w_down || !y) return ops_fail(TP_EINVAL, "null argument");
  if ((uintptr_t)saved & 255) return ops_fail(TP_EINVAL, "saved must be 256-byte aligned");
  if (!workspace || ((uintptr_t)workspace & 255)) return ops_fail(TP_EINVAL, "the workspace must be 256-byte aligned");
  const Geo g(rows, d, f, d_out, precision);
  Carver c(workspace);
  void* own = c.take(Saved(g, nullptr).h_bytes);
  const Saved sv(g, saved ? saved : own);
  cudaStream_t stream = (cudaStream_t)cuda_stream;
  // a few rows: the weights stream past them, twice, with nothing in between
  if (by_rows(g)) {
    if (workspace_bytes < c.used) return ops_fail(TP_EINVAL, "a workspace of %lld bytes is needed", (long long)c.used);
    if ((s = ops_device()) != TP_OK) return s;
    // h for the second product: a bf16 block's kept one, a 32-bit block's in fp32
    const int64_t ldh = g.f32 ? f : g.ldf;
    void* h = g.f32 ? own : sv.h;
    cudaError_t e = rows_gated(RowsGated{x, w_gate_up, ldx, rows, d, f, act, g.f32, h, ldh, saved ? sv.a : nullptr,
                                         saved ? sv.p : nullptr, sv.h, g.ldf, rows * g.ldf, sv.a_lo,
                                         sv.p_lo}, stream);
    if (e == cudaSuccess) e = rows_plain(h, ldh, w_down, rows, f, d_out, g.f32, y, stream);
    if (e == cudaSuccess) return TP_OK;
    cudaGetLastError();   // reported here
    return ops_fail(TP_ECUDA, "pack_gated_forward: %s", cudaGetErrorString(e));
  }
  Stager st(g, c);
  const ProdOperand xo = st.operand(x, ldx, rows, d, 1), wgu = st.operand(w_gate_up, d, 2 * (int64_t)f, d, 2);
  const ProdOperand wd = st.operand(w_down, f, d_out, f, 1);
  Plans p;
  plan_forward(p, g, act, xo, wgu, wd, sv, saved != nullptr, y);
  return run(p, st, c, workspace_bytes, stream, "pack_gated_forward");
}

tp_status pack_gated_backward(const void* dy, int64_t lddy, const void* x, int64_t ldx, const void* w_gate_up,
                              const void* w_down, const void* saved, int64_t rows, int32_t d, int32_t f, int32_t d_out,
                              int32_t precision, void* dx, void* dw_gate_up, void* dw_down, void* workspace,
                              int64_t workspace_bytes, void* cuda_stream) {
  tp_status s = check(rows, d, f, d_out, precision);
  if (s != TP_OK) return s;
  if (ldx < d) return ops_fail(TP_EINVAL, "ldx %lld is less than d %d", (long long)ldx, d);
  if (lddy < d_out) return ops_fail(TP_EINVAL, "lddy %lld is less than d_out %d", (long long)lddy, d_out);
  if (!dw_gate_up || !dw_down) return ops_fail(TP_EINVAL, "null argument");
  cudaStream_t stream = (cudaStream_t)cuda_stream;
  if (rows == 0) {   // sums over no rows
    if ((s = ops_device()) != TP_OK) return s;
    const int64_t e = precision == TP_FP32 ? 4 : 2;
    cudaError_t er = cudaMemsetAsync(dw_gate_up, 0, 2 * e * f * d, stream);
    if (er == cudaSuccess) er = cudaMemsetAsync(dw_down, 0, e * f * d_out, stream);
    if (er == cudaSuccess) return TP_OK;
    cudaGetLastError();   // reported here
    return ops_fail(TP_ECUDA, "pack_gated_backward: %s", cudaGetErrorString(er));
  }
  if (!dy || !x || !w_gate_up || !w_down || !saved || !dx) return ops_fail(TP_EINVAL, "null argument");
  if ((uintptr_t)saved & 255) return ops_fail(TP_EINVAL, "saved must be 256-byte aligned");
  if (!workspace || ((uintptr_t)workspace & 255)) return ops_fail(TP_EINVAL, "the workspace must be 256-byte aligned");
  const Geo g(rows, d, f, d_out, precision);
  const Saved sv(g, const_cast<void*>(saved));
  Carver c(workspace);
  void* dgu = c.take(2 * g.parts * rows * g.ldf * 2);
  Stager st(g, c);
  const ProdOperand dyo = st.operand(dy, lddy, rows, d_out, 1), xo = st.operand(x, ldx, rows, d, 1);
  const ProdOperand wgu = st.operand(w_gate_up, d, 2 * (int64_t)f, d, 2), wd = st.operand(w_down, f, d_out, f, 1);
  Plans p;
  plan_backward(p, g, dyo, xo, wgu, wd, sv, dgu, dx, dw_gate_up, dw_down);
  return run(p, st, c, workspace_bytes, stream, "pack_gated_backward");
}

}  // extern "C"
