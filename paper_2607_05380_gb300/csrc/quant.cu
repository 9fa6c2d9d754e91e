// quant.cu -- the 8-bit product with a scale per row and output channel (entry
// point in tabpack_ops.h).
//
// sm_103a's tensor cores have no fast 8-bit integer rate, so the integers go
// through them as fp16, in which every int8 and every product of two is
// exact, with fp32 accumulators: sums are exact below 2^24.  A staging launch
// writes them out as fp16 first, so that TMA can feed them: 8192 rows, 2048 ->
// 4096, 85 us, of which the product takes 72 at the measured tensor rate; in
// the product's own pipeline the conversion would need more than the shared
// memory's 128 bytes a cycle.  A few rows take the weights as they are (rows.cu).
#include "prod.cuh"
#include "rows.cuh"

using namespace tp;

namespace {

constexpr int32_t kMaxDim = 1 << 17;
constexpr int64_t kMaxRows = (int64_t(1) << 31) - 256, kMaxElems = int64_t(1) << 40;   // (tiles are numbered in 32 bits)

tp_status check(int64_t rows, int32_t k, int32_t n, int32_t precision) {
  if (rows < 0 || rows > kMaxRows) return ops_fail(TP_EINVAL, "rows %lld out of range", (long long)rows);
  if (k < 1 || n < 1 || k > kMaxDim || n > kMaxDim)
    return ops_fail(TP_EINVAL, "k %d and n %d must be in 1..%d", k, n, kMaxDim);
  if (rows * (k > n ? k : n) > kMaxElems) return ops_fail(TP_EINVAL, "more than 2^40 elements in a matrix");
  if (precision != TP_BF16 && precision != TP_FP32) return ops_fail(TP_EINVAL, "unknown precision %d", precision);
  return TP_OK;
}

struct Work {
  ProdLaunch l;
  int64_t ldk, qx, qw, bytes;
  Work(int64_t rows, int32_t k, int32_t n, int32_t precision) {
    l = ProdLaunch{};
    l.epi = kEpiQuant, l.fp16 = 1, l.f32 = precision == TP_FP32, l.n_jobs = 1;
    ProdJob& j = l.job[0];
    j.M = (int32_t)rows, j.N = n, j.K = k;
    j.map_a = 0, j.map_b = 1, j.n_pairs = 1;
    prod_plan(l);
    ldk = round_up(k, 8);
    qx = round_up(rows * ldk * 2, 256), qw = round_up(n * ldk * 2, 256);
    bytes = qx + qw + prod_bytes(&l, 1);
  }
};

}  // namespace

extern "C" {

tp_status pack_product_q8_bytes(int64_t rows, int32_t k, int32_t n, int32_t precision, int64_t* workspace) {
  const tp_status s = check(rows, k, n, precision);
  if (s != TP_OK) return s;
  if (!workspace) return ops_fail(TP_EINVAL, "null argument");
  *workspace = rows == 0 || rows_take(rows, (int64_t)k * n, k, true) ? 0 : Work(rows, k, n, precision).bytes;
  return TP_OK;
}

tp_status pack_product_q8(const int8_t* q, int64_t ldq, const float* scale, const int8_t* w, const float* w_scale,
                          const float* bias, int64_t rows, int32_t k, int32_t n, int32_t precision, void* y,
                          void* workspace, int64_t workspace_bytes, void* cuda_stream) {
  tp_status s = check(rows, k, n, precision);
  if (s != TP_OK) return s;
  if (ldq < k) return ops_fail(TP_EINVAL, "ldq %lld is less than k %d", (long long)ldq, k);
  if (rows == 0) return TP_OK;
  if (!q || !scale || !w || !w_scale || !y) return ops_fail(TP_EINVAL, "null argument");
  cudaStream_t st = (cudaStream_t)cuda_stream;
  if (rows_take(rows, (int64_t)k * n, k, true)) {   // a few rows: the weights stream past them
    if ((s = ops_device()) != TP_OK) return s;
    const cudaError_t e = rows_quant(q, ldq, scale, w, w_scale, bias, rows, k, n, precision == TP_FP32, y, st);
    if (e == cudaSuccess) return TP_OK;
    cudaGetLastError();   // reported here
    return ops_fail(TP_ECUDA, "pack_product_q8: %s", cudaGetErrorString(e));
  }
  Work o(rows, k, n, precision);
  if (workspace_bytes < o.bytes || !workspace || ((uintptr_t)workspace & 255))
    return ops_fail(TP_EINVAL, "a workspace of %lld bytes, 256-byte aligned, is needed", (long long)o.bytes);
  if ((s = ops_device()) != TP_OK) return s;
  char* x16 = (char*)workspace;
  char* w16 = x16 + o.qx;
  StageLaunch sl;
  sl.n = 2;
  sl.job[0] = StageJob{q, x16, ldq, rows, rows, o.ldk, k, kStageS8};
  sl.job[1] = StageJob{w, w16, k, n, n, o.ldk, k, kStageS8};
  o.l.op[0] = ProdOperand{x16, o.ldk, rows, k, 0, 1};
  o.l.op[1] = ProdOperand{w16, o.ldk, n, k, 0, 1};
  ProdJob& j = o.l.job[0];
  j.out = y, j.ldo = n, j.sx = scale, j.sw = w_scale, j.bias = bias;
  const char* what = "";
  const cudaError_t e = prod_run_all(sl, &o.l, 1, w16 + o.qw, st, &what);
  if (e == cudaSuccess) return TP_OK;
  cudaGetLastError();   // reported here
  return ops_fail(TP_ECUDA, "pack_product_q8: %s: %s", what, cudaGetErrorString(e));
}

}  // extern "C"
