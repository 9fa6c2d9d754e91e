// distill.cu -- distillation of m students from one teacher's top logits:
// loss and gradient in one call (entry points in tabpack_ops.h).
//
// Per row, with zm = max z, S = sum exp((z - zm) / tau), S1 = sum exp(z - zm)
// and the teacher's p over its k entries:
//   kd = tau^2 sum_j p_j (log p_j - (z_idj - zm) / tau + log S)
//   ce = log S1 - (z_y - zm)
//   dz = [alpha tau (exp((z - zm) / tau) / S - p) + (1 - alpha) (exp(z - zm) / S1 - onehot)] / rows
// The gradient's dense part is written for every class; then, after a barrier
// of the row's threads, the thread of each entry writes the whole value at
// its class (summing the entries of the same class itself), so no value is
// added to in memory and the result does not depend on any order.
//
// Bound by HBM (z read, dz written) for many classes, by latency for few.
// Up to 1024 classes a group of 8 to 32 lanes holds a row in registers.
// Above, a block takes a row: running maximum and sums in one pass, and the
// gradient in a second one that finds the row in L2.
#include <algorithm>

#include "prod.cuh"

using namespace tp;

namespace {

constexpr int kMaxK = 128;
constexpr float kLog2e = 1.44269504088896340736f;
__device__ __forceinline__ float neg_inf() { return __uint_as_float(0xFF800000u); }

template <typename T>
struct Args {
  const T* z;
  const int32_t *ids, *labels;
  const float* top;
  T* dz;
  float* row_loss;     // [m * rows]
  int64_t all, rows;   // m * rows
  int32_t n, k;
  int32_t power;       // exp(v) from e = exp(v / tau): 1: e, 2: e^2, 4: e^4, 0: an exponential of its own
  int32_t soft, hard;  // alpha > 0; alpha < 1 and there are labels
  float inv_tau, tau, alpha, inv_rows;
};

// exp(v / tau) and exp(v) for v <= 0
template <typename T>
__device__ __forceinline__ float exp_tau(const Args<T>& g, float v) {
  return exp2f(v * (g.inv_tau * kLog2e));
}
template <typename T>
__device__ __forceinline__ float exp_one(const Args<T>& g, float v, float e) {
  if (g.power == 1) return e;
  if (g.power == 2) return e * e;
  if (g.power == 4) {
    const float s = e * e;
    return s * s;
  }
  return exp2f(v * kLog2e);
}

// What a row's threads agree on once its sums are known.
struct Row {
  float zm, ca, c1, log_s, log_s1;   // ca = alpha tau / (S rows), c1 = (1 - alpha) / (S1 rows); 0 without a teacher / label
  int label;                         // -1: none
};

// The dense part of the gradient at a class of logit z.
template <typename T>
__device__ __forceinline__ float dense(const Args<T>& g, const Row& r, float z) {
  const float v = z - r.zm, e = exp_tau(g, v);
  float d = r.ca * e;
  if (r.c1 != 0.f) d += r.c1 * exp_one(g, v, e);
  return d;
}

// Entry j's share of kd / tau^2 and its class's gradient.
template <typename T>
__device__ __forceinline__ float entry(const Args<T>& g, const Row& r, const T* z, T* dz, const int* ids, const float* p,
                                       float log_p, int j) {
  const int id = ids[j];
  if (id < 0) return 0.f;
  const float zi = Elem<T>::to_f(z[id]), pj = p[j];
  if (dz) {
    float same = 0.f;
    for (int i = 0; i < g.k; ++i) same += ids[i] == id ? p[i] : 0.f;
    float d = dense(g, r, zi) - g.alpha * g.tau * g.inv_rows * same;
    if (id == r.label) d -= (1.f - g.alpha) * g.inv_rows;
    dz[id] = Elem<T>::from_f(d);
  }
  return pj == 0.f ? 0.f : pj * (log_p - (zi - r.zm) * g.inv_tau + r.log_s);
}

template <int kG>
__device__ __forceinline__ float group_sum(float v) {
#pragma unroll
  for (int o = kG / 2; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}
template <int kG>
__device__ __forceinline__ float group_max(float v) {
#pragma unroll
  for (int o = kG / 2; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, o));
  return v;
}
template <int kG>
__device__ __forceinline__ bool group_any(bool b, int lane) {
  const uint32_t m = __ballot_sync(0xffffffffu, b);
  const uint32_t mine = kG == 32 ? 0xffffffffu : ((1u << kG) - 1u) << (lane & ~(kG - 1));
  return (m & mine) != 0;
}

// The teacher's entries of a row into shared memory: ids (-1: none) and p; a
// group's lane gl takes entries gl, gl + kG, ...  Returns whether there is an
// entry; log p_j = (top_j - hi) / tau - log_tot.
template <typename T, int kG>
__device__ __forceinline__ bool teacher(const Args<T>& g, int64_t b, int gl, int lane, int* ids, float* p, float& hi,
                                        float& log_tot) {
  const int32_t* gi = g.ids + b * g.k;
  const float* gt = g.top + b * g.k;
  hi = neg_inf();
  bool any = false;
  for (int j = gl; j < g.k; j += kG) {
    const int id = gi[j];
    const float t = gt[j];
    const bool ok = id >= 0 && id < g.n && t != neg_inf();
    ids[j] = ok ? id : -1;
    if (ok) hi = fmaxf(hi, t);
    any |= ok;
  }
  hi = group_max<kG>(hi);
  any = group_any<kG>(any, lane);
  float tot = 0.f;
  for (int j = gl; j < g.k; j += kG) {
    const float e = ids[j] < 0 ? 0.f : exp2f((gt[j] - hi) * (g.inv_tau * kLog2e));
    p[j] = e;
    tot += e;
  }
  tot = group_sum<kG>(tot);
  const float inv = any ? 1.f / tot : 0.f;
  for (int j = gl; j < g.k; j += kG) p[j] *= inv;
  log_tot = logf(tot);
  __syncwarp();
  return any;
}

template <typename T, int kG, int kV>
__global__ void __launch_bounds__(256) k_distill_group(const Args<T> g) {
  extern __shared__ uint8_t raw[];
  constexpr int kGroups = 256 / kG;
  const int lane = threadIdx.x & 31, gl = threadIdx.x & (kG - 1), grp = threadIdx.x / kG;
  int* ids = (int*)raw + grp * g.k;
  float* p = (float*)raw + (kGroups + grp) * g.k;
  pdl_trigger();
  pdl_wait();
  const int64_t rr = (int64_t)blockIdx.x * kGroups + grp;
  const bool live = rr < g.all;
  const int64_t row = live ? rr : g.all - 1, b = row % g.rows;   // lanes past the last row go along with it
  const T* z = g.z + row * g.n;
  float v[kV];
  float zm = neg_inf();
  bool alive = false;
#pragma unroll
  for (int i = 0; i < kV; ++i) {
    const int c = gl + kG * i;
    v[i] = c < g.n ? Elem<T>::to_f(z[c]) : neg_inf();
    alive |= v[i] != neg_inf();
    zm = fmaxf(zm, v[i]);
  }
  float hi = 0.f, log_tot = 0.f;
  const bool has = g.soft && teacher<T, kG>(g, b, gl, lane, ids, p, hi, log_tot);
  int label = g.hard ? g.labels[b] : -1;
  if (label >= g.n || label < 0) label = -1;
  zm = group_max<kG>(zm);
  alive = group_any<kG>(alive, lane);
  float s = 0.f, s1 = 0.f;
#pragma unroll
  for (int i = 0; i < kV; ++i)
    if (gl + kG * i < g.n) {
      const float e = exp_tau(g, v[i] - zm);
      s += e;
      if (g.hard) s1 += exp_one(g, v[i] - zm, e);
    }
  s = group_sum<kG>(s);
  s1 = group_sum<kG>(s1);
  Row r;
  r.zm = zm, r.label = label;
  r.log_s = logf(s), r.log_s1 = logf(s1);
  r.ca = has ? g.alpha * g.tau * g.inv_rows / s : 0.f;
  r.c1 = label >= 0 ? (1.f - g.alpha) * g.inv_rows / s1 : 0.f;
  T* dz = g.dz && live ? g.dz + row * g.n : nullptr;
  if (dz) {
#pragma unroll
    for (int i = 0; i < kV; ++i) {
      const int c = gl + kG * i;
      if (c < g.n) {
        float d = alive ? dense(g, r, v[i]) : 0.f;
        if (alive && c == label) d -= (1.f - g.alpha) * g.inv_rows;
        dz[c] = Elem<T>::from_f(d);
      }
    }
  }
  __syncwarp();
  float kd = 0.f;
  if (has && alive)
    for (int j = gl; j < g.k; j += kG)
      kd += entry(g, r, z, dz, ids, p, (g.top[b * g.k + j] - hi) * g.inv_tau - log_tot, j);
  kd = group_sum<kG>(kd);
  if (gl == 0 && live) {
    float loss = 0.f;
    if (has && alive) loss += g.alpha * g.tau * g.tau * kd;
    if (label >= 0 && alive) loss += (1.f - g.alpha) * (r.log_s1 - (Elem<T>::to_f(z[label]) - zm));
    g.row_loss[row] = loss;
  }
}

// ------------------------------------------------- many classes: a block a row
// Walks a row: f(first class, number, values) over groups of eight aligned
// classes and, at the ends, single ones.
template <typename T, int kThreads, typename F>
__device__ __forceinline__ void walk(const T* z, int n, F f) {
  constexpr int kV = 16 / sizeof(T);
  const int head = min(n, (int)((16 - ((uintptr_t)z & 15)) & 15) / (int)sizeof(T));
  const int body = (n - head) / kV, tail0 = head + body * kV;
  if ((int)threadIdx.x < head) {
    float v[1] = {Elem<T>::to_f(z[threadIdx.x])};
    f(std::integral_constant<int, 1>(), (int)threadIdx.x, v);
  }
  for (int i = threadIdx.x; i < body; i += kThreads) {
    const int c = head + i * kV;
    const uint4 w = *reinterpret_cast<const uint4*>(z + c);
    const uint32_t u[4] = {w.x, w.y, w.z, w.w};
    float v[kV];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      if constexpr (sizeof(T) == 4) {
        v[e] = __uint_as_float(u[e]);
      } else {
        v[2 * e] = __uint_as_float(u[e] << 16);
        v[2 * e + 1] = __uint_as_float(u[e] & 0xFFFF0000u);
      }
    }
    f(std::integral_constant<int, kV>(), c, v);
  }
  const int c = tail0 + threadIdx.x;
  if (c < n) {
    float v[1] = {Elem<T>::to_f(z[c])};
    f(std::integral_constant<int, 1>(), c, v);
  }
}

template <typename T, int kThreads>
__global__ void __launch_bounds__(kThreads) k_distill_row(const Args<T> g) {
  constexpr int kWarps = kThreads / 32;
  __shared__ int ids[kMaxK];
  __shared__ float p[kMaxK];
  __shared__ float rm[kWarps], rs[kWarps], rs1[kWarps];
  __shared__ int has_s, alive_s;
  __shared__ float hi_s, log_tot_s;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  pdl_trigger();
  pdl_wait();
  const int64_t row = blockIdx.x, b = row % g.rows;
  const T* z = g.z + row * g.n;
  if (threadIdx.x == 0) alive_s = 0;
  int label = g.hard ? g.labels[b] : -1;
  if (label >= g.n || label < 0) label = -1;
  if (warp == 0 && g.soft) {
    float hi = 0.f, log_tot = 0.f;
    const bool has = teacher<T, 32>(g, b, lane, lane, ids, p, hi, log_tot);
    if (lane == 0) has_s = has, hi_s = hi, log_tot_s = log_tot;
  }
  // running maximum and sums of a thread's classes
  float m = neg_inf(), s = 0.f, s1 = 0.f;
  bool alive = false;
  walk<T, kThreads>(z, g.n, [&](auto nv, int, float* v) {
    constexpr int kN = nv.value;
    float hi = v[0];
#pragma unroll
    for (int e = 1; e < kN; ++e) hi = fmaxf(hi, v[e]);
#pragma unroll
    for (int e = 0; e < kN; ++e) alive |= v[e] != neg_inf();
    if (hi > m) {
      const float f = exp_tau(g, m - hi);   // 0 at first
      s *= f;
      s1 *= exp_one(g, m - hi, f);
      m = hi;
    }
    if (m == neg_inf()) {
      // nothing but -inf (or NaN) so far: a NaN has to reach the sum
#pragma unroll
      for (int e = 0; e < kN; ++e)
        if (v[e] != v[e]) s = v[e], s1 = v[e];
      return;
    }
#pragma unroll
    for (int e = 0; e < kN; ++e) {
      const float x = exp_tau(g, v[e] - m);
      s += x;
      if (g.hard) s1 += exp_one(g, v[e] - m, x);
    }
  });
  const float wm = group_max<32>(m);
  // a thread without a class above -inf adds what it has (0 or NaN)
  const float f = m == neg_inf() ? 1.f : exp_tau(g, m - wm);
  s = group_sum<32>(s * f);
  s1 = group_sum<32>(s1 * (m == neg_inf() ? 1.f : exp_one(g, m - wm, f)));
  if (lane == 0) rm[warp] = wm, rs[warp] = s, rs1[warp] = s1;
  __syncthreads();
  if (__any_sync(0xffffffffu, alive) && lane == 0) alive_s = 1;
  float zm = neg_inf();
#pragma unroll
  for (int k = 0; k < kWarps; ++k) zm = fmaxf(zm, rm[k]);
  s = s1 = 0.f;
#pragma unroll 4
  for (int k = 0; k < kWarps; ++k) {
    const float q = rm[k] == neg_inf() ? 1.f : exp_tau(g, rm[k] - zm);
    s += rs[k] * q;
    s1 += rs1[k] * (rm[k] == neg_inf() ? 1.f : exp_one(g, rm[k] - zm, q));
  }
  __syncthreads();
  const bool has = g.soft && has_s;
  alive = alive_s;
  Row r;
  r.zm = zm, r.label = label;
  r.log_s = logf(s), r.log_s1 = logf(s1);
  r.ca = has ? g.alpha * g.tau * g.inv_rows / s : 0.f;
  r.c1 = label >= 0 ? (1.f - g.alpha) * g.inv_rows / s1 : 0.f;
  T* dz = g.dz ? g.dz + row * g.n : nullptr;
  if (dz) {
    const bool vec = (((uintptr_t)z ^ (uintptr_t)dz) & 15) == 0;
    walk<T, kThreads>(z, g.n, [&](auto nv, int c, float* v) {
      constexpr int kN = nv.value;
      float d[kN];
#pragma unroll
      for (int e = 0; e < kN; ++e) {
        d[e] = alive ? dense(g, r, v[e]) : 0.f;
        if (alive && c + e == label) d[e] -= (1.f - g.alpha) * g.inv_rows;
      }
      if constexpr (kN == 4) {
        if (vec) {
          *reinterpret_cast<float4*>(dz + c) = make_float4(d[0], d[1], d[2], d[3]);
          return;
        }
      } else if constexpr (kN == 8) {
        if (vec) {
          uint32_t u[4];
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const __nv_bfloat162 h = __floats2bfloat162_rn(d[2 * e], d[2 * e + 1]);
            u[e] = *reinterpret_cast<const uint32_t*>(&h);
          }
          *reinterpret_cast<uint4*>(dz + c) = make_uint4(u[0], u[1], u[2], u[3]);
          return;
        }
      }
#pragma unroll
      for (int e = 0; e < kN; ++e) dz[c + e] = Elem<T>::from_f(d[e]);
    });
    __syncthreads();
  }
  if (warp == 0) {
    float kd = 0.f;
    if (has && alive)
      for (int j = lane; j < g.k; j += 32)
        kd += entry(g, r, z, dz, ids, p, (g.top[b * g.k + j] - hi_s) * g.inv_tau - log_tot_s, j);
    kd = group_sum<32>(kd);
    if (lane == 0) {
      float loss = 0.f;
      if (has && alive) loss += g.alpha * g.tau * g.tau * kd;
      if (label >= 0 && alive) loss += (1.f - g.alpha) * (r.log_s1 - (Elem<T>::to_f(z[label]) - zm));
      g.row_loss[row] = loss;
    }
  }
}

// A student's mean over its rows, in a fixed order.
__global__ void __launch_bounds__(256) k_distill_mean(const float* row_loss, int64_t rows, float* loss) {
  __shared__ float s[8];
  pdl_trigger();
  pdl_wait();
  const float* p = row_loss + blockIdx.x * rows;
  float a = 0.f;
#pragma unroll 4
  for (int64_t i = threadIdx.x; i < rows; i += 256) a += p[i];
  a = group_sum<32>(a);
  if ((threadIdx.x & 31) == 0) s[threadIdx.x >> 5] = a;
  __syncthreads();
  if (threadIdx.x == 0) {
    for (int k = 1; k < 8; ++k) a += s[k];
    loss[blockIdx.x] = a / (float)rows;
  }
}

template <typename T, int kG, int kV>
void group(const Args<T>& a, cudaStream_t st) {
  launch_pdl(k_distill_group<T, kG, kV>, dim3((unsigned)ceil_div(a.all, 256 / kG)), dim3(256),
             (size_t)(256 / kG) * a.k * 8, st, a);
}

template <typename T>
void rows(const Args<T>& a, cudaStream_t st) {
  if (a.n <= 16) group<T, 8, 2>(a, st);
  else if (a.n <= 32) group<T, 8, 4>(a, st);
  else if (a.n <= 64) group<T, 16, 4>(a, st);
  else if (a.n <= 128) group<T, 32, 4>(a, st);
  else if (a.n <= 256) group<T, 32, 8>(a, st);
  else if (a.n <= 512) group<T, 32, 16>(a, st);
  else if (a.n <= 1024) group<T, 32, 32>(a, st);
  else if (a.n <= 8192) launch_pdl(k_distill_row<T, 256>, dim3((unsigned)a.all), dim3(256), 0, st, a);
  else launch_pdl(k_distill_row<T, 1024>, dim3((unsigned)a.all), dim3(1024), 0, st, a);
}

tp_status check(int64_t m, int64_t rows) {
  if (m < 1 || m > 65535 || rows < 0 || rows > (int64_t(1) << 31) / m - 1)
    return ops_fail(TP_EINVAL, "m %lld (1..65535) students of %lld rows: fewer than 2^31 rows in all are taken",
                    (long long)m, (long long)rows);
  return TP_OK;
}

}  // namespace

extern "C" {

tp_status pack_distill_bytes(int64_t m, int64_t rows, int64_t* workspace) {
  const tp_status s = check(m, rows);
  if (s != TP_OK) return s;
  if (!workspace) return ops_fail(TP_EINVAL, "null argument");
  *workspace = m * rows * 4;
  return TP_OK;
}

tp_status pack_distill(const void* z, int64_t m, int64_t n_rows, int32_t n, const int32_t* ids, const float* top,
                       int32_t k, const int32_t* labels, float tau, float alpha, int32_t precision, float* loss,
                       void* dz, void* workspace, int64_t workspace_bytes, void* cuda_stream) {
  tp_status s = check(m, n_rows);
  if (s != TP_OK) return s;
  if (n < 2) return ops_fail(TP_EINVAL, "n %d must be at least 2", n);
  if (k < 1 || k > kMaxK) return ops_fail(TP_EINVAL, "k %d must be in 1..%d", k, kMaxK);
  if (!(tau > 0.f) || !(tau <= 3.4e38f)) return ops_fail(TP_EINVAL, "tau must be positive and finite");
  if (!(alpha >= 0.f && alpha <= 1.f)) return ops_fail(TP_EINVAL, "alpha must be in 0..1");
  if (precision != TP_BF16 && precision != TP_FP32) return ops_fail(TP_EINVAL, "unknown precision %d", precision);
  if (!loss) return ops_fail(TP_EINVAL, "null argument");
  cudaStream_t st = (cudaStream_t)cuda_stream;
  cudaError_t e;
  if (n_rows == 0) {   // a mean over no rows: 0
    if ((s = ops_device()) != TP_OK) return s;
    e = cudaMemsetAsync(loss, 0, (size_t)m * 4, st);
  } else {
    if (!z || !ids || !top) return ops_fail(TP_EINVAL, "null argument");
    if (workspace_bytes < m * n_rows * 4 || !workspace || ((uintptr_t)workspace & 255))
      return ops_fail(TP_EINVAL, "a workspace of %lld bytes, 256-byte aligned, is needed", (long long)(m * n_rows * 4));
    if ((s = ops_device()) != TP_OK) return s;
    float* rl = (float*)workspace;
    const int power = tau == 1.f ? 1 : tau == 2.f ? 2 : tau == 4.f ? 4 : 0;
    const int soft = alpha > 0.f, hard = alpha < 1.f && labels != nullptr;
    if (precision == TP_FP32)
      rows(Args<float>{(const float*)z, ids, labels, top, (float*)dz, rl, m * n_rows, n_rows, n, k, power, soft, hard,
                       1.f / tau, tau, alpha, 1.f / (float)n_rows}, st);
    else
      rows(Args<__nv_bfloat16>{(const __nv_bfloat16*)z, ids, labels, top, (__nv_bfloat16*)dz, rl, m * n_rows, n_rows, n, k,
                               power, soft, hard, 1.f / tau, tau, alpha, 1.f / (float)n_rows}, st);
    launch_pdl(k_distill_mean, dim3((unsigned)m), dim3(256), 0, st, (const float*)rl, n_rows, loss);
    e = cudaGetLastError();
  }
  if (e == cudaSuccess) return TP_OK;
  cudaGetLastError();   // reported here
  return ops_fail(TP_ECUDA, "pack_distill: %s", cudaGetErrorString(e));
}

}  // extern "C"
