// distill.cu -- distillation of m students from one teacher's top logits:
// loss and gradient in one call (entry points in tabpack_ops.h).
//
// Per row, with zm = max z, c = log2(e) / tau, e_i = 2^((z_i - zm) c), S = sum
// e_i, and e1_i, S1 likewise for tau = 1, and the teacher's p:
//   log softmax(z / tau)_i = ((z_i - zm) c - log2 S) / log2(e)
//   kd = tau^2 sum_j p_j (log p_j - log softmax(z / tau)[id_j])
//   dz = [alpha tau (e / S - p) + (1 - alpha) (e1 / S1 - onehot)] / rows
// z_i c - o in one multiply-add, o = zm c rounded, is off by that rounding, the
// same for every class, so it drops out; but for a row that a mask left at
// -10^10 or at the type's lowest value its power of two overflows: such rows
// ("far"), and all rows of a tau beyond 2^-18 .. 2^18, take the difference
// first.  For tau = 1, 2 and 4 e1 is the first, second or fourth power of e, so that a
// class costs one exponential a pass.
//
// The gradient's dense part is written for every class; then, after a barrier
// of the row's threads, the thread of each entry writes the whole value at
// its class (summing the entries of the same class itself), and one thread
// that at the label, if no entry has it: no value is added to in memory and
// the result does not depend on any order.
//
// Bound by HBM (z read, dz written) for many classes (2048 rows of 50021, bf16:
// 80 us, 0.76 of the measured copy rate, issue slots 60 % taken; fp32 182 us,
// 0.66; a tau without a shared exponential, bf16: 89 us), by latency for few (64
// students, 1024 rows of 10: 8.4 us) and by its loads of single elements
// between (80000 rows of 512, bf16: 85 us, 0.29).
//   up to 32 classes    of many rows, few entries: a thread takes a row, which blocks of 128
//                       rows stage in shared memory: no exchanges between lanes
//   up to 1024          8 to 32 lanes hold a row in registers
//   above               a block takes a row: running maximum and sums in one
//                       pass, the gradient in a second that finds the row in
//                       L2; one warp more works out the teacher's side meanwhile
#include <algorithm>
#include <type_traits>

#include "prod.cuh"

namespace tp {
namespace {

constexpr int kMaxK = 128;
constexpr int kMaxN = 2147482624;   // 2^31 - 1024: a thread's number past a row's last class (Span) is still an int
constexpr float kMinTau = 8.67361738e-19f;   // 2^-60: tau^2, log2(e) / tau and their like stay normal numbers
constexpr float kLog2e = 1.44269504088896340736f, kLn2 = 0.69314718055994530942f;
__device__ __forceinline__ float neg_inf() { return __uint_as_float(0xFF800000u); }
__device__ __forceinline__ float ex2(float v) {   // 2^v to 2 ulp; results below 2^-126 are 0
  float r;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(v));
  return r;
}

// The label's part: none, or e1 from e: the first, second, fourth power, or an
// exponential of its own.
enum Hard : int32_t { kNone = 0, kPow1 = 1, kPow2 = 2, kPow4 = 4, kOwn = 5 };

template <typename T>
struct Args {
  const T* z;
  const int32_t *ids, *labels;
  const float* top;
  T* dz;
  float* row_loss;     // [m * rows]
  int64_t all, rows;   // m * rows
  int32_t n, k;
  int32_t soft, hard;  // alpha > 0; Hard
  float c, tau, alpha, inv_rows;
};

template <int kHard>
__device__ __forceinline__ float pow_tau(float e) {
  return kHard == kPow2 ? e * e : kHard == kPow4 ? (e * e) * (e * e) : e;
}

// What a row's threads agree on once its sums are known.
struct Row {
  float zm, o, o1;            // maximum; zm c and zm log2(e), rounded
  bool far;                   // exponents from z - zm, not from z c - o
  float log_s, log_s1;        // base 2
  float ca, c1;               // alpha tau / (S rows), 0 without a teacher; (1 - alpha) / (S1 rows), 0 without a label
  int label;                  // -1: none
  bool alive;                 // a class above -inf (or NaN)
};

// (all -inf: zm = -inf, s = 0)
template <typename T>
__device__ __forceinline__ Row make_row(const Args<T>& g, float zm, bool far, float s, float s1, bool has, int label) {
  Row r;
  r.alive = !(zm == neg_inf() && s == 0.f);
  r.zm = r.alive ? zm : 0.f;
  r.o = __fmul_rn(r.zm, g.c), r.o1 = __fmul_rn(r.zm, kLog2e);
  r.far = far;
  r.log_s = log2f(s);
  r.log_s1 = log2f(s1);
  r.ca = has && r.alive ? g.alpha * g.tau * g.inv_rows / s : 0.f;
  r.c1 = label >= 0 && r.alive ? (1.f - g.alpha) * g.inv_rows / s1 : 0.f;
  r.label = r.alive ? label : -1;
  return r;
}

// log2 of e and of e1 (by an exponential of its own) at a class of logit z
__device__ __forceinline__ float power(float c, const Row& r, float z) { return r.far ? (z - r.zm) * c : fmaf(z, c, -r.o); }
__device__ __forceinline__ float power1(const Row& r, float z) {
  return r.far ? (z - r.zm) * kLog2e : fmaf(z, kLog2e, -r.o1);
}

// The dense part of the gradient at a class of logit z.
template <int kHard>
__device__ __forceinline__ float dense(float c, const Row& r, float z) {
  const float e = ex2(power(c, r, z));
  if (kHard == kNone) return e * r.ca;
  if (kHard == kPow1) return e * (r.ca + r.c1);
  if (kHard == kPow2) return e * fmaf(r.c1, e, r.ca);
  if (kHard == kPow4) return e * fmaf(r.c1 * e, e * e, r.ca);
  return fmaf(r.ca, e, r.c1 * ex2(power1(r, z)));
}
template <typename T>
__device__ __forceinline__ float dense_any(const Args<T>& g, const Row& r, float z) {
  switch (g.hard) {
    case kNone: return dense<kNone>(g.c, r, z);
    case kPow1: return dense<kPow1>(g.c, r, z);
    case kPow2: return dense<kPow2>(g.c, r, z);
    case kPow4: return dense<kPow4>(g.c, r, z);
    default: return dense<kOwn>(g.c, r, z);
  }
}

// log softmax(z / tau) and -log softmax(z) at a class of logit z
template <typename T>
__device__ __forceinline__ float log_q(const Args<T>& g, const Row& r, float z) {
  return (power(g.c, r, z) - r.log_s) * kLn2;
}
template <typename T>
__device__ __forceinline__ float cross_entropy(const Args<T>& g, const Row& r, float z) {
  const float v = g.hard == kOwn ? power1(r, z) : (float)g.hard * power(g.c, r, z);   // (kPow1, 2, 4: tau itself)
  return (r.log_s1 - v) * kLn2;
}
template <typename T>
__device__ __forceinline__ int label_of(const Args<T>& g, int64_t b) {
  const int y = g.hard ? g.labels[b] : -1;
  return y >= 0 && y < g.n ? y : -1;
}
template <typename T>
__device__ __forceinline__ float row_loss(const Args<T>& g, const Row& r, bool has, float kd, float z_label) {
  float loss = 0.f;
  if (has && r.alive) loss = g.alpha * g.tau * g.tau * kd;
  if (r.label >= 0) loss += (1.f - g.alpha) * cross_entropy(g, r, z_label);
  return loss;
}

// Entry j's share of kd / tau^2 and its class's gradient; twice: entries of the
// row may have the same class, whose shares each of them then adds up.
template <typename T>
__device__ __forceinline__ float entry(const Args<T>& g, const Row& r, const T* z, T* dz, const int* ids, const float* p,
                                       bool twice, float log_p, int j) {
  const int id = ids[j];
  if (id < 0) return 0.f;
  const float zi = Elem<T>::to_f(z[id]), pj = p[j];
  if (dz) {
    float same = twice ? 0.f : pj;
    if (twice)
      for (int i = 0; i < g.k; ++i) same += ids[i] == id ? p[i] : 0.f;
    float d = dense_any(g, r, zi) - g.alpha * g.tau * g.inv_rows * same;
    if (id == r.label) d -= (1.f - g.alpha) * g.inv_rows;
    dz[id] = Elem<T>::from_f(d);
  }
  return pj == 0.f ? 0.f : pj * (log_p - log_q(g, r, zi));
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

// Is (id, t) an entry of the teacher's?
template <typename T>
__device__ __forceinline__ bool is_entry(const Args<T>& g, int id, float t) {
  return id >= 0 && id < g.n && t != neg_inf();
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
    const bool ok = is_entry(g, id, t);
    ids[j] = ok ? id : -1;
    if (ok) hi = fmaxf(hi, t);
    any |= ok;
  }
  hi = group_max<kG>(hi);
  any = group_any<kG>(any, lane);
  float tot = 0.f;
  for (int j = gl; j < g.k; j += kG) {
    const float e = ids[j] < 0 ? 0.f : ex2((gt[j] - hi) * g.c);
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

// Marks the classes that have an entry, a bit each (class modulo the bits, a
// power of two or more than the classes).  Returns whether two entries have
// the same bit: with that question answered in k steps, the k^2 comparisons
// are left to rows that need them.
template <int kG>
__device__ __forceinline__ bool mark(const int* ids, int k, uint32_t* bits, int mask, int gl, int lane) {
  bool twice = false;
  for (int j = gl; j < k; j += kG) {
    const int id = ids[j];
    if (id < 0) continue;
    const uint32_t bit = 1u << (id & 31);
    twice |= (atomicOr(bits + ((id & mask) >> 5), bit) & bit) != 0;
  }
  twice = group_any<kG>(twice, lane);
  __syncwarp();
  return twice;
}

// f(the row's Hard as a constant)
template <typename F>
__device__ __forceinline__ void by_hard(int hard, F f) {
  switch (hard) {
    case kNone: f(std::integral_constant<int, kNone>()); break;
    case kPow1: f(std::integral_constant<int, kPow1>()); break;
    case kPow2: f(std::integral_constant<int, kPow2>()); break;
    case kPow4: f(std::integral_constant<int, kPow4>()); break;
    default: f(std::integral_constant<int, kOwn>()); break;
  }
}

// ---------------------------------------------- few classes: a thread a row
constexpr int kSmallRows = 128, kSmallN = 32;

template <typename T>
__global__ void __launch_bounds__(kSmallRows) k_distill_thread(const Args<T> g, uint32_t div) {
  extern __shared__ float buf[];
  const int n = g.n, ld = n | 1;   // an odd pitch: threads of a warp read different banks
  pdl_trigger();
  pdl_wait();
  const int64_t row0 = (int64_t)blockIdx.x * kSmallRows;
  const int rows = (int)min((int64_t)kSmallRows, g.all - row0), count = rows * n;
  const T* z = g.z + row0 * n;
  for (int i = threadIdx.x; i < count; i += kSmallRows)
    buf[n & 1 ? i : i + (int)(((uint32_t)i * div) >> 20)] = Elem<T>::to_f(z[i]);   // i + i / n
  __syncthreads();
  if ((int)threadIdx.x < rows) {
    float* v = buf + threadIdx.x * ld;
    const int64_t row = row0 + threadIdx.x, b = row % g.rows;
    const int32_t* gi = g.ids + b * g.k;
    const float* gt = g.top + b * g.k;
    const int label = label_of(g, b);
    // the teacher's maximum and sum
    float hi = neg_inf(), tot = 0.f;
    bool has = false;
    if (g.soft) {
      for (int j = 0; j < g.k; ++j)
        if (is_entry(g, gi[j], gt[j])) hi = fmaxf(hi, gt[j]), has = true;
      for (int j = 0; j < g.k; ++j)
        if (is_entry(g, gi[j], gt[j])) tot += ex2((gt[j] - hi) * g.c);
    }
    float zm = neg_inf();
    for (int i = 0; i < n; ++i) zm = fmaxf(zm, v[i]);
    float s = 0.f, s1 = 0.f;
    if (zm == neg_inf()) {   // nothing but -inf, or a NaN, which has to reach the sums
      for (int i = 0; i < n; ++i)
        if (v[i] != v[i]) s = s1 = v[i];
    } else {
      by_hard(g.hard, [&](auto h) {
        for (int i = 0; i < n; ++i) {
          const float e = ex2((v[i] - zm) * g.c);
          s += e;
          if (h.value == kOwn) s1 += ex2((v[i] - zm) * kLog2e);
          else if (h.value != kNone) s1 += pow_tau<h.value>(e);
        }
      });
    }
    const Row r = make_row(g, zm, true, s, s1, has, label);
    float kd = 0.f;
    const float inv = 1.f / tot, log_tot = logf(tot);
    if (has && r.alive)
      for (int j = 0; j < g.k; ++j) {
        const int id = gi[j];
        const float t = gt[j];
        if (!is_entry(g, id, t)) continue;
        const float p = ex2((t - hi) * g.c) * inv;
        if (p != 0.f) kd += p * ((t - hi) * (g.c * kLn2) - log_tot - log_q(g, r, v[id]));
      }
    g.row_loss[row] = row_loss(g, r, has, kd, r.label >= 0 ? v[r.label] : 0.f);
    if (g.dz) {
      by_hard(g.hard, [&](auto h) {
        for (int i = 0; i < n; ++i) v[i] = dense<h.value>(g.c, r, v[i]);
      });
      if (has && r.alive)
        for (int j = 0; j < g.k; ++j) {
          const int id = gi[j];
          if (is_entry(g, id, gt[j])) v[id] -= g.alpha * g.tau * g.inv_rows * (ex2((gt[j] - hi) * g.c) * inv);
        }
      if (r.label >= 0) v[r.label] -= (1.f - g.alpha) * g.inv_rows;
    }
  }
  if (g.dz == nullptr) return;
  __syncthreads();
  T* dz = g.dz + row0 * n;
  for (int i = threadIdx.x; i < count; i += kSmallRows)
    dz[i] = Elem<T>::from_f(buf[n & 1 ? i : i + (int)(((uint32_t)i * div) >> 20)]);
}

// --------------------------------------------- up to 1024: a group of lanes
template <typename T, int kG, int kV>
__global__ void __launch_bounds__(256) k_distill_group(const Args<T> g) {
  extern __shared__ uint8_t raw[];
  constexpr int kGroups = 256 / kG;
  const int lane = threadIdx.x & 31, gl = threadIdx.x & (kG - 1), grp = threadIdx.x / kG;
  int* ids = (int*)raw + grp * g.k;
  float* p = (float*)raw + (kGroups + grp) * g.k;
  constexpr int kWords = kG * kV / 32;
  uint32_t* bits = (uint32_t*)raw + 2 * kGroups * g.k + grp * kWords;
  for (int i = gl; i < kWords; i += kG) bits[i] = 0;
  pdl_trigger();
  pdl_wait();
  const int64_t rr = (int64_t)blockIdx.x * kGroups + grp;
  const bool live = rr < g.all;
  const int64_t row = live ? rr : g.all - 1, b = row % g.rows;   // lanes past the last row go along with it
  const T* z = g.z + row * g.n;
  float v[kV];
  float zm = neg_inf();
#pragma unroll
  for (int i = 0; i < kV; ++i) {
    const int c = gl + kG * i;
    v[i] = c < g.n ? Elem<T>::to_f(z[c]) : neg_inf();
  }
  float hi = 0.f, log_tot = 0.f;
  const bool has = g.soft && teacher<T, kG>(g, b, gl, lane, ids, p, hi, log_tot);
  const bool twice = g.soft && g.dz && mark<kG>(ids, g.k, bits, ~0, gl, lane);
  const int label = label_of(g, b);
#pragma unroll
  for (int i = 0; i < kV; ++i) zm = fmaxf(zm, v[i]);
  zm = group_max<kG>(zm);
  float s = 0.f, s1 = 0.f;
  if (zm == neg_inf()) {   // nothing but -inf, or a NaN, which has to reach the sums
#pragma unroll
    for (int i = 0; i < kV; ++i)
      if (v[i] != v[i]) s = s1 = v[i];
  } else {
    by_hard(g.hard, [&](auto h) {
#pragma unroll
      for (int i = 0; i < kV; ++i) {
        const float e = ex2((v[i] - zm) * g.c);
        s += e;
        if (h.value == kOwn) s1 += ex2((v[i] - zm) * kLog2e);
        else if (h.value != kNone) s1 += pow_tau<h.value>(e);
      }
    });
  }
  s = group_sum<kG>(s);
  s1 = group_sum<kG>(s1);
  const Row r = make_row(g, zm, true, s, s1, has, label);
  T* dz = g.dz && live ? g.dz + row * g.n : nullptr;
  if (dz) {
    by_hard(g.hard, [&](auto h) {
#pragma unroll
      for (int i = 0; i < kV; ++i) {
        const int c = gl + kG * i;
        if (c < g.n) dz[c] = Elem<T>::from_f(dense<h.value>(g.c, r, v[i]));
      }
    });
  }
  __syncwarp();
  float kd = 0.f;
  if (has && r.alive)
    for (int j = gl; j < g.k; j += kG)
      kd += entry(g, r, z, dz, ids, p, twice, (g.top[b * g.k + j] - hi) * (g.c * kLn2) - log_tot, j);
  kd = group_sum<kG>(kd);
  if (gl == 0) {
    const float zl = r.label >= 0 ? Elem<T>::to_f(z[r.label]) : 0.f;
    if (dz && r.label >= 0 && !(has && (bits[r.label >> 5] >> (r.label & 31) & 1)))   // a label no entry has
      dz[r.label] = Elem<T>::from_f(dense_any(g, r, zl) - (1.f - g.alpha) * g.inv_rows);
    if (live) g.row_loss[row] = row_loss(g, r, has, kd, zl);
  }
}

// ------------------------------------------------- many classes: a block a row
constexpr int kMarks = 32768;   // bits for classes that have an entry
constexpr int kTurn = 4;   // 16-byte groups that a thread asks for at a time

template <typename T>
struct Vec;   // 16 bytes of T
template <>
struct Vec<float> {
  static constexpr int kN = 4;
  static __device__ __forceinline__ uint4 none() { return make_uint4(0xFF800000u, 0xFF800000u, 0xFF800000u, 0xFF800000u); }
  static __device__ __forceinline__ float top(const uint4& u) {
    return fmaxf(fmaxf(__uint_as_float(u.x), __uint_as_float(u.y)), fmaxf(__uint_as_float(u.z), __uint_as_float(u.w)));
  }
  static __device__ __forceinline__ void get(const uint4& u, float (&v)[4]) {
    v[0] = __uint_as_float(u.x), v[1] = __uint_as_float(u.y), v[2] = __uint_as_float(u.z), v[3] = __uint_as_float(u.w);
  }
  static __device__ __forceinline__ uint4 put(const float (&v)[4]) {
    return make_uint4(__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3]));
  }
};
template <>
struct Vec<__nv_bfloat16> {
  static constexpr int kN = 8;
  static __device__ __forceinline__ uint4 none() { return make_uint4(0xFF80FF80u, 0xFF80FF80u, 0xFF80FF80u, 0xFF80FF80u); }
  static __device__ __forceinline__ __nv_bfloat162 h2(uint32_t u) { return *reinterpret_cast<__nv_bfloat162*>(&u); }
  static __device__ __forceinline__ float top(const uint4& u) {
    const __nv_bfloat162 m = __hmax2(__hmax2(h2(u.x), h2(u.y)), __hmax2(h2(u.z), h2(u.w)));
    return fmaxf(__low2float(m), __high2float(m));
  }
  static __device__ __forceinline__ void get(const uint4& u, float (&v)[8]) {
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int e = 0; e < 4; ++e) v[2 * e] = __uint_as_float(w[e] << 16), v[2 * e + 1] = __uint_as_float(w[e] & 0xFFFF0000u);
  }
  static __device__ __forceinline__ uint4 put(const float (&v)[8]) {
    uint32_t w[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const __nv_bfloat162 h = __floats2bfloat162_rn(v[2 * e], v[2 * e + 1]);
      w[e] = *reinterpret_cast<const uint32_t*>(&h);
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
  }
};

// 2^(v c - o) of two classes, or 2^((v - o) c), o then being the maximum itself
template <bool kFar>
__device__ __forceinline__ float2 exp2_of(float2 v, float o, float c) {
  const float2 t = kFar ? __fmul2_rn(__fadd2_rn(v, make_float2(-o, -o)), make_float2(c, c))
                        : __ffma2_rn(v, make_float2(c, c), make_float2(-o, -o));
  return make_float2(ex2(t.x), ex2(t.y));
}
template <int kHard, bool kFar>
__device__ __forceinline__ float2 dense2(float c, const Row& r, float2 v) {
  const float2 e = exp2_of<kFar>(v, kFar ? r.zm : r.o, c);
  const float2 ca = make_float2(r.ca, r.ca), c1 = make_float2(r.c1, r.c1);
  if (kHard == kNone) return __fmul2_rn(e, ca);
  if (kHard == kPow1) return __fmul2_rn(e, __fadd2_rn(ca, c1));
  if (kHard == kPow2) return __fmul2_rn(e, __ffma2_rn(c1, e, ca));
  if (kHard == kPow4) return __fmul2_rn(e, __ffma2_rn(__fmul2_rn(c1, e), __fmul2_rn(e, e), ca));
  return __ffma2_rn(ca, e, __fmul2_rn(c1, exp2_of<kFar>(v, kFar ? r.zm : r.o1, kLog2e)));
}

// m c rounded (not folded into a multiply-add, which would be another offset)
// and kept finite, so that two equal ones differ by 0.
__device__ __forceinline__ float offset(float m, float c) {
  return fminf(fmaxf(__fmul_rn(m, c), -3.402823466e38f), 3.402823466e38f);
}

// A thread's running maximum m, the offsets its exponents were taken with, and
// its sums (of even and odd classes).
template <int kHard, bool kFar>
struct Running {
  float m = neg_inf(), o = neg_inf(), o1 = neg_inf();
  float2 s{0.f, 0.f}, s1{0.f, 0.f};
  __device__ __forceinline__ void raise(float top, float c) {
    if (!(top > m)) return;
    m = top;
    const float to = kFar ? m : offset(m, c), to1 = kFar ? m : offset(m, kLog2e);
    const float f = ex2(kFar ? (o - to) * c : o - to);   // 0 at first
    const float f1 = kHard == kOwn ? ex2(kFar ? (o1 - to1) * kLog2e : o1 - to1) : pow_tau<kHard>(f);
    s = __fmul2_rn(s, make_float2(f, f));
    s1 = __fmul2_rn(s1, make_float2(f1, f1));
    o = to, o1 = to1;
  }
  __device__ __forceinline__ void add(float2 v, float c) {
    const float2 e = exp2_of<kFar>(v, o, c);
    s = __fadd2_rn(s, e);
    if (kHard == kOwn) s1 = __fadd2_rn(s1, exp2_of<kFar>(v, o1, kLog2e));
    else if (kHard == kPow2) s1 = __ffma2_rn(e, e, s1);
    else if (kHard == kPow4) s1 = __ffma2_rn(__fmul2_rn(e, e), __fmul2_rn(e, e), s1);
    else if (kHard == kPow1) s1 = s;
  }
  __device__ __forceinline__ void only_nan(float v) {
    if (v != v) s.x = s1.x = v;
  }
};

// |zm c| from which on a row is far: below, the product's rounding is less than 2^3
constexpr float kFarPower = 67108864.f;
// Of temperatures further than this from 1 every row is far: a gap of 2^26 in
// the larger of the two exponents (see nothing()) leaves at least 2^8 in the
// other one up to here, and may leave less beyond.
constexpr float kFarTau = 262144.f;

// A row's 16-byte groups and the single classes at its ends.
template <typename T>
struct Span {
  const T* z;
  const uint4* zv;
  int head, body, single;
  bool mine;
  __device__ __forceinline__ Span(const T* p, int n, int tid) : z(p) {
    constexpr int kN = Vec<T>::kN;
    head = min(n, (int)((16 - ((uintptr_t)z & 15)) & 15) / (int)sizeof(T));
    body = (n - head) / kN;
    const int tail = head + body * kN;
    zv = reinterpret_cast<const uint4*>(z + head);
    single = tid < head ? tid : tail + tid - head;   // at most 2 (kN - 1) of them
    mine = single < n;
  }
};

// sums of the offset of maximum m brought to that of maximum `to`
template <int kHard, bool kFar>
__device__ __forceinline__ void bring(float& s, float& s1, float m, float to, float c) {
  if (to == neg_inf()) return;   // no class above -inf: 0 or NaN as it is
  const float f = ex2(kFar ? (m - to) * c : offset(m, c) - offset(to, c));
  s *= f;
  s1 *= kHard == kOwn ? ex2(kFar ? (m - to) * kLog2e : offset(m, kLog2e) - offset(to, kLog2e)) : pow_tau<kHard>(f);
}

// What a thread sees while its maximum is -inf, or twice as far out as a row
// that is not far may lie, counts only if it is NaN: either the row's own
// maximum is 2^26 or more above it in the larger of the two exponents, so that
// it adds 0 to both sums (see kFarTau), or the row is far and the sums are taken
// again.
template <int kHard, bool kFar>
__device__ __forceinline__ bool nothing(const Running<kHard, kFar>& q, float c) {
  return kFar ? q.m == neg_inf() : !(fabsf(q.m) * fmaxf(c, kLog2e) < 2.f * kFarPower);
}
// (out of line: predicated into the loop, its comparisons were a quarter of it)
template <typename T>
__device__ __noinline__ float find_nan(uint4 u) {
  using V = Vec<T>;
  float v[V::kN], s = 0.f;
  V::get(u, v);
#pragma unroll
  for (int e = 0; e < V::kN; ++e) s = v[e] != v[e] ? v[e] : s;
  return s;
}
// kCount groups of a thread into its sums.
template <typename T, int kHard, bool kFar, int kCount>
__device__ __forceinline__ void take(Running<kHard, kFar>& q, const uint4 (&u)[kCount], float c) {
  using V = Vec<T>;
  float top = V::top(u[0]);
#pragma unroll
  for (int k = 1; k < kCount; ++k) top = fmaxf(top, V::top(u[k]));
  q.raise(top, c);
  if (nothing(q, c)) {
#pragma unroll
    for (int k = 0; k < kCount; ++k) q.only_nan(find_nan<T>(u[k]));
    return;
  }
#pragma unroll
  for (int k = 0; k < kCount; ++k) {
    float v[V::kN];
    V::get(u[k], v);
#pragma unroll
    for (int e = 0; e < V::kN; e += 2) q.add(make_float2(v[e], v[e + 1]), c);
  }
}
// A warp's maximum and sums: the thread's single class, then the lanes joined.
template <typename T, int kHard, bool kFar, int kWarps>
__device__ __forceinline__ void finish(Running<kHard, kFar>& q, const Span<T>& sp, float c, float (*red)[kWarps]) {
  if (sp.mine) {
    const float v = Elem<T>::to_f(sp.z[sp.single]);
    q.raise(v, c);
    if (nothing(q, c)) q.only_nan(v);
    else q.add(make_float2(v, neg_inf()), c);
  }
  float s = q.s.x + q.s.y, s1 = q.s1.x + q.s1.y;
  const float wm = group_max<32>(q.m);
  bring<kHard, kFar>(s, s1, q.m, wm, c);
  s = group_sum<32>(s);
  s1 = group_sum<32>(s1);
  if ((threadIdx.x & 31) == 0) {
    const int w = threadIdx.x >> 5;
    red[0][w] = wm, red[1][w] = s, red[2][w] = s1;
  }
}
struct Sums { float zm, s, s1; };
template <int kHard, bool kFar, int kWarps>
__device__ __forceinline__ Sums row_join(float c, const float (*red)[kWarps]) {
  Sums t{neg_inf(), 0.f, 0.f};
#pragma unroll
  for (int k = 0; k < kWarps; ++k) t.zm = fmaxf(t.zm, red[0][k]);
#pragma unroll 4
  for (int k = 0; k < kWarps; ++k) {
    float a = red[1][k], a1 = red[2][k];
    bring<kHard, kFar>(a, a1, red[0][k], t.zm, c);
    t.s += a;
    t.s1 += a1;
  }
  return t;
}

// A row's sums by kWarps warps.
template <typename T, int kHard, bool kFar, int kWarps>
__device__ __forceinline__ void row_part(const Span<T>& sp, float c, float (*red)[kWarps]) {
  constexpr int kThreads = 32 * kWarps;
  Running<kHard, kFar> q;
  int i = threadIdx.x;
  for (; i + (kTurn - 1) * kThreads < sp.body; i += kTurn * kThreads) {
    uint4 u[kTurn];
#pragma unroll
    for (int k = 0; k < kTurn; ++k) u[k] = sp.zv[i + k * kThreads];
    take<T, kHard, kFar, kTurn>(q, u, c);
  }
  // the last turn: at once, past the row's end -inf, which adds 0; group by group in a row of many turns, which
  // wants the registers (2048 rows of 50021 bf16: 80 us, at once 81.6; 16384 of 4000: 95 us, at once 82)
  if constexpr (kWarps <= 4) {
    if (i < sp.body) {
      uint4 u[kTurn];
#pragma unroll
      for (int k = 0; k < kTurn; ++k) u[k] = i + k * kThreads < sp.body ? sp.zv[i + k * kThreads] : Vec<T>::none();
      take<T, kHard, kFar, kTurn>(q, u, c);
    }
  } else {
    for (; i < sp.body; i += kThreads) {
      const uint4 u[1] = {sp.zv[i]};
      take<T, kHard, kFar, 1>(q, u, c);
    }
  }
  finish<T, kHard, kFar, kWarps>(q, sp, c, red);
}

// A row's dense gradient by kWarps warps; kSame: dz lies as z does in its
// 16-byte groups.
template <typename T, int kHard, bool kFar, bool kSame, int kWarps>
__device__ __forceinline__ void row_dense(const Span<T>& sp, float c, const Row& r, T* dz) {
  using V = Vec<T>;
  constexpr int kN = V::kN, kThreads = 32 * kWarps;
  auto put = [&](int at, const uint4& u) {
    float v[kN];
    V::get(u, v);
#pragma unroll
    for (int e = 0; e < kN; e += 2) {
      const float2 d = dense2<kHard, kFar>(c, r, make_float2(v[e], v[e + 1]));
      v[e] = d.x, v[e + 1] = d.y;
    }
    if constexpr (kSame) {
      reinterpret_cast<uint4*>(dz + sp.head)[at] = V::put(v);
    } else {
#pragma unroll
      for (int e = 0; e < kN; ++e) dz[sp.head + at * kN + e] = Elem<T>::from_f(v[e]);
    }
  };
  int i = threadIdx.x;
  for (; i + (kTurn - 1) * kThreads < sp.body; i += kTurn * kThreads) {
    uint4 u[kTurn];
#pragma unroll
    for (int k = 0; k < kTurn; ++k) u[k] = sp.zv[i + k * kThreads];
#pragma unroll
    for (int k = 0; k < kTurn; ++k) put(i + k * kThreads, u[k]);
  }
  if constexpr (kWarps <= 4) {   // (as in row_part)
    if (i < sp.body) {
      uint4 u[kTurn];
#pragma unroll
      for (int k = 0; k < kTurn; ++k) u[k] = i + k * kThreads < sp.body ? sp.zv[i + k * kThreads] : V::none();
#pragma unroll
      for (int k = 0; k < kTurn; ++k)
        if (i + k * kThreads < sp.body) put(i + k * kThreads, u[k]);
    }
  } else {
    for (; i < sp.body; i += kThreads) put(i, sp.zv[i]);
  }
  if (sp.mine) dz[sp.single] = Elem<T>::from_f(dense<kHard>(c, r, Elem<T>::to_f(sp.z[sp.single])));
}

// kWarps warps take the classes; one more works out the teacher's distribution
// while they take the sums, and the entries' gradients and the loss while they
// write the dense part; its values go over theirs after the last barrier.
template <typename T, int kHard, int kWarps>
__global__ void __launch_bounds__(32 * kWarps + 32, kWarps > 4 ? 3 : 32 / kWarps) k_distill_row(const Args<T> g) {
  constexpr int kPer = kMaxK / 32;   // entries of a lane
  __shared__ int ids[kMaxK];
  __shared__ float p[kMaxK];
  __shared__ float red[2][3][kWarps];
  __shared__ uint32_t bits[kMarks / 32];   // (of the extra warp)
  __shared__ int has_s;
  const int lane = threadIdx.x & 31;
  const bool extra = threadIdx.x >= 32 * kWarps;
  pdl_trigger();
  pdl_wait();
  const int64_t row = blockIdx.x, b = row % g.rows;
  const T* z = g.z + row * g.n;
  T* dz = g.dz ? g.dz + row * g.n : nullptr;
  const int label = label_of(g, b);
  const Span<T> sp(z, g.n, threadIdx.x);
  float hi = 0.f, log_tot = 0.f, z_entry[kPer], z_label = 0.f;
  bool twice = true;
  if (extra) {
    bool any = false;
    const bool marks = dz && g.k > 16;   // fewer entries are compared as fast
    if (marks)
      for (int i = lane; 32 * i < min(g.n, kMarks); i += 32) bits[i] = 0;
    if (g.soft) any = teacher<T, 32>(g, b, lane, lane, ids, p, hi, log_tot);
    if (marks && g.soft) twice = mark<32>(ids, g.k, bits, kMarks - 1, lane, lane);
    if (lane == 0) has_s = any;
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      const int j = lane + 32 * i;
      z_entry[i] = any && j < g.k && ids[j] >= 0 ? Elem<T>::to_f(z[ids[j]]) : 0.f;
    }
    if (label >= 0) z_label = Elem<T>::to_f(z[label]);
  } else {
    row_part<T, kHard, false, kWarps>(sp, g.c, red[0]);
  }
  __syncthreads();
  Sums a = row_join<kHard, false, kWarps>(g.c, red[0]);
  const float wide = fmaxf(g.c, kLog2e), narrow = fminf(g.c, kLog2e);
  // (an infinite maximum: NaN either way)
  const bool far = (fabsf(a.zm) * wide >= kFarPower || wide > kFarTau * narrow) && a.zm != neg_inf();
  if (far) {
    if (!extra) row_part<T, kHard, true, kWarps>(sp, g.c, red[1]);
    __syncthreads();
    a = row_join<kHard, true, kWarps>(g.c, red[1]);
  }
  const bool has = has_s;
  const Row r = make_row(g, a.zm, far, a.s, a.s1, has, label);
  if (!extra) {
    if (dz == nullptr) return;
    const bool same = (((uintptr_t)z ^ (uintptr_t)dz) & 15) == 0;
    if (far) row_dense<T, kHard, true, false, kWarps>(sp, g.c, r, dz);
    else if (same) row_dense<T, kHard, false, true, kWarps>(sp, g.c, r, dz);
    else row_dense<T, kHard, false, false, kWarps>(sp, g.c, r, dz);
    __syncthreads();
    return;
  }
  // the entries' gradients and the loss, while the dense part is written
  float d_entry[kPer], d_label = 0.f, kd = 0.f;
  const float ones = (1.f - g.alpha) * g.inv_rows;
  bool found = false;
#pragma unroll
  for (int i = 0; i < kPer; ++i) {
    const int j = lane + 32 * i, id = has && r.alive && j < g.k ? ids[j] : -1;
    d_entry[i] = 0.f;
    if (id < 0) continue;
    float same = twice ? 0.f : p[j];
    if (dz && twice)
      for (int q = 0; q < g.k; ++q) same += ids[q] == id ? p[q] : 0.f;
    d_entry[i] = dense<kHard>(g.c, r, z_entry[i]) - g.alpha * g.tau * g.inv_rows * same;
    if (id == r.label) d_entry[i] -= ones, found = true;
    if (p[j] != 0.f)
      kd += p[j] * ((g.top[b * g.k + j] - hi) * (g.c * kLn2) - log_tot - log_q(g, r, z_entry[i]));
  }
  const bool label_apart = !__any_sync(0xffffffffu, found) && r.label >= 0;
  if (label_apart) d_label = dense<kHard>(g.c, r, z_label) - ones;
  kd = group_sum<32>(kd);
  if (lane == 0) g.row_loss[row] = row_loss(g, r, has, kd, z_label);
  if (dz == nullptr) return;
  __syncthreads();   // over the dense part
#pragma unroll
  for (int i = 0; i < kPer; ++i) {
    const int j = lane + 32 * i;
    if (has && r.alive && j < g.k && ids[j] >= 0) dz[ids[j]] = Elem<T>::from_f(d_entry[i]);
  }
  if (label_apart && lane == 0) dz[r.label] = Elem<T>::from_f(d_label);
}

// A student's mean over its rows, in a fixed order: 256 to 1024 threads with four
// loads in flight (a whole call of 100000 rows, 256 threads: 55 us; 1024: 37).
__global__ void __launch_bounds__(1024) k_distill_mean(const float* row_loss, int64_t rows, float* loss) {
  __shared__ float s[32];
  pdl_trigger();
  pdl_wait();
  const float* p = row_loss + blockIdx.x * rows;
  float a = 0.f;
#pragma unroll 4
  for (int64_t i = threadIdx.x; i < rows; i += blockDim.x) a += p[i];
  a = group_sum<32>(a);
  if ((threadIdx.x & 31) == 0) s[threadIdx.x >> 5] = a;
  __syncthreads();
  if (threadIdx.x < 32) {
    a = group_sum<32>(32 * threadIdx.x < blockDim.x ? s[threadIdx.x] : 0.f);   // (warps that there are)
    if (threadIdx.x == 0) loss[blockIdx.x] = a / (float)rows;
  }
}

template <typename T, int kG, int kV>
void group(const Args<T>& a, cudaStream_t st) {
  launch_pdl(k_distill_group<T, kG, kV>, dim3((unsigned)ceil_div(a.all, 256 / kG)), dim3(256),
             (size_t)(256 / kG) * (a.k * 8 + kG * kV / 8), st, a);
}

template <typename T, int kWarps>
void wide(const Args<T>& a, cudaStream_t st) {
  const dim3 grid((unsigned)a.all), block(32 * kWarps + 32);
  if (a.hard == kNone) launch_pdl(k_distill_row<T, kNone, kWarps>, grid, block, 0, st, a);
  else if (a.hard == kPow1) launch_pdl(k_distill_row<T, kPow1, kWarps>, grid, block, 0, st, a);
  else if (a.hard == kPow2) launch_pdl(k_distill_row<T, kPow2, kWarps>, grid, block, 0, st, a);
  else if (a.hard == kPow4) launch_pdl(k_distill_row<T, kPow4, kWarps>, grid, block, 0, st, a);
  else launch_pdl(k_distill_row<T, kOwn, kWarps>, grid, block, 0, st, a);
}

template <typename T>
cudaError_t rows(const Args<T>& a, cudaStream_t st) {
  // Launches of many rows want few lanes a row, launches of few rows short
  // chains a lane (a whole call, us, bf16 / fp32; the other way in brackets):
  //   10 classes, 80000 rows: 8 entries, a thread 21.7 / 21.1 (eight lanes 24.5 / 24.0), 2 entries 15.1 / 14.9
  //   (24.7 / 24.2); 32 classes, 16 entries: eight lanes 27.7 / 27.2 (a thread 66.9 / 66.5); 10 classes, 8 entries,
  //   4096 rows: eight lanes 5.3 / 5.1 (a thread 8.6 / 8.4), 24000 rows 9.6 / 9.4 (10.8 / 10.7)
  //   64 classes, 80000 rows: eight lanes 26.7 / 26.0 (sixteen 38.6 / 37.8)
  //   128, 80000 rows: sixteen 41.8 / 41.5 (thirty-two 64.7 / 64.2; eight would take 32.5 / 31.5), 4096 rows 6.5 / 6.5
  //   (8.2 / 8.1)
  //   256, 80000 rows: sixteen 53.0 / 55.4 (thirty-two 73.2 / 76.0), 128 rows: thirty-two 5.2 / 4.9 (5.5 / 5.1)
  //   512, 80000 rows: sixteen 85.2 / 73.6 (thirty-two 108 / 96.7), 128 rows: thirty-two 5.5 / 5.1 (6.5 / 5.7)
  //   1000, 16384 rows: a warp 28.5 / 32.3 (a block 36.9 / 38.8), 128 rows: a block 4.8 / 5.1 (6.6 / 5.9)
  const bool few = a.all <= 4096;
  if (a.n <= kSmallN && a.k <= 8 && a.all > 24576) {
    const uint32_t div = ((1u << 20) + a.n - 1) / a.n;   // i / n = i div >> 20 for i < 128 * 32
    launch_pdl(k_distill_thread<T>, dim3((unsigned)ceil_div(a.all, kSmallRows)), dim3(kSmallRows),
               (size_t)kSmallRows * (a.n | 1) * 4, st, a, div);
  } else if (a.n <= 32) {
    group<T, 8, 4>(a, st);
  } else if (a.n <= 64) {
    group<T, 8, 8>(a, st);
  } else if (a.n <= 128) {
    group<T, 16, 8>(a, st);
  } else if (a.n <= 256) {
    if (few) group<T, 32, 8>(a, st);
    else group<T, 16, 16>(a, st);
  } else if (a.n <= 512) {
    if (few) group<T, 32, 16>(a, st);
    else group<T, 16, 32>(a, st);
  } else if (a.n <= 1024 && a.all > 1024) {
    group<T, 32, 32>(a, st);
  } else if (a.n * (int64_t)sizeof(T) <= 16384) {
    // two warps a row: 16384 rows of 2000, bf16 48 us (four 68), fp32 57 (71); of 4000, 65 (82), 95 (101)
    wide<T, 2>(a, st);
  } else if (a.n * (int64_t)sizeof(T) <= 32768) {
    // four: 16384 rows of 16000 bf16, 182 us (two 230, fifteen 264); fp32, by fifteen, 349 us (four 433)
    wide<T, 4>(a, st);
  } else {
    wide<T, 15>(a, st);
  }
  return cudaGetLastError();
}

tp_status check(int64_t m, int64_t rows) {
  if (m < 1 || m > 65535 || rows < 0 || rows > (int64_t(1) << 31) / m - 1)
    return ops_fail(TP_EINVAL, "m %lld (1..65535) students of %lld rows: fewer than 2^31 rows in all are taken",
                    (long long)m, (long long)rows);
  return TP_OK;
}

}  // namespace
}  // namespace tp

using namespace tp;

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
  if (n < 2 || n > kMaxN) return ops_fail(TP_EINVAL, "n %d must be in 2..%d", n, kMaxN);
  if (k < 1 || k > kMaxK) return ops_fail(TP_EINVAL, "k %d must be in 1..%d", k, kMaxK);
  if (!(tau >= kMinTau && tau <= 1.f / kMinTau)) return ops_fail(TP_EINVAL, "tau must be in 2^-60..2^60");
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
    const int soft = alpha > 0.f;
    const int hard = !(alpha < 1.f && labels) ? kNone : tau == 1.f ? kPow1 : tau == 2.f ? kPow2 : tau == 4.f ? kPow4 : kOwn;
    const float c = kLog2e / tau;
    if (precision == TP_FP32)
      e = rows(Args<float>{(const float*)z, ids, labels, top, (float*)dz, rl, m * n_rows, n_rows, n, k, soft, hard, c, tau,
                       alpha, 1.f / (float)n_rows}, st);
    else
      e = rows(Args<__nv_bfloat16>{(const __nv_bfloat16*)z, ids, labels, top, (__nv_bfloat16*)dz, rl, m * n_rows, n_rows, n, k,
                               soft, hard, c, tau, alpha, 1.f / (float)n_rows}, st);
    if (e == cudaSuccess) {
      const int64_t threads = std::min<int64_t>(1024, std::max<int64_t>(256, round_up(ceil_div(n_rows, 4), 32)));
      launch_pdl(k_distill_mean, dim3((unsigned)m), dim3((unsigned)threads), 0, st, (const float*)rl, n_rows, loss);
      e = cudaGetLastError();
    }
  }
  if (e == cudaSuccess) return TP_OK;
  cudaGetLastError();   // reported here
  return ops_fail(TP_ECUDA, "pack_distill: %s", cudaGetErrorString(e));
}

}  // extern "C"
