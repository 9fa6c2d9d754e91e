// distill.cu -- distillation of m students from one teacher's top logits:
// loss and gradient in one call (entry points in tabpack_ops.h).
//
// Per row, with zm = max z, c = log2(e) / tau, e_i = 2^((z_i - zm) c), S = sum
// e_i, and e1_i, S1 likewise for tau = 1, and the teacher's p:
//   log softmax(z / tau)_i = ((z_i - zm) c - log2 S) / log2(e)
//   kd = tau^2 sum_j p_j (log p_j - log softmax(z / tau)[id_j])
//   dz = [alpha tau (e / S - p) + (1 - alpha) (e1 / S1 - onehot)] / rows
// (The difference is taken first: z_i c - zm c in one multiply-add would be off
// by zm c's rounding, whose power of two overflows for a row that a mask left
// at -10^10 or at the type's lowest value.)  For tau = 1, 2 and 4 e1 is the first, second or fourth power of e, so that a
// class costs one exponential a pass.
//
// The gradient's dense part is written for every class; then, after a barrier
// of the row's threads, the thread of each entry writes the whole value at
// its class (summing the entries of the same class itself), and one thread
// that at the label, if no entry has it: no value is added to in memory and
// the result does not depend on any order.
//
// Bound by HBM (z read, dz written) for many classes, by latency for few.
//   up to 32 classes    a thread takes a row, which blocks of 128 rows stage in
//                       shared memory: no exchanges between lanes at all
//   up to 1024          16 or 32 lanes hold a row in registers
//   above               a block takes a row: running maximum and sums in one
//                       pass, the gradient in a second that finds the row in
//                       L2; four 16-byte groups per thread and turn, one
//                       comparison of maxima for each turn
#include <algorithm>
#include <type_traits>

#include "prod.cuh"

using namespace tp;

namespace {

constexpr int kMaxK = 128;
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
  float zm;
  float log_s, log_s1;        // base 2
  float ca, c1;               // alpha tau / (S rows), 0 without a teacher; (1 - alpha) / (S1 rows), 0 without a label
  int label;                  // -1: none
  bool alive;                 // a class above -inf (or NaN)
};

// (all -inf: zm = -inf, s = 0)
template <typename T>
__device__ __forceinline__ Row make_row(const Args<T>& g, float zm, float s, float s1, bool has, int label) {
  Row r;
  r.alive = !(zm == neg_inf() && s == 0.f);
  r.zm = r.alive ? zm : 0.f;
  r.log_s = log2f(s);
  r.log_s1 = log2f(s1);
  r.ca = has && r.alive ? g.alpha * g.tau * g.inv_rows / s : 0.f;
  r.c1 = label >= 0 && r.alive ? (1.f - g.alpha) * g.inv_rows / s1 : 0.f;
  r.label = r.alive ? label : -1;
  return r;
}

// The dense part of the gradient at a class of logit z.
template <int kHard>
__device__ __forceinline__ float dense(float c, const Row& r, float z) {
  const float e = ex2((z - r.zm) * c);
  if (kHard == kNone) return e * r.ca;
  if (kHard == kPow1) return e * (r.ca + r.c1);
  if (kHard == kPow2) return e * fmaf(r.c1, e, r.ca);
  if (kHard == kPow4) return e * fmaf(r.c1 * e, e * e, r.ca);
  return fmaf(r.ca, e, r.c1 * ex2((z - r.zm) * kLog2e));
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
  return ((z - r.zm) * g.c - r.log_s) * kLn2;
}
template <typename T>
__device__ __forceinline__ float cross_entropy(const Args<T>& g, const Row& r, float z) {
  return (r.log_s1 - (z - r.zm) * kLog2e) * kLn2;
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

// Entry j's share of kd / tau^2; its class's gradient, and by the first entry's
// thread that of a label no entry has.
template <typename T>
__device__ __forceinline__ float entry(const Args<T>& g, const Row& r, const T* z, T* dz, const int* ids, const float* p,
                                       float log_p, int j) {
  const int id = ids[j];
  if (id < 0) return 0.f;
  const float zi = Elem<T>::to_f(z[id]), pj = p[j];
  if (dz) {
    float same = 0.f;
    for (int i = 0; i < g.k; ++i) same += ids[i] == id ? p[i] : 0.f;
    float d = dense_any(g, r, zi) - g.alpha * g.tau * g.inv_rows * same;
    if (id == r.label) d -= (1.f - g.alpha) * g.inv_rows;
    dz[id] = Elem<T>::from_f(d);
  }
  return pj == 0.f ? 0.f : pj * (log_p - log_q(g, r, zi));
}
template <typename T>
__device__ __forceinline__ void label_entry(const Args<T>& g, const Row& r, const T* z, T* dz, const int* ids, bool has) {
  if (dz == nullptr || r.label < 0) return;
  if (has)
    for (int i = 0; i < g.k; ++i)
      if (ids[i] == r.label) return;
  dz[r.label] = Elem<T>::from_f(dense_any(g, r, Elem<T>::to_f(z[r.label])) - (1.f - g.alpha) * g.inv_rows);
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
    const Row r = make_row(g, zm, s, s1, has, label);
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
  const Row r = make_row(g, zm, s, s1, has, label);
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
      kd += entry(g, r, z, dz, ids, p, (g.top[b * g.k + j] - hi) * (g.c * kLn2) - log_tot, j);
  kd = group_sum<kG>(kd);
  if (gl == 0) {
    label_entry(g, r, z, dz, ids, has);
    if (live) g.row_loss[row] = row_loss(g, r, has, kd, r.label >= 0 ? Elem<T>::to_f(z[r.label]) : 0.f);
  }
}

// ------------------------------------------------- many classes: a block a row
constexpr int kRowThreads = 512, kTurn = 4;

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

// Two fp32 operations in one instruction.
struct F2 { float x, y; };
__device__ __forceinline__ uint64_t pack2(F2 a) {
  uint64_t r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a.x), "f"(a.y));
  return r;
}
__device__ __forceinline__ F2 unpack2(uint64_t v) {
  F2 r;
  asm("mov.b64 {%0, %1}, %2;" : "=f"(r.x), "=f"(r.y) : "l"(v));
  return r;
}
__device__ __forceinline__ F2 add2(F2 a, F2 b) {
  uint64_t r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(pack2(a)), "l"(pack2(b)));
  return unpack2(r);
}
__device__ __forceinline__ F2 mul2(F2 a, F2 b) {
  uint64_t r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(pack2(a)), "l"(pack2(b)));
  return unpack2(r);
}
__device__ __forceinline__ F2 fma2(F2 a, F2 b, F2 c) {
  uint64_t r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(pack2(a)), "l"(pack2(b)), "l"(pack2(c)));
  return unpack2(r);
}
__device__ __forceinline__ F2 both(float v) { return F2{v, v}; }
// 2^((v - zm) c) of two
__device__ __forceinline__ F2 exp2_of(F2 v, float zm, float c) {
  const F2 t = mul2(add2(v, both(-zm)), both(c));
  return F2{ex2(t.x), ex2(t.y)};
}
template <int kHard>
__device__ __forceinline__ F2 dense2(float c, const Row& r, F2 v) {
  const F2 e = exp2_of(v, r.zm, c);
  if (kHard == kNone) return mul2(e, both(r.ca));
  if (kHard == kPow1) return mul2(e, both(r.ca + r.c1));
  if (kHard == kPow2) return mul2(e, fma2(both(r.c1), e, both(r.ca)));
  if (kHard == kPow4) return mul2(e, fma2(mul2(both(r.c1), e), mul2(e, e), both(r.ca)));
  return fma2(both(r.ca), e, mul2(both(r.c1), exp2_of(v, r.zm, kLog2e)));
}

// A thread's running maximum and sums (of even and odd classes).
template <int kHard>
struct Running {
  float m = neg_inf();
  F2 s{0.f, 0.f}, s1{0.f, 0.f};
  __device__ __forceinline__ void raise(float top, float c) {
    if (!(top > m)) return;
    const float f = ex2((m - top) * c);   // 0 at first
    s = mul2(s, both(f));
    s1 = mul2(s1, both(kHard == kOwn ? ex2((m - top) * kLog2e) : pow_tau<kHard>(f)));
    m = top;
  }
  __device__ __forceinline__ void add(F2 v, float c) {
    const F2 e = exp2_of(v, m, c);
    s = add2(s, e);
    if (kHard == kOwn) s1 = add2(s1, exp2_of(v, m, kLog2e));
    else if (kHard == kPow2) s1 = fma2(e, e, s1);
    else if (kHard == kPow4) s1 = fma2(mul2(e, e), mul2(e, e), s1);
    else if (kHard == kPow1) s1 = s;
  }
  // nothing above -inf so far: only a NaN counts
  __device__ __forceinline__ void only_nan(float v) {
    if (v != v) s.x = s1.x = v;
  }
};

template <typename T, int kHard>
__global__ void __launch_bounds__(kRowThreads, 3) k_distill_row(const Args<T> g) {
  using V = Vec<T>;
  constexpr int kWarps = kRowThreads / 32, kN = V::kN;
  __shared__ int ids[kMaxK];
  __shared__ float p[kMaxK];
  __shared__ float rm[kWarps], rs[kWarps], rs1[kWarps];
  __shared__ int has_s;
  __shared__ float hi_s, log_tot_s;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, tid = threadIdx.x;
  pdl_trigger();
  pdl_wait();
  const int64_t row = blockIdx.x, b = row % g.rows;
  const T* z = g.z + row * g.n;
  const int label = label_of(g, b);
  if (warp == 0 && g.soft) {
    float hi = 0.f, log_tot = 0.f;
    const bool any = teacher<T, 32>(g, b, lane, lane, ids, p, hi, log_tot);
    if (lane == 0) has_s = any, hi_s = hi, log_tot_s = log_tot;
  }
  // single classes up to the first 16-byte boundary, groups, and single ones at the end
  const int head = min(g.n, (int)((16 - ((uintptr_t)z & 15)) & 15) / (int)sizeof(T));
  const int body = (g.n - head) / kN, tail = head + body * kN;
  const uint4* zv = reinterpret_cast<const uint4*>(z + head);
  const int single = tid < head ? tid : tail + tid - head;   // at most 2 (kN - 1) of them
  const bool mine = single < g.n && (tid < head || single >= tail);
  Running<kHard> q;
  for (int i = tid; i < body; i += kTurn * kRowThreads) {
    uint4 u[kTurn];
#pragma unroll
    for (int k = 0; k < kTurn; ++k) u[k] = i + k * kRowThreads < body ? zv[i + k * kRowThreads] : V::none();
    float top = V::top(u[0]);
#pragma unroll
    for (int k = 1; k < kTurn; ++k) top = fmaxf(top, V::top(u[k]));
    q.raise(top, g.c);
#pragma unroll
    for (int k = 0; k < kTurn; ++k) {
      float v[kN];
      V::get(u[k], v);
      if (q.m == neg_inf()) {
#pragma unroll
        for (int e = 0; e < kN; ++e) q.only_nan(v[e]);
      } else {
#pragma unroll
        for (int e = 0; e < kN; e += 2) q.add(F2{v[e], v[e + 1]}, g.c);
      }
    }
  }
  if (mine) {
    const float v = Elem<T>::to_f(z[single]);
    q.raise(v, g.c);
    if (q.m == neg_inf()) q.only_nan(v);
    else q.add(F2{v, neg_inf()}, g.c);
  }
  auto join = [&](float& s, float& s1, float m, float to) {
    if (to == neg_inf()) return;   // no class above -inf: 0 or NaN as it is
    const float f = ex2((m - to) * g.c);
    s *= f;
    s1 *= kHard == kOwn ? ex2((m - to) * kLog2e) : pow_tau<kHard>(f);
  };
  float s = q.s.x + q.s.y, s1 = q.s1.x + q.s1.y;
  const float wm = group_max<32>(q.m);
  join(s, s1, q.m, wm);
  s = group_sum<32>(s);
  s1 = group_sum<32>(s1);
  if (lane == 0) rm[warp] = wm, rs[warp] = s, rs1[warp] = s1;
  __syncthreads();
  float zm = neg_inf();
  s = s1 = 0.f;
#pragma unroll
  for (int k = 0; k < kWarps; ++k) zm = fmaxf(zm, rm[k]);
#pragma unroll 4
  for (int k = 0; k < kWarps; ++k) {
    float a = rs[k], a1 = rs1[k];
    join(a, a1, rm[k], zm);
    s += a;
    s1 += a1;
  }
  const bool has = g.soft && has_s;
  const Row r = make_row(g, zm, s, s1, has, label);
  T* dz = g.dz ? g.dz + row * g.n : nullptr;
  if (dz) {
    if ((((uintptr_t)z ^ (uintptr_t)dz) & 15) == 0) {
      uint4* dv = reinterpret_cast<uint4*>(dz + head);
      for (int i = tid; i < body; i += kTurn * kRowThreads) {
        uint4 u[kTurn];
#pragma unroll
        for (int k = 0; k < kTurn; ++k) u[k] = i + k * kRowThreads < body ? zv[i + k * kRowThreads] : V::none();
#pragma unroll
        for (int k = 0; k < kTurn; ++k) {
          float v[kN];
          V::get(u[k], v);
#pragma unroll
          for (int e = 0; e < kN; e += 2) {
            const F2 d = dense2<kHard>(g.c, r, F2{v[e], v[e + 1]});
            v[e] = d.x, v[e + 1] = d.y;
          }
          if (i + k * kRowThreads < body) dv[i + k * kRowThreads] = V::put(v);
        }
      }
      if (mine) dz[single] = Elem<T>::from_f(dense<kHard>(g.c, r, Elem<T>::to_f(z[single])));
    } else {   // dz starts at another place of a 16-byte group than z
      for (int i = tid; i < g.n; i += kRowThreads) dz[i] = Elem<T>::from_f(dense<kHard>(g.c, r, Elem<T>::to_f(z[i])));
    }
    __syncthreads();
  }
  if (warp == 0) {
    float kd = 0.f;
    if (has && r.alive)
      for (int j = lane; j < g.k; j += 32)
        kd += entry(g, r, z, dz, ids, p, (g.top[b * g.k + j] - hi_s) * (g.c * kLn2) - log_tot_s, j);
    kd = group_sum<32>(kd);
    if (lane == 0) {
      label_entry(g, r, z, dz, ids, has);
      g.row_loss[row] = row_loss(g, r, has, kd, r.label >= 0 ? Elem<T>::to_f(z[r.label]) : 0.f);
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
  if (a.n <= kSmallN) {
    const uint32_t div = ((1u << 20) + a.n - 1) / a.n;   // i / n = i div >> 20 for i < 128 * 32
    launch_pdl(k_distill_thread<T>, dim3((unsigned)ceil_div(a.all, kSmallRows)), dim3(kSmallRows),
               (size_t)kSmallRows * (a.n | 1) * 4, st, a, div);
  } else if (a.n <= 64) {
    group<T, 16, 4>(a, st);
  } else if (a.n <= 128) {
    group<T, 32, 4>(a, st);
  } else if (a.n <= 256) {
    group<T, 32, 8>(a, st);
  } else if (a.n <= 512) {
    group<T, 32, 16>(a, st);
  } else if (a.n <= 1024) {
    group<T, 32, 32>(a, st);
  } else {
    const dim3 grid((unsigned)a.all), block(kRowThreads);
    if (a.hard == kNone) launch_pdl(k_distill_row<T, kNone>, grid, block, 0, st, a);
    else if (a.hard == kPow1) launch_pdl(k_distill_row<T, kPow1>, grid, block, 0, st, a);
    else if (a.hard == kPow2) launch_pdl(k_distill_row<T, kPow2>, grid, block, 0, st, a);
    else if (a.hard == kPow4) launch_pdl(k_distill_row<T, kPow4>, grid, block, 0, st, a);
    else launch_pdl(k_distill_row<T, kOwn>, grid, block, 0, st, a);
  }
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
    const int soft = alpha > 0.f;
    const int hard = !(alpha < 1.f && labels) ? kNone : tau == 1.f ? kPow1 : tau == 2.f ? kPow2 : tau == 4.f ? kPow4 : kOwn;
    const float c = kLog2e / tau;
    if (precision == TP_FP32)
      rows(Args<float>{(const float*)z, ids, labels, top, (float*)dz, rl, m * n_rows, n_rows, n, k, soft, hard, c, tau,
                       alpha, 1.f / (float)n_rows}, st);
    else
      rows(Args<__nv_bfloat16>{(const __nv_bfloat16*)z, ids, labels, top, (__nv_bfloat16*)dz, rl, m * n_rows, n_rows, n, k,
                               soft, hard, c, tau, alpha, 1.f / (float)n_rows}, st);
    launch_pdl(k_distill_mean, dim3((unsigned)m), dim3(256), 0, st, (const float*)rl, n_rows, loss);
    e = cudaGetLastError();
  }
  if (e == cudaSuccess) return TP_OK;
  cudaGetLastError();   // reported here
  return ops_fail(TP_ECUDA, "pack_distill: %s", cudaGetErrorString(e));
}

}  // extern "C"
