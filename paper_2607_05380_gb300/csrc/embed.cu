// embed.cu -- embedding lookup with scaling, and the table's gradient by sorted
// tokens (entry points in tabpack_ops.h).
//
//   y[i] = scale table[ids[i]],   dtable[v] = scale sum_{i: ids[i] = v} dy[i]
//
// Lookup: a gather, bound by HBM (800 440 tokens of 64 columns from a table of a
// million rows, fp32 to bf16: 38 us, 4.8 TB/s of what it has to move); a few lanes
// a token, ids one turn ahead.
//
// Gradient of more than a few tokens: they are sorted by id (radix sort, stable), so
// that each row of the gradient is the sum of a run of tokens and is written once, in
// a fixed order of additions, without atomics on values.  A group of lanes adds up a
// chunk of sorted tokens: runs inside the chunk are finished there; what crosses its
// ends is joined with the block's other groups' in shared memory, and what crosses
// the block's ends, at most two 32-bit rows, is a sorted list again, which the same
// kernel takes until one block is left.  A value with many thousands of tokens is so
// spread over the GPU like any others.  The first level says, in a byte a row, which
// rows have tokens; beside the second the others are zeroed.
//
// Of few tokens bound by the chain of launches (49 152 of 128 columns, 20 011 rows:
// sort 18 us, sums 9.5, the join and the zeroes 8.5), of many by the sort's scattered
// stores and HBM (800 440 of 64 and a million rows: sort 52 us, sums 38, zeroes 28).
#include <algorithm>
#include <type_traits>

#include "lanes.cuh"
#include "prod.cuh"

using namespace tp;

namespace {

constexpr int32_t kMaxD = 1 << 17;
constexpr int64_t kMaxN = (int64_t(1) << 31) - 4096, kMaxElems = int64_t(1) << 40;
constexpr uint32_t kSkip = 0x80000000u;   // an entry of the partial rows that holds nothing
constexpr uint32_t kEnds = 0x80000000u;   // beside a row's number: the last entry of its run

struct Ids {
  const void* p;
  int32_t wide, vocab;
  // the id, or vocab for one outside the table
  __device__ __forceinline__ uint32_t at(int64_t i) const {
    const int64_t v = wide ? ((const int64_t*)p)[i] : (int64_t)((const int32_t*)p)[i];
    return v >= 0 && v < vocab ? (uint32_t)v : (uint32_t)vocab;
  }
};

// kE neighbouring columns of a row, as they were read, by loads and stores of up
// to 16 bytes that their address is a multiple of.
template <typename T, int kE>
struct Cols {
  static constexpr int kBytes = (int)sizeof(T) * kE, kWords = kBytes < 4 ? 1 : kBytes / 4;
  uint32_t w[kWords];
  __device__ __forceinline__ void load(const T* p, bool there) {
    if constexpr (kBytes == 2) {
      w[0] = there ? *reinterpret_cast<const uint16_t*>(p) : 0u;
    } else if constexpr (kBytes == 4) {
      w[0] = there ? *reinterpret_cast<const uint32_t*>(p) : 0u;
    } else if constexpr (kBytes == 8) {
      const uint2 v = there ? *reinterpret_cast<const uint2*>(p) : make_uint2(0u, 0u);
      w[0] = v.x, w[1] = v.y;
    } else {
#pragma unroll
      for (int h = 0; h < kBytes / 16; ++h) {
        const uint4 v = there ? reinterpret_cast<const uint4*>(p)[h] : make_uint4(0u, 0u, 0u, 0u);
        w[4 * h] = v.x, w[4 * h + 1] = v.y, w[4 * h + 2] = v.z, w[4 * h + 3] = v.w;
      }
    }
  }
  __device__ __forceinline__ float get(int e) const {
    if constexpr (sizeof(T) == 4) return __uint_as_float(w[e]);
    else return __uint_as_float(e & 1 ? w[e >> 1] & 0xFFFF0000u : w[e >> 1] << 16);
  }
  static __device__ __forceinline__ void put(T* p, const float (&v)[kE]) {
    uint32_t w[kWords];
    if constexpr (kBytes == 2) {
      *p = Elem<T>::from_f(v[0]);
      return;
    } else {
#pragma unroll
      for (int i = 0; i < kWords; ++i) {
        if constexpr (sizeof(T) == 4) {
          w[i] = __float_as_uint(v[i]);
        } else {
          const __nv_bfloat162 b = __floats2bfloat162_rn(v[2 * i], v[2 * i + 1]);
          w[i] = *reinterpret_cast<const uint32_t*>(&b);
        }
      }
      if constexpr (kBytes == 4) {
        *reinterpret_cast<uint32_t*>(p) = w[0];
      } else if constexpr (kBytes == 8) {
        *reinterpret_cast<uint2*>(p) = make_uint2(w[0], w[1]);
      } else {
#pragma unroll
        for (int h = 0; h < kBytes / 16; ++h)
          reinterpret_cast<uint4*>(p)[h] = make_uint4(w[4 * h], w[4 * h + 1], w[4 * h + 2], w[4 * h + 3]);
      }
    }
  }
};
// Do rows of d elements of `bytes` each, ld apart, allow loads of e of them at once?
bool fits(const void* p, int64_t ld, int d, int bytes, int e) {
  const int b = std::min(16, bytes * e);
  return d % e == 0 && ((uintptr_t)p % b) == 0 && (ld * bytes) % b == 0;
}

// How a row's columns are spread: 2^shift lanes a row, kI = `items` groups of
// kE = e columns a lane, the lanes' groups side by side.
struct Split {
  int e, shift, items;
  int64_t width() const { return (int64_t)(e * items) << shift; }
};
// The sums' split of n tokens: a warp a row where the row is wide enough for it, in
// as few columns a lane as blocks for the whole GPU allow, because the longest chain
// of a lane's work is what counts (1000 tokens of 192 columns: eight columns a lane
// 24 us, one 16); but of more tokens than keep it busy, more columns a lane,
// because then the instructions a token are (800 440 tokens of 64
// columns, both passes: two columns a lane 187 us, four 164, eight 179).  e_most:
// what the addresses allow.
Split split_cols(int64_t n, int d, int e_most) {
  Split s{1, 5, 1};
  while (s.width() < d && ceil_div(n, 256) * ceil_div(d, s.width()) > 2 * kSms)
    if (s.e < e_most) s.e *= 2;
    else if (s.e == 1 && s.items < 4) ++s.items;
    else break;
  while (s.shift > 3 && (s.e << (s.shift - 1)) >= d) --s.shift;   // (lanes idle in rows of less than eight columns: more, shorter lists)
  while (s.e < e_most && s.shift > 3 && (n >> 4) << (s.shift - 1) >= (int64_t)128 * 32 * kSms) s.e *= 2, --s.shift;
  if (s.e > 1) s.items = 1;
  return s;
}
// f(kE, kI) of a split
template <typename F>
void with_split(const Split& s, F f) {
  using std::integral_constant;
  using One = integral_constant<int, 1>;
  if (s.e == 8) f(integral_constant<int, 8>(), One());
  else if (s.e == 4) f(integral_constant<int, 4>(), One());
  else if (s.e == 2) f(integral_constant<int, 2>(), One());
  else if (s.items == 1) f(One(), One());
  else if (s.items == 2) f(One(), integral_constant<int, 2>());
  else if (s.items == 3) f(One(), integral_constant<int, 3>());
  else f(One(), integral_constant<int, 4>());
}

// ------------------------------------------------------------------- lookup
template <typename T, typename O>
struct LookArgs {
  Ids ids;
  const T* table;
  O* y;
  int64_t n, ldt;
  int32_t d, shift;
  float scale;
};
template <typename T, typename O, int kE, int kI>
__global__ void __launch_bounds__(256) k_lookup(const LookArgs<T, O> g) {
  constexpr int kU = 2;   // tokens in flight
  const int lanes = 1 << g.shift, groups = 256 >> g.shift;
  const int at = threadIdx.x & (lanes - 1), grp = threadIdx.x >> g.shift;
  const int64_t c0 = ((int64_t)blockIdx.y * kI * lanes + at) * kE, step = (int64_t)gridDim.x * groups * kU;
  pdl_trigger();
  pdl_wait();
  int64_t t0 = (int64_t)blockIdx.x * (groups * kU) + grp;
  uint32_t next[kU];   // the ids asked for
  auto ask = [&](int64_t from) {
#pragma unroll
    for (int u = 0; u < kU; ++u) next[u] = from + u * groups < g.n ? g.ids.at(from + u * groups) : (uint32_t)g.ids.vocab;
  };
  ask(t0);
  for (; t0 < g.n; t0 += step) {
    uint32_t id[kU];
#pragma unroll
    for (int u = 0; u < kU; ++u) id[u] = next[u];
    Cols<T, kE> v[kU][kI];
#pragma unroll
    for (int u = 0; u < kU; ++u) {
      const bool there = id[u] < (uint32_t)g.ids.vocab;
      const T* row = g.table + (there ? (int64_t)id[u] * g.ldt : 0) + c0;
#pragma unroll
      for (int i = 0; i < kI; ++i) v[u][i].load(row + i * lanes * kE, there && c0 + i * lanes * kE < g.d);
    }
    ask(t0 + step);
#pragma unroll
    for (int u = 0; u < kU; ++u) {
      const int64_t t = t0 + u * groups;
      if (t >= g.n) break;
      const bool there = id[u] < (uint32_t)g.ids.vocab;
#pragma unroll
      for (int i = 0; i < kI; ++i) {
        if (c0 + i * lanes * kE >= g.d) break;
        float f[kE];
#pragma unroll
        for (int e = 0; e < kE; ++e) f[e] = there ? v[u][i].get(e) * g.scale : 0.f;   // (no -0, no NaN by the scale)
        Cols<O, kE>::put(g.y + t * g.d + c0 + i * lanes * kE, f);
      }
    }
  }
}

// Rows of an odd number of columns: 16 bytes of y a thread, whatever rows they belong
// to.  A block's tokens are a multiple of eight, so that it starts at a multiple of
// 16 bytes.  (140 077 tokens of 33 columns, fp32: a warp a row 13 us, this 10.)  Of fewer
// tokens, whose blocks do not fill the GPU, lanes over a row (bf16, us, this and
// those: 2000 of 129 2.8 and 2.7, of 2047 11.3 and 8.4; 10 000 5.1 and 5.5, 25 and
// 34; of 33 3.2 and 3.3).
constexpr int kFlatTokens = 2048;   // of a block, at most
constexpr int64_t kFlatFrom = 8192;
template <typename T, typename O>
__global__ void __launch_bounds__(256) k_lookup_flat(const LookArgs<T, O> g, int tokens) {
  constexpr int kE = 16 / sizeof(O);
  __shared__ uint32_t id[kFlatTokens + 1];
  pdl_trigger();
  pdl_wait();
  const int64_t t0 = (int64_t)blockIdx.x * tokens;
  const int here = (int)min((int64_t)tokens, g.n - t0);
  for (int i = threadIdx.x; i <= here; i += 256) id[i] = i < here ? g.ids.at(t0 + i) : (uint32_t)g.ids.vocab;
  __syncthreads();
  const uint32_t total = (uint32_t)here * (uint32_t)g.d;
  O* y = g.y + t0 * g.d;
#pragma unroll 2
  for (uint32_t e = threadIdx.x * kE; e < total; e += 256 * kE) {
    uint32_t row = e / (uint32_t)g.d, c = e - row * (uint32_t)g.d;
    float v[kE];
#pragma unroll
    for (int i = 0; i < kE; ++i) {
      const uint32_t k = row < (uint32_t)here ? id[row] : (uint32_t)g.ids.vocab;
      const bool there = k < (uint32_t)g.ids.vocab;
      v[i] = there ? Elem<T>::to_f(g.table[(int64_t)k * g.ldt + c]) * g.scale : 0.f;
      if (++c == (uint32_t)g.d) c = 0, ++row;
    }
    if (e + kE <= total) {
      Cols<O, kE>::put(y + e, v);
    } else {
#pragma unroll
      for (int i = 0; i < kE; ++i)
        if (e + i < total) y[e + i] = Elem<O>::from_f(v[i]);
    }
  }
}

// --------------------------------------------------------------------- sort
// Radix sort, stable, by digits of at most kMaxBits bits.  A block ranks the
// tokens of a tile by its warps' counts of each digit.
constexpr int kMaxBits = 10;   // the warps' counts of a digit's values fit in shared memory beside a tile
constexpr int kFewBits = 8;    // of the sorts in one launch, whose passes clear and add up the counts of fewer tokens

struct SortArgs {
  Ids ids;                      // the first pass's keys; their places are its values
  const uint32_t *key, *val;    // the later ones'
  uint32_t *key_out, *val_out;
  uint32_t *count, *total;      // [bins][blocks]; [bins]
  uint8_t* seen;                // a byte per row of the table: whether it has a token
  int64_t n;
  int32_t first, shift, bits_all, blocks;
};
constexpr uint32_t kLast = 0xffffffffu;   // the key of a place past the last token: behind all others in every pass
__device__ __forceinline__ uint32_t key_at(const SortArgs& g, int64_t i) { return g.first ? g.ids.at(i) : g.key[i]; }

__device__ __forceinline__ void clear_seen(const SortArgs& g, int64_t thread, int64_t threads) {
  const int64_t words = ((int64_t)g.ids.vocab + 15) >> 4;
  for (int64_t i = thread; i < words; i += threads) reinterpret_cast<uint4*>(g.seen)[i] = make_uint4(0u, 0u, 0u, 0u);
}

// Of a launch whose first block sorts alone: the others, where the table is large
// enough for some, clear its bytes.  Is this one of them?
__device__ __forceinline__ bool clears(const SortArgs& g) {
  if (blockIdx.x > 0) clear_seen(g, (int64_t)(blockIdx.x - 1) * blockDim.x + threadIdx.x, (int64_t)(gridDim.x - 1) * blockDim.x);
  else if (gridDim.x == 1) clear_seen(g, threadIdx.x, blockDim.x);
  return blockIdx.x > 0;
}

// Exclusive prefix sums of v[0 .. bins - 1] in shared memory, by the whole block.
template <int kThreads>
__device__ __forceinline__ void block_scan(uint32_t* v, int bins, uint32_t* warps) {
  constexpr int kPer = (1 << kMaxBits) / kThreads, kWarps = kThreads / 32;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  uint32_t c[kPer], s = 0;
#pragma unroll
  for (int i = 0; i < kPer; ++i) {
    const int at = threadIdx.x * kPer + i;
    c[i] = at < bins ? v[at] : 0u;
    s += c[i];
  }
  uint32_t t = s;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const uint32_t u = __shfl_up_sync(0xffffffffu, t, o);
    if (lane >= o) t += u;
  }
  if (lane == 31) warps[warp] = t;
  __syncthreads();
  uint32_t before = lane < warp && lane < kWarps ? warps[lane] : 0u;   // the warps before this one
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) before += __shfl_xor_sync(0xffffffffu, before, o);
  before += t - s;
#pragma unroll
  for (int i = 0; i < kPer; ++i) {
    const int at = threadIdx.x * kPer + i;
    if (at < bins) v[at] = before;
    before += c[i];
  }
  __syncthreads();
}

// Each token's number among those of its digit in its warp (in order), and in
// wh the warps' counts; afterwards wh holds, per warp and digit, the tokens of
// the warps before it, and sum (if wanted) the block's counts.  The lanes of one
// digit find each other by a ballot per bit, the most of a pass's work (masks or-ed
// in shared memory, or match.any: as much for spread digits, more for frequent ones).
template <int kThreads, int kBits, int kR>
__device__ __forceinline__ void rank_tile(const uint32_t (&key)[kR], int shift, uint16_t* wh, uint32_t* sum,
                                          uint32_t (&rank)[kR]) {
  constexpr int kWarps = kThreads / 32, bins = 1 << kBits;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  for (int i = threadIdx.x; i < bins * kWarps / 2; i += kThreads) ((uint32_t*)wh)[i] = 0;
  __syncthreads();
  uint16_t* mine = wh + warp * bins;
#pragma unroll
  for (int r = 0; r < kR; ++r) {
    const uint32_t digit = key[r] >> shift & (bins - 1);
    uint32_t same = 0xffffffffu;
#pragma unroll
    for (int b = 0; b < kBits; ++b) {
      const uint32_t set = __ballot_sync(0xffffffffu, digit >> b & 1);
      same &= ~(set ^ (uint32_t)((int32_t)(digit << (31 - b)) >> 31));   // the lanes whose bit is this one's
    }
    const uint32_t before = mine[digit], lower = same & ((1u << lane) - 1);
    rank[r] = before + __popc(lower);
    __syncwarp();
    if (lower == 0) mine[digit] = (uint16_t)(before + __popc(same));
    __syncwarp();
  }
  __syncthreads();
  for (int i = threadIdx.x; i < bins; i += kThreads) {
    uint32_t s = 0;
#pragma unroll 1
    for (int w0 = 0; w0 < kWarps; w0 += 8) {   // eight loads in flight
      uint32_t c[8];
#pragma unroll
      for (int w = 0; w < 8; ++w) c[w] = wh[(w0 + w) * bins + i];
#pragma unroll
      for (int w = 0; w < 8; ++w) {
        wh[(w0 + w) * bins + i] = (uint16_t)s;
        s += c[w];
      }
    }
    if (sum) sum[i] = s;
  }
  __syncthreads();
}

// Many tokens: three launches a pass, a tile of kRounds tokens a thread a block (800 440
// tokens, two passes: counts 12 us, their scans 6, scattered stores 34; a bit per
// row of the table set by atomics beside them 150 more).
constexpr int kSortThreads = 512;

template <int kRounds, int kBits>
__global__ void __launch_bounds__(kSortThreads) k_sort_count(const SortArgs g) {
  __shared__ uint32_t h[1 << kBits];
  pdl_trigger();
  pdl_wait();
  constexpr int bins = 1 << kBits;
  for (int i = threadIdx.x; i < bins; i += kSortThreads) h[i] = 0;
  uint32_t key[kRounds];
#pragma unroll
  for (int r = 0; r < kRounds; ++r) {
    const int64_t i = (int64_t)blockIdx.x * (kSortThreads * kRounds) + r * kSortThreads + threadIdx.x;
    key[r] = i < g.n ? key_at(g, i) : kLast;
  }
  __syncthreads();
#pragma unroll
  for (int r = 0; r < kRounds; ++r)
    if (key[r] != kLast) atomicAdd(&h[key[r] >> g.shift & (bins - 1)], 1u);
  __syncthreads();
  for (int i = threadIdx.x; i < bins; i += kSortThreads) g.count[(int64_t)i * g.blocks + blockIdx.x] = h[i];
  if (g.first) clear_seen(g, (int64_t)blockIdx.x * kSortThreads + threadIdx.x, (int64_t)g.blocks * kSortThreads);
}

// Where each block's tokens of a digit begin among the digit's: a warp a digit.
__global__ void __launch_bounds__(256) k_sort_scan(uint32_t* count, uint32_t* total, int blocks, int bins) {
  pdl_trigger();
  pdl_wait();
  const int bin = blockIdx.x * 8 + (threadIdx.x >> 5), lane = threadIdx.x & 31;
  if (bin >= bins) return;
  uint32_t* row = count + (int64_t)bin * blocks;
  uint32_t before = 0;
  for (int b = 0; b < blocks; b += 128) {   // four a lane
    uint32_t c[4], s = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int at = b + 4 * lane + i;
      c[i] = at < blocks ? row[at] : 0u;
      s += c[i];
    }
    uint32_t t = s;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const uint32_t v = __shfl_up_sync(0xffffffffu, t, o);
      if (lane >= o) t += v;
    }
    uint32_t at_lane = before + t - s;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if (b + 4 * lane + i < blocks) row[b + 4 * lane + i] = at_lane;
      at_lane += c[i];
    }
    before += __shfl_sync(0xffffffffu, t, 31);
  }
  if (lane == 0) total[bin] = before;
}

template <int kRounds, int kBits>
__global__ void __launch_bounds__(kSortThreads, kRounds <= 4 ? 3 : 2) k_sort_scatter(const SortArgs g) {
  extern __shared__ uint32_t sm[];
  constexpr int bins = 1 << kBits;
  uint32_t* base = sm;
  uint16_t* wh = (uint16_t*)(sm + bins + 32);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  pdl_trigger();
  pdl_wait();
  const int64_t i0 = (int64_t)blockIdx.x * (kSortThreads * kRounds) + warp * (32 * kRounds) + lane;
  uint32_t key[kRounds], val[kRounds], rank[kRounds];
#pragma unroll
  for (int r = 0; r < kRounds; ++r) {
    const int64_t i = i0 + 32 * r;
    key[r] = i < g.n ? key_at(g, i) : kLast;
    val[r] = g.first ? (uint32_t)i : i < g.n ? g.val[i] : 0u;
  }
  for (int i = threadIdx.x; i < bins; i += kSortThreads) base[i] = g.total[i];
  __syncthreads();
  block_scan<kSortThreads>(base, bins, sm + bins);
  for (int i = threadIdx.x; i < bins; i += kSortThreads) base[i] += g.count[(int64_t)i * g.blocks + blockIdx.x];
  rank_tile<kSortThreads, kBits>(key, g.shift, wh, nullptr, rank);
#pragma unroll
  for (int r = 0; r < kRounds; ++r) {
    if (i0 + 32 * r >= g.n) continue;
    const uint32_t digit = key[r] >> g.shift & (bins - 1);
    const uint32_t to = base[digit] + wh[warp * bins + digit] + rank[r];
    g.key_out[to] = key[r];
    g.val_out[to] = val[r];
  }
}

// Up to 64 K tokens: every pass in one launch of a cluster of kCluster blocks,
// which keep the tokens in registers and hand them over through each other's
// shared memory.  A block sorts its own by the digit first: neighbours then go
// to neighbouring places (49 152 tokens, two passes: 18 us; one 4-byte store each to
// a place of its own 38).  A pass takes 8 us: the ranks 2.8, the blocks' counts and
// scans 1.5, handing over 1 to 2, two barriers of the cluster 1.5.
constexpr int kCluster = 16, kClusterThreads = 512;
__device__ __forceinline__ uint32_t cluster_address(const void* p, uint32_t rank) {
  uint32_t a;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(a) : "r"((uint32_t)__cvta_generic_to_shared(p)), "r"(rank));
  return a;
}
__device__ __forceinline__ void cluster_barrier() {
  asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
template <int kR>
constexpr int cluster_smem() {   // tokens sent and received; counts, three bases and the scan's; the warps' counts
  return 2 * kR * kClusterThreads * 8 + (4 * (1 << kFewBits) + 32) * 4 +
         (1 << kFewBits) * (kClusterThreads / 32) * 2;
}
template <int kR>
__global__ void __launch_bounds__(kClusterThreads, 1) k_sort_cluster(const SortArgs g) {
  constexpr int kPer = kR * kClusterThreads;   // tokens a block
  extern __shared__ __align__(16) uint32_t sm[];
  constexpr int bins = 1 << kFewBits;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  uint2 *sent = (uint2*)sm, *got = sent + kPer;
  uint32_t *cnt = (uint32_t*)(got + kPer), *local = cnt + bins, *below = local + bins, *base = below + bins;
  uint16_t* wh = (uint16_t*)(base + bins + 32);
  const uint32_t rank_of = blockIdx.x;         // (one cluster)
  pdl_trigger();
  pdl_wait();
  const int at0 = warp * (32 * kR) + lane;
  uint32_t key[kR], val[kR], rank[kR];
#pragma unroll
  for (int r = 0; r < kR; ++r) {
    val[r] = rank_of * kPer + at0 + 32 * r;
    key[r] = (int64_t)val[r] < g.n ? g.ids.at(val[r]) : kLast;
  }
  clear_seen(g, rank_of * kClusterThreads + threadIdx.x, kCluster * kClusterThreads);
  for (int shift = 0; shift < g.bits_all; shift += kFewBits) {
    rank_tile<kClusterThreads, kFewBits>(key, shift, wh, cnt, rank);
    cluster_barrier();   // all counts are there, and all tokens of the pass before have been read
    // what the blocks have of a digit: four lanes a digit look at four blocks each
    for (int i = threadIdx.x; i < 4 * bins; i += kClusterThreads) {
      const int bin = i >> 2, b0 = (i & 3) * (kCluster / 4);
      uint32_t c[kCluster / 4], all = 0, low = 0;
#pragma unroll
      for (int b = 0; b < kCluster / 4; ++b)
        asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(c[b]) : "r"(cluster_address(cnt + bin, b0 + b)));
#pragma unroll
      for (int b = 0; b < kCluster / 4; ++b) all += c[b], low += b0 + b < (int)rank_of ? c[b] : 0u;
#pragma unroll
      for (int o = 1; o < 4; o <<= 1) {
        all += __shfl_xor_sync(0xffffffffu, all, o);
        low += __shfl_xor_sync(0xffffffffu, low, o);
      }
      if ((i & 3) == 0) base[bin] = all, local[bin] = cnt[bin], below[bin] = low;
    }
    __syncthreads();
    block_scan<kClusterThreads>(local, bins, base + bins);
    block_scan<kClusterThreads>(base, bins, base + bins);
#pragma unroll
    for (int r = 0; r < kR; ++r) {
      const uint32_t digit = key[r] >> shift & (bins - 1);
      sent[local[digit] + wh[warp * bins + digit] + rank[r]] = make_uint2(key[r], val[r]);
    }
    for (int i = threadIdx.x; i < bins; i += kClusterThreads)   // from a block's own place to the cluster's
      base[i] += below[i] - local[i];
    __syncthreads();
#pragma unroll
    for (int r = 0; r < kR; ++r) {
      const int i = threadIdx.x + r * kClusterThreads;
      const uint2 t = sent[i];
      const uint32_t to = base[t.x >> shift & (bins - 1)] + i, block = to / kPer, place = to % kPer;
      asm volatile("st.shared::cluster.v2.u32 [%0], {%1, %2};" ::"r"(cluster_address(got + place, block)), "r"(t.x), "r"(t.y)
                   : "memory");
    }
    cluster_barrier();
#pragma unroll
    for (int r = 0; r < kR; ++r) {
      const uint2 t = got[at0 + 32 * r];
      key[r] = t.x, val[r] = t.y;
    }
  }
  const int64_t i0 = (int64_t)rank_of * kPer + at0;
#pragma unroll
  for (int r = 0; r < kR; ++r)
    if (i0 + 32 * r < g.n) g.key_out[i0 + 32 * r] = key[r], g.val_out[i0 + 32 * r] = val[r];
}

// Up to 4096 tokens: every pass in one block.
constexpr int kTileThreads = 1024;
template <int kR>
constexpr int tile_smem() {
  return kR * kTileThreads * 8 + ((1 << kFewBits) + 32) * 4 + (1 << kFewBits) * (kTileThreads / 32) * 2;
}
template <int kR>
__global__ void __launch_bounds__(kTileThreads, 1) k_sort_tile(const SortArgs g) {
  extern __shared__ __align__(16) uint32_t sm[];
  constexpr int bins = 1 << kFewBits;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  uint2* sorted = (uint2*)sm;
  uint32_t *base = (uint32_t*)(sorted + kR * kTileThreads);
  uint16_t* wh = (uint16_t*)(base + bins + 32);
  pdl_trigger();
  pdl_wait();
  if (clears(g)) return;
  const int at0 = warp * (32 * kR) + lane;
  uint32_t key[kR], val[kR], rank[kR];
#pragma unroll
  for (int r = 0; r < kR; ++r) {
    val[r] = at0 + 32 * r;
    key[r] = (int)val[r] < g.n ? g.ids.at(val[r]) : kLast;
  }
  for (int shift = 0; shift < g.bits_all; shift += kFewBits) {
    rank_tile<kTileThreads, kFewBits>(key, shift, wh, base, rank);
    block_scan<kTileThreads>(base, bins, base + bins);
#pragma unroll
    for (int r = 0; r < kR; ++r) {
      const uint32_t digit = key[r] >> shift & (bins - 1);
      sorted[base[digit] + wh[warp * bins + digit] + rank[r]] = make_uint2(key[r], val[r]);
    }
    __syncthreads();
#pragma unroll
    for (int r = 0; r < kR; ++r) {
      const uint2 t = sorted[at0 + 32 * r];
      key[r] = t.x, val[r] = t.y;
    }
  }
#pragma unroll
  for (int r = 0; r < kR; ++r)
    if (at0 + 32 * r < g.n) g.key_out[at0 + 32 * r] = key[r], g.val_out[at0 + 32 * r] = val[r];
}

// --------------------------------------------------------------------- runs
template <typename T, typename O>
struct RunArgs {
  const uint32_t *key, *val;    // val: the rows of src (NULL: one after another)
  const T* src;
  O* out;
  uint32_t* key_out;            // two entries a block
  float* part;
  uint8_t* seen;                // the table's rows that have a token: the first level says, beside the second the others
                                // are zeroed
  int64_t m, ld;
  int32_t chunk, d, vocab, shift, run_blocks, first, wide;   // wide: zero_rows by 16 bytes
  float scale;
};

// Rows without a token become zero: a thread takes 16 bytes of the table, whatever
// rows they belong to.
template <typename O>
__device__ __forceinline__ void zero_flat(const uint8_t* seen, O* out, int64_t vocab, int d, int64_t block, int64_t blocks) {
  constexpr int kE = 16 / sizeof(O);
  const int64_t total = vocab * d, step = blocks * blockDim.x * kE;
  for (int64_t base = (block * blockDim.x + (threadIdx.x & ~31)) * kE; base < total; base += step) {
    const int64_t row0 = base / d;   // of the warp's first element
    const uint32_t off = (uint32_t)(base - row0 * d) + (threadIdx.x & 31) * kE, row = off / (uint32_t)d;
    const int64_t at = base + (threadIdx.x & 31) * kE;
    if (at >= total) continue;
    uint32_t c = off - row * (uint32_t)d;
    int64_t r = row0 + row;
    uint32_t keep = 0, here = seen[r];
#pragma unroll
    for (int e = 0; e < kE; ++e) {
      if (at + e < total) keep |= (here ? 1u : 0u) << e;
      if (++c == (uint32_t)d && e + 1 < kE) c = 0, here = ++r < vocab ? seen[r] : 1u;
    }
    const float zero[kE] = {};
    if (keep == 0 && at + kE <= total) {
      Cols<O, kE>::put(out + at, zero);
    } else {
#pragma unroll
      for (int e = 0; e < kE; ++e)
        if (!(keep >> e & 1) && at + e < total) out[at + e] = Elem<O>::from_f(0.f);
    }
  }
}
// The same with fewer instructions where there is a warp's turn for every 32 rows:
// 2^shift lanes a row, by 16-byte stores where the rows lie on multiples of 16 bytes;
// and for a table that does not start at one.  (3000 rows of 192, where 94 warps had
// one: 22 us of a backward pass, 16 the other way.)
template <typename O, int kE>
__device__ __forceinline__ void zero_rows(const uint8_t* seen, O* out, int64_t vocab, int d, int64_t block, int64_t blocks) {
  const int lane = threadIdx.x & 31, warps = (int)blockDim.x >> 5;
  int shift = 0;
  while (shift < 5 && (kE << shift) < d) ++shift;
  const int at = lane & ((1 << shift) - 1), sub = lane >> shift, step = 32 >> shift;
  const float zero[kE] = {};
  for (int64_t r0 = (block * warps + (threadIdx.x >> 5)) * 32; r0 < vocab; r0 += blocks * warps * 32) {
    const uint32_t absent = __ballot_sync(0xffffffffu, r0 + lane < vocab && seen[r0 + lane] == 0);
#pragma unroll 4
    for (int r = sub; r < 32; r += step)
      if (absent >> r & 1)
        for (int64_t c = at * kE; c < d; c += kE << shift) Cols<O, kE>::put(out + (r0 + r) * d + c, zero);
  }
}

// A group of 2^shift lanes takes `chunk` entries of the sorted list, kI kE of
// their columns a lane, a block the chunks of its groups.  What the groups leave
// is joined in shared memory, what the block leaves goes to the next level.
constexpr int kRunThreads = 512, kJoinThreads = 1024;   // of the first level; of the later ones
constexpr int kMostEntries = 4096;                      // of a block
template <typename T, typename O, int kE, int kI>
__global__ void __launch_bounds__(1024) k_runs(const RunArgs<T, O> g) {
  constexpr int kWords = Cols<T, kE>::kWords * kI, kU = kWords >= 8 ? 4 : 8;   // rows in flight
  extern __shared__ __align__(16) float rows[];           // two a group, then the block's keys and places
  __shared__ uint32_t keys[2 * 1024];
  pdl_trigger();
  pdl_wait();
  if ((int)blockIdx.x >= g.run_blocks) {
    constexpr int kWide = 16 / sizeof(O);
    const int64_t block = (int64_t)(blockIdx.x - g.run_blocks) * gridDim.y + blockIdx.y;
    const int64_t blocks = (int64_t)(gridDim.x - g.run_blocks) * gridDim.y;
    if (g.wide) zero_rows<O, kWide>(g.seen, g.out, g.vocab, g.d, block, blocks);
    else if (((uintptr_t)g.out & 15) == 0) zero_flat(g.seen, g.out, g.vocab, g.d, block, blocks);
    else zero_rows<O, 1>(g.seen, g.out, g.vocab, g.d, block, blocks);
    return;
  }
  const int lanes = 1 << g.shift, groups = (int)blockDim.x >> g.shift, at = threadIdx.x & (lanes - 1);
  const int grp = threadIdx.x >> g.shift, per_block = groups * g.chunk;
  uint2* entry = (uint2*)(rows + 2 * blockDim.x * (kI * kE));   // a row of src, kEnds on the last one of a run; the key
  const int64_t b0 = (int64_t)blockIdx.x * per_block, c0 = ((int64_t)blockIdx.y * kI * lanes + at) * kE;
  const int n_here = (int)min((int64_t)per_block, g.m - b0);
  const int i_first = min(grp * g.chunk, n_here), count = min(g.chunk, n_here - i_first);
  float acc[kI][kE];
  bool any = false;
  auto clear = [&] {
#pragma unroll
    for (int i = 0; i < kI; ++i)
#pragma unroll
      for (int e = 0; e < kE; ++e) acc[i][e] = 0.f;
    any = false;
  };
  auto write = [&](uint32_t row) {   // a finished sum
    O* out = g.out + (int64_t)row * g.d + c0;
#pragma unroll
    for (int i = 0; i < kI; ++i) {
      float v[kE];
#pragma unroll
      for (int e = 0; e < kE; ++e) v[e] = acc[i][e] * g.scale;
      if (c0 + i * lanes * kE < g.d) Cols<O, kE>::put(out + i * lanes * kE, v);
    }
  };
  // an entry's row, the lanes' columns side by side
  auto slot = [&](int entry, int i) { return rows + (entry * kI + i) * (lanes * kE) + at * kE; };
  for (int i = threadIdx.x; i < n_here; i += blockDim.x) {
    const uint32_t key = g.key[b0 + i], next = b0 + i + 1 < g.m ? g.key[b0 + i + 1] & ~kSkip : kLast;
    entry[i] = make_uint2((g.val ? g.val[b0 + i] : (uint32_t)(b0 + i)) | ((key & ~kSkip) != next ? kEnds : 0u), key);
    // the first token of a row says that the row has one
    if (g.first && blockIdx.y == 0 && key < (uint32_t)g.vocab && (b0 + i == 0 || g.key[b0 + i - 1] != key)) g.seen[key] = 1;
  }
  const uint32_t block_before = b0 ? g.key[b0 - 1] & ~kSkip : kLast;
  const uint32_t block_after = b0 + n_here < g.m ? g.key[b0 + n_here] & ~kSkip : kLast;
  __syncthreads();
  const uint32_t before = i_first ? entry[i_first - 1].y & ~kSkip : block_before;
  const uint32_t key0 = count ? entry[i_first].y & ~kSkip : kLast, key1 = count ? entry[i_first + count - 1].y & ~kSkip : kLast;
  uint32_t left0 = key0 | kSkip, left1 = key1 | kSkip;   // what the group leaves: nothing yet
  bool open = before == key0;                            // the run began before the group
  auto leave = [&](int which, uint32_t key) {
#pragma unroll
    for (int i = 0; i < kI; ++i) Cols<float, kE>::put(slot(2 * grp + which, i), acc[i]);
    if (which) left1 = key;
    else left0 = key;
  };
  clear();
  // all groups of a warp take the same number of steps, so that they meet again after each
#pragma unroll 1
  for (int i0 = 0; i0 < g.chunk; i0 += kU) {
    Cols<T, kE> v[kU][kI];
    uint2 in[kU];
#pragma unroll
    for (int u = 0; u < kU; ++u) {
      in[u] = i0 + u < count ? entry[i_first + i0 + u] : make_uint2(0u, kLast);
      const bool there = in[u].y < (uint32_t)g.vocab;   // (neither skipped nor outside the table)
      const T* row = g.src + (there ? (int64_t)(in[u].x & ~kEnds) * g.ld : 0) + c0;
#pragma unroll
      for (int i = 0; i < kI; ++i) v[u][i].load(row + i * lanes * kE, there && c0 + i * lanes * kE < g.d);
    }
#pragma unroll
    for (int u = 0; u < kU; ++u) {
      any = any || in[u].y < (uint32_t)g.vocab;
#pragma unroll
      for (int i = 0; i < kI; ++i)
#pragma unroll
        for (int e = 0; e < kE; ++e) acc[i][e] += v[u][i].get(e);   // (zeros where there is none)
      if (in[u].x & kEnds) {
        const uint32_t key = in[u].y & ~kSkip;
        if (any) {
          if (open) leave(0, key);
          else write(key);
        }
        clear();
        open = false;
      }
      __syncwarp();
    }
  }
  if (any) leave(open ? 0 : 1, key1);   // a run that goes on
  if (at == 0) {   // (a group without entries: kLast)
    keys[2 * grp] = left0;
    keys[2 * grp + 1] = left1;
  }
  __syncthreads();
  const int n = 2 * ((n_here + g.chunk - 1) / g.chunk);   // entries that the block's groups have left
  // a run of entries is summed by the group that left its first one
#pragma unroll 1
  for (int e = 2 * grp; e < min(2 * grp + 2, n); ++e) {
    const uint32_t key = keys[e] & ~kSkip;
    if (e && (keys[e - 1] & ~kSkip) == key) continue;
    clear();
    int j = e;
    for (bool more = true; more;) {   // four entries at a time
      uint32_t k[4];
      float v[4][kI][kE];
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        k[u] = j + u < n ? keys[j + u] : kLast;
#pragma unroll
        for (int i = 0; i < kI; ++i)
#pragma unroll
          for (int c = 0; c < kE; ++c) v[u][i][c] = k[u] == key ? slot(j + u, i)[c] : 0.f;
      }
      int same = 0;
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        more = more && (k[u] & ~kSkip) == key && k[u] != kLast;
        same += more;
        any = any || (more && k[u] == key);
#pragma unroll
        for (int i = 0; i < kI; ++i)
#pragma unroll
          for (int c = 0; c < kE; ++c) acc[i][c] += v[u][i][c];   // (an entry of the key lies in its run)
      }
      j += same;
    }
    const bool from = e == 0 && block_before == key, on = j == n && block_after == key;
    if (any && !from && !on) write(key);
    if (!g.key_out) continue;
    const bool left = any && (from || on);
    if (left) {
      float* part = g.part + (2 * (int64_t)blockIdx.x + (from ? 0 : 1)) * g.d + c0;
#pragma unroll
      for (int i = 0; i < kI; ++i)
        if (c0 + i * lanes * kE < g.d) Cols<float, kE>::put(part + i * lanes * kE, acc[i]);
    }
    // the block's two entries: of its first run and of its last; where these are one run, the second holds nothing
    if (at == 0 && blockIdx.y == 0) {
      uint32_t* out = g.key_out + 2 * (int64_t)blockIdx.x;
      if (e == 0) out[0] = left && from ? key : key | kSkip;
      if (j == n) out[1] = left && !from ? key : key | kSkip;
    }
  }
}

// --------------------------------------------------------------- few tokens
// A few tokens: one launch without a sort.  A block zeroes a run of the table's rows,
// but those that have tokens; it sums those rows that are its number modulo the
// blocks', for each of which its eight warps look through 32 tokens each, and their
// sums are joined in order.  (Sorted, and summed and joined in launches of their own: 12 us
// instead of 5 for 36 tokens.)
constexpr int kFew = 256;
template <typename T, typename O>
struct FewArgs {
  Ids ids;
  const T* dy;
  O* out;
  int64_t ld;
  int32_t n, d;
  float scale;
};
template <typename T, typename O, int kE>
__global__ void __launch_bounds__(kFew) k_grad_few(const FewArgs<T, O> g) {
  constexpr int kWarps = kFew / 32, kU = 4;   // kU: rows in flight
  __shared__ uint32_t key[kFew], hit[kFew], near[kFew];
  __shared__ int n_hit, n_near;
  __shared__ __align__(16) float part[kWarps][32 * kE];
  const int t = threadIdx.x, warp = t >> 5, lane = t & 31;
  const uint32_t blocks = gridDim.x, vocab = (uint32_t)g.ids.vocab;
  pdl_trigger();
  pdl_wait();
  key[t] = t < g.n ? g.ids.at(t) : kLast;
  if (t == 0) n_hit = n_near = 0;
  __syncthreads();
  if (key[t] < vocab && key[t] % blocks == blockIdx.x) {
    bool first = true;
    for (int j = 0; j < t; ++j) first = first && key[j] != key[t];
    if (first) hit[atomicAdd(&n_hit, 1)] = key[t];   // (in any order: it decides on no sum)
  }
  // rows to be zeroed: a run of the table's, at once where no token has one of them
  const int64_t per = ceil_div(vocab, blocks), z0 = min((int64_t)vocab, blockIdx.x * per), z1 = min((int64_t)vocab, z0 + per);
  if (key[t] >= z0 && key[t] < z1) near[atomicAdd(&n_near, 1)] = key[t];
  __syncthreads();
  const int hits = n_hit, nears = n_near;
  constexpr int kWide = 16 / sizeof(O);
  const int64_t e0 = z0 * g.d, e1 = z1 * g.d;
  const int64_t v0 = min(e1, e0 + (int64_t)(-(uintptr_t)(g.out + e0) / sizeof(O) % kWide)), v1 = v0 + (e1 - v0) / kWide * kWide;
  // has one of the rows from a to b a token?
  auto taken = [&](int64_t a, int64_t b) {
    bool is = false;
    for (int i = 0; i < nears; ++i) is = is || (near[i] >= a && near[i] <= b);
    return is;
  };
  auto one = [&](int64_t e) {
    const int64_t r = nears ? e / g.d : 0;
    if (!nears || !taken(r, r)) g.out[e] = Elem<O>::from_f(0.f);
  };
  const float wide[kWide] = {};
  for (int64_t e = v0 + t * kWide; e < v1; e += kFew * kWide) {
    const int64_t r = nears ? e / g.d : 0, last = nears ? (e + kWide - 1) / g.d : 0;
    if (!nears || !taken(r, last)) {
      Cols<O, kWide>::put(g.out + e, wide);
    } else {
      for (int i = 0; i < kWide; ++i) one(e + i);
    }
  }
  for (int64_t e = e0 + t; e < v0; e += kFew) one(e);
  for (int64_t e = v1 + t; e < e1; e += kFew) one(e);
  for (int h = 0; h < hits; ++h) {
    const uint32_t row = hit[h];
    const uint32_t mine = __ballot_sync(0xffffffffu, key[t] == row);
    for (int64_t c0 = 0; c0 < g.d; c0 += 32 * kE) {
      const int64_t c = c0 + lane * kE;
      float acc[kE] = {};
      for (uint32_t left = mine; left;) {
        Cols<T, kE> v[kU];
#pragma unroll
        for (int u = 0; u < kU; ++u) {
          const int i = 32 * warp + __ffs(left) - 1;
          v[u].load(g.dy + (left ? (int64_t)i * g.ld : 0) + c, left != 0 && c < g.d);
          left &= left - 1;
        }
#pragma unroll
        for (int u = 0; u < kU; ++u)
#pragma unroll
          for (int e = 0; e < kE; ++e) acc[e] += v[u].get(e);   // (zeros where there is none)
      }
      Cols<float, kE>::put(&part[warp][lane * kE], acc);
      __syncthreads();
      for (int i = t; i < 32 * kE; i += kFew) {
        float sum = part[0][i];
#pragma unroll
        for (int w = 1; w < kWarps; ++w) sum += part[w][i];
        if (c0 + i < g.d) g.out[(int64_t)row * g.d + c0 + i] = Elem<O>::from_f(sum * g.scale);
      }
      __syncthreads();
    }
  }
}

// --------------------------------------------------------------------- host
constexpr int kLevels = 16;   // a level has at most a quarter of the entries before

// Sizes of a backward call and where its workspace's parts begin; e: columns a
// lane takes at once.
struct Plan {
  Split split;
  int32_t bits_all, bits, passes, rounds, chunk[kLevels], levels = 0;
  int64_t blocks, m[kLevels], run_blocks[kLevels];
  int64_t key[2], val[2], count, total, seen, part_key[kLevels], part[kLevels], bytes;
  Plan(int64_t n, int32_t vocab, int32_t d, int e) {
    split = split_cols(n, d, e);
    bits_all = 0;
    while (bits_all < 31 && (uint32_t)vocab >> bits_all) ++bits_all;
    passes = (int32_t)ceil_div(bits_all, kMaxBits);   // of the sort in many launches
    bits = std::max<int32_t>(8, (int32_t)ceil_div(bits_all, passes));
    rounds = n <= 2 * kSortThreads * 2 * kSms ? 2 : n <= 4 * kSortThreads * 4 * kSms ? 4 : 8;   // a wave or two of blocks
    blocks = ceil_div(n, kSortThreads * rounds);
    Carver c(nullptr);
    auto take = [&](int64_t b) {
      const int64_t at = c.used;
      c.take(b);
      return at;
    };
    for (int i = 0; i < 2; ++i) key[i] = take(n * 4), val[i] = take(n * 4);
    count = take(blocks * 4 << bits);
    total = take(4 << bits);
    seen = take(round_up(vocab, 16));
    for (int64_t left = n;;) {
      // entries a group: 16, or 32 where the blocks then fill the GPU all the same; one block takes what is
      // left once it can with 32
      const int64_t groups = (levels ? kJoinThreads : kRunThreads) >> split.shift;
      int64_t per = 16;
      while (levels == 0 && per < 32 && left > groups * per * 2 * kSms) per *= 2;
      per = std::min(per, kMostEntries / groups);
      if (levels && left <= std::min<int64_t>(32 * groups, kMostEntries)) per = std::max<int64_t>(1, ceil_div(left, groups));
      m[levels] = left, chunk[levels] = (int32_t)per, run_blocks[levels] = ceil_div(left, groups * per);
      left = 2 * run_blocks[levels];
      if (run_blocks[levels++] == 1 && levels > 1) break;   // (two at least: the second one zeroes)
      part_key[levels - 1] = take(left * 4), part[levels - 1] = take(left * d * 4);
    }
    bytes = c.used;
  }
};

// Of a call whatever its addresses allow.
int64_t plan_bytes(int64_t n, int32_t vocab, int32_t d) {
  int64_t most = 0;
  for (int e = 1; e <= 8 && d % e == 0; e *= 2) most = std::max(most, Plan(n, vocab, d, e).bytes);
  return most;
}

template <typename T, typename O>
cudaError_t run_level(RunArgs<T, O> a, const Split& s, int threads, int64_t zero_blocks, cudaStream_t st) {
  a.shift = s.shift;
  const int64_t across = ceil_div(a.d, s.width());
  const dim3 grid((unsigned)(a.run_blocks + ceil_div(zero_blocks, across)), (unsigned)across);
  const size_t smem = (size_t)2 * threads * s.e * s.items * 4 + (size_t)(threads >> s.shift) * a.chunk * 8;
  cudaError_t e = cudaSuccess;
  with_split(s, [&](auto c, auto i) {
    if (smem > 32 * 1024) {
      static OncePerDevice once;
      e = once([] {
        return cudaFuncSetAttribute(k_runs<T, O, decltype(c)::value, decltype(i)::value>,
                                    cudaFuncAttributeMaxDynamicSharedMemorySize, 128 * 1024);
      });
    }
    if (e == cudaSuccess) launch_pdl(k_runs<T, O, c.value, i.value>, grid, dim3((unsigned)threads), smem, st, a);
  });
  return e;
}

template <int kRounds, int kBits>
void sort_pass(const SortArgs& s, cudaStream_t st) {
  constexpr int bins = 1 << kBits;
  const dim3 grid((unsigned)s.blocks), block(kSortThreads);
  launch_pdl(k_sort_count<kRounds, kBits>, grid, block, 0, st, s);
  launch_pdl(k_sort_scan, dim3((unsigned)ceil_div(bins, 8)), dim3(256), 0, st, s.count, s.total, (int)s.blocks, bins);
  launch_pdl(k_sort_scatter<kRounds, kBits>, grid, block, (bins + 32) * 4 + bins * (kSortThreads / 32) * 2, st, s);
}

template <int kR>
cudaError_t sort_cluster(const SortArgs& s, cudaStream_t st) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(kCluster);
  cfg.blockDim = dim3(kClusterThreads);
  cfg.dynamicSmemBytes = cluster_smem<kR>();
  cfg.stream = st;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = kCluster;
  attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
  attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[1].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 2;
  static OncePerDevice once;
  const cudaError_t e = once([&] {
    cudaError_t a = cudaFuncSetAttribute(k_sort_cluster<kR>, cudaFuncAttributeMaxDynamicSharedMemorySize, cluster_smem<kR>());
    if (a == cudaSuccess) a = cudaFuncSetAttribute(k_sort_cluster<kR>, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
    int fit = 0;
    if (a == cudaSuccess) a = cudaOccupancyMaxActiveClusters(&fit, k_sort_cluster<kR>, &cfg);
    return a == cudaSuccess && fit < 1 ? cudaErrorNotSupported : a;
  });
  return e == cudaSuccess ? cudaLaunchKernelEx(&cfg, k_sort_cluster<kR>, s) : e;
}

template <typename T, typename O>
cudaError_t backward(const T* dy, int64_t lddy, const Ids& ids, int64_t n, int32_t d, float scale, O* out, char* ws,
                     cudaStream_t st) {
  int most = 8;
  while (most > 1 && !(fits(dy, lddy, d, sizeof(T), most) && fits(out, d, d, sizeof(O), most))) most /= 2;
  if (n <= kFew) {
    const FewArgs<T, O> a{ids, dy, out, lddy, (int32_t)n, d, scale};
    while (most > 1 && 16 * most >= d) most /= 2;   // (no idle lanes)
    const dim3 grid((unsigned)std::min(ids.vocab, 8 * kSms)), block(kFew);
    if (most == 8) launch_pdl(k_grad_few<T, O, 8>, grid, block, 0, st, a);
    else if (most == 4) launch_pdl(k_grad_few<T, O, 4>, grid, block, 0, st, a);
    else if (most == 2) launch_pdl(k_grad_few<T, O, 2>, grid, block, 0, st, a);
    else launch_pdl(k_grad_few<T, O, 1>, grid, block, 0, st, a);
    return cudaGetLastError();
  }
  const Plan p(n, ids.vocab, d, most);
  SortArgs s{};
  s.ids = ids, s.n = n, s.bits_all = p.bits_all, s.blocks = (int32_t)p.blocks;
  s.count = (uint32_t*)(ws + p.count), s.total = (uint32_t*)(ws + p.total), s.seen = (uint8_t*)(ws + p.seen);
  uint32_t* key[2] = {(uint32_t*)(ws + p.key[0]), (uint32_t*)(ws + p.key[1])};
  uint32_t* val[2] = {(uint32_t*)(ws + p.val[0]), (uint32_t*)(ws + p.val[1])};
  s.first = 1, s.key_out = key[0], s.val_out = val[0];
  cudaError_t e = cudaSuccess;
  int at = 0;
  const dim3 one(1 + (unsigned)std::min<int64_t>(ids.vocab >> 16, kSms));   // the block that sorts, and 64 KB to clear a block
  if (n <= kTileThreads) {
    launch_pdl(k_sort_tile<1>, one, dim3(kTileThreads), tile_smem<1>(), st, s);
  } else if (n <= 4 * kTileThreads) {
    static_assert(tile_smem<4>() <= 64 * 1024, "a block's shared memory");
    static OncePerDevice once;
    e = once([] { return cudaFuncSetAttribute(k_sort_tile<4>, cudaFuncAttributeMaxDynamicSharedMemorySize, 64 * 1024); });
    if (e != cudaSuccess) return e;
    launch_pdl(k_sort_tile<4>, one, dim3(kTileThreads), tile_smem<4>(), st, s);
  } else {
    e = n <= 2 * kCluster * kClusterThreads   ? sort_cluster<2>(s, st)
        : n <= 4 * kCluster * kClusterThreads ? sort_cluster<4>(s, st)
        : n <= 8 * kCluster * kClusterThreads ? sort_cluster<8>(s, st)
                                              : cudaErrorNotSupported;
    if (e == cudaErrorNotSupported) {   // too many, or a part of a GPU that no such cluster fits on
      cudaGetLastError();
      e = cudaSuccess;
      at = -1;
    }
  }
  if (e != cudaSuccess) return e;
  if (at < 0) {
    at = 0;
    for (int i = 0; i < p.passes; ++i) {
      s.first = i == 0, s.shift = i * p.bits;
      s.key = key[at ^ 1], s.val = val[at ^ 1], s.key_out = key[at], s.val_out = val[at];
      auto of_bits = [&](auto r) {
        if (p.bits == 8) sort_pass<r.value, 8>(s, st);
        else if (p.bits == 9) sort_pass<r.value, 9>(s, st);
        else sort_pass<r.value, kMaxBits>(s, st);
      };
      if (p.rounds == 2) of_bits(std::integral_constant<int, 2>());
      else if (p.rounds == 4) of_bits(std::integral_constant<int, 4>());
      else of_bits(std::integral_constant<int, 8>());
      at ^= 1;
    }
    at ^= 1;
  }
  const uint32_t *k = key[at], *v = val[at];
  for (int l = 0; l < p.levels; ++l) {
    const bool last = l + 1 == p.levels;
    auto fill = [&](auto& a) {
      a.key = k, a.val = v, a.out = out, a.m = p.m[l], a.chunk = p.chunk[l], a.run_blocks = (int32_t)p.run_blocks[l];
      a.key_out = last ? nullptr : (uint32_t*)(ws + p.part_key[l]), a.part = last ? nullptr : (float*)(ws + p.part[l]);
      a.d = d, a.vocab = ids.vocab, a.scale = scale, a.seen = s.seen, a.wide = fits(out, d, d, sizeof(O), 16 / sizeof(O)) && ids.vocab >= 32 * 32 * 2 * kSms;
    };
    if (l == 0) {
      RunArgs<T, O> a{};
      fill(a);
      a.src = dy, a.ld = lddy, a.first = 1;
      e = run_level(a, p.split, kRunThreads, 0, st);
    } else {
      RunArgs<float, O> a{};
      fill(a);
      a.src = (const float*)(ws + p.part[l - 1]), a.ld = d;
      const int64_t zero_blocks = l > 1 ? 0 : std::min<int64_t>(ceil_div((int64_t)ids.vocab * d, 1024 * 8), 2 * kSms);
      e = run_level(a, p.split, kJoinThreads, zero_blocks, st);
    }
    if (e != cudaSuccess) return e;
    if (!last) k = (const uint32_t*)(ws + p.part_key[l]), v = nullptr;
  }
  return cudaGetLastError();
}

template <typename T, typename O>
void lookup(const Ids& ids, int64_t n, const T* table, int64_t ldt, int32_t d, float scale, O* y, cudaStream_t st) {
  int most = 8;
  while (most > 1 && !(fits(table, ldt, d, sizeof(T), most) && fits(y, d, d, sizeof(O), most))) most /= 2;
  // no chains here: the widest loads
  Split s{most, 0, most == 1 ? (int)std::min<int64_t>(4, ceil_div(d, 32)) : 1};
  while (s.shift < 5 && (s.e << s.shift) < d) ++s.shift;
  LookArgs<T, O> a{ids, table, y, n, ldt, d, s.shift, scale};
  if (most == 1 && n >= kFlatFrom && ((uintptr_t)y & 15) == 0) {
    const int64_t share = std::max<int64_t>(8, ceil_div(n, 2 * kSms) / 8 * 8);   // no fewer blocks than two an SM
    const int tokens = (int)std::min<int64_t>(std::min(kFlatTokens, std::max(8, 8192 / d / 8 * 8)), share);
    launch_pdl(k_lookup_flat<T, O>, dim3((unsigned)ceil_div(n, tokens)), dim3(256), 0, st, a, tokens);
    return;
  }
  // no more blocks than run at once, which take the same number of turns
  const int64_t turns = ceil_div(n, (int64_t)(256 >> s.shift) * 2), each = ceil_div(turns, 8 * kSms);
  const dim3 grid((unsigned)ceil_div(turns, each), (unsigned)ceil_div(d, s.width()));
  with_split(s, [&](auto c, auto i) { launch_pdl(k_lookup<T, O, c.value, i.value>, grid, dim3(256), 0, st, a); });
}

tp_status check(int64_t n, int32_t id_bytes, int32_t vocab, int32_t d) {
  if (n < 0 || n > kMaxN) return ops_fail(TP_EINVAL, "n %lld out of range", (long long)n);
  if (id_bytes != 4 && id_bytes != 8) return ops_fail(TP_EINVAL, "ids must be of 4 or 8 bytes, not %d", id_bytes);
  if (vocab < 1 || vocab > (int32_t)kMaxN) return ops_fail(TP_EINVAL, "vocab %d must be in 1..%lld", vocab, (long long)kMaxN);
  if (d < 1 || d > kMaxD) return ops_fail(TP_EINVAL, "d %d must be in 1..%d", d, kMaxD);
  if (n * d > kMaxElems || (int64_t)vocab * d > kMaxElems) return ops_fail(TP_EINVAL, "more than 2^40 elements in a matrix");
  return TP_OK;
}
bool known(int32_t precision) { return precision == TP_BF16 || precision == TP_FP32; }

tp_status done(cudaError_t e, const char* who) {
  if (e == cudaSuccess) return TP_OK;
  cudaGetLastError();   // reported here
  return ops_fail(TP_ECUDA, "%s: %s", who, cudaGetErrorString(e));
}
using Half = __nv_bfloat16;

}  // namespace

extern "C" {

tp_status pack_embed(const void* ids, int32_t id_bytes, int64_t n, const void* table, int64_t ldt, int32_t vocab, int32_t d,
                     float scale, int32_t table_precision, int32_t precision, void* y, void* cuda_stream) {
  tp_status s = check(n, id_bytes, vocab, d);
  if (s != TP_OK) return s;
  if (!known(table_precision) || !known(precision))
    return ops_fail(TP_EINVAL, "unknown precision %d", known(precision) ? table_precision : precision);
  if (ldt < d) return ops_fail(TP_EINVAL, "ldt %lld is less than d %d", (long long)ldt, d);
  if (n == 0) return TP_OK;
  if (!ids || !table || !y) return ops_fail(TP_EINVAL, "null argument");
  if ((uintptr_t)ids & (id_bytes - 1)) return ops_fail(TP_EINVAL, "ids must be aligned to their size");
  if ((s = ops_device()) != TP_OK) return s;
  cudaStream_t st = (cudaStream_t)cuda_stream;
  const Ids i{ids, id_bytes == 8, vocab};
  if (table_precision == TP_FP32) {
    if (precision == TP_FP32) lookup(i, n, (const float*)table, ldt, d, scale, (float*)y, st);
    else lookup(i, n, (const float*)table, ldt, d, scale, (Half*)y, st);
  } else {
    if (precision == TP_FP32) lookup(i, n, (const Half*)table, ldt, d, scale, (float*)y, st);
    else lookup(i, n, (const Half*)table, ldt, d, scale, (Half*)y, st);
  }
  return done(cudaGetLastError(), "pack_embed");
}

tp_status pack_embed_bytes(int64_t n, int32_t vocab, int32_t d, int64_t* backward_bytes) {
  const tp_status s = check(n, 4, vocab, d);
  if (s != TP_OK) return s;
  if (!backward_bytes) return ops_fail(TP_EINVAL, "null argument");
  *backward_bytes = n > kFew ? plan_bytes(n, vocab, d) : 0;
  return TP_OK;
}

tp_status pack_embed_backward(const void* dy, int64_t lddy, const void* ids, int32_t id_bytes, int64_t n, int32_t vocab,
                              int32_t d, float scale, int32_t precision, int32_t table_precision, void* dtable,
                              void* workspace, int64_t workspace_bytes, void* cuda_stream) {
  tp_status s = check(n, id_bytes, vocab, d);
  if (s != TP_OK) return s;
  if (!known(table_precision) || !known(precision))
    return ops_fail(TP_EINVAL, "unknown precision %d", known(precision) ? table_precision : precision);
  if (lddy < d) return ops_fail(TP_EINVAL, "lddy %lld is less than d %d", (long long)lddy, d);
  if (!dtable) return ops_fail(TP_EINVAL, "null argument");
  cudaStream_t st = (cudaStream_t)cuda_stream;
  if (n == 0) {   // sums over no tokens
    if ((s = ops_device()) != TP_OK) return s;
    return done(cudaMemsetAsync(dtable, 0, (size_t)vocab * d * (table_precision == TP_FP32 ? 4 : 2), st),
                "pack_embed_backward");
  }
  if (!dy || !ids) return ops_fail(TP_EINVAL, "null argument");
  if ((uintptr_t)ids & (id_bytes - 1)) return ops_fail(TP_EINVAL, "ids must be aligned to their size");
  const int64_t need = n > kFew ? plan_bytes(n, vocab, d) : 0;
  if (need && (workspace_bytes < need || !workspace || ((uintptr_t)workspace & 255)))
    return ops_fail(TP_EINVAL, "a workspace of %lld bytes, 256-byte aligned, is needed", (long long)need);
  if ((s = ops_device()) != TP_OK) return s;
  const Ids i{ids, id_bytes == 8, vocab};
  char* ws = (char*)workspace;
  cudaError_t e;
  if (precision == TP_FP32) {
    if (table_precision == TP_FP32) e = backward((const float*)dy, lddy, i, n, d, scale, (float*)dtable, ws, st);
    else e = backward((const float*)dy, lddy, i, n, d, scale, (Half*)dtable, ws, st);
  } else {
    if (table_precision == TP_FP32) e = backward((const Half*)dy, lddy, i, n, d, scale, (float*)dtable, ws, st);
    else e = backward((const Half*)dy, lddy, i, n, d, scale, (Half*)dtable, ws, st);
  }
  return done(e, "pack_embed_backward");
}

}  // extern "C"
