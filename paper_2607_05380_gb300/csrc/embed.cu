// embed.cu -- embedding lookup with scaling, and the table's gradient by sorted
// tokens (entry points in tabpack_ops.h).
//
//   y[i] = scale table[ids[i]],   dtable[v] = scale sum_{i: ids[i] = v} dy[i]
//
// Lookup: a gather, bound by HBM; a few lanes a token, several tokens in flight.
//
// Gradient: the tokens are sorted by id (radix sort, stable), so that each row of
// the gradient is the sum of a run of tokens and is written once, in a fixed
// order of additions, without atomics on values.  A group of lanes adds up a
// chunk of C sorted tokens: runs inside the chunk are finished there; a run
// that crosses its ends leaves a 32-bit partial row, at most two a chunk, and
// these are a sorted list again, which the same kernel takes until one chunk is
// left.  A value with many thousands of tokens is so spread over the GPU like
// any others.  Rows without a token are zeroed beside the first level's sums: a
// bit per row says which they are.
#include <algorithm>

#include "lanes.cuh"
#include "prod.cuh"

using namespace tp;

namespace {

constexpr int32_t kMaxD = 1 << 17;
constexpr int64_t kMaxN = (int64_t(1) << 31) - 4096, kMaxElems = int64_t(1) << 40;
constexpr uint32_t kSkip = 0x80000000u;   // an entry of the partial rows that holds nothing

struct Ids {
  const void* p;
  int32_t wide, vocab;
  // the id, or vocab for one outside the table
  __device__ __forceinline__ uint32_t at(int64_t i) const {
    const int64_t v = wide ? ((const int64_t*)p)[i] : (int64_t)((const int32_t*)p)[i];
    return v >= 0 && v < vocab ? (uint32_t)v : (uint32_t)vocab;
  }
};

// kE = 8 columns by 16-byte loads and stores, or one.
template <typename T, int kE>
__device__ __forceinline__ void load_cols(const T* p, float (&v)[kE], bool there) {
  if constexpr (kE == 1) {
    v[0] = there ? Elem<T>::to_f(p[0]) : 0.f;
  } else {
    Lane<T, 1, 1, 8> l;
    l.load(p, 0, there ? 8 : 0);
    l.get(0, v);
  }
}
template <typename T, int kE>
__device__ __forceinline__ void store_cols(T* p, const float (&v)[kE]) {
  if constexpr (kE == 1) p[0] = Elem<T>::from_f(v[0]);
  else Lane<T, 1, 1, 8>::put(p, 0, 0, 8, v);
}

// Lanes a row (a power of two) and the columns they take together: kI groups
// of kE columns a lane.
struct Split {
  int shift, items;
};
Split split_cols(int d, int e) {
  const int groups = (int)ceil_div(d, e);
  Split best{5, 1};
  int64_t least = INT64_MAX;
  for (int items = 1; items <= (e == 1 ? 5 : 1); ++items)
    for (int shift = e == 1 && d >= 8 ? 3 : 0; shift <= 5; ++shift) {
      // idle lanes cost most, then the keys that every block of columns reads again
      const int64_t w = (int64_t)items << shift, cost = ceil_div(groups, w) * (w * 16 + 24) + (1 << shift) / 8;
      if (cost < least) least = cost, best = Split{shift, items};
    }
  return best;
}

// ------------------------------------------------------------------- lookup
template <typename T, typename O>
struct LookArgs {
  Ids ids;
  const T* table;
  O* y;
  int64_t n, ldt;
  int32_t d, shift, items;
  float scale;
};
template <typename T, typename O, int kE>
__global__ void __launch_bounds__(256) k_lookup(const LookArgs<T, O> g) {
  constexpr int kU = 4;   // tokens in flight
  const int lanes = 1 << g.shift, groups = 256 >> g.shift;
  const int at = threadIdx.x & (lanes - 1), grp = threadIdx.x >> g.shift;
  const int64_t t0 = (int64_t)blockIdx.x * (groups * kU) + grp;
  pdl_trigger();
  pdl_wait();
  uint32_t id[kU];
#pragma unroll
  for (int u = 0; u < kU; ++u) {
    const int64_t t = t0 + u * groups;
    id[u] = t < g.n ? g.ids.at(t) : (uint32_t)g.ids.vocab;
  }
  for (int i = 0; i < g.items; ++i) {
    const int64_t c = ((int64_t)blockIdx.y * g.items + i) * (lanes * kE) + at * kE;
    if (c >= g.d) break;
    float v[kU][kE];
#pragma unroll
    for (int u = 0; u < kU; ++u) {
      const bool there = id[u] < (uint32_t)g.ids.vocab;
      load_cols<T, kE>(g.table + (there ? (int64_t)id[u] * g.ldt : 0) + c, v[u], there);
    }
#pragma unroll
    for (int u = 0; u < kU; ++u) {
      const int64_t t = t0 + u * groups;
      if (t >= g.n) break;
      const bool there = id[u] < (uint32_t)g.ids.vocab;
#pragma unroll
      for (int e = 0; e < kE; ++e) v[u][e] = there ? v[u][e] * g.scale : 0.f;
      store_cols<O, kE>(g.y + t * g.d + c, v[u]);
    }
  }
}

// --------------------------------------------------------------------- sort
// A block takes a tile of kTile tokens, a warp 32 kRounds of them in order.
constexpr int kSortThreads = 512, kRounds = 8, kTile = kSortThreads * kRounds, kSortWarps = kSortThreads / 32;
constexpr int kMaxBits = 10;   // of a pass: the warps' counts of a digit's values fit in shared memory beside a tile

struct SortArgs {
  Ids ids;                      // the first pass's keys; their places are its values
  const uint32_t *key, *val;    // the later ones'
  uint32_t *key_out, *val_out;
  uint32_t *count, *total;      // [bins][blocks]; [bins]
  uint32_t* seen;               // a bit per row of the table
  int64_t n;
  int32_t first, last, shift, bits, blocks;
};
__device__ __forceinline__ uint32_t key_at(const SortArgs& g, int64_t i) { return g.first ? g.ids.at(i) : g.key[i]; }
__device__ __forceinline__ int64_t seen_words(const SortArgs& g) { return ((int64_t)g.ids.vocab + 31) >> 5; }
__device__ __forceinline__ void mark(const SortArgs& g, uint32_t key) {
  if (key >= (uint32_t)g.ids.vocab) return;
  uint32_t* w = g.seen + (key >> 5);
  if (!(*(volatile uint32_t*)w >> (key & 31) & 1)) atomicOr(w, 1u << (key & 31));   // frequent values: once, then reads
}

__global__ void __launch_bounds__(kSortThreads) k_sort_count(const SortArgs g) {
  __shared__ uint32_t h[1 << kMaxBits];
  pdl_trigger();
  pdl_wait();
  const int bins = 1 << g.bits;
  for (int i = threadIdx.x; i < bins; i += kSortThreads) h[i] = 0;
  __syncthreads();
#pragma unroll
  for (int r = 0; r < kRounds; ++r) {
    const int64_t i = (int64_t)blockIdx.x * kTile + r * kSortThreads + threadIdx.x;
    if (i < g.n) atomicAdd(&h[key_at(g, i) >> g.shift & (bins - 1)], 1u);
  }
  __syncthreads();
  for (int i = threadIdx.x; i < bins; i += kSortThreads) g.count[(int64_t)i * g.blocks + blockIdx.x] = h[i];
  if (g.first)
    for (int64_t i = (int64_t)blockIdx.x * kSortThreads + threadIdx.x; i < seen_words(g); i += (int64_t)g.blocks * kSortThreads)
      g.seen[i] = 0;
}

// Where each block's tokens of a digit begin among the digit's: a warp a digit.
__global__ void __launch_bounds__(256) k_sort_scan(uint32_t* count, uint32_t* total, int blocks, int bins) {
  pdl_trigger();
  pdl_wait();
  const int bin = blockIdx.x * 8 + (threadIdx.x >> 5), lane = threadIdx.x & 31;
  if (bin >= bins) return;
  uint32_t* row = count + (int64_t)bin * blocks;
  uint32_t before = 0;
  for (int b = 0; b < blocks; b += 32) {
    const uint32_t c = b + lane < blocks ? row[b + lane] : 0u;
    uint32_t s = c;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const uint32_t v = __shfl_up_sync(0xffffffffu, s, o);
      if (lane >= o) s += v;
    }
    if (b + lane < blocks) row[b + lane] = before + s - c;
    before += __shfl_sync(0xffffffffu, s, 31);
  }
  if (lane == 0) total[bin] = before;
}

// Exclusive prefix sums of v[0 .. bins - 1] in shared memory, by the whole block.
__device__ __forceinline__ void block_scan(uint32_t* v, int bins, uint32_t* warps) {
  constexpr int kPer = (1 << kMaxBits) / kSortThreads;
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
  uint32_t before = t - s;
  for (int w = 0; w < warp; ++w) before += warps[w];
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
// the warps before it, and sum (if wanted) the block's counts.
__device__ __forceinline__ void rank_tile(const uint32_t (&key)[kRounds], int shift, int bits, uint16_t* wh, uint32_t* sum,
                                          uint32_t (&rank)[kRounds]) {
  const int bins = 1 << bits, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  for (int i = threadIdx.x; i < bins * kSortWarps; i += kSortThreads) wh[i] = 0;
  __syncthreads();
  uint16_t* mine = wh + warp * bins;
#pragma unroll
  for (int r = 0; r < kRounds; ++r) {
    const uint32_t digit = key[r] >> shift & (bins - 1);
    uint32_t same = 0xffffffffu;
    for (int b = 0; b < bits; ++b) {
      const uint32_t set = __ballot_sync(0xffffffffu, digit >> b & 1);
      same &= digit >> b & 1 ? set : ~set;
    }
    const uint32_t before = mine[digit], lower = same & ((1u << lane) - 1);
    rank[r] = before + __popc(lower);
    __syncwarp();
    if (lower == 0) mine[digit] = (uint16_t)(before + __popc(same));
    __syncwarp();
  }
  __syncthreads();
  for (int i = threadIdx.x; i < bins; i += kSortThreads) {
    uint32_t s = 0;
#pragma unroll
    for (int w = 0; w < kSortWarps; ++w) {
      const uint32_t c = wh[w * bins + i];
      wh[w * bins + i] = (uint16_t)s;
      s += c;
    }
    if (sum) sum[i] = s;
  }
  __syncthreads();
}

__global__ void __launch_bounds__(kSortThreads) k_sort_scatter(const SortArgs g) {
  extern __shared__ uint32_t sm[];
  uint32_t* base = sm;
  uint16_t* wh = (uint16_t*)(sm + (1 << g.bits) + 32);
  const int bins = 1 << g.bits, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  pdl_trigger();
  pdl_wait();
  const int64_t i0 = (int64_t)blockIdx.x * kTile + warp * (32 * kRounds) + lane;
  uint32_t key[kRounds], rank[kRounds];
#pragma unroll
  for (int r = 0; r < kRounds; ++r) key[r] = i0 + 32 * r < g.n ? key_at(g, i0 + 32 * r) : 0xffffffffu;
  for (int i = threadIdx.x; i < bins; i += kSortThreads) base[i] = g.total[i];
  __syncthreads();
  block_scan(base, bins, sm + bins);
  for (int i = threadIdx.x; i < bins; i += kSortThreads) base[i] += g.count[(int64_t)i * g.blocks + blockIdx.x];
  rank_tile(key, g.shift, g.bits, wh, nullptr, rank);
#pragma unroll
  for (int r = 0; r < kRounds; ++r) {
    const int64_t i = i0 + 32 * r;
    if (i >= g.n) break;
    const uint32_t digit = key[r] >> g.shift & (bins - 1);
    const uint32_t to = base[digit] + wh[warp * bins + digit] + rank[r];
    g.key_out[to] = key[r];
    g.val_out[to] = g.first ? (uint32_t)i : g.val[i];
    if (g.last) mark(g, key[r]);
  }
}

// Up to kTile tokens: every pass in one block.
__global__ void __launch_bounds__(kSortThreads) k_sort_tile(const SortArgs g, int bits_all) {
  extern __shared__ uint32_t sm[];
  uint32_t *ks = sm, *vs = sm + kTile, *base = vs + kTile;
  uint16_t* wh = (uint16_t*)(base + (1 << g.bits) + 32);
  const int bins = 1 << g.bits, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  pdl_trigger();
  pdl_wait();
  const int i0 = warp * (32 * kRounds) + lane;
  uint32_t key[kRounds], val[kRounds], rank[kRounds];
#pragma unroll
  for (int r = 0; r < kRounds; ++r) {
    val[r] = i0 + 32 * r;
    key[r] = (int)val[r] < g.n ? key_at(g, val[r]) : 0xffffffffu;   // (behind all others in every pass)
  }
  for (int64_t i = threadIdx.x; i < seen_words(g); i += kSortThreads) g.seen[i] = 0;
  for (int shift = 0; shift < bits_all; shift += g.bits) {
    rank_tile(key, shift, g.bits, wh, base, rank);
    block_scan(base, bins, base + bins);
#pragma unroll
    for (int r = 0; r < kRounds; ++r) {
      const uint32_t digit = key[r] >> shift & (bins - 1);
      const uint32_t to = base[digit] + wh[warp * bins + digit] + rank[r];
      ks[to] = key[r], vs[to] = val[r];
    }
    __syncthreads();
#pragma unroll
    for (int r = 0; r < kRounds; ++r) key[r] = ks[i0 + 32 * r], val[r] = vs[i0 + 32 * r];
    __syncthreads();
  }
#pragma unroll
  for (int r = 0; r < kRounds; ++r) {
    const int i = i0 + 32 * r;
    if (i >= g.n) break;
    g.key_out[i] = key[r], g.val_out[i] = val[r];
    mark(g, key[r]);
  }
}

// --------------------------------------------------------------------- runs
template <typename T, typename O>
struct RunArgs {
  const uint32_t *key, *val;    // val: the rows of src (NULL: one after another)
  const T* src;
  O* out;
  uint32_t* key_out;            // two entries a chunk
  float* part;
  const uint32_t* seen;         // first level: rows to be zeroed (NULL: none)
  int64_t m, ld, chunks;
  int32_t chunk, d, vocab, shift, items, run_blocks;
  float scale;
};

template <typename O, int kE>
__device__ __forceinline__ void zero_rows(const uint32_t* seen, O* out, int64_t vocab, int d, int shift, int64_t block,
                                          int64_t blocks) {
  const int lanes = 1 << shift, at = threadIdx.x & (lanes - 1);
  const float zero[kE] = {};
  for (int64_t r = block * (256 >> shift) + (threadIdx.x >> shift); r < vocab; r += blocks * (256 >> shift)) {
    if (seen[r >> 5] >> (r & 31) & 1) continue;
    for (int64_t c = at * kE; c < d; c += lanes * kE) store_cols<O, kE>(out + r * d + c, zero);
  }
}

// A group of lanes takes a chunk of the sorted list and kI * kE of their
// columns each.
template <typename T, typename O, int kE, int kI>
__global__ void __launch_bounds__(256) k_runs(const RunArgs<T, O> g) {
  constexpr int kU = kE == 1 ? 8 : 4;   // rows in flight
  pdl_trigger();
  pdl_wait();
  if ((int)blockIdx.x >= g.run_blocks) {
    if (blockIdx.y == 0)
      zero_rows<O, kE>(g.seen, g.out, g.vocab, g.d, g.shift, blockIdx.x - g.run_blocks, gridDim.x - g.run_blocks);
    return;
  }
  const int lanes = 1 << g.shift, at = threadIdx.x & (lanes - 1);
  const int64_t q = (int64_t)blockIdx.x * (256 >> g.shift) + (threadIdx.x >> g.shift);
  if (q >= g.chunks) return;
  const int64_t first = q * g.chunk, end = min(first + g.chunk, g.m);
  const int64_t c0 = (int64_t)blockIdx.y * kI * (lanes * kE) + at * kE;
  const uint32_t none = 0xffffffffu;
  const uint32_t before = first ? g.key[first - 1] & ~kSkip : none, after = end < g.m ? g.key[end] & ~kSkip : none;
  uint32_t cur = g.key[first] & ~kSkip;
  // what the chunk leaves in its two entries: nothing yet
  uint32_t left0 = cur | kSkip, left1 = kSkip;
  float acc[kI][kE];
  bool any = false, head = true;
  auto clear = [&] {
#pragma unroll
    for (int i = 0; i < kI; ++i)
#pragma unroll
      for (int e = 0; e < kE; ++e) acc[i][e] = 0.f;
    any = false;
  };
  auto finish = [&](bool tail) {
    const bool from = head && before == cur, on = tail && after == cur;
    if (any) {
      if (!from && !on) {
#pragma unroll
        for (int i = 0; i < kI; ++i) {
          const int64_t c = c0 + (int64_t)i * (lanes * kE);
          float v[kE];
#pragma unroll
          for (int e = 0; e < kE; ++e) v[e] = acc[i][e] * g.scale;
          if (c < g.d) store_cols<O, kE>(g.out + (int64_t)cur * g.d + c, v);
        }
      } else {
#pragma unroll
        for (int i = 0; i < kI; ++i) {
          const int64_t c = c0 + (int64_t)i * (lanes * kE);
          if (c < g.d) store_cols<float, kE>(g.part + (2 * q + (from ? 0 : 1)) * g.d + c, acc[i]);
        }
        if (from) left0 = cur;
        else left1 = cur;
      }
    }
    head = false;
  };
  clear();
  for (int64_t i0 = first; i0 < end; i0 += kU) {
    uint32_t key[kU];
    float v[kU][kI][kE];
#pragma unroll
    for (int u = 0; u < kU; ++u) key[u] = i0 + u < end ? g.key[i0 + u] : none;
#pragma unroll
    for (int u = 0; u < kU; ++u) {
      const bool there = key[u] < (uint32_t)g.vocab;   // (neither skipped nor outside the table)
      const int64_t row = !there ? 0 : g.val ? (int64_t)g.val[i0 + u] : i0 + u;
#pragma unroll
      for (int i = 0; i < kI; ++i) {
        const int64_t c = c0 + (int64_t)i * (lanes * kE);
        load_cols<T, kE>(g.src + row * g.ld + c, v[u][i], there && c < g.d);
      }
    }
#pragma unroll
    for (int u = 0; u < kU; ++u) {
      if (i0 + u >= end) break;
      const uint32_t k = key[u] & ~kSkip;
      if (k != cur) {
        finish(false);
        clear();
        cur = k;
      }
      if (key[u] < (uint32_t)g.vocab) {
        any = true;
#pragma unroll
        for (int i = 0; i < kI; ++i)
#pragma unroll
          for (int e = 0; e < kE; ++e) acc[i][e] += v[u][i][e];
      }
    }
  }
  finish(true);
  if (g.key_out && at == 0 && blockIdx.y == 0) {
    g.key_out[2 * q] = left0;
    g.key_out[2 * q + 1] = left1 == kSkip ? cur | kSkip : left1;
  }
}

// --------------------------------------------------------------------- host
// Sizes of a backward call and where its workspace's parts begin.
constexpr int kLevels = 12;   // a level has at most an eighth of the entries before
struct Plan {
  int32_t bits_all, bits, passes, chunk[kLevels], levels = 0;
  int64_t blocks, m[kLevels];
  int64_t key[2], val[2], count, total, seen, part_key[kLevels], part[kLevels], bytes;
  Plan(int64_t n, int32_t vocab, int32_t d) {
    bits_all = 0;
    while (bits_all < 31 && (uint32_t)vocab >> bits_all) ++bits_all;
    passes = (int32_t)ceil_div(bits_all, kMaxBits);
    bits = (int32_t)ceil_div(bits_all, passes);
    blocks = ceil_div(n, kTile);
    Carver c(nullptr);
    auto take = [&](int64_t b) {
      const int64_t at = c.used;
      c.take(b);
      return at;
    };
    for (int i = 0; i < 2; ++i) key[i] = take(n * 4), val[i] = take(n * 4);
    count = take(blocks * 4 << bits);
    total = take(4 << bits);
    seen = take(ceil_div(vocab, 32) * 4);
    // tokens a chunk: enough chunks for every lane of the GPU, but partial rows are written and read again
    int64_t left = n;
    do {
      int64_t c2 = 16;
      while (c2 < 64 && ceil_div(left, 2 * c2) * std::min<int64_t>(d, 256) >= int64_t(kSms) * 2048 * 4) c2 *= 2;
      chunk[levels] = (int32_t)c2;
      m[levels] = left;
      left = 2 * ceil_div(left, c2);
      if (m[levels] > c2) part_key[levels] = take(left * 4), part[levels] = take(left * d * 4);
      ++levels;
    } while (m[levels - 1] > chunk[levels - 1]);
    bytes = c.used;
  }
};

template <typename T, typename O, int kE>
void run_level(RunArgs<T, O> a, int64_t zero_blocks, cudaStream_t st) {
  const Split s = split_cols(a.d, kE);
  a.shift = s.shift, a.items = s.items;
  a.run_blocks = (int32_t)ceil_div(a.chunks, 256 >> s.shift);
  const dim3 grid((unsigned)(a.run_blocks + zero_blocks), (unsigned)ceil_div(a.d, (int64_t)s.items * kE << s.shift));
  if constexpr (kE == 8) {
    launch_pdl(k_runs<T, O, 8, 1>, grid, dim3(256), 0, st, a);
  } else {
    if (s.items == 1) launch_pdl(k_runs<T, O, 1, 1>, grid, dim3(256), 0, st, a);
    else if (s.items == 2) launch_pdl(k_runs<T, O, 1, 2>, grid, dim3(256), 0, st, a);
    else if (s.items == 3) launch_pdl(k_runs<T, O, 1, 3>, grid, dim3(256), 0, st, a);
    else if (s.items == 4) launch_pdl(k_runs<T, O, 1, 4>, grid, dim3(256), 0, st, a);
    else launch_pdl(k_runs<T, O, 1, 5>, grid, dim3(256), 0, st, a);
  }
}

template <typename T, typename O>
void backward(const T* dy, int64_t lddy, const Ids& ids, int64_t n, int32_t d, float scale, O* out, char* ws, cudaStream_t st) {
  const Plan p(n, ids.vocab, d);
  SortArgs s{};
  s.ids = ids, s.n = n, s.bits = p.bits, s.blocks = (int32_t)p.blocks;
  s.count = (uint32_t*)(ws + p.count), s.total = (uint32_t*)(ws + p.total), s.seen = (uint32_t*)(ws + p.seen);
  uint32_t* key[2] = {(uint32_t*)(ws + p.key[0]), (uint32_t*)(ws + p.key[1])};
  uint32_t* val[2] = {(uint32_t*)(ws + p.val[0]), (uint32_t*)(ws + p.val[1])};
  const int bins = 1 << p.bits;
  const size_t sm = (size_t)(bins + 32) * 4 + (size_t)bins * kSortWarps * 2;
  int at = 0;
  if (n <= kTile) {
    s.first = s.last = 1, s.key_out = key[0], s.val_out = val[0];
    const size_t all = sm + 2 * kTile * 4;
    cudaFuncSetAttribute(k_sort_tile, cudaFuncAttributeMaxDynamicSharedMemorySize, 96 * 1024);
    launch_pdl(k_sort_tile, dim3(1), dim3(kSortThreads), all, st, s, (int)p.bits_all);
  } else {
    for (int i = 0; i < p.passes; ++i) {
      s.first = i == 0, s.last = i + 1 == p.passes, s.shift = i * p.bits;
      s.key = key[at ^ 1], s.val = val[at ^ 1], s.key_out = key[at], s.val_out = val[at];
      launch_pdl(k_sort_count, dim3((unsigned)p.blocks), dim3(kSortThreads), 0, st, s);
      launch_pdl(k_sort_scan, dim3((unsigned)ceil_div(bins, 8)), dim3(256), 0, st, s.count, s.total, (int)p.blocks, bins);
      launch_pdl(k_sort_scatter, dim3((unsigned)p.blocks), dim3(kSortThreads), sm, st, s);
      at ^= 1;
    }
    at ^= 1;
  }
  const bool out_ok = d % 8 == 0 && aligned16(out, 0, 4), in_ok = aligned16(dy, lddy, sizeof(T));
  const uint32_t *k = key[at], *v = val[at];
  for (int l = 0; l < p.levels; ++l) {
    const bool last = l + 1 == p.levels;
    auto fill = [&](auto& a) {
      a.key = k, a.val = v, a.out = out, a.m = p.m[l], a.chunk = p.chunk[l], a.chunks = ceil_div(p.m[l], p.chunk[l]);
      a.key_out = last ? nullptr : (uint32_t*)(ws + p.part_key[l]), a.part = last ? nullptr : (float*)(ws + p.part[l]);
      a.d = d, a.vocab = ids.vocab, a.scale = scale;
    };
    if (l == 0) {
      RunArgs<T, O> a{};
      fill(a);
      a.src = dy, a.ld = lddy, a.seen = s.seen;
      const int64_t zero_blocks = std::min<int64_t>(ceil_div((int64_t)ids.vocab * d, 256 * 64), 4 * kSms);
      if (out_ok && in_ok) run_level<T, O, 8>(a, zero_blocks, st);
      else run_level<T, O, 1>(a, zero_blocks, st);
    } else {
      RunArgs<float, O> a{};
      fill(a);
      a.src = (const float*)(ws + p.part[l - 1]), a.ld = d;
      if (out_ok) run_level<float, O, 8>(a, 0, st);
      else run_level<float, O, 1>(a, 0, st);
    }
    if (!last) k = (const uint32_t*)(ws + p.part_key[l]), v = nullptr;
  }
}

template <typename T, typename O>
void lookup(const Ids& ids, int64_t n, const T* table, int64_t ldt, int32_t d, float scale, O* y, cudaStream_t st) {
  const bool vec = d % 8 == 0 && aligned16(table, ldt, sizeof(T)) && aligned16(y, 0, 4);
  LookArgs<T, O> a{ids, table, y, n, ldt, d, 0, 0, scale};
  const Split s = split_cols(d, vec ? 8 : 1);
  a.shift = s.shift, a.items = s.items;
  const dim3 grid((unsigned)ceil_div(n, (int64_t)(256 >> s.shift) * 4), (unsigned)ceil_div(d, (int64_t)s.items * (vec ? 8 : 1) << s.shift));
  if (vec) launch_pdl(k_lookup<T, O, 8>, grid, dim3(256), 0, st, a);
  else launch_pdl(k_lookup<T, O, 1>, grid, dim3(256), 0, st, a);
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
  *backward_bytes = n ? Plan(n, vocab, d).bytes : 0;
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
  const int64_t need = Plan(n, vocab, d).bytes;
  if (workspace_bytes < need || !workspace || ((uintptr_t)workspace & 255))
    return ops_fail(TP_EINVAL, "a workspace of %lld bytes, 256-byte aligned, is needed", (long long)need);
  if ((s = ops_device()) != TP_OK) return s;
  const Ids i{ids, id_bytes == 8, vocab};
  char* ws = (char*)workspace;
  if (precision == TP_FP32) {
    if (table_precision == TP_FP32) backward((const float*)dy, lddy, i, n, d, scale, (float*)dtable, ws, st);
    else backward((const float*)dy, lddy, i, n, d, scale, (Half*)dtable, ws, st);
  } else {
    if (table_precision == TP_FP32) backward((const Half*)dy, lddy, i, n, d, scale, (float*)dtable, ws, st);
    else backward((const Half*)dy, lddy, i, n, d, scale, (Half*)dtable, ws, st);
  }
  return done(cudaGetLastError(), "pack_embed_backward");
}

}  // extern "C"
