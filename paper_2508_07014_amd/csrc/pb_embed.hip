// Rows of a table for tokens, scaled (pb_embed_tokens), and the table's gradient (pb_embed_tokens_backward).
#include <algorithm>

#include "pb_logit_rows.hpp"
#include "pb_student.hpp"

namespace pb {
namespace em {

using namespace lr;
using wv::first_lane;

// Elements that a lane takes at once: 16 bytes of the type that is written, so that the lanes of a store lie next to each other (lookup of 32768
// x 2048 fp32 rows into fp32 67 us, with 32 bytes a lane 93; 8 bytes a lane into bf16 52 instead of 46; the gradient of 16384 x 1024
// bf16 on 32001 fp32 rows 40 instead of 63).
template <typename From, typename To>
constexpr int step_of() { return To::N; }

// K (4 or 8) elements at p, any alignment of its elements, to and from fp32.
typedef unsigned v2u __attribute__((ext_vector_type(2)));
template <typename E, int K>
__device__ __forceinline__ void load_vector(const typename E::type* p, float (&x)[K]) {
  if constexpr (E::N == K) {
    E::unpack(any_vector<E>(p), x);
  } else if constexpr (K == 8) {
    float lo[4], hi[4];
    E::unpack(any_vector<E>(p), lo);
    E::unpack(any_vector<E>(p + 4), hi);
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = lo[i], x[4 + i] = hi[i];
  } else {
    typedef unsigned any2 __attribute__((ext_vector_type(2), aligned(2)));
    const v2u half = *reinterpret_cast<const any2*>(p);
    float both[8];
    E::unpack(v4u{half.x, half.y, 0u, 0u}, both);
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = both[i];
  }
}
template <typename E, bool STREAM, int K>
__device__ __forceinline__ void store_vector_of(typename E::type* p, const float (&x)[K]) {
  if constexpr (E::N == K) {
    if constexpr (STREAM) stream_vector<E>(p, E::pack(x));
    else store_vector<E>(p, E::pack(x));
  } else if constexpr (K == 8) {
    const float lo[4] = {x[0], x[1], x[2], x[3]}, hi[4] = {x[4], x[5], x[6], x[7]};
    store_vector<E>(p, E::pack(lo));
    store_vector<E>(p + 4, E::pack(hi));
  } else {
    typedef unsigned any2 __attribute__((ext_vector_type(2), aligned(2)));
    const float both[8] = {x[0], x[1], x[2], x[3], 0.0f, 0.0f, 0.0f, 0.0f};
    const v4u r = E::pack(both);
    __builtin_nontemporal_store(v2u{r.x, r.y}, reinterpret_cast<any2*>(p));
  }
}

// The columns of a lane: SL vectors of K, `lanes` lanes apart.  The last one of a row is loaded from dim - K on (nothing outside
// the row is touched), `skip` of it columns of the lane before; NARROW: dim < K, single elements.
template <int K, int SL, bool NARROW>
struct Columns {
  int at[SL], skip[SL], dim;  // skip = K: none
  __device__ __forceinline__ Columns(int dim_, int first, int lanes, int lane) : dim(dim_) {
#pragma unroll
    for (int s = 0; s < SL; ++s) {
      const int d = first + (s * lanes + lane) * K;
      at[s] = NARROW ? 0 : min(d, dim - K);
      skip[s] = min(K, NARROW ? (d > 0 ? K : 0) : d - at[s]);
    }
  }
  template <typename E>
  __device__ __forceinline__ void load(const typename E::type* row, int s, float (&x)[K]) const {
    if constexpr (NARROW) {
#pragma unroll
      for (int i = 0; i < K; ++i) x[i] = i < dim ? E::up(row[i]) : 0.0f;
    } else {
      load_vector<E>(row + at[s], x);
    }
  }
  template <typename E, bool STREAM = true>
  __device__ __forceinline__ void store(typename E::type* row, int s, const float (&x)[K]) const {
    if constexpr (NARROW) {
#pragma unroll
      for (int i = 0; i < K; ++i)
        if (skip[s] == 0 && i < dim) row[i] = E::down(x[i]);
      return;
    }
    if (skip[s] == 0) return store_vector_of<E, STREAM>(row + at[s], x);
#pragma unroll
    for (int i = 1; i < K; ++i)
      if (i >= skip[s]) row[at[s] + i] = E::down(x[i]);
  }
};

// Lanes that take a row: a power of 2, at most a wave.
int lanes_for(int dim, int step) {
  int lanes = 1;
  while (lanes < 64 && lanes * step < dim) lanes *= 2;
  return lanes;
}

// Rows for tokens, SL vectors of a lane at once.  Bound by HBM: 32768 x 2048 fp32 rows of 131072 into bf16 46 us, 134 MB written and about as much
// read; past the caches bf16 into bf16 32.5 us, through them 41.8.
template <typename E, typename O, int SL, bool NARROW>
__global__ __launch_bounds__(256) void embed_kernel(EmbedArgs a, int lanes) {
  constexpr int K = step_of<E, O>();
  const int64_t i = static_cast<int64_t>(blockIdx.x) * (256 / lanes) + threadIdx.x / lanes;
  if (i >= a.n) return;
  const int t = a.tokens[i];
  const bool there = static_cast<unsigned>(t) < static_cast<unsigned>(a.V);
  const typename E::type* from = static_cast<const typename E::type*>(a.table) + (there ? t : 0) * a.table_stride;
  typename O::type* to = static_cast<typename O::type*>(a.out) + i * a.out_stride;
  const Columns<K, SL, NARROW> cols(a.dim, blockIdx.y * lanes * K * SL, lanes, threadIdx.x & (lanes - 1));
  float x[SL][K] = {};
  if (there) {
#pragma unroll
    for (int u = 0; u < SL; ++u) cols.template load<E>(from, u, x[u]);
  }
#pragma unroll
  for (int u = 0; u < SL; ++u) {
#pragma unroll
    for (int k = 0; k < K; ++k) x[u][k] = there ? product(x[u][k], a.scale) : 0.0f;
    cols.template store<O>(to, u, x[u]);
  }
}

// The gradient: positions sorted by token, then sums over each token's positions.
//
// Sorting.  A workgroup takes a range of the vocabulary, 2^shift tokens, and reads all tokens: those of its range it counts, for each
// wave's share of the positions apart, and places in a second pass; those below its range it counts for the place its range
// begins at.  So the order is that of the positions, without an atomic on memory and with one launch.  Reading all tokens in every
// workgroup takes time with their number (16384 of them: 9 us, 131072: 42), so from kManyTokens on the positions are
// split by range first, in chunks: then a workgroup reads its own alone (131072: 7 and 16 us).  Gradients of 32001 x 256 fp32, split / not:
// 24000 tokens 32.9 / 28.5 us, 36000 36.2 / 32.6, 48000 37.9 / 37.8, 64000 41.4 / 42.2, 90000 58.5 / 61.3.
constexpr int kSortThreads = 1024, kSortWaves = kSortThreads / 64;
constexpr int kAhead = 16, kTail = 4;  // tokens that a lane requests at once, and of the last ones
constexpr int kMaxShift = 9;    // (ranges of 512 tokens: 32 KiB of counts)
constexpr int kMaxRanges = (kLogitsMaxV + (1 << kMaxShift) - 1) >> kMaxShift;
static_assert(kMaxRanges <= kSortThreads, "a thread a range");
constexpr int kManyTokens = 40960;
constexpr int kSplit = 4096;    // positions of a chunk at most: 12 bits beside those of a token in its range
// Positions of a chunk, so that the waves that merge them have as many each (67251 x 40 on 193 rows 47.0 -> 41.8 us, 200000 x 64 on
// 32001 51.6 -> 48.3; always kSplit of them before).
int64_t turns_for(int n) { return (static_cast<int64_t>(n) + kSortWaves * kSplit - 1) / (kSortWaves * kSplit); }
int span_for(int n) {
  const int64_t chunks = kSortWaves * turns_for(n);
  return static_cast<int>(((n + chunks - 1) / chunks + 63) / 64 * 64);
}

// Workgroups a range: the one with the most frequent token takes longest, and two of them place half the positions each (they count all).  Two /
// one: 8000 x 640 fp32 on 8192 rows 22.9 / 24.4 us, 40000 x 128 on 4097 28.8 / 31.2; where the ranges are as many as CUs already 16000 x 64 on
// 131072 26.9 / 25.3.
int parts_for(int n, int V) { return n >= 4096 && n < kManyTokens && V <= 128 << kMaxShift ? 2 : 1; }
int shift_for(int n, int V) {  // about as many workgroups as there are CUs
  int shift = 0;
  while (shift < kMaxShift && ((V - 1) >> shift) >= 256 / parts_for(n, V)) ++shift;
  return shift;
}

// Sums of all threads' values up to each (`total`: of all); s: a place a wave.
__device__ __forceinline__ int group_upto(int v, int* s, int* total) {
  const int lane = threadIdx.x & 63, wave = uniform_i(threadIdx.x >> 6);
  int upto = v;
#pragma unroll
  for (int d = 1; d < 64; d *= 2) {
    const int w = __shfl_up(upto, d, 64);
    if (lane >= d) upto += w;
  }
  __syncthreads();
  if (lane == 63) s[wave] = upto;
  __syncthreads();
  int ahead = 0, all = 0;
  for (int w = 0; w < kSortWaves; ++w) {
    if (w < wave) ahead += s[w];
    all += s[w];
  }
  *total = all;
  return ahead + upto;
}

// Tokens of a range that occur more than kFew times, for the launch that joins their pieces (in any order).
constexpr int kFew = 32;
struct Owner {
  int v, begin, end;
};
struct Owners {
  int32_t* count;  // [ranges]
  Owner* list;     // [ranges << shift]
};
// By all threads of the range's workgroup, the thread's own token with its places (n: a place in LDS).
__device__ __forceinline__ void write_owners(const Owners& o, int range, int v0, int size, int at, int end, int* n) {
  const int tid = threadIdx.x;
  if (tid == 0) *n = 0;
  __syncthreads();
  if (tid < size && end - at > kFew) o.list[v0 + atomicAdd(n, 1)] = Owner{v0 + tid, at, end};
  __syncthreads();
  if (tid == 0) o.count[range] = *n;
}

// counts[wave][i], i < size: how many of each wave; becomes the place of the wave's first, `base` ahead of them all.  Returns
// the place of the thread's i (and in *end what follows it).  PARTS: two more rows of counts, of what lies ahead of all waves' and behind.
template <bool PARTS = false>
__device__ __forceinline__ int places(int* counts, int stride, int size, int base, int* s, int* end) {
  const int tid = threadIdx.x;
  int total = 0, all, ahead = 0, each[kSortWaves];
  if (tid < size) {
    if (PARTS) {
      ahead = counts[kSortWaves * stride + tid];
      total = ahead + counts[(kSortWaves + 1) * stride + tid];
    }
#pragma unroll
    for (int w = 0; w < kSortWaves; ++w) each[w] = counts[w * stride + tid];
#pragma unroll
    for (int w = 0; w < kSortWaves; ++w) total += each[w];
  }
  const int first = base + group_upto(total, s, &all) - total;
  if (tid < size) {
    int at = first + ahead;
#pragma unroll
    for (int w = 0; w < kSortWaves; ++w) {
      counts[w * stride + tid] = at;
      at += each[w];
    }
  }
  *end = first + total;
  __syncthreads();
  return first;
}

// Counts a wave's keys (`in`: the lane has one) in the wave's own counters.  A token of many positions fills whole waves, whose additions to
// one place the LDS would take one after the other: the lanes with the first one's key are counted at once.
template <int ROUNDS>
__device__ __forceinline__ void count_keys(int* counters, unsigned key, bool in, int lane) {
  u64 left = __ballot(in);
  for (int round = 0; round < ROUNDS && left; ++round) {
    const unsigned k = static_cast<unsigned>(__builtin_amdgcn_readlane(static_cast<int>(key), first_lane(left)));
    const u64 same = left & __ballot(key == k);
    if (lane == 0) atomicAdd(&counters[k], __builtin_popcountll(same));
    left &= ~same;
  }
  if ((left >> lane) & 1) atomicAdd(&counters[key], 1);
}
// Places a wave's keys (of `bits` bits) at their counters, in the order of the lanes.  Which lanes have the same key is found key by key
// while there are few or one has many lanes, for what is left after that bit by bit; the counters are read and moved on once for all.
template <int ROUNDS, typename Put>
__device__ __forceinline__ void place_keys(int* counters, unsigned key, bool in, int bits, int lane, Put&& put) {
  u64 left = __ballot(in), same = 0;
  if (!left) return;
  for (int round = 0; left && (round < ROUNDS || __builtin_popcountll(left) <= 4); ++round) {
    const unsigned k = static_cast<unsigned>(__builtin_amdgcn_readlane(static_cast<int>(key), first_lane(left)));
    const u64 these = left & __ballot(key == k);
    if ((these >> lane) & 1) same = these;
    left &= ~these;
  }
  if (left) {
    u64 those = left;
    for (int b = 0; b < bits; ++b) {
      const bool one = (key >> b) & 1u;
      const u64 ones = __ballot(one);
      those &= one ? ones : ~ones;
    }
    if ((left >> lane) & 1) same = those;
  }
  if (in) {
    const int to = counters[key], rank = __builtin_popcountll(same & ((1ull << lane) - 1));
    __builtin_amdgcn_wave_barrier();
    if (rank == 0) counters[key] = to + __builtin_popcountll(same);
    put(to + rank);
  }
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}

__global__ __launch_bounds__(kSortThreads) void embed_sort_kernel(const int32_t* tokens, int n, int V, int shift, int32_t* begin, int32_t* order, Owners owners) {
  extern __shared__ int counts[];  // [kSortWaves + 2][2^shift]
  __shared__ int s[kSortWaves];
  const int tid = threadIdx.x, lane = tid & 63, wave = uniform_i(tid >> 6), range = 1 << shift, part = blockIdx.y, parts = gridDim.y;
  const int v0 = blockIdx.x << shift, size = min(range, V - v0);
  for (int i = tid; i < (kSortWaves + 2) * range; i += kSortThreads) counts[i] = 0;
  __syncthreads();
  const int shares = kSortWaves * parts, share = ((n + shares - 1) / shares + 63) / 64 * 64;
  const int p0 = min(n, (part * kSortWaves + wave) * share), p1 = min(n, p0 + share);
  int* mine = counts + wave * range;
  int below = 0;
  auto count = [&](int* to, int t) {  // (an id below 0 is a large one without its sign)
    const unsigned u = static_cast<unsigned>(t) - static_cast<unsigned>(v0);
    below += static_cast<unsigned>(t) < static_cast<unsigned>(v0);
    if (u < static_cast<unsigned>(size)) atomicAdd(&to[u], 1);
  };
  auto count_share = [&](int* to, int p, int end) {
    for (; p + 64 * kAhead <= end; p += 64 * kAhead) {
      int t[kAhead];
#pragma unroll
      for (int k = 0; k < kAhead; ++k) t[k] = tokens[p + 64 * k + lane];
#pragma unroll
      for (int k = 0; k < kAhead; ++k) count(to, t[k]);
    }
    for (; p < end; p += 64 * kTail) {
      int t[kTail];
#pragma unroll
      for (int k = 0; k < kTail; ++k) t[k] = p + 64 * k + lane < end ? tokens[p + 64 * k + lane] : -1;
#pragma unroll
      for (int k = 0; k < kTail; ++k) count(to, t[k]);
    }
  };
  for (int q = 0; q < parts; ++q) {
    const int from = min(n, (q * kSortWaves + wave) * share);
    count_share(q == part ? mine : counts + (q < part ? kSortWaves : kSortWaves + 1) * range, from, min(n, from + share));
  }
  int base, end;
  group_upto(below, s, &base);
  const int at = places<true>(counts, range, size, base, s, &end);
  if (part == 0) {
    if (tid < size) {
      begin[v0 + tid] = at;
      if (v0 + tid == V - 1) begin[V] = end;
    }
    write_owners(owners, blockIdx.x, v0, size, at, end, s);
  }
  auto put = [&](int t, int from) {
    const unsigned u = static_cast<unsigned>(t) - static_cast<unsigned>(v0);
    place_keys<1>(mine, u, u < static_cast<unsigned>(size), shift, lane, [&](int to) { order[to] = from; });
  };
  int p = p0;  // (the same in all lanes of a wave)
  for (; p + 64 * kAhead <= p1; p += 64 * kAhead) {
    int t[kAhead];
#pragma unroll
    for (int k = 0; k < kAhead; ++k) t[k] = tokens[p + 64 * k + lane];
#pragma unroll
    for (int k = 0; k < kAhead; ++k) put(t[k], p + 64 * k + lane);
  }
  for (; p < p1; p += 64 * kTail) {
    int t[kTail];
#pragma unroll
    for (int k = 0; k < kTail; ++k) t[k] = p + 64 * k + lane < p1 ? tokens[p + 64 * k + lane] : -1;
#pragma unroll
    for (int k = 0; k < kTail; ++k) put(t[k], p + 64 * k + lane);
  }
}

// A chunk's positions by the range of their tokens, in order: an entry is the token's place in its range and the position's in the
// chunk; starts[chunk][range] is where the range's begin in the chunk, starts[chunk][ranges] how many there are.
__global__ __launch_bounds__(kSortThreads) void embed_split_kernel(const int32_t* tokens, int n, int V, int shift, int ranges, int span, unsigned* entries, int32_t* starts) {
  __shared__ int counts[kSortWaves * kMaxRanges], s[kSortWaves];
  constexpr int kTurns = kSplit / kSortThreads;
  const int tid = threadIdx.x, lane = tid & 63, wave = uniform_i(tid >> 6), p0 = blockIdx.x * span, p1 = min(n, p0 + span), at0 = wave * (kSplit / kSortWaves) + lane;
  for (int i = tid; i < kSortWaves * ranges; i += kSortThreads) counts[i] = 0;
  int t[kTurns];
#pragma unroll
  for (int k = 0; k < kTurns; ++k) t[k] = p0 + at0 + 64 * k < p1 ? tokens[p0 + at0 + 64 * k] : -1;
  __syncthreads();
  int* mine = counts + wave * ranges;
#pragma unroll
  for (int k = 0; k < kTurns; ++k)
    count_keys<1>(mine, static_cast<unsigned>(t[k]) >> shift, static_cast<unsigned>(t[k]) < static_cast<unsigned>(V), lane);
  __syncthreads();
  int end;
  const int at = places(counts, ranges, ranges, 0, s, &end);
  int32_t* to = starts + static_cast<int64_t>(blockIdx.x) * (ranges + 1);
  if (tid < ranges) to[tid] = at;
  if (tid == ranges - 1) to[ranges] = end;
  int bits = 0;
  while (((ranges - 1) >> bits) > 0) ++bits;
#pragma unroll
  for (int k = 0; k < kTurns; ++k)
    place_keys<0>(mine, static_cast<unsigned>(t[k]) >> shift, static_cast<unsigned>(t[k]) < static_cast<unsigned>(V), bits, lane, [&](int q) {
      entries[p0 + q] = static_cast<unsigned>(t[k] & ((1 << shift) - 1)) * kSplit + static_cast<unsigned>(at0 + 64 * k);
    });
}

// A range's positions from all chunks: each wave takes some chunks next to each other.
__global__ __launch_bounds__(kSortThreads) void embed_merge_kernel(const unsigned* entries, const int32_t* starts, int chunks, int span, int V, int shift, int ranges,
                                                                  int32_t* begin, int32_t* order, Owners owners) {
  extern __shared__ int counts[];  // [kSortWaves][2^shift]
  __shared__ int s[kSortWaves];
  const int tid = threadIdx.x, lane = tid & 63, wave = uniform_i(tid >> 6), range = 1 << shift, b = blockIdx.x;
  const int v0 = b << shift, size = min(range, V - v0);
  for (int i = tid; i < kSortWaves * range; i += kSortThreads) counts[i] = 0;
  int below = 0;
  for (int c = tid; c < chunks; c += kSortThreads) below += starts[static_cast<int64_t>(c) * (ranges + 1) + b];
  int base, end;
  group_upto(below, s, &base);  // (waits for the counts to be 0, too)
  const int share = (chunks + kSortWaves - 1) / kSortWaves, c0 = min(chunks, wave * share), c1 = min(chunks, c0 + share);
  int* mine = counts + wave * range;
  // Calls f(entry, is one, chunk) for 64 entries at a time, in order, those of four chunks requested together.
  auto all = [&](auto&& f) {
    for (int q = c0; q < c1; q += 64) {
      const int c = min(q + lane, c1 - 1), from = starts[static_cast<int64_t>(c) * (ranges + 1) + b], to = starts[static_cast<int64_t>(c) * (ranges + 1) + b + 1];
      const int many = min(64, c1 - q);
      for (int k0 = 0; k0 < many; k0 += 4) {
        unsigned e[4];
        int i0[4], i1[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const int from_lane = min(k0 + k, many - 1);
          i0[k] = __builtin_amdgcn_readlane(from, from_lane);
          i1[k] = k0 + k < many ? __builtin_amdgcn_readlane(to, from_lane) : i0[k];
          e[k] = i0[k] + lane < i1[k] ? entries[static_cast<int64_t>(q + k0 + k) * span + i0[k] + lane] : 0u;
        }
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          if (i0[k] < i1[k]) f(e[k], i0[k] + lane < i1[k], q + k0 + k);
          for (int i = i0[k] + 64; i < i1[k]; i += 64 * 8) {
            unsigned more[8];
#pragma unroll
            for (int u = 0; u < 8; ++u) more[u] = i + 64 * u + lane < i1[k] ? entries[static_cast<int64_t>(q + k0 + k) * span + i + 64 * u + lane] : 0u;
#pragma unroll
            for (int u = 0; u < 8; ++u)
              if (i + 64 * u < i1[k]) f(more[u], i + 64 * u + lane < i1[k], q + k0 + k);
          }
        }
      }
    }
  };
  all([&](unsigned e, bool is, int) { count_keys<2>(mine, e / kSplit, is, lane); });
  __syncthreads();
  const int at = places(counts, range, size, base, s, &end);
  if (tid < size) {
    begin[v0 + tid] = at;
    if (v0 + tid == V - 1) begin[V] = end;
  }
  write_owners(owners, b, v0, size, at, end, s);
  all([&](unsigned e, bool is, int c) {
    place_keys<2>(mine, e / kSplit, is, shift, lane, [&](int to) { order[to] = c * span + static_cast<int>(e % kSplit); });
  });
}

// Sums.  Tokens with up to kFew positions are summed by `lanes` lanes at once; those with more in pieces, cut at every kFew-th place of
// the order, which a second launch joins (kFew = 16 / 32 / 64: 131072 x 2048 bf16 299 / 285 / 272 us, 16384 x 1024 on fp32 rows 43.4 / 43.5 / 48.8,
// 8000 x 640 fp32 22.7 / 23.6 / 26.8).  A stretch of kFew places holds pieces of two such tokens at most: one that
// began before it or at its first place, and one that begins later in it.
struct SumArgs {
  EmbedGradArgs a;
  const int32_t* begin;  // [V + 1]
  const int32_t* order;  // [n]
  float* pieces;         // [stretches][2][dim]
  int lanes;
};

// Adds the rows of `U` positions from order[i] on, requested together.
template <int U, typename G, typename Order, int K, int SL, bool NARROW>
__device__ __forceinline__ void add_rows(const EmbedGradArgs& a, const Order* order, const Columns<K, SL, NARROW>& cols, int i, float (&sum)[SL][K]) {
  const typename G::type* g = static_cast<const typename G::type*>(a.grad);
  int p[U];
  float x[U][SL][K];
#pragma unroll
  for (int k = 0; k < U; ++k) p[k] = order[i + k];
#pragma unroll
  for (int k = 0; k < U; ++k)
#pragma unroll
    for (int v = 0; v < SL; ++v) cols.template load<G>(g + p[k] * a.grad_stride, v, x[k][v]);
#pragma unroll
  for (int k = 0; k < U; ++k)
#pragma unroll
    for (int v = 0; v < SL; ++v)
#pragma unroll
      for (int c = 0; c < K; ++c) sum[v][c] += x[k][v][c];
}
template <typename G, typename Order, int K, int SL, bool NARROW>
__device__ __forceinline__ void sum_positions(const EmbedGradArgs& a, const Order* order, const Columns<K, SL, NARROW>& cols, int i, int j, float (&sum)[SL][K]) {
  constexpr int U = 64 / (K * SL);
  for (; i + U <= j; i += U) add_rows<U, G>(a, order, cols, i, sum);
  if constexpr (U > 4)
    for (; i + 4 <= j; i += 4) add_rows<4, G>(a, order, cols, i, sum);
  if constexpr (U > 2)
    if (i + 2 <= j) add_rows<2, G>(a, order, cols, i, sum), i += 2;
  for (; i < j; ++i) add_rows<1, G>(a, order, cols, i, sum);
}
template <typename T, int K, int SL, bool NARROW>
__device__ __forceinline__ void write_columns(const EmbedGradArgs& a, const Columns<K, SL, NARROW>& cols, int v, float (&sum)[SL][K]) {
  typename T::type* to = static_cast<typename T::type*>(a.table_grad) + v * a.table_stride;
  float old[SL][K];
  if (a.accumulate) {
#pragma unroll
    for (int u = 0; u < SL; ++u) cols.template load<T>(to, u, old[u]);
  }
#pragma unroll
  for (int u = 0; u < SL; ++u) {
#pragma unroll
    for (int c = 0; c < K; ++c) sum[u][c] = a.accumulate ? product(a.scale, sum[u][c]) + old[u][c] : product(a.scale, sum[u][c]);
    cols.template store<T>(to, u, sum[u]);
  }
}
template <int K, int SL, bool NARROW>
__device__ __forceinline__ void write_piece(float* to, const Columns<K, SL, NARROW>& cols, const float (&sum)[SL][K]) {
#pragma unroll
  for (int u = 0; u < SL; ++u) cols.template store<F32, false>(to, u, sum[u]);
}

// A stretch's pieces: `lanes` lanes a vector of each of its columns, and where these are few, subs_for() groups of them a part of the positions each. (112956 x 32
// bf16 on 4599 rows 54.0 -> 48.7 us, 18419 x 64 fp32 on 11821 21.1 -> 18.7, 8470 x 96 on 3412 20.6 -> 17.6)
__host__ __device__ __forceinline__ int subs_for(int lanes) { return lanes <= 16 ? 4 : lanes <= 32 ? 2 : 1; }
template <typename G, int K, bool NARROW>
__device__ __forceinline__ void sum_piece(const SumArgs& s, const Columns<K, 1, NARROW>& cols, int i, int j, int sub, float* piece) {
  const int subs = subs_for(s.lanes), share = (j - i + subs - 1) / subs;
  float sum[1][K] = {};
  sum_positions<G>(s.a, s.order, cols, i + sub * share, min(j, i + (sub + 1) * share), sum);
  for (int d = s.lanes; d < s.lanes * subs; d *= 2)
#pragma unroll
    for (int e = 0; e < K; ++e) sum[0][e] += __shfl_xor(sum[0][e], d, 64);
  if (sub == 0) write_piece(piece, cols, sum);
}
template <typename G, int K, bool NARROW>
__device__ __forceinline__ void sum_stretch(const SumArgs& s, int c, int vector, int end, int lane, int sub) {
  const EmbedGradArgs& a = s.a;
  const Columns<K, 1, NARROW> cols(a.dim, vector * s.lanes * K, s.lanes, lane);
  const int i0 = c * kFew, i1 = min(end, i0 + kFew);
  const int first = a.tokens[s.order[i0]], last = a.tokens[s.order[i1 - 1]];
  float* pieces = s.pieces + static_cast<int64_t>(c) * 2 * a.dim;
  if (s.begin[first + 1] - s.begin[first] > kFew) sum_piece<G>(s, cols, i0, min(i1, s.begin[first + 1]), sub, pieces);
  if (last != first && s.begin[last + 1] - s.begin[last] > kFew) sum_piece<G>(s, cols, s.begin[last], i1, sub, pieces + a.dim);
}

// The first stretch_blocks workgroups take stretches (a piece takes longer than other rows), the others tokens, `lanes` lanes SL vectors of a
// row.  What belongs to a row lies next to each other in the grid, so that rows are read whole (131072 x 2048 bf16 285 -> 262 us).  The gradient is
// written past the caches (262 us and, 16384 x 1024 on fp32 rows, 40; otherwise 283 and 66).  Bound by HBM: 1.07 GB in 215 us of those 262.
// ROWS: rows that lanes take one after the other, where a row is one vector of each lane and there are more rows than the chip holds at
// once twice over: where they begin is read at once (60000 x 512 bf16 on 50000 49.3 -> 44.2 us, 100000 x 200 on 131072 fp32 rows 74 -> 61; two rows
// 45.6 and 63; few rows lose by it: 40000 x 128 on 4097 rows 28.6 -> 32.3, longer ones as well: 8000 x 640 22.5 -> 24.5).
template <typename G, typename T, int SL, int ROWS, bool NARROW>
__global__ __launch_bounds__(256) void embed_sums_kernel(SumArgs s, int stretch_blocks, unsigned vectors) {
  constexpr int K = step_of<G, T>();
  const EmbedGradArgs& a = s.a;
  const int lane = threadIdx.x & (s.lanes - 1), each = 256 / s.lanes;
  if (static_cast<int>(blockIdx.x) < stretch_blocks) {
    const int subs = subs_for(s.lanes), group = threadIdx.x / s.lanes;
    const unsigned unit = blockIdx.x * (each / subs) + group / subs;
    const int c = static_cast<int>(unit / vectors), end = s.begin[a.V];
    if (static_cast<int64_t>(c) * kFew < end) sum_stretch<G, K, NARROW>(s, c, static_cast<int>(unit % vectors), end, lane, group & (subs - 1));
    return;
  }
  const unsigned of_row = SL == 1 ? 1 : (vectors + SL - 1) / SL, first = (blockIdx.x - stretch_blocks) * (each * ROWS) + threadIdx.x / s.lanes;
  int from[ROWS], to[ROWS];
#pragma unroll
  for (int r = 0; r < ROWS; ++r) {
    const unsigned v = min((first + r * each) / of_row, static_cast<unsigned>(a.V) - 1);
    from[r] = s.begin[v];
    to[r] = s.begin[v + 1];
  }
#pragma unroll
  for (int r = 0; r < ROWS; ++r) {
    const unsigned v = (first + r * each) / of_row;
    if (v >= static_cast<unsigned>(a.V)) return;
    if (to[r] - from[r] > kFew || (to[r] == from[r] && a.accumulate)) continue;
    const Columns<K, SL, NARROW> cols(a.dim, static_cast<int>((first + r * each) % of_row) * s.lanes * K * SL, s.lanes, lane);
    float sum[SL][K] = {};
    sum_positions<G>(a, s.order, cols, from[r], to[r], sum);
    write_columns<T>(a, cols, static_cast<int>(v), sum);
  }
}

// Pieces of a token, in the order of their stretches: a workgroup a range (and vectors of its columns).  Its groups of lanes take the tokens
// of few pieces one each; of the others, each group sums a share of the pieces, and the first of them those sums.
// (Shares are added one after the other in fp32: of a token with 131072 positions 512 pieces by each of 8 groups of 64 lanes.)
constexpr int kJoinThreads = 512;  // (1024 / 512 / 256: 131072 x 2048 bf16 259 / 256 / 285 us, 8000 x 640 fp32 27.5 / 26.7 / 25.7, 40000 x 128 34.8 / 32.9 / 32.7)
template <typename T, int K, bool NARROW>
__global__ __launch_bounds__(kJoinThreads) void embed_join_kernel(SumArgs s, Owners owners, int shift) {
  __shared__ float shares[kJoinThreads * K];
  const EmbedGradArgs& a = s.a;
  const int n_owners = owners.count[blockIdx.x];
  const Owner* list = owners.list + (static_cast<int64_t>(blockIdx.x) << shift);
  if (n_owners == 0) return;
  const int tid = threadIdx.x, groups = kJoinThreads / s.lanes, group = tid / s.lanes, lane = tid & (s.lanes - 1);
  const Columns<K, 1, NARROW> cols(a.dim, blockIdx.y * s.lanes * K, s.lanes, lane);
  const int64_t row = 2 * static_cast<int64_t>(a.dim);
  constexpr int U = 2 * K, kFewPieces = 16;
  auto add = [&](int first_place, int k, int k1, float (&sum)[1][K]) {  // pieces of stretches k .. k1 - 1
    const int c = first_place / kFew;
    for (; k < k1; k += U) {
      float x[U][K];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int q = min(k + u, k1 - 1);
        cols.template load<F32>(s.pieces + q * row + (q == c && first_place != c * kFew ? a.dim : 0), 0, x[u]);
      }
#pragma unroll
      for (int u = 0; u < U; ++u)
#pragma unroll
        for (int e = 0; e < K; ++e) sum[0][e] += k + u < k1 ? x[u][e] : 0.0f;
    }
  };
  for (int o = group; o < n_owners; o += groups) {
    const Owner w = list[o];
    const int c = w.begin / kFew, last = (w.end + kFew - 1) / kFew;
    if (last - c > kFewPieces) continue;
    float sum[1][K] = {};
    add(w.begin, c, last, sum);
    write_columns<T>(a, cols, w.v, sum);
  }
  for (int o = 0; o < n_owners; ++o) {
    const Owner w = list[o];
    const int c = w.begin / kFew, last = (w.end + kFew - 1) / kFew;
    if (last - c <= kFewPieces) continue;
    const int share = (last - c + groups - 1) / groups;
    float sum[1][K] = {};
    add(w.begin, c + group * share, min(last, c + (group + 1) * share), sum);
#pragma unroll
    for (int e = 0; e < K; ++e) shares[e * kJoinThreads + tid] = sum[0][e];
    __syncthreads();
    if (group == 0) {
      for (int q = 1; q < groups && c + q * share < last; ++q)
#pragma unroll
        for (int e = 0; e < K; ++e) sum[0][e] += shares[e * kJoinThreads + q * s.lanes + lane];
      write_columns<T>(a, cols, w.v, sum);
    }
    __syncthreads();
  }
}

// Few tokens on a small table, all in one launch: a workgroup a token (and vectors of its columns) looks through the tokens for its
// positions, waves in their order, its groups of lanes sum a share of those each, and the first of them those sums.  TURNS: 256 tokens each,
// held from the count of the positions to their list; LOOP: read again for that, TURNS at a time.
constexpr int kSmallTokens = 16384;
static_assert(kSmallTokens <= 65536, "positions in 16 bits");
template <int K, int TURNS, bool LOOP>
struct SmallShared {
  unsigned short list[LOOP ? kSmallTokens : 256 * TURNS];
  int found[4];
  float shares[256 * K];
};
// A wave's tokens from turn `from` on.
template <int TURNS>
__device__ __forceinline__ void request_tokens(const EmbedGradArgs& a, int turns, int p0, int from, int (&t)[TURNS]) {
#pragma unroll
  for (int k = 0; k < TURNS; ++k) t[k] = from + k < turns && p0 + 64 * (from + k) < a.n ? a.tokens[p0 + 64 * (from + k)] : -1;
}
// Token v's row of the gradient, by the workgroup; t: its tokens (of the first turns, where there are more than TURNS of them).
// A group of lanes adds its share one after the other in fp32: up to 1024 of them where small() ends (4096 positions of one token, 64 lanes; 16384, 16).
template <typename G, typename T, int TURNS, bool LOOP, int K, bool NARROW>
__device__ __forceinline__ void sum_token(const SumArgs& s, int v, const Columns<K, 1, NARROW>& cols, int (&t)[TURNS], int turns, int p0, SmallShared<K, TURNS, LOOP>& sh) {
  const EmbedGradArgs& a = s.a;
  const int tid = threadIdx.x, wave = uniform_i(tid >> 6), lane64 = tid & 63;
  int count = 0;
  for (int from = 0; from < (LOOP ? turns : 1); from += TURNS) {
    if (LOOP && from > 0) request_tokens(a, turns, p0, from, t);
#pragma unroll
    for (int k = 0; k < TURNS; ++k) count += __builtin_popcountll(__ballot(t[k] == v));
  }
  if (lane64 == 0) sh.found[wave] = count;
  __syncthreads();
  int at = 0;
  for (int w = 0; w < wave; ++w) at += sh.found[w];
  if (count > 0) {
    for (int from = 0; from < (LOOP ? turns : 1); from += TURNS) {
      if (LOOP) request_tokens(a, turns, p0, from, t);
#pragma unroll
      for (int k = 0; k < TURNS; ++k) {
        const u64 here = __ballot(t[k] == v);
        if (t[k] == v) sh.list[at + __builtin_popcountll(here & ((1ull << lane64) - 1))] = static_cast<unsigned short>(p0 + 64 * (from + k));
        at += __builtin_popcountll(here);
      }
    }
  }
  count = sh.found[0] + sh.found[1] + sh.found[2] + sh.found[3];
  if (count == 0 && a.accumulate) return;
  __syncthreads();
  const int lane = tid & (s.lanes - 1), group = tid / s.lanes, groups = 256 / s.lanes;
  const int share = max(8, (count + groups - 1) / groups);
  float sum[1][K] = {};
  sum_positions<G>(a, sh.list, cols, group * share, min(count, (group + 1) * share), sum);
  if (count > share) {
#pragma unroll
    for (int e = 0; e < K; ++e) sh.shares[e * 256 + tid] = sum[0][e];
    __syncthreads();
    if (group == 0)
      for (int q = 1; q * share < count; ++q)
#pragma unroll
        for (int e = 0; e < K; ++e) sum[0][e] += sh.shares[e * 256 + q * s.lanes + lane];
  }
  if (group == 0) write_columns<T>(a, cols, v, sum);
}
template <typename G, typename T, int TURNS, bool LOOP, bool NARROW>
__global__ __launch_bounds__(256) void embed_small_kernel(SumArgs s) {
  constexpr int K = step_of<G, T>();
  __shared__ SmallShared<K, TURNS, LOOP> sh;
  const int turns = (s.a.n + 255) / 256, p0 = uniform_i(threadIdx.x >> 6) * turns * 64 + (threadIdx.x & 63);
  int t[TURNS];
  request_tokens(s.a, turns, p0, 0, t);
  const Columns<K, 1, NARROW> cols(s.a.dim, blockIdx.y * s.lanes * K, s.lanes, threadIdx.x & (s.lanes - 1));
  sum_token<G, T, TURNS, LOOP>(s, blockIdx.x, cols, t, turns, p0, sh);
}

// Few tokens on a large table, all in one launch: a workgroup takes some rows (and a vector of their columns), most of which no token has.  us, so / in
// three launches, fp32: 88 tokens, 44224 x 320 bf16 8.9 / 17.4; 500, 32001 x 640 18.3 / 23.2; 1000, 8192 x 256 7.9 / 12.4, 32001 x 256 9.1 / 16.1, 65000 x 256
// 13.8 / 21.5, 131072 x 64 10.5 / 17.1; all of them one token, 32001 x 256 16.0 / 17.4.  2000: 32001 x 256 11.9 / 16.6, but where they are one
// token 29 / 16.  Rows a workgroup, 8 / 16 / 32: 1000, 8192 x 256 7.9 / 10.1 / -, 32001 x 256 10.1 / 9.1 / 9.2, 131072 x 64 19.9 / 13.6 / 10.5.
constexpr int kFewTokens = 1024;
int few_rows(int V) { return V <= 8 * 2048 ? 8 : V <= 16 * 2048 ? 16 : 32; }
template <typename G, typename T>
__global__ __launch_bounds__(256) void embed_few_kernel(SumArgs s, int rows) {
  constexpr int K = step_of<G, T>(), TURNS = kFewTokens / 256;
  __shared__ SmallShared<K, TURNS, false> sh;
  __shared__ unsigned occur;
  const EmbedGradArgs& a = s.a;
  const int turns = (a.n + 255) / 256, p0 = uniform_i(threadIdx.x >> 6) * turns * 64 + (threadIdx.x & 63);
  const int v0 = blockIdx.x * rows, size = min(rows, a.V - v0);
  int t[TURNS];
  request_tokens(a, turns, p0, 0, t);
  if (threadIdx.x == 0) occur = 0;
  __syncthreads();
  unsigned mine = 0;
#pragma unroll
  for (int k = 0; k < TURNS; ++k) {
    const unsigned u = static_cast<unsigned>(t[k]) - static_cast<unsigned>(v0);
    mine |= u < static_cast<unsigned>(size) ? 1u << u : 0u;
  }
  if (mine != 0) atomicOr(&occur, mine);
  __syncthreads();
  const unsigned has = occur;
  const Columns<K, 1, false> cols(a.dim, blockIdx.y * s.lanes * K, s.lanes, threadIdx.x & (s.lanes - 1));
  if (!a.accumulate) {
    const float zero[K] = {};
    for (int r = threadIdx.x / s.lanes; r < size; r += 256 / s.lanes)
      if (!((has >> r) & 1u)) cols.template store<T>(static_cast<typename T::type*>(a.table_grad) + (v0 + r) * a.table_stride, 0, zero);
  }
  for (unsigned left = has; left != 0; left &= left - 1) {
    sum_token<G, T, TURNS, false>(s, v0 + __builtin_ctz(left), cols, t, turns, p0, sh);
    __syncthreads();
  }
}

template <typename Do>
int with_type(int dtype, Do&& f) {
  return dtype == PB_F32 ? f(F32{}) : dtype == PB_F16 ? f(F16{}) : f(BF16{});
}
int done() { return hipGetLastError() == hipSuccess ? PB_OK : PB_EHIP; }

int64_t padded(int64_t bytes) { return (bytes + 255) / 256 * 256; }

}  // namespace em

int launch_embed_tokens(int table_dtype, int out_dtype, const EmbedArgs& a, hipStream_t stream) {
  return em::with_type(table_dtype, [&](auto e) {
    return em::with_type(out_dtype, [&](auto o) {
      using E = decltype(e);
      using O = decltype(o);
      constexpr int K = em::step_of<E, O>();
      const int lanes = em::lanes_for(a.dim, K), vectors = (a.dim + lanes * K - 1) / (lanes * K), groups = (a.n + 256 / lanes - 1) / (256 / lanes);
      auto go = [&](auto kernel, int sl) {
        kernel<<<dim3(groups, (vectors + sl - 1) / sl), 256, 0, stream>>>(a, lanes);
        return em::done();
      };
      if (a.dim < K) return go(em::embed_kernel<E, O, 1, true>, 1);
      if (vectors == 1) return go(em::embed_kernel<E, O, 1, false>, 1);
      if (vectors == 2) return go(em::embed_kernel<E, O, 2, false>, 2);
      return go(em::embed_kernel<E, O, 4, false>, 4);
    });
  });
}

namespace em {
// What lies where in the workspace.  Its size does not fall with n: one for many tokens does for fewer.
struct Layout {
  int64_t begin, order, count, list, pieces, entries, starts, bytes;
};
Layout layout(int32_t n, int32_t V, int32_t dim) {
  Layout l;
  l.begin = 0;
  l.order = padded((static_cast<int64_t>(V) + 1) * 4);
  l.count = l.order + padded(static_cast<int64_t>(n) * 4);
  l.list = l.count + kMaxRanges * 4;
  l.pieces = l.list + padded((static_cast<int64_t>(V) + (1 << kMaxShift)) * static_cast<int64_t>(sizeof(Owner)));
  l.bytes = l.pieces + (n > kFew ? padded((static_cast<int64_t>(n) + kFew - 1) / kFew * 2 * dim * 4) : 0);
  l.entries = l.starts = l.pieces;  // (entries and starts are done with before there are pieces)
  if (n >= kManyTokens) {
    l.starts = l.entries + padded(static_cast<int64_t>(n) * 4);
    l.bytes = std::max(l.bytes, l.starts + turns_for(n) * kSortWaves * ((((V - 1) >> shift_for(n, V)) + 2) * 4));
  }
  return l;
}
}  // namespace em

int64_t embed_tokens_backward_workspace(int32_t n, int32_t V, int32_t dim) { return em::layout(n, V, dim).bytes; }

namespace em {
template <typename G, typename T>
struct Shape {
  static constexpr int K = step_of<G, T>();
  int lanes, vectors;
  explicit Shape(int dim) : lanes(lanes_for(dim, K)), vectors((dim + lanes * K - 1) / (lanes * K)) {}
};
// us, a workgroup a token / in three launches, fp32 where not said: 500 tokens, 1025 x 640 5.7 / 12.4; 2000, 4096 x 64 9.1 / 14.0, 8192 x 64 15.2 / 14.1;
// 2900, 6000 x 64 12.2 / 13.9; 4096, 4096 x 64 10.0 / 14.8, 1025 x 640 12.7 / 17.0, 8192 x 512 bf16 21.6 / 16.3; 5000, 4096 x 64 19.7 / 16.7; 8192, 2048 x 64
// 15.1 / 17.7; 16384, 166 x 64 18.4 / 21.3, 1025 x 64 17.4 / 20.1; and, where a token of many positions has few groups of lanes for them, 8192, 300 x 512
// bf16 17.4 / 17.8, 300 x 1024 bf16 27.1 / 23.7; 16384, 166 x 2048 71 / 51.  Few tokens, a workgroup a token / some rows: 1000, 2048 x 64 4.7 / 9.9, 4096 x 64
// 6.6 / 10.2, 3000 x 512 8.9 / 7.1, 6000 x 64 8.6 / 6.3; 300, 6000 x 64 7.8 / 4.6.
bool small(int64_t n, int64_t V, int lanes, int vectors) {
  return n <= kSmallTokens && n * lanes <= 4096 * 64 && V * vectors <= (n <= kFewTokens ? 4608 : 6144) && V * vectors * n <= 17 << 20;
}

template <typename G, typename T>
int backward(const EmbedGradArgs& a, char* ws, hipStream_t stream) {
  const Shape<G, T> shape(a.dim);
  constexpr int K = Shape<G, T>::K;
  const int lanes = shape.lanes, each = 256 / lanes, vectors = shape.vectors;
  const Layout l = layout(a.n, a.V, a.dim);
  int32_t* begin = reinterpret_cast<int32_t*>(ws + l.begin);
  int32_t* order = reinterpret_cast<int32_t*>(ws + l.order);
  const SumArgs s{a, begin, order, reinterpret_cast<float*>(ws + l.pieces), lanes};
  if (small(a.n, a.V, lanes, vectors)) {
    auto go = [&](auto kernel) {
      kernel<<<dim3(a.V, vectors), 256, 0, stream>>>(s);
      return done();
    };
    if (a.dim < K) return go(embed_small_kernel<G, T, 16, true, true>);
    if (a.n <= 1024) return go(embed_small_kernel<G, T, 4, false, false>);
    if (a.n <= 4096) return go(embed_small_kernel<G, T, 16, false, false>);
    return go(embed_small_kernel<G, T, 16, true, false>);
  }
  if (a.n <= kFewTokens && a.dim >= K) {  // (narrower rows are seldom: three launches)
    const int rows = few_rows(a.V);
    embed_few_kernel<G, T><<<dim3((a.V + rows - 1) / rows, vectors), 256, 0, stream>>>(s, rows);
    return done();
  }
  const int shift = shift_for(a.n, a.V), ranges = ((a.V - 1) >> shift) + 1, stretches = (a.n + kFew - 1) / kFew;
  const size_t counts = static_cast<size_t>(kSortWaves) * 4 << shift;
  const Owners owners{reinterpret_cast<int32_t*>(ws + l.count), reinterpret_cast<Owner*>(ws + l.list)};
  if (a.n >= kManyTokens) {
    unsigned* entries = reinterpret_cast<unsigned*>(ws + l.entries);
    int32_t* starts = reinterpret_cast<int32_t*>(ws + l.starts);
    const int span = span_for(a.n), chunks = (a.n + span - 1) / span;
    embed_split_kernel<<<chunks, kSortThreads, 0, stream>>>(a.tokens, a.n, a.V, shift, ranges, span, entries, starts);
    if (done() != PB_OK) return PB_EHIP;
    embed_merge_kernel<<<ranges, kSortThreads, counts, stream>>>(entries, starts, chunks, span, a.V, shift, ranges, begin, order, owners);
  } else {
    embed_sort_kernel<<<dim3(ranges, parts_for(a.n, a.V)), kSortThreads, counts + (static_cast<size_t>(8) << shift), stream>>>(a.tokens, a.n, a.V, shift, begin, order, owners);
  }
  if (done() != PB_OK) return PB_EHIP;
  const int stretch_each = each / subs_for(lanes);
  const int64_t stretch_blocks = a.n > kFew ? (static_cast<int64_t>(stretches) * vectors + stretch_each - 1) / stretch_each : 0;
  auto sums = [&](auto kernel, int sl, int rows) {
    const int64_t of_block = static_cast<int64_t>(each) * rows, row_blocks = (static_cast<int64_t>(a.V) * ((vectors + sl - 1) / sl) + of_block - 1) / of_block;
    kernel<<<static_cast<unsigned>(stretch_blocks + row_blocks), 256, 0, stream>>>(s, static_cast<int>(stretch_blocks), static_cast<unsigned>(vectors));
    return done();
  };
  int rc;
  const bool many = static_cast<int64_t>(a.V) * lanes > 64 * 16384;  // (waves of 64 lanes)
  if (a.dim < K) rc = sums(embed_sums_kernel<G, T, 1, 1, true>, 1, 1);
  else if (vectors == 1 && many) rc = sums(embed_sums_kernel<G, T, 1, 4, false>, 1, 4);
  else if (vectors == 1) rc = sums(embed_sums_kernel<G, T, 1, 1, false>, 1, 1);
  else if (vectors == 2) rc = sums(embed_sums_kernel<G, T, 2, 1, false>, 2, 1);
  else rc = sums(embed_sums_kernel<G, T, 4, 1, false>, 4, 1);
  if (rc != PB_OK || stretch_blocks == 0) return rc;
  const dim3 grid(ranges, vectors);
  if (a.dim < K) embed_join_kernel<T, K, true><<<grid, kJoinThreads, 0, stream>>>(s, owners, shift);
  else embed_join_kernel<T, K, false><<<grid, kJoinThreads, 0, stream>>>(s, owners, shift);
  return done();
}
}  // namespace em

int launch_embed_tokens_backward(int grad_dtype, int table_dtype, const EmbedGradArgs& a, void* workspace, hipStream_t stream) {
  return em::with_type(grad_dtype, [&](auto g) {
    return em::with_type(table_dtype, [&](auto t) { return em::backward<decltype(g), decltype(t)>(a, static_cast<char*>(workspace), stream); });
  });
}

}  // namespace pb
