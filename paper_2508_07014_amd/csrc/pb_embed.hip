// Rows of a table for tokens, scaled (pb_embed_tokens), and the table's gradient (pb_embed_tokens_backward).
#include "pb_logit_rows.hpp"
#include "pb_student.hpp"

namespace pb {
namespace em {

using namespace lr;
using wv::first_lane;

// Eight elements at p, any alignment of its elements, to and from fp32.
constexpr int kStep = 8;
template <typename E>
__device__ __forceinline__ void load8(const typename E::type* p, float (&x)[kStep]) {
  if constexpr (E::N == 8) {
    E::unpack(any_vector<E>(p), x);
  } else {
    float lo[4], hi[4];
    E::unpack(any_vector<E>(p), lo);
    E::unpack(any_vector<E>(p + 4), hi);
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = lo[i], x[4 + i] = hi[i];
  }
}
template <typename E>
__device__ __forceinline__ void store8(typename E::type* p, const float (&x)[kStep]) {
  if constexpr (E::N == 8) {
    store_vector<E>(p, E::pack(x));
  } else {
    const float lo[4] = {x[0], x[1], x[2], x[3]}, hi[4] = {x[4], x[5], x[6], x[7]};
    store_vector<E>(p, E::pack(lo));
    store_vector<E>(p + 4, E::pack(hi));
  }
}
// The first n (1 .. 8) of them.
template <typename E>
__device__ __forceinline__ void load_some(const typename E::type* p, int n, float (&x)[kStep]) {
  if (n == kStep) return load8<E>(p, x);
#pragma unroll
  for (int i = 0; i < kStep; ++i) x[i] = i < n ? E::up(p[i]) : 0.0f;
}
template <typename E>
__device__ __forceinline__ void store_some(typename E::type* p, int n, const float (&x)[kStep]) {
  if (n == kStep) return store8<E>(p, x);
#pragma unroll
  for (int i = 0; i < kStep; ++i)
    if (i < n) p[i] = E::down(x[i]);
}

// `lanes` (a power of 2 up to 64) take a row, 8 elements each a turn.
template <typename E, typename O>
__global__ __launch_bounds__(256) void embed_kernel(EmbedArgs a, int lanes) {
  const int64_t i = static_cast<int64_t>(blockIdx.x) * (256 / lanes) + threadIdx.x / lanes;
  if (i >= a.n) return;
  const int t = a.tokens[i], lane = threadIdx.x & (lanes - 1);
  const bool there = static_cast<unsigned>(t) < static_cast<unsigned>(a.V);
  const typename E::type* from = static_cast<const typename E::type*>(a.table) + (there ? t : 0) * a.table_stride;
  typename O::type* to = static_cast<typename O::type*>(a.out) + i * a.out_stride;
  for (int d = lane * kStep; d < a.dim; d += lanes * kStep) {
    const int n = min(kStep, a.dim - d);
    float x[kStep] = {0, 0, 0, 0, 0, 0, 0, 0};
    if (there) {
      load_some<E>(from + d, n, x);
#pragma unroll
      for (int k = 0; k < kStep; ++k) x[k] *= a.scale;
    }
    store_some<O>(to + d, n, x);
  }
}

// The gradient: positions sorted by token, then sums over each token's positions.
//
// Sorting.  A workgroup takes a range of the vocabulary and reads all tokens: those of its range it counts, for each wave's share of
// the positions apart, and places in a second pass; those below its range it counts for the place its range begins at.
// So the order is that of the positions, without an atomic on memory and with one launch: the workgroups read the tokens
// as often as there are of them, from the caches (131072 tokens: 128 MB in all).
constexpr int kSortThreads = 1024, kSortWaves = kSortThreads / 64;
constexpr int kMostRange = 896;   // tokens of a range: 64 bytes of LDS each
constexpr int kRanges = 256;      // at least so many workgroups where there are as many tokens

__global__ __launch_bounds__(kSortThreads) void embed_sort_kernel(const int32_t* tokens, int n, int V, int range, int32_t* begin, int32_t* order) {
  extern __shared__ int counts[];  // [kSortWaves][range]
  __shared__ int shared_sum[kSortWaves], base;
  const int tid = threadIdx.x, lane = tid & 63, wave = uniform_i(tid >> 6);
  const int v0 = blockIdx.x * range, size = min(range, V - v0);
  for (int i = tid; i < kSortWaves * range; i += kSortThreads) counts[i] = 0;
  __syncthreads();
  const int share = ((n + kSortWaves - 1) / kSortWaves + 63) / 64 * 64, p0 = min(n, wave * share), p1 = min(n, p0 + share);
  int* mine = counts + wave * range;
  int below = 0;
  for (int p = p0 + lane; p < p1; p += 64) {
    const int t = tokens[p];
    if (t >= v0 && t < v0 + size) atomicAdd(&mine[t - v0], 1);
    below += t >= 0 && t < v0;
  }
#pragma unroll
  for (int d = 1; d < 64; d *= 2) below += __shfl_xor(below, d, 64);
  if (lane == 0) shared_sum[wave] = below;
  __syncthreads();
  if (tid == 0) {
    int s = 0;
    for (int w = 0; w < kSortWaves; ++w) s += shared_sum[w];
    base = s;
  }
  __syncthreads();
  // counts[w][v] becomes the place of wave w's first position of token v: sums over tokens, then over the waves before.
  int total = 0;
  if (tid < size)
    for (int w = 0; w < kSortWaves; ++w) total += counts[w * range + tid];
  int upto = total;
#pragma unroll
  for (int d = 1; d < 64; d *= 2) {
    const int v = __shfl_up(upto, d, 64);
    if (lane >= d) upto += v;
  }
  __syncthreads();
  if (lane == 63) shared_sum[wave] = upto;
  __syncthreads();
  int at = base + upto - total;
  for (int w = 0; w < wave; ++w) at += shared_sum[w];
  if (tid < size) {
    begin[v0 + tid] = at;
    if (v0 + tid == V - 1) begin[V] = at + total;
    for (int w = 0; w < kSortWaves; ++w) {
      const int c = counts[w * range + tid];
      counts[w * range + tid] = at;
      at += c;
    }
  }
  __syncthreads();
  for (int p = p0; p < p1; p += 64) {  // (all lanes of a wave: p0 is the wave's)
    const int t = p + lane < p1 ? tokens[p + lane] : -1;
    const bool in = t >= v0 && t < v0 + size;
    u64 left = __ballot(in);
    while (left) {
      const int v = __builtin_amdgcn_readlane(t, first_lane(left));
      const u64 same = __ballot(in && t == v);
      const int to = mine[v - v0];
      if (in && t == v) order[to + __builtin_popcountll(same & ((1ull << lane) - 1))] = p + lane;
      if (lane == 0) mine[v - v0] = to + __builtin_popcountll(same);
      left &= ~same;
      __builtin_amdgcn_wave_barrier();
    }
  }
}

// Sums.  Tokens with up to kFew positions are summed by `lanes` lanes at once; those with more in pieces, cut at every kFew-th place of
// the order, which a second launch joins.  A stretch of kFew places holds pieces of two such tokens at most: one that
// began before it or at its first place, and one that begins later in it.
constexpr int kFew = 64;

struct SumArgs {
  EmbedGradArgs a;
  const int32_t* begin;  // [V + 1]
  const int32_t* order;  // [n]
  float* pieces;         // [stretches][2][dim]
  int lanes;
};

// Eight columns from d on over the positions order[i] .. order[j - 1], in that order.
template <typename G>
__device__ __forceinline__ void sum_positions(const SumArgs& s, int i, int j, int d, int n, float (&sum)[kStep]) {
  const typename G::type* g = static_cast<const typename G::type*>(s.a.grad) + d;
  for (; i + 4 <= j; i += 4) {
    int p[4];
    float x[4][kStep];
#pragma unroll
    for (int k = 0; k < 4; ++k) p[k] = s.order[i + k];
#pragma unroll
    for (int k = 0; k < 4; ++k) load_some<G>(g + p[k] * s.a.grad_stride, n, x[k]);
#pragma unroll
    for (int k = 0; k < 4; ++k)
#pragma unroll
      for (int c = 0; c < kStep; ++c) sum[c] += x[k][c];
  }
  for (; i < j; ++i) {
    float x[kStep];
    load_some<G>(g + s.order[i] * s.a.grad_stride, n, x);
#pragma unroll
    for (int c = 0; c < kStep; ++c) sum[c] += x[c];
  }
}
template <typename T>
__device__ __forceinline__ void write_columns(const EmbedGradArgs& a, int v, int d, int n, float (&sum)[kStep]) {
  typename T::type* to = static_cast<typename T::type*>(a.table_grad) + v * a.table_stride + d;
  float old[kStep];
  if (a.accumulate) load_some<T>(to, n, old);
#pragma unroll
  for (int c = 0; c < kStep; ++c) sum[c] = a.accumulate ? __builtin_fmaf(a.scale, sum[c], old[c]) : a.scale * sum[c];
  store_some<T>(to, n, sum);
}

template <typename G, typename T>
__global__ __launch_bounds__(256) void embed_sums_kernel(SumArgs s, int rows_blocks, int stretches) {
  const EmbedGradArgs& a = s.a;
  const int lane = threadIdx.x & (s.lanes - 1), sub = threadIdx.x / s.lanes, each = 256 / s.lanes;
  const int d = (blockIdx.y * s.lanes + lane) * kStep, n = min(kStep, a.dim - d);
  if (n <= 0) return;
  float sum[kStep] = {0, 0, 0, 0, 0, 0, 0, 0};
  if (static_cast<int>(blockIdx.x) < rows_blocks) {
    const int64_t v = static_cast<int64_t>(blockIdx.x) * each + sub;
    if (v >= a.V) return;
    const int i = s.begin[v], j = s.begin[v + 1];
    if (j - i > kFew || (j == i && a.accumulate)) return;
    sum_positions<G>(s, i, j, d, n, sum);
    write_columns<T>(a, static_cast<int>(v), d, n, sum);
    return;
  }
  const int c = (static_cast<int>(blockIdx.x) - rows_blocks) * each + sub, end = s.begin[a.V];
  if (c >= stretches || c * kFew >= end) return;
  const int i0 = c * kFew, i1 = min(end, i0 + kFew);
  const int first = a.tokens[s.order[i0]], last = a.tokens[s.order[i1 - 1]];
  if (s.begin[first + 1] - s.begin[first] > kFew) {
    sum_positions<G>(s, i0, min(i1, s.begin[first + 1]), d, n, sum);
    store_some<F32>(s.pieces + (static_cast<int64_t>(c) * 2) * a.dim + d, n, sum);
  }
  if (last != first && s.begin[last + 1] - s.begin[last] > kFew) {
    float other[kStep] = {0, 0, 0, 0, 0, 0, 0, 0};
    sum_positions<G>(s, s.begin[last], i1, d, n, other);
    store_some<F32>(s.pieces + (static_cast<int64_t>(c) * 2 + 1) * a.dim + d, n, other);
  }
}

// Pieces of a token in the order of their stretches, by the workgroup of the stretch in which it begins.
template <typename T>
__global__ __launch_bounds__(256) void embed_join_kernel(SumArgs s, int stretches) {
  const EmbedGradArgs& a = s.a;
  const int c = blockIdx.x * (256 / s.lanes) + threadIdx.x / s.lanes, end = s.begin[a.V];
  const int d = (blockIdx.y * s.lanes + (threadIdx.x & (s.lanes - 1))) * kStep, n = min(kStep, a.dim - d);
  if (c >= stretches || c * kFew >= end || n <= 0) return;
  const int v = a.tokens[s.order[min(end, c * kFew + kFew) - 1]], i = s.begin[v], j = s.begin[v + 1];
  if (j - i <= kFew || i / kFew != c) return;
  float sum[kStep], x[kStep];
  load_some<F32>(s.pieces + (static_cast<int64_t>(c) * 2 + (i == c * kFew ? 0 : 1)) * a.dim + d, n, sum);
  for (int k = c + 1; k * kFew < j; ++k) {
    load_some<F32>(s.pieces + static_cast<int64_t>(k) * 2 * a.dim + d, n, x);
#pragma unroll
    for (int e = 0; e < kStep; ++e) sum[e] += x[e];
  }
  write_columns<T>(a, v, d, n, sum);
}

int lanes_for(int dim) {
  int lanes = 1;
  while (lanes < 64 && lanes * kStep < dim) lanes *= 2;
  return lanes;
}

template <typename Do>
int with_type(int dtype, Do&& f) {
  return dtype == PB_F32 ? f(F32{}) : dtype == PB_F16 ? f(F16{}) : f(BF16{});
}
int done() { return hipGetLastError() == hipSuccess ? PB_OK : PB_EHIP; }

int sort_range(int V) {
  const int even = (V + kRanges - 1) / kRanges;
  return even < kMostRange ? even : kMostRange;
}
int64_t padded(int64_t bytes) { return (bytes + 255) / 256 * 256; }

}  // namespace em

int launch_embed_tokens(int table_dtype, int out_dtype, const EmbedArgs& a, hipStream_t stream) {
  const int lanes = em::lanes_for(a.dim);
  const unsigned grid = static_cast<unsigned>((static_cast<int64_t>(a.n) * lanes + 255) / 256);
  return em::with_type(table_dtype, [&](auto e) {
    return em::with_type(out_dtype, [&](auto o) {
      em::embed_kernel<decltype(e), decltype(o)><<<grid, 256, 0, stream>>>(a, lanes);
      return em::done();
    });
  });
}

int64_t embed_tokens_backward_workspace(int32_t n, int32_t V, int32_t dim) {
  const int64_t stretches = (static_cast<int64_t>(n) + em::kFew - 1) / em::kFew;
  return em::padded((static_cast<int64_t>(V) + 1) * 4) + em::padded(static_cast<int64_t>(n) * 4) + stretches * 2 * dim * 4;
}
int launch_embed_tokens_backward(int grad_dtype, int table_dtype, const EmbedGradArgs& a, void* workspace, hipStream_t stream) {
  char* ws = static_cast<char*>(workspace);
  int32_t* begin = reinterpret_cast<int32_t*>(ws);
  int32_t* order = reinterpret_cast<int32_t*>(ws + em::padded((static_cast<int64_t>(a.V) + 1) * 4));
  float* pieces = reinterpret_cast<float*>(ws + em::padded((static_cast<int64_t>(a.V) + 1) * 4) + em::padded(static_cast<int64_t>(a.n) * 4));
  const int range = em::sort_range(a.V), lanes = em::lanes_for(a.dim), each = 256 / lanes;
  const int stretches = (a.n + em::kFew - 1) / em::kFew, slices = (a.dim + lanes * em::kStep - 1) / (lanes * em::kStep);
  em::embed_sort_kernel<<<(a.V + range - 1) / range, em::kSortThreads, static_cast<size_t>(range) * em::kSortWaves * 4, stream>>>(a.tokens, a.n, a.V, range, begin, order);
  if (em::done() != PB_OK) return PB_EHIP;
  const em::SumArgs s{a, begin, order, pieces, lanes};
  const int rows_blocks = (a.V + each - 1) / each, stretch_blocks = (stretches + each - 1) / each;
  const int rc = em::with_type(grad_dtype, [&](auto g) {
    return em::with_type(table_dtype, [&](auto t) {
      em::embed_sums_kernel<decltype(g), decltype(t)><<<dim3(rows_blocks + stretch_blocks, slices), 256, 0, stream>>>(s, rows_blocks, stretches);
      return em::done();
    });
  });
  if (rc != PB_OK || a.n <= em::kFew) return rc;
  return em::with_type(table_dtype, [&](auto t) {
    em::embed_join_kernel<decltype(t)><<<dim3(stretch_blocks, slices), 256, 0, stream>>>(s, stretches);
    return em::done();
  });
}

}  // namespace pb
