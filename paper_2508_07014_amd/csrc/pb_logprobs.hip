// pb_token_logprobs and its gradient (gfx950): rows read once, in 16-byte vectors, by a wave or a workgroup each.
#include <hip/hip_runtime.h>

#include "pb_kernels.hpp"
#include "pb_logit_rows.hpp"

namespace pb {
namespace lr {
namespace {

constexpr int kUnroll = 4;            // vectors of a thread in flight
constexpr int kGroups = 256;          // parts of a row whose maxima bound the alternatives

// Maximum, sum of exponentials and entropy in one pass.  With c = log2(e) / T every term is e = exp2(d), d = x c - rc, and the
// reference rc = m c, m the largest element that the lane has seen: batch by batch (kUnroll vectors), since a move costs an
// exponential and a product a sum.  So e <= 1, and the sum X of e d holds no term of the maximum's size that the entropy
// would have to cancel.  The sum of the batch in which the maximum lies, P, is kept apart from the others', S, down to the
// logarithm: log(P + S) = log1p((P - 1) + S), so that what lies beside a likely token is not rounded to its unit (entropies of
// such rows: errors of 5e-6 without, 1e-7 with it); where less than an eighth of the maximum's term lies beside it, that batch is
// summed once more without it.  d is rounded once; what rc was rounded by is the same for all terms and comes off a wave's sums.
// Elements below -far (see kFar) are masks of a lowest value: nothing beside any ordinary logit.
struct Sums {
  float m = -INFINITY, thr, rc = 0.0f, P = 0.0f, S = 0.0f, X = 0.0f;
  int at = -1;  // first vector of the batch that P is the sum of; -1: the edge
  __device__ __forceinline__ explicit Sums(float far) : thr(-far) {}
};
// (S, X) seen from a reference that lies `apart` = rc - new rc higher.
template <bool ENT>
__device__ __forceinline__ void rebase(float& S, float& X, float apart) {
  const float f = exp2_fast(apart);  // (may be infinite where the sums are 0)
  if constexpr (ENT) X = S == 0.0f ? 0.0f : f * __builtin_fmaf(apart, S, X);
  S = S == 0.0f ? 0.0f : f * S;
}
template <bool ENT, int U, int N>
__device__ __forceinline__ void add_batch(Sums& s, const float (&x)[U][N], float m, float c, int at) {
  const bool up = m > s.thr;
  if (__ballot(up) != 0) {
    asm volatile("");  // (a branch: selects would take the move's exponential in every batch)
    if (up) {
      const float next = m * c;
      s.S += s.P;
      rebase<ENT>(s.S, s.X, s.rc - next);
      s.rc = next;
      s.thr = m;
      s.at = at;
    }
  }
  float sum, sum_x;
#pragma unroll
  for (int u = 0; u < U; ++u) {
    float e[N], ed[N];
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const float d = __builtin_fmaf(x[u][i], c, -s.rc);
      e[i] = exp2_fast(d);
      if constexpr (ENT) ed[i] = mul_0(e[i], d);  // (-inf: nothing)
    }
    if constexpr (ENT) sum_x = u == 0 ? vec_sum(ed) : sum_x + vec_sum(ed);
    sum = u == 0 ? vec_sum(e) : sum + vec_sum(e);
  }
  s.P = up ? sum : s.P;
  s.S += up ? 0.0f : sum;
  if constexpr (ENT) s.X += sum_x;
}

// Sums of a part of a row, d = (x - m) c.  P is negative where it lacks the maximum's term, 1: then -P is the rest of the batch's.
// A part of nothing but -inf has sums of 0.
struct __align__(16) Part {
  float m, P, S, X;
};
__device__ __forceinline__ float whole(float P) { return __float_as_int(P) < 0 ? 1.0f - P : P; }
// How far sums seen from m are to move: from below 2^-1000 nothing is left of them.  (A part of nothing but masks of a lowest value
// beside an ordinary one: apart S would pass the fp32 range, and X be 0 times that.  Lanes that lie so far apart inside a wave
// are summed again, see wave_part; the clamp there cost 16384 x 2049 bf16 2 %.)
__device__ __forceinline__ float parted(float m, float from, float c) { return fmaxf((m - from) * c, -1000.0f); }
// The parts that the lanes of a wave hold as one, the same in every lane: one lane's P stays apart.  `apart(m)`: how far the
// lane's sums are to move to be seen from m.
template <bool ENT, typename Apart>
__device__ __forceinline__ Part join_lanes(float m, float P, float S, float X, Apart&& apart) {
  Part p;
  p.m = wave_max(m);
  const int first = wv::first_lane(__ballot(m == p.m) | (1ull << 63));
  p.P = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(P), first));
  if (static_cast<int>(threadIdx.x & 63) != first) {
    S += whole(P);
    rebase<ENT>(S, X, apart(p.m));
  }
  p.S = wave_sum(S);
  p.X = ENT ? wave_sum(X) : 0.0f;
  return p;
}
template <bool ENT>
__device__ __forceinline__ Part join_parts(const Part& q, float c) {
  return join_lanes<ENT>(q.m, q.P, q.S, q.X, [&](float m) { return parted(q.m, m, c); });
}
// A batch of a lane is of U vectors, `stride` apart, all below `end`.  again(add) goes over the wave's elements a second time, where
// the maximum lies far from 0.
template <bool ENT, int U, typename E, typename Again>
__device__ __forceinline__ Part wave_part(const Row<E>& row, const Sums& s, float c, int stride, int end, Again&& again) {
  Part p = join_lanes<ENT>(s.m, s.P, s.S, s.X, [&](float m) { return s.rc - m * c; });
  const float mc = p.m * c;
  if (fabsf(mc) <= kFar) {
    const float rounded = __builtin_fmaf(p.m, c, -mc), f = exp2_fast(-rounded);
    if constexpr (ENT) p.X = f * __builtin_fmaf(-rounded, p.P + p.S, p.X);
    p.P *= f;
    p.S *= f;
    if (p.P + p.S < 1.125f) {
      const int lane = threadIdx.x & 63, at = __builtin_amdgcn_readlane(s.at, wv::first_lane(__ballot(s.m == p.m)));
      float rest = 0.0f;
      if (lane < U * E::N && at >= 0 && at + lane / E::N * stride < end) {
        const float x = E::up(row.x[row.token(at + lane / E::N * stride, lane % E::N)]);
        rest = x == p.m ? 0.0f : exp2_fast((x - p.m) * c);
      }
      p.P = -wave_sum(rest);
    }
  } else if (fabsf(p.m) != INFINITY) {
    float S = 0.0f, X = 0.0f;
    again([&](float x) {
      const float d = (x - p.m) * c, e = exp2_fast(d);
      S += e;
      if constexpr (ENT) X = __builtin_fmaf(e, fmaxf(d, -1000.0f), X);
    });
    p.P = wave_sum(S);
    p.S = 0.0f;
    p.X = ENT ? wave_sum(X) : 0.0f;
  }
  return p;
}

// W parts as one.
template <bool ENT, int W>
__device__ __forceinline__ Part join_set(const Part (&q)[W], float c) {
  Part p{q[0].m, 0.0f, 0.0f, 0.0f};
#pragma unroll
  for (int w = 1; w < W; ++w) p.m = fmaxf(p.m, q[w].m);
  bool taken = false;
#pragma unroll
  for (int w = 0; w < W; ++w) {
    const bool top = !taken && q[w].m == p.m;
    float S = q[w].S + (top ? 0.0f : whole(q[w].P)), X = q[w].X;
    float S1 = S, X1 = X;
    rebase<ENT>(S1, X1, parted(q[w].m, p.m, c));
    p.P = top ? q[w].P : p.P;
    p.S += top ? S : S1;
    p.X += top ? X : X1;
    taken = taken || top;
  }
  return p;
}

struct RowSums {  // the same in every thread of the row
  float base;     // the maximum, 0 for a row of nothing but -inf
  float m;        // the maximum
  float log_s;    // log of the sum of exp((x - base) / T), 0 for such a row
  float H;        // entropy
  bool bad;       // the row holds a NaN or +inf
};
__device__ __forceinline__ RowSums finish(const Part& p) {
  const bool empty = p.m == -INFINITY;
  const float S = whole(p.P) + p.S, log_s = log_1p((__float_as_int(p.P) < 0 ? -p.P : p.P - 1.0f) + p.S);
  RowSums r;
  r.bad = S != S || p.m == INFINITY;
  r.m = r.bad ? NAN : p.m;
  r.base = empty ? 0.0f : p.m;
  r.log_s = r.bad ? NAN : empty ? 0.0f : log_s;
  r.H = r.bad ? NAN : empty ? 0.0f : log_s - p.X * kLn2 * __builtin_amdgcn_rcpf(S);
  return r;
}

// The row from its waves' parts (`lds`: NT / 64 of them).
template <int NT, bool ENT>
__device__ __forceinline__ RowSums join_waves(const Part& p, int tid, float c, Part* lds) {
  constexpr int W = NT / 64;
  if constexpr (W == 1) return finish(p);
  if ((tid & 63) == 0) lds[tid >> 6] = p;
  __syncthreads();
  if constexpr (W <= 4) {
    Part q[W];
#pragma unroll
    for (int w = 0; w < W; ++w) q[w] = lds[w];
    return finish(join_set<ENT, W>(q, c));
  }
  // (a lane each: the waves of one row share a CU, and sixteen joins one after the other took longer than the reductions)
  const Part q = (tid & 63) < W ? lds[tid & 63] : Part{-INFINITY, 0.0f, 0.0f, 0.0f};
  return finish(join_parts<ENT>(q, c));
}

// The alternatives.  Every lane keeps the largest element of its vectors (m1), the first vector that holds it (k1) and the
// largest element of its other vectors (m2).  The N-th largest of the lanes' (or, past 256 threads, of 256 groups of
// lanes') m1 is a bound that N elements reach; hardly more than those lie above it (with G groups G ln(G / (G - N)) are
// expected), and all lie in vectors k1, except where an m2 reaches it too.  So after one pass over the row a few vectors
// are read a second time, from cache, and a list of N and some candidates is put in order by counting.
template <int N>
constexpr int list_size() { return 64 * N + 64; }
struct Tops {
  float m1 = -INFINITY, m2 = -INFINITY;
  int k1 = 0;
  __device__ __forceinline__ void add(float vm, int k) {
    k1 = vm > m1 ? k : k1;
    m2 = __builtin_amdgcn_fmed3f(vm, m1, m2);  // (m2 <= m1)
    m1 = max3(m1, vm, vm);
  }
};

__device__ __forceinline__ unsigned order32(float x) { return ukey(__fadd_rn(x, 0.0f)); }  // (-0.0 as 0.0)
__device__ __forceinline__ u64 order64(unsigned key, int token) { return (static_cast<u64>(key) << 32) | static_cast<unsigned>(~token); }

template <int NT, int N>
struct TopLds {
  unsigned group[NT == 64 ? 1 : NT];
  int first[NT == 64 ? 1 : NT];
  __align__(16) u64 list[list_size<N>()];
  u64 best;
  int rank[NT == 64 ? 1 : 128];
  int count;
  __device__ __forceinline__ void clear(int tid) {  // (before a barrier)
    if (tid == 0) count = 0;
    if (NT > 64 && tid < 128) rank[tid] = 0;
  }
};

// The largest b that at least `n` keys of the row's groups reach (0: there are fewer); a wave holds them all, PER per lane.
template <int PER>
__device__ __forceinline__ int how_many(const unsigned (&key)[PER], unsigned b) {
  int n = 0;
#pragma unroll
  for (int i = 0; i < PER; ++i) n += __builtin_popcountll(__ballot(key[i] >= b));
  return n;
}
// For few of 64 keys: one maximum after the other.  Otherwise between the smallest and the largest key, in quarters (three counts
// at a time do not wait for each other): four or five steps until exactly n reach one of the three, 16 at most (equal keys).
// (16384 x 1025 fp32 with entropy, 4 / 8 / 12 / 20 alternatives: 17.4 19.4 21.8 26.8 us by maxima, 18.7 20.1 21.5 24.7 in quarters.)
constexpr int kFewSteps = 8;
template <int PER>
__device__ __forceinline__ unsigned bound_of(const unsigned (&key)[PER], int n) {
  if (how_many(key, 1u) < n) return 0u;
  if (PER == 1 && n <= kFewSteps) {
    unsigned left = key[0];
    for (int reached = 0;;) {
      const unsigned b = wv::wave_max_u(left);
      reached += __builtin_popcountll(__ballot(left == b));
      if (reached >= n) return b;
      left = left == b ? 0u : left;
    }
  }
  unsigned most = key[0], least = key[0] - 1u;  // (a key of 0 is none)
#pragma unroll
  for (int i = 1; i < PER; ++i) {
    most = max(most, key[i]);
    least = min(least, key[i] - 1u);
  }
  unsigned lo = ~wv::wave_max_u(~least) + 1u, hi = wv::wave_max_u(most);  // n keys or more reach lo, fewer reach hi + 1
  while (lo < hi) {
    const unsigned step = (hi - lo) / 4 + 1, t1 = lo + step, t2 = t1 + min(hi - t1, step), t3 = t2 + min(hi - t2, step);
    const int n1 = how_many(key, t1), n2 = how_many(key, t2), n3 = how_many(key, t3);
    hi = n1 < n ? t1 - 1 : n2 < n ? t2 - 1 : n3 < n ? t3 - 1 : hi;
    lo = n3 >= n ? t3 : n2 >= n ? t2 : n1 >= n ? t1 : lo;
    if (n3 == n || n2 == n || n1 == n) break;
  }
  return lo;
}

// The same, from a lane's largest key alone where there are lanes enough (a bound of 20 from 64 groups instead of 256 admits 24
// candidates instead of 21, and takes a quarter of the instructions).
template <int PER>
__device__ __forceinline__ unsigned some_bound_of(const unsigned (&key)[PER], int n) {
  if (PER == 1 || n > 24) return bound_of(key, n);
  unsigned most[1] = {key[0]};
#pragma unroll
  for (int i = 1; i < PER; ++i) most[0] = max(most[0], key[i]);
  const unsigned b = bound_of(most, n);
  return b != 0u ? b : bound_of(key, n);
}

// Candidates into the list: of every lane that calls, the elements of vector v that the bound admits, an element of all lanes
// after the other (additions of a number of its own by every lane to the count became a loop over the lanes: 13540 x 704 fp16,
// the largest element 13.4 -> 11.4 us).
template <int NT, int M>
__device__ __forceinline__ int places(TopLds<NT, M>& lds, int n) {  // of n candidates of the wave
  int at = 0;
  if (__lane_id() == static_cast<unsigned>(wv::first_lane(__ballot(true)))) at = atomicAdd(&lds.count, n);
  return uniform_i(at);
}
__device__ __forceinline__ int lanes_before(u64 who) {
  return __builtin_amdgcn_mbcnt_hi(static_cast<unsigned>(who >> 32), __builtin_amdgcn_mbcnt_lo(static_cast<unsigned>(who), 0u));
}
template <typename E, int NT>
__device__ __forceinline__ void push_vector(const Row<E>& row, const float (&x)[E::N], int v, unsigned b, int last, TopLds<NT, E::N>& lds) {
  const float least = b == 0u ? -INFINITY : ukey_val(v <= last ? b : b + 1);  // (as good an order as the keys', -0.0 as 0.0)
  u64 who[E::N];
  int n = 0;
#pragma unroll
  for (int i = 0; i < E::N; ++i) {
    who[i] = __ballot(x[i] >= least);
    n += __builtin_popcountll(who[i]);
  }
  if (n == 0) return;
  int at = places(lds, n);
#pragma unroll
  for (int i = 0; i < E::N; ++i)
    if (who[i] != 0) {
      const int to = at + lanes_before(who[i]);
      if (x[i] >= least && to < list_size<E::N>()) lds.list[to] = order64(order32(x[i]), row.token(v, i));
      at += __builtin_popcountll(who[i]);
    }
}
template <typename E, int NT>
__device__ __forceinline__ void push_edge(const Row<E>& row, int tid, float edge, unsigned b, TopLds<NT, E::N>& lds) {
  if (tid < row.edges && order32(edge) >= b) {
    const int at = atomicAdd(&lds.count, 1);
    if (at < list_size<E::N>()) lds.list[at] = order64(order32(edge), row.edge_token(tid));
  }
}

// The first n elements of the vectors that equal the bound (some may fall behind larger elements of the list).
template <typename E, int NT>
__device__ __forceinline__ void push_equal(const Row<E>& row, int tid, unsigned b, int n, int* found, TopLds<NT, E::N>& lds) {
  constexpr int W = NT / 64;
  for (int before = 0, at = 0; at < row.nv && before < n; at += NT) {
    unsigned equal = 0;
    float x[E::N];
    if (at + tid < row.nv) {
      E::unpack(row.vec(at + tid), x);
#pragma unroll
      for (int i = 0; i < E::N; ++i) equal |= order32(x[i]) == b ? 1u << i : 0u;
    }
    int mine = 0, wave = 0;  // equal elements of the wave's lanes before this one, and of all
#pragma unroll
    for (int i = 0; i < E::N; ++i) {
      const u64 who = __ballot((equal >> i) & 1u);
      mine += __builtin_amdgcn_mbcnt_hi(static_cast<unsigned>(who >> 32), __builtin_amdgcn_mbcnt_lo(static_cast<unsigned>(who), 0u));
      wave += __builtin_popcountll(who);
    }
    if ((tid & 63) == 0) found[tid >> 6] = wave;
    __syncthreads();
    int total = 0;
    for (int w = 0; w < W; ++w) {
      if (w < (tid >> 6)) mine += found[w];
      total += found[w];
    }
    mine += before;
#pragma unroll
    for (int i = 0; i < E::N; ++i)
      if ((equal >> i) & 1u) {
        if (mine < n) {
          const int to = atomicAdd(&lds.count, 1);
          if (to < list_size<E::N>()) lds.list[to] = order64(b, row.token(at + tid, i));
        }
        ++mine;
      }
    before += total;
    __syncthreads();
  }
}

// (x - base) / T - log of the sum.  The difference is taken of halves, which changes no bit of it: of the largest and the lowest value
// of a type it passes the fp32 range, where the quotient need not.
__device__ __forceinline__ float log_prob(float x, float base, float inv, float logs) {
  return __builtin_fmaf(__builtin_fmaf(x, 0.5f, -0.5f * base), 2.0f * inv, -logs);
}

struct TopOut {
  int n;
  float base, inv, logs;
  int32_t* tokens;
  float* logp;
  __device__ __forceinline__ void write(int rank, u64 k) const {
    tokens[rank] = static_cast<int32_t>(~static_cast<unsigned>(k));
    logp[rank] = log_prob(ukey_val(static_cast<unsigned>(k >> 32)), base, inv, logs);
  }
};
// The list in order.  Where there were more candidates than it holds (the largest values crowd in a few groups): one
// alternative after the other, each a pass over the row.
template <typename E, int NT>
__device__ __forceinline__ void write_list(const Row<E>& row, int tid, float edge, const TopOut& out, TopLds<NT, E::N>& lds) {
  row_sync<NT>();
  int count = uniform_i(lds.count);
  if (count <= list_size<E::N>()) {
    constexpr int W = NT / 64;
    if (W > 1 && count <= 128) {  // (every wave compares all of them with its share of the list)
      const int share = (count + W - 1) / W, from = share * (tid >> 6), to = min(from + share, count);
      for (int i = tid & 63; i < count; i += 64) {
        const u64 k = lds.list[i];
        int rank = 0;
        for (int j = from; j < to; ++j) rank += lds.list[j] > k ? 1 : 0;
        if (rank) atomicAdd(&lds.rank[i], rank);
      }
      row_sync<NT>();
      if (tid < count && lds.rank[tid] < out.n) out.write(lds.rank[tid], lds.list[tid]);
      return;
    }
    if (NT == 64 && count > 64) {
      // Few groups for so many alternatives, or fewer tokens left by a mask: a bound of the candidates themselves (the lower
      // tokens among those that equal it), and those that reach it to the front.  (10 x 192 fp32, 56 alternatives: 15.9 us with
      // each of the 192 compared with all, 7.2 so; 9024 x 769 bf16, 95 % masked, 48 of them: 174 and 58.)
      constexpr int PER = list_size<E::N>() / 64;
      u64 held[PER];
      unsigned key[PER], place[PER];
#pragma unroll
      for (int i = 0; i < PER; ++i) {
        held[i] = 64 * i + tid < count ? lds.list[64 * i + tid] : 0u;
        key[i] = static_cast<unsigned>(held[i] >> 32);
      }
      const unsigned b = bound_of(key, out.n);
      unsigned first = 0u;
      if (how_many(key, b) > 64) {
#pragma unroll
        for (int i = 0; i < PER; ++i) place[i] = key[i] == b ? static_cast<unsigned>(held[i]) : 0u;
        first = bound_of(place, out.n - how_many(key, b + 1));
      }
      const u64 least = (static_cast<u64>(b) << 32) | first;
      int n = 0;
#pragma unroll
      for (int i = 0; i < PER; ++i) {
        const u64 who = __ballot(held[i] >= least);
        const int before = __builtin_popcountll(who & ((u64{1} << tid) - 1));
        if (held[i] >= least) lds.list[n + before] = held[i];
        n += __builtin_popcountll(who);
      }
      count = n;
      row_sync<64>();
    }
    for (int i = tid; i < count; i += NT) {
      const u64 k = lds.list[i];
      int rank = 0;
      for (int j = 0; j < count; j += 2) {
        const ulonglong2 q = *reinterpret_cast<const ulonglong2*>(lds.list + j);  // (behind the last one: anything)
        rank += (q.x > k ? 1 : 0) + (j + 1 < count && q.y > k ? 1 : 0);
      }
      if (rank < out.n) out.write(rank, k);
    }
    return;
  }
  u64 before = ~0ull;
  for (int n = 0; n < out.n; ++n) {
    u64 best = 0;
    auto take = [&](float x, int token) {
      const u64 k = order64(order32(x), token);
      best = k < before && k > best ? k : best;
    };
    for (int v = tid; v < row.nv; v += NT) {
      float x[E::N];
      E::unpack(row.vec(v), x);
#pragma unroll
      for (int i = 0; i < E::N; ++i) take(x[i], row.token(v, i));
    }
    if (tid < row.edges) take(edge, row.edge_token(tid));
    if (tid == 0) lds.best = 0;
    row_sync<NT>();
    atomicMax(&lds.best, best);
    row_sync<NT>();
    before = lds.best;
    if (tid == 0) out.write(n, before);
    row_sync<NT>();
  }
}

template <typename E, int NT>
__device__ __forceinline__ void write_alternatives(const Row<E>& row, int tid, const Tops& tops, float edge, const TopOut& out,
                                                   TopLds<NT, E::N>& lds) {
  constexpr int GROUPS = NT < kGroups ? NT : kGroups, PER = GROUPS / 64, PARTS = NT / GROUPS;
  const int lane = tid & 63;
  const bool some = tid < row.nv;
  const unsigned own = some ? order32(tops.m1) : 0u;
  lds.clear(tid);
  unsigned key[PER];
  if constexpr (NT == 64) {
    key[0] = own;
  } else {
    lds.group[tid] = own;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      key[i] = 0u;
#pragma unroll
      for (int p = 0; p < PARTS; ++p) key[i] = max(key[i], lds.group[GROUPS * p + 64 * i + lane]);
    }
  }
  const unsigned b = some_bound_of(key, out.n);
  // Elements equal to the bound count in the order of their tokens.  Where many groups have it for their maximum (masked
  // rows with fewer tokens left than alternatives wanted, flat rows), only those up to vector `last` are wanted: the groups
  // above it are not enough by `need`, and the `need` lowest vectors in which a group has its maximum hold so many.
  // (68 x 129 fp16, 95 % of it masked, one alternative: 14.7 us with all of a masked row's elements ranked, 4.6 so; the bound of
  // an ordinary row admits up to some 5 groups more than n and goes without.)
  int last = INT_MAX;
  if (b != 0u && how_many(key, b) > out.n + 8) {
    int first[PER];
    if constexpr (NT == 64) {
      first[0] = tops.k1 * NT + tid;
    } else {
      lds.first[tid] = tops.k1 * NT + tid;
      __syncthreads();
#pragma unroll
      for (int i = 0; i < PER; ++i) {
        first[i] = INT_MAX;
#pragma unroll
        for (int p = 0; p < PARTS; ++p) {
          const int at = GROUPS * p + 64 * i + lane;
          if (lds.group[at] == b) first[i] = min(first[i], lds.first[at]);
        }
      }
    }
    unsigned place[PER];  // (the need-th smallest is the need-th largest of the complements)
#pragma unroll
    for (int i = 0; i < PER; ++i) place[i] = key[i] == b ? static_cast<unsigned>(INT_MAX - first[i]) : 0u;
    last = INT_MAX - static_cast<int>(bound_of(place, out.n - how_many(key, b + 1)));
  }
  row_sync<NT>();
  const int v1 = tops.k1 * NT + tid;
  const bool mine = some && (own > b || (own == b && v1 <= last));
  if (mine) {
    float x[E::N];
    E::unpack(row.vec(v1), x);
    push_vector<E, NT>(row, x, v1, b, last, lds);
  }
  // the other vectors of lanes that have more above the bound: of one such lane after the other by the whole wave, or, where
  // they are many, by all of them at once
  if (row.nv > NT) {
    const unsigned k2 = order32(tops.m2);
    u64 more = __ballot(mine && (k2 > b || (k2 == b && (v1 == tid ? tid + NT : tid) <= last)));
    if (__builtin_popcountll(more) < row.nv / NT) {
      for (; more; more &= more - 1) {
        const int from = wv::first_lane(more), skip = __builtin_amdgcn_readlane(v1, from);
        for (int v = lane * NT + (tid & ~63) + from; v < row.nv; v += 64 * NT)
          if (v != skip) {
            float x[E::N];
            E::unpack(row.vec(v), x);
            push_vector<E, NT>(row, x, v, b, last, lds);
          }
      }
    } else if ((more >> lane) & 1u) {
      for (int v = tid; v < row.nv; v += NT)
        if (v != v1) {
          float x[E::N];
          E::unpack(row.vec(v), x);
          push_vector<E, NT>(row, x, v, b, last, lds);
        }
    }
  }
  push_edge<E, NT>(row, tid, edge, b, lds);
  write_list<E, NT>(row, tid, edge, out, lds);
}

// What a row's sums say, and the scores of the given tokens.
__device__ __forceinline__ void write_scores(const LogprobArgs& a, int64_t r, int tid, const RowSums& sums, int given, float given_x) {
  if (tid < a.n_tokens) a.logp[r * a.n_tokens + tid] = given < 0 ? NAN : log_prob(given_x, sums.base, a.in.inv_temp, sums.log_s);
  if (tid == 0) {
    if (a.entropy) a.entropy[r] = sums.H;
    if (a.stats) {
      a.stats[3 * r + 0] = sums.m;
      a.stats[3 * r + 1] = sums.log_s;
      a.stats[3 * r + 2] = sums.H;
    }
  }
  if (sums.bad && tid < a.n_top) {
    a.top_tokens[r * a.n_top + tid] = -1;
    a.top_logp[r * a.n_top + tid] = NAN;
  }
}
template <typename E>
__device__ __forceinline__ int load_given(const LogprobArgs& a, int64_t r, const Row<E>& row, int tid, float& x) {
  x = 0.0f;
  if (tid >= a.n_tokens) return -1;
  const int t = a.tokens[r * a.n_tokens + tid];
  if (static_cast<unsigned>(t) >= static_cast<unsigned>(row.V)) return -1;
  x = E::up(row.x[t]);
  return t;
}

// One row, by a workgroup, or (NT == 64: rows of up to kWaveVectors vectors) by a wave, four in a workgroup.  Large calls of long
// rows are bound by HBM (8192 x 32001 bf16, 32 alternatives: 100 us, 5.2 TB/s), those of short rows by vector instructions (16000 x
// 1025 fp32 with entropy: 12.5 us, 5.2 TB/s; with 5 alternatives 17.2 us, 509 instructions a wave, 79 - 80 % of the cycles), small ones
// by the launch and one row's chain of loads and reductions (32 x 1024 fp32: 3.1 us).
static_assert(kWaveVectors == 2 * 64 * kUnroll, "a wave requests its row in two batches");
template <typename E, int NT, bool ENT, bool TOP>
__global__ __launch_bounds__(NT == 64 ? 256 : NT) void logprobs_kernel(LogprobArgs a) {
  constexpr int ROWS = NT == 64 ? 4 : 1;
  __shared__ Part s_sums[ROWS][NT / 64];
  __shared__ TopLds<TOP ? NT : 64, TOP ? E::N : 1> s_top[TOP ? ROWS : 1];
  const int sub = NT == 64 ? uniform_i(threadIdx.x >> 6) : 0, tid = NT == 64 ? threadIdx.x & 63 : threadIdx.x;
  const int64_t r = static_cast<int64_t>(blockIdx.x) * ROWS + sub;
  if (ROWS > 1 && r >= a.in.rows) return;
  const Row<E> row = row_at<E>(a.in.x, a.in.stride, r, a.in.V);
  const float inv = a.in.inv_temp, c = a.in.c;
  // (all that does not depend on other loads is requested before the first wait: the token, the first vectors, the edge)
  int given = -1;
  if (tid < a.n_tokens) given = a.tokens[r * a.n_tokens + tid];
  constexpr bool AHEAD = NT == 64;  // (a wave requests all of its row at once; more waves hide each other's waits)
  v4u raw[kUnroll], more[AHEAD ? kUnroll : 1];
  auto load = [&](auto& to, int k) {  // vectors k, k + 1, ... of the thread; behind the row's end its last one again
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) to[u] = row.vec(min((k + u) * NT + tid, row.nv - 1));
  };
  if (row.nv > 0) load(raw, 0);
  if constexpr (AHEAD)
    if (row.nv > kUnroll * NT) load(more, kUnroll);
  float edge = -INFINITY;
  if (tid < row.edges) edge = E::up(row.x[row.edge_token(tid)]);
  float given_x = 0.0f;
  if (static_cast<unsigned>(given) < static_cast<unsigned>(row.V)) given_x = E::up(row.x[given]);
  else given = -1;
  Sums s(a.in.far);
  Tops tops;
  auto batch = [&](auto count, const auto& raw, int k) {
    constexpr int U = decltype(count)::value;
    float x[U][E::N], m = -INFINITY;
#pragma unroll
    for (int u = 0; u < U; ++u) {
      E::unpack(raw[u], x[u]);
      const float vm = vec_max(x[u]);
      if constexpr (TOP) tops.add(vm, k + u);
      m = u == 0 ? vm : max3(m, vm, vm);
    }
    s.m = max3(s.m, m, m);
    add_batch<ENT>(s, x, m, c, k * NT + tid);
  };
  using std::integral_constant;
  auto run = [&](auto& raw, int k) {
    const int left = row.nv - k * NT;  // (uniform, > 0)
    if (left < kUnroll * NT) {
#pragma unroll
      for (int u = 0; u < kUnroll; ++u)
        if ((k + u) * NT + tid >= row.nv) raw[u] = E::nothing();
    }
    if (left > 3 * NT) batch(integral_constant<int, 4>{}, raw, k);
    else if (left > 2 * NT) batch(integral_constant<int, 3>{}, raw, k);
    else if (left > NT) batch(integral_constant<int, 2>{}, raw, k);
    else batch(integral_constant<int, 1>{}, raw, k);
  };
  static_assert(kUnroll == 4, "run() takes up to four vectors");
  if constexpr (AHEAD) {
    if (row.nv > 0) run(raw, 0);
    if (row.nv > kUnroll * NT) run(more, kUnroll);
  } else {
    for (int k = 0; k * NT < row.nv; k += kUnroll) {
      if (k > 0) load(raw, k);
      run(raw, k);
    }
  }
  if (tid < row.edges) {
    const float x[1][1] = {{edge}};
    s.m = fmaxf(s.m, edge);
    add_batch<ENT>(s, x, edge, c, -1);
  }
  const Part part = wave_part<ENT, kUnroll>(row, s, c, NT, row.nv, [&](auto&& add) {
    for (int v = tid; v < row.nv; v += NT) {
      float x[E::N];
      E::unpack(row.vec(v), x);
#pragma unroll
      for (int i = 0; i < E::N; ++i) add(x[i]);
    }
    if (tid < row.edges) add(edge);
  });
  const RowSums sums = join_waves<NT, ENT>(part, tid, c, s_sums[sub]);
  write_scores(a, r, tid, sums, given, given_x);
  if constexpr (TOP) {
    if (!sums.bad)
      write_alternatives<E, NT>(row, tid, tops, edge, TopOut{a.n_top, sums.base, inv, sums.log_s, a.top_tokens + r * a.n_top, a.top_logp + r * a.n_top},
                                s_top[sub]);
  }
}

// Few long rows: every wave takes 64 * `each` vectors of a row and leaves their part in the workspace, with the largest element
// of the vectors, its token and the largest of the others; a workgroup per row joins them.  The parts' largest elements bound
// the alternatives as the lanes' do above, and are candidates themselves; the few parts with a second one are read again.
// Both are bound by latency: 1 x 131072 bf16, 20 alternatives, 3.5 us and 5.6 us.
struct PartRecord {
  Part sums;
  float top, second;
  int token, unused;
};
template <typename E, bool ENT, bool TOP>
__global__ __launch_bounds__(256) void logprobs_parts_kernel(LogprobArgs a, int parts, int each, PartRecord* __restrict__ out) {
  const int64_t at = static_cast<int64_t>(blockIdx.x) * 4 + uniform_i(threadIdx.x >> 6);
  const int64_t r = at / parts;
  if (r >= a.in.rows) return;
  const int lane = threadIdx.x & 63, begin = static_cast<int>(at - r * parts) * 64 * each;
  const Row<E> row = row_at<E>(a.in.x, a.in.stride, r, a.in.V);
  const float c = a.in.c;
  const int end = min(begin + 64 * each, row.nv);
  Sums s(a.in.far);
  Tops tops;
  for (int v0 = begin + lane; v0 < end; v0 += 64 * kUnroll) {
    v4u raw[kUnroll];
#pragma unroll
    for (int u = 0; u < kUnroll; ++u)
      if (v0 + 64 * u < end) raw[u] = row.vec(v0 + 64 * u);
#pragma unroll
    for (int u = 0; u < kUnroll; ++u)
      if (v0 + 64 * u < end) {
        float x[1][E::N];
        E::unpack(raw[u], x[0]);
        const float vm = vec_max(x[0]);
        if constexpr (TOP) tops.add(vm, v0 + 64 * u);
        s.m = fmaxf(s.m, vm);
        add_batch<ENT>(s, x, vm, c, v0 + 64 * u);
      }
  }
  const bool has_edge = begin == 0 && lane < row.edges;  // (the first part has the edge as well)
  float edge = -INFINITY;
  if (has_edge) {
    edge = E::up(row.x[row.edge_token(lane)]);
    const float x[1][1] = {{edge}};
    s.m = fmaxf(s.m, edge);
    add_batch<ENT>(s, x, edge, c, -1);
  }
  const Part p = wave_part<ENT, 1>(row, s, c, 64, end, [&](auto&& add) {
    for (int v = begin + lane; v < end; v += 64) {
      float x[E::N];
      E::unpack(row.vec(v), x);
#pragma unroll
      for (int i = 0; i < E::N; ++i) add(x[i]);
    }
    if (has_edge) add(edge);
  });
  PartRecord rec{p, -INFINITY, -INFINITY, 0, 0};
  if constexpr (TOP) {
    // (a lane without vectors, or with nothing but -inf in them, keeps its first one in k1)
    const int own = tops.m1 == -INFINITY ? begin + lane : tops.k1;
    rec.top = wave_max(tops.m1);
    const int v = wv::wave_min_nn(tops.m1 == rec.top && own < end ? own : INT_MAX);
    if (v < end) {
      float x[E::N], rest = -INFINITY;
      E::unpack(row.vec(v), x);
      int i = E::N;
#pragma unroll
      for (int k = E::N - 1; k >= 0; --k) i = x[k] == rec.top ? k : i;
#pragma unroll
      for (int k = 0; k < E::N; ++k) rest = k == i ? rest : fmaxf(rest, x[k]);
      rec.token = row.token(v, min(i, E::N - 1));
      rec.second = fmaxf(rest, wave_max(own == v ? tops.m2 : tops.m1));
    }
  }
  if (lane == 0) out[at] = rec;
}

// Every wave joins all parts by itself (a few instructions, no barrier); the parts that reach the bound are dealt out to the
// waves.
constexpr int kJoinThreads = 512;
template <typename E, bool ENT, bool TOP>
__global__ __launch_bounds__(kJoinThreads) void logprobs_join_kernel(LogprobArgs a, int parts, int each, const PartRecord* __restrict__ in) {
  constexpr int NT = kJoinThreads, W = NT / 64, PER = kMaxParts / 64;
  __shared__ TopLds<TOP ? NT : 64, TOP ? E::N : 1> lds;
  __shared__ int s_found[W];
  __shared__ short s_part[W][kMaxParts];
  const int64_t r = blockIdx.x;
  const int tid = threadIdx.x, lane = tid & 63, wave = uniform_i(tid >> 6);
  if constexpr (TOP) {
    lds.clear(tid);
    __syncthreads();
  }
  const Row<E> row = row_at<E>(a.in.x, a.in.stride, r, a.in.V);
  const float c = a.in.c;
  Part p[PER];
  unsigned key[PER];
  float top[PER], second[PER];
  int token[PER];
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const int at = 64 * i + lane;
    p[i] = Part{-INFINITY, 0.0f, 0.0f, 0.0f};
    top[i] = second[i] = -INFINITY;
    token[i] = 0;
    if (at < parts) {
      const PartRecord rec = in[r * parts + at];
      p[i] = rec.sums;
      top[i] = rec.top;
      second[i] = rec.second;
      token[i] = rec.token;
    }
    // (a row's head may leave its last part empty)
    key[i] = at < parts && at * 64 * each < row.nv ? order32(top[i]) : 0u;
  }
  float given_x, edge = -INFINITY;
  const int given = load_given<E>(a, r, row, tid, given_x);
  if (tid < row.edges) edge = E::up(row.x[row.edge_token(tid)]);
  const Part all = join_set<ENT, PER>(p, c);
  const RowSums sums = finish(join_parts<ENT>(all, c));
  if (wave == 0) write_scores(a, r, tid, sums, given, given_x);
  if constexpr (TOP) {
    if (sums.bad) return;
    const TopOut out{a.n_top, sums.base, a.in.inv_temp, sums.log_s, a.top_tokens + r * a.n_top, a.top_logp + r * a.n_top};
    const unsigned b = some_bound_of(key, out.n);
    const bool ties = b != 0u && how_many(key, b) > out.n + 16;  // (then the elements equal to the bound are looked for in order)
    const int last = ties ? -1 : INT_MAX;
    int n = 0;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const bool take = key[i] > b || (key[i] == b && key[i] != 0u && !ties);
      if (wave == W - 1 && take) {
        const int to = atomicAdd(&lds.count, 1);
        if (to < list_size<E::N>()) lds.list[to] = order64(key[i], token[i]);
      }
      const unsigned k2 = order32(second[i]);
      const bool again = take && (ties ? k2 > b : k2 >= b);
      const u64 who = __ballot(again);
      if (again) s_part[wave][n + __builtin_amdgcn_mbcnt_hi(static_cast<unsigned>(who >> 32), __builtin_amdgcn_mbcnt_lo(static_cast<unsigned>(who), 0u))] = static_cast<short>(64 * i + lane);
      n += __builtin_popcountll(who);
    }
    row_sync<64>();
    for (int t0 = wave; t0 < n * each; t0 += W) {  // (64 vectors of a part a turn)
      const int i = t0 / each, part = uniform_i(s_part[wave][i]), v = part * 64 * each + (t0 - i * each) * 64 + lane;
      if (v < row.nv) {
        float x[E::N];
        E::unpack(row.vec(v), x);
        const int skip = in[r * parts + part].token - row.token(v, 0);  // (the part's largest element is a candidate already)
#pragma unroll
        for (int k = 0; k < E::N; ++k) x[k] = k == skip ? NAN : x[k];
        push_vector<E, NT>(row, x, v, b, last, lds);
      }
    }
    push_edge<E, NT>(row, tid, edge, b, lds);
    if (ties) push_equal<E, NT>(row, tid, b, out.n, s_found, lds);
    write_list<E, NT>(row, tid, edge, out, lds);
  }
}

// Gradient: p (A + B log2 p) with A = -(G + h H) / T, B = -h ln(2) / T for all tokens, plus what the given ones take.  A
// workgroup takes kUnroll vectors a thread of one row (a wave, four rows a workgroup, where those hold the row).  The
// gradients on the given tokens are computed before anything is written and stored behind the rest.  Bound by HBM (4096 x 50000
// bf16: 134 us, 6.1 TB/s, more than a plain copy's 5.2), small calls by the launch.
template <typename E, int NT, bool STREAM>
__global__ __launch_bounds__(256) void logprobs_backward_kernel(LogprobGradArgs a, int parts) {
  constexpr int ROWS = 256 / NT, PART = NT * kUnroll;
  const int sub = ROWS > 1 ? uniform_i(threadIdx.x / NT) : 0, tid = threadIdx.x % NT;
  const int64_t r = ROWS > 1 ? static_cast<int64_t>(blockIdx.x) * ROWS + sub : blockIdx.x / parts;
  const int part = ROWS > 1 ? 0 : blockIdx.x % parts;
  if (ROWS > 1 && r >= a.in.rows) return;
  const Row<E> row = row_at<E, 64>(a.in.x, a.in.stride, r, a.in.V);
  typename E::type* out = static_cast<typename E::type*>(a.grad) + r * a.grad_stride;
  v4u raw[kUnroll];
#pragma unroll
  for (int u = 0; u < kUnroll; ++u)
    if (part * PART + u * NT + tid < row.nv) raw[u] = row.template vec_once<STREAM>(part * PART + u * NT + tid);
  const bool has_edge = part == 0 && tid < row.edges;
  float edge = 0.0f;
  if (has_edge) edge = E::up(row.x[row.edge_token(tid)]);
  const float inv = a.in.inv_temp, c = a.in.c;
  const float m = a.stats[3 * r], logs = a.stats[3 * r + 1], H = a.stats[3 * r + 2];
  const float h = a.grad_entropy ? a.grad_entropy[r] : 0.0f;
  const int lane = threadIdx.x & 63;
  int given = -1;
  bool mine = false;  // the token lies in this part, which writes it, after its other stores
  float g = 0.0f, given_x = 0.0f;
  if (lane < a.n_tokens && a.grad_logp) {
    given = a.tokens[r * a.n_tokens + lane];
    if (static_cast<unsigned>(given) < static_cast<unsigned>(a.in.V)) {
      g = a.grad_logp[r * a.n_tokens + lane];
      mine = part == (given < row.head || given >= row.head + row.nv * E::N ? 0 : (given - row.head) / E::N / PART);
      if (mine) given_x = E::up(row.x[given]);
    } else {
      given = -1;
    }
  }
  const float G = wave_sum(g);
  const bool none = (__ballot(g != 0.0f) == 0 && h == 0.0f) || m == -INFINITY;
  const float hH = h == 0.0f ? 0.0f : h * H;  // (H counts for nothing where h does)
  const float A = none ? 0.0f : m != m ? NAN : -(G + hH) * inv, B = none ? 0.0f : -h * kLn2 * inv, log2s = logs * kLog2e;
  auto pull = [&](float x) {
    const float d = fmaxf(__builtin_fmaf(x - m, c, -log2s), -1000.0f);
    return exp2_fast(d) * __builtin_fmaf(B, d, A);
  };
  float onto = g, rest = 0.0f;  // what the given token takes, listed once or several times, and what the others do
  if (a.n_tokens > 1 && a.grad_logp) {
    onto = 0.0f;
    for (int k = 0; k < a.n_tokens; ++k) {
      const float gk = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(g), k));
      const bool same = __builtin_amdgcn_readlane(given, k) == given;
      onto += same ? gk : 0.0f;
      rest += same ? 0.0f : gk;
    }
  }
  // (onto - p G as (1 - p) onto - p rest: the difference would have the rounding of onto where p is near 1, and of G where p is small and
  // little falls onto the token; and 1 - p = 1 - e^l comes from its series where p is near 1, the next term l^6 / 5040 of it)
  const float l = __builtin_fmaf(given_x - m, inv, -logs), d = fmaxf(__builtin_fmaf(given_x - m, c, -log2s), -1000.0f), p = exp2_fast(d);
  float series = __builtin_fmaf(l, 1.0f / 6, 1.0f);
  series = __builtin_fmaf(l * series, 1.0f / 5, 1.0f);
  series = __builtin_fmaf(l * series, 1.0f / 4, 1.0f);
  series = __builtin_fmaf(l * series, 1.0f / 3, 1.0f);
  series = __builtin_fmaf(l * series, 1.0f / 2, 1.0f);
  const float not_p = l > -0.25f ? -l * series : 1.0f - p;
  const float taken = m != m ? NAN : p * __builtin_fmaf(B, d, -hH * inv) + __builtin_fmaf(-p, rest, not_p * onto) * inv;
  if constexpr (NT > 64) __syncthreads();
#pragma unroll
  for (int u = 0; u < kUnroll; ++u) {
    const int v = part * PART + u * NT + tid;
    if (v < row.nv) {
      float x[E::N];
      E::unpack(raw[u], x);
#pragma unroll
      for (int i = 0; i < E::N; ++i) x[i] = none ? 0.0f : pull(x[i]);
      stream_vector<E>(out + row.token(v, 0), E::pack(x));
    }
  }
  if (has_edge) out[row.edge_token(tid)] = E::down(none ? 0.0f : pull(edge));
  row_sync<NT>();
  if (threadIdx.x % NT < 64 && mine && !none) out[given] = E::down(taken);
}

template <typename E>
int forward(const LogprobArgs& a, void* workspace, hipStream_t stream) {
  const bool ent = a.entropy || a.stats, top = a.n_top > 0;
  auto done = [] { return hipGetLastError() == hipSuccess ? PB_OK : PB_EHIP; };
  const RowSplit split = split_logprobs(a.in.V / E::N, a.in.all_rows, a.in.V);
  if (split.parts > 0) {
    PartRecord* ws = static_cast<PartRecord*>(workspace);
    const int grid = static_cast<int>((static_cast<int64_t>(a.in.rows) * split.parts + 3) / 4);
    auto begin = [&](auto kernel) { kernel<<<grid, 256, 0, stream>>>(a, split.parts, split.each, ws); };
    if (ent && top) begin(logprobs_parts_kernel<E, true, true>);
    else if (ent) begin(logprobs_parts_kernel<E, true, false>);
    else if (top) begin(logprobs_parts_kernel<E, false, true>);
    else begin(logprobs_parts_kernel<E, false, false>);
    if (done() != PB_OK) return PB_EHIP;
    auto finish = [&](auto kernel) { kernel<<<a.in.rows, kJoinThreads, 0, stream>>>(a, split.parts, split.each, ws); return done(); };
    if (ent && top) return finish(logprobs_join_kernel<E, true, true>);
    if (ent) return finish(logprobs_join_kernel<E, true, false>);
    if (top) return finish(logprobs_join_kernel<E, false, true>);
    return finish(logprobs_join_kernel<E, false, false>);
  }
  auto pick = [&](auto nt) {
    constexpr int NT = decltype(nt)::value;
    constexpr int ROWS = NT == 64 ? 4 : 1, THREADS = NT == 64 ? 256 : NT;
    auto go = [&](auto kernel) { kernel<<<(a.in.rows + ROWS - 1) / ROWS, THREADS, 0, stream>>>(a); return done(); };
    if (ent && top) return go(logprobs_kernel<E, NT, true, true>);
    if (ent) return go(logprobs_kernel<E, NT, true, false>);
    if (top) return go(logprobs_kernel<E, NT, false, true>);
    return go(logprobs_kernel<E, NT, false, false>);
  };
  // Threads a row, us with 128 / 256 / 512 / 1024, bf16: 16384 x 8192, 8 alternatives: 59 73 114 312; 5000 x 4104 without: 11.5 12.6
  // 17.4 29; 1024 x 16384, 20 of them: 14.6 14.9 19.0 35; 8192 x 32001, 8 of them: 103 99 106 209; 400 x 33000, 5 of them and entropy:
  // 15.1 11.7 11.7 16.6.  A row a CU and fewer, 5 of them and entropy: 200 x 6000 6.4 6.1 6.0 6.3; 64 x 12000 7.0 6.5 6.1 6.8; 256 x 33000
  // 12.9 10.0 8.7 9.8; 64 x 50000 13.7 9.9 8.7 9.0; 256 x 60000 18.3 12.9 11.1 11.7.
  const int nv = a.in.V / E::N;
  if (nv <= kWaveVectors) return pick(std::integral_constant<int, 64>{});
  if (nv <= 2048 && a.in.rows >= 1024) return pick(std::integral_constant<int, 128>{});
  if (nv <= 1024 || (nv <= 8192 && a.in.rows > 256)) return pick(std::integral_constant<int, 256>{});
  return pick(std::integral_constant<int, 512>{});
}

// Logits that with their gradient do not fit in the last cache (256 MB) are not kept there either: 8192 x 32001 bf16 192 -> 188 us,
// fp32 379 -> 368; 1024 x 32001 bf16, which fits, 21.6 us against 25.2.  The gradient goes past the caches in any case (there 29 -> 22 us).
constexpr int64_t kStreamBytes = 256ll << 20;
template <typename E>
int backward(const LogprobGradArgs& a, hipStream_t stream) {
  const int64_t nv = a.in.V / E::N;
  const bool large = 2 * static_cast<int64_t>(a.in.rows) * a.in.V * static_cast<int64_t>(sizeof(typename E::type)) > kStreamBytes;
  const int parts = nv <= 64 * kUnroll ? 1 : static_cast<int>((nv + 256 * kUnroll - 1) / (256 * kUnroll));
  auto go = [&](auto kernel, int grid) { kernel<<<grid, 256, 0, stream>>>(a, parts); };
  if (nv <= 64 * kUnroll) {
    if (large) go(logprobs_backward_kernel<E, 64, true>, (a.in.rows + 3) / 4);
    else go(logprobs_backward_kernel<E, 64, false>, (a.in.rows + 3) / 4);
  } else {
    if (large) go(logprobs_backward_kernel<E, 256, true>, a.in.rows * parts);
    else go(logprobs_backward_kernel<E, 256, false>, a.in.rows * parts);
  }
  return hipGetLastError() == hipSuccess ? PB_OK : PB_EHIP;
}

}  // namespace
}  // namespace lr

int64_t token_logprobs_workspace(int dtype, int32_t rows, int32_t V) {
  return static_cast<int64_t>(rows) * split_logprobs(V / (dtype == PB_F32 ? lr::F32::N : lr::F16::N), rows, V).parts * static_cast<int64_t>(sizeof(lr::PartRecord));
}
int launch_token_logprobs(int dtype, const LogprobArgs& a, void* workspace, hipStream_t stream) {
  return dtype == PB_F32   ? lr::forward<lr::F32>(a, workspace, stream)
         : dtype == PB_F16 ? lr::forward<lr::F16>(a, workspace, stream)
                           : lr::forward<lr::BF16>(a, workspace, stream);
}
int launch_token_logprobs_backward(int dtype, const LogprobGradArgs& a, hipStream_t stream) {
  return dtype == PB_F32 ? lr::backward<lr::F32>(a, stream) : dtype == PB_F16 ? lr::backward<lr::F16>(a, stream) : lr::backward<lr::BF16>(a, stream);
}

}  // namespace pb
