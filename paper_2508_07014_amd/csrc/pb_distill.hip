// pb_distill_topk (gfx950): the loss and the gradient of a row in one go, the row held in registers between the two.
#include <hip/hip_runtime.h>

#include "pb_kernels.hpp"
#include "pb_logit_rows.hpp"

namespace pb {
namespace lr {
namespace {

// Sums of exponentials: every term is e = exp2(d), d = x c - rc with c = log2(e) / T and the reference rc = m c, m the largest
// element that the lane has seen (a reference below the maximum would add its distance to the rounding of d).  d is rounded
// once; what rc itself was rounded by is the same for all terms of the lane and is made up for at the end (wave_part).
// Elements below -far (see kFar) are masks of a lowest value: nothing beside any ordinary logit.  With LISTED a second sum, X,
// takes the terms of listed tokens, which S then lacks.
// (S, X) seen from a reference that lies `apart` = rc - new rc higher:
template <bool LISTED>
__device__ __forceinline__ void rebase(float& S, float& X, float apart) {
  const float f = exp2_fast(apart);  // (may be infinite where the sums are 0)
  if constexpr (LISTED) X = X == 0.0f ? 0.0f : f * X;
  S = S == 0.0f ? 0.0f : f * S;
}
struct Sums {
  float rc = 0.0f, thr, S = 0.0f, X = 0.0f, m = -INFINITY;
  __device__ __forceinline__ explicit Sums(float far) : thr(-far) {}
};
// Moves the reference to `m`, the largest of the elements that are about to be added, if they exceed it.
template <bool LISTED>
__device__ __forceinline__ void look_at(Sums& s, float m, float c) {
  s.m = fmaxf(s.m, m);
  if (__ballot(m > s.thr) != 0) {  // (of the wave: a branch, not selects)
    if (m > s.thr) {
      const float next = m * c;
      rebase<LISTED>(s.S, s.X, s.rc - next);
      s.rc = next;
      s.thr = m;
    }
  }
}
template <bool LISTED, int N>
__device__ __forceinline__ void add_vector(Sums& s, const float (&x)[N], float c, unsigned listed) {  // (a bit per element)
  float e[N];
#pragma unroll
  for (int i = 0; i < N; ++i) e[i] = exp2_fast(__builtin_fmaf(x[i], c, -s.rc));
  if (LISTED && listed != 0u) {
    float on[N];
#pragma unroll
    for (int i = 0; i < N; ++i) {
      on[i] = (listed >> i) & 1u ? e[i] : 0.0f;
      e[i] = (listed >> i) & 1u ? 0.0f : e[i];
    }
    s.X += vec_sum(on);
  }
  s.S += vec_sum(e);
}

// Sums of a part of a row, seen from its maximum: d = (x - m) c.  Where less than an eighth of the maximum's term lies beside it,
// the sums lack that term, so that the rest is not rounded to its unit: `one` says where it belongs, 1: S, 2: X (0: nothing
// lacks).  A part of nothing but -inf has sums of 0.
struct Part {
  float m, S, X;
  int one;
};
__device__ __forceinline__ Part whole(const Part& p) { return Part{p.m, p.one == 1 ? p.S + 1.0f : p.S, p.one == 2 ? p.X + 1.0f : p.X, 0}; }
// The part of a wave from its lanes', the same in every lane.  again(add) goes over the wave's elements a second time, with
// add(x, listed): where the maximum lies so far from 0 that x c and m c no longer resolve what is between them, the
// difference does.  lane_again(tid, add) goes over the elements of one lane, by the whole wave.
template <bool LISTED, typename Again, typename LaneAgain>
__device__ __forceinline__ Part wave_part(const Sums& s, float c, Again&& again, LaneAgain&& lane_again) {
  Part p{wave_max(s.m), s.S, s.X, 0};
  const float mc = p.m * c;
  rebase<LISTED>(p.S, p.X, s.rc - mc);
  const Part own = p;
  p.S = wave_sum(p.S);
  if constexpr (LISTED) p.X = wave_sum(p.X);
  const float back = -__builtin_fmaf(p.m, c, -mc);  // (from the rounded m c to m c)
  rebase<LISTED>(p.S, p.X, back);
  float S = 0.0f, X = 0.0f;
  if (fabsf(mc) <= kFar) {
    if (p.S + p.X < 1.125f) {
      const int first = wv::first_lane(__ballot(s.m == p.m));
      bool on_max = false;
      lane_again(first, [&](float x, bool on) {
        const float e = x == p.m ? 0.0f : exp2_fast((x - p.m) * c);
        on_max = on_max || (x == p.m && on);
        S += LISTED && on ? 0.0f : e;
        if constexpr (LISTED) X += on ? e : 0.0f;
      });
      Part rest = own;  // (of the other lanes)
      rebase<LISTED>(rest.S, rest.X, back);
      const bool other = static_cast<int>(threadIdx.x & 63) != first;
      p.S = wave_sum(S + (other ? rest.S : 0.0f));
      if constexpr (LISTED) p.X = wave_sum(X + (other ? rest.X : 0.0f));
      p.one = LISTED && __ballot(on_max) != 0 ? 2 : 1;
    }
  } else if (fabsf(p.m) != INFINITY) {
    again([&](float x, bool on) {
      const float d = (x - p.m) * c, e = exp2_fast(d);
      S += LISTED && on ? 0.0f : e;
      if constexpr (LISTED) X += on ? e : 0.0f;
    });
    p.S = wave_sum(S);
    if constexpr (LISTED) p.X = wave_sum(X);
  }
  return p;
}
// Parts seen from the larger of their maxima keep their 1 apart, the others take it along.
template <bool LISTED>
__device__ __forceinline__ Part see_from(Part p, float m, float c) {
  if (p.m == m) return p;
  p = whole(p);
  rebase<LISTED>(p.S, p.X, (p.m - m) * c);
  p.m = m;
  return p;
}
// Two parts, or the parts that the lanes of a wave hold, as one (two that have the same maximum: the second's 1 joins the sums).
template <bool LISTED>
__device__ __forceinline__ Part join(const Part& p, const Part& q, float c) {
  const float m = fmaxf(p.m, q.m);
  const Part a = see_from<LISTED>(p, m, c);
  Part b = see_from<LISTED>(q, m, c);
  if (a.one != 0) b = whole(b);
  return Part{m, a.S + b.S, a.X + b.X, a.one | b.one};
}
template <bool LISTED>
__device__ __forceinline__ Part join_lanes(const Part& p, float c) {
  Part q = see_from<LISTED>(p, wave_max(p.m), c);
  const u64 ones = __ballot(q.one != 0);
  const int first = wv::first_lane(ones | (1ull << 63)), one = __builtin_amdgcn_readlane(q.one, first);
  if (static_cast<int>(threadIdx.x & 63) != first) q = whole(q);
  return Part{q.m, wave_sum(q.S), LISTED ? wave_sum(q.X) : 0.0f, one};
}

struct RowSums {  // the same in every thread of the row
  float m;        // maximum, -inf for a row of nothing but -inf, NaN for a marked one
  float base;     // m, 0 for such a row
  double S, all;  // the sum without the listed tokens, and the whole one, d = (x - base) c; 1 + a little, if so, in 64 bits
  bool bad;       // the row holds a NaN or +inf
};
// The row from its waves' parts (`lds`: NT / 64 of them).
template <int NT, bool LISTED>
__device__ __forceinline__ RowSums join_waves(Part p, int tid, float c, Part* lds) {
  constexpr int W = NT / 64;
  if constexpr (W > 1) {
    if ((tid & 63) == 0) lds[tid >> 6] = p;
    __syncthreads();
    p = lds[0];
    float M = p.m;
#pragma unroll
    for (int w = 1; w < W; ++w) M = fmaxf(M, lds[w].m);
    p = see_from<LISTED>(p, M, c);
#pragma unroll
    for (int w = 1; w < W; ++w) {
      Part q = see_from<LISTED>(lds[w], M, c);
      if (p.one != 0) q = whole(q);
      p = Part{M, p.S + q.S, p.X + q.X, p.one | q.one};
    }
    p = Part{uniform_f(p.m), uniform_f(p.S), uniform_f(p.X), uniform_i(p.one)};
  }
  RowSums r;
  r.S = (p.one == 1 ? 1.0 : 0.0) + p.S;
  r.all = (p.one != 0 ? 1.0 : 0.0) + (static_cast<double>(p.S) + p.X);
  r.bad = r.all != r.all || p.m == INFINITY;
  r.m = r.bad ? NAN : p.m;  // (a row of NaN and -inf has -inf for its largest number, and is no row of nothing but -inf)
  r.base = r.m == -INFINITY ? 0.0f : r.m;
  return r;
}

template <int CTRL>
__device__ __forceinline__ double dpp_add(double v) {
  const long long b = __double_as_longlong(v);
  const unsigned lo = static_cast<unsigned>(__builtin_amdgcn_update_dpp(0, static_cast<int>(b), CTRL, 0xf, 0xf, true));
  const unsigned hi = static_cast<unsigned>(__builtin_amdgcn_update_dpp(0, static_cast<int>(b >> 32), CTRL, 0xf, 0xf, true));
  return v + __longlong_as_double((static_cast<long long>(hi) << 32) | lo);
}
__device__ __forceinline__ double wave_sum(double v) {
  v = dpp_add<0x111>(v);
  v = dpp_add<0x112>(v);
  v = dpp_add<0x114>(v);
  v = dpp_add<0x118>(v);
  v = dpp_add<0x142>(v);
  v = dpp_add<0x143>(v);
  const long long b = __double_as_longlong(v);
  const unsigned lo = __builtin_amdgcn_readlane(static_cast<int>(b), 63), hi = __builtin_amdgcn_readlane(static_cast<int>(b >> 32), 63);
  return __longlong_as_double((static_cast<long long>(hi) << 32) | lo);
}

// 1 / v and log(v), v a positive number, to 1e-14: v = 2^k m, m in [sqrt(1/2), sqrt(2)), log m = 2 atanh(t), t = (m - 1) / (m + 1), by
// its series up to t^15 (the library's takes three times the instructions for the last bits).
__device__ __forceinline__ double over_64(double v) {
  double r = __builtin_amdgcn_rcp(v);
  r = __builtin_fma(r, __builtin_fma(-v, r, 1.0), r);
  return __builtin_fma(r, __builtin_fma(-v, r, 1.0), r);
}
__device__ __forceinline__ double log_64(double v) {
  const int k = (static_cast<int>(__double_as_longlong(v) >> 32) - 0x3fe6a09e) >> 20;
  const double m = ldexp(v, -k);
  const double t = (m - 1.0) * over_64(m + 1.0), t2 = t * t;
  double s = 1.0 / 15.0;
  s = __builtin_fma(s, t2, 1.0 / 13.0);
  s = __builtin_fma(s, t2, 1.0 / 11.0);
  s = __builtin_fma(s, t2, 1.0 / 9.0);
  s = __builtin_fma(s, t2, 1.0 / 7.0);
  s = __builtin_fma(s, t2, 1.0 / 5.0);
  s = __builtin_fma(s, t2, 1.0 / 3.0);
  s = __builtin_fma(s, t2, 1.0);
  return __builtin_fma(static_cast<double>(k), 0.69314718055994530942, 2.0 * t * s);
}

// The teacher's list of a row, an entry a lane.
// (Probabilities of the list and the student's on it in 64 bits: losses and gradients are small differences of them, and fp32 would
// leave 6e-8 of a probability, as much as 1e-4 of a gradient.)
struct Entry {
  int token;    // -1: absent
  float x;      // the student's logit
  double log_q, q;
};
struct List {   // the same in every lane
  double rest;  // what the entries leave of 1
  double shift; // log q = l - shift
  double Q;     // sum of q and rest
  int any;      // there is something to learn from
};
__device__ __forceinline__ double mass_from(double log_q) { return log_q == INFINITY ? NAN : exp(log_q); }  // (+inf: marked)
template <typename E, bool TAIL>
__device__ __forceinline__ List load_list(const DistillArgs& a, int64_t r, const Row<E>& row, int lane, Entry& e) {
  e = Entry{-1, 0.0f, -INFINITY, 0.0};
  if (lane < a.K) {
    const int t = a.tokens[r * a.K + lane];
    const float value = a.logp[r * a.K + lane];
    if (static_cast<unsigned>(t) < static_cast<unsigned>(row.V)) {
      e.token = t;
      e.x = E::up(row.x[t]);
      e.log_q = value;
    }
  }
  List l;
  if constexpr (TAIL) {
    e.q = mass_from(e.log_q);
    const double sum = wave_sum(e.q), left = 1.0 - sum;
    l.rest = left < 0x1p-20 ? 0.0 : left;  // (NaN stays)
    l.any = __ballot(e.token >= 0) != 0 ? 1 : 0;
    l.Q = l.rest > 0.0 ? 1.0 : sum;  // (NaN stays)
    l.shift = 0.0;
  } else {
    const float top = wave_max(static_cast<float>(e.log_q));
    l.any = __ballot(e.token >= 0 && e.log_q != -INFINITY) != 0 ? 1 : 0;
    const double part = e.token >= 0 ? exp(e.log_q - (l.any ? top : 0.0f)) : 0.0, sum = wave_sum(part);
    l.rest = 0.0;
    l.shift = top + log_64(sum);
    l.Q = sum == sum ? 1.0 : NAN;
    e.log_q -= l.shift;
    e.q = part * over_64(sum);
  }
  return l;
}

struct Student {
  float S;       // sum over all tokens
  double p_rest; // what the student leaves to the tokens that are not listed
  float A, lift; // their gradient is A exp2((x - base) c + lift)
};
template <bool TAIL>
__device__ __forceinline__ Student student(const RowSums& sums, const List& list, float w, float inv) {
  Student s{static_cast<float>(sums.all), 0.0, 0.0f, 0.0f};
  double share = list.Q;
  if constexpr (TAIL) {
    s.p_rest = sums.m == -INFINITY ? 0.0 : sums.S * over_64(sums.all);
    if (s.p_rest < 0x1p-126) s.p_rest = 0.0;  // (NaN stays)
    // (q' / p' may pass the fp32 range together with a row's weight, q' p_j / p' does not: the power of 2 goes into p_j)
    if (list.rest > 0.0 && s.p_rest > 0.0) {
      const int k = 1023 - static_cast<int>(__double_as_longlong(s.p_rest) >> 52);
      s.lift = static_cast<float>(k);
      share = ldexp(share, -k) - list.rest * over_64(ldexp(s.p_rest, k));
    }
  }
  s.A = static_cast<float>(share) * w * inv / s.S;
  return s;
}
// Sum of q over the entries of the lane's token (it may be listed more than once).  By one wave; `table`, kHashBits bits of
// LDS, finds the few tokens that can be the same as another (in lists of 64 different ones every fifth has such a pair):
// 64 comparisons of every lane took 3.2 us.
constexpr int kHashBits = 8192;
__device__ __forceinline__ double mass_of(const Entry& e, unsigned* table) {
  const v4u none = {0u, 0u, 0u, 0u};
#pragma unroll
  for (int i = 0; i < kHashBits / 128; i += 64) reinterpret_cast<v4u*>(table)[i + (threadIdx.x & 63)] = none;
  row_sync<64>();
  unsigned seen = 0u;
  if (e.token >= 0) {
    const unsigned h = static_cast<unsigned>(e.token) * 2654435761u >> 19;
    seen = atomicOr(&table[h >> 5], 1u << (h & 31)) >> (h & 31) & 1u;
  }
  double mass = e.q;
  for (u64 left = __ballot(seen != 0u); left != 0;) {
    const int token = __builtin_amdgcn_readlane(e.token, wv::first_lane(left));
    const u64 same = __ballot(e.token == token);
    if (__builtin_popcountll(same) > 1) {
      const double sum = wave_sum(e.token == token ? e.q : 0.0);
      mass = e.token == token ? sum : mass;
    }
    left &= ~same;
  }
  return mass;
}
// By one wave: the row's loss.  Terms that cancel, and log-probs of masked tokens that may pass the fp32 range: in 64 bits.
template <bool TAIL>
__device__ __forceinline__ void write_loss(const DistillArgs& a, int64_t r, int lane, const Entry& e, const List& list, const RowSums& sums,
                                           const Student& st, float inv) {
  const double lp = (static_cast<double>(e.x) - sums.base) * inv - (sums.m == -INFINITY ? 0.0 : log_64(sums.all));
  double loss = wave_sum(e.q > 0.0 ? e.q * (e.log_q - lp) : e.q);  // (0, or NaN)
  if (TAIL && list.rest != 0.0) loss += st.p_rest == 0.0 ? INFINITY : list.rest * (log_64(list.rest) - log_64(st.p_rest));
  if (lane == 0) a.loss[r] = sums.bad ? NAN : static_cast<float>(loss);
}
// The gradient on a listed token: the difference of two probabilities, of which one may be near 1, in 64 bits.
__device__ __forceinline__ float listed_grad(float x, double mass, const List& list, const RowSums& sums, float c, float w, float inv) {
  const double p = exp2_fast((x - sums.base) * c) * over_64(sums.all);
  return static_cast<float>(p * list.Q - mass) * w * inv;
}

// Has the compiler unpack held vectors again, rather than keep them unpacked in twice the registers.
template <int HELD>
__device__ __forceinline__ void reload(v4u (&held)[HELD]) {
#pragma unroll
  for (int u = 0; u < HELD; ++u) asm volatile("" : "+v"(held[u]));
}

// One row, by a wave (four rows a workgroup) or a workgroup.  Thread t holds vectors t, t + NT, ... of the row, HELD of them
// in registers; what a row has beyond HELD * NT vectors is read a second time for the gradient (from cache: only the rows
// at work are in between).  With TAIL the tokens that are not listed have a sum of their own, so that little mass does not
// vanish in a difference: bits in LDS say which elements are listed, and most vectors have none.  Bound by HBM where rows are
// long (8192 x 32001 bf16, 32 entries: 192 us, 5.5 TB/s), by the 600 instructions a row needs anyway where they are short (13686 x
// 129 bf16: 15.4 us with 4 entries, 16.8 with 64), by latency where they are few (500 x 1025 fp32: 4.4 us).
template <typename E, int NT, int HELD, bool TAIL, bool STREAM>
__global__ __launch_bounds__(NT == 64 ? 256 : NT) void distill_kernel(DistillArgs a, int mark_bytes) {
  constexpr int ROWS = NT == 64 ? 4 : 1;
  extern __shared__ __align__(16) unsigned char s_all[];
  __shared__ Part s_sums[ROWS][NT / 64];
  __shared__ List s_list;
  __shared__ u64 s_edge[ROWS];
  __shared__ __align__(16) unsigned s_table[ROWS][kHashBits / 32];
  const int sub = NT == 64 ? uniform_i(threadIdx.x >> 6) : 0, tid = NT == 64 ? threadIdx.x & 63 : threadIdx.x;
  const int64_t r = static_cast<int64_t>(blockIdx.x) * ROWS + sub;
  if (ROWS > 1 && r >= a.in.rows) return;
  const Row<E> row = row_at<E, NT == 64 ? 16 : 64>(a.in.x, a.in.stride, r, a.in.V);
  unsigned char* marks = s_all + sub * mark_bytes;
  v4u held[HELD];  // (behind the row's end: its last vector again; loads under conditions took 230 registers instead of 50)
  if (row.nv > 0) {
#pragma unroll
    for (int u = 0; u < HELD; ++u) held[u] = row.template vec_once<STREAM>(min(u * NT + tid, row.nv - 1));
  }
  float edge = -INFINITY;
  if (tid < row.edges) edge = E::up(row.x[row.edge_token(tid)]);
  const float w = a.row_grads ? a.row_grads[r] : 1.0f, inv = a.in.inv_temp, c = a.in.c;
  const bool lister = NT == 64 || tid < 64;
  if constexpr (TAIL) {
    for (int i = tid; i < mark_bytes / 4; i += NT) reinterpret_cast<unsigned*>(marks)[i] = 0u;
    if (tid == 0) s_edge[sub] = 0;
  }
  Entry e{-1, 0.0f, 0.0, 0.0};
  List list{0.0, 0.0, 0.0, 0};
  double mass = 0.0;
  if (lister) {
    list = load_list<E, TAIL>(a, r, row, tid & 63, e);
    if (a.grad) mass = mass_of(e, s_table[sub]);
  }
  if constexpr (NT > 64) {
    if (tid == 0) s_list = list;
  }
  if constexpr (TAIL || NT > 64) row_sync<NT>();
  if constexpr (NT > 64) list = s_list;
  if constexpr (TAIL) {
    if (lister && e.token >= 0) {
      const int at = e.token - row.head, v = at / E::N;
      if (at < 0 || v >= row.nv) {
        atomicOr(&s_edge[sub], 1ull << (at < 0 ? e.token : e.token - row.nv * E::N));
      } else {
        atomicOr(&reinterpret_cast<unsigned*>(marks)[at >> 5], 1u << (at & 31));
      }
    }
    row_sync<NT>();
  }
  typename E::type* out = a.grad ? static_cast<typename E::type*>(a.grad) + r * a.grad_stride : nullptr;
  auto zeros = [&] {
    const v4u z = {0u, 0u, 0u, 0u};
    for (int v = tid; v < row.nv; v += NT) store_vector<E>(out + row.token(v, 0), z);
    if (tid < row.edges) out[row.edge_token(tid)] = E::down(0.0f);
  };
  if (!uniform_i(list.any)) {
    if (a.loss && tid == 0) a.loss[r] = 0.0f;
    if (out) zeros();
    return;
  }
  Sums s(a.in.far);
  auto listed = [&](int v) -> unsigned { return !TAIL ? 0u : E::N == 8 ? marks[v] : (marks[v >> 1] >> (4 * (v & 1))) & 15u; };
  auto edge_listed = [&](int t) -> bool { return TAIL && ((s_edge[sub] >> t) & 1u); };
  float most = edge;
#pragma unroll
  for (int u = 0; u < HELD; ++u)
    if (u * NT + tid < row.nv) {
      float x[E::N];
      E::unpack(held[u], x);
      most = fmaxf(most, vec_max(x));
    }
  look_at<TAIL>(s, most, c);
  reload(held);
#pragma unroll
  for (int u = 0; u < HELD; ++u)
    if (u * NT + tid < row.nv) {
      float x[E::N];
      E::unpack(held[u], x);
      add_vector<TAIL>(s, x, c, listed(u * NT + tid));
    }
  if (tid < row.edges) {
    const float x[1] = {edge};
    add_vector<TAIL>(s, x, c, edge_listed(tid) ? 1u : 0u);
  }
  for (int v = HELD * NT + tid; v < row.nv; v += NT) {
    float x[E::N];
    E::unpack(row.vec(v), x);
    look_at<TAIL>(s, vec_max(x), c);
    add_vector<TAIL>(s, x, c, listed(v));
  }
  const Part part = wave_part<TAIL>(s, c, [&](auto&& add) {
    for (int v = tid; v < row.nv; v += NT) {
      float x[E::N];
      E::unpack(row.vec(v), x);
      const unsigned on = listed(v);
#pragma unroll
      for (int i = 0; i < E::N; ++i) add(x[i], (on >> i) & 1u);
    }
    if (tid < row.edges) add(edge, edge_listed(tid));
  }, [&](int lane, auto&& add) {
    const int me = tid & 63, one = (tid & ~63) + lane;
    for (int k = me; k < (row.nv - one + NT - 1) / NT * E::N; k += 64) {
      const int v = one + k / E::N * NT, i = k % E::N;
      add(E::up(row.x[row.token(v, i)]), (listed(v) >> i) & 1u);
    }
    if (me == lane && tid < row.edges) add(edge, edge_listed(tid));
  });
  const RowSums sums = join_waves<NT, TAIL>(part, tid, c, s_sums[sub]);
  const bool empty = sums.m == -INFINITY;
  const Student st = student<TAIL>(sums, list, w, inv);
  if (lister && a.loss) write_loss<TAIL>(a, r, tid, e, list, sums, st, inv);
  if (!out) return;
  if (empty || w == 0.0f) {
    if constexpr (NT > 64) __syncthreads();  // (the gradient may take the logits' place: all of them have been read)
    zeros();
    return;
  }
  auto grad = [&](float x) { return exp2_fast(__builtin_fmaf(x - sums.base, c, st.lift)) * st.A; };
  auto put = [&](const v4u& raw, int v) {
    float x[E::N];
    E::unpack(raw, x);
#pragma unroll
    for (int i = 0; i < E::N; ++i) x[i] = grad(x[i]);
    if constexpr (NT > 64 && E::N == 8) stream_vector<E>(out + row.token(v, 0), E::pack(x));
    else store_vector<E>(out + row.token(v, 0), E::pack(x));
  };
  if constexpr (NT > 64) __syncthreads();
  reload(held);
#pragma unroll
  for (int u = 0; u < HELD; ++u)
    if (u * NT + tid < row.nv) put(held[u], u * NT + tid);
  for (int v = HELD * NT + tid; v < row.nv; v += NT) put(row.vec(v), v);
  if (tid < row.edges) out[row.edge_token(tid)] = E::down(grad(edge));
  const float own = lister ? listed_grad(e.x, mass, list, sums, c, w, inv) : 0.0f;
  row_sync<NT>();
  if (lister && e.token >= 0) out[e.token] = E::down(own);
}

constexpr int kGradUnroll = 4;

// Few long rows, and rows too long for the registers of a workgroup: every wave takes 64 * `each` vectors of a row and
// leaves their part of the sums in the workspace, and one more wave the list's (with the student's logits on it, since the
// gradient may take the logits' place); the second kernel joins the parts and writes the gradient.  64 x 131072 bf16, 64 entries:
// 7.3 us, the list's wave being the last to end, and 8.0 us.
struct DistillSpace {
  float4* parts;  // [rows, parts]
  List* lists;    // [rows]
  double* mass;   // [rows, 64]
  float* x;       // [rows, 64]
};
template <typename E, bool TAIL>
__global__ __launch_bounds__(256) void distill_parts_kernel(DistillArgs a, int parts, int each, DistillSpace ws) {
  __shared__ unsigned s_marks[4][64 * kMaxEach / 4];  // a byte per vector
  __shared__ u64 s_edge[4];
  __shared__ __align__(16) unsigned s_table[kHashBits / 32];  // (of the one list wave that a workgroup has at most)
  const int sub = uniform_i(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int64_t at = static_cast<int64_t>(blockIdx.x) * 4 + sub;
  const int64_t r = at / (parts + 1);
  if (r >= a.in.rows) return;
  const int part = static_cast<int>(at - r * (parts + 1)) - 1, begin = part * 64 * each;  // (-1: the list, the longest way)
  const Row<E> row = row_at<E>(a.in.x, a.in.stride, r, a.in.V);
  const float c = a.in.c;
  const int end = min(begin + 64 * each, row.nv);
  if (part < 0) {
    Entry e;
    const List l = load_list<E, TAIL>(a, r, row, lane, e);
    if (lane == 0) ws.lists[r] = l;
    ws.x[r * 64 + lane] = e.x;
    ws.mass[r * 64 + lane] = mass_of(e, s_table);
    return;
  }
  v4u raw[kGradUnroll];  // (requested before the list)
  auto load = [&](int v0) {
#pragma unroll
    for (int u = 0; u < kGradUnroll; ++u) raw[u] = row.vec(min(v0 + 64 * u, row.nv - 1));
  };
  load(begin + lane);
  if constexpr (TAIL) {
    if (lane < 16 * each) s_marks[sub][lane] = 0u;
    if (16 * each > 64 && lane < 16 * each - 64) s_marks[sub][64 + lane] = 0u;
    if (lane == 0) s_edge[sub] = 0;
    row_sync<64>();
    if (lane < a.K) {
      const int t = a.tokens[r * a.K + lane], e = t - row.head, v = e / E::N;
      if (static_cast<unsigned>(t) < static_cast<unsigned>(a.in.V)) {
        if (e < 0 || v >= row.nv)
          atomicOr(&s_edge[sub], 1ull << (e < 0 ? t : t - row.nv * E::N));
        else if (v >= begin && v < end)
          atomicOr(&s_marks[sub][(v - begin) >> 2], 1u << (8 * ((v - begin) & 3) + e % E::N));
      }
    }
    row_sync<64>();
  }
  auto listed = [&](int v) -> unsigned { return TAIL ? reinterpret_cast<const unsigned char*>(s_marks[sub])[v - begin] : 0u; };
  Sums s(a.in.far);
  for (int v0 = begin + lane; v0 < end; v0 += 64 * kGradUnroll) {
    if (v0 > begin + lane) load(v0);
#pragma unroll
    for (int u = 0; u < kGradUnroll; ++u)
      if (v0 + 64 * u < end) {
        float x[E::N];
        E::unpack(raw[u], x);
        look_at<TAIL>(s, vec_max(x), c);
        add_vector<TAIL>(s, x, c, listed(v0 + 64 * u));
      }
  }
  const bool has_edge = begin == 0 && lane < row.edges;
  const bool on_edge = TAIL && has_edge && ((s_edge[sub] >> lane) & 1u);
  float edge = -INFINITY;
  if (has_edge) {
    edge = E::up(row.x[row.edge_token(lane)]);
    const float x[1] = {edge};
    look_at<TAIL>(s, edge, c);
    add_vector<TAIL>(s, x, c, on_edge ? 1u : 0u);
  }
  const Part p = wave_part<TAIL>(s, c, [&](auto&& add) {
    for (int v = begin + lane; v < end; v += 64) {
      float x[E::N];
      E::unpack(row.vec(v), x);
      const unsigned on = listed(v);
#pragma unroll
      for (int i = 0; i < E::N; ++i) add(x[i], (on >> i) & 1u);
    }
    if (has_edge) add(edge, on_edge);
  }, [&](int one, auto&& add) {
    for (int k = lane; k < (end - begin - one + 63) / 64 * E::N; k += 64) {
      const int v = begin + one + k / E::N * 64, i = k % E::N;
      add(E::up(row.x[row.token(v, i)]), (listed(v) >> i) & 1u);
    }
    if (lane == one && has_edge) add(edge, on_edge);
  });
  if (lane == 0) ws.parts[r * parts + part] = make_float4(p.m, p.S, p.X, static_cast<float>(p.one));
}

template <typename E, bool TAIL>
__global__ __launch_bounds__(256) void distill_grad_kernel(DistillArgs a, int parts, int blocks, DistillSpace ws) {
  constexpr int BLOCK = 256 * kGradUnroll;
  const int64_t r = blockIdx.x / blocks;
  const int block = blockIdx.x % blocks, tid = threadIdx.x, lane = tid & 63;
  const Row<E> row = row_at<E>(a.in.x, a.in.stride, r, a.in.V);
  typename E::type* out = a.grad ? static_cast<typename E::type*>(a.grad) + r * a.grad_stride : nullptr;
  v4u raw[kGradUnroll];
  if (out) {  // (a row behind its end: its last vector again)
#pragma unroll
    for (int u = 0; u < kGradUnroll; ++u) raw[u] = row.vec(min(block * BLOCK + u * 256 + tid, row.nv - 1));
  }
  const bool has_edge = block == 0 && tid < row.edges;
  float edge = 0.0f;
  if (has_edge) edge = E::up(row.x[row.edge_token(tid)]);
  const float w = a.row_grads ? a.row_grads[r] : 1.0f, inv = a.in.inv_temp, c = a.in.c;
  const List list = ws.lists[r];
  Part p{-INFINITY, 0.0f, 0.0f, 0};
#pragma unroll
  for (int i = 0; i < kMaxParts / 64; ++i)
    if (64 * i + lane < parts) {
      const float4 q = ws.parts[r * parts + 64 * i + lane];
      p = join<TAIL>(p, Part{q.x, q.y, q.z, static_cast<int>(q.w)}, c);
    }
  const RowSums sums = join_waves<64, TAIL>(join_lanes<TAIL>(p, c), lane, c, nullptr);
  const Student st = student<TAIL>(sums, list, w, inv);
  const bool learn = list.any != 0, none = !learn || sums.m == -INFINITY || w == 0.0f;
  Entry e{-1, 0.0f, -INFINITY, 0.0};
  double mass = 0.0;
  bool mine = false;  // the lane's listed token lies in this block, whose first wave writes it after the other stores
  if (tid < 64) {
    if (learn && tid < a.K) {
      const int t = a.tokens[r * a.K + tid];
      if (static_cast<unsigned>(t) < static_cast<unsigned>(a.in.V)) {
        e.token = t;
        e.x = ws.x[r * 64 + tid];
        mass = ws.mass[r * 64 + tid];
        e.log_q = a.logp[r * a.K + tid] - list.shift;
        if (block == 0) e.q = mass_from(e.log_q);
        mine = block == (t < row.head || t >= row.head + row.nv * E::N ? 0 : (t - row.head) / E::N / BLOCK);
      }
    }
  }
  auto grad = [&](float x) { return exp2_fast(__builtin_fmaf(x - sums.base, c, st.lift)) * st.A; };
  if (out) {
#pragma unroll
    for (int u = 0; u < kGradUnroll; ++u) {
      const int v = block * BLOCK + u * 256 + tid;
      if (v < row.nv) {
        float x[E::N];
        E::unpack(raw[u], x);
#pragma unroll
        for (int i = 0; i < E::N; ++i) x[i] = none ? 0.0f : grad(x[i]);
        stream_vector<E>(out + row.token(v, 0), E::pack(x));
      }
    }
    if (has_edge) out[row.edge_token(tid)] = E::down(none ? 0.0f : grad(edge));
  }
  if (block == 0 && tid < 64 && a.loss) {
    if (learn) write_loss<TAIL>(a, r, tid, e, list, sums, st, inv);
    else if (tid == 0) a.loss[r] = 0.0f;
  }
  if (!out) return;
  __syncthreads();
  if (mine && !none) out[e.token] = E::down(listed_grad(e.x, mass, list, sums, c, w, inv));
}

DistillSpace space_in(void* p, int32_t rows, int parts) {
  DistillSpace ws;
  ws.parts = static_cast<float4*>(p);
  ws.lists = reinterpret_cast<List*>(ws.parts + static_cast<int64_t>(rows) * parts);
  ws.mass = reinterpret_cast<double*>(ws.lists + rows);
  ws.x = reinterpret_cast<float*>(ws.mass + static_cast<int64_t>(rows) * 64);
  return ws;
}

template <typename E>
int distill_split(const DistillArgs& a, const RowSplit& split, void* workspace, hipStream_t stream) {
  const DistillSpace ws = space_in(workspace, a.in.rows, split.parts);
  const int grid = static_cast<int>((static_cast<int64_t>(a.in.rows) * (split.parts + 1) + 3) / 4);
  const int blocks = a.grad ? (a.in.V / E::N + 256 * kGradUnroll - 1) / (256 * kGradUnroll) : 1;
  auto go = [&](auto tail) {
    constexpr bool TAIL = decltype(tail)::value;
    distill_parts_kernel<E, TAIL><<<grid, 256, 0, stream>>>(a, split.parts, split.each, ws);
    if (hipGetLastError() != hipSuccess) return PB_EHIP;
    distill_grad_kernel<E, TAIL><<<a.in.rows * blocks, 256, 0, stream>>>(a, split.parts, blocks, ws);
    return hipGetLastError() == hipSuccess ? PB_OK : PB_EHIP;
  };
  return a.tail ? go(std::true_type{}) : go(std::false_type{});
}

template <typename E>
int distill(const DistillArgs& a, void* workspace, hipStream_t stream) {
  const RowSplit split = split_distill(a.in.V / E::N, a.in.all_rows);
  if (split.parts > 0) return distill_split<E>(a, split, workspace, stream);
  const int nv = a.in.V / E::N, mark_bytes = (a.in.V + 127) / 128 * 16;  // (a bit per element behind the head)
  // (logits of 16 bits that do not fit in the last cache with their gradient, in long rows, are not kept there either:
  // 8192 x 32001 195 -> 191 us, 16384 x 16000 201 -> 190; 32768 x 8193 207 against 213, 1024 x 32001, which fits, 28 against 30.
  // The gradient of such types goes past the caches (there 36 -> 28 us; fp32 8192 x 32000 397 us against 420).)
  const bool large = E::N == 8 && nv > 1024 && 4 * static_cast<int64_t>(a.in.rows) * a.in.V > (256ll << 20);
  auto go = [&](auto nt, auto held) {
    constexpr int NT = decltype(nt)::value, HELD = decltype(held)::value, ROWS = NT == 64 ? 4 : 1, THREADS = NT == 64 ? 256 : NT;
    constexpr bool CAN = E::N == 8 && NT * HELD > 1024 && NT < 1024;  // (too few rows for that)
    const int grid = (a.in.rows + ROWS - 1) / ROWS, lds = a.tail ? ROWS * mark_bytes : 0;
    auto launch = [&](auto kernel) { kernel<<<grid, THREADS, lds, stream>>>(a, a.tail ? mark_bytes : 0); };
    if (a.tail) {
      if (CAN && large) launch(distill_kernel<E, NT, HELD, true, CAN>);
      else launch(distill_kernel<E, NT, HELD, true, false>);
    } else {
      if (CAN && large) launch(distill_kernel<E, NT, HELD, false, CAN>);
      else launch(distill_kernel<E, NT, HELD, false, false>);
    }
    return hipGetLastError() == hipSuccess ? PB_OK : PB_EHIP;
  };
  using std::integral_constant;
  // Threads x vectors held, us at the best and its neighbours: 16384 x 300 bf16 64x4 20.4, 64x8 21.9; 500 x 1025 fp32 64x4 5.2, 64x8 5.8,
  // 16384 x 1025 fp32 37.2 35.4; 16384 x 4096 bf16 64x8 61, 64x16 59, 256x4 70; 16384 x 8192 256x4 103, 256x8 110, 64x16 114;
  // 16384 x 16000 256x8 188, 512x4 191, 512x8 206; 8192 x 32001 256x8 208, 512x8 191, 512x16 204; 4096 x 65000 512x8 216, 512x16 203,
  // 1024x8 259; 3000 x 32001 fp32 173 149 168.  Longer rows: 256 x 131072 bf16 512x16 38, 1024x8 34; 1000 x 90000 75 87.
  if (nv <= 128 || (nv <= 256 && a.in.rows < 4096)) return go(integral_constant<int, 64>{}, integral_constant<int, 4>{});
  if (nv <= 512) return go(integral_constant<int, 64>{}, integral_constant<int, 8>{});
  if (nv <= 1024) return go(integral_constant<int, 256>{}, integral_constant<int, 4>{});
  if (nv <= 2048) return go(integral_constant<int, 256>{}, integral_constant<int, 8>{});
  if (nv <= 4096) return go(integral_constant<int, 512>{}, integral_constant<int, 8>{});
  if (nv <= 8192 || a.in.rows > 256) return go(integral_constant<int, 512>{}, integral_constant<int, 16>{});
  return go(integral_constant<int, 1024>{}, integral_constant<int, 8>{});
}

}  // namespace
}  // namespace lr

int64_t distill_topk_workspace(int dtype, int32_t rows, int32_t V) {
  const RowSplit split = split_distill(V / (dtype == PB_F32 ? lr::F32::N : lr::F16::N), rows);
  if (split.parts == 0) return 0;
  return static_cast<int64_t>(rows) * (split.parts * static_cast<int64_t>(sizeof(float4)) + sizeof(lr::List) + 64 * (sizeof(double) + sizeof(float)));
}
int launch_distill_topk(int dtype, const DistillArgs& a, void* workspace, hipStream_t stream) {
  return dtype == PB_F32   ? lr::distill<lr::F32>(a, workspace, stream)
         : dtype == PB_F16 ? lr::distill<lr::F16>(a, workspace, stream)
                           : lr::distill<lr::BF16>(a, workspace, stream);
}

}  // namespace pb
