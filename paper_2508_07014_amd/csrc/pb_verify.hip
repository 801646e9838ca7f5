// Verification of drafted tokens (pb_verify_draft): which of them a target's rows accept, and the token drawn behind them.
//
//   p_i = softmax(x_i / T), q_i = softmax(y_i / T') (or 1 at t_i): t_i is accepted where those before it are and u_i q_i(t_i) < p_i(t_i);
//   behind the k accepted ones a token is drawn from max(p_k - q_k, 0), or from p_k where no drafted token was refused: the first
//   v whose sum over all tokens up to it exceeds w times the sum over all.
//
// A drawn token is a border between two of V sums: with sums in fp32, off by 1e-7 of the whole, one draw in a hundred from a
// row of 131072 tokens would be another token than the definition's.  So the row that decides is summed in 64 bits.  The other
// rows are only compared: their sums in fp32 decide wherever u q lies apart from p by more than those can be off, and where it
// does not the two rows are summed in 64 bits as well.
//
// Long rows take three launches: sums of all rows, a wave a part; then the decision and the deciding row's sums, several workgroups a
// sequence; then the draw.  max(p - q, 0) needs the ratio of the two rows' sums, which the second launch has in fp32 only:
// with it, it says which tokens lie above the line e_p = ratio e_q and sums both sides of those, so that the third can put
// the exact ratio in; tokens that lie too near to the line for the first ratio are summed apart, with how near they come.
#include <algorithm>

#include "pb_logit_rows.hpp"
#include "pb_student.hpp"

namespace pb {
namespace vd {

using namespace lr;
using wv::first_lane;

// Of a part of a row: the largest element m (-inf: nothing) and how many there are of it, the sum of e = 2^t, t = (x - m) c, over the others in fp32
// (NaN where the part holds a NaN or +inf; beside a near-certain token the others' weight is not lost in its 1); beside the
// first part, what the row has of the token drafted there.
struct Sums {
  float m, ones, s, at;
};
// How far a row's sum s is off at most, relative to itself: each exponent by three roundings (of the difference, of c, of the product),
// 3 ln 2 |t| 2^-24 of its term, its exponential by 2 x 2^-24, the sum by 13 additions one after the other at most (3 in a vector, 3 of vectors, the
// edge, 6 in a wave; parts are joined in 64 bits).  The mean of |t| = log2 (1 / e) over the row's probabilities e / s is at most the
// logarithm of the mean of 1 / e, which is V / s (s >= 1).
__device__ __forceinline__ double off_by(double s, int V) {
  return static_cast<double>((2.1f * __builtin_amdgcn_logf(static_cast<float>(V) / static_cast<float>(s)) + 17.0f) * 0x1p-24f);
}
constexpr double kBeside = 0x1p-34;      // products of two such bounds, and what the sums in 64 bits are off by
constexpr double kSmallBeside = 0x1p-20; // of a row's weight beside its largest element, apart from which it is kept below this
constexpr double kNothing = 0x1p-40;     // a rest of the target's mass below this is none (equal rows differ by their roundings)
// p - ratio q below this, relative to p, is none: the ratio of two sums in 64 bits, of at most 30 additions one after the other each, is off by up to
// 2^-47 of itself, and a token of p = q would be drawn for it.
constexpr double kEven = 0x1p-46;
constexpr double kNoWeight = 0x1p-960;   // weights below this, masked tokens' among them, are none

typedef VerifyArgs::Scale Scale;

// 2^((x - m) c) for x <= m, at least 2^-1000, off by 4e-14 of itself: with n the nearest integer to the exponent (in the low word of
// the sum with 1.5 2^52) and r what is left, 1 + r P(r), P by interpolation at Chebyshev's nodes, and n added to the exponent: 16
// instructions in 64 bits, 4 cycles each like those in fp32.  (With rounding, conversion and ldexp as instructions of their own it is 19;
// all rows of 128 x 17 of 131072 bf16 in these weights took 209 us and 190; in fp32 they take 89.)
__device__ __forceinline__ double weight(float x, float m, const Scale& k) {
  const double d = fmax(static_cast<double>(x) - static_cast<double>(m), k.low);
  const double s = fma(d, k.c, 0x1.8p52), r = fma(d, k.c, -(s - 0x1.8p52));
  double p = 0x1.b63880a30e9ffp-24;
  p = fma(p, r, 0x1.63d136366db24p-20);
  p = fma(p, r, 0x1.ffcb9515a8016p-17);
  p = fma(p, r, 0x1.4308ac85aa947p-13);
  p = fma(p, r, 0x1.5d87fe86fe88ep-10);
  p = fma(p, r, 0x1.3b2ab7181b755p-7);
  p = fma(p, r, 0x1.c6b08d7047e52p-5);
  p = fma(p, r, 0x1.ebfbdff823cedp-3);
  p = fma(p, r, 0x1.62e42fefa39efp-1);
  p = fma(p, r, 1.0);
  return __hiloint2double(__double2hiint(p) + (__double2loint(s) << 20), __double2loint(p));
}

__device__ __forceinline__ double readlane64(double v, int lane) {
  return __hiloint2double(__builtin_amdgcn_readlane(__double2hiint(v), lane), __builtin_amdgcn_readlane(__double2loint(v), lane));
}
// v plus what the lane has that CTRL names, in the rows of ROWS.
template <int CTRL, int ROWS>
__device__ __forceinline__ double dpp_add64(double v) {
  const int lo = __builtin_amdgcn_update_dpp(0, __double2loint(v), CTRL, ROWS, 0xf, ROWS == 0xf);
  const int hi = __builtin_amdgcn_update_dpp(0, __double2hiint(v), CTRL, ROWS, 0xf, ROWS == 0xf);
  return v + __hiloint2double(hi, lo);
}
// Sums over the lanes up to each, and over the wave.
__device__ __forceinline__ double wave_upto64(double v) {
  v = dpp_add64<0x111, 0xf>(v);
  v = dpp_add64<0x112, 0xf>(v);
  v = dpp_add64<0x114, 0xf>(v);
  v = dpp_add64<0x118, 0xf>(v);
  v = dpp_add64<0x142, 0xa>(v);
  return dpp_add64<0x143, 0xc>(v);
}
__device__ __forceinline__ double wave_sum64(double v) { return readlane64(wave_upto64(v), 63); }

// Part of a row, by a wave: vectors first .. first + 64 EACH - 1, and the row's edge where `edge`.
template <typename E, int EACH>
__device__ __forceinline__ Sums part_sums(const Row<E>& row, int first, bool edge, double c64, int lane) {
  v4u raw[EACH];
  float xe = -INFINITY;
#pragma unroll
  for (int u = 0; u < EACH; ++u) {
    const int v = first + 64 * u + lane;
    raw[u] = v < row.nv ? row.vec(v) : E::nothing();
  }
  if (edge && lane < row.edges) xe = E::up(row.x[row.edge_token(lane)]);
  float m = fmaxf(-INFINITY, xe), most[EACH];
#pragma unroll
  for (int u = 0; u < EACH; ++u) {
    float x[E::N];
    E::unpack(raw[u], x);
    most[u] = vec_max(x);
    m = fmaxf(m, most[u]);
  }
  m = wave_max(m);
  const float c = static_cast<float>(c64), from = m == -INFINITY ? 0.0f : m;
  float s[EACH];
  int ones = 0;
#pragma unroll
  for (int u = 0; u < EACH; ++u) {
    s[u] = 0.0f;
    if (first + 64 * u >= row.nv) continue;
    float x[E::N];
    E::unpack(raw[u], x);
#pragma unroll
    for (int i = 0; i < E::N; ++i) x[i] = exp2_fast((x[i] - from) * c);
    s[u] = vec_sum(x);
    if (__ballot(most[u] == from) == 0) continue;
    E::unpack(raw[u], x);  // (again, without the largest elements)
#pragma unroll
    for (int i = 0; i < E::N; ++i) {
      ones += __builtin_popcountll(__ballot(x[i] == from));
      x[i] = x[i] == from ? 0.0f : exp2_fast((x[i] - from) * c);
    }
    s[u] = vec_sum(x);
  }
  const float e = xe == from ? 0.0f : exp2_fast((xe - from) * c);
  ones += __builtin_popcountll(__ballot(xe == from));
  return Sums{m, static_cast<float>(ones), wave_sum(vec_sum(s) + e) + (from - from), 0.0f};  // (inf - inf: NaN)
}

// The rows of a sequence: 0 .. n the target's, n + 1 .. 2 n the draft's.
template <typename E>
__device__ __forceinline__ Row<E> row_of(const VerifyArgs& a, int64_t b, int j) {
  return j <= a.n ? row_at<E>(static_cast<const typename E::type*>(a.target) + b * a.target_seq, a.target_row, j, a.V)
                  : row_at<E>(static_cast<const typename E::type*>(a.draft) + b * a.draft_seq, a.draft_row, j - a.n - 1, a.V);
}
// The drafted tokens of a sequence, a lane each, and how many there are before the first that is absent.
struct Drafted {
  int t, count;
  float u;  // their numbers
};
__device__ __forceinline__ Drafted drafted_tokens(const VerifyArgs& a, int64_t b, int lane) {
  Drafted r;
  r.t = lane < a.n ? a.tokens[b * a.n + lane] : -1;
  r.u = lane < a.n ? a.numbers[b * (a.n + 1) + lane] : 0.0f;
  const u64 none = ~__ballot(static_cast<unsigned>(r.t) < static_cast<unsigned>(a.V));
  r.count = first_lane(none);  // (n <= 63: lane 63 holds none)
  r.u = fminf(fmaxf(r.u, 0.0f), 0x1.fffffep-1f);
  return r;
}
template <typename E>
__device__ __forceinline__ float target_at(const VerifyArgs& a, int64_t b, int i, int t) {
  return E::up((static_cast<const typename E::type*>(a.target) + b * a.target_seq + i * a.target_row)[t]);
}
template <typename E>
__device__ __forceinline__ float draft_at(const VerifyArgs& a, int64_t b, int i, int t) {
  return E::up((static_cast<const typename E::type*>(a.draft) + b * a.draft_seq + i * a.draft_row)[t]);
}

// A row is split in parts of 64 EACH vectors, a wave each; at least one.  Of 2048 elements (16-bit rows 4096 / 2048 / 1024 us: 32 x 9 of 32001 22.0 / 21.0 /
// 21.6, 64 x 9 of 50000 without rows of the draft 26.3 / 25.4 / 26.7, 128 x 17 of 131072 146 / 145 / 173; fp32 2048 / 1024: 8 x 9 of 131072 22.7 /
// 23.1); 64 kSmallEach vectors where one workgroup takes all of a sequence.
template <typename E>
constexpr int kEach = 32 / E::N;
constexpr int kSmallEach = 8;
template <typename E>
__host__ __device__ __forceinline__ int parts_of(int V, int each) {
  const int parts = (V / E::N + 64 * each - 1) / (64 * each);
  return parts > 0 ? parts : 1;
}

// A wave a part of a row.  Rows behind the end of a draft are not looked at.  Bound by HBM where there are many (128 x 17 rows of 131072 bf16: 89 us,
// 6.4 TB/s), at 9 instructions an element.
template <typename E>
__global__ __launch_bounds__(256) void verify_sums_kernel(VerifyArgs a, int rows, int parts, Sums* sums) {
  const int lane = threadIdx.x & 63;
  const unsigned item = blockIdx.x * 4 + uniform_i(threadIdx.x >> 6), of_seq = static_cast<unsigned>(rows) * parts;  // (see verify_draft_slice)
  const unsigned b = item / of_seq, within = item - b * of_seq;
  if (b >= static_cast<unsigned>(a.sequences)) return;
  const int j = static_cast<int>(within / parts), part = static_cast<int>(within) - j * parts;
  const Drafted tokens = drafted_tokens(a, b, lane);
  const int i = j <= a.n ? j : j - a.n - 1;
  if (j <= a.n ? i > tokens.count : i >= tokens.count) return;
  const Row<E> row = row_of<E>(a, b, j);
  float at = 0.0f;
  if (part == 0 && i < tokens.count) at = E::up(row.x[__builtin_amdgcn_readlane(tokens.t, i)]);
  Sums s = part_sums<E, kEach<E>>(row, part * 64 * kEach<E>, part == 0, j <= a.n ? a.target_scale.c : a.draft_scale.c, lane);
  s.at = at;
  if (lane == 0) sums[item] = s;
}

// What is decided from the sums of a sequence's rows.
struct Verdict {
  int k;           // accepted tokens
  int none;        // no token is drawn: the target's row there is nothing but -inf, or it, or the draft's, holds a NaN or +inf
  int refused;     // the token that was refused, -1: none
  float pm, qm;    // largest elements of the rows that decide; qm = -inf: no draft's row counts
  double ratio;    // of their sums, about
  double near;     // how far that is off at most, relative to itself
};
struct LeftVerdict {  // for the next launch
  Verdict d;
  double beside;  // of the target's row, as in RowSums
};

constexpr int kMaxRows = 2 * kMaxDrafts + 1;
struct RowSums {
  float m[kMaxRows];
  double s[kMaxRows];
  double off[kMaxRows];     // how far s is off at most, relative to itself
  double turn[16];          // a place a wave
  // Where s is 1 and less than kSmallBeside, this; else no less than that.  (Behind the others: decide() takes 8 registers more with it among them,
  // and a workgroup of 1024 threads then leaves no room for the next one's first waves: 128 x 17 rows of 131072 bf16 137 -> 140 us.)
  double beside[kMaxRows];
};

__device__ __forceinline__ double share(float x, float m, double s, const Scale& k) {  // (a row of nothing but -inf: s = 0; a marked one: NaN)
  if (m == -INFINITY) return s;
  const double w = weight(x, m, k);
  return (w > kNoWeight ? w : 0.0) / s;
}
// (Next to a near-certain token, the others' weight is all of the logarithm, and would be lost in a sum with its 1: log(1 + r) is r - r^2 / 2
// within 2^-40 of itself.  From kSmallBeside on what a sum in 64 bits keeps of it is nearer than the fp32 sums of long rows' parts.)
__device__ __forceinline__ float log_share(float x, float m, double s, double beside, double c) {
  const double all = beside < kSmallBeside ? fma(-0.5 * beside, beside, beside) : log2(s) * 0.69314718055994530942;
  return static_cast<float>((static_cast<double>(x) - static_cast<double>(m)) * c * 0.69314718055994530942 - all);
}

// Elements v .. v + N - 1 of a row of V; -inf past it.
template <typename E>
__device__ __forceinline__ void load_at(const typename E::type* x, int v, int V, float (&xs)[E::N]) {
  if (v + E::N <= V) {
    E::unpack(any_vector<E>(x + v), xs);
  } else {
#pragma unroll
    for (int i = 0; i < E::N; ++i) xs[i] = v + i < V ? E::up(x[v + i]) : -INFINITY;
  }
}
// A slice of a row: 64 vectors from a whole number of them on, in a wave.
template <typename E>
__host__ __device__ __forceinline__ int slices_of(int V) { return (V + 64 * E::N - 1) / (64 * E::N); }
template <int N>
__device__ __forceinline__ double lane_sum(const double (&w)[N]) {
  double s = w[0];
#pragma unroll
  for (int i = 1; i < N; ++i) s += w[i];
  return s;
}

// A row's sum in 64 bits, by the whole workgroup.
template <typename E, int WAVES>
__device__ __forceinline__ double row_sum(const typename E::type* x, int V, float m, const Scale& k, double (&turn)[16]) {
  const int lane = threadIdx.x & 63, wave = uniform_i(threadIdx.x >> 6);
  double s = 0.0;
  for (int slice = wave; slice < slices_of<E>(V); slice += WAVES) {
    float xs[E::N];
    load_at<E>(x, (slice * 64 + lane) * E::N, V, xs);
#pragma unroll
    for (int i = 0; i < E::N; ++i) s += weight(xs[i], m, k);
  }
  s = wave_sum64(s);
  __syncthreads();
  if (lane == 0) turn[wave] = s;
  __syncthreads();
  s = 0.0;
  for (int w = 0; w < WAVES; ++w) s += turn[w];
  return s;
}

// Joins the parts of all rows (waves of the workgroup take turns).
template <int WAVES>
__device__ __forceinline__ void join_rows(const VerifyArgs& a, const Sums* sums, int rows, int parts, RowSums& joined) {
  const int lane = threadIdx.x & 63, wave = uniform_i(threadIdx.x >> 6);
  const Sums none{-INFINITY, 0.0f, 0.0f, 0.0f};
  Sums next = wave < rows && lane < parts ? sums[wave * parts + lane] : none;
  for (int j = wave; j < rows; j += WAVES) {  // (rows behind the end of the draft too, whose sums nobody has written and nobody looks at)
    const Scale k = j <= a.n ? a.target_scale : a.draft_scale;
    Sums part = next;
    if (j + WAVES < rows && lane < parts) next = sums[(j + WAVES) * parts + lane];
    float m = part.m;
    for (int p = lane + 64; p < parts; p += 64) m = fmaxf(m, sums[j * parts + p].m);
    m = wave_max(m);
    double s = 0.0;
    for (int p = lane; p < parts; p += 64) {
      if (p > lane) part = sums[j * parts + p];
      s += part.m == -INFINITY ? static_cast<double>(part.s)  // (0, or NaN)
                               : (static_cast<double>(part.ones) + static_cast<double>(part.s)) * weight(part.m, m, k);
    }
    s = wave_sum64(s);
    double beside = s;
    if (s < kSmallBeside + 1.0) {  // (again, without the largest element)
      beside = 0.0;
      for (int p = lane; p < parts; p += 64) {
        part = sums[j * parts + p];
        beside += part.m == m || part.m == -INFINITY ? static_cast<double>(part.s) : (static_cast<double>(part.ones) + static_cast<double>(part.s)) * weight(part.m, m, k);
      }
      beside = wave_sum64(beside);
    }
    if (lane == 0) {
      joined.m[j] = m;
      joined.beside[j] = beside;
      joined.s[j] = s;
      joined.off[j] = off_by(s, a.V);
    }
  }
}

// Decides from the rows' sums, the same in every wave.  Writes the accepted tokens if `writes`, in the last wave.
template <typename E, int WAVES>
__device__ __forceinline__ Verdict decide(const VerifyArgs& a, int64_t b, const Drafted& tokens, float xt, float yt, RowSums& joined, bool writes) {
  const int lane = threadIdx.x & 63, wave = uniform_i(threadIdx.x >> 6), t = tokens.t, count = tokens.count;
  const float u = tokens.u;
  const typename E::type* target = static_cast<const typename E::type*>(a.target) + b * a.target_seq;
  const typename E::type* draft = a.draft ? static_cast<const typename E::type*>(a.draft) + b * a.draft_seq : nullptr;
  __syncthreads();
  bool takes = false;
  for (u64 exact = 0;;) {
    bool unsure = false;
    takes = false;
    if (lane < count) {
      const double p = share(xt, joined.m[lane], joined.s[lane], a.target_scale);
      const double q = draft ? share(yt, joined.m[a.n + 1 + lane], joined.s[a.n + 1 + lane], a.draft_scale) : 1.0;
      const double uq = static_cast<double>(u) * q;
      takes = uq < p;  // (false for NaN)
      unsure = p > 0.0 && fabs(uq - p) <= p * (joined.off[lane] + (draft ? joined.off[a.n + 1 + lane] : 0.0) + kBeside) && !((exact >> lane) & 1u);
    }
    const int stop = first_lane(~__ballot(takes || unsure));  // (the first that is refused for sure; lane 63 takes none)
    const u64 open = __ballot(unsure) & ((1ull << stop) - 1);
    if (open == 0) break;
    const int i = first_lane(open);
    const double ps = row_sum<E, WAVES>(target + i * a.target_row, a.V, joined.m[i], a.target_scale, joined.turn);
    const double qs = draft ? row_sum<E, WAVES>(draft + i * a.draft_row, a.V, joined.m[a.n + 1 + i], a.draft_scale, joined.turn) : 0.0;
    __syncthreads();
    if (threadIdx.x == 0) {
      if (joined.m[i] != -INFINITY) joined.s[i] = ps;
      if (draft && joined.m[a.n + 1 + i] != -INFINITY) joined.s[a.n + 1 + i] = qs;
    }
    exact |= 1ull << i;
    __syncthreads();
  }
  Verdict r;
  r.k = first_lane(~__ballot(takes));
  r.refused = r.k < count ? __builtin_amdgcn_readlane(t, r.k) : -1;
  const double ps = joined.s[r.k];
  r.pm = joined.m[r.k];
  r.qm = -INFINITY;
  r.ratio = r.near = 0.0;
  r.none = r.pm == -INFINITY || ps != ps;
  if (r.refused >= 0 && draft) {
    const double qs = joined.s[a.n + 1 + r.k];
    r.qm = joined.m[a.n + 1 + r.k];
    if (r.qm != -INFINITY) {
      r.ratio = ps / qs;
      r.near = joined.off[r.k] + joined.off[a.n + 1 + r.k] + kBeside;
    }
    r.none |= qs != qs;
  }
  if (writes && wave == WAVES - 1) {
    if (lane <= a.n && (lane != r.k || r.none)) {  // (the token at k is drawn later)
      a.out[b * (a.n + 1) + lane] = lane < r.k ? t : -1;
      if (a.logp) a.logp[b * (a.n + 1) + lane] = lane < r.k ? log_share(xt, joined.m[lane], joined.s[lane], joined.beside[lane], a.target_scale.c) : NAN;
    }
    if (lane == 0) a.accepted[b] = r.k;
  }
  return r;
}

// The same from the sums of a launch before.
template <typename E, int WAVES>
__device__ __forceinline__ Verdict decide_rows(const VerifyArgs& a, int64_t b, const Sums* sums, int rows, int parts, RowSums& joined, bool writes) {
  const int lane = threadIdx.x & 63;
  sums += b * rows * parts;
  float xt = 0.0f, yt = 0.0f;
  if (lane < a.n) {
    xt = sums[lane * parts].at;
    if (a.draft) yt = sums[(a.n + 1 + lane) * parts].at;
  }
  const Drafted tokens = drafted_tokens(a, b, lane);
  join_rows<WAVES>(a, sums, rows, parts, joined);
  return decide<E, WAVES>(a, b, tokens, xt, yt, joined, writes);
}

// The rows that decide, as weights.
template <typename E>
struct Rest {
  const typename E::type* x;
  const typename E::type* y;  // null: no draft's row counts
  int V, barred;              // the token that a draft without rows was sure of, -1: none
  float pm, qm;
  Scale pk, qk;
  __device__ __forceinline__ Rest(const VerifyArgs& a, int64_t b, const Verdict& d)
      : x(static_cast<const typename E::type*>(a.target) + b * a.target_seq + d.k * a.target_row),
        y(d.qm == -INFINITY ? nullptr : static_cast<const typename E::type*>(a.draft) + b * a.draft_seq + d.k * a.draft_row),
        V(a.V), barred(a.draft ? -1 : d.refused), pm(d.pm), qm(d.qm), pk(a.target_scale), qk(a.draft_scale) {}
  // Of elements v .. v + N - 1 (next to nothing past the row).
  __device__ __forceinline__ void weights(int v, double (&p)[E::N], double (&q)[E::N]) const {
    float xs[E::N], ys[E::N];
    load_at<E>(x, v, V, xs);
    if (y) load_at<E>(y, v, V, ys);
#pragma unroll
    for (int i = 0; i < E::N; ++i) {
      p[i] = weight(xs[i], pm, pk);
      q[i] = y ? weight(ys[i], qm, qk) : 0.0;
    }
  }
  // What a token may be drawn from: p - ratio q where that is more than nothing, in units of the target's largest weight; all of p
  // where `whole`.
  __device__ __forceinline__ void rest(int v, const double (&p)[E::N], const double (&q)[E::N], double ratio, bool whole, double (&r)[E::N]) const {
#pragma unroll
    for (int i = 0; i < E::N; ++i) {  // (what is compared hangs on d: kEven p alone is taken out of draw_held()'s loop, into registers that it does not have)
      const double d = whole ? p[i] : fma(-ratio, q[i], p[i]);
      r[i] = fma(-kEven, p[i], d) > kNoWeight && (whole || v + i != barred) ? d : 0.0;
    }
  }
};

// Where in the sums of the slices the drawn token lies, by any wave (the same in each).
struct Place {
  int slice;
  double before, target;  // what lies ahead of the slice, what the token's sum is to pass
};
__device__ __forceinline__ double sum_of(const double* sums, int n, int lane) {
  double all = 0.0;
  for (int s = lane; s < n; s += 64) all += sums[s];
  return wave_sum64(all);
}
__device__ __forceinline__ Place place_of(const double* sums, int slices, float w, double all, int lane) {
  Place r{0, 0.0, static_cast<double>(fminf(fmaxf(w, 0.0f), 0x1.fffffep-1f)) * all};
  double ahead = 0.0;
  for (int s0 = 0; s0 < slices; s0 += 64) {
    const double mine = s0 + lane < slices ? sums[s0 + lane] : 0.0;
    const double upto = ahead + wave_upto64(mine);
    const u64 has = __ballot(mine > 0.0 && upto > r.target), some = __ballot(mine > 0.0);
    if (some) {  // (the last slice with any mass, where roundings leave none past the target)
      const int at = has ? first_lane(has) : 63 - __builtin_clzll(some);
      r.slice = s0 + at;
      r.before = readlane64(upto - mine, at);
    }
    if (has) break;
    ahead = readlane64(upto, 63);
  }
  return r;
}

// The token within its slice: the first one up to which the sum passes the target; the last one with any mass where
// roundings leave none.
template <int N>
__device__ __forceinline__ int find_in_slice(const double (&w)[N], const Place& at, int lane) {
  const double s = lane_sum(w);
  double upto = at.before + (wave_upto64(s) - s);
  int found = -1, any = -1;
  const int v = (at.slice * 64 + lane) * N;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    upto += w[i];
    any = w[i] > 0.0 ? v + i : any;
    found = found < 0 && w[i] > 0.0 && upto > at.target ? v + i : found;
  }
  const u64 has = __ballot(found >= 0), some = __ballot(any >= 0);
  if (has) return __builtin_amdgcn_readlane(found, first_lane(has));
  return some ? __builtin_amdgcn_readlane(any, 63 - __builtin_clzll(some)) : -1;
}

template <typename E>
__device__ __forceinline__ void write_drawn(const VerifyArgs& a, int64_t b, const Verdict& d, double ps, double beside, int token, int lane) {
  if (lane != 0) return;
  const int64_t at = b * (a.n + 1) + d.k;
  a.out[at] = token;
  if (a.logp) a.logp[at] = token < 0 ? NAN : log_share(target_at<E>(a, b, d.k, token), d.pm, ps, beside, a.target_scale.c);
}

// Rows of up to WAVES * HELD slices: a workgroup a sequence holds the rows that decide in registers.
constexpr int kHeld = 2;  // at most
template <int WAVES>
struct DrawShared {
  double p[WAVES], q[WAVES], slices[WAVES * kHeld];
};
template <typename E, int WAVES, int HELD>
__device__ __forceinline__ void draw_held(const VerifyArgs& a, int64_t b, const Verdict& d, const RowSums& joined, DrawShared<WAVES>& shared) {
  const int lane = threadIdx.x & 63, wave = uniform_i(threadIdx.x >> 6), slices = slices_of<E>(a.V);
  const float number = a.numbers[b * (a.n + 1) + a.n];
  const Rest<E> r(a, b, d);
  double p[HELD][E::N], q[HELD][E::N], ps = 0.0, qs = 0.0;
#pragma unroll
  for (int h = 0; h < HELD; ++h) {
    if (wave + h * WAVES >= slices) break;
    r.weights(((wave + h * WAVES) * 64 + lane) * E::N, p[h], q[h]);
    ps += lane_sum(p[h]);
    qs += lane_sum(q[h]);
  }
  ps = wave_sum64(ps);
  qs = wave_sum64(qs);
  if (lane == 0) {
    shared.p[wave] = ps;
    shared.q[wave] = qs;
  }
  __syncthreads();
  ps = wave_sum64(lane < WAVES ? shared.p[lane] : 0.0);
  qs = wave_sum64(lane < WAVES ? shared.q[lane] : 0.0);
  const double ratio = r.y ? ps / qs : 0.0;
  for (bool whole = d.refused < 0;; whole = true) {
    double w[HELD][E::N];
#pragma unroll
    for (int h = 0; h < HELD; ++h) {
      const int s = wave + h * WAVES;
      if (s >= slices) break;
      r.rest((s * 64 + lane) * E::N, p[h], q[h], ratio, whole, w[h]);
      const double v = wave_sum64(lane_sum(w[h]));
      if (lane == 0) shared.slices[s] = v;
    }
    __syncthreads();
    const double all = sum_of(shared.slices, slices, lane);
    if (!whole && !(all > kNothing * ps)) {  // (the same in every wave)
      __syncthreads();
      continue;
    }
    const Place at = place_of(shared.slices, slices, number, all, lane);
#pragma unroll
    for (int h = 0; h < HELD; ++h)
      if (at.slice == wave + h * WAVES) write_drawn<E>(a, b, d, ps, joined.beside[d.k], find_in_slice(w[h], at, lane), lane);
    return;
  }
}
template <typename E, int WAVES, int HELD>
__global__ __launch_bounds__(64 * WAVES) void verify_draw_kernel(VerifyArgs a, int rows, int parts, const Sums* sums) {
  __shared__ RowSums joined;
  __shared__ DrawShared<WAVES> shared;
  const int64_t b = blockIdx.x;
  const Verdict d = decide_rows<E, WAVES>(a, b, sums, rows, parts, joined, true);
  if (!d.none) draw_held<E, WAVES, HELD>(a, b, d, joined, shared);
}

// All of a sequence in one workgroup, where its rows have few parts.
constexpr int kSmallItems = 32;
template <typename E, int WAVES, int EACH, int HELD>
__global__ __launch_bounds__(64 * WAVES) void verify_small_kernel(VerifyArgs a, int rows, int parts) {
  __shared__ RowSums joined;
  __shared__ Sums sums[kSmallItems];
  __shared__ DrawShared<WAVES> shared;
  const int lane = threadIdx.x & 63, wave = uniform_i(threadIdx.x >> 6);
  const int64_t b = blockIdx.x;
  const Drafted tokens = drafted_tokens(a, b, lane);
  float xt = 0.0f, yt = 0.0f;
  if (lane < tokens.count) {
    xt = target_at<E>(a, b, lane, tokens.t);
    if (a.draft) yt = draft_at<E>(a, b, lane, tokens.t);
  }
  for (int item = wave; item < rows * parts; item += WAVES) {
    const int j = item / parts, part = item - j * parts;
    if (j <= a.n ? j > tokens.count : j - a.n - 1 >= tokens.count) continue;
    const Sums s = part_sums<E, EACH>(row_of<E>(a, b, j), part * 64 * EACH, part == 0, j <= a.n ? a.target_scale.c : a.draft_scale.c, lane);
    if (lane == 0) sums[item] = s;
  }
  __syncthreads();
  join_rows<WAVES>(a, sums, rows, parts, joined);
  const Verdict d = decide<E, WAVES>(a, b, tokens, xt, yt, joined, true);
  if (!d.none) draw_held<E, WAVES, HELD>(a, b, d, joined, shared);
}

// Long rows: several workgroups a sequence decide, each for itself, and sum their slices; the first leaves the verdict.
struct Slice {
  double p, q;              // sums of the weights
  double above;             // of p - ratio q over the tokens above the line (the draft's token without rows aside), with the verdict's ratio
  double above_q;           // of q over those
  double near_p, near_q;    // of p and q over tokens that may lie on either side, which are not among those
  double low, high;         // the least and the largest p / q - ratio of these (none: inf, -inf)
};
// Bound by instructions in 64 bits, 46 an element of both rows (128 sequences of 131072: 43 us); few sequences by the chain of reads up to the
// decision and the row behind it (9 us).
constexpr int kRestWaves = 16;
template <typename E>
__global__ __launch_bounds__(64 * kRestWaves) void verify_rest_kernel(VerifyArgs a, int rows, int parts, const Sums* sums, LeftVerdict* verdicts, Slice* out) {
  __shared__ RowSums joined;
  const int lane = threadIdx.x & 63, wave = uniform_i(threadIdx.x >> 6), slices = slices_of<E>(a.V);
  const int64_t b = blockIdx.y;
  const Verdict d = decide_rows<E, kRestWaves>(a, b, sums, rows, parts, joined, blockIdx.x == 0);
  if (blockIdx.x == 0 && threadIdx.x == 0) verdicts[b] = LeftVerdict{d, joined.beside[d.k]};
  if (d.none) return;
  const Rest<E> r(a, b, d);
  for (int s = blockIdx.x * kRestWaves + wave; s < slices; s += gridDim.x * kRestWaves) {
    const int v = (s * 64 + lane) * E::N;
    Slice to{0.0, 0.0, 0.0, 0.0, 0.0, 0.0, INFINITY, -INFINITY};
    if (r.y) {
      float xs[E::N], ys[E::N];
      load_at<E>(r.x, v, r.V, xs);
      load_at<E>(r.y, v, r.V, ys);
      double near = INFINITY;
#pragma unroll
      for (int i = 0; i < E::N; ++i) {
        const double p = weight(xs[i], r.pm, r.pk), q = weight(ys[i], r.qm, r.qk), rest = fma(-d.ratio, q, p);
        near = fmin(near, fma(-d.near * d.ratio, q, fabs(rest)));
        to.p += p;
        to.q += q;
        to.above += fmax(rest, 0.0);
        to.above_q += rest > 0.0 ? q : 0.0;
      }
      if (__ballot(near <= 0.0) != 0) {
        to.above = to.above_q = 0.0;
#pragma unroll 1
        for (int i = 0; i < E::N; ++i) {
          const double p = weight(xs[i], r.pm, r.pk), q = weight(ys[i], r.qm, r.qk), rest = fma(-d.ratio, q, p);
          if (fabs(rest) <= d.near * d.ratio * q) {
            to.near_p += p;
            to.near_q += q;
            to.low = fmin(to.low, rest / q);
            to.high = fmax(to.high, rest / q);
          } else if (rest > 0.0) {
            to.above += rest;
            to.above_q += q;
          }
        }
        to.near_p = wave_sum64(to.near_p);
        to.near_q = wave_sum64(to.near_q);
#pragma unroll
        for (int l = 1; l < 64; l *= 2) {
          to.low = fmin(to.low, __shfl_xor(to.low, l, 64));
          to.high = fmax(to.high, __shfl_xor(to.high, l, 64));
        }
      }
      to.q = wave_sum64(to.q);
      to.above = wave_sum64(to.above);
      to.above_q = wave_sum64(to.above_q);
    } else {
      double p[E::N], q[E::N], w[E::N];
      r.weights(v, p, q);
      to.p = lane_sum(p);
      if (r.barred >= 0) {
        r.rest(v, p, q, 0.0, false, w);
        to.above = wave_sum64(lane_sum(w));
      }
    }
    to.p = wave_sum64(to.p);
    if (lane == 0) out[b * slices + s] = to;
  }
}
// Draws from the slices' sums (in LDS), by a wave.
template <typename E>
__device__ __forceinline__ void draw_from(const VerifyArgs& a, int64_t b, const Verdict& d, const Rest<E>& r, double* sums, int slices, float number, double ratio,
                                          bool whole, double ps, double beside, double all, int lane) {
  for (;;) {
    const Place at = place_of(sums, slices, number, all, lane);
    const int v = (at.slice * 64 + lane) * E::N;
    double p[E::N], q[E::N], w[E::N];
    r.weights(v, p, q);
    r.rest(v, p, q, ratio, whole, w);
    const int token = find_in_slice(w, at, lane);
    if (token >= 0 || !(sums[at.slice] > 0.0)) return write_drawn<E>(a, b, d, ps, beside, token, lane);
    // (nothing but weights that are none each, and together are one: not a slice to draw from)
    __builtin_amdgcn_wave_barrier();
    if (lane == 0) sums[at.slice] = 0.0;
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
    all = sum_of(sums, slices, lane);
  }
}
// And a workgroup a sequence draws.
constexpr int kPickWaves = 8;
template <typename E>
__global__ __launch_bounds__(64 * kPickWaves) void verify_pick_kernel(VerifyArgs a, const LeftVerdict* verdicts, const Slice* in) {
  __shared__ double sums[kLogitsMaxV / (64 * E::N)], turn[2 * kPickWaves];
  __shared__ int again;
  const int lane = threadIdx.x & 63, wave = uniform_i(threadIdx.x >> 6), slices = slices_of<E>(a.V);
  constexpr int kMine = (kLogitsMaxV / (64 * E::N) + 64 * kPickWaves - 1) / (64 * kPickWaves);
  const int64_t b = blockIdx.x;
  in += b * slices;
  Slice mine[kMine];
  double ps = 0.0, qs = 0.0;
#pragma unroll
  for (int k = 0; k < kMine; ++k) {
    const int s = threadIdx.x + k * 64 * kPickWaves;
    mine[k] = s < slices ? in[s] : Slice{0.0, 0.0, 0.0, 0.0, 0.0, 0.0, INFINITY, -INFINITY};
  }
  const float number = a.numbers[b * (a.n + 1) + a.n];
  const Verdict d = verdicts[b].d;
  if (d.none) return;  // (and nothing was summed)
#pragma unroll
  for (int k = 0; k < kMine; ++k) {
    ps += mine[k].p;
    qs += mine[k].q;
  }
  ps = wave_sum64(ps);
  qs = wave_sum64(qs);
  if (lane == 0) {
    turn[wave] = ps;
    turn[kPickWaves + wave] = qs;
  }
  if (threadIdx.x == 0) again = 0;
  __syncthreads();
  ps = wave_sum64(lane < kPickWaves ? turn[lane] : 0.0);
  qs = wave_sum64(lane < kPickWaves ? turn[kPickWaves + lane] : 0.0);
  const Rest<E> r(a, b, d);
  const double ratio = r.y ? ps / qs : 0.0;
  bool whole = d.refused < 0 || (!r.y && r.barred < 0);  // (a draft's row of nothing but -inf takes nothing away)
  for (;; whole = true) {
#pragma unroll
    for (int k = 0; k < kMine; ++k) {
      const int s = threadIdx.x + k * 64 * kPickWaves;
      double v = whole ? mine[k].p : mine[k].above;
      if (!whole && r.y) {  // (a slice with tokens on both sides of the ratio that the last bits of their weights decide is summed again)
        const double further = ratio - d.ratio, bits = ratio * 0x1p-44;
        v = fma(-further, mine[k].above_q, v);
        if (mine[k].low > further + bits) v += fma(-ratio, mine[k].near_q, mine[k].near_p);
        else if (!(mine[k].high < further - bits)) v = NAN;
      }
      if (s < slices) sums[s] = v != v || v > kNoWeight ? v : 0.0;
      if (s < slices && v != v) again = 1;
    }
    __syncthreads();
    for (int s = wave; s < slices && !whole && again; s += kPickWaves) {
      if (sums[s] == sums[s]) continue;
      const int from = (s * 64 + lane) * E::N;
      double p[E::N], q[E::N], w[E::N];
      r.weights(from, p, q);
      r.rest(from, p, q, ratio, false, w);
      const double again = wave_sum64(lane_sum(w));
      if (lane == 0) sums[s] = again;
    }
    __syncthreads();
    const double all = sum_of(sums, slices, lane);
    if (!whole && !(all > kNothing * ps)) {
      __syncthreads();
      continue;
    }
    if (wave == 0) draw_from(a, b, d, r, sums, slices, number, ratio, whole, ps, verdicts[b].beside, all, lane);
    return;
  }
}

// Rows without a draft, and a few of one that was sure of its tokens, need no ratio: all are summed in 64 bits, slice by slice, and one launch more
// decides and draws from those sums.  us, this way / in three launches, bf16 where not said: 1 x 1 row of 131072 11.7 / 12.6, 70 x 1 of 89793 16.5 / 20.1,
// 254 x 1 of 34124 17.4 / 20.6, 64 x 1 of 131072 fp32 19.8 / 26.6, 256 x 1 of 131072 34.8 / 46.3; 1 x 5 of 131072 13.9 / 14.4, 22 x 5 of 42561 16.9 / 16.6,
// 10 x 16 of 41282 fp32 19.0 / 18.3, 98 x 5 of 39809 28.3 / 25.3, 64 x 9 of 50000 34.5 / 25.9.  (256 x 1 of 131072: 32 and 8 us, the first bound by its 16
// instructions in 64 bits an element, where reading takes 10.)
constexpr int64_t kSureElements = 5 << 20;  // of rows of a draft
constexpr int32_t kHeldTwice = 128;         // sequences up to which no workgroup holds two slices of 16-bit rows a wave
struct SliceSum {
  float m;     // the largest element of the slices that a wave has summed
  float ones;  // how many of them the slice has
  double s;    // of the others' weights, in units of its own (NaN where one of these slices holds a NaN or +inf)
  __device__ __forceinline__ double in_units_of(float most, const Scale& k) const { return m == -INFINITY ? s : (ones + s) * weight(m, most, k); }
};
constexpr int kSureSlices = 4;  // a wave
template <typename E>
__global__ __launch_bounds__(256) void verify_slices_kernel(VerifyArgs a, int parts, SliceSum* out) {
  const int lane = threadIdx.x & 63, rows = a.n + 1, slices = slices_of<E>(a.V);
  const unsigned item = blockIdx.x * 4 + uniform_i(threadIdx.x >> 6), of_seq = static_cast<unsigned>(rows) * parts;
  const unsigned b = item / of_seq, within = item - b * of_seq;
  if (b >= static_cast<unsigned>(a.sequences)) return;
  const int j = static_cast<int>(within / parts), first = (static_cast<int>(within) - j * parts) * kSureSlices;
  const typename E::type* row = static_cast<const typename E::type*>(a.target) + b * a.target_seq + j * a.target_row;
  float x[kSureSlices][E::N], most[kSureSlices], m = -INFINITY;
  const int t = lane < j ? a.tokens[static_cast<int64_t>(b) * a.n + lane] : 0;
  if (__ballot(static_cast<unsigned>(t) >= static_cast<unsigned>(a.V))) return;  // (a row behind the end of the draft)
#pragma unroll
  for (int k = 0; k < kSureSlices; ++k) load_at<E>(row, ((first + k) * 64 + lane) * E::N, a.V, x[k]);
  bool marked = false;
#pragma unroll
  for (int k = 0; k < kSureSlices; ++k) {
    most[k] = vec_max(x[k]);
    m = fmaxf(m, most[k]);
#pragma unroll
    for (int i = 0; i < E::N; ++i) marked |= !(x[k][i] < INFINITY);
  }
  m = wave_max(m);
  const bool none = __ballot(marked) != 0;
  const float from = m == -INFINITY ? 0.0f : m;
#pragma unroll
  for (int k = 0; k < kSureSlices; ++k) {
    double s = 0.0;
    int ones = 0;
#pragma unroll
    for (int i = 0; i < E::N; ++i) s += weight(x[k][i], from, a.target_scale);
    if (__ballot(most[k] == from) != 0) {  // (again, without the largest elements)
      s = 0.0;
#pragma unroll
      for (int i = 0; i < E::N; ++i) {
        const double w = weight(x[k][i], from, a.target_scale);
        s += x[k][i] == from ? 0.0 : w;
        ones += __builtin_popcountll(__ballot(x[k][i] == from));
      }
    }
    s = wave_sum64(s);
    if (lane == 0 && first + k < slices)
      out[(static_cast<int64_t>(b) * rows + j) * slices + first + k] = SliceSum{m, static_cast<float>(ones), none ? NAN : m == -INFINITY ? 0.0 : s};
  }
}
constexpr int kSureWaves = 16;
template <typename E>
__global__ __launch_bounds__(64 * kSureWaves) void verify_sure_kernel(VerifyArgs a, const SliceSum* in) {
  __shared__ RowSums joined;
  __shared__ double sums[kLogitsMaxV / (64 * E::N)];
  const int lane = threadIdx.x & 63, wave = uniform_i(threadIdx.x >> 6), slices = slices_of<E>(a.V);
  const int64_t b = blockIdx.x;
  in += b * (a.n + 1) * slices;
  const Drafted tokens = drafted_tokens(a, b, lane);
  const float xt = lane < tokens.count ? target_at<E>(a, b, lane, tokens.t) : 0.0f, number = a.numbers[b * (a.n + 1) + a.n];
  for (int j = wave; j <= tokens.count; j += kSureWaves) {
    float m = -INFINITY;
    for (int s = lane; s < slices; s += 64) m = fmaxf(m, in[j * slices + s].m);
    m = wave_max(m);
    double all = 0.0, ones = 0.0;  // (see log_share)
    for (int s = lane; s < slices; s += 64) {
      const SliceSum part = in[j * slices + s];
      all += part.m == m ? part.s : part.in_units_of(m, a.target_scale);
      ones += part.m == m ? part.ones : 0.0f;
    }
    all = wave_sum64(all);
    ones = wave_sum64(ones);
    if (lane == 0) {
      joined.m[j] = m;
      joined.beside[j] = ones > 1.0 ? ones : all;
      joined.s[j] = ones + all;
      joined.off[j] = 0.0;
    }
  }
  const Verdict d = decide<E, kSureWaves>(a, b, tokens, xt, 0.0f, joined, true);
  if (d.none) return;
  const Rest<E> r(a, b, d);
  const int own = d.refused < 0 ? -1 : d.refused / (64 * E::N);  // the slice of the token that may not be drawn
  const double ps = joined.s[d.k];
  for (bool whole = d.refused < 0;; whole = true) {
    for (int s = threadIdx.x; s < slices; s += 64 * kSureWaves) {
      const SliceSum part = in[d.k * slices + s];
      const double v = part.in_units_of(d.pm, a.target_scale);
      if (whole || s != own) sums[s] = v > kNoWeight ? v : 0.0;
    }
    if (!whole && wave == kSureWaves - 1) {
      double p[E::N], q[E::N], w[E::N];
      r.weights((own * 64 + lane) * E::N, p, q);
      r.rest((own * 64 + lane) * E::N, p, q, 0.0, false, w);
      const double v = wave_sum64(lane_sum(w));
      if (lane == 0) sums[own] = v;
    }
    __syncthreads();
    const double all = sum_of(sums, slices, lane);
    if (!whole && !(all > kNothing * ps)) {  // (the same in every wave)
      __syncthreads();
      continue;
    }
    if (wave == 0) draw_from(a, b, d, r, sums, slices, number, 0.0, whole, ps, joined.beside[d.k], all, lane);
    return;
  }
}

// How a call is laid out.  us, one launch / two, 16 waves a sequence: 1 x 9 rows of 1024 fp32 8.3 / 10.0, 64 x 17 of 1025 bf16 10.4 / 11.8, 256 x 31 of
// 1025 13.2 / 15.9, 1 x 17 of 4096 12.8 / 11.8, 256 x 17 of 4096 16.7 / 18.5, 1 x 9 of 8192 13.9 / 13.0, 256 x 9 of 8192 18.7 / 20.8, 64 x 3 of 16384 17.3 /
// 18.1.  Two launches / three: 1 x 9 rows of 16000 bf16 16.5 / 15.4, 64 x 9 22.0 / 21.2, 128 x 9 24.6 / 24.1, 256 x 9 29.5 / 32.4, 64 x 9 of 8000
// 15.9 / 20.2, 1 x 9 of 8000 fp32 13.7 / 14.3, 256 x 5 20.7 / 23.6; past what the registers of a workgroup hold there are three.  Workgroups a sequence for 256 / 512 in all: 128 x 17 of 131072 bf16 155 /
// 149, 200 x 3 of 131072 fp32 139.5 / 134.5, 64 x 3 of 131072 bf16 40.0 / 41.4, 64 x 9 of 50000 without rows of the draft 27.0 / 29.2, 128 x 9 of 50000 51.0 /
// 52.1, 256 x 5 of 65536 72.0 / 73.6, 128 x 17 of 32001 fp32 70.7 / 73.7.
struct Plan {
  int rows, parts;
  int groups;  // workgroups a sequence that sum the row that decides; 0: one workgroup decides and draws; -1: one does everything; -2: from sums of all
               // slices in 64 bits, one decides and draws
  int64_t verdicts, slice_sums, bytes;  // places in the workspace, its size
};
template <typename E>
Plan plan(int32_t sequences, int32_t n, bool drafted, int32_t V) {
  Plan p;
  p.rows = drafted ? 2 * n + 1 : n + 1;
  p.parts = parts_of<E>(V, kSmallEach);
  const int slices = slices_of<E>(V);
  if (p.rows * p.parts <= kSmallItems && slices <= 16 * kHeld) {
    p.groups = -1;
    p.verdicts = p.slice_sums = p.bytes = 0;
    return p;
  }
  p.parts = parts_of<E>(V, kEach<E>);
  const int held = E::N == 8 && sequences <= kHeldTwice ? 16 : 16 * kHeld;  // slices that one workgroup decides and draws from
  if (!drafted && slices > held && (n == 0 || static_cast<int64_t>(sequences) * p.rows * V <= kSureElements)) {
    p.groups = -2;
    p.verdicts = p.slice_sums = 0;
    p.bytes = static_cast<int64_t>(sequences) * p.rows * slices * static_cast<int64_t>(sizeof(SliceSum));
    return p;
  }
  int64_t groups = 256 / sequences;
  if (slices >= 256) groups = std::max<int64_t>(groups, std::min(512 / sequences, slices / (4 * kRestWaves)));  // (four slices a wave)
  p.groups = slices <= held ? 0 : static_cast<int>(std::min<int64_t>((slices + kRestWaves - 1) / kRestWaves, std::max<int64_t>(1, groups)));
  p.verdicts = (static_cast<int64_t>(sequences) * p.rows * p.parts * static_cast<int64_t>(sizeof(Sums)) + 15) / 16 * 16;
  p.slice_sums = p.verdicts + (p.groups > 0 ? (static_cast<int64_t>(sequences) * static_cast<int64_t>(sizeof(LeftVerdict)) + 15) / 16 * 16 : 0);
  p.bytes = p.slice_sums + (p.groups > 0 ? static_cast<int64_t>(sequences) * slices * static_cast<int64_t>(sizeof(Slice)) : 0);
  return p;
}

template <typename E>
int forward(const VerifyArgs& a, void* workspace, hipStream_t stream) {
  auto done = [] { return hipGetLastError() == hipSuccess ? PB_OK : PB_EHIP; };
  const Plan p = plan<E>(a.sequences, a.n, a.draft != nullptr, a.V);
  if (p.groups == -1) {
    if (a.V <= 4 * 64 * E::N) verify_small_kernel<E, 16, 4, 1><<<a.sequences, 1024, 0, stream>>>(a, p.rows, p.parts);
    else if (slices_of<E>(a.V) <= 16) verify_small_kernel<E, 16, kSmallEach, 1><<<a.sequences, 1024, 0, stream>>>(a, p.rows, p.parts);
    else verify_small_kernel<E, 16, kSmallEach, 2><<<a.sequences, 1024, 0, stream>>>(a, p.rows, p.parts);
    return done();
  }
  if (p.groups == -2) {
    const int parts = (slices_of<E>(a.V) + kSureSlices - 1) / kSureSlices;
    SliceSum* slices = static_cast<SliceSum*>(workspace);
    verify_slices_kernel<E><<<static_cast<unsigned>((static_cast<int64_t>(a.sequences) * p.rows * parts + 3) / 4), 256, 0, stream>>>(a, parts, slices);
    if (done() != PB_OK) return PB_EHIP;
    verify_sure_kernel<E><<<a.sequences, 64 * kSureWaves, 0, stream>>>(a, slices);
    return done();
  }
  char* ws = static_cast<char*>(workspace);
  Sums* sums = reinterpret_cast<Sums*>(ws);
  const unsigned grid = static_cast<unsigned>((static_cast<int64_t>(a.sequences) * p.rows * p.parts + 3) / 4);
  verify_sums_kernel<E><<<grid, 256, 0, stream>>>(a, p.rows, p.parts, sums);
  if (done() != PB_OK) return PB_EHIP;
  if (p.groups == 0) {
    if (slices_of<E>(a.V) <= 16) verify_draw_kernel<E, 16, 1><<<a.sequences, 1024, 0, stream>>>(a, p.rows, p.parts, sums);
    else verify_draw_kernel<E, 16, 2><<<a.sequences, 1024, 0, stream>>>(a, p.rows, p.parts, sums);
    return done();
  }
  LeftVerdict* verdicts = reinterpret_cast<LeftVerdict*>(ws + p.verdicts);
  Slice* slice_sums = reinterpret_cast<Slice*>(ws + p.slice_sums);
  verify_rest_kernel<E><<<dim3(p.groups, a.sequences), 64 * kRestWaves, 0, stream>>>(a, p.rows, p.parts, sums, verdicts, slice_sums);
  if (done() != PB_OK) return PB_EHIP;
  verify_pick_kernel<E><<<a.sequences, 64 * kPickWaves, 0, stream>>>(a, verdicts, slice_sums);
  return done();
}

}  // namespace vd

// (Sequences are the second dimension of a grid, which holds 65535 at most.)
int32_t verify_draft_slice(int dtype, int32_t n, int32_t V) {
  const int parts = dtype == PB_F32 ? vd::parts_of<lr::F32>(V, vd::kEach<lr::F32>) : vd::parts_of<lr::F16>(V, vd::kEach<lr::F16>);
  return static_cast<int32_t>(std::min<int64_t>(32768, 4 * kMostGroups / ((2 * n + 1) * static_cast<int64_t>(parts))));
}
// (The size is that of the call with rows of the draft and of that without, whichever is larger, and no less than that of fewer sequences: those
// that a rule of plan() ends at are asked for too.)
int64_t verify_draft_workspace(int dtype, int32_t sequences, int32_t n, int32_t V) {
  const int32_t most = std::min(sequences, verify_draft_slice(dtype, n, V));
  const int32_t sure = static_cast<int32_t>(std::min<int64_t>(most, vd::kSureElements / ((n + 1) * static_cast<int64_t>(V))));
  int64_t bytes = 0;
  for (const int32_t count : {most, std::min(most, vd::kHeldTwice), sure})
    for (const bool drafted : {false, true})
      if (count > 0) bytes = std::max(bytes, (dtype == PB_F32 ? vd::plan<lr::F32>(count, n, drafted, V) : vd::plan<lr::F16>(count, n, drafted, V)).bytes);
  return bytes;
}
int launch_verify_draft(int dtype, const VerifyArgs& a, void* workspace, hipStream_t stream) {
  return dtype == PB_F32   ? vd::forward<lr::F32>(a, workspace, stream)
         : dtype == PB_F16 ? vd::forward<lr::F16>(a, workspace, stream)
                           : vd::forward<lr::BF16>(a, workspace, stream);
}

}  // namespace pb
