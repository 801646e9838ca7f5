// Verification of drafted tokens (pb_verify_draft): which of them a target's rows accept, and the token drawn behind them.
//
//   p_i = softmax(x_i / T), q_i = softmax(y_i / T') (or 1 at t_i): t_i is accepted where those before it are and u_i q_i(t_i) < p_i(t_i);
//   behind the k accepted ones a token is drawn from max(p_k - q_k, 0), or from p_k where no drafted token was refused: the first
//   v whose sum over all tokens up to it exceeds w times the sum over all.
//
// A drawn token is a border between two of V sums: with sums in fp32, off by 1e-7 of the whole, one draw in a hundred from a
// row of 131072 tokens would be another token than the definition's.  So exponentials and sums are in 64 bits throughout, which
// the chip's vector units take at the rate of fp32.
#include <algorithm>

#include "pb_logit_rows.hpp"
#include "pb_student.hpp"

namespace pb {
namespace vd {

using namespace lr;
using wv::first_lane;

// Of one row, or of a part of it: the largest element and the sum of 2^((x - m) c); bad: it holds a NaN or +inf.
struct Sums {
  float m;
  int bad;
  double s;
};

constexpr double kNothing = 0x1p-40;     // a rest of the target's mass below this is none (equal rows differ by their roundings)
constexpr double kNoWeight = 0x1p-960;   // weights below this, masked tokens' among them, are none

// What turns x - m into a weight: log2(e) / T, and the difference below which weights do not go (2^-1000).
struct Scale {
  double c, low;
};
__device__ __forceinline__ Scale scale_of(double c) { return Scale{c, -1000.0 / c}; }

// 2^((x - m) c) for x <= m, at least 2^-1000, off by 4e-14 of itself: with n the nearest integer to the exponent (in the low word of
// the sum with 1.5 2^52) and r what is left, 1 + r P(r), P by interpolation at Chebyshev's nodes, and n added to the exponent.  (16
// instructions in 64 bits; with rounding, conversion and ldexp as instructions of their own, 19, of which those are slower than the
// others: 128 x 17 rows of 131072 bf16 209 us against ...)
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
__device__ __forceinline__ Sums part_sums(const Row<E>& row, int first, bool edge, double c, int lane) {
  v4u raw[EACH];
  float m = -INFINITY, xe = -INFINITY;
#pragma unroll
  for (int u = 0; u < EACH; ++u) {
    const int v = first + 64 * u + lane;
    raw[u] = v < row.nv ? row.vec(v) : E::nothing();
  }
  if (edge && lane < row.edges) xe = E::up(row.x[row.edge_token(lane)]);
  bool bad = xe != xe;
  m = fmaxf(m, xe);
#pragma unroll
  for (int u = 0; u < EACH; ++u) {
    float x[E::N];
    E::unpack(raw[u], x);
#pragma unroll
    for (int i = 0; i < E::N; i += 2) bad |= __builtin_isunordered(x[i], x[i + 1]);
    m = fmaxf(m, vec_max(x));
  }
  m = wave_max(m);
  bad = __ballot(bad) != 0 || m == INFINITY;
  if (m == -INFINITY || bad) return Sums{m, bad, 0.0};
  const Scale k = scale_of(c);
  double s = edge && lane < row.edges ? weight(xe, m, k) : 0.0;
#pragma unroll
  for (int u = 0; u < EACH; ++u) {
    if (first + 64 * u >= row.nv) break;
    float x[E::N];
    E::unpack(raw[u], x);
#pragma unroll
    for (int i = 0; i < E::N; ++i) s += weight(x[i], m, k);
  }
  return Sums{m, 0, wave_sum64(s)};
}

// The rows of a sequence: 0 .. n the target's, n + 1 .. 2 n the draft's.
template <typename E>
__device__ __forceinline__ Row<E> row_of(const VerifyArgs& a, int64_t b, int j) {
  return j <= a.n ? row_at<E>(static_cast<const typename E::type*>(a.target) + b * a.target_seq, a.target_row, j, a.V)
                  : row_at<E>(static_cast<const typename E::type*>(a.draft) + b * a.draft_seq, a.draft_row, j - a.n - 1, a.V);
}
// Drafted tokens of a sequence, and those of them before the first that is absent.
__device__ __forceinline__ int drafted_tokens(const VerifyArgs& a, int64_t b, int lane, int* count) {
  const int t = lane < a.n ? a.tokens[b * a.n + lane] : -1;
  const u64 none = ~__ballot(static_cast<unsigned>(t) < static_cast<unsigned>(a.V));
  *count = none ? first_lane(none) : 64;  // (n <= 63: lane 63 holds none)
  return t;
}

// A row is split in parts of 64 EACH vectors, a wave each; at least one.
template <typename E>
__host__ __device__ __forceinline__ int parts_of(int V, int each) {
  const int parts = (V / E::N + 64 * each - 1) / (64 * each);
  return parts > 0 ? parts : 1;
}

// A wave a part of a row.  Rows behind the end of a draft are not looked at.
template <typename E, int EACH>
__global__ __launch_bounds__(256) void verify_sums_kernel(VerifyArgs a, int rows, int parts, Sums* sums) {
  const int lane = threadIdx.x & 63;
  const int64_t item = static_cast<int64_t>(blockIdx.x) * 4 + uniform_i(threadIdx.x >> 6);
  if (item >= static_cast<int64_t>(a.sequences) * rows * parts) return;
  const int part = static_cast<int>(item % parts), j = static_cast<int>(item / parts % rows);
  const int64_t b = item / parts / rows;
  int count;
  drafted_tokens(a, b, lane, &count);
  if (j <= a.n ? j > count : j - a.n - 1 >= count) return;
  const Row<E> row = row_of<E>(a, b, j);
  const Sums s = part_sums<E, EACH>(row, part * 64 * EACH, part == 0, j <= a.n ? a.target_c : a.draft_c, lane);
  if (lane == 0) sums[item] = s;
}

// What is decided from the sums of a sequence's rows.
struct Verdict {
  int k;           // accepted tokens
  int none;        // no token is drawn: the target's row there is nothing but -inf, or it, or the draft's, holds a NaN or +inf
  int refused;     // a drafted token was refused: the draft's row counts
  int token;       // that one
  float pm, qm;    // of the rows that decide
  double pw, qw;   // 1 / their sums (the draft's: 0 for a row of nothing but -inf)
  double ps;       // the target's sum
};

constexpr int kMaxRows = 2 * kMaxDrafts + 1;
struct RowSums {
  float m[kMaxRows];
  double s[kMaxRows];
};

__device__ __forceinline__ double share(float x, float m, double s, double c) {  // (a row of nothing but -inf: s = 0; a marked one: NaN)
  if (m == -INFINITY) return s;
  const double w = weight(x, m, scale_of(c));
  return (w > kNoWeight ? w : 0.0) / s;
}
__device__ __forceinline__ float log_share(float x, float m, double s, double c) {
  return static_cast<float>(((static_cast<double>(x) - static_cast<double>(m)) * c - log2(s)) * 0.69314718055994530942);
}

// Joins the parts of all rows (waves of the workgroup take turns), then decides, the same in every wave.  Writes the accepted tokens
// if `writes`, in the last wave.
template <typename E, int WAVES>
__device__ __forceinline__ Verdict decide(const VerifyArgs& a, int64_t b, const Sums* sums, int rows, int parts, RowSums& joined, bool writes) {
  const int lane = threadIdx.x & 63, wave = uniform_i(threadIdx.x >> 6);
  int count;
  const int t = drafted_tokens(a, b, lane, &count);
  float xt = 0.0f, yt = 0.0f, u = 0.0f;
  if (lane < count) {
    xt = E::up((static_cast<const typename E::type*>(a.target) + b * a.target_seq + lane * a.target_row)[t]);
    if (a.draft) yt = E::up((static_cast<const typename E::type*>(a.draft) + b * a.draft_seq + lane * a.draft_row)[t]);
    u = fminf(fmaxf(a.numbers[b * (a.n + 1) + lane], 0.0f), 0x1.fffffep-1f);
  }
  for (int j = wave; j < rows; j += WAVES) {
    if (j <= a.n ? j > count : j - a.n - 1 >= count) continue;
    const double c = j <= a.n ? a.target_c : a.draft_c;
    float m = -INFINITY;
    bool bad = false;
    for (int p = lane; p < parts; p += 64) {
      m = fmaxf(m, sums[j * parts + p].m);
      bad |= sums[j * parts + p].bad != 0;
    }
    m = wave_max(m);
    double s = 0.0;
    if (m != -INFINITY)
      for (int p = lane; p < parts; p += 64) s += sums[j * parts + p].s * weight(sums[j * parts + p].m, m, scale_of(c));
    s = wave_sum64(s);
    if (__ballot(bad) != 0) s = NAN;
    if (lane == 0) {
      joined.m[j] = m;
      joined.s[j] = s;
    }
  }
  __syncthreads();
  bool takes = false;
  if (lane < count) {
    const double p = share(xt, joined.m[lane], joined.s[lane], a.target_c);
    const double q = a.draft ? share(yt, joined.m[a.n + 1 + lane], joined.s[a.n + 1 + lane], a.draft_c) : 1.0;
    takes = static_cast<double>(u) * q < p;  // (false for NaN)
  }
  Verdict r;
  r.k = first_lane(~__ballot(takes));  // (lane 63 takes none)
  r.refused = r.k < count;
  r.token = __builtin_amdgcn_readlane(t, r.k);
  r.pm = joined.m[r.k];
  r.ps = joined.s[r.k];
  r.pw = 1.0 / r.ps;
  r.qm = -INFINITY;
  r.qw = 0.0;
  r.none = r.pm == -INFINITY || r.ps != r.ps;
  if (r.refused && a.draft) {
    const double qs = joined.s[a.n + 1 + r.k];
    r.qm = joined.m[a.n + 1 + r.k];
    r.qw = r.qm == -INFINITY ? 0.0 : 1.0 / qs;
    r.none |= qs != qs;
  }
  if (writes && wave == WAVES - 1) {
    if (lane <= a.n && (lane != r.k || r.none)) {  // (the token at k is drawn later)
      a.out[b * (a.n + 1) + lane] = lane < r.k ? t : -1;
      if (a.logp) a.logp[b * (a.n + 1) + lane] = lane < r.k ? log_share(xt, joined.m[lane], joined.s[lane], a.target_c) : NAN;
    }
    if (lane == 0) a.accepted[b] = r.k;
  }
  return r;
}

// The row that decides, as what a token may be drawn from: max(p - q, 0), or p where `whole`.
template <typename E>
struct Rest {
  const typename E::type* x;
  const typename E::type* y;  // null: no draft's row counts
  int V, barred;              // the token that a draft without rows was sure of, -1: none
  float pm, qm;
  double pw, qw;
  Scale pk, qk;
  // Elements v .. v + N - 1 (0 past the row).
  __device__ __forceinline__ void at(int v, double (&r)[E::N]) const {
    float xs[E::N], ys[E::N];
    if (v + E::N <= V) {
      E::unpack(any_vector<E>(x + v), xs);
      if (y) E::unpack(any_vector<E>(y + v), ys);
    } else {
#pragma unroll
      for (int i = 0; i < E::N; ++i) {
        xs[i] = v + i < V ? E::up(x[v + i]) : -INFINITY;
        if (y) ys[i] = v + i < V ? E::up(y[v + i]) : -INFINITY;
      }
    }
#pragma unroll
    for (int i = 0; i < E::N; ++i) {
      double p = weight(xs[i], pm, pk) * pw;
      if (y) p -= weight(ys[i], qm, qk) * qw;
      r[i] = p > kNoWeight && v + i != barred ? p : 0.0;
    }
  }
};
template <typename E>
__device__ __forceinline__ Rest<E> rest_of(const VerifyArgs& a, int64_t b, const Verdict& d, bool whole) {
  Rest<E> r;
  r.x = static_cast<const typename E::type*>(a.target) + b * a.target_seq + d.k * a.target_row;
  const bool held = d.refused && !whole;
  r.y = held && a.draft && d.qw > 0.0 ? static_cast<const typename E::type*>(a.draft) + b * a.draft_seq + d.k * a.draft_row : nullptr;
  r.barred = held && !a.draft ? d.token : -1;
  r.V = a.V;
  r.pm = d.pm;
  r.qm = d.qm;
  r.pw = d.pw;
  r.qw = d.qw;
  r.pk = scale_of(a.target_c);
  r.qk = scale_of(a.draft ? a.draft_c : 1.0);
  return r;
}

// A slice of the row that decides: 64 vectors from a whole number of them on, in a wave.
template <typename E>
__host__ __device__ __forceinline__ int slices_of(int V) { return (V + 64 * E::N - 1) / (64 * E::N); }
template <int N>
__device__ __forceinline__ double slice_sum(const double (&w)[N]) {
  double s = w[0];
#pragma unroll
  for (int i = 1; i < N; ++i) s += w[i];
  return wave_sum64(s);
}

// Where in the sums of the slices the drawn token lies, by any wave (the same in each).
struct Place {
  int slice;              // -1: there is no mass
  double before, target;  // what lies ahead of the slice, what the token's sum is to pass
};
__device__ __forceinline__ Place place_of(const double* sums, int slices, float w, double* total, int lane) {
  double all = 0.0;
  for (int s = lane; s < slices; s += 64) all += sums[s];
  all = wave_sum64(all);
  *total = all;
  Place r{-1, 0.0, static_cast<double>(fminf(fmaxf(w, 0.0f), 0x1.fffffep-1f)) * all};
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
  double s = w[0];
#pragma unroll
  for (int i = 1; i < N; ++i) s += w[i];
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
__device__ __forceinline__ void write_drawn(const VerifyArgs& a, int64_t b, const Verdict& d, int token, int lane) {
  if (lane != 0) return;
  const int64_t at = b * (a.n + 1) + d.k;
  a.out[at] = token;
  if (a.logp) a.logp[at] = log_share(E::up((static_cast<const typename E::type*>(a.target) + b * a.target_seq + d.k * a.target_row)[token]), d.pm, d.ps, a.target_c);
}

// Draws for a sequence, by a workgroup that goes through the slices of the row that decides (LDS: slice_sums, again).
template <typename E, int WAVES>
__device__ __forceinline__ void draw(const VerifyArgs& a, int64_t b, const Verdict& d, bool whole, double* slice_sums) {
  const int lane = threadIdx.x & 63, wave = uniform_i(threadIdx.x >> 6), slices = slices_of<E>(a.V);
  const float number = a.numbers[b * (a.n + 1) + a.n];
  for (;; whole = true) {
    const Rest<E> r = rest_of<E>(a, b, d, whole);
    double w[E::N];
    for (int s = wave; s < slices; s += WAVES) {
      r.at((s * 64 + lane) * E::N, w);
      const double v = slice_sum(w);
      if (lane == 0) slice_sums[s] = v;
    }
    __syncthreads();
    double total;
    const Place at = place_of(slice_sums, slices, number, &total, lane);
    if (!whole && !(total > kNothing)) {  // (the same in every wave)
      __syncthreads();
      continue;
    }
    if (at.slice % WAVES == wave) {  // (some slice has mass: the row's largest element does)
      if (slices > WAVES) r.at((at.slice * 64 + lane) * E::N, w);  // (otherwise it is the one that it has)
      write_drawn<E>(a, b, d, find_in_slice(w, at, lane), lane);
    }
    return;
  }
}

// The rest of a sequence, a workgroup each: decides and draws.
template <typename E, int WAVES>
__global__ __launch_bounds__(64 * WAVES) void verify_draw_kernel(VerifyArgs a, int rows, int parts, const Sums* sums) {
  __shared__ RowSums joined;
  __shared__ double slice_sums[kLogitsMaxV / (64 * E::N) + 1];
  const int64_t b = blockIdx.x;
  const Verdict d = decide<E, WAVES>(a, b, sums + b * rows * parts, rows, parts, joined, true);
  if (!d.none) draw<E, WAVES>(a, b, d, !d.refused, slice_sums);
}

// All of a sequence in one workgroup, where its rows have few parts.
constexpr int kSmallItems = 64;
template <typename E, int WAVES, int EACH>
__global__ __launch_bounds__(64 * WAVES) void verify_small_kernel(VerifyArgs a, int rows, int parts) {
  __shared__ RowSums joined;
  __shared__ Sums sums[kSmallItems];
  __shared__ double slice_sums[kSmallItems * EACH + 1];
  const int lane = threadIdx.x & 63, wave = uniform_i(threadIdx.x >> 6);
  const int64_t b = blockIdx.x;
  int count;
  drafted_tokens(a, b, lane, &count);
  for (int item = wave; item < rows * parts; item += WAVES) {
    const int j = item / parts, part = item - j * parts;
    if (j <= a.n ? j > count : j - a.n - 1 >= count) continue;
    const Sums s = part_sums<E, EACH>(row_of<E>(a, b, j), part * 64 * EACH, part == 0, j <= a.n ? a.target_c : a.draft_c, lane);
    if (lane == 0) sums[item] = s;
  }
  __syncthreads();
  const Verdict d = decide<E, WAVES>(a, b, sums, rows, parts, joined, true);
  if (!d.none) draw<E, WAVES>(a, b, d, !d.refused, slice_sums);
}

// Long rows: several workgroups a sequence decide, each for itself, and sum their slices; the first leaves the verdict.
constexpr int kRestWaves = 16;
template <typename E>
__global__ __launch_bounds__(64 * kRestWaves) void verify_rest_kernel(VerifyArgs a, int rows, int parts, const Sums* sums, Verdict* verdicts, double* slice_sums) {
  __shared__ RowSums joined;
  const int lane = threadIdx.x & 63, wave = uniform_i(threadIdx.x >> 6), slices = slices_of<E>(a.V);
  const int64_t b = blockIdx.y;
  const Verdict d = decide<E, kRestWaves>(a, b, sums + b * rows * parts, rows, parts, joined, blockIdx.x == 0);
  if (blockIdx.x == 0 && threadIdx.x == 0) verdicts[b] = d;
  if (d.none) return;
  const Rest<E> r = rest_of<E>(a, b, d, !d.refused);
  for (int s = blockIdx.x * kRestWaves + wave; s < slices; s += gridDim.x * kRestWaves) {
    double w[E::N];
    r.at((s * 64 + lane) * E::N, w);
    const double v = slice_sum(w);
    if (lane == 0) slice_sums[b * slices + s] = v;
  }
}
// And a wave a sequence draws.
template <typename E>
__global__ __launch_bounds__(256) void verify_pick_kernel(VerifyArgs a, const Verdict* verdicts, const double* slice_sums) {
  __shared__ double whole_sums[kLogitsMaxV / (64 * E::N) + 1];
  const int lane = threadIdx.x & 63, wave = uniform_i(threadIdx.x >> 6), slices = slices_of<E>(a.V);
  const int64_t b = blockIdx.x;
  const Verdict d = verdicts[b];
  if (d.none) return;
  double total;
  const Place at = place_of(slice_sums + b * slices, slices, a.numbers[b * (a.n + 1) + a.n], &total, lane);
  if (d.refused && !(total > kNothing)) return draw<E, 4>(a, b, d, true, whole_sums);
  if (wave != 0) return;
  double w[E::N];
  rest_of<E>(a, b, d, !d.refused).at((at.slice * 64 + lane) * E::N, w);
  write_drawn<E>(a, b, d, find_in_slice(w, at, lane), lane);
}

// How a call is laid out.
struct Plan {
  int rows, each, parts;
  int groups;  // workgroups a sequence that sum the row that decides; 0: one workgroup decides and draws; -1: one does everything
  int64_t verdicts, slice_sums, bytes;  // places in the workspace, its size
};
template <typename E>
Plan plan(int32_t sequences, int32_t n, bool drafted, int32_t V) {
  Plan p;
  p.rows = drafted ? 2 * n + 1 : n + 1;
  p.each = 8;
  p.parts = parts_of<E>(V, 8);
  const int slices = slices_of<E>(V);
  if (p.rows * p.parts <= 32 && slices <= 32) {
    p.groups = -1;
    p.verdicts = p.slice_sums = p.bytes = 0;
    return p;
  }
  if (static_cast<int64_t>(sequences) * p.rows * p.parts < 2048) {
    p.each = 2;
    p.parts = parts_of<E>(V, 2);
  }
  p.groups = slices <= 32 ? 0 : static_cast<int>(std::min<int64_t>((slices + kRestWaves - 1) / kRestWaves, std::max<int64_t>(1, 1024 / sequences)));
  p.verdicts = (static_cast<int64_t>(sequences) * p.rows * p.parts * static_cast<int64_t>(sizeof(Sums)) + 15) / 16 * 16;
  p.slice_sums = p.verdicts + (p.groups > 0 ? static_cast<int64_t>(sequences) * static_cast<int64_t>(sizeof(Verdict)) : 0);
  p.bytes = p.slice_sums + (p.groups > 0 ? static_cast<int64_t>(sequences) * slices * 8 : 0);
  return p;
}

template <typename E>
int forward(const VerifyArgs& a, void* workspace, hipStream_t stream) {
  auto done = [] { return hipGetLastError() == hipSuccess ? PB_OK : PB_EHIP; };
  const Plan p = plan<E>(a.sequences, a.n, a.draft != nullptr, a.V);
  if (p.groups < 0) {
    verify_small_kernel<E, 16, 8><<<a.sequences, 1024, 0, stream>>>(a, p.rows, p.parts);
    return done();
  }
  char* ws = static_cast<char*>(workspace);
  Sums* sums = reinterpret_cast<Sums*>(ws);
  const unsigned grid = static_cast<unsigned>((static_cast<int64_t>(a.sequences) * p.rows * p.parts + 3) / 4);
  if (p.each == 2) verify_sums_kernel<E, 2><<<grid, 256, 0, stream>>>(a, p.rows, p.parts, sums);
  else verify_sums_kernel<E, 8><<<grid, 256, 0, stream>>>(a, p.rows, p.parts, sums);
  if (done() != PB_OK) return PB_EHIP;
  if (p.groups == 0) {
    verify_draw_kernel<E, 16><<<a.sequences, 1024, 0, stream>>>(a, p.rows, p.parts, sums);
    return done();
  }
  Verdict* verdicts = reinterpret_cast<Verdict*>(ws + p.verdicts);
  double* slice_sums = reinterpret_cast<double*>(ws + p.slice_sums);
  verify_rest_kernel<E><<<dim3(p.groups, a.sequences), 64 * kRestWaves, 0, stream>>>(a, p.rows, p.parts, sums, verdicts, slice_sums);
  if (done() != PB_OK) return PB_EHIP;
  verify_pick_kernel<E><<<a.sequences, 256, 0, stream>>>(a, verdicts, slice_sums);
  return done();
}

}  // namespace vd

// (Sequences are the second dimension of a grid, which holds 65535 at most.)
int32_t verify_draft_slice(int dtype, int32_t n, int32_t V) {
  const int parts = dtype == PB_F32 ? vd::parts_of<lr::F32>(V, 2) : vd::parts_of<lr::F16>(V, 2);
  return static_cast<int32_t>(std::min<int64_t>(32768, 4 * kMostGroups / ((2 * n + 1) * static_cast<int64_t>(parts))));
}
// (The size is that of the call with rows of the draft, and without them, whichever is larger: it does not depend on them.)
int64_t verify_draft_workspace(int dtype, int32_t sequences, int32_t n, int32_t V) {
  const int32_t some = std::min(sequences, verify_draft_slice(dtype, n, V)), last = sequences % std::max(1, some);
  int64_t most = 0;
  for (const int32_t count : {some, last})
    for (const bool drafted : {false, true})
      if (count > 0) most = std::max(most, (dtype == PB_F32 ? vd::plan<lr::F32>(count, n, drafted, V) : vd::plan<lr::F16>(count, n, drafted, V)).bytes);
  return most;
}
int launch_verify_draft(int dtype, const VerifyArgs& a, void* workspace, hipStream_t stream) {
  return dtype == PB_F32   ? vd::forward<lr::F32>(a, workspace, stream)
         : dtype == PB_F16 ? vd::forward<lr::F16>(a, workspace, stream)
                           : vd::forward<lr::BF16>(a, workspace, stream);
}

}  // namespace pb
