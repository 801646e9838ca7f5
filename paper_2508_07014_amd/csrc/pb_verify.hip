// Verification of drafted tokens (pb_verify_draft): which of them a target's rows accept, and the token drawn behind them.
//
//   p_i = softmax(x_i / T), q_i = softmax(y_i / T') (or 1 at t_i): t_i is accepted where those before it are and u_i q_i(t_i) < p_i(t_i);
//   behind the k accepted ones a token is drawn from max(p_k - q_k, 0), or from p_k where no drafted token was refused: the first
//   v whose sum over all tokens up to it exceeds w times the sum over all.
//
// A drawn token is a border between two of V sums: with sums in fp32, off by 1e-7 of the whole, one draw in a hundred from a
// row of 131072 tokens would be another token than the definition's.  So exponentials and sums are in 64 bits throughout, which
// the chip's vector units take at the rate of fp32.
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

constexpr int kEach = 8;                     // vectors of a lane in a part of a row
constexpr double kNothing = 0x1p-40;         // a rest of the target's mass below this is none (equal rows differ by their roundings)

// 2^t for t <= 0: 1 + r P(r), |r| <= 1/2, P by interpolation at Chebyshev's nodes, 6e-16 of the value.  Past 2^-1074: 0.
__device__ __forceinline__ double exp2_64(double t) {
  t = fmax(t, -1100.0);
  const double n = rint(t), r = t - n;
  double p = 0x1.e5e9f548e5725p-28;
  p = fma(p, r, 0x1.b6571de2f2351p-24);
  p = fma(p, r, 0x1.62bfe46117445p-20);
  p = fma(p, r, 0x1.ffcb76789860fp-17);
  p = fma(p, r, 0x1.4309130378460p-13);
  p = fma(p, r, 0x1.5d87fe908f88ap-10);
  p = fma(p, r, 0x1.3b2ab6fba385fp-7);
  p = fma(p, r, 0x1.c6b08d7044119p-5);
  p = fma(p, r, 0x1.ebfbdff82c590p-3);
  p = fma(p, r, 0x1.62e42fefa39f7p-1);
  p = fma(p, r, 1.0);
  return ldexp(p, static_cast<int>(n));
}

// Sum over a wave, the same bits in every lane.
__device__ __forceinline__ double wave_sum64(double v) {
#pragma unroll
  for (int d = 1; d < 64; d *= 2) v += __shfl_xor(v, d, 64);
  return v;
}
// Sums over the lanes up to each.
__device__ __forceinline__ double wave_upto64(double v, int lane) {
#pragma unroll
  for (int d = 1; d < 64; d *= 2) {
    const double w = __shfl_up(v, d, 64);
    if (lane >= d) v += w;
  }
  return v;
}
__device__ __forceinline__ double readlane64(double v, int lane) {
  const int lo = __builtin_amdgcn_readlane(__double2loint(v), lane), hi = __builtin_amdgcn_readlane(__double2hiint(v), lane);
  return __hiloint2double(hi, lo);
}

// What element x has beside m.
__device__ __forceinline__ double weight(float x, float m, double c) {
  return exp2_64((static_cast<double>(x) - static_cast<double>(m)) * c);
}

// Part of a row, by a wave: vectors first .. first + 64 kEach - 1, and the row's edge where `edge`.
template <typename E>
__device__ __forceinline__ Sums part_sums(const Row<E>& row, int first, bool edge, double c, int lane) {
  v4u raw[kEach];
  float m = -INFINITY, xe = -INFINITY;
#pragma unroll
  for (int u = 0; u < kEach; ++u) {
    const int v = first + 64 * u + lane;
    raw[u] = v < row.nv ? row.vec(v) : E::nothing();
  }
  if (edge && lane < row.edges) xe = E::up(row.x[row.edge_token(lane)]);
  bool bad = xe != xe;
  m = fmaxf(m, xe);
#pragma unroll
  for (int u = 0; u < kEach; ++u) {
    float x[E::N];
    E::unpack(raw[u], x);
#pragma unroll
    for (int i = 0; i < E::N; i += 2) bad |= __builtin_isunordered(x[i], x[i + 1]);
    m = fmaxf(m, vec_max(x));
  }
  m = wave_max(m);
  bad = __ballot(bad) != 0 || m == INFINITY;
  if (m == -INFINITY || bad) return Sums{m, bad, 0.0};
  double s = weight(xe, m, c);
#pragma unroll
  for (int u = 0; u < kEach; ++u) {
    if (first + 64 * u >= row.nv) break;
    float x[E::N];
    E::unpack(raw[u], x);
#pragma unroll
    for (int i = 0; i < E::N; ++i) s += weight(x[i], m, c);
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
__device__ __forceinline__ int drafted(const VerifyArgs& a, int64_t b, int lane, int* count) {
  const int t = lane < a.n ? a.tokens[b * a.n + lane] : -1;
  const u64 none = ~__ballot(static_cast<unsigned>(t) < static_cast<unsigned>(a.V));
  *count = none ? first_lane(none) : 64;  // (n <= 63: lane 63 holds none)
  return t;
}

// A wave a part of a row.  Rows behind the end of a draft are not looked at.
template <typename E>
__global__ __launch_bounds__(256) void verify_sums_kernel(VerifyArgs a, int rows, int parts, Sums* sums) {
  const int lane = threadIdx.x & 63;
  const int64_t item = static_cast<int64_t>(blockIdx.x) * 4 + uniform_i(threadIdx.x >> 6);
  if (item >= static_cast<int64_t>(a.sequences) * rows * parts) return;
  const int part = static_cast<int>(item % parts), j = static_cast<int>(item / parts % rows);
  const int64_t b = item / parts / rows;
  int count;
  drafted(a, b, lane, &count);
  if (j <= a.n ? j > count : j - a.n - 1 >= count) return;
  const Row<E> row = row_of<E>(a, b, j);
  const Sums s = part_sums<E>(row, part * 64 * kEach, part == 0, j <= a.n ? a.target_c : a.draft_c, lane);
  if (lane == 0) sums[item] = s;
}

// What is decided from the sums of a sequence's rows.
struct Verdict {
  int k;           // accepted tokens
  int marked;      // the row that decides holds a NaN or +inf
  int refused;     // a drafted token was refused: the draft's row counts
  int token;       // that one
  float pm, qm;    // of the rows that decide
  double pw, qw;   // 1 / their sums; 0 for a row of nothing but -inf
  double log2_p;   // log2 of the target's sum
};

template <int ROWS>
struct RowSums {
  float m[ROWS];
  double s[ROWS];
};

// Joins the parts of all rows (waves of the workgroup take turns), then decides, the same in every wave.  Writes the accepted tokens
// if `writes`, in the first wave.
template <typename E, int WAVES>
__device__ __forceinline__ Verdict decide(const VerifyArgs& a, int64_t b, const Sums* sums, int rows, int parts, RowSums<2 * kMaxDrafts + 1>& joined,
                                          bool writes) {
  const int lane = threadIdx.x & 63, wave = uniform_i(threadIdx.x >> 6);
  int count;
  const int t = drafted(a, b, lane, &count);
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
      for (int p = lane; p < parts; p += 64) s += sums[j * parts + p].s * weight(sums[j * parts + p].m, m, c);
    s = wave_sum64(s);
    if (__ballot(bad) != 0) s = NAN;
    if (lane == 0) {
      joined.m[j] = m;
      joined.s[j] = s;
    }
  }
  __syncthreads();
  const bool mine = lane < count;
  bool takes = false;
  if (mine) {
    const float pm = joined.m[lane];
    const double ps = joined.s[lane];
    const double p = pm == -INFINITY ? ps : weight(xt, pm, a.target_c) / ps;  // (ps: 0, or NaN)
    double q = 1.0;
    if (a.draft) {
      const float qm = joined.m[a.n + 1 + lane];
      const double qs = joined.s[a.n + 1 + lane];
      q = qm == -INFINITY ? qs : weight(yt, qm, a.draft_c) / qs;
    }
    takes = static_cast<double>(u) * q < p;  // (false for NaN)
  }
  Verdict r;
  r.k = first_lane(~__ballot(takes));  // (lane 63 takes none)
  r.refused = r.k < count;
  r.token = __builtin_amdgcn_readlane(t, r.k);
  r.pm = joined.m[r.k];
  const double ps = joined.s[r.k];
  r.pw = r.pm == -INFINITY ? 0.0 : 1.0 / ps;
  r.log2_p = log2(ps);
  r.qm = -INFINITY;
  r.qw = 0.0;
  r.marked = ps != ps;
  if (r.refused && a.draft) {
    const double qs = joined.s[a.n + 1 + r.k];
    r.qm = joined.m[a.n + 1 + r.k];
    r.qw = r.qm == -INFINITY ? 0.0 : 1.0 / qs;
    r.marked |= qs != qs;
  }
  if (writes && wave == 0 && lane <= a.n && lane != r.k) {  // (the token at k is drawn later)
    a.out[b * (a.n + 1) + lane] = lane < r.k ? t : -1;
    if (a.logp) {
      float l = NAN;
      if (lane < r.k)
        l = static_cast<float>(((static_cast<double>(xt) - static_cast<double>(joined.m[lane])) * a.target_c - log2(joined.s[lane])) * 0.69314718055994530942);
      a.logp[b * (a.n + 1) + lane] = l;
    }
  }
  if (writes && wave == 0 && lane == 0) a.accepted[b] = r.k;
  return r;
}

// The row that decides, as what a token may be drawn from: max(p - q, 0), or p where `whole`.
template <typename E>
struct Rest {
  const typename E::type* x;
  const typename E::type* y;  // null: no draft's row counts
  int V, barred;              // the token that a draft without rows was sure of, -1: none
  float pm, qm;
  double pw, qw, pc, qc;
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
      double p = weight(xs[i], pm, pc) * pw;
      if (y) p -= weight(ys[i], qm, qc) * qw;
      r[i] = p > 0.0 && v + i != barred ? p : 0.0;
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
  r.pm = d.pm == -INFINITY ? 0.0f : d.pm;  // (pw is 0 then)
  r.qm = d.qm;
  r.pw = d.pw;
  r.qw = d.qw;
  r.pc = a.target_c;
  r.qc = a.draft_c;
  return r;
}

// A slice of the row that decides: 64 vectors, in a wave.
template <typename E>
__device__ __forceinline__ double slice_sum(const Rest<E>& r, int slice, int lane) {
  double w[E::N], s = 0.0;
  r.at((slice * 64 + lane) * E::N, w);
#pragma unroll
  for (int i = 0; i < E::N; ++i) s += w[i];
  return wave_sum64(s);
}
template <typename E>
__host__ __device__ __forceinline__ int slices_of(int V) { return (V + 64 * E::N - 1) / (64 * E::N); }

// The token within a slice, by a wave: the first one up to which the sum passes `target` with `before` ahead of the slice; the
// last one with any mass where roundings leave none.
template <typename E>
__device__ __forceinline__ int find_in_slice(const Rest<E>& r, int slice, double before, double target, int lane) {
  double w[E::N], s = 0.0;
  const int v = (slice * 64 + lane) * E::N;
  r.at(v, w);
  int any = -1;
#pragma unroll
  for (int i = 0; i < E::N; ++i) {
    s += w[i];
    any = w[i] > 0.0 ? v + i : any;
  }
  double upto = before + (wave_upto64(s, lane) - s);
  int found = -1;
#pragma unroll
  for (int i = 0; i < E::N; ++i) {
    upto += w[i];
    found = found < 0 && w[i] > 0.0 && upto > target ? v + i : found;
  }
  const u64 has = __ballot(found >= 0), some = __ballot(any >= 0);
  if (has) return __builtin_amdgcn_readlane(found, first_lane(has));
  return some ? __builtin_amdgcn_readlane(any, 63 - __builtin_clzll(some)) : -1;
}

// By one wave from the slices' sums: the drawn token, or -1 where there is no mass.  *total: of all slices.
template <typename E>
__device__ __forceinline__ int draw(const Rest<E>& r, const double* sums, int slices, double w, double* total, int lane) {
  double all = 0.0;
  for (int s = lane; s < slices; s += 64) all += sums[s];
  all = wave_sum64(all);
  *total = all;
  if (!(all > 0.0)) return -1;
  const double target = w * all;
  double before = 0.0, ahead = 0.0;
  int slice = -1, last = -1;
  for (int s0 = 0; s0 < slices && slice < 0; s0 += 64) {
    const double mine = s0 + lane < slices ? sums[s0 + lane] : 0.0;
    const double upto = ahead + wave_upto64(mine, lane);
    const u64 has = __ballot(mine > 0.0 && upto > target), some = __ballot(mine > 0.0);
    if (some) {
      last = s0 + 63 - __builtin_clzll(some);
      before = readlane64(upto - mine, 63 - __builtin_clzll(some));
    }
    if (has) {
      slice = s0 + first_lane(has);
      before = readlane64(upto - mine, first_lane(has));
    }
    ahead = readlane64(upto, 63);
  }
  return find_in_slice(r, slice >= 0 ? slice : last, before, target, lane);
}

template <typename E>
__device__ __forceinline__ void write_drawn(const VerifyArgs& a, int64_t b, const Verdict& d, int token, int lane) {
  if (lane != 0) return;
  const int64_t at = b * (a.n + 1) + d.k;
  a.out[at] = token;
  if (!a.logp) return;
  float l = NAN;
  if (token >= 0) {
    const float x = E::up((static_cast<const typename E::type*>(a.target) + b * a.target_seq + d.k * a.target_row)[token]);
    l = static_cast<float>(((static_cast<double>(x) - static_cast<double>(d.pm)) * a.target_c - d.log2_p) * 0.69314718055994530942);
  }
  a.logp[at] = l;
}

// The rest of a sequence, a workgroup each: decides, sums the row that decides slice by slice, draws.
template <typename E, int WAVES>
__global__ __launch_bounds__(64 * WAVES) void verify_draw_kernel(VerifyArgs a, int rows, int parts, const Sums* sums) {
  __shared__ RowSums<2 * kMaxDrafts + 1> joined;
  __shared__ double slice_sums[kLogitsMaxV / (64 * E::N) + 1];
  __shared__ int again;
  const int lane = threadIdx.x & 63, wave = uniform_i(threadIdx.x >> 6);
  const int64_t b = blockIdx.x;
  const Verdict d = decide<E, WAVES>(a, b, sums + b * rows * parts, rows, parts, joined, true);
  if (d.marked) {
    if (wave == 0) write_drawn<E>(a, b, d, -1, lane);
    return;
  }
  const int slices = slices_of<E>(a.V);
  for (bool whole = !d.refused;; whole = true) {
    const Rest<E> r = rest_of<E>(a, b, d, whole);
    for (int s = wave; s < slices; s += WAVES) {
      const double v = slice_sum<E>(r, s, lane);
      if (lane == 0) slice_sums[s] = v;
    }
    __syncthreads();
    if (wave == 0) {
      double total;
      const float w = fminf(fmaxf(a.numbers[b * (a.n + 1) + a.n], 0.0f), 0x1.fffffep-1f);
      const int token = draw<E>(r, slice_sums, slices, static_cast<double>(w), &total, lane);
      const bool redo = !whole && !(total > kNothing);
      if (!redo) write_drawn<E>(a, b, d, token, lane);
      if (lane == 0) again = redo;
    }
    __syncthreads();
    if (!again) break;
  }
}

template <typename E>
int forward(const VerifyArgs& a, void* workspace, hipStream_t stream) {
  const int rows = a.draft ? 2 * a.n + 1 : a.n + 1;
  const int parts = (a.V / E::N + 64 * kEach - 1) / (64 * kEach) + (a.V / E::N == 0);
  Sums* sums = static_cast<Sums*>(workspace);
  const int64_t waves = static_cast<int64_t>(a.sequences) * rows * parts;
  verify_sums_kernel<E><<<static_cast<unsigned>((waves + 3) / 4), 256, 0, stream>>>(a, rows, parts, sums);
  if (hipGetLastError() != hipSuccess) return PB_EHIP;
  verify_draw_kernel<E, 16><<<a.sequences, 1024, 0, stream>>>(a, rows, parts, sums);
  return hipGetLastError() == hipSuccess ? PB_OK : PB_EHIP;
}

}  // namespace vd

static int verify_parts(int dtype, int32_t V) {
  const int nv = V / (dtype == PB_F32 ? lr::F32::N : lr::F16::N);
  return (nv + 64 * vd::kEach - 1) / (64 * vd::kEach) + (nv == 0);
}
int32_t verify_draft_slice(int dtype, int32_t n, int32_t V) {
  return static_cast<int32_t>(4 * kMostGroups / ((2 * n + 1) * static_cast<int64_t>(verify_parts(dtype, V))));
}
int64_t verify_draft_workspace(int dtype, int32_t sequences, int32_t n, int32_t V) {
  const int32_t most = verify_draft_slice(dtype, n, V);
  return static_cast<int64_t>(sequences < most ? sequences : most) * (2 * n + 1) * verify_parts(dtype, V) * static_cast<int64_t>(sizeof(vd::Sums));
}
int launch_verify_draft(int dtype, const VerifyArgs& a, void* workspace, hipStream_t stream) {
  return dtype == PB_F32   ? vd::forward<lr::F32>(a, workspace, stream)
         : dtype == PB_F16 ? vd::forward<lr::F16>(a, workspace, stream)
                           : vd::forward<lr::BF16>(a, workspace, stream);
}

}  // namespace pb
