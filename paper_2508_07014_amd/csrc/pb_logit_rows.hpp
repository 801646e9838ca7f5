// Device helpers of the kernels on rows of logits (gfx950, wave64): a row as aligned 16-byte vectors, sums of exponentials in
// one pass, the tokens on a row.
#pragma once
#include <hip/hip_runtime.h>

#include <climits>
#include <cmath>
#include <cstdint>

#include "pb_logits.hpp"
#include "pb_wave.hpp"

namespace pb {
namespace lr {

using wv::u64;
using wv::ukey;
using wv::ukey_val;
using wv::uniform_f;
using wv::uniform_i;

typedef unsigned v4u __attribute__((ext_vector_type(4)));
typedef float v2f __attribute__((ext_vector_type(2)));
typedef _Float16 v2h __attribute__((ext_vector_type(2)));
typedef __bf16 v2b __attribute__((ext_vector_type(2)));

constexpr float kLog2e = 1.44269504088896340736f, kLn2 = 0.69314718055994530942f;

// Element types: N of them in a 16-byte vector, to and from fp32 (one rounding, to nearest even).
struct F32 {
  typedef float type;
  typedef unsigned any4 __attribute__((ext_vector_type(4), aligned(4)));  // 16 bytes at any element
  static constexpr int N = 4;
  static __device__ __forceinline__ float up(float v) { return v; }
  static __device__ __forceinline__ void unpack(const v4u& r, float (&x)[N]) {
#pragma unroll
    for (int i = 0; i < N; ++i) x[i] = __uint_as_float(r[i]);
  }
  static __device__ __forceinline__ v4u pack(const float (&x)[N]) {
    v4u r;
#pragma unroll
    for (int i = 0; i < N; ++i) r[i] = __float_as_uint(x[i]);
    return r;
  }
  static __device__ __forceinline__ float down(float v) { return v; }
};
struct F16 {
  typedef _Float16 type;
  typedef unsigned any4 __attribute__((ext_vector_type(4), aligned(2)));
  static constexpr int N = 8;
  static __device__ __forceinline__ float up(_Float16 v) { return static_cast<float>(v); }
  static __device__ __forceinline__ void unpack(const v4u& r, float (&x)[N]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const unsigned w = r[i];
      const v2h h = __builtin_bit_cast(v2h, w);
      x[2 * i] = static_cast<float>(h.x);
      x[2 * i + 1] = static_cast<float>(h.y);
    }
  }
  static __device__ __forceinline__ v4u pack(const float (&x)[N]) {
    v4u r;
#pragma unroll
    for (int i = 0; i < 4; ++i) r[i] = __builtin_bit_cast(unsigned, v2h{static_cast<_Float16>(x[2 * i]), static_cast<_Float16>(x[2 * i + 1])});
    return r;
  }
  static __device__ __forceinline__ _Float16 down(float v) { return static_cast<_Float16>(v); }
};
struct BF16 {
  typedef __bf16 type;
  typedef unsigned any4 __attribute__((ext_vector_type(4), aligned(2)));
  static constexpr int N = 8;
  static __device__ __forceinline__ float up(__bf16 v) { return static_cast<float>(v); }
  static __device__ __forceinline__ void unpack(const v4u& r, float (&x)[N]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      x[2 * i] = __uint_as_float(r[i] << 16);
      x[2 * i + 1] = __uint_as_float(r[i] & 0xffff0000u);
    }
  }
  static __device__ __forceinline__ v4u pack(const float (&x)[N]) {
    v4u r;
#pragma unroll
    for (int i = 0; i < 4; ++i) r[i] = __builtin_bit_cast(unsigned, __builtin_convertvector((v2f{x[2 * i], x[2 * i + 1]}), v2b));
    return r;
  }
  static __device__ __forceinline__ __bf16 down(float v) { return static_cast<__bf16>(v); }
};

// A row of V elements at any alignment: up to N - 1 elements before the first 16-byte boundary and as many behind the last
// one (the edge, one lane each), `nv` aligned vectors between them.  Nothing outside the row is touched.
template <typename E>
struct Row {
  const typename E::type* x;
  const v4u* body;
  int V, head, nv, edges;
  __device__ __forceinline__ v4u vec(int v) const {  // (a 32-bit offset from a uniform base)
    return *reinterpret_cast<const v4u*>(reinterpret_cast<const char*>(body) + static_cast<unsigned>(v) * 16u);
  }
  __device__ __forceinline__ int edge_token(int t) const { return t + (t >= head ? nv * E::N : 0); }
  __device__ __forceinline__ int token(int v, int i) const { return head + v * E::N + i; }
};
template <typename E>
__device__ __forceinline__ Row<E> row_at(const void* base, int64_t stride, int64_t row, int V) {
  Row<E> r;
  r.x = static_cast<const typename E::type*>(base) + row * stride;
  r.V = V;
  r.head = min(V, static_cast<int>((0u - static_cast<unsigned>(reinterpret_cast<uintptr_t>(r.x))) & 15u) / static_cast<int>(sizeof(typename E::type)));
  r.nv = (V - r.head) / E::N;
  r.edges = V - r.nv * E::N;
  r.body = reinterpret_cast<const v4u*>(r.x + r.head);
  return r;
}

__device__ __forceinline__ float exp2_fast(float v) { return __builtin_amdgcn_exp2f(v); }

template <int CTRL>
__device__ __forceinline__ float dpp_f(float v, float none) {
  return __int_as_float(__builtin_amdgcn_update_dpp(__float_as_int(none), __float_as_int(v), CTRL, 0xf, 0xf, false));
}
__device__ __forceinline__ float wave_sum(float v) {
  v += dpp_f<0x111>(v, 0.0f);
  v += dpp_f<0x112>(v, 0.0f);
  v += dpp_f<0x114>(v, 0.0f);
  v += dpp_f<0x118>(v, 0.0f);
  // (row_bcast writes rows 1 and 3, then 2 and 3, alone: the other rows add their `none`)
  v += __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), 0x142, 0xa, 0xf, false));
  v += __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), 0x143, 0xc, 0xf, false));
  return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), 63));
}
__device__ __forceinline__ float wave_max(float v) { return ukey_val(wv::wave_max_u(ukey(v))); }

// Waves of one row that wait for each other: a workgroup, or one wave of it.
template <int NT>
__device__ __forceinline__ void row_sync() {
  if constexpr (NT == 64) {
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
  } else {
    __syncthreads();
  }
}

// 16 bytes to any element of a row.
template <typename E>
__device__ __forceinline__ void store_vector(typename E::type* p, const v4u& r) {
  *reinterpret_cast<typename E::any4*>(p) = r;
}

// max and sums of exponentials in one pass.  With c = log2(e) / T every term is e = exp2(d), d = x c - rc; the reference rc
// is the lane's own and is moved, with the sums, only when an element exceeds it by more than 2^kRoom: the first vector
// sets it, after that a lane hardly ever comes back (one fused multiply-add and one exponential a term, no running maximum
// in the chain).  d is rounded once; what rc itself was rounded by is the same for all terms of the lane, and is made up for
// at the end (row_sums).  Elements below -kFar / c are masks of a lowest value: nothing beside any ordinary logit.  A row whose
// maximum lies beyond +-kFar / c is summed again from differences (row_sums).
// A second sum goes along: of e d (for the entropy), or of the terms of listed tokens, which the first one then lacks.
constexpr float kRoom = 30.0f, kFar = 1048576.0f;
enum Second : int { kAlone = 0, kEntropy = 1, kListed = 2 };

// (S, X) seen from a reference that lies `apart` = rc - new rc higher.
template <int SECOND>
__device__ __forceinline__ void rebase(float& S, float& X, float apart) {
  const float f = exp2_fast(apart);  // (may be infinite where the sums are 0)
  if constexpr (SECOND == kEntropy) X = S == 0.0f ? 0.0f : f * __builtin_fmaf(apart, S, X);
  if constexpr (SECOND == kListed) X = X == 0.0f ? 0.0f : f * X;
  S = S == 0.0f ? 0.0f : f * S;
}
struct Sums {
  float rc = 0.0f, thr, S = 0.0f, X = 0.0f, m = -INFINITY;
  __device__ __forceinline__ explicit Sums(float far) : thr(-far) {}
};
template <int N>
__device__ __forceinline__ float vec_max(const float (&x)[N]) {
  if constexpr (N == 1) return x[0];
  float m = x[0];
#pragma unroll
  for (int i = 1; i + 1 < N; i += 2) m = fmaxf(fmaxf(m, x[i]), x[i + 1]);
  if constexpr (N % 2 == 0) m = fmaxf(m, x[N - 1]);
  return m;
}
// A vector into the sums; `vm` its largest element, `listed` a bit per element that goes to the second sum (kListed).
template <int SECOND, int N>
__device__ __forceinline__ void add_vector(Sums& s, const float (&x)[N], float vm, float c, float room, unsigned listed = 0u) {
  if (__ballot(vm > s.thr) != 0) {  // (of the wave: a branch, not selects in every vector)
    if (vm > s.thr) {
      const float next = vm * c;
      rebase<SECOND>(s.S, s.X, s.rc - next);
      s.rc = next;
      s.thr = vm + room;
    }
  }
  if (SECOND == kListed && listed != 0u) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const float e = exp2_fast(__builtin_fmaf(x[i], c, -s.rc));
      const bool on = (listed >> i) & 1u;
      s.S += on ? 0.0f : e;
      s.X += on ? e : 0.0f;
    }
    return;
  }
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const float d = __builtin_fmaf(x[i], c, -s.rc), e = exp2_fast(d);
    s.S += e;
    if constexpr (SECOND == kEntropy) s.X = __builtin_fmaf(e, fmaxf(d, -1000.0f), s.X);  // (-inf: nothing)
  }
}

// Sums of a part of a row, seen from its maximum: d = (x - m) c.  A part of nothing but -inf has sums of 0.
struct Part {
  float m, S, X;
};
// The part of a wave from its lanes', the same in every lane.  again(add) goes over the wave's elements a second time, with
// add(x, listed): where the maximum lies so far from 0 that x c and m c no longer resolve what is between them, the
// difference does.
template <int SECOND, typename Again>
__device__ __forceinline__ Part wave_part(const Sums& s, float c, Again&& again) {
  Part p{wave_max(s.m), s.S, s.X};
  const float mc = p.m * c;
  rebase<SECOND>(p.S, p.X, s.rc - mc);
  p.S = wave_sum(p.S);
  if constexpr (SECOND != kAlone) p.X = wave_sum(p.X);
  rebase<SECOND>(p.S, p.X, -__builtin_fmaf(p.m, c, -mc));  // (from the rounded m c to m c)
  if (!(fabsf(mc) <= kFar) && fabsf(p.m) != INFINITY) {
    float S = 0.0f, X = 0.0f;
    again([&](float x, bool on) {
      const float d = (x - p.m) * c, e = exp2_fast(d);
      S += SECOND == kListed && on ? 0.0f : e;
      if constexpr (SECOND == kEntropy) X = __builtin_fmaf(e, fmaxf(d, -1000.0f), X);
      if constexpr (SECOND == kListed) X += on ? e : 0.0f;
    });
    p.S = wave_sum(S);
    if constexpr (SECOND != kAlone) p.X = wave_sum(X);
  }
  return p;
}
template <int SECOND>
__device__ __forceinline__ Part see_from(Part p, float m, float c) {
  rebase<SECOND>(p.S, p.X, (p.m - m) * c);
  p.m = m;
  return p;
}
// Two parts, or the parts that the lanes of a wave hold, as one.
template <int SECOND>
__device__ __forceinline__ Part join(const Part& p, const Part& q, float c) {
  const float m = fmaxf(p.m, q.m);
  const Part a = see_from<SECOND>(p, m, c), b = see_from<SECOND>(q, m, c);
  return Part{m, a.S + b.S, a.X + b.X};
}
template <int SECOND>
__device__ __forceinline__ Part join_lanes(const Part& p, float c) {
  const Part q = see_from<SECOND>(p, wave_max(p.m), c);
  return Part{q.m, wave_sum(q.S), SECOND != kAlone ? wave_sum(q.X) : 0.0f};
}

struct RowSums {  // the same in every thread of the row
  float m;        // maximum, -inf for a row of nothing but -inf
  float base;     // m, 0 for such a row
  float S, X;     // the sums, d = (x - base) c
  bool bad;       // the row holds a NaN or +inf
};
// The row from its waves' parts (`lds`: 3 * NT / 64 floats).
template <int NT, int SECOND>
__device__ __forceinline__ RowSums join_waves(Part p, int tid, float c, float* lds) {
  constexpr int W = NT / 64;
  if constexpr (W > 1) {
    if ((tid & 63) == 0) {
      lds[tid >> 6] = p.m;
      lds[W + (tid >> 6)] = p.S;
      lds[2 * W + (tid >> 6)] = p.X;
    }
    __syncthreads();
    float M = lds[0], S = 0.0f, X = 0.0f;
#pragma unroll
    for (int w = 1; w < W; ++w) M = fmaxf(M, lds[w]);
#pragma unroll
    for (int w = 0; w < W; ++w) {
      const Part q = see_from<SECOND>(Part{lds[w], lds[W + w], lds[2 * W + w]}, M, c);
      S += q.S;
      X += q.X;
    }
    p = Part{uniform_f(M), uniform_f(S), uniform_f(X)};
  }
  RowSums r{p.m, p.m == -INFINITY ? 0.0f : p.m, p.S, p.X, false};
  r.bad = r.S != r.S || r.X != r.X || r.m == INFINITY;
  return r;
}

}  // namespace lr
}  // namespace pb
