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
  static __device__ __forceinline__ v4u nothing() { return v4u{0xff800000u, 0xff800000u, 0xff800000u, 0xff800000u}; }  // -inf throughout
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
  static __device__ __forceinline__ v4u nothing() { return v4u{0xfc00fc00u, 0xfc00fc00u, 0xfc00fc00u, 0xfc00fc00u}; }  // -inf throughout
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
  static __device__ __forceinline__ v4u nothing() { return v4u{0xff80ff80u, 0xff80ff80u, 0xff80ff80u, 0xff80ff80u}; }  // -inf throughout
  static __device__ __forceinline__ v4u pack(const float (&x)[N]) {
    v4u r;
#pragma unroll
    for (int i = 0; i < 4; ++i) r[i] = __builtin_bit_cast(unsigned, __builtin_convertvector((v2f{x[2 * i], x[2 * i + 1]}), v2b));
    return r;
  }
  static __device__ __forceinline__ __bf16 down(float v) { return static_cast<__bf16>(v); }
};

// A row of V elements at any alignment: the elements before the first boundary and the fewer than N behind the last vector
// (the edge, one lane each), `nv` aligned vectors between them.  Nothing outside the row is touched.
template <typename E>
struct Row {
  const typename E::type* x;
  const v4u* body;
  int V, head, nv, edges;
  __device__ __forceinline__ v4u vec(int v) const {  // (a 32-bit offset from a uniform base)
    return *reinterpret_cast<const v4u*>(reinterpret_cast<const char*>(body) + static_cast<unsigned>(v) * 16u);
  }
  template <bool STREAM>
  __device__ __forceinline__ v4u vec_once(int v) const {  // (STREAM: past the caches)
    if constexpr (!STREAM) return vec(v);
    return __builtin_nontemporal_load(reinterpret_cast<const v4u*>(reinterpret_cast<const char*>(body) + static_cast<unsigned>(v) * 16u));
  }
  __device__ __forceinline__ int edge_token(int t) const { return t + (t >= head ? nv * E::N : 0); }
  __device__ __forceinline__ int token(int v, int i) const { return head + v * E::N + i; }
};
// ALIGN: the boundary that the vectors begin at, 16, or 64, so that a wave's stores fill whole cache lines but for the first
// and last (odd rows of bf16 in one pass over 2 x 500 MB: 192 -> 188 us; the longer edge costs short rows 5 %).
template <typename E, unsigned ALIGN = 16>
__device__ __forceinline__ Row<E> row_at(const void* base, int64_t stride, int64_t row, int V) {
  Row<E> r;
  r.x = static_cast<const typename E::type*>(base) + row * stride;
  r.V = V;
  r.head = min(V, static_cast<int>((0u - static_cast<unsigned>(reinterpret_cast<uintptr_t>(r.x))) & (ALIGN - 1u)) / static_cast<int>(sizeof(typename E::type)));
  r.nv = (V - r.head) / E::N;
  r.edges = V - r.nv * E::N;
  r.body = reinterpret_cast<const v4u*>(r.x + r.head);
  return r;
}

__device__ __forceinline__ float exp2_fast(float v) { return __builtin_amdgcn_exp2f(v); }

// Sum over a wave, in lane 63 of the last step and from there in every lane.  (row_bcast:15 adds a row's sum to the next row's,
// row_bcast:31 that of the first two to the others': what rows 0 to 2 are left with is not used.  Lanes without a source add 0 by
// bound_ctrl, so the additions take the moves along.)
template <int CTRL>
__device__ __forceinline__ float dpp_add(float v) {
  return v + __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), CTRL, 0xf, 0xf, true));
}
__device__ __forceinline__ float wave_sum(float v) {
  v = dpp_add<0x111>(v);
  v = dpp_add<0x112>(v);
  v = dpp_add<0x114>(v);
  v = dpp_add<0x118>(v);
  v = dpp_add<0x142>(v);
  v = dpp_add<0x143>(v);
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

// 16 bytes to any element of a row, and the same past the caches.
template <typename E>
__device__ __forceinline__ void stream_vector(typename E::type* p, const v4u& r) {
  __builtin_nontemporal_store(r, reinterpret_cast<typename E::any4*>(p));
}
template <typename E>
__device__ __forceinline__ void store_vector(typename E::type* p, const v4u& r) {
  *reinterpret_cast<typename E::any4*>(p) = r;
}

// The larger of three (a NaN is passed over, as by fmaxf, which would first quiet each operand by an instruction of its own).
__device__ __forceinline__ float max3(float a, float b, float c) {
  float r;
  asm("v_max3_f32 %0, %1, %2, %3" : "=v"(r) : "v"(a), "v"(b), "v"(c));
  return r;
}
template <int N>
__device__ __forceinline__ float vec_max(const float (&x)[N]) {
  if constexpr (N == 1) return x[0];
  float m = max3(x[0], x[1], x[2]);
#pragma unroll
  for (int i = 3; i + 1 < N; i += 2) m = max3(m, x[i], x[i + 1]);
  if constexpr (N % 2 == 0) m = max3(m, x[N - 1], x[N - 1]);
  return m;
}
// a b, and 0 where a is 0 and b is infinite (or NaN, which the sums of a find anyway).
__device__ __forceinline__ float mul_0(float a, float b) {
  float r;
  asm("v_mul_legacy_f32 %0, %1, %2" : "=v"(r) : "v"(a), "v"(b));
  return r;
}
// log(1 + r), r > -1/2: the logarithm of u = 1 + r, rounded, by what u lacks of r (Kahan); of u = 2^k m, m in [sqrt(1/2), sqrt(2)),
// k ln 2 + log m, so that what the hardware's log is off by counts relative to log m (64 rows of 50000: log-probs off by up to
// 5.2e-8 of themselves without, 3.5e-8 with it, in the same time).
__device__ __forceinline__ float log_1p(float r) {
  const float u = 1.0f + r, d = u - 1.0f;
  const int k = (static_cast<int>(__float_as_uint(u)) - 0x3f3504f3) >> 23;
  const float m = __uint_as_float(__float_as_uint(u) - (static_cast<unsigned>(k) << 23));
  const float l = __builtin_fmaf(static_cast<float>(k), kLn2, __builtin_amdgcn_logf(m) * kLn2);  // (the hardware's has base 2)
  return d == 0.0f ? r : fabsf(d) < 0.5f ? l * (r * __builtin_amdgcn_rcpf(d)) : l;
}
template <int N>
__device__ __forceinline__ float vec_sum(float (&x)[N]) {  // (in pairs: fewer roundings in a row)
#pragma unroll
  for (int n = N / 2; n > 0; n /= 2)
#pragma unroll
    for (int i = 0; i < n; ++i) x[i] += x[i + n];
  return x[0];
}

}  // namespace lr
}  // namespace pb
