// Log-probs of given tokens, entropy and alternatives of rows of logits, their gradient, and the distillation loss from a
// teacher's alternatives with its gradient: one workgroup per row.
#include <hip/hip_bf16.h>
#include <hip/hip_fp16.h>
#include <hip/hip_runtime.h>

#include <cmath>

#include "pb_kernels.hpp"
#include "pb_logits.hpp"

namespace pb {
namespace {

constexpr int kThreads = 256;
using u64 = unsigned long long;

__device__ __forceinline__ float to_f(float v) { return v; }
__device__ __forceinline__ float to_f(__half v) { return __half2float(v); }
__device__ __forceinline__ float to_f(__hip_bfloat16 v) { return __bfloat162float(v); }
__device__ __forceinline__ void put(float* p, float v) { *p = v; }
__device__ __forceinline__ void put(__half* p, float v) { *p = __float2half(v); }
__device__ __forceinline__ void put(__hip_bfloat16* p, float v) { *p = __float2bfloat16(v); }

template <typename V, typename F>
__device__ V block_reduce(V v, V* lds, F f) {  // (the result in every thread)
  __syncthreads();
  lds[threadIdx.x] = v;
  __syncthreads();
  for (int n = kThreads / 2; n > 0; n >>= 1) {
    if (static_cast<int>(threadIdx.x) < n) lds[threadIdx.x] = f(lds[threadIdx.x], lds[threadIdx.x + n]);
    __syncthreads();
  }
  return lds[0];
}

// Order of the alternatives: value descending (0.0 and -0.0 alike), token ascending.
__device__ __forceinline__ u64 order_key(float x, int v) {
  const int b = __float_as_int(__fadd_rn(x, 0.0f));
  const unsigned k = static_cast<unsigned>(b) ^ (static_cast<unsigned>(b >> 31) | 0x80000000u);
  return (static_cast<u64>(k) << 32) | static_cast<unsigned>(~v);
}

// max x (0 in the place of -inf), sum of exp((x - max) / T) over all tokens, sum of that times (x - max) / T
struct RowSums {
  float m, base, S, E;
};
template <typename T>
__device__ RowSums row_sums(const T* x, int V, float inv, float* lds) {
  RowSums r;
  float m = -INFINITY;
  for (int v = threadIdx.x; v < V; v += kThreads) m = fmaxf(m, to_f(x[v]));
  r.m = block_reduce(m, lds, [](float a, float b) { return fmaxf(a, b); });
  r.base = r.m == -INFINITY ? 0.0f : r.m;
  float S = 0.0f, E = 0.0f;
  for (int v = threadIdx.x; v < V; v += kThreads) {
    const float d = (to_f(x[v]) - r.base) * inv, e = expf(d);
    S += e;
    E += e * fmaxf(d, -1000.0f);
  }
  r.S = block_reduce(S, lds, [](float a, float b) { return a + b; });
  r.E = block_reduce(E, lds, [](float a, float b) { return a + b; });
  return r;
}

template <typename T>
__global__ __launch_bounds__(kThreads) void token_logprobs_kernel(LogprobArgs a) {
  __shared__ float lds[kThreads];
  __shared__ u64 keys[kThreads];
  const int64_t row = blockIdx.x;
  const T* x = static_cast<const T*>(a.in.x) + row * a.in.stride;
  const int V = a.in.V;
  const float inv = a.in.inv_temp;
  const RowSums r = row_sums(x, V, inv, lds);
  const bool empty = r.S == 0.0f, bad = r.S != r.S;
  const float logs = empty ? 0.0f : logf(r.S);
  const float H = bad ? NAN : empty ? 0.0f : logs - r.E / r.S;
  const int tid = threadIdx.x;
  for (int k = tid; k < a.n_tokens; k += kThreads) {
    const int t = a.tokens[row * a.n_tokens + k];
    float lp = NAN;
    if (static_cast<unsigned>(t) < static_cast<unsigned>(V) && !bad) lp = (to_f(x[t]) - r.base) * inv - logs;
    a.logp[row * a.n_tokens + k] = lp;
  }
  if (tid == 0) {
    if (a.entropy) a.entropy[row] = H;
    if (a.stats) {
      a.stats[3 * row + 0] = bad ? NAN : r.m;
      a.stats[3 * row + 1] = bad ? NAN : logs;
      a.stats[3 * row + 2] = H;
    }
  }
  u64 last = ~0ull;
  for (int k = 0; k < a.n_top; ++k) {
    u64 best = 0;
    for (int v = tid; v < V; v += kThreads) {
      const u64 key = order_key(to_f(x[v]), v);
      if (key < last && key > best) best = key;
    }
    best = block_reduce(best, keys, [](u64 p, u64 q) { return p > q ? p : q; });
    last = best;
    if (tid == 0) {
      const int v = bad ? -1 : static_cast<int>(~static_cast<unsigned>(best));
      a.top_tokens[row * a.n_top + k] = v;
      a.top_logp[row * a.n_top + k] = bad ? NAN : (to_f(x[v]) - r.base) * inv - logs;
    }
  }
}

template <typename T>
__global__ __launch_bounds__(kThreads) void logprobs_backward_kernel(LogprobGradArgs a) {
  __shared__ float at[kMaxGiven];
  __shared__ float sum;
  __shared__ int any;
  const int64_t row = blockIdx.x;
  const T* x = static_cast<const T*>(a.in.x) + row * a.in.stride;
  T* out = static_cast<T*>(a.grad) + row * a.grad_stride;
  const int V = a.in.V, tid = threadIdx.x;
  const float inv = a.in.inv_temp;
  const float m = a.stats[3 * row], logs = a.stats[3 * row + 1], H = a.stats[3 * row + 2];
  const float gh = a.grad_entropy ? a.grad_entropy[row] : 0.0f;
  if (tid == 0) {
    float G = 0.0f;
    bool some = gh != 0.0f;
    for (int k = 0; k < a.n_tokens && a.grad_logp; ++k) {
      const unsigned t = a.tokens[row * a.n_tokens + k];
      const float g = a.grad_logp[row * a.n_tokens + k];
      if (t < static_cast<unsigned>(V)) {
        G += g;
        some = some || g != 0.0f;
      }
    }
    sum = G;
    any = some && m != -INFINITY;
  }
  __syncthreads();
  if (!any) {
    for (int v = tid; v < V; v += kThreads) put(out + v, 0.0f);
    return;
  }
  auto pull = [&](float xv) {
    const float lp = (xv - m) * inv - logs;
    return -expf(lp) * (sum + gh * (fmaxf(lp, -1000.0f) + H)) * inv;
  };
  if (tid < a.n_tokens && a.grad_logp) {  // (before anything is written: the gradient may take the logits' place)
    const int t = a.tokens[row * a.n_tokens + tid];
    if (static_cast<unsigned>(t) < static_cast<unsigned>(V)) {
      float g = 0.0f;
      for (int k = 0; k < a.n_tokens; ++k)
        if (a.tokens[row * a.n_tokens + k] == t) g += a.grad_logp[row * a.n_tokens + k];
      at[tid] = pull(to_f(x[t])) + g * inv;
    }
  }
  __syncthreads();
  for (int v = tid; v < V; v += kThreads) put(out + v, pull(to_f(x[v])));
  __syncthreads();
  if (tid < a.n_tokens && a.grad_logp) {
    const int t = a.tokens[row * a.n_tokens + tid];
    if (static_cast<unsigned>(t) < static_cast<unsigned>(V)) put(out + t, at[tid]);
  }
}

template <typename T>
__global__ __launch_bounds__(kThreads) void distill_kernel(DistillArgs a) {
  __shared__ float lds[kThreads];
  __shared__ float at[kMaxGiven], q[kMaxGiven], l[kMaxGiven];
  __shared__ double terms[kMaxGiven];  // (cancel in the sum, and a masked token's log-prob may pass the fp32 range)
  __shared__ int tok[kMaxGiven];
  __shared__ unsigned marks[kLogitsMaxV / 32];
  __shared__ float s_rest;
  __shared__ int s_any;
  const int64_t row = blockIdx.x;
  const T* x = static_cast<const T*>(a.in.x) + row * a.in.stride;
  T* out = a.grad ? static_cast<T*>(a.grad) + row * a.grad_stride : nullptr;
  const int V = a.in.V, tid = threadIdx.x;
  const float inv = a.in.inv_temp;
  const float w = a.row_grads ? a.row_grads[row] : 1.0f;
  if (a.tail)
    for (int i = tid; i < (V + 31) / 32; i += kThreads) marks[i] = 0u;
  if (tid < a.K) {
    tok[tid] = a.tokens[row * a.K + tid];
    const bool there = static_cast<unsigned>(tok[tid]) < static_cast<unsigned>(V);
    if (!there) tok[tid] = -1;
    l[tid] = there ? a.logp[row * a.K + tid] : -INFINITY;
  }
  __syncthreads();
  if (a.tail && tid < a.K && tok[tid] >= 0) atomicOr(&marks[tok[tid] >> 5], 1u << (tok[tid] & 31));
  if (tid == 0) {
    bool any = false;
    float top = -INFINITY;
    for (int k = 0; k < a.K; ++k) {
      any = any || (tok[k] >= 0 && (a.tail || l[k] != -INFINITY));
      top = fmaxf(top, l[k]);
    }
    double sum = 0.0;
    for (int k = 0; k < a.K; ++k) sum += a.tail ? exp(static_cast<double>(l[k])) : exp(static_cast<double>(l[k]) - (any ? top : 0.0f));
    for (int k = 0; k < a.K && !a.tail; ++k) l[k] = l[k] - top - static_cast<float>(log(sum));
    for (int k = 0; k < a.K; ++k) q[k] = tok[k] >= 0 ? expf(l[k]) : 0.0f;
    s_rest = a.tail && 1.0 - sum >= 0x1p-20 ? static_cast<float>(1.0 - sum) : 0.0f;
    s_any = any;
  }
  __syncthreads();
  if (!s_any) {
    if (a.loss && tid == 0) a.loss[row] = 0.0f;
    for (int v = tid; v < V && out; v += kThreads) put(out + v, 0.0f);
    return;
  }
  const RowSums r = row_sums(x, V, inv, lds);
  const bool empty = r.S == 0.0f;
  const float logs = empty ? 0.0f : logf(r.S);
  float p_rest = 0.0f;
  if (a.tail) {
    float S = 0.0f;
    for (int v = tid; v < V; v += kThreads)
      if (!((marks[v >> 5] >> (v & 31)) & 1u)) S += expf((to_f(x[v]) - r.base) * inv);
    p_rest = block_reduce(S, lds, [](float p, float s) { return p + s; }) / (empty ? 1.0f : r.S);
  }
  float Q = s_rest;
  for (int k = 0; k < a.K; ++k) Q += q[k];
  const float share = s_rest > 0.0f && p_rest > 0.0f ? Q - s_rest / p_rest : Q;
  if (tid < a.K && tok[tid] >= 0) {
    const float lp = (to_f(x[tok[tid]]) - r.base) * inv - logs;
    const double exact = (static_cast<double>(to_f(x[tok[tid]])) - r.base) * inv - (empty ? 0.0 : log(static_cast<double>(r.S)));
    terms[tid] = q[tid] > 0.0f ? q[tid] * (l[tid] - exact) : 0.0;
    float mass = 0.0f;
    for (int k = 0; k < a.K; ++k)
      if (tok[k] == tok[tid]) mass += q[k];
    at[tid] = (expf(lp) * Q - mass) * w * inv;
  }
  __syncthreads();
  if (tid == 0 && a.loss) {
    double loss = s_rest > 0.0f ? s_rest * log(static_cast<double>(s_rest) / p_rest) : 0.0;
    for (int k = 0; k < a.K; ++k)
      if (tok[k] >= 0) loss += terms[k];
    a.loss[row] = r.S != r.S ? NAN : static_cast<float>(loss);
  }
  if (!out) return;
  const bool none = empty || w == 0.0f;
  const float scale = w * inv;
  for (int v = tid; v < V; v += kThreads)
    put(out + v, none ? 0.0f : expf((to_f(x[v]) - r.base) * inv - logs) * share * scale);
  __syncthreads();
  if (tid < a.K && tok[tid] >= 0 && !none) put(out + tok[tid], at[tid]);
}

template <template <typename> class Launch, typename Args>
int by_type(int dtype, const Args& a, hipStream_t stream) {
  switch (dtype) {
    case PB_F32: Launch<float>::go(a, stream); break;
    case PB_F16: Launch<__half>::go(a, stream); break;
    default: Launch<__hip_bfloat16>::go(a, stream); break;
  }
  return hipGetLastError() == hipSuccess ? PB_OK : PB_EHIP;
}
template <typename T>
struct Logprobs {
  static void go(const LogprobArgs& a, hipStream_t s) { token_logprobs_kernel<T><<<a.in.rows, kThreads, 0, s>>>(a); }
};
template <typename T>
struct Backward {
  static void go(const LogprobGradArgs& a, hipStream_t s) { logprobs_backward_kernel<T><<<a.in.rows, kThreads, 0, s>>>(a); }
};
template <typename T>
struct Distill {
  static void go(const DistillArgs& a, hipStream_t s) { distill_kernel<T><<<a.in.rows, kThreads, 0, s>>>(a); }
};

}  // namespace

int launch_token_logprobs(int dtype, const LogprobArgs& a, hipStream_t stream) { return by_type<Logprobs>(dtype, a, stream); }
int launch_token_logprobs_backward(int dtype, const LogprobGradArgs& a, hipStream_t stream) { return by_type<Backward>(dtype, a, stream); }
int launch_distill_topk(int dtype, const DistillArgs& a, hipStream_t stream) { return by_type<Distill>(dtype, a, stream); }

}  // namespace pb
