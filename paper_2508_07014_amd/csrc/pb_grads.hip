// The norm over all gradients of a model and their clipping (pb_grad_norm, pb_grad_clip).
//
// A set of tensors is a table of pieces of at most kChunk elements on the device; workgroups take them in turn.  Squares are exact in
// 64 bits and summed there: no scale of gradients overflows or vanishes.
#include "pb_logit_rows.hpp"
#include "pb_student.hpp"

namespace pb {
namespace gr {

using namespace lr;

constexpr int kGroups = 2048;  // workgroups at most: eight a CU
// Sets that do not fit in the last cache (256 MB) are read past it, both times: 800 MB of bf16 norm 135 -> 120 us, clipping 295 -> 282; 200
// MB, which fits, both 99 -> 96 us the other way.
constexpr int64_t kStreamBytes = 256ll << 20;
constexpr int kAhead = 8;      // vectors that a lane requests at once: a piece of kChunk 16-bit elements in one turn

template <int WAVES>
__device__ __forceinline__ double block_sum(double v, double (&shared)[WAVES]) {
#pragma unroll
  for (int d = 1; d < 64; d *= 2) v += __shfl_xor(v, d, 64);
  if ((threadIdx.x & 63) == 0) shared[threadIdx.x >> 6] = v;
  __syncthreads();
  v = 0.0;
  for (int w = 0; w < WAVES; ++w) v += shared[w];
  return v;
}

// Of a piece, the thread's own share of THREADS.
template <typename E, bool STREAM, int THREADS>
__device__ __forceinline__ double squares(const GradChunk& c, int tid) {
  const Row<E> row = row_at<E>(c.x, 0, 0, c.n);
  double s[4] = {0.0, 0.0, 0.0, 0.0};
  auto add = [&](const v4u& raw) {
    float x[E::N];
    E::unpack(raw, x);
#pragma unroll
    for (int i = 0; i < E::N; ++i) s[i % 4] = fma(static_cast<double>(x[i]), static_cast<double>(x[i]), s[i % 4]);
  };
  if (tid < row.edges) {
    const double x = E::up(row.x[row.edge_token(tid)]);
    s[0] = x * x;
  }
  int v = tid;
  for (; v + THREADS * (kAhead - 1) < row.nv; v += THREADS * kAhead) {
    v4u raw[kAhead];
#pragma unroll
    for (int k = 0; k < kAhead; ++k) raw[k] = row.template vec_once<STREAM>(v + THREADS * k);
#pragma unroll
    for (int k = 0; k < kAhead; ++k) add(raw[k]);
  }
  for (; v < row.nv; v += THREADS) add(row.vec(v));
  return (s[0] + s[1]) + (s[2] + s[3]);
}

template <bool STREAM, int THREADS>
__device__ __forceinline__ double squares_of(const GradChunk& c, int tid) {
  return c.dtype == PB_F32   ? squares<F32, STREAM, THREADS>(c, tid)
         : c.dtype == PB_F16 ? squares<F16, STREAM, THREADS>(c, tid)
                             : squares<BF16, STREAM, THREADS>(c, tid);
}

// Bound by HBM (800 MB of bf16: 120 us, 6.7 TB/s); small sets by the launch and three reads one after the other (8 MB of fp32: 3.8 us).
template <bool STREAM>
__global__ __launch_bounds__(256) void grad_squares_kernel(const GradChunk* chunks, int64_t n, double* sums) {
  __shared__ double shared[4];
  double s = 0.0;
  for (int64_t c = blockIdx.x; c < n; c += gridDim.x) {
    s += squares_of<STREAM, 256>(chunks[c], threadIdx.x);
  }
  s = block_sum<4>(s, shared);
  if (threadIdx.x == 0) sums[blockIdx.x] = s;
}
__global__ __launch_bounds__(1024) void grad_norm_kernel(const double* sums, int n, float* norm) {
  __shared__ double shared[16];
  static_assert(kGroups <= 2048, "two a thread");
  double s = static_cast<int>(threadIdx.x) < n ? sums[threadIdx.x] : 0.0;
  if (static_cast<int>(threadIdx.x) + 1024 < n) s += sums[threadIdx.x + 1024];
  s = block_sum<16>(s, shared);
  if (threadIdx.x == 0) *norm = static_cast<float>(sqrt(s));
}
// A set of few pieces, which are small then, in one launch: a wave a piece (us, one launch / two: 5 tensors of 300 bf16 2.5 / 5.7, 16 of 2000 3.4 /
// 6.0, 60 of 1000 4.7 / 5.6, 60 of 2000 6.4 / 6.0; with the clipping behind it 6.5 / 10.0, 7.2 / 9.6, 7.7 / 10.0, 9.1 / 10.0).
constexpr int kFewPieces = 64;
__global__ __launch_bounds__(1024) void grad_norm_small_kernel(const GradChunk* chunks, int n, float* norm) {
  __shared__ double shared[16];
  const int wave = threadIdx.x >> 6;
  GradChunk mine[kFewPieces / 16];
#pragma unroll
  for (int k = 0; k < kFewPieces / 16; ++k) mine[k] = wave + 16 * k < n ? chunks[wave + 16 * k] : GradChunk{nullptr, 0, PB_F32};
  double s = 0.0;
#pragma unroll
  for (int k = 0; k < kFewPieces / 16; ++k)
    if (mine[k].n > 0) s += squares_of<false, 64>(mine[k], threadIdx.x & 63);
  s = block_sum<16>(s, shared);
  if (threadIdx.x == 0) *norm = static_cast<float>(sqrt(s));
}

template <typename E, bool STREAM>
__device__ __forceinline__ void scaled(const GradChunk& c, const GradChunk& out, float by) {
  const Row<E> row = row_at<E>(c.x, 0, 0, c.n);
  typename E::type* to = static_cast<typename E::type*>(out.x);
  auto put = [&](int v, const v4u& raw) {
    float x[E::N];
    E::unpack(raw, x);
#pragma unroll
    for (int i = 0; i < E::N; ++i) x[i] = product(x[i], by);
    stream_vector<E>(to + row.token(v, 0), E::pack(x));
  };
  if (static_cast<int>(threadIdx.x) < row.edges) {
    const int i = row.edge_token(threadIdx.x);
    to[i] = E::down(product(E::up(row.x[i]), by));
  }
  int v = threadIdx.x;
  for (; v + 256 * (kAhead - 1) < row.nv; v += 256 * kAhead) {
    v4u raw[kAhead];
#pragma unroll
    for (int k = 0; k < kAhead; ++k) raw[k] = row.template vec_once<STREAM>(v + 256 * k);
#pragma unroll
    for (int k = 0; k < kAhead; ++k) put(v + 256 * k, raw[k]);
  }
  for (; v < row.nv; v += 256) put(v, row.vec(v));
}

// (A norm that is not finite clips nothing: there is no factor for it.)  A workgroup takes the pieces that it has taken for the norm, from
// the last to the first: the last ones are those that the norm has left in the caches, in that of its own part of the chip.  Bound by HBM (800 MB of
// bf16 into as many: 282 us, 5.7 TB/s).
template <bool STREAM>
__global__ __launch_bounds__(256) void grad_clip_kernel(const GradChunk* chunks, const GradChunk* out, int64_t n, const float* norm, float max_norm) {
  const float is = *norm;
  const bool clips = is > max_norm && is < INFINITY;
  const float by = clips ? max_norm / is : 1.0f;
  if (!clips && out == chunks) return;
  const int64_t grid = gridDim.x, full = grid < kGroups ? 0 : n / kGroups * kGroups;  // (a smaller grid has a piece for each workgroup)
  for (int64_t c = blockIdx.x + (full + blockIdx.x < n ? full : full - grid); c >= 0; c -= grid) {
    const GradChunk from = chunks[c], to = out[c];
    if (from.dtype == PB_F32) scaled<F32, STREAM>(from, to, by);
    else if (from.dtype == PB_F16) scaled<F16, STREAM>(from, to, by);
    else scaled<BF16, STREAM>(from, to, by);
  }
}

int groups_for(int64_t chunks) { return static_cast<int>(chunks < kGroups ? chunks : kGroups); }

}  // namespace gr

int64_t grad_norm_workspace(int64_t chunks) { return gr::groups_for(chunks) * 8; }
int launch_grad_norm(const GradChunk* chunks, int64_t n, int64_t bytes, float* norm, void* workspace, hipStream_t stream) {
  double* sums = static_cast<double*>(workspace);
  const int groups = gr::groups_for(n);
  if (n <= gr::kFewPieces) {
    gr::grad_norm_small_kernel<<<1, 1024, 0, stream>>>(chunks, groups, norm);
    return hipGetLastError() == hipSuccess ? PB_OK : PB_EHIP;
  }
  if (bytes > gr::kStreamBytes) gr::grad_squares_kernel<true><<<groups, 256, 0, stream>>>(chunks, n, sums);
  else gr::grad_squares_kernel<false><<<groups, 256, 0, stream>>>(chunks, n, sums);
  if (hipGetLastError() != hipSuccess) return PB_EHIP;
  gr::grad_norm_kernel<<<1, 1024, 0, stream>>>(sums, groups, norm);
  return hipGetLastError() == hipSuccess ? PB_OK : PB_EHIP;
}
int launch_grad_clip(const GradChunk* chunks, const GradChunk* out, int64_t n, int64_t bytes, const float* norm, float max_norm, hipStream_t stream) {
  if (n == 0) return PB_OK;
  const int groups = gr::groups_for(n);
  if (bytes > gr::kStreamBytes) gr::grad_clip_kernel<true><<<groups, 256, 0, stream>>>(chunks, out, n, norm, max_norm);
  else gr::grad_clip_kernel<false><<<groups, 256, 0, stream>>>(chunks, out, n, norm, max_norm);
  return hipGetLastError() == hipSuccess ? PB_OK : PB_EHIP;
}

}  // namespace pb
