// A student of the teacher whose alternatives pb_distill_topk learns from: rows of its table for tokens and their gradient
// (pb_embed.hip), the norm over all gradients and their clipping (pb_grads.hip), and the verification of what it drafts
// (pb_verify.hip).  Arguments of the calls as the kernels get them, and the launch wrappers.
#pragma once
#include <hip/hip_runtime.h>

#include <cstdint>
#include <vector>

#include "pb.h"
#include "pb_logits.hpp"

namespace pb {

// A product that is rounded to fp32 by itself: the compiler would fold it into the conversion to fp16 behind it in some places and
// not in others, and a row's bits would depend on the length of the row.
__device__ __forceinline__ float product(float a, float b) {
  float r = a * b;
  asm("" : "+v"(r));
  return r;
}

constexpr int kMaxDrafts = 63;             // drafted tokens a sequence: with the row behind them a lane each
constexpr int kMostTokens = 1 << 24;       // looked up in a call
constexpr int kMostDim = 1 << 16;          // columns of a table
constexpr int64_t kMostGroups = 1 << 22;   // workgroups a launch (its threads are counted in 32 bits); more go out in slices

struct VerifyArgs {
  const void* target;  // [sequences, n + 1] rows
  const void* draft;   // [sequences, n] rows; null: the draft was sure of its tokens
  int64_t target_seq, target_row, draft_seq, draft_row;  // strides in elements
  int32_t sequences, n, V;
  struct Scale {
    double c, low;  // log2(e) / T, and the difference below which weights do not go (2^-1000)
  } target_scale, draft_scale;
  const int32_t* tokens;     // [sequences, n]
  const float* numbers;      // [sequences, n + 1]
  int32_t* out;              // [sequences, n + 1]
  int32_t* accepted;         // [sequences]
  float* logp;               // [sequences, n + 1]; null: not wanted
};
int64_t verify_draft_workspace(int dtype, int32_t sequences, int32_t n, int32_t V);
int32_t verify_draft_slice(int dtype, int32_t n, int32_t V);  // sequences a launch at most
int launch_verify_draft(int dtype, const VerifyArgs& a, void* workspace, hipStream_t stream);

struct EmbedArgs {
  const void* table;
  int64_t table_stride;
  int32_t V, dim;
  float scale;
  const int32_t* tokens;
  int32_t n;
  void* out;
  int64_t out_stride;
};
int launch_embed_tokens(int table_dtype, int out_dtype, const EmbedArgs& a, hipStream_t stream);

struct EmbedGradArgs {
  const void* grad;  // [n, dim] on the rows that were looked up
  int64_t grad_stride;
  const int32_t* tokens;
  int32_t n, V, dim;
  float scale;
  int32_t accumulate;
  void* table_grad;  // [V, dim]
  int64_t table_stride;
};
int64_t embed_tokens_backward_workspace(int32_t n, int32_t V, int32_t dim);
int launch_embed_tokens_backward(int grad_dtype, int table_dtype, const EmbedGradArgs& a, void* workspace, hipStream_t stream);

// A set of tensors as the kernels see it: pieces of at most kChunk elements, fewer in small sets (which are to fill the chip), in the
// order of the tensors.
constexpr int64_t kMostElements = 1ll << 40;
constexpr int kChunk = 16384, kLeastChunk = 2048;
inline int64_t chunk_for(int64_t elements) {
  const int64_t even = (elements / 2048 + kLeastChunk - 1) / kLeastChunk * kLeastChunk;
  return even < kLeastChunk ? kLeastChunk : even < kChunk ? even : kChunk;
}
struct GradChunk {
  void* x;
  int32_t n;
  int32_t dtype;
};
int64_t grad_norm_workspace(int64_t chunks);
int launch_grad_norm(const GradChunk* chunks, int64_t n, int64_t bytes, float* norm, void* workspace, hipStream_t stream);
int launch_grad_clip(const GradChunk* chunks, const GradChunk* out, int64_t n, int64_t bytes, const float* norm, float max_norm, hipStream_t stream);

}  // namespace pb

struct pb_tensors {
  pb::GradChunk* d_chunks = nullptr;
  int64_t count = 0;  // pieces
  int64_t bytes = 0;  // of the tensors
  int device = -1;
  std::vector<int64_t> sizes;
  std::vector<int32_t> dtypes;
  struct Span {
    uintptr_t begin, end;
    int32_t tensor;  // -1: several that share memory
  };
  std::vector<Span> spans;  // by address, apart from each other
  bool shares = false;      // whether any of them is of several tensors
};
