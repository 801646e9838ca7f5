// Log-probs, entropy and alternatives of rows of logits, and distillation from a teacher's alternatives: arguments of the
// calls as the kernels get them, and the launch wrappers (pb_logits.hip).
#pragma once
#include <hip/hip_runtime.h>

#include <cstdint>

#include "pb.h"

namespace pb {

constexpr int kLogitsMaxV = 1 << 19;   // widest row: a bit per token fits in LDS
constexpr int kMaxGiven = 64;          // tokens scored, alternatives kept or teacher's entries a row: one lane each

struct LogitRows {
  const void* x;       // [rows, stride], enum pb_dtype
  int64_t stride;      // in elements
  int32_t rows, V;
  float inv_temp;
};

struct LogprobArgs {
  LogitRows in;
  const int32_t* tokens;  // [rows, n_tokens]
  int32_t n_tokens, n_top;
  float* logp;            // each may be null
  float* entropy;
  int32_t* top_tokens;
  float* top_logp;
  float* stats;
};

struct LogprobGradArgs {
  LogitRows in;
  const float* stats;
  const int32_t* tokens;
  int32_t n_tokens;
  const float* grad_logp;     // [rows, n_tokens]; null: none
  const float* grad_entropy;  // [rows]; null: none
  void* grad;
  int64_t grad_stride;
};

struct DistillArgs {
  LogitRows in;
  const int32_t* tokens;  // [rows, K]
  const float* logp;      // [rows, K]
  int32_t K, tail;
  const float* row_grads;  // null: 1
  float* loss;             // null: not wanted
  void* grad;              // null: not wanted
  int64_t grad_stride;
};

int launch_token_logprobs(int dtype, const LogprobArgs& a, hipStream_t stream);
int launch_token_logprobs_backward(int dtype, const LogprobGradArgs& a, hipStream_t stream);
int launch_distill_topk(int dtype, const DistillArgs& a, hipStream_t stream);

}  // namespace pb
