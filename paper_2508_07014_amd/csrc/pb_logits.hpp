// Log-probs, entropy and alternatives of rows of logits, and distillation from a teacher's alternatives: arguments of the
// calls as the kernels get them, and the launch wrappers (pb_logprobs.hip, pb_distill.hip).
#pragma once
#include <hip/hip_runtime.h>

#include <cstdint>

#include "pb.h"

namespace pb {

constexpr int kLogitsMaxV = 3 << 17;   // widest row: a bit per token fits in 64 KiB of LDS with room to spare
constexpr int kMaxGiven = 64;          // tokens scored, alternatives kept or teacher's entries a row: one lane each

struct LogitRows {
  const void* x;       // [rows, stride], enum pb_dtype
  int64_t stride;      // in elements
  int32_t rows, V;
  int32_t all_rows;    // of the call, of which these are a slice: what decides whether rows are split
  float inv_temp;      // 1 / T
  float c;             // log2(e) / T
  float far;           // logits below -far are masks: see kFar
};
// Where a wave's largest element m lies further than kFar / c from 0, |m c| > kFar, x c is too coarse for the differences between
// elements, and its sums are formed from (x - m) c instead.  Other waves leave out the elements below -far, masks of a lowest
// value.  Those lie as far again below the line, so that beside any m above it they are nothing (2^-kFar of its term).
constexpr float kFar = 1048576.0f;
inline LogitRows logit_rows(const void* x, int64_t stride, int32_t rows, int32_t V, float temperature) {
  const double c = 1.44269504088896340736 / temperature;
  return LogitRows{x, stride, rows, V, rows, static_cast<float>(1.0 / temperature), static_cast<float>(c), static_cast<float>(2 * kFar / c)};
}

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

// Few long rows are split over the chip: `parts` waves a row, each with 64 * `each` vectors of 16 bytes (0: not split).
// At most kMaxParts, so that one wave can join them; at least `few`; and about kSplitWaves in all.
constexpr int kWaveVectors = 512;  // longest row that one wave takes, in vectors
constexpr int kMaxParts = 256, kSplitWaves = 4096;
constexpr int kMaxEach = 8;  // (the marks of a part's listed tokens lie in LDS)
static_assert(kMaxEach * 64 * kMaxParts >= kLogitsMaxV / 4, "the widest row is split");
struct RowSplit {
  int parts, each;
};
inline RowSplit row_split(int vectors, int32_t rows, int few) {
  const int least = (vectors + 64 * kMaxParts - 1) / (64 * kMaxParts), most = vectors / (64 * few) < kMaxEach ? vectors / (64 * few) : kMaxEach;
  const int64_t want = static_cast<int64_t>(rows) * vectors / (64 * kSplitWaves);
  const int each = static_cast<int>(want < least ? least : want > most ? (most > least ? most : least) : want);
  return RowSplit{(vectors + 64 * each - 1) / (64 * each), each};
}

// Which calls are split.  us, split / a workgroup a row.  Log-probs with entropy and 5 alternatives, bf16: V = 80000, 1 row 7.6 / 9.3, 12
// rows 8.3 / 9.7, 32 rows 9.7 / 9.9; V = 131072, 1 row 8.0 / 12.2, 72 rows 12.5 / 13.4, 120 rows 15.3 / 13.7; V = 250000, 1 row 8.3 / 19.8,
// 138 rows 21.5 / 22.4; V = 393216, 120 rows 25.7 / 34.8, 218 rows 39.4 / 38.0.  fp32: V = 80000, 1 row 7.7 / 10.0, 32 rows 9.8 / 11.6; V =
// 131072, 72 rows 14.7 / 16.2, 120 rows 18.2 / 17.0; V = 250000, 138 rows 31.7 / 37.6; V = 393216, 218 rows 64.0 / 62.9.  Without
// alternatives, bf16: V = 80000, 32 rows 6.9 / 7.7; V = 131072, 72 rows 9.0 / 10.8, 120 rows 11.4 / 11.2.  So the line (12 rows at V = 80000, 72
// at 131072, 138 at 250000, 218 at 393216) lies within 4 % of where both are equal or on the side of one workgroup a row; short of
// it, V = 80000 with 13 to 32 rows, a split would be 2 to 15 % faster.  At V = 50000 it was slower (bf16 1 row 8.6 / 8.1, 32 rows 9.5 / 8.5; fp32
// 16 rows 9.4 / 8.9).
// Distillation, 32 entries and the rest, bf16: V = 32001, 16 rows 8.9 / 9.2, 40 rows 9.5 / 9.5, 64 rows 10.3 / 9.6; V = 50000, 32 rows 10.0 /
// 11.7, 62 rows 12.0 / 11.9, 100 rows 12.8 / 12.5; V = 131072, 64 rows 14.9 / 24.1, 160 rows 25.4 / 26.5, 200 rows 30.0 / 30.1.  fp32: V =
// 131072, 64 rows 19.0 / 33.6, 327 rows 84.8 / 123; on the short side the line is drawn for 16 bits, and a workgroup a row would be
// faster: V = 16001, 40 rows 9.1 / 7.5; V = 32001, 16 rows 9.4 / 9.1, 80 rows 12.1 / 10.7.
inline RowSplit split_logprobs(int vectors, int32_t rows, int32_t V) {
  return rows <= (V - 70000) / 800 && rows <= V / 1800 ? row_split(vectors, rows, 80) : RowSplit{0, 0};  // (the parts are to bound 64 alternatives)
}
static_assert(70000 / 8 >= 80 * 64, "rows that are split have 80 parts of 64 vectors");
inline RowSplit split_distill(int vectors, int32_t rows) {
  return vectors >= 3500 && rows <= vectors / 100 ? row_split(vectors, rows, 16) : RowSplit{0, 0};
}

int64_t token_logprobs_workspace(int dtype, int32_t rows, int32_t V);
int64_t distill_topk_workspace(int dtype, int32_t rows, int32_t V);
int launch_token_logprobs(int dtype, const LogprobArgs& a, void* workspace, hipStream_t stream);
int launch_token_logprobs_backward(int dtype, const LogprobGradArgs& a, hipStream_t stream);
int launch_distill_topk(int dtype, const DistillArgs& a, void* workspace, hipStream_t stream);

}  // namespace pb
