// Token scores: what the kernel is given.
#pragma once
#include <cuda_runtime.h>
#include <stddef.h>
#include <stdint.h>

namespace icc {

constexpr int SCORE_MAX_TOP = 32;
constexpr int SCORE_MAX_SPLIT = 32;       // pieces of a row
constexpr int SCORE_SLOTS = 1024;         // partial results, and rows that are split, of a launch

// What one CTA knows of its piece of a row: largest logit m, sum of 2^d and of 2^d d with d = (x - m) scale log2(e), and the best keys.
struct ScorePartial {
  float top, sum, weighted, unused;
  uint64_t keys[SCORE_MAX_TOP];
};

struct ScoreParams {
  const unsigned char* logits;
  int64_t row_stride;       // elements
  int64_t n_rows;
  const int* targets;
  float* log_probs;
  float* entropy;
  int* top_ids;
  float* top_log_probs;
  int vocab, n_top, split;  // pieces of a row
  float scale, scale_log2;  // scale_log2 = scale * log2(e)
  ScorePartial* partials;   // [rows, split] where split > 1
  int* arrivals;            // [rows]: pieces that have arrived, zero between launches
  int* host_status;         // mapped host word
};

// dtype: 0 bf16, 1 fp16, 2 fp32
cudaError_t score_launch(ScoreParams p, int dtype, int sm_count, cudaStream_t st);

}  // namespace icc
