// Distributions cut by top-k, top-p and min-p: tokens drawn from them, scores without what is cut off (ad_truncate.hip).
#pragma once

#include "ad_internal.h"

namespace ad {

struct TruncateArgs {
  const void* x;                 // scores [rows, vocab], rows `stride` elements apart
  size_t stride;
  int vocab, n_seq, rows;
  const int* row_start;          // [n_seq + 1]; null: sequence b is row b
  const float* temperature;      // [n_seq] each; null: 1, not cut
  const int* top_k;
  const float *top_p, *min_p;
  const float* u;                // drawn: [rows], and where the tokens and their logarithms of probabilities (null: not wanted) go
  int* tokens;
  float* log_probs;
  void* out;                     // truncated: scores [rows, vocab] of the same type, rows out_stride apart
  size_t out_stride;
};
void launch_sample(int dtype, const TruncateArgs& a, hipStream_t s);
void launch_truncate(int dtype, const TruncateArgs& a, hipStream_t s);

}  // namespace ad
