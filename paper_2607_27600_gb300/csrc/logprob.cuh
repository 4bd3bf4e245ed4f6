// logprob.cuh -- interface of the token log-probability kernel.
#pragma once
#include "cc_common.cuh"

namespace cc {

constexpr int kMaxTop = 32;   // alternatives of a row at most: one per lane

struct LogprobParams {
  const void *logits;        // [rows][vocab], rows ld elements apart
  int dtype;                 // cc_dtype
  int rows, vocab;
  long long ld;
  const int32_t *targets;    // device [rows], or null
  float *logprob, *entropy;  // device [rows], or null
  int top;                   // 0 .. kMaxTop, at most vocab
  int32_t *top_ids;          // device [rows][top], or null
  float *top_logprob;
  unsigned *status;
};

cudaError_t launch_token_logprobs(const LogprobParams &p, int sms, cudaStream_t st);

}  // namespace cc
