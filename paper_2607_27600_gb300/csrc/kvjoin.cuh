// kvjoin.cuh -- interface of the join of attention over disjoint slots.
#pragma once
#include "cc_common.cuh"

namespace cc {

constexpr int kMaxJoinParts = 16;

struct KvJoinParams {
  int n_rows, hq, head_dim, n_parts;
  int dtype;                          // cc_dtype of the parts and of out
  const void *part[kMaxJoinParts];    // [n_rows][hq * head_dim], rows part_ld elements apart
  long long part_ld[kMaxJoinParts];
  const float *part_lse[kMaxJoinParts];   // [n_rows][hq]
  void *out;
  long long out_ld;
  float *lse;                         // [n_rows][hq], or null
};

cudaError_t launch_kv_join(const KvJoinParams &p, cudaStream_t st);

}  // namespace cc
