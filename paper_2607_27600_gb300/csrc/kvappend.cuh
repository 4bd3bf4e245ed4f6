// kvappend.cuh -- interface of the cache-writing kernels of a serving step.
#pragma once
#include "rows.cuh"

namespace cc {

struct KvAppendParams {
  StepRows rows;
  const int32_t *pos;        // device [n_rows], or nullptr: those following the cache's
  const int32_t *cache_pos;  // device [batch][cap] (read where pos is null)
  const void *k, *v, *q;     // rows of hkv (hq) heads of head_dim; q may be null
  void *q_out;
  long long k_ld, v_ld, q_ld, q_out_ld;   // elements between rows
  int dtype;                 // cc_dtype of k, v, q, q_out
  void *kc, *vc;             // cache buffers of the layer
  uint8_t *ke, *ve;          // block format: scale exponents
  int format;                // cc_kv_format
  int block;                 // slots per scale (block format), else slots per unit of work
  float k_qscale, v_qscale;  // CC_KV_E4M3: 1 / scale
  KvLayout pg;
  int hq, hkv, head_dim;
  int rotate;
  unsigned long long turns[64];   // RoPE: inv_freq / (2 pi), 0.64 fixed point
  unsigned *status;
};

cudaError_t launch_kv_append(const KvAppendParams &p, int sms, cudaStream_t st);
// Positions and token ids (tokens may be null) of the rows into the cache, then
// seq_len grows.
cudaError_t launch_kv_advance(const StepRows &rows, const int32_t *pos, const int32_t *tokens,
                              int32_t *seq_len, int32_t *cache_tokens, int32_t *cache_pos,
                              unsigned *status, cudaStream_t st);

}  // namespace cc
