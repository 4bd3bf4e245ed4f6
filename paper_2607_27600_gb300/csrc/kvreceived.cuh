// kvreceived.cuh -- interface of the attention that cached slots receive.
#pragma once
#include "rows.cuh"

namespace cc {

struct KvReceivedParams {
  StepRows rows;
  int memory_only, first;
  int f16;                      // q is fp16 (else bf16)
  const void *q;
  long long q_ld;               // elements between rows
  const float *lse;             // [n_rows][hq]
  const uint8_t *k, *ke;
  int block;                    // slots per scale
  KvLayout pg;
  int hq, hkv, head_dim;
  float scale_log2;             // log2(e) / sqrt(head_dim)
  float *acc;                   // [batch][cap]
  unsigned *status;
  // set by kv_received_plan
  int heads_at_once;            // KV heads of a pass over a share's slots
  int tiles_at_once;            // eights of query rows of a KV head in a pass
  int shares;                   // CTAs
};

void kv_received_plan(KvReceivedParams &p, int sms);
cudaError_t launch_kv_received(const KvReceivedParams &p, cudaStream_t st);

}  // namespace cc
