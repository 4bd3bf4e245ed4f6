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
  float kappa, kappa_lo;        // scale_log2 sqrt(head_dim) as two fp32
  float *acc;                   // [batch][cap]
  unsigned *status;
  // set by kv_received_plan
  int heads_at_once;            // KV heads of a pass over a share's slots
  int tiles_at_once;            // eights of query rows of a KV head in a pass
  int shares;                   // CTAs
  int resident;                 // of them on an SM
  // chunks (set by launch_kv_received_tiles)
  int P;                        // positions of a query tile
  float *part;                  // [hkv][batch][cap][2]: the sums of whole units, over half of the rows each
  float *cut;                   // [2 * shares][256][2]: of a share's pieces of units
};

CC_DEV float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// A row's lse in the scores' log2 domain.  Rounded to fp32 it would cost the weights what it
// drops (4e-6 of them at a score of 60), so y is the rounded part and `rest` what it leaves, in
// natural units; and the log2(e) in it is the one in scale_log2 as that was rounded, so that
// the two roundings cancel.  Not finite: y = +inf, the row adds nothing.
struct RowLse {
  float y, rest;
};
CC_DEV RowLse row_lse(const KvReceivedParams &p, float lse) {
  const float y = lse * p.kappa;
  if (!(fabsf(y) < INFINITY)) return {INFINITY, 0.f};
  return {y, 0.69314718055994531f * fmaf(lse, p.kappa_lo, fmaf(lse, p.kappa, -y))};
}

void kv_received_plan(KvReceivedParams &p, int sms);
cudaError_t launch_kv_received(const KvReceivedParams &p, cudaStream_t st);

// Chunks: tiles of up to 96 query rows, kv_received_positions consecutive ones of a KV head's
// heads.  tq: q as [n_rows][hq][head_dim], box {64, heads of a KV head, positions}.
constexpr int kReceivedMaxGroup = 96;   // heads of a KV head
int kv_received_positions(int group);
size_t kv_received_part_bytes(const KvReceivedParams &p, int sms);
cudaError_t launch_kv_received_tiles(KvReceivedParams p, const CUtensorMap &tq, void *ws, int sms, cudaStream_t st);

}  // namespace cc
