// kvattn.cuh -- interface of the attention over a block-scaled 8-bit cache.
#pragma once
#include "rows.cuh"

namespace cc {

struct KvAttnParams {
  StepRows rows;
  int memory_only;
  int f16;                      // q and out are fp16 (else bf16)
  const void *q;
  void *out;
  long long q_ld, out_ld;       // elements between rows
  float *lse;                   // [n_rows][hq], or null
  const uint8_t *k, *v, *ke, *ve;
  int block;                    // slots per scale
  KvLayout pg;
  int hq, hkv, head_dim;
  float scale_log2;             // log2(e) / sqrt(head_dim)
  // set by kv_attn_plan
  int nt;                       // query rows of a unit / 8: 1, 2 or 4
  int ctas;                     // CTAs that share the units' key tiles
  float *part_o;                // [2 * ctas][8 * nt][head_dim]: what a CTA leaves of the unit
  float4 *part_ml;              // [2 * ctas][8 * nt]            before and after its share
  unsigned *status;
};

// Rows of a unit and CTAs of a launch: p.nt and p.ctas from rows.max_rows and
// the head counts.
void kv_attn_plan(KvAttnParams &p, int sms);
size_t kv_attn_part_bytes(const KvAttnParams &p);
cudaError_t launch_kv_attn(const KvAttnParams &p, cudaStream_t st);

// The seen slots of one layer as a bf16 slot-major copy (exact) in rows
// b * cap + i of ko, vo, and the ends seq_len + rows (memory_only: seq_len) of
// the sequences in `ends`; a sequence without rows is not copied.
cudaError_t launch_kv_block_copy(const KvAttnParams &p, void *ko, void *vo, int32_t *ends,
                                 cudaStream_t st);

}  // namespace cc
