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
  long long exp_bytes;          // bytes of ke (and of ve)
  KvLayout pg;
  int hq, hkv, head_dim;
  float scale_log2;             // log2(e) / sqrt(head_dim)
  // set by kv_attn_plan
  int nt;                       // query rows of a unit / 8: 1 to 4
  int resident;                 // shares of a KV head's key tiles that the SMs work on at once
  int shares;                   // shares at most, each one CTA per KV head
  int ctas;                     // shares * hkv
  int most_groups;              // units of a KV head and sequence at most
  int spread;                   // few units, of many shares each
  float *part_o;                // [2 * ctas][8 * nt][head_dim]: what a CTA leaves of the unit
  float4 *part_ml;              // [2 * ctas][8 * nt]            before and after its share
  int4 *cut;                    // [ctas]: the unit that starts in a CTA's share and goes on;
                                // spread: the shares of each unit
  unsigned *status;
};

// Rows of a unit and CTAs of a launch: p.nt and p.ctas from rows.max_rows and
// the head counts.
void kv_attn_plan(KvAttnParams &p, int sms);
// Bytes of the three, and where they lie in a workspace.
size_t kv_attn_part_bytes(const KvAttnParams &p);
void kv_attn_bind(KvAttnParams &p, void *ws);
cudaError_t launch_kv_attn(const KvAttnParams &p, cudaStream_t st);

// Around the tile attention (attn.cu) of larger chunks:
//   the seen slots of one layer as a bf16 slot-major copy (exact) in rows
//   b * cap + i of ko, vo; for each sequence the first and end slot of its rows
//   (lo, hi: seq_len and on) and the first of them (base).  A sequence that is not
//   ok has lo = hi; one without rows is not copied.  NaN codes among the values
//   of new tokens, which earlier rows do not see, are copied as 0 ...
struct KvTileRows {
  int32_t *lo, *hi, *base;   // device [batch]
};
//   (and, meanwhile, how the SMs share the tile attention's work: AttnParams' pieces and
//   joins, where they are asked for)
struct KvTilePlan {
  int4 *pieces;     // device [n_pieces], then as many again of scratch; or null
  int4 *joins;      // device [n_joins]
  int n_pieces, n_joins;
  int units;        // with rows, at most
  int sms;          // partial rows of 2 * sms pieces at most
  int P;            // positions of a unit
};
constexpr int kTilePlanBatch = 256;   // sequences of a plan at most
cudaError_t launch_kv_block_copy(const KvAttnParams &p, void *ko, void *vo, const KvTileRows &t,
                                 const KvTilePlan &plan, cudaStream_t st);
//   ... and put into the rows that do, afterwards (p.lse: of every row, by the tile attention);
cudaError_t launch_kv_restore_nan(const KvAttnParams &p, cudaStream_t st);
//   fp16 rows as bf16 pairs (exact): [n_rows][hi: hq * head_dim | lo: hq * head_dim].
cudaError_t launch_kv_split_rows(const KvAttnParams &p, void *pairs, cudaStream_t st);

}  // namespace cc
