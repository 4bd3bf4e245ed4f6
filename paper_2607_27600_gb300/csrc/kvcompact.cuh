// kvcompact.cuh -- interface of the in-place compaction of a block-scaled cache.
#pragma once
#include "cc_common.cuh"

namespace cc {

constexpr int kMaxBlockArrays = 2 * 128;   // K and V of each layer
constexpr int kCompactChunk = 128;         // destination slots of a unit: whole blocks and pages
constexpr int kCompactWidth = 128;         // bytes of a slot that a unit moves

struct KvCompactParams {
  int batch, cap;
  int n_arrays;
  uint8_t *codes[kMaxBlockArrays];   // of each layer's K or V
  uint8_t *exps[kMaxBlockArrays];
  int hkv, head_dim, block;
  KvLayout pg;
  int32_t *tokens, *pos;             // [batch][cap]
  float *acc;                        // [batch][cap], or null
  uint8_t *h;                        // [batch][cap] rows of h_bytes, or null
  int h_bytes;
  const int32_t *keep_idx;           // [batch][cap]
  const int32_t *keep_count;         // [batch]
  int32_t *seq_len;                  // [batch], set to keep_count
  // workspace (kv_compact_bind)
  int *first_chunk;                  // [batch + 1]: chunks of the sequences before
  int *reader;                       // [batch][reader_ld]: first kept slot with a source at or past chunk c
  unsigned *flags;                   // of each unit: its sources are read
  // set by kv_compact_plan
  int planes;                        // units of a chunk of slots
  int array_planes, h_planes;        // of an array of codes, of h
  int reader_ld;                     // chunks of cap, and one
  size_t flag_count;
  unsigned *status;
};

void kv_compact_plan(KvCompactParams &p);
size_t kv_compact_bytes(const KvCompactParams &p);
void kv_compact_bind(KvCompactParams &p, void *ws);
cudaError_t launch_kv_compact(const KvCompactParams &p, int sms, cudaStream_t st);

}  // namespace cc
