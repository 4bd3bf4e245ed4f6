// kvreceived.cu -- the attention that the slots of a block-scaled cache receive
// from a step's rows: what an eviction by accumulated attention ranks by.
//
// With x_rj = q_r . K_j 2^(ek_j - 127) log2(e) / sqrt(dh) and y_r = lse_r log2(e),
//   acc[j] += sum over the rows r (of all heads) that see j of 2^(x_rj - y_r):
// the softmax's denominator comes with the rows, so that a slot's sum needs nothing of
// any other slot and the values are not read.  Sums are fp32 in a fixed order.
//
// Few rows a sequence: bound by the bytes of the key codes, read once for all rows.
// The products are m16n8k16 with 16 slots on the M side and 8 query rows on the N
// side, S^T = K Q^T, so that the slots of a lane stay the same from head to head and its
// sums in registers.  A warp takes 16 slots of all heads, each lane 32 bytes of a slot's
// 128 straight into the registers that the products read (which element of a row meets
// which k index is free as long as Q agrees), several heads ahead.  The queries of a
// share's sequence lie in shared memory as fp16 operands, scaled by a power of two per row and head:
// exact but for elements more than 2^24 (fp16 rows: 2^21) below the largest, which are off by at
// most 2^-32 of that one.
//
// 64 sequences of 1500 to 32767 slots, a row each of 32 heads of 128 on 8: 213 us, 5.3 TB/s
// of codes and exponents; 16 sequences of 250 to 9001, five rows each: 33 us, 2.3 TB/s: too short for
// more, and with 24 columns of scores 16 warps an SM instead of 24.  Bound by the latency of
// the loads (long scoreboard first among the stalls, DRAM busy 67 % at 32 sequences).
#include "kvreceived.cuh"

#include <algorithm>
#include <type_traits>

namespace cc {

namespace {

constexpr int kWarps = 8;
constexpr int kStep = 16;            // slots of a warp's step
// CTAs per SM: two, and three where one tile of query rows leaves the registers and the cache has
// room for so many slots that it pays.  Two and three, a row each: 64 sequences of 32000 slots, 16/4
// heads, 212 and 203 us; 32 of 16600, 32/8 heads, 114 and 114; four of 16384, 16/4 heads, 12.8 and 14.9; one of
// 8191, 28/4 heads, 8.2 and 10.6.
constexpr long long kManySteps = 128;   // of a CTA
constexpr int kSegment = 32;         // steps between joins of the warps' sums
constexpr int kQueryBytes = 92 * 1024;   // of the queries in shared memory, at most

CC_DEV uint32_t widen2(uint32_t two) {   // e4m3 pair (low 16 bits) -> fp16 pair, exact
  uint32_t r;
  asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(r) : "h"((unsigned short)two));
  return r;
}
CC_DEV void mma_f16(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0,
                    uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, "
      "{%0,%1,%2,%3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
CC_DEV uint4 load_once(const uint8_t *p) {
  uint4 u;
  asm("ld.global.nc.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(u.x), "=r"(u.y), "=r"(u.z), "=r"(u.w) : "l"(p));
  return u;
}

// What a share sees of sequence b: `keys` slots (0: no rows, or a bad sequence).
struct Seen {
  SeqRows s;
  int keys;
};
CC_DEV Seen seen_of(const KvReceivedParams &p, int b) {
  Seen v;
  v.s = seq_rows(p.rows, b, !p.memory_only);
  v.keys = v.s.count == 0 ? 0 : v.s.seq + (p.memory_only ? 0 : v.s.count);
  return v;
}
CC_DEV int steps_of(const KvReceivedParams &p, int b) { return (seen_of(p, b).keys + kStep - 1) / kStep; }
CC_DEV long long total_steps(const KvReceivedParams &p) {   // a whole warp calls
  long long all = 0;
  for (int b = threadIdx.x & 31; b < p.rows.batch; b += 32) all += steps_of(p, b);
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) all += __shfl_xor_sync(0xFFFFFFFFu, all, o);
  return all;
}
// The sequence that holds step `at` (below the total) and the steps before it.
CC_DEV int find_step(const KvReceivedParams &p, long long at, long long &before) {
  const int lane = threadIdx.x & 31;
  before = 0;
  for (int b0 = 0; b0 < p.rows.batch; b0 += 32) {
    const long long w = b0 + lane < p.rows.batch ? steps_of(p, b0 + lane) : 0;
    long long sum = w;   // inclusive prefix over the lanes
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const long long x = __shfl_up_sync(0xFFFFFFFFu, sum, o);
      if (lane >= o) sum += x;
    }
    const unsigned past = __ballot_sync(0xFFFFFFFFu, before + sum > at);
    if (past) {
      const int k = __ffs(past) - 1;
      before += __shfl_sync(0xFFFFFFFFu, sum - w, k);
      return b0 + k;
    }
    before += __shfl_sync(0xFFFFFFFFu, sum, 31);
  }
  return p.rows.batch;
}

// Per query row: what makes its products scores, its log2-sum-exp, and the slots that it sees
// (none where it adds nothing).
struct __align__(16) RowTerm {
  float f, y, rest;   // rest: in the log2 domain
  int seen;
};

// TILES: eights of query rows of a KV head in a pass where there are few, all of which take the
// slots' widened codes as they are made; 0: any number, which are widened first.
template <typename T, int DH, int TILES, int RESIDENT>
__global__ void __launch_bounds__(kWarps * 32, RESIDENT)
    kv_received_kernel(const __grid_constant__ KvReceivedParams p) {
  constexpr int KS = DH / 16;        // k steps of K Q^T
  constexpr int W = DH / 16;         // words of a slot that a lane holds
  extern __shared__ __align__(16) uint8_t smem[];
  __shared__ float sum_sh[kWarps][kSegment * kStep];
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, n8 = lane >> 2, quad = lane & 3;
  const long long total = total_steps(p);
  const int n_shares = (int)min((long long)p.shares, total);
  if (blockIdx.x == 0)   // reported once: sequences whose rows or lengths are bad
    for (int b = tid; b < p.rows.batch; b += kWarps * 32)
      if (!seq_rows(p.rows, b, !p.memory_only).ok) set_status(p.status, CC_ERR_DEVICE_ARG);
  const int share = blockIdx.x;
  if (share >= n_shares) return;
  long long at = total * share / n_shares;
  const long long end = total * (share + 1) / n_shares;
  long long before;
  int b = find_step(p, at, before);
  const int G = p.hq / p.hkv;
  const int hs = p.pg.head_major ? 1 : p.hkv;
  const int log_block = 31 - __clz(p.block), slot_bytes = hs * DH;
  const long long head_bytes = (p.pg.head_major ? (long long)p.rows.cap : 1) * DH;
  const long long head_exps = p.pg.head_major ? p.rows.cap >> log_block : 1;
  const int NT = p.tiles_at_once, HC = p.heads_at_once;
  uint4 *q_sh = reinterpret_cast<uint4 *>(smem);                         // [HC][NT][KS / 2][32]
  RowTerm *r_sh = reinterpret_cast<RowTerm *>(smem + (size_t)HC * NT * KS * 256);   // [HC][NT * 8]
  // whether a lane's 32 bytes may be one load
  const bool wide = (reinterpret_cast<uintptr_t>(p.k) & 31) == 0;

  for (; at < end; ++b) {
    const Seen v = seen_of(p, b);
    const int steps = (v.keys + kStep - 1) / kStep;
    if (before + steps <= at) {
      before += steps;
      continue;
    }
    const int from = (int)(at - before), to = (int)min((long long)steps, from + (end - at));
    at += to - from;
    before += steps;
    const SeqRows s = v.s;
    const int q_rows = s.count * G;   // of a KV head
    bool fresh = p.first != 0;        // the new rows' slots start from 0
    for (int g0 = 0; g0 < p.hkv; g0 += HC)
      for (int R0 = 0; R0 < q_rows; R0 += 8 * NT) {
        const int heads = min(HC, p.hkv - g0), tiles = TILES > 0 ? TILES : min(NT, (q_rows - R0 + 7) / 8);
        // ---- where this warp's items lie: every kWarps-th pair of heads, through the steps
        const int pairs = (heads + 1) / 2;
        const int step_skip = kWarps / pairs, pair_skip = kWarps - step_skip * pairs;
        uint32_t kw[2][2][W], ke[2];
        int next_step = 0, next_pair = 0, left = 0;
        int run = 0;   // steps from next_step on that lie one after the other
        int row = 0;   // of a slot-major buffer or pool, next_step's first slot's; -1: no page
        const uint8_t *at[2], *at_e;   // of the next item: the lane's slots, their scale
        // Where the next item lies.
        auto find = [&]() {
          const int slot = next_step * kStep;
          if (run <= 0) {
            if (!p.pg.table || p.pg.head_major) {
              row = b * p.rows.cap + slot;
              run = 0x7FFFFFFF;
            } else {   // a page that is none: its slots receive nothing
              row = (int)kv_row(p.pg, p.rows.cap, b, slot);
              run = (p.pg.page - slot % p.pg.page) / kStep;
              if (row < 0 && lane == 0) set_status(p.status, CC_ERR_DEVICE_ARG);
            }
          }
          const int g = g0 + 2 * next_pair;
          const long long vec = p.pg.head_major ? (long long)(b * p.hkv + g) * p.rows.cap + slot
                                                : (long long)max(0, row) * p.hkv + g;
          const uint8_t *src = p.k + vec * DH + quad * (DH / 4);
          const int last = min(kStep - 1, v.keys - 1 - slot);   // (past the last seen slot: that one)
          at[0] = src + min(n8, last) * slot_bytes;
          at[1] = src + min(n8 + 8, last) * slot_bytes;
          at_e = p.ke + (p.pg.head_major ? vec >> log_block : (long long)(max(0, row) >> log_block) * p.hkv + g);
        };
        auto load = [&](int i) {   // the i-th head of the pair
          if (2 * next_pair + i >= heads) return;
#pragma unroll
          for (int r = 0; r < 2; ++r) {
            const uint8_t *src = at[r] + i * head_bytes;
            if constexpr (DH == 128) {
              if (wide) {
                asm volatile("ld.global.nc.v8.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
                             : "=r"(kw[i][r][0]), "=r"(kw[i][r][1]), "=r"(kw[i][r][2]), "=r"(kw[i][r][3]),
                               "=r"(kw[i][r][4]), "=r"(kw[i][r][5]), "=r"(kw[i][r][6]), "=r"(kw[i][r][7])
                             : "l"(src));
              } else {
                *reinterpret_cast<uint4 *>(&kw[i][r][0]) = load_once(src);
                *reinterpret_cast<uint4 *>(&kw[i][r][4]) = load_once(src + 16);
              }
            } else {
              *reinterpret_cast<uint4 *>(&kw[i][r][0]) = load_once(src);
            }
          }
          ke[i] = row < 0 ? 256u : at_e[i * head_exps];
        };
        auto advance = [&]() {
          int on = step_skip;
          next_pair += pair_skip;
          if (next_pair >= pairs) {
            next_pair -= pairs;
            ++on;
          }
          next_step += on;
          run -= on;
          if (row >= 0) row += on * kStep;
        };
        // The first of this warp's items of the segment at `seg` on their way.
        auto begin = [&](int seg) {
          const int n = min(kSegment, to - seg);   // (may be <= 0)
          left = max(0, (n * pairs - warp + kWarps - 1) / kWarps);
          next_step = seg + warp / pairs;
          next_pair = warp % pairs;
          run = 0;
          if (left > 0) {
            find();
            load(0);
            load(1);
          }
        };
        begin(from);
        // ---- the queries: row 8 t + n8 of a head as the second operand, fp16, scaled
        // to a largest magnitude of [2^7, 2^8)
        __syncthreads();   // the last pass is done with them
        for (int i = warp; i < heads * tiles; i += kWarps) {
          const int h = i / tiles, t = i - h * tiles;
          const int R = R0 + 8 * t + n8, pos = R / G, head = (g0 + h) * G + R - pos * G;
          const bool live = R < q_rows;
          const long long row = s.r0 + pos;
          float x[DH / 4], top = 0.f;
          const T *src = reinterpret_cast<const T *>(p.q) + row * p.q_ld + (long long)head * DH + quad * (DH / 4);
#pragma unroll
          for (int c = 0; c < DH / 32; ++c) {
            const uint4 u = live ? reinterpret_cast<const uint4 *>(src)[c] : make_uint4(0, 0, 0, 0);
            const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              float2 f;
              if constexpr (std::is_same_v<T, __half>)
                f = __half22float2(*reinterpret_cast<const __half2 *>(&w[j]));
              else
                f = make_float2(bf16_lo(w[j]), bf16_hi(w[j]));
              x[c * 8 + 2 * j] = f.x;
              x[c * 8 + 2 * j + 1] = f.y;
              top = fmaxf(top, fmaxf(fabsf(f.x), fabsf(f.y)));
            }
          }
          top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, 1));
          top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, 2));
          // 2^(7 - exponent of top), kept in the range whose inverse is normal
          const int e = top > 0.f && top < INFINITY ? max((int)(__float_as_uint(top) >> 23), 8) : 134;
          const float up = __uint_as_float((uint32_t)min(261 - e, 253) << 23);
          const float down = p.scale_log2 * __uint_as_float((uint32_t)max(e - 7, 1) << 23);
#pragma unroll
          for (int k = 0; k < KS / 2; ++k)
            q_sh[((h * NT + t) * (KS / 2) + k) * 32 + lane] =
                make_uint4(pack_f16x2(x[8 * k] * up, x[8 * k + 1] * up), pack_f16x2(x[8 * k + 2] * up, x[8 * k + 3] * up),
                           pack_f16x2(x[8 * k + 4] * up, x[8 * k + 5] * up), pack_f16x2(x[8 * k + 6] * up, x[8 * k + 7] * up));
          if (quad == 0) {
            const RowLse y = row_lse(p, live ? p.lse[row * p.hq + head] : INFINITY);
            const int seen = p.memory_only ? s.seq : s.seq + pos + 1;
            r_sh[h * NT * 8 + 8 * t + n8] = {down, y.y, y.rest * 1.44269504f, y.y < INFINITY ? seen : 0};
          }
        }
        __syncthreads();
        // ---- segments of kSegment steps: 16 slots of two heads at a time, a step's heads by
        // neighbouring warps, so that a slot's bytes are read at about one time
        for (int seg = from; seg < to; seg += kSegment) {
          const int seg_end = min(to, seg + kSegment);
          float *mine = sum_sh[warp];
          for (int i = lane; i < (seg_end - seg) * kStep; i += 32) mine[i] = 0.f;
          __syncwarp();
#pragma unroll 1
          for (; left > 0; --left) {
            const int step = next_step, pair = next_pair, slot = step * kStep + n8;
            advance();
            if (left > 1) find();
            float sum[2] = {0.f, 0.f};
#pragma unroll
            for (int i = 0; i < 2; ++i) {
              const int h = 2 * pair + i;
              if (h >= heads) break;
              const uint32_t e = ke[i];
              const float scale = __uint_as_float((e & 255u) << 23), kf = fmaf(scale, 0.f, scale);   // (e = 255: NaN)
              const RowTerm *rt = r_sh + h * NT * 8 + 2 * quad;
              const uint4 *qh = q_sh + (size_t)h * NT * (KS / 2) * 32 + lane;
              auto weigh = [&](const float (&d)[4], const RowTerm *of) {
#pragma unroll
                for (int c = 0; c < 2; ++c) {
                  const RowTerm r = of[c];
                  const float f = r.f * kf;
                  // (a row that adds nothing sees no slot)
#pragma unroll
                  for (int k = 0; k < 2; ++k) {
                    const float x = ex2(fmaf(d[2 * k + c], f, -r.y) - r.rest);
                    sum[k] += slot + 8 * k < r.seen && e < 256u ? x : 0.f;
                  }
                }
              };
              // (two chains of products: a step drops the bits below its sum's last, always downwards;
              // one chain's totals are 2.2e-6 off over 8192 slots, two chains' 0.9e-6)
              auto add = [](float (&d)[4], const float (&d2)[4]) {
#pragma unroll
                for (int c = 0; c < 4; ++c) d[c] += d2[c];
              };
              if constexpr (TILES > 0) {
                float d[TILES][4], d2[TILES][4];
#pragma unroll
                for (int t = 0; t < TILES; ++t)
#pragma unroll
                  for (int c = 0; c < 4; ++c) d[t][c] = d2[t][c] = 0.f;
#pragma unroll
                for (int k = 0; k < KS; k += 2) {
                  uint32_t op[2][4];
#pragma unroll
                  for (int j = 0; j < 2; ++j) {
                    op[j][0] = widen2(kw[i][0][k + j]);
                    op[j][1] = widen2(kw[i][1][k + j]);
                    op[j][2] = widen2(kw[i][0][k + j] >> 16);
                    op[j][3] = widen2(kw[i][1][k + j] >> 16);
                  }
#pragma unroll
                  for (int t = 0; t < TILES; ++t) {
                    const uint4 q4 = qh[(t * (KS / 2) + k / 2) * 32];
                    mma_f16(d[t], op[0][0], op[0][1], op[0][2], op[0][3], q4.x, q4.y);
                    mma_f16(d2[t], op[1][0], op[1][1], op[1][2], op[1][3], q4.z, q4.w);
                  }
                }
                if (left > 1) load(i);
#pragma unroll
                for (int t = 0; t < TILES; ++t) {
                  add(d[t], d2[t]);
                  weigh(d[t], rt + 8 * t);
                }
              } else {
                uint32_t op[KS][4];
#pragma unroll
                for (int k = 0; k < KS; ++k) {
                  op[k][0] = widen2(kw[i][0][k]);
                  op[k][1] = widen2(kw[i][1][k]);
                  op[k][2] = widen2(kw[i][0][k] >> 16);
                  op[k][3] = widen2(kw[i][1][k] >> 16);
                }
                if (left > 1) load(i);
#pragma unroll 1
                for (int t = 0; t < tiles; ++t, qh += KS / 2 * 32) {
                  float d[4] = {0.f, 0.f, 0.f, 0.f}, d2[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                  for (int k = 0; k < KS / 2; ++k) {
                    const uint4 q4 = qh[k * 32];
                    mma_f16(d, op[2 * k][0], op[2 * k][1], op[2 * k][2], op[2 * k][3], q4.x, q4.y);
                    mma_f16(d2, op[2 * k + 1][0], op[2 * k + 1][1], op[2 * k + 1][2], op[2 * k + 1][3], q4.z, q4.w);
                  }
                  add(d, d2);
                  weigh(d, rt + 8 * t);
                }
              }
            }
            // (an odd last head: the pair's second was not there, the next one's may be)
            if (2 * pair + 1 >= heads && left > 1) load(1);
#pragma unroll
            for (int k = 0; k < 2; ++k) {
              sum[k] += __shfl_xor_sync(0xFFFFFFFFu, sum[k], 1);
              sum[k] += __shfl_xor_sync(0xFFFFFFFFu, sum[k], 2);
            }
            if (quad < 2) mine[(step - seg) * kStep + n8 + 8 * quad] += quad ? sum[1] : sum[0];
          }
          begin(seg + kSegment);
          // the warps' sums in their order
          __syncthreads();
          for (int i = tid; i < (seg_end - seg) * kStep; i += kWarps * 32) {
            const int slot = seg * kStep + i;
            if (slot >= v.keys) break;
            float x = 0.f;
#pragma unroll
            for (int w = 0; w < kWarps; ++w) x += sum_sh[w][i];
            float *dst = p.acc + (long long)b * p.rows.cap + slot;
            *dst = (fresh && slot >= s.seq ? 0.f : *dst) + x;
          }
          __syncthreads();
        }
        fresh = false;
      }
  }
}

size_t smem_bytes(const KvReceivedParams &p) {
  return (size_t)p.heads_at_once * p.tiles_at_once * (p.head_dim / 16 * 256 + 8 * sizeof(RowTerm));
}

template <typename T, int DH, int TILES, int RESIDENT = 2>
cudaError_t launch_tiles(const KvReceivedParams &p, cudaStream_t st) {
  static bool attr_set[64] = {};
  int dev = 0;
  cudaGetDevice(&dev);
  if (dev < 64 && !attr_set[dev]) {
    const cudaError_t e = cudaFuncSetAttribute(kv_received_kernel<T, DH, TILES, RESIDENT>,
                                               cudaFuncAttributeMaxDynamicSharedMemorySize, kQueryBytes);
    if (e != cudaSuccess) return e;
    attr_set[dev] = true;
  }
  kv_received_kernel<T, DH, TILES, RESIDENT><<<p.shares, kWarps * 32, smem_bytes(p), st>>>(p);
  return cudaGetLastError();
}
template <typename T, int DH>
cudaError_t launch(const KvReceivedParams &p, cudaStream_t st) {
  switch (p.tiles_at_once) {
    case 1: return p.resident == 3 ? launch_tiles<T, DH, 1, 3>(p, st) : launch_tiles<T, DH, 1>(p, st);
    case 2: return launch_tiles<T, DH, 2>(p, st);
    case 3: return launch_tiles<T, DH, 3>(p, st);
    default: return launch_tiles<T, DH, 0>(p, st);
  }
}

}  // namespace

void kv_received_plan(KvReceivedParams &p, int sms) {
  const int G = p.hq / p.hkv;
  const int tile = p.head_dim / 16 * 256 + 8 * (int)sizeof(RowTerm);   // bytes of 8 query rows of a head
  const int room = kQueryBytes / tile;
  p.heads_at_once = std::min(p.hkv, room);
  const long long tiles = ((long long)p.rows.max_rows * G + 7) / 8;
  p.tiles_at_once = (int)std::min<long long>(tiles, room / p.heads_at_once);
  const long long most = (long long)p.rows.batch * ((p.rows.cap + kStep - 1) / kStep);
  p.resident = p.tiles_at_once == 1 && most > sms * 3 * kManySteps ? 3 : 2;
  // (two steps a CTA at least: each brings the queries in for itself)
  p.shares = (int)std::min<long long>((long long)sms * p.resident, (most + 1) / 2);
}

cudaError_t launch_kv_received(const KvReceivedParams &p, cudaStream_t st) {
  if (p.head_dim == 128)
    return p.f16 ? launch<__half, 128>(p, st) : launch<__nv_bfloat16, 128>(p, st);
  return p.f16 ? launch<__half, 64>(p, st) : launch<__nv_bfloat16, 64>(p, st);
}

}  // namespace cc
