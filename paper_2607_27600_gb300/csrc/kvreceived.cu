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
// share's sequence lie in shared memory as operands, scaled by a power of two per row so
// that bf16 ones fit fp16 exactly.
#include "kvreceived.cuh"

#include <algorithm>
#include <type_traits>

namespace cc {

namespace {

constexpr int kWarps = 8;
constexpr int kStep = 16;            // slots of a warp's step
constexpr int kResident = 2;         // CTAs per SM
constexpr int kAhead = 3;            // heads of a step in flight per warp
constexpr int kQueryBytes = 96 * 1024;   // of the queries in shared memory, at most

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

// Per query row: what makes its products scores, its log2-sum-exp (+inf where it adds
// nothing), and the slots that it sees.
struct __align__(16) RowTerm {
  float f, y, rest;   // rest: in the log2 domain
  int seen;
};

template <typename T, int DH>
__global__ void __launch_bounds__(kWarps * 32, kResident)
    kv_received_kernel(const __grid_constant__ KvReceivedParams p) {
  constexpr int KS = DH / 16;        // k steps of K Q^T
  constexpr int W = DH / 16;         // words of a slot that a lane holds
  extern __shared__ __align__(16) uint8_t smem[];
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
  const int log_block = 31 - __clz(p.block);
  const int NT = p.tiles_at_once, HC = p.heads_at_once;
  uint2 *q_sh = reinterpret_cast<uint2 *>(smem);                         // [HC][NT][KS][32]
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
        const int heads = min(HC, p.hkv - g0), tiles = min(NT, (q_rows - R0 + 7) / 8);
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
          for (int k = 0; k < KS; ++k)
            q_sh[((h * NT + t) * KS + k) * 32 + lane] =
                make_uint2(pack_f16x2(x[4 * k] * up, x[4 * k + 1] * up),
                           pack_f16x2(x[4 * k + 2] * up, x[4 * k + 3] * up));
          if (quad == 0) {
            const RowLse y = row_lse(p, live ? p.lse[row * p.hq + head] : INFINITY);
            r_sh[h * NT * 8 + 8 * t + n8] = {down, y.y, y.rest * 1.44269504f,
                                             p.memory_only ? s.seq : s.seq + pos + 1};
          }
        }
        __syncthreads();
        // ---- this warp's steps: 16 slots of every head of the pass, kAhead heads ahead
        const int mine = (to - from - warp + kWarps - 1) / kWarps;   // (may be <= 0)
        const int items = max(mine, 0) * heads;
        uint32_t kw[kAhead][2][W], ke[kAhead];
        int next_step = from + warp, next_head = 0, left = items;
        long long vec0 = 0;   // of slot 0 of the step: vector index of head 0
        long long exp0 = 0;
        bool ok = true;
        auto enter = [&]() {   // where the step's slots lie
          const int slot = next_step * kStep;
          if (p.pg.head_major) {
            vec0 = ((long long)b * p.hkv + g0) * p.rows.cap + slot;
            exp0 = vec0 >> log_block;
            return;
          }
          const long long row = kv_row(p.pg, p.rows.cap, b, slot);
          ok = row >= 0;
          if (!ok && lane == 0) set_status(p.status, CC_ERR_DEVICE_ARG);
          vec0 = (ok ? row : 0) * hs + g0;
          exp0 = ((ok ? row : 0) >> log_block) * hs + g0;
        };
        const long long head_step = p.pg.head_major ? p.rows.cap : 1;
        const long long head_exps = p.pg.head_major ? p.rows.cap >> log_block : 1;
        auto load = [&](uint32_t (&w)[2][W], uint32_t &e) {
          if (left <= 0) return;
          --left;
          if (next_head == 0) enter();
          const int slot = next_step * kStep + n8;
#pragma unroll
          for (int r = 0; r < 2; ++r) {
            const bool there = ok && slot + 8 * r < v.keys;
            const uint8_t *src = p.k + (vec0 + next_head * head_step + (long long)(n8 + 8 * r) * hs) * DH + quad * (DH / 4);
#pragma unroll
            for (int i = 0; i < W; ++i) w[r][i] = 0;
            if (there) {
              if constexpr (DH == 128) {
                if (wide) {
                  asm("ld.global.nc.v8.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
                      : "=r"(w[r][0]), "=r"(w[r][1]), "=r"(w[r][2]), "=r"(w[r][3]), "=r"(w[r][4]),
                        "=r"(w[r][5]), "=r"(w[r][6]), "=r"(w[r][7])
                      : "l"(src));
                } else {
                  *reinterpret_cast<uint4 *>(&w[r][0]) = load_once(src);
                  *reinterpret_cast<uint4 *>(&w[r][4]) = load_once(src + 16);
                }
              } else {
                *reinterpret_cast<uint4 *>(&w[r][0]) = load_once(src);
              }
            }
          }
          // (a page that is none: its slots receive nothing)
          e = ok ? p.ke[exp0 + next_head * head_exps] : 256u;
          if (++next_head == heads) {
            next_head = 0;
            next_step += kWarps;
          }
        };
#pragma unroll
        for (int a = 0; a < kAhead; ++a) load(kw[a], ke[a]);
        int step = from + warp, h = 0;
        float sum[2] = {0.f, 0.f};
#pragma unroll 1
        for (int it = 0; it < items; it += kAhead) {
#pragma unroll
          for (int a = 0; a < kAhead; ++a) {
            if (it + a < items) {
              const int slot = step * kStep + n8;
              uint32_t wa[W], wb[W];
              const uint32_t e = ke[a];
#pragma unroll
              for (int i = 0; i < W; ++i) {
                wa[i] = kw[a][0][i];
                wb[i] = kw[a][1][i];
              }
              load(kw[a], ke[a]);
              const float scale = __uint_as_float((e & 255u) << 23), kf = fmaf(scale, 0.f, scale);   // (e = 255: NaN)
              const RowTerm *rt = r_sh + h * NT * 8;
              const uint2 *qh = q_sh + (size_t)h * NT * KS * 32 + lane;
              for (int t = 0; t < tiles; ++t) {
                float d[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int k = 0; k < KS; ++k) {
                  const uint2 q2 = qh[(t * KS + k) * 32];
                  mma_f16(d, widen2(wa[k]), widen2(wb[k]), widen2(wa[k] >> 16), widen2(wb[k] >> 16), q2.x, q2.y);
                }
#pragma unroll
                for (int c = 0; c < 2; ++c) {
                  const RowTerm r = rt[8 * t + 2 * quad + c];
                  const float f = r.f * kf;
                  const bool adds = r.y < INFINITY && e < 256u;
#pragma unroll
                  for (int k = 0; k < 2; ++k)
                    if (adds && slot + 8 * k < r.seen) sum[k] += ex2(fmaf(d[2 * k + c], f, -r.y) - r.rest);
                }
              }
              if (++h == heads) {   // the slots' sums of this pass
                h = 0;
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                  float x = sum[k];
                  x += __shfl_xor_sync(0xFFFFFFFFu, x, 1);
                  x += __shfl_xor_sync(0xFFFFFFFFu, x, 2);
                  if (quad == 0 && slot + 8 * k < v.keys) {
                    float *dst = p.acc + (long long)b * p.rows.cap + slot + 8 * k;
                    *dst = (fresh && slot + 8 * k >= s.seq ? 0.f : *dst) + x;
                  }
                  sum[k] = 0.f;
                }
                step += kWarps;
              }
            }
          }
        }
        fresh = false;
      }
  }
}

size_t smem_bytes(const KvReceivedParams &p) {
  return (size_t)p.heads_at_once * p.tiles_at_once * (p.head_dim / 16 * 256 + 8 * sizeof(RowTerm));
}

template <typename T, int DH>
cudaError_t launch(const KvReceivedParams &p, cudaStream_t st) {
  static bool attr_set[64] = {};
  int dev = 0;
  cudaGetDevice(&dev);
  if (dev < 64 && !attr_set[dev]) {
    const cudaError_t e = cudaFuncSetAttribute(kv_received_kernel<T, DH>,
                                               cudaFuncAttributeMaxDynamicSharedMemorySize, kQueryBytes);
    if (e != cudaSuccess) return e;
    attr_set[dev] = true;
  }
  kv_received_kernel<T, DH><<<p.shares, kWarps * 32, smem_bytes(p), st>>>(p);
  return cudaGetLastError();
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
  p.shares = (int)std::min<long long>((long long)sms * kResident, most);
}

cudaError_t launch_kv_received(const KvReceivedParams &p, cudaStream_t st) {
  if (p.head_dim == 128)
    return p.f16 ? launch<__half, 128>(p, st) : launch<__nv_bfloat16, 128>(p, st);
  return p.f16 ? launch<__half, 64>(p, st) : launch<__nv_bfloat16, 64>(p, st);
}

}  // namespace cc
