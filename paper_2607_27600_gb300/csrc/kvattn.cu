// kvattn.cu -- attention of a few query rows per sequence over a paged cache of
// e4m3 codes with a power-of-two scale for each block of slots and KV head.
//
// With x_j = q . K_j 2^ek_j log2(e) / sqrt(dh) and lv_j the V exponent,
//   out = sum_j 2^(x_j + lv_j) code_j / sum_j 2^x_j,
// in one pass over the keys with two running references per row: m for the
// sum below, so that 2^(x - m) neither overflows nor vanishes, and mv for the sum
// above, so that the largest 2^(x + lv - mv) fills fp16, in which the
// probabilities meet the codes (exact in fp16) on the tensor cores.  Both are
// whole numbers: every rescaling is by a power of two.  Queries are scaled by a
// power of two per row so that bf16 ones fit fp16 exactly; sums are fp32.
//
// Bound by the cache's bytes: a tcgen05 tile of 128 query rows would be
// nearly all padding, so the products are m16n8k16 with the keys (then the head
// dimension) on the M side and the 8 * NT query rows of a unit (the heads of a KV head
// at consecutive positions) on the N side: S^T = K Q^T, O^T = V^T P^T.  A
// unit's key tiles of 64 are one long line over all units, cut into equal shares
// for the CTAs of one resident wave, so that ragged batches balance; a unit that
// spans shares is joined by kv_combine_kernel in share order.
//
// A lane copies exactly the 16-byte pieces that it will itself multiply
// (cp.async into a slot of its own), so the ring needs no barrier: K rows
// lane/4 and lane/4 + 8, V rows 2 (lane%4) + {0, 1, 8, 9}.  Which element of a
// piece meets which k index is free as long as Q agrees; transposing V is a byte
// permute of two rows' words before they are widened.
#include "kvattn.cuh"

#include <algorithm>
#include <type_traits>

namespace cc {

namespace {

constexpr int kWarps = 4;          // of a CTA, each every fourth 16 keys of a tile
constexpr int kTile = 16 * kWarps; // keys of a tile
constexpr int kMinTiles = 2;       // of a share at least
constexpr float kNone = -1e30f;    // reference of a row that has seen no key
constexpr float kSumLimit = 64.f;  // log2 of a term of the sum below
constexpr float kTop = 15.f, kHead = 8.f;   // log2 of a term above: limit, and what a new reference leaves

template <int NT>
constexpr int stages() { return 4; }

template <int DH, int NT>
struct KvSmem {
  static constexpr int KP = DH / 32;              // 16-byte pieces of K per lane and stage
  static constexpr int VB = DH / 8;               // bytes of V per lane and row
  static constexpr int STAGE = 32 * (KP * 16 + 4 * VB);   // bytes of a warp's stage
  static constexpr int ST = stages<NT>();
  static constexpr int RING = ST * STAGE;         // bytes of a warp's ring
  static constexpr int ROWS = 8 * NT;
  static constexpr int MERGE = ROWS * DH * 4;     // a warp's partial rows
  static constexpr int BYTES = kWarps * (RING > MERGE ? RING : MERGE);
};

CC_DEV float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
CC_DEV uint32_t widen2(uint32_t two) {   // e4m3 pair (low 16 bits) -> fp16 pair, exact
  uint32_t r;
  asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(r) : "h"((unsigned short)two));
  return r;
}
CC_DEV uint32_t transpose8(uint32_t x) {
  uint32_t r;
  asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(x));
  return r;
}
CC_DEV void mma_f16(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0,
                    uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, "
      "{%0,%1,%2,%3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
template <int BYTES>
CC_DEV void copy_async(uint32_t dst, const void *src, bool there) {   // else zeros
  if constexpr (BYTES == 16)
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src),
                 "r"(there ? 16 : 0) : "memory");
  else
    asm volatile("cp.async.ca.shared.global [%0], [%1], 8, %2;" ::"r"(dst), "l"(src),
                 "r"(there ? 8 : 0) : "memory");
}
CC_DEV void copy_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
CC_DEV void copy_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

// ---------------------------------------------------------------------------
// the line of key tiles
// ---------------------------------------------------------------------------
struct SeqPlan {
  SeqRows s;
  int keys;     // seen slots of the last row
  int tiles;    // key tiles of a unit (at least one, so that empty rows are written)
  int groups;   // units of a KV head
};
template <int NT>
CC_DEV SeqPlan seq_plan(const KvAttnParams &p, int b) {
  SeqPlan q;
  q.s = seq_rows(p.rows, b, !p.memory_only);
  q.keys = q.s.ok ? q.s.seq + (p.memory_only ? 0 : q.s.count) : 0;
  q.tiles = max(1, (q.keys + kTile - 1) / kTile);
  q.groups = (q.s.count * (p.hq / p.hkv) + 8 * NT - 1) / (8 * NT);
  return q;
}
// Tiles of a sequence's units, and of all sequences'.  A whole warp calls the latter.
CC_DEV long long seq_tiles(const KvAttnParams &p, const SeqPlan &q) {
  return (long long)q.groups * q.tiles * p.hkv;
}
template <int NT>
CC_DEV long long total_tiles(const KvAttnParams &p) {
  long long all = 0;
  for (int b = threadIdx.x & 31; b < p.rows.batch; b += 32) all += seq_tiles(p, seq_plan<NT>(p, b));
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) all += __shfl_xor_sync(0xFFFFFFFFu, all, o);
  return all;
}
// The sequence that holds tile `at` (less than the total) and the tiles before
// it.  A whole warp calls.
template <int NT>
CC_DEV int find_tile(const KvAttnParams &p, long long at, long long &before) {
  const int lane = threadIdx.x & 31;
  before = 0;
  for (int b0 = 0; b0 < p.rows.batch; b0 += 32) {
    const long long w = b0 + lane < p.rows.batch ? seq_tiles(p, seq_plan<NT>(p, b0 + lane)) : 0;
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
// CTAs that get a share of `total` tiles; CTA c's starts at total * c / n.
CC_DEV int sharing_ctas(const KvAttnParams &p, long long total) {
  return (int)max(1ll, min((long long)p.ctas, (total + kMinTiles - 1) / kMinTiles));
}
CC_DEV int cta_of_tile(long long t, long long total, int n) {   // the last c with total * c / n <= t
  return (int)(((t + 1) * n - 1) / total);
}

template <typename T>
CC_DEV uint32_t pack2(float a, float b) {
  return std::is_same_v<T, __half> ? pack_f16x2(a, b) : pack_bf16x2(a, b);
}

// Row R of a unit's group: which row of the buffers and which head.
struct RowAt {
  int row, head;
  bool live;
};
CC_DEV RowAt row_at(const KvAttnParams &p, const SeqRows &s, int g, int R) {
  const int G = p.hq / p.hkv, pos = R / G;
  return {s.r0 + pos, g * G + R - pos * G, pos < s.count};
}

// out and lse of one row's share of the head dimension: the joined sums.
template <typename T>
CC_DEV void store2(const KvAttnParams &p, const RowAt &r, int d, int dh, float o0, float o1, float m,
                   float mv, float l) {
  const bool good = l > 0.f && l < INFINITY;
  const int shift = good ? (int)(mv - m) : 0;
  const float inv = good ? 1.f / l : 0.f;
  const uint32_t w = good ? pack2<T>(ldexpf(o0 * inv, shift), ldexpf(o1 * inv, shift)) : 0u;
  *reinterpret_cast<uint32_t *>(reinterpret_cast<T *>(p.out) + r.row * p.out_ld +
                                (long long)r.head * dh + d) = w;
  if (p.lse && d == 0)
    p.lse[(long long)r.row * p.hq + r.head] =
        l == 0.f ? -INFINITY : (m + log2f(l)) * 0.69314718055994531f;
}

// ---------------------------------------------------------------------------
// the kernel
// ---------------------------------------------------------------------------
template <typename T, int DH, int NT>
__global__ void __launch_bounds__(kWarps * 32, NT == 4 ? 2 : 3)
    kv_attn_kernel(const __grid_constant__ KvAttnParams p) {
  using L = KvSmem<DH, NT>;
  constexpr int KS = DH / 16;        // k steps of K Q^T
  constexpr int DT = DH / 16;        // M tiles of V^T P^T
  constexpr int KP = L::KP, ST = L::ST, VW = DH / 32;
  extern __shared__ __align__(16) uint8_t smem[];
  __shared__ float s_m[kWarps][L::ROWS], s_mv[kWarps][L::ROWS], s_l[kWarps][L::ROWS];
  pdl_trigger();   // the combine may launch: it waits for this grid
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, n8 = lane >> 2, quad = lane & 3;
  const long long total = total_tiles<NT>(p);
  const int n_ctas = sharing_ctas(p, total), cta = blockIdx.x;
  if (cta >= n_ctas) return;
  long long at = total * cta / n_ctas;
  const long long end = total * (cta + 1) / n_ctas;
  // reported once, by the first CTA: sequences whose rows or lengths are bad
  if (cta == 0)
    for (int b = tid; b < p.rows.batch; b += kWarps * 32)
      if (!seq_rows(p.rows, b, !p.memory_only).ok) set_status(p.status, CC_ERR_DEVICE_ARG);
  if (at >= end) return;

  long long before;
  int b = find_tile<NT>(p, at, before);
  if (b >= p.rows.batch) return;   // (at < total)
  const uint32_t ring = smem_u32(smem) + warp * L::RING;
  const int vstep = p.pg.head_major ? 1 : p.hkv;
  SeqPlan sq = seq_plan<NT>(p, b);
  bool first = true;   // the share's first segment
  while (at < end) {
    while (before + seq_tiles(p, sq) <= at) {   // the next sequence with rows
      before += seq_tiles(p, sq);
      sq = seq_plan<NT>(p, ++b);
    }
    const long long in_seq = at - before;
    const int unit = (int)(in_seq / sq.tiles), g = unit / sq.groups, grp = unit - g * sq.groups;
    const int tile0 = (int)(in_seq - (long long)unit * sq.tiles);
    const int tile1 = (int)min((long long)sq.tiles, tile0 + (end - at));
    const SeqRows s = sq.s;
    const int G = p.hq / p.hkv, R0 = grp * L::ROWS;
    // seen slots of the group's first and last row
    const int last_pos = min(s.count - 1, (R0 + L::ROWS - 1) / G);
    const int seen_lo = p.memory_only ? s.seq : s.seq + R0 / G + 1;
    const int seen_hi = p.memory_only ? s.seq : s.seq + last_pos + 1;

    // ---- the ring of 16-key steps of this warp: step i is keys
    // (tile0 + i) * 64 + 16 warp + [0, 16)
    const int steps = tile1 - tile0;
    int issued = 0;
    auto issue = [&](int &ek, int &ev) {
      const int slot = (tile0 + issued) * kTile + warp * 16;
      const uint32_t dst = ring + (issued % ST) * L::STAGE;
      ek = ev = 127;
      if (issued < steps && slot < seen_hi) {
        const long long vec = kv_vec(p.pg, p.rows.cap, b, g, slot);
        const bool ok = vec >= 0;
        const long long v0 = ok ? vec : 0;
        if (!ok && lane == 0) set_status(p.status, CC_ERR_DEVICE_ARG);
        const int left = ok ? seen_hi - slot : 0;
        const long long ei = p.pg.head_major ? v0 / p.block : v0 / p.hkv / p.block * p.hkv + g;
        ek = p.ke[ei];
        ev = p.ve[ei];
        const uint8_t *kp = p.k + v0 * DH + quad * 16, *vp = p.v + v0 * DH + n8 * L::VB;
#pragma unroll
        for (int r = 0; r < 2; ++r) {
          const int row = n8 + 8 * r;
          const bool there = row < left;
          const uint8_t *src = kp + (there ? row * vstep * DH : 0);
#pragma unroll
          for (int h = 0; h < KP / 2; ++h)
            copy_async<16>(dst + ((r * (KP / 2) + h) * 32 + lane) * 16, src + h * 64, there);
        }
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const int row = 2 * quad + (r & 1) + 8 * (r >> 1);
          const bool there = row < left;
          copy_async<L::VB>(dst + KP * 512 + (r * 32 + lane) * L::VB,
                            vp + (there ? row * vstep * DH : 0), there);
        }
        if (!ok) ek = -1;   // its slots are not seen
      }
      ++issued;
      copy_commit();
    };
    int ek_q[ST], ev_q[ST];
#pragma unroll
    for (int i = 0; i < ST - 1; ++i) issue(ek_q[i], ev_q[i]);

    // ---- queries: row 8 t + n8 of the group as the second operand, fp16,
    // scaled to a largest magnitude of [2^7, 2^8)
    uint32_t qb[NT][KS][2];
    float qf[NT][2];           // of rows 2 quad, 2 quad + 1: what undoes the scale, with the softmax's
    int seen[NT][2];           // slots they see
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      const RowAt r = row_at(p, s, g, R0 + 8 * t + n8);
      float x[DH / 4];
      float top = 0.f;
#pragma unroll
      for (int h = 0; h < DH / 64; ++h) {
        const T *src = reinterpret_cast<const T *>(p.q) + r.row * p.q_ld + (long long)r.head * DH +
                       h * 64 + quad * 16;
#pragma unroll
        for (int c = 0; c < 2; ++c) {
          const uint4 u = r.live ? reinterpret_cast<const uint4 *>(src)[c] : make_uint4(0, 0, 0, 0);
          const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            float2 f;
            if constexpr (std::is_same_v<T, __half>)
              f = __half22float2(*reinterpret_cast<const __half2 *>(&w[i]));
            else
              f = make_float2(bf16_lo(w[i]), bf16_hi(w[i]));
            x[h * 16 + c * 8 + 2 * i] = f.x;
            x[h * 16 + c * 8 + 2 * i + 1] = f.y;
            top = fmaxf(top, fmaxf(fabsf(f.x), fabsf(f.y)));
          }
        }
      }
      top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, 1));
      top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, 2));
      // 2^(7 - exponent of top), kept in the range whose inverse is normal
      const int e = top > 0.f && top < INFINITY ? max((int)(__float_as_uint(top) >> 23), 8) : 134;
      const float up = __uint_as_float((uint32_t)min(261 - e, 253) << 23);
      const float down = p.scale_log2 * __uint_as_float((uint32_t)max(e - 7, 1) << 23);
#pragma unroll
      for (int k = 0; k < KS; ++k) {
        qb[t][k][0] = pack_f16x2(x[4 * k] * up, x[4 * k + 1] * up);
        qb[t][k][1] = pack_f16x2(x[4 * k + 2] * up, x[4 * k + 3] * up);
      }
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        qf[t][c] = __shfl_sync(0xFFFFFFFFu, down, (2 * quad + c) * 4);
        const int pos = (R0 + 8 * t + 2 * quad + c) / G;
        seen[t][c] = p.memory_only ? s.seq : s.seq + pos + 1;
      }
    }
    float o[NT][DT][4], m[NT][2], mv[NT][2], l[NT][2];
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      m[t][0] = m[t][1] = mv[t][0] = mv[t][1] = kNone;
      l[t][0] = l[t][1] = 0.f;
#pragma unroll
      for (int d = 0; d < DT; ++d)
#pragma unroll
        for (int k = 0; k < 4; ++k) o[t][d][k] = 0.f;
    }

#pragma unroll 1
    for (int i0 = 0; i0 < steps; i0 += ST) {
#pragma unroll
      for (int u = 0; u < ST; ++u) {
        const int i = i0 + u;
        if (i >= steps) break;
        issue(ek_q[(u + ST - 1) % ST], ev_q[(u + ST - 1) % ST]);
        copy_wait<ST - 1>();
        const int slot = (tile0 + i) * kTile + warp * 16;
        if (slot >= seen_hi || ek_q[u] < 0) continue;
        const uint8_t *st = smem + warp * L::RING + (i % ST) * L::STAGE;
        // ---- S^T: keys n8, n8 + 8 x rows 2 quad, 2 quad + 1
        float sc[NT][4];
#pragma unroll
        for (int t = 0; t < NT; ++t) sc[t][0] = sc[t][1] = sc[t][2] = sc[t][3] = 0.f;
#pragma unroll
        for (int h = 0; h < KP / 2; ++h) {
          const uint4 ua = *reinterpret_cast<const uint4 *>(st + (h * 32 + lane) * 16);
          const uint4 ub = *reinterpret_cast<const uint4 *>(st + ((KP / 2 + h) * 32 + lane) * 16);
          const uint32_t wa[4] = {ua.x, ua.y, ua.z, ua.w}, wb[4] = {ub.x, ub.y, ub.z, ub.w};
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const uint32_t a0 = widen2(wa[j]), a2 = widen2(wa[j] >> 16);
            const uint32_t a1 = widen2(wb[j]), a3 = widen2(wb[j] >> 16);
#pragma unroll
            for (int t = 0; t < NT; ++t)
              mma_f16(sc[t], a0, a1, a2, a3, qb[t][4 * h + j][0], qb[t][4 * h + j][1]);
          }
        }
        // ---- scores in the log2 domain, against the references
        const float kf = __uint_as_float((uint32_t)ek_q[u] << 23);
        const float lv = (float)(ev_q[u] - 127);
        const bool mask = slot + 16 > seen_lo;   // uniform over the warp
        bool over = false;
#pragma unroll
        for (int t = 0; t < NT; ++t) {
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            sc[t][k] *= qf[t][k & 1] * kf;
            if (mask && slot + n8 + 8 * (k >> 1) >= seen[t][k & 1]) sc[t][k] = -INFINITY;
          }
#pragma unroll
          for (int c = 0; c < 2; ++c)
            over |= fmaxf(sc[t][c], sc[t][2 + c]) - m[t][c] > fminf(kSumLimit, kTop - (lv + m[t][c] - mv[t][c]));
        }
        if (__any_sync(0xFFFFFFFFu, over)) {
#pragma unroll
          for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int c = 0; c < 2; ++c) {
              float x = fmaxf(sc[t][c], sc[t][2 + c]);
              x = fmaxf(x, __shfl_xor_sync(0xFFFFFFFFu, x, 4));
              x = fmaxf(x, __shfl_xor_sync(0xFFFFFFFFu, x, 8));
              x = ceilf(fmaxf(x, __shfl_xor_sync(0xFFFFFFFFu, x, 16)));
              const float m1 = fmaxf(m[t][c], x), mv1 = fmaxf(mv[t][c], x + lv - kHead);
              l[t][c] *= ex2(m[t][c] - m1);
              const float f = ex2(mv[t][c] - mv1);
              m[t][c] = m1;
              mv[t][c] = mv1;
#pragma unroll
              for (int d = 0; d < DT; ++d) {
                o[t][d][c] *= f;
                o[t][d][2 + c] *= f;
              }
            }
        }
        uint32_t pb[NT][2];
#pragma unroll
        for (int t = 0; t < NT; ++t) {
          float y[4];
#pragma unroll
          for (int c = 0; c < 2; ++c) {
            const float f = ex2(lv + m[t][c] - mv[t][c]);
            const float p0 = ex2(sc[t][c] - m[t][c]), p1 = ex2(sc[t][2 + c] - m[t][c]);
            l[t][c] += p0 + p1;
            y[c] = p0 * f;
            y[2 + c] = p1 * f;
          }
          pb[t][0] = transpose8(pack_f16x2(y[0], y[1]));   // rows of P^T: keys
          pb[t][1] = transpose8(pack_f16x2(y[2], y[3]));
        }
        // ---- O^T += V^T P^T
        uint32_t w[4][VW];
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const uint8_t *src = st + KP * 512 + (r * 32 + lane) * L::VB;
          if constexpr (VW == 4)
            *reinterpret_cast<uint4 *>(w[r]) = *reinterpret_cast<const uint4 *>(src);
          else
            *reinterpret_cast<uint2 *>(w[r]) = *reinterpret_cast<const uint2 *>(src);
        }
#pragma unroll
        for (int j = 0; j < VW; ++j)
#pragma unroll
          for (int h = 0; h < 2; ++h) {   // bytes 4 j + 2 h, + 1 of the rows: M tile 2 j + h
            const uint32_t sel = h ? 0x7362u : 0x5140u;
            const uint32_t lo = __byte_perm(w[0][j], w[1][j], sel), hi = __byte_perm(w[2][j], w[3][j], sel);
            const uint32_t a0 = widen2(lo), a1 = widen2(lo >> 16), a2 = widen2(hi), a3 = widen2(hi >> 16);
#pragma unroll
            for (int t = 0; t < NT; ++t) mma_f16(o[t][2 * j + h], a0, a1, a2, a3, pb[t][0], pb[t][1]);
          }
      }
    }

    // ---- the four warps' rows meet
    copy_wait<0>();
    __syncthreads();   // every warp is done with its ring
    float *so = reinterpret_cast<float *>(smem);   // [warp][row][DH]
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        float x = l[t][c];
        x += __shfl_xor_sync(0xFFFFFFFFu, x, 4);
        x += __shfl_xor_sync(0xFFFFFFFFu, x, 8);
        x += __shfl_xor_sync(0xFFFFFFFFu, x, 16);
        const int row = 8 * t + 2 * quad + c;
        if (n8 == 0) {
          s_m[warp][row] = m[t][c];
          s_mv[warp][row] = mv[t][c];
          s_l[warp][row] = x;
        }
        float4 *dst = reinterpret_cast<float4 *>(so + (warp * L::ROWS + row) * DH + n8 * L::VB);
#pragma unroll
        for (int j = 0; j < VW; ++j)
          dst[j] = make_float4(o[t][2 * j][c], o[t][2 * j][2 + c], o[t][2 * j + 1][c], o[t][2 * j + 1][2 + c]);
      }
    __syncthreads();
    const bool whole = tile0 == 0 && tile1 == sq.tiles;
    // a unit in several shares: what this one has of it, after (0) or from (1) its start
    const long long slot = 2ll * cta + (first && tile0 > 0 ? 0 : 1);
    for (int i = tid; i < L::ROWS * DH / 2; i += kWarps * 32) {
      const int R = i / (DH / 2), d = (i - R * (DH / 2)) * 2;
      const RowAt r = row_at(p, s, g, R0 + R);
      if (!r.live) continue;
      float mt = kNone, mvt = kNone, lt = 0.f, o0 = 0.f, o1 = 0.f;
#pragma unroll
      for (int w = 0; w < kWarps; ++w) {
        mt = fmaxf(mt, s_m[w][R]);
        mvt = fmaxf(mvt, s_mv[w][R]);
      }
#pragma unroll
      for (int w = 0; w < kWarps; ++w) {   // a warp without keys holds zeros
        lt += s_l[w][R] * ex2(s_m[w][R] - mt);
        const float f = ex2(s_mv[w][R] - mvt);
        const float2 x = *reinterpret_cast<const float2 *>(so + (w * L::ROWS + R) * DH + d);
        o0 = fmaf(f, x.x, o0);
        o1 = fmaf(f, x.y, o1);
      }
      if (whole) {
        store2<T>(p, r, d, DH, o0, o1, mt, mvt, lt);
      } else {
        *reinterpret_cast<float2 *>(p.part_o + (slot * L::ROWS + R) * DH + d) = make_float2(o0, o1);
        if (d == 0) p.part_ml[slot * L::ROWS + R] = make_float4(mt, mvt, lt, 0.f);
      }
    }
    __syncthreads();   // the rows are read: the ring may be refilled
    at += tile1 - tile0;
    first = false;
  }
}

// Joins the shares of a unit, one row of it per CTA, in share order: kGroups
// groups of DH / 2 threads take every kGroups-th share.  CTA (c, row) joins the
// unit that the boundary between shares c and c + 1 cuts, if it is the first
// that does.
constexpr int kGroups = 4;

template <typename T, int DH, int NT>
__global__ void __launch_bounds__(kGroups * DH / 2)
    kv_combine_kernel(const __grid_constant__ KvAttnParams p) {
  constexpr int ROWS = 8 * NT;
  __shared__ float2 part[kGroups][DH / 2];
  __shared__ float part_l[kGroups];
  pdl_trigger();
  pdl_wait();
  const int c0 = blockIdx.x, R = blockIdx.y;
  const long long total = total_tiles<NT>(p);
  const int n_ctas = sharing_ctas(p, total);
  if (c0 + 1 >= n_ctas) return;
  const long long cut = total * (c0 + 1) / n_ctas;   // the first tile of the next share
  long long before;
  const int b = find_tile<NT>(p, cut, before);
  if (b >= p.rows.batch) return;
  const SeqPlan sq = seq_plan<NT>(p, b);
  const int unit = (int)((cut - before) / sq.tiles), g = unit / sq.groups, grp = unit - g * sq.groups;
  const long long t0 = before + (long long)unit * sq.tiles;
  if (t0 == cut || cta_of_tile(t0, total, n_ctas) != c0) return;
  const RowAt r = row_at(p, sq.s, g, grp * ROWS + R);
  if (!r.live) return;
  const int c1 = cta_of_tile(t0 + sq.tiles - 1, total, n_ctas);
  const int part_id = threadIdx.x / (DH / 2), d = (threadIdx.x - part_id * (DH / 2)) * 2;
  // share c0 holds the unit's start, those after it start inside the unit
  auto slot = [&](int c) { return (2ll * c + (c == c0 ? 1 : 0)) * ROWS + R; };
  float m = kNone, mv = kNone;
  for (int c = c0 + (threadIdx.x & 31); c <= c1; c += 32) {
    const float4 x = p.part_ml[slot(c)];
    m = fmaxf(m, x.x);
    mv = fmaxf(mv, x.y);
  }
  m = warp_max(m);
  mv = warp_max(mv);
  float l = 0.f, o0 = 0.f, o1 = 0.f;
#pragma unroll 4
  for (int c = c0 + part_id; c <= c1; c += kGroups) {
    const float4 x = p.part_ml[slot(c)];
    const float2 v = *reinterpret_cast<const float2 *>(p.part_o + slot(c) * DH + d);
    l += x.z * ex2(x.x - m);
    const float f = ex2(x.y - mv);
    o0 = fmaf(f, v.x, o0);
    o1 = fmaf(f, v.y, o1);
  }
  part[part_id][d / 2] = make_float2(o0, o1);
  if (d == 0) part_l[part_id] = l;
  __syncthreads();
  if (part_id > 0) return;
  l = o0 = o1 = 0.f;
#pragma unroll
  for (int k = 0; k < kGroups; ++k) {
    l += part_l[k];
    o0 += part[k][d / 2].x;
    o1 += part[k][d / 2].y;
  }
  store2<T>(p, r, d, DH, o0, o1, m, mv, l);
}

template <typename T, int DH, int NT>
cudaError_t launch_as(const KvAttnParams &p, cudaStream_t st) {
  using L = KvSmem<DH, NT>;
  auto kern = kv_attn_kernel<T, DH, NT>;
  static bool attr_set[64] = {};
  int dev = 0;
  cudaGetDevice(&dev);
  if (dev < 64 && !attr_set[dev]) {
    const cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, L::BYTES);
    if (e != cudaSuccess) return e;
    attr_set[dev] = true;
  }
  kern<<<(unsigned)p.ctas, kWarps * 32, L::BYTES, st>>>(p);
  cudaError_t e = cudaGetLastError();
  if (e != cudaSuccess) return e;
  return launch_pdl(kv_combine_kernel<T, DH, NT>, dim3((unsigned)p.ctas, L::ROWS),
                    dim3(kGroups * DH / 2), 0, st, p);
}
template <typename T, int DH>
cudaError_t launch_nt(const KvAttnParams &p, cudaStream_t st) {
  switch (p.nt) {
    case 1: return launch_as<T, DH, 1>(p, st);
    case 2: return launch_as<T, DH, 2>(p, st);
    case 4: return launch_as<T, DH, 4>(p, st);
    default: return cudaErrorInvalidValue;
  }
}
template <typename T>
cudaError_t launch_dh(const KvAttnParams &p, cudaStream_t st) {
  return p.head_dim == 128 ? launch_nt<T, 128>(p, st) : launch_nt<T, 64>(p, st);
}

// A slot's 16 elements of K and V per thread.
__global__ void __launch_bounds__(256)
    kv_block_copy_kernel(const __grid_constant__ KvAttnParams p, uint16_t *ko, uint16_t *vo, int32_t *ends) {
  const int dh = p.head_dim, chunks = p.hkv * dh / 16, cap = p.rows.cap;
  const long long idx = (long long)blockIdx.x * blockDim.x + threadIdx.x;
  if (idx >= (long long)p.rows.batch * cap * chunks) return;
  const long long row = idx / chunks;
  const int c = (int)(idx - row * chunks);
  const int b = (int)(row / cap), i = (int)(row - (long long)b * cap);
  const SeqRows s = seq_rows(p.rows, b, !p.memory_only);
  const int end = s.ok ? s.seq + (p.memory_only ? 0 : s.count) : 0;
  if (i == 0 && c == 0) {
    ends[b] = end;
    if (!s.ok) set_status(p.status, CC_ERR_DEVICE_ARG);
  }
  if (i >= end || s.count == 0) return;
  const int h = c * 16 / dh, e = c * 16 - h * dh;
  const long long vec = kv_vec(p.pg, cap, b, h, i);
  const size_t dst = (size_t)row * p.hkv * dh + (size_t)h * dh + e;
  if (vec < 0) {
    set_status(p.status, CC_ERR_DEVICE_ARG);
    return;
  }
  const long long ei = p.pg.head_major ? vec / p.block : vec / p.hkv / p.block * p.hkv + h;
  auto convert = [&](const uint8_t *in, int exp, uint16_t *out) {
    const uint4 x = *reinterpret_cast<const uint4 *>(in);
    const uint32_t w[4] = {x.x, x.y, x.z, x.w};
    const float f = __uint_as_float((uint32_t)exp << 23);
    uint32_t o[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const uint32_t h2 = widen2(w[j / 2] >> (16 * (j & 1)));
      const float2 y = __half22float2(*reinterpret_cast<const __half2 *>(&h2));
      o[j] = pack_bf16x2(y.x * f, y.y * f);
    }
    uint4 *d = reinterpret_cast<uint4 *>(out);
    d[0] = make_uint4(o[0], o[1], o[2], o[3]);
    d[1] = make_uint4(o[4], o[5], o[6], o[7]);
  };
  convert(p.k + vec * dh + e, p.ke[ei], ko + dst);
  convert(p.v + vec * dh + e, p.ve[ei], vo + dst);
}

}  // namespace

void kv_attn_plan(KvAttnParams &p, int sms) {
  const long long rows = (long long)p.rows.max_rows * (p.hq / p.hkv);
  p.nt = rows <= 8 ? 1 : rows <= 16 ? 2 : 4;
  p.ctas = sms * (p.nt == 4 ? 2 : 3);
}

size_t kv_attn_part_bytes(const KvAttnParams &p) {
  return (size_t)2 * p.ctas * 8 * p.nt * (p.head_dim * sizeof(float) + sizeof(float4));
}

cudaError_t launch_kv_attn(const KvAttnParams &p, cudaStream_t st) {
  if (p.head_dim != 64 && p.head_dim != 128) return cudaErrorInvalidValue;
  return p.f16 ? launch_dh<__half>(p, st) : launch_dh<__nv_bfloat16>(p, st);
}

cudaError_t launch_kv_block_copy(const KvAttnParams &p, void *ko, void *vo, int32_t *ends,
                                 cudaStream_t st) {
  const long long n = (long long)p.rows.batch * p.rows.cap * (p.hkv * p.head_dim / 16);
  const long long blocks = (n + 255) / 256;
  if (blocks > 0x7FFFFFFFll) return cudaErrorInvalidValue;
  kv_block_copy_kernel<<<(unsigned)blocks, 256, 0, st>>>(
      p, reinterpret_cast<uint16_t *>(ko), reinterpret_cast<uint16_t *>(vo), ends);
  return cudaGetLastError();
}

}  // namespace cc
