// kvattn.cu -- attention of a few query rows per sequence over a paged cache of
// e4m3 codes with a power-of-two scale for each block of slots and KV head.
//
// With x_j = q . K_j 2^ek_j log2(e) / sqrt(dh) and lv_j the V exponent,
//   out = sum_j 2^(x_j + lv_j) code_j / sum_j 2^x_j,
// in one pass over the keys with two running references per row: m for the
// sum below, so that 2^(x - m) neither overflows nor vanishes, and mv for the sum
// above, so that the largest 2^(x + lv - mv) fills fp16, in which the
// probabilities meet the codes (exact in fp16) on the tensor cores.  Both are
// whole numbers: every rescaling is by a power of two.  mv is held as dv = mv - m, which
// stays exact where scores are past 2^24.  Queries come to fp16 scaled by a
// power of two per row: exact but for elements more than 2^24 (fp16 rows: 2^21) below the row's
// largest, which are off by at most 2^-32 of that one; sums are fp32.  A bf16 row's
// probabilities are one fp16 each (out against 64 bits 0.00165, with fp32 ones 0.00163).
//
// Bound by the cache's bytes: a tcgen05 tile of 128 query rows would be
// nearly all padding, so the products are m16n8k16 with the keys (then the head
// dimension) on the M side and the 8 * NT query rows of a unit (the heads of a KV head
// at consecutive positions) on the N side: S^T = K Q^T, O^T = V^T P^T.  The key
// tiles of 64 of all units of a KV head are one long line, cut into equal shares so
// that ragged batches balance; the KV heads' CTAs of a share are neighbours, so that
// the pieces of a slot are read at about one time.  A unit that spans shares is
// joined by kv_combine_kernel in share order.
//
// Each warp streams its own 16 keys a step through a ring of its own (cp.async, no
// barrier wider than the warp).  A copy takes whole 128-byte lines: with the two
// halves of a line in two instructions the same stream ran at 5.1 instead of 6.9 TB/s.
// Which element of a row meets which k index is free as long as Q agrees, so a lane
// reads 16 bytes of a K row as four k steps' operands; transposing V is a byte
// permute of two rows' words before they are widened.  The 16 keys are taken in an
// order (row_of) in which, with the rows' pieces swizzled, neither product's reads
// meet in a bank.
//
// 64 ragged sequences of 1500 to 32767 slots, a row each, 32/8 heads: 2.25 GB in 345 us
// (6.5 TB/s); one of 8192 slots, 28/4 heads: 12.3 us, of which the stream is 1.3.  Units
// of 24 rows wait for their own latencies (40 % of the issue slots): 16 sequences' 5 rows of
// fp16, 153 MB in 59 us.
#include "kvattn.cuh"

#include <algorithm>
#include <type_traits>

namespace cc {

namespace {

constexpr int kWarps = 4;          // of a CTA, each every fourth 16 keys of a tile
constexpr int kTile = 16 * kWarps; // keys of a tile
constexpr int kMinTiles = 4;       // of a share at least
constexpr int kGroups = 8;         // of the join
// What a unit costs besides its tiles (its queries, the first loads' latency, its
// rows at the end: 5 to 6 us where a tile takes 1), in tiles.
constexpr int kUnitTiles = 5;
constexpr uint32_t kNoScale = 255;   // a scale exponent: elements that are no numbers (0: a scale of 0)
constexpr uint32_t kNanCodes = 0x7F7F7F7Fu;
constexpr uint32_t kBadPage = 0xFFFFFFFFu;   // in place of the scales' place: nothing to see
constexpr float kNone = -3.402823466e38f;   // reference of a row that has seen no key: the lowest fp32
constexpr float kFar = 0x1p22f;    // of a reference from which scores are rounded before it is taken off
constexpr float kSumLimit = 64.f;  // log2 of a term of the sum below
constexpr float kTop = 15.f, kHead = 8.f;   // log2 of a term above: limit, and what a new reference leaves

// CTAs per SM.  More streams in flight cost DRAM more than they hide: 64 ragged
// sequences, 2.25 GB: two 344 us (6.5 TB/s), three 384, four 414.
constexpr int kResident = 2;

template <int DH, int NT>
struct KvSmem {
  static constexpr int HALF = 16 * DH;            // bytes of K (or V) of a warp's stage
  static constexpr int STAGE = 2 * HALF + 16;     // and a word of K's scales, of V's, their place in it
  static constexpr int VB = DH / 8;               // bytes of a V row that a lane reads
  static constexpr int PIECES = DH / 16;          // 16-byte pieces of a row
  static constexpr int RPC = 32 / PIECES;         // rows of one copy instruction of the warp
  static constexpr int ST = 3;                    // (four: 7 % slower)
  static constexpr int RING = ST * STAGE;         // bytes of a warp's ring
  // piece c of row r: eight consecutive pieces of 128 bytes differ for the
  // rows that are read at once
  CC_DEV static int at(int r, int c) {
    return DH == 128 ? r * DH + ((c ^ (r & 7)) << 4) : r * DH + ((c ^ ((r >> 1) & 3)) << 4);
  }
  static constexpr int ROWS = 8 * NT;
  static constexpr int MERGE = ROWS * DH * 4;     // a warp's partial rows
  static constexpr int WARP = RING > MERGE ? RING : MERGE;
  // the queries as operands: in registers, or past 16 rows in shared memory
  static constexpr bool Q_SHARED = NT > 2;
  static constexpr int OFF_Q = kWarps * WARP;
  static constexpr int BYTES = OFF_Q + (Q_SHARED ? NT * (DH / 16) * 32 * 8 : 0);
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
CC_DEV uint32_t nan_bytes(uint32_t w) {   // 0xFF in every byte of w that is a NaN code
  return __vcmpeq4(w & kNanCodes, kNanCodes);
}
// Key of index n of the products' 16: odd ones half an 8-row group away.
CC_DEV int row_of(int n) { return n ^ ((n & 1) << 2); }
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
CC_DEV void copy16(uint32_t dst, const void *src) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}
CC_DEV void copy4(uint32_t dst, const void *src, int bytes) {   // fewer than 4: zeros after them
  asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(dst), "l"(src), "r"(bytes) : "memory");
}
// From src + off where it is there, else zeros (then src, which is, is named but not read).
CC_DEV void copy16_if(uint32_t dst, const uint8_t *src, int off, bool there) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src + (there ? off : 0)),
               "r"(there ? 16 : 0) : "memory");
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
// Tiles of a sequence's units of one KV head on the line, each unit's own after
// kUnitTiles for its cost, and of all sequences'.  A whole warp calls the latter.
CC_DEV long long seq_tiles(const SeqPlan &q) {
  return (long long)q.groups * (q.tiles + kUnitTiles);
}
template <int NT>
CC_DEV long long total_tiles(const KvAttnParams &p) {
  long long all = 0;
  for (int b = threadIdx.x & 31; b < p.rows.batch; b += 32) all += seq_tiles(seq_plan<NT>(p, b));
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
    const long long w = b0 + lane < p.rows.batch ? seq_tiles(seq_plan<NT>(p, b0 + lane)) : 0;
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
// Shares of the line of `total` tiles where `resident` are worked on at once; share
// c starts at total * c / n.  (Three times as many shorter ones, so that a slower SM
// takes fewer, measured within 1 %.)
__host__ __device__ __forceinline__ int line_shares(int resident, long long total) {
  const long long few = (total + kMinTiles - 1) / kMinTiles;
  return few >= resident ? resident : few < 1 ? 1 : (int)few;
}
CC_DEV int share_of_tile(long long t, long long total, int n) {   // the last c with total * c / n <= t
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

// What the sum above of a row is multiplied by: 2^dv / l as two factors,
// neither of which leaves fp32's range (0 for a row without a finite sum below).
struct OutScale {
  float a, b;
};
CC_DEV OutScale out_scale(float dv, float l) {
  if (!(l > 0.f && l < INFINITY)) return {0.f, 0.f};
  const int shift = min(max((int)dv, -250), 250), half = shift / 2;
  return {__uint_as_float((uint32_t)(127 + half) << 23) / l, __uint_as_float((uint32_t)(127 + shift - half) << 23)};
}
CC_DEV float row_lse(float m, float l) {
  return l == 0.f ? -INFINITY : (m + log2f(l)) * 0.69314718055994531f;
}

// ---------------------------------------------------------------------------
// the kernel
// ---------------------------------------------------------------------------
template <typename T, int DH, int NT>
__global__ void __launch_bounds__(kWarps * 32, kResident)
    kv_attn_kernel(const __grid_constant__ KvAttnParams p) {
  using L = KvSmem<DH, NT>;
  constexpr int KS = DH / 16;        // k steps of K Q^T
  constexpr int DT = DH / 16;        // M tiles of V^T P^T
  constexpr int ST = L::ST, VW = DH / 32;
  // an fp16 output would show the probabilities' rounding: two fp16 parts of each
  // (out against 64 bits 2.9e-4 with one, 2.1e-4 with two, the output's own rounding)
  constexpr bool PAIRS = std::is_same_v<T, __half>;
  extern __shared__ __align__(16) uint8_t smem[];
  __shared__ float s_m[kWarps][L::ROWS], s_dv[kWarps][L::ROWS], s_l[kWarps][L::ROWS];
  __shared__ float4 s_f[L::ROWS];
  __shared__ float s_b[L::ROWS];
  __shared__ long long s_to[L::ROWS];
  static_assert(kWarps == 4, "a row's weights are a float4");
  pdl_trigger();   // the combine may launch: it waits for this grid
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, n8 = lane >> 2, quad = lane & 3;
  const long long total = total_tiles<NT>(p);
  const int n_shares = min(p.shares, line_shares(p.resident, total)), cta = blockIdx.x;
  const int share = cta / p.hkv, g = cta - share * p.hkv;
  int4 cut = make_int4(0, -1, 0, 0);   // the unit that starts here and goes on in the next share
  if (share >= n_shares) {
    if (tid == 0 && !p.spread) p.cut[cta] = cut;
    return;
  }
  long long at = total * share / n_shares;
  const long long end = total * (share + 1) / n_shares;
  // reported once, by the first CTA: sequences whose rows or lengths are bad
  if (cta == 0)
    for (int b = tid; b < p.rows.batch; b += kWarps * 32)
      if (!seq_rows(p.rows, b, !p.memory_only).ok) set_status(p.status, CC_ERR_DEVICE_ARG);
  long long before = 0;
  int b = at < end ? find_tile<NT>(p, at, before) : 0;   // (below the batch: at < total)
  const uint32_t ring = smem_u32(smem) + warp * L::RING;
  const int hs = p.pg.head_major ? 1 : p.hkv, step = hs * DH;   // bytes from a slot to the next
  const int log_block = 31 - __clz(p.block);
  SeqPlan sq = seq_plan<NT>(p, b);
  bool first = true;   // the share's first segment
  while (at < end) {
    while (before + seq_tiles(sq) <= at) {   // the next sequence with rows
      before += seq_tiles(sq);
      sq = seq_plan<NT>(p, ++b);
    }
    const long long in_seq = at - before;
    const int span = sq.tiles + kUnitTiles;
    const int grp = (int)(in_seq / span), from = (int)(in_seq - (long long)grp * span);
    const int to = (int)min((long long)span, from + (end - at));
    const long long unit_at = at - from;
    at += to - from;
    const int tile0 = max(0, from - kUnitTiles), tile1 = to - kUnitTiles;
    if (tile1 <= 0) break;   // the share ends before the unit's first tile
    const SeqRows s = sq.s;
    const int gs = p.pg.head_major ? 0 : g;
    const int G = p.hq / p.hkv, R0 = grp * L::ROWS;
    // seen slots of the group's first and last row
    const int last_pos = min(s.count - 1, (R0 + L::ROWS - 1) / G);
    const int seen_lo = p.memory_only ? s.seq : s.seq + R0 / G + 1;
    const int seen_hi = p.memory_only ? s.seq : s.seq + last_pos + 1;

    // ---- the ring of 16-key steps of this warp: step i is keys
    // (tile0 + i) * 64 + 16 warp + [0, 16), which lie in one page
    int next = tile0 * kTile + warp * 16;   // slot of the next step to issue
    const int steps = min(tile1 - tile0, max(0, seen_hi - next + kTile - 1) / kTile);
    // where slot 0 (of the page) of this head lies, and the step's slot in it
    const int crow = lane / L::PIECES, cpiece = lane % L::PIECES;   // of this lane's copies
    const long long lane_off = (long long)crow * step + cpiece * 16;
    const uint8_t *kb, *vb;
    long long e0;   // of the slot's (page's) first scale exponent
    int off = next, page = 0, page_end = 0x7FFFFFFF;
    bool ok = true;
    auto enter = [&](long long row0) {   // rows of hs vectors, of which this head's is the gs-th
      const long long vec = row0 * hs + gs;
      kb = p.k + vec * DH + lane_off;
      vb = p.v + vec * DH + lane_off;
      e0 = (row0 >> log_block) * hs + gs;
    };
    auto enter_page = [&]() {
      const int e = p.pg.table[(long long)b * p.pg.pages_per_seq + page];
      ok = e >= 0 && e < p.pg.n_pages;
      enter(ok ? (long long)e * p.pg.page : 0);
    };
    if (p.pg.table) {
      page = next / p.pg.page;
      off = next - page * p.pg.page;
      page_end = p.pg.page;
      if (steps > 0) enter_page();
    } else {
      enter(p.pg.head_major ? ((long long)b * p.hkv + g) * p.rows.cap : (long long)b * p.rows.cap);
    }
    int left_to_issue = steps;
    uint32_t write_at = 0, read_at = 0;   // stages of the ring
    auto issue = [&]() {
      if (left_to_issue > 0) {
        --left_to_issue;
        const uint32_t dst = ring + write_at;
        write_at = write_at + L::STAGE == L::RING ? 0 : write_at + L::STAGE;
        if (off >= page_end) {
          off -= page_end;
          ++page;
          enter_page();
        }
        if (!ok && lane == 0) set_status(p.status, CC_ERR_DEVICE_ARG);
        // the block's scale exponents: the aligned words that hold them
        const long long eo = e0 + (long long)(off >> log_block) * hs;
        if (ok && lane < 2)
          copy4(dst + 2 * L::HALF + lane * 4, (lane ? p.ve : p.ke) + (eo & ~3ll),
                (int)min(4ll, p.exp_bytes - (eo & ~3ll)));
        if (lane == 0)
          asm volatile("st.shared.u32 [%0], %1;" ::"r"(dst + 2 * L::HALF + 8),
                       "r"(ok ? (uint32_t)(eo & 3) * 8 : kBadPage) : "memory");
        if (ok) {
          const uint8_t *kp = kb + (long long)off * step, *vp = vb + (long long)off * step;
          const int left = seen_hi - next;
          if (left >= 16) {
#pragma unroll
            for (int c = 0; c < 16 / L::RPC; ++c) {
              const int to = L::at(crow + c * L::RPC, cpiece), from = c * L::RPC * step;
              copy16(dst + to, kp + from);
              copy16(dst + L::HALF + to, vp + from);
            }
          } else {   // what lies past the end reads as zeros
#pragma unroll
            for (int c = 0; c < 16 / L::RPC; ++c) {
              const int row = crow + c * L::RPC, to = L::at(row, cpiece);
              // (the step's first row is there: named from there)
              copy16_if(dst + to, kp - lane_off, (int)lane_off + c * L::RPC * step, row < left);
              copy16_if(dst + L::HALF + to, vp - lane_off, (int)lane_off + c * L::RPC * step, row < left);
            }
          }
        }
        off += kTile;
        next += kTile;
      }
      copy_commit();
    };
#pragma unroll 1
    for (int i = 0; i < ST - 1; ++i) issue();

    // ---- queries: row 8 t + n8 of the group as the second operand, fp16,
    // scaled to a largest magnitude of [2^7, 2^8)
    uint32_t qb[L::Q_SHARED ? 1 : NT][KS][2];
    uint2 *q_sh = reinterpret_cast<uint2 *>(smem + L::OFF_Q);   // [NT][KS][lane]
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
        const uint32_t b0 = pack_f16x2(x[4 * k] * up, x[4 * k + 1] * up);
        const uint32_t b1 = pack_f16x2(x[4 * k + 2] * up, x[4 * k + 3] * up);
        if constexpr (L::Q_SHARED) {
          if (t % kWarps == warp) q_sh[(t * KS + k) * 32 + lane] = make_uint2(b0, b1);
        } else {
          qb[t][k][0] = b0;
          qb[t][k][1] = b1;
        }
      }
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        qf[t][c] = __shfl_sync(0xFFFFFFFFu, down, (2 * quad + c) * 4);
        const int pos = (R0 + 8 * t + 2 * quad + c) / G;
        seen[t][c] = p.memory_only ? s.seq : s.seq + pos + 1;
      }
    }
    if constexpr (L::Q_SHARED) __syncthreads();
    float o[NT][DT][4], m[NT][2], dv[NT][2], l[NT][2];
    bool far = false;   // a reference of this lane's rows is past kFar
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      m[t][0] = m[t][1] = kNone;
      dv[t][0] = dv[t][1] = l[t][0] = l[t][1] = 0.f;
#pragma unroll
      for (int d = 0; d < DT; ++d)
#pragma unroll
        for (int k = 0; k < 4; ++k) o[t][d][k] = 0.f;
    }

    // where this lane reads in a stage: K row row_of(n8), piece quad (+ 4); V rows
    // row_of(2 quad), row_of(2 quad + 1), bytes n8 * VB
    const int k_at = L::at(row_of(n8), quad);
    int v_at[2];
#pragma unroll
    for (int r = 0; r < 2; ++r)
      v_at[r] = L::at(row_of(2 * quad + r), n8 * L::VB / 16) + n8 * L::VB % 16;
#pragma unroll 1   // (one copy of the body: four overran the instruction cache)
    for (int i = 0; i < steps; ++i) {
      copy_wait<ST - 2>();
      __syncwarp();   // every lane's copies of this step; every lane is done with the last one
      issue();
      const int slot = (tile0 + i) * kTile + warp * 16;
      const uint8_t *st = smem + warp * L::RING + read_at;
      read_at = read_at + L::STAGE == L::RING ? 0 : read_at + L::STAGE;
      const uint4 ew = *reinterpret_cast<const uint4 *>(st + 2 * L::HALF);
      if (ew.z == kBadPage) continue;
      const uint32_t ek = (ew.x >> ew.z) & 255u, ev = (ew.y >> ew.z) & 255u;
      // ---- S^T: keys n8, n8 + 8 x rows 2 quad, 2 quad + 1
      float sc[NT][4];
#pragma unroll
      for (int t = 0; t < NT; ++t) sc[t][0] = sc[t][1] = sc[t][2] = sc[t][3] = 0.f;
#pragma unroll
      for (int h = 0; h < DH / 64; ++h) {
        const uint4 ua = *reinterpret_cast<const uint4 *>(st + (k_at ^ (h * 64)));
        const uint4 ub = *reinterpret_cast<const uint4 *>(st + 8 * DH + (k_at ^ (h * 64)));
        const uint32_t wa[4] = {ua.x, ua.y, ua.z, ua.w}, wb[4] = {ub.x, ub.y, ub.z, ub.w};
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const uint32_t a0 = widen2(wa[j]), a2 = widen2(wa[j] >> 16);
          const uint32_t a1 = widen2(wb[j]), a3 = widen2(wb[j] >> 16);
#pragma unroll
          for (int t = 0; t < NT; ++t) {
            if constexpr (L::Q_SHARED) {
              const uint2 q2 = q_sh[(t * KS + 4 * h + j) * 32 + lane];
              mma_f16(sc[t], a0, a1, a2, a3, q2.x, q2.y);
            } else {
              mma_f16(sc[t], a0, a1, a2, a3, qb[t][4 * h + j][0], qb[t][4 * h + j][1]);
            }
          }
        }
      }
      // ---- scores in the log2 domain, against the references
      const float scale_k = __uint_as_float(ek << 23), kf = fmaf(scale_k, 0.f, scale_k);   // (e = 255: NaN)
      const float lv = (float)((int)ev - 127);
      const bool mask = slot + 16 > seen_lo;   // uniform over the warp
      float qk[NT][2];   // what makes them scores: 1 where they are scores already
#pragma unroll
      for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int c = 0; c < 2; ++c) qk[t][c] = qf[t][c] * kf;
      if (mask || far) {
#pragma unroll
        for (int t = 0; t < NT; ++t) {
#pragma unroll
          for (int k = 0; k < 4; ++k)
            sc[t][k] = slot + row_of(n8) + 8 * (k >> 1) >= seen[t][k & 1] ? -INFINITY : sc[t][k] * qk[t][k & 1];
          qk[t][0] = qk[t][1] = 1.f;
        }
      }
      const float room = kTop - lv;
      bool over = false;
#pragma unroll
      for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int c = 0; c < 2; ++c)
          over |= fmaf(fmaxf(sc[t][c], sc[t][2 + c]), qk[t][c], -m[t][c]) > fminf(kSumLimit, dv[t][c] + room);
      if (__any_sync(0xFFFFFFFFu, over)) {
        far = false;
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
          for (int c = 0; c < 2; ++c) {
            float x = fmaxf(sc[t][c], sc[t][2 + c]) * qk[t][c];
            x = fmaxf(x, __shfl_xor_sync(0xFFFFFFFFu, x, 4));
            x = fmaxf(x, __shfl_xor_sync(0xFFFFFFFFu, x, 8));
            x = ceilf(fmaxf(x, __shfl_xor_sync(0xFFFFFFFFu, x, 16)));
            const float m1 = fmaxf(m[t][c], x), fall = m[t][c] - m1;
            const float dv1 = fmaxf(dv[t][c] + fall, x - m1 + (lv - kHead));
            l[t][c] = m1 < INFINITY ? l[t][c] * ex2(fall) : NAN;   // (a score past fp32)
            const float f = ex2(dv[t][c] + fall - dv1);
            m[t][c] = m1;
            dv[t][c] = dv1;
            far |= fabsf(m1) >= kFar && m1 > kNone;
#pragma unroll
            for (int d = 0; d < DT; ++d) {
              o[t][d][c] *= f;
              o[t][d][2 + c] *= f;
            }
          }
        if (far) {   // the product's rounding, which counts here, is to be the reference's
#pragma unroll
          for (int t = 0; t < NT; ++t) {
#pragma unroll
            for (int k = 0; k < 4; ++k) sc[t][k] *= qk[t][k & 1];
            qk[t][0] = qk[t][1] = 1.f;
          }
        }
      }
      uint32_t pb[NT][2], pl[PAIRS ? NT : 1][2];
#pragma unroll
      for (int t = 0; t < NT; ++t) {
        float y[4];
#pragma unroll
        for (int c = 0; c < 2; ++c) {
          // (finite: a key of probability 0 may have any scale)
          const float f = ex2(fminf(lv - dv[t][c], 126.f));
          const float p0 = ex2(fmaf(sc[t][c], qk[t][c], -m[t][c])), p1 = ex2(fmaf(sc[t][2 + c], qk[t][c], -m[t][c]));
          l[t][c] += p0 + p1;
          y[c] = p0 * f;
          y[2 + c] = p1 * f;
        }
#pragma unroll
        for (int k = 0; k < 2; ++k) {   // rows of P^T: keys
          const uint32_t hi = pack_f16x2(y[2 * k], y[2 * k + 1]);
          pb[t][k] = transpose8(hi);
          if constexpr (PAIRS) {
            const float2 f = __half22float2(*reinterpret_cast<const __half2 *>(&hi));
            pl[t][k] = transpose8(pack_f16x2(y[2 * k] - f.x, y[2 * k + 1] - f.y));
          }
        }
      }
      // ---- O^T += V^T P^T
      uint32_t w[4][VW];
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const uint8_t *src = st + L::HALF + (r >> 1) * 8 * DH + v_at[r & 1];
        if constexpr (VW == 4)
          *reinterpret_cast<uint4 *>(w[r]) = *reinterpret_cast<const uint4 *>(src);
        else
          *reinterpret_cast<uint2 *>(w[r]) = *reinterpret_cast<const uint2 *>(src);
      }
      if (mask || ev - 1u >= kNoScale - 1u) {
        if (ev - 1u >= kNoScale - 1u) {   // a scale of 0, or none: codes that say so
#pragma unroll
          for (int r = 0; r < 4; ++r)
#pragma unroll
            for (int j = 0; j < VW; ++j) w[r][j] = ev ? kNanCodes : nan_bytes(w[r][j]) & kNanCodes;
        }
        // keys that some rows do not see: a NaN among their values may reach only
        // the rows that do (0 times NaN is NaN), so it leaves the product
        uint32_t any = 0;
#pragma unroll
        for (int r = 0; r < 4; ++r)
#pragma unroll
          for (int j = 0; j < VW; ++j) any |= nan_bytes(w[r][j]);
        if (__any_sync(0xFFFFFFFFu, any != 0)) {
          uint32_t bits[4];   // of row r: which of the lane's VB values
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            bits[r] = 0;
#pragma unroll
            for (int j = 0; j < VW; ++j) {
              const uint32_t x = nan_bytes(w[r][j]);
              w[r][j] &= ~x;
              bits[r] |= ((x & 1u) | ((x >> 7) & 2u) | ((x >> 14) & 4u) | ((x >> 21) & 8u)) << (4 * j);
            }
          }
#pragma unroll 1
          for (int k = 0; k < 4; ++k) {   // of the quad's lane k, which holds keys of its own
            uint32_t hit[4];
#pragma unroll
            for (int r = 0; r < 4; ++r) hit[r] = __shfl_sync(0xFFFFFFFFu, bits[r], (lane & ~3) | k);
#pragma unroll
            for (int t = 0; t < NT; ++t)
#pragma unroll
              for (int c = 0; c < 2; ++c) {
                uint32_t here = 0;
#pragma unroll
                for (int r = 0; r < 4; ++r)
                  here |= slot + row_of(2 * k + (r & 1)) + 8 * (r >> 1) < seen[t][c] ? hit[r] : 0u;
#pragma unroll
                for (int d = 0; d < L::VB; ++d)
                  if ((here >> d) & 1u) o[t][d >> 1][(d & 1) * 2 + c] = NAN;
              }
          }
        }
      }
#pragma unroll
      for (int j = 0; j < VW; ++j)
#pragma unroll
        for (int h = 0; h < 2; ++h) {   // bytes 4 j + 2 h, + 1 of the rows: M tile 2 j + h
          const uint32_t sel = h ? 0x7362u : 0x5140u;
          const uint32_t lo = __byte_perm(w[0][j], w[1][j], sel), hi = __byte_perm(w[2][j], w[3][j], sel);
          const uint32_t a0 = widen2(lo), a1 = widen2(lo >> 16), a2 = widen2(hi), a3 = widen2(hi >> 16);
#pragma unroll
          for (int t = 0; t < NT; ++t) {
            mma_f16(o[t][2 * j + h], a0, a1, a2, a3, pb[t][0], pb[t][1]);
            if constexpr (PAIRS) mma_f16(o[t][2 * j + h], a0, a1, a2, a3, pl[t][0], pl[t][1]);
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
          s_dv[warp][row] = dv[t][c];
          s_l[warp][row] = x;
        }
        float4 *dst = reinterpret_cast<float4 *>(so + (warp * L::ROWS + row) * DH + n8 * L::VB);
#pragma unroll
        for (int j = 0; j < VW; ++j)
          dst[j] = make_float4(o[t][2 * j][c], o[t][2 * j][2 + c], o[t][2 * j + 1][c], o[t][2 * j + 1][2 + c]);
      }
    __syncthreads();
    const bool whole = tile0 == 0 && tile1 == sq.tiles;
    if (tile0 == 0 && (!whole || p.spread)) {
      cut = make_int4(share, share_of_tile(unit_at + span - 1, total, n_shares), b, grp);
      if (p.spread && tid == 0) p.cut[((long long)b * p.most_groups + grp) * p.hkv + g] = cut;
    }
    // a unit in several shares: what this one has of it, after (0) or from (1) its start
    const long long part = (2ll * cta + (first && tile0 > 0 ? 0 : 1)) * L::ROWS;
    if (tid < L::ROWS) {   // per row: the warps' weights, and where it goes
      const RowAt r = row_at(p, s, g, R0 + tid);
      float mt = kNone, dvt = -INFINITY, lt = 0.f, f[kWarps];
#pragma unroll
      for (int w = 0; w < kWarps; ++w) mt = fmaxf(mt, s_m[w][tid]);
#pragma unroll
      for (int w = 0; w < kWarps; ++w) {   // a warp without keys holds zeros
        const float fall = s_m[w][tid] - mt;
        lt += s_l[w][tid] * ex2(fall);
        f[w] = s_dv[w][tid] + fall;
        dvt = fmaxf(dvt, f[w]);
      }
#pragma unroll
      for (int w = 0; w < kWarps; ++w) f[w] = ex2(f[w] - dvt);
      OutScale k{1.f, 1.f};
      long long to = r.live ? (part + tid) * DH : -1;
      if (whole) {
        k = out_scale(dvt, lt);
        if (r.live) to = r.row * p.out_ld + (long long)r.head * DH;
        if (r.live && p.lse) p.lse[(long long)r.row * p.hq + r.head] = row_lse(mt, lt);
      } else {
        p.part_ml[part + tid] = make_float4(mt, dvt, lt, 0.f);
      }
      s_f[tid] = make_float4(f[0] * k.a, f[1] * k.a, f[2] * k.a, f[3] * k.a);
      s_b[tid] = k.b;
      s_to[tid] = to;
    }
    __syncthreads();
#pragma unroll
    for (int i0 = 0; i0 < L::ROWS * DH / 4; i0 += kWarps * 32) {
      const int i = i0 + tid, R = i / (DH / 4), d = (i - R * (DH / 4)) * 4;
      const long long to = s_to[R];
      if (to < 0) continue;
      const float4 f = s_f[R];
      float4 y = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
      for (int w = 0; w < kWarps; ++w) {
        const float4 x = *reinterpret_cast<const float4 *>(so + (w * L::ROWS + R) * DH + d);
        const float fw = w == 0 ? f.x : w == 1 ? f.y : w == 2 ? f.z : f.w;
        y = make_float4(fmaf(fw, x.x, y.x), fmaf(fw, x.y, y.y), fmaf(fw, x.z, y.z), fmaf(fw, x.w, y.w));
      }
      if (whole) {
        const float k = s_b[R];
        // (0 times an infinite sum would be NaN: such a row is 0)
        const bool zero = k == 0.f;
        *reinterpret_cast<uint2 *>(reinterpret_cast<T *>(p.out) + to + d) =
            zero ? make_uint2(0u, 0u) : make_uint2(pack2<T>(y.x * k, y.y * k), pack2<T>(y.z * k, y.w * k));
      } else {
        *reinterpret_cast<float4 *>(p.part_o + to + d) = y;
      }
    }
    __syncthreads();   // the rows are read: the ring may be refilled
    first = false;
  }
  if (tid == 0 && !p.spread) p.cut[cta] = cut;
}

// Joins the shares of a unit that starts in share c0 and goes on past it, as that
// share's CTA wrote it down, in share order.  SPREAD (few units, of many shares): a CTA
// per unit and row, its kGroups groups of DH / 2 threads each take every kGroups-th
// share; else CTAs per share, a group per row.  A group loads eight shares at a time; in
// the second form, where a unit has a few and many CTAs find none, four, so that two
// CTAs fit an SM (16 sequences' 5 rows: fp16 62.1 -> 60.1 us, bf16 57.0 -> 55.0; two at a
// time and four CTAs: the same, and single rows 1 us slower).
template <typename T, int DH, int NT, bool SPREAD>
__global__ void __launch_bounds__(kGroups * DH / 2, SPREAD ? 1 : 1024 / (kGroups * DH / 2))
    kv_combine_kernel(const __grid_constant__ KvAttnParams p) {
  constexpr int ROWS = 8 * NT, kJoin = SPREAD ? 8 : 4;
  __shared__ float4 part[SPREAD ? kGroups : 1][DH / 2];   // m, dv and the two sums
  __shared__ float part_l[kGroups];
  const int group = threadIdx.x / (DH / 2), d = (threadIdx.x - group * (DH / 2)) * 2;
  const int R = SPREAD ? blockIdx.y : blockIdx.y * kGroups + group;
  const int unit = blockIdx.x / p.hkv, g = blockIdx.x - unit * p.hkv;
  pdl_trigger();
  pdl_wait();
  // (SPREAD: a unit without rows was not written down)
  const int b = SPREAD ? unit / p.most_groups : 0, grp = unit - b * p.most_groups;
  RowAt r{0, 0, false};
  if (SPREAD && R < ROWS) r = row_at(p, seq_rows(p.rows, b, !p.memory_only), g, grp * ROWS + R);
  if (SPREAD && !r.live) return;
  const int4 u = p.cut[blockIdx.x];   // first and last share; sequence and group of rows
  const int c0 = u.x, c1 = u.y;
  if (c1 <= c0 || R >= ROWS) return;
  // (the row is needed last: its lookup runs beside the loads)
  if (!SPREAD) r = row_at(p, seq_rows(p.rows, u.z, !p.memory_only), g, u.w * ROWS + R);
  // share c0 holds the unit's start, those after it start inside the unit
  auto slot = [&](int c) { return (2ll * ((long long)c * p.hkv + g) + (c == c0 ? 1 : 0)) * ROWS + R; };
  constexpr int STEP = SPREAD ? kGroups : 1;
  float m = kNone, dv = 0.f, l = 0.f, o0 = 0.f, o1 = 0.f;
  auto join = [&](float xm, float xdv, float xl, float x0, float x1) {
    const float m1 = fmaxf(m, xm), fall = m - m1, x_fall = xm - m1;
    const float a = dv + fall, b = xdv + x_fall, dv1 = fmaxf(a, b);
    l = l * ex2(fall) + xl * ex2(x_fall);
    const float f = ex2(a - dv1), g = ex2(b - dv1);
    o0 = o0 * f + x0 * g;
    o1 = o1 * f + x1 * g;
    m = m1;
    dv = dv1;
  };
#pragma unroll 1
  for (int c = c0 + (SPREAD ? group : 0); c <= c1; c += kJoin * STEP) {
    float4 x[kJoin];
    float2 v[kJoin];
#pragma unroll
    for (int k = 0; k < kJoin; ++k)
      if (c + k * STEP <= c1) {
        x[k] = p.part_ml[slot(c + k * STEP)];
        v[k] = *reinterpret_cast<const float2 *>(p.part_o + slot(c + k * STEP) * DH + d);
      }
#pragma unroll
    for (int k = 0; k < kJoin; ++k)
      if (c + k * STEP <= c1) join(x[k].x, x[k].y, x[k].z, v[k].x, v[k].y);
  }
  if constexpr (SPREAD) {
    part[group][d / 2] = make_float4(m, dv, o0, o1);
    if (d == 0) part_l[group] = l;
    __syncthreads();
    if (group > 0) return;
#pragma unroll
    for (int k = 1; k < kGroups; ++k) {
      const float4 x = part[k][d / 2];
      join(x.x, x.y, part_l[k], x.z, x.w);
    }
  }
  if (!r.live) return;
  const OutScale k = out_scale(dv, l);
  *reinterpret_cast<uint32_t *>(reinterpret_cast<T *>(p.out) + r.row * p.out_ld + (long long)r.head * DH + d) =
      k.b == 0.f ? 0u : pack2<T>(o0 * k.a * k.b, o1 * k.a * k.b);
  if (p.lse && d == 0) p.lse[(long long)r.row * p.hq + r.head] = row_lse(m, l);
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
  const unsigned rows = (unsigned)std::min<long long>(L::ROWS, (long long)p.rows.max_rows * (p.hq / p.hkv));
  if (p.spread)
    return launch_pdl(kv_combine_kernel<T, DH, NT, true>,
                      dim3((unsigned)(p.rows.batch * p.most_groups * p.hkv), rows), dim3(kGroups * DH / 2),
                      0, st, p);
  return launch_pdl(kv_combine_kernel<T, DH, NT, false>, dim3((unsigned)p.ctas, (rows + kGroups - 1) / kGroups),
                    dim3(kGroups * DH / 2), 0, st, p);
}
template <typename T, int DH>
cudaError_t launch_nt(const KvAttnParams &p, cudaStream_t st) {
  switch (p.nt) {
    case 1: return launch_as<T, DH, 1>(p, st);
    case 2: return launch_as<T, DH, 2>(p, st);
    case 3: return launch_as<T, DH, 3>(p, st);
    case 4: return launch_as<T, DH, 4>(p, st);
    default: return cudaErrorInvalidValue;
  }
}
template <typename T>
cudaError_t launch_dh(const KvAttnParams &p, cudaStream_t st) {
  return p.head_dim == 128 ? launch_nt<T, 128>(p, st) : launch_nt<T, 64>(p, st);
}

// ---------------------------------------------------------------------------
// around the tile attention
// ---------------------------------------------------------------------------
// How the tile attention's CTAs, one per SM at a time, share its units.  Nearly equal
// units stay whole as far as they fill the SMs evenly; what is left of them, or all where
// they differ, is left whole, cut into equal pieces while there are SMs for each, or
// laid end to end as a line that is cut into one share per SM, whichever has the
// least estimate: key tiles of 1.45 us and what pieces cost besides.  Units in step, on
// the same key tiles, share them in L2, which only the line gives up.  Longest pieces
// come first, so that the SMs, which take them in order, end at about one time.
// Against as many equal pieces of every unit as SMs allow (none past one wave), 32/8
// heads: 2048 rows after 14336 slots 407 -> 385 us, after 129024 3.10 -> 2.82 ms; eight
// chunks of 1 to 2000 rows 315 -> 230; three of fp16, 100 to 30000 slots, 802 -> 250; four
// equal ones 263 -> 269 and 128 rows after 2048 slots 36 -> 39 (the join's launch, the plan).
constexpr int kPieceCost = 5;    // of a piece besides its key tiles, in tiles (7 us)
constexpr int kPieceTiles = 4;   // of a piece at least
constexpr int kJoinCost = 4, kJoinParts = 25;   // the join: its launch, and partial rows a tile
constexpr int kLineCost = 2 * kPieceCost + 22;  // of the line: two pieces an SM, the join, uneven ends
constexpr int kPlanThreads = 256, kPlanBins = 64;

__device__ __noinline__ void plan_tiles(const KvAttnParams &p, const KvTilePlan &t) {
  __shared__ int s_unit[kTilePlanBatch + 1], s_at[kTilePlanBatch + 1];   // a sequence's first, and the end
  __shared__ int s_seq[kTilePlanBatch], s_count[kTilePlanBatch], s_bin[kPlanBins];
  __shared__ int s_most, s_pieces, s_parts, s_joins;
  const int tid = threadIdx.x, batch = p.rows.batch, P = t.P, heads = p.hkv, sms = t.sms;
  // key tiles of position block i
  auto tiles_of = [&](int seq, int count, int i) {
    const int n = p.memory_only ? seq : seq + count, last = seq + min((i + 1) * P, count) - 1;
    return n > 0 ? min(last, n - 1) / 128 + 1 : 0;
  };
  if (tid == 0) s_most = s_pieces = s_parts = s_joins = s_unit[0] = s_at[0] = 0;
  if (tid < kPlanBins) s_bin[tid] = 0;
  __syncthreads();
  if (tid < batch) {
    const SeqRows s = seq_rows(p.rows, tid, !p.memory_only);
    s_seq[tid] = s.seq;
    s_count[tid] = s.count;
    const int blocks = (s.count + P - 1) / P;
    int weight = 0;
    for (int i = 0; i < blocks; ++i) weight += tiles_of(s.seq, s.count, i) + kPieceCost;
    if (blocks) atomicMax(&s_most, tiles_of(s.seq, s.count, blocks - 1));
    s_unit[tid + 1] = blocks * heads;
    s_at[tid + 1] = weight * heads;
  }
  __syncthreads();
#pragma unroll 1
  for (int o = 1; o < batch; o *= 2) {   // running sums
    const int u = tid >= o && tid < batch ? s_unit[tid + 1 - o] : 0, w = tid >= o && tid < batch ? s_at[tid + 1 - o] : 0;
    __syncthreads();
    if (tid < batch) {
      s_unit[tid + 1] += u;
      s_at[tid + 1] += w;
    }
    __syncthreads();
  }
  // (more units than fit: sequences share rows, which is reported; no sum is used then)
  const int units = min(s_unit[batch], t.units), all = s_at[batch], most = s_most;
  struct Unit {
    int id, tiles, at;
  };
  auto unit_at = [&](int j) {
    int b = 0;
#pragma unroll 1
    for (int o = kTilePlanBatch / 2; o; o /= 2)
      if (b + o < batch && s_unit[b + o] <= j) b += o;
    const int seq = s_seq[b], count = s_count[b], blocks = (count + P - 1) / P;
    const int r = j - s_unit[b], g = r / blocks, i = r - g * blocks;
    Unit u{(i * batch + b) * heads + g, tiles_of(seq, count, i), s_at[b] + (s_at[b + 1] - s_at[b]) / heads * g};
#pragma unroll 1
    for (int k = 0; k < i; ++k) u.at += tiles_of(seq, count, k) + kPieceCost;
    return u;
  };
  const int top = most + kPieceCost;
  const bool even = 4ll * top * s_unit[batch] <= 5ll * all;   // none a quarter above the mean
  const int whole = even ? units / sms * sms : 0, rest = units - whole;
  const int from = rest > 0 ? unit_at(whole).at : all;
  const int share = max((all - from + sms - 1) / sms, kPieceTiles);
  // estimates
  const int equal = even && rest > 0 ? min(sms / rest, most / kPieceTiles) : 1;
  const int uncut = rest <= sms ? top : share + top / 2;
  const int in_equal = most / max(equal, 1) + kPieceCost + kJoinCost + rest * equal / kJoinParts;
  const int in_line = share + share / 16 + kLineCost;
  const bool sound = rest > 0 && s_unit[batch] <= t.units;
  const bool line = sound && in_line < uncut && (equal < 2 || in_line < in_equal);
  const bool equally = sound && !line && equal > 1 && in_equal < uncut;
  int4 *raw = t.pieces + t.n_pieces;
  const float per_tile = (kPlanBins - 1) / (float)max(most, 1);
  auto bin_of = [&](int tiles) { return max(0, kPlanBins - 1 - (int)((float)tiles * per_tile)); };
#pragma unroll 1
  for (int j = tid; j < units; j += kPlanThreads) {
    const Unit u = unit_at(j);
    auto walk = [&](auto piece) {
      int last = 0, k = 0;
      if (j >= whole && line) {
        const int x = u.at - from;
        for (int y = (x / share + 1) * share - x - kPieceCost; y <= u.tiles - kPieceTiles; y += share)
          if (y >= last + kPieceTiles) {
            piece(k++, last, y - last);
            last = y;
          }
      } else if (j >= whole && equally) {
        for (int to = 1; to < equal; ++to) {
          const int y = (int)((long long)u.tiles * to / equal);
          if (y - last >= kPieceTiles && u.tiles - y >= kPieceTiles) {
            piece(k++, last, y - last);
            last = y;
          }
        }
      }
      piece(k++, last, u.tiles - last);
      return k;
    };
    const int n = walk([](int, int, int) {});
    const int at = atomicAdd(&s_pieces, n), part = n > 1 ? atomicAdd(&s_parts, n) : -1;
    if (at + n > t.n_pieces || part + n > 2 * sms) continue;   // (never: there are fewer cuts than SMs)
    walk([&](int k, int off, int tiles) {
      raw[at + k] = make_int4(u.id, off, tiles, n > 1 ? part + k : -1);
      atomicAdd(&s_bin[bin_of(tiles)], 1);
    });
    if (n > 1) {
      const int to = atomicAdd(&s_joins, 1);
      if (to < t.n_joins) t.joins[to] = make_int4(u.id, part, n, 0);
    }
  }
  __syncthreads();
  const int pieces = min(s_pieces, t.n_pieces);
  for (int i = s_joins + tid; i < t.n_joins; i += kPlanThreads) t.joins[i] = make_int4(-1, 0, 0, 0);
  for (int i = pieces + tid; i < t.n_pieces; i += kPlanThreads) t.pieces[i] = make_int4(-1, 0, 0, -1);
  int before = 0;   // pieces of longer bins
  if (tid < kPlanBins)
    for (int i = 0; i < tid; ++i) before += s_bin[i];
  __syncthreads();
  if (tid < kPlanBins) s_bin[tid] = before;
  __syncthreads();
  for (int i = tid; i < pieces; i += kPlanThreads) {
    const int4 x = raw[i];
    t.pieces[atomicAdd(&s_bin[bin_of(x.z)], 1)] = x;
  }
}
static_assert(kTilePlanBatch <= kPlanThreads && kPlanBins <= kPlanThreads, "a thread a sequence, and a bin");

// 16 elements of K and of V per thread (four, all loads ahead, changed no time by more
// than 2 %).  Registers for eight CTAs per SM, which the plan alone exceeds: with five
// the copy of 130000 slots took 13 us more.
__global__ void __launch_bounds__(256, 8)
    kv_block_copy_kernel(const __grid_constant__ KvAttnParams p, uint16_t *ko, uint16_t *vo, KvTileRows t,
                         const __grid_constant__ KvTilePlan plan, int per_seq) {
  int block = blockIdx.x;
  if (plan.pieces && block-- == 0) {
    plan_tiles(p, plan);
    return;
  }
  const int dh = p.head_dim, chunks = p.hkv * dh / 16, cap = p.rows.cap;
  const int b = block / per_seq;
  const uint32_t idx = (uint32_t)(block - b * per_seq) * 256u + threadIdx.x;   // in the sequence
  const int i = (int)(idx / chunks), c = (int)(idx - (uint32_t)i * chunks);
  const long long row = (long long)b * cap + i;
  const SeqRows s = seq_rows(p.rows, b, !p.memory_only);
  if (i == 0 && c == 0) {
    t.lo[b] = s.ok ? s.seq : 0;
    t.hi[b] = s.ok ? s.seq + s.count : 0;
    t.base[b] = s.r0;
    if (!s.ok) set_status(p.status, CC_ERR_DEVICE_ARG);
  }
  if (s.count == 0 || i >= s.seq + (p.memory_only ? 0 : s.count)) return;   // (at most cap)
  const int h = c * 16 / dh, e = c * 16 - h * dh;
  const long long vec = kv_vec(p.pg, cap, b, h, i);
  const size_t dst = (size_t)row * p.hkv * dh + (size_t)h * dh + e;
  if (vec < 0) set_status(p.status, CC_ERR_DEVICE_ARG);
  const long long at = vec < 0 ? 0 : vec;
  const long long ei = p.pg.head_major ? at / p.block : at / p.hkv / p.block * p.hkv + h;
  auto convert = [&](const uint8_t *in, int exp, bool clean, uint16_t *out) {
    const uint4 x = *reinterpret_cast<const uint4 *>(in);
    uint32_t w[4] = {x.x, x.y, x.z, x.w};
    const bool none = exp == (int)kNoScale;
    const float f = none ? 1.f : __uint_as_float((uint32_t)exp << 23);
    uint32_t o[8];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      if (none) w[j] = kNanCodes;
      if (clean) w[j] &= ~nan_bytes(w[j]);
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        const uint32_t h2 = widen2(w[j] >> (16 * k));
        const float2 y = __half22float2(*reinterpret_cast<const __half2 *>(&h2));
        o[2 * j + k] = pack_bf16x2(y.x * f, y.y * f);
      }
    }
    uint4 *d = reinterpret_cast<uint4 *>(out);
    d[0] = make_uint4(o[0], o[1], o[2], o[3]);
    d[1] = make_uint4(o[4], o[5], o[6], o[7]);
  };
  // (the slots of a bad page: keys of NaN, so that the rows that see them are 0)
  convert(p.k + at * dh + e, vec < 0 ? (int)kNoScale : p.ke[ei], false, ko + dst);
  convert(p.v + at * dh + e, vec < 0 ? 0 : p.ve[ei], i >= s.seq || vec < 0, vo + dst);
}

// 16 values of a new token and KV head per thread: where they hold NaN codes, the
// outputs of the token's own and the later rows of its sequence get NaN, but for rows
// that are 0 (a score that is no number: their lse is none either).
template <typename T>
__global__ void __launch_bounds__(256) kv_restore_nan_kernel(const __grid_constant__ KvAttnParams p) {
  const int dh = p.head_dim, chunks = p.hkv * dh / 16, G = p.hq / p.hkv;
  const long long idx = (long long)blockIdx.x * 256 + threadIdx.x;
  const int r = (int)(idx / chunks), c = (int)(idx - (long long)r * chunks), lane = threadIdx.x & 31;
  // Whose row it is: every sequence is looked at, a lane each, for the few rows of the warp in
  // turn (where some are bad, row_start is not in order).
  int b = -1;
  const int last = min(__shfl_sync(0xFFFFFFFFu, r, 31), p.rows.n_rows - 1);
  for (int row = __shfl_sync(0xFFFFFFFFu, r, 0); row <= last; ++row)
    for (int b0 = 0; b0 < p.rows.batch; b0 += 32) {
      bool in = false;
      if (b0 + lane < p.rows.batch) {
        const SeqRows s = seq_rows(p.rows, b0 + lane, true);
        in = row >= s.r0 && row < s.r0 + s.count;
      }
      const unsigned hit = __ballot_sync(0xFFFFFFFFu, in);
      if (!hit) continue;
      if (row == r) b = b0 + __ffs(hit) - 1;
      break;
    }
  if (b < 0) return;
  const SeqRows s = seq_rows(p.rows, b, true);
  const int g = c * 16 / dh, e = c * 16 - g * dh;
  const long long vec = kv_vec(p.pg, p.rows.cap, b, g, s.seq + r - s.r0);
  if (vec < 0) return;
  const long long ei = p.pg.head_major ? vec / p.block : vec / p.hkv / p.block * p.hkv + g;
  const bool none = p.ve[ei] == kNoScale;
  const uint4 u = *reinterpret_cast<const uint4 *>(p.v + vec * dh + e);
  if (!none && !(nan_bytes(u.x) | nan_bytes(u.y) | nan_bytes(u.z) | nan_bytes(u.w))) return;
  const T nan = std::is_same_v<T, __half> ? T(__ushort_as_half(0x7FFF)) : T(__ushort_as_bfloat16(0x7FFF));
  for (int d = 0; d < 16; ++d) {
    if (!none && (p.v[vec * dh + e + d] & 0x7F) != 0x7F) continue;
    for (int i = r; i < s.r0 + s.count; ++i)
      for (int h = 0; h < G; ++h)
        if (fabsf(p.lse[(long long)i * p.hq + g * G + h]) < INFINITY)
          reinterpret_cast<T *>(p.out)[i * p.out_ld + (long long)(g * G + h) * dh + e + d] = nan;
  }
}

// 8 elements per thread.
__global__ void __launch_bounds__(256)
    kv_split_rows_kernel(const __grid_constant__ KvAttnParams p, __nv_bfloat16 *pairs) {
  const int width = p.hq * p.head_dim, per = width / 8;
  const long long idx = (long long)blockIdx.x * blockDim.x + threadIdx.x;
  if (idx >= (long long)p.rows.n_rows * per) return;
  const long long r = idx / per;
  const int e = (int)(idx - r * per) * 8;
  const uint4 u = *reinterpret_cast<const uint4 *>(reinterpret_cast<const __half *>(p.q) + r * p.q_ld + e);
  const uint32_t w[4] = {u.x, u.y, u.z, u.w};
  uint32_t hi[4], lo[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float2 x = __half22float2(*reinterpret_cast<const __half2 *>(&w[i]));
    hi[i] = pack_bf16x2(x.x, x.y);
    lo[i] = pack_bf16x2(pair_rest(x.x, bf16_lo(hi[i])), pair_rest(x.y, bf16_hi(hi[i])));
  }
  __nv_bfloat16 *dst = pairs + r * 2 * width + e;
  *reinterpret_cast<uint4 *>(dst) = make_uint4(hi[0], hi[1], hi[2], hi[3]);
  *reinterpret_cast<uint4 *>(dst + width) = make_uint4(lo[0], lo[1], lo[2], lo[3]);
}

}  // namespace

void kv_attn_plan(KvAttnParams &p, int sms) {
  const long long rows = (long long)p.rows.max_rows * (p.hq / p.hkv);
  p.nt = (int)std::min<long long>(4, (rows + 7) / 8);
  p.resident = std::max(1, sms * kResident / p.hkv);
  // (as if every sequence were as long as its buffer)
  const long long groups = (rows + 8 * p.nt - 1) / (8 * p.nt), tiles = (p.rows.cap + kTile - 1) / kTile + kUnitTiles;
  p.shares = line_shares(p.resident, p.rows.batch * groups * tiles);
  p.ctas = p.shares * p.hkv;
  p.spread = p.shares >= kGroups * p.rows.batch * groups;
  p.most_groups = (int)groups;
}

size_t kv_attn_part_bytes(const KvAttnParams &p) {
  return (size_t)2 * p.ctas * 8 * p.nt * (p.head_dim * sizeof(float) + sizeof(float4)) +
         p.ctas * sizeof(int4);
}
void kv_attn_bind(KvAttnParams &p, void *ws) {
  const size_t rows = (size_t)2 * p.ctas * 8 * p.nt;
  p.part_o = reinterpret_cast<float *>(ws);
  p.part_ml = reinterpret_cast<float4 *>(p.part_o + rows * p.head_dim);
  p.cut = reinterpret_cast<int4 *>(p.part_ml + rows);
}

cudaError_t launch_kv_attn(const KvAttnParams &p, cudaStream_t st) {
  if (p.head_dim != 64 && p.head_dim != 128) return cudaErrorInvalidValue;
  return p.f16 ? launch_dh<__half>(p, st) : launch_dh<__nv_bfloat16>(p, st);
}

cudaError_t launch_kv_block_copy(const KvAttnParams &p, void *ko, void *vo, const KvTileRows &t,
                                 const KvTilePlan &plan, cudaStream_t st) {
  const long long n = (long long)p.rows.cap * (p.hkv * p.head_dim / 16), per_seq = (n + 255) / 256;
  const long long blocks = per_seq * p.rows.batch + (plan.pieces ? 1 : 0);
  if (blocks > 0x7FFFFFFFll || n > 0xFFFFFF00ll) return cudaErrorInvalidValue;
  if (plan.pieces && p.rows.batch > kTilePlanBatch) return cudaErrorInvalidValue;
  kv_block_copy_kernel<<<(unsigned)blocks, 256, 0, st>>>(
      p, reinterpret_cast<uint16_t *>(ko), reinterpret_cast<uint16_t *>(vo), t, plan, (int)per_seq);
  return cudaGetLastError();
}

cudaError_t launch_kv_restore_nan(const KvAttnParams &p, cudaStream_t st) {
  const long long blocks = ((long long)p.rows.n_rows * (p.hkv * p.head_dim / 16) + 255) / 256;
  if (blocks > 0x7FFFFFFFll) return cudaErrorInvalidValue;
  if (p.f16) kv_restore_nan_kernel<__half><<<(unsigned)blocks, 256, 0, st>>>(p);
  else kv_restore_nan_kernel<__nv_bfloat16><<<(unsigned)blocks, 256, 0, st>>>(p);
  return cudaGetLastError();
}

cudaError_t launch_kv_split_rows(const KvAttnParams &p, void *pairs, cudaStream_t st) {
  const long long blocks = ((long long)p.rows.n_rows * p.hq * p.head_dim / 8 + 255) / 256;
  if (blocks > 0x7FFFFFFFll) return cudaErrorInvalidValue;
  kv_split_rows_kernel<<<(unsigned)blocks, 256, 0, st>>>(p, reinterpret_cast<__nv_bfloat16 *>(pairs));
  return cudaGetLastError();
}

}  // namespace cc
