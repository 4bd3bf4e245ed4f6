// kvreceived_tiles.cu -- the attention that the slots of a block-scaled cache receive
// from chunks of rows (kvreceived.cu has the definition, and few rows).
//
// The floor is the tensor cores' and, about as high, the exponentials': 128 slots are the
// M rows of a tcgen05 product and 96 query rows its N, so that a lane keeps the same slots
// from tile to tile, adds their weights in registers, and has their scales as factors.
// The key codes become bf16 (fp16 for fp16 rows; exact, without
// their scale) once per unit and stay in tensor memory as the A operand; the query
// tiles stream through shared memory by TMA, each for both of a CTA's slot tiles.
//
// A unit is 256 slots of one KV head against all query tiles that see them.  The units
// of all sequences form one line, each with a little for its start, cut into equal
// shares, a CTA per share; the sums of a unit that spans shares are added up in share
// order, then the heads' in theirs (finish_kernel): fixed orders, no atomics.
//
//   warps 0-7, 8-15  a slot tile each: codes to tensor memory, then per query tile the
//                    scores from tensor memory (four warps half of the columns), weights, sums
//   warps 16, 17     the products of a slot tile each, in two buffers of scores of its own
//                    (warp 17 has the tensor memory)
//   warp 18          query tiles (TMA)
//   warp 19          the rows' terms
//
// A chunk of 2048 rows behind 14336 slots, 32 query heads of 128 on 8: 221 us (1.17 PFLOP/s).  One
// behind 16384 slots took 241 us when the products alone took 150, tensor pipe and
// exponentials each busy half of the time, instructions issued in 63 % of it; without the slots'
// warps' arithmetic the hand-overs of a tile between the roles still took 215 us.
// A score's k steps are one chain of products: totals are 3.6e-7 off (300 fp16 rows of 28/4 heads 6.4e-7),
// where two chains a score keep few rows (kvreceived.cu) below 1.4e-6 and plain fp32 gives 2e-7.
// Measured slower: weights of a tile's 96 columns by every other four warps (277 us; a buffer
// of scores is held for longer), scores taken 16 columns at a time (298), the next unit's codes
// fetched ahead (the same).
//
// A row's y is its rounded part, which the scores' multiply-add takes off, and a factor
// e^-rest of its weights.
#include "kvreceived.cuh"

#include <type_traits>

namespace cc {

namespace {

constexpr int KT = 128;             // slots of a tile
constexpr int QT = 96;              // query rows of a tile: two buffers of scores for each of two slot tiles
constexpr int CH = QT / 2;          // of them (columns of the scores) a warp's
constexpr int kUnitSlots = 2 * KT;
constexpr int kStages = 6;
constexpr int kThreads = 640;
// Registers of a launch's 640 threads at 96 shared out anew between its five warpgroups.
constexpr int kRegsSlots = 104, kRegsOthers = 64;
static_assert(4 * kRegsSlots + kRegsOthers <= 5 * 96, "more registers than the block is launched with");
// Of a unit's start, in query tiles; and of one that some rows do not see, whose masked tiles take longer.
// (With 3 for both the last shares end 10 % behind the others: 276 against 250 us for a chunk of 2048 rows
// behind 16384 slots, 32 query heads of 128 on 8: the only shape at which the two were chosen.)
constexpr int kUnitCost = 5, kEdgeCost = 7;

template <int DH>
struct RtSmem {
  static constexpr int NH = DH / 64;                   // 64-column (128-byte) halves
  static constexpr int TILE = NH * QT * 128;
  static constexpr int OFF_Q = 0;
  // [stage][QT / 2] float4: of two query rows -y, -y, e^-rest, e^-rest
  static constexpr int OFF_TERM = OFF_Q + kStages * TILE;
  static constexpr int OFF_LIVE = OFF_TERM + kStages * QT * 8;     // [stage]: bit h: columns 48 h ... all add
  static constexpr int OFF_BAR = OFF_LIVE + kStages * 4;
  static constexpr int BYTES = OFF_BAR + 256 + 1024;               // barriers + alignment slack
};

// ---------------------------------------------------------------------------
// the line of units
// ---------------------------------------------------------------------------
struct SeqLine {
  SeqRows s;
  int keys;       // slots that some row sees
  int nk;         // units of a KV head
  int tiles;      // query tiles of a KV head
  int nfull;      // units (from the first) that all query tiles see
};
CC_DEV SeqLine seq_line(const KvReceivedParams &p, int b) {
  SeqLine q;
  q.s = seq_rows(p.rows, b, !p.memory_only);
  q.keys = q.s.count == 0 ? 0 : q.s.seq + (p.memory_only ? 0 : q.s.count);
  q.nk = (q.keys + kUnitSlots - 1) / kUnitSlots;
  q.tiles = (q.s.count + p.P - 1) / p.P;
  q.nfull = p.memory_only ? q.nk : min(q.nk, (q.s.seq + p.P - 1) / kUnitSlots + 1);
  return q;
}
// The first query tile that sees a slot of unit kt.
CC_DEV int first_tile(const KvReceivedParams &p, const SeqLine &q, int kt) {
  return p.memory_only ? 0 : max(0, kt * kUnitSlots - q.s.seq) / p.P;
}
CC_DEV long long seq_length(const KvReceivedParams &p, const SeqLine &q) {
  long long n = (long long)q.nfull * (q.tiles + kUnitCost);
  for (int kt = q.nfull; kt < q.nk; ++kt) n += q.tiles - first_tile(p, q, kt) + kEdgeCost;
  return n * p.hkv;
}
CC_DEV long long line_length(const KvReceivedParams &p) {   // a whole warp calls
  long long all = 0;
  for (int b = threadIdx.x & 31; b < p.rows.batch; b += 32) all += seq_length(p, seq_line(p, b));
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) all += __shfl_xor_sync(0xFFFFFFFFu, all, o);
  return all;
}
CC_DEV long long length_before(const KvReceivedParams &p, int seq) {   // a whole warp calls
  long long all = 0;
  for (int b = threadIdx.x & 31; b < seq; b += 32) all += seq_length(p, seq_line(p, b));
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) all += __shfl_xor_sync(0xFFFFFFFFu, all, o);
  return all;
}
__host__ __device__ __forceinline__ int line_shares(int most, long long total) { return total < most ? (int)total : most; }
CC_DEV int share_at(long long t, long long total, int n) {   // the last c with total * c / n <= t
  return (int)(((t + 1) * n - 1) / total);
}

// The pieces of units in a share, in order; every warp walks them for itself.
struct Pieces {
  long long at, end, before;   // position, the share's end, the line before sequence b
  int b;
  SeqLine q;
  // the piece: unit kt of KV head g, query tiles [t0, t1); where its sums go
  int kt, g, t0, t1;
  bool whole, begins;
  CC_DEV void start(const KvReceivedParams &p, long long total, int n, int share) {
    at = total * share / n;
    end = total * (share + 1) / n;
    before = 0;
    // the sequence that holds `at`, 32 at a time
    const int lane = threadIdx.x & 31;
    b = 0;
    for (int b0 = 0; b0 < p.rows.batch; b0 += 32) {
      const long long w = b0 + lane < p.rows.batch ? seq_length(p, seq_line(p, b0 + lane)) : 0;
      long long sum = w;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const long long x = __shfl_up_sync(0xFFFFFFFFu, sum, o);
        if (lane >= o) sum += x;
      }
      const unsigned past = __ballot_sync(0xFFFFFFFFu, before + sum > at);
      if (past) {
        const int k = __ffs(past) - 1;
        before += __shfl_sync(0xFFFFFFFFu, sum - w, k);
        b = b0 + k;
        break;
      }
      before += __shfl_sync(0xFFFFFFFFu, sum, 31);
    }
    q = seq_line(p, b);
  }
  CC_DEV bool next(const KvReceivedParams &p) {
    while (at < end) {
      long long x = at - before;
      const int span0 = q.tiles + kUnitCost;
      const long long full = (long long)q.nfull * p.hkv * span0;
      int span = span0, unit = 0, cost = kUnitCost;
      t0 = 0;
      if (x < full) {
        unit = (int)(x / span0);
        x -= (long long)unit * span0;
        kt = unit / p.hkv;
        g = unit - kt * p.hkv;
      } else {
        x -= full;
        cost = kEdgeCost;
        for (kt = q.nfull; kt < q.nk; ++kt) {
          t0 = first_tile(p, q, kt);
          span = q.tiles - t0 + kEdgeCost;
          if (x < (long long)span * p.hkv) break;
          x -= (long long)span * p.hkv;
        }
        if (kt >= q.nk) {   // the next sequence
          before += seq_length(p, q);
          q = seq_line(p, ++b);
          continue;
        }
        g = (int)(x / span);
        x -= (long long)g * span;
      }
      const int from = (int)x, to = (int)min((long long)span, x + (end - at));
      at += to - from;
      begins = from == 0;
      whole = begins && to == span;
      t1 = t0 + to - cost;
      t0 += max(0, from - cost);
      if (t1 > t0) return true;   // (else the share ends before the unit's first tile)
    }
    return false;
  }
};

// Two e4m3 codes (lo and hi byte of `two`) -> the operand type's pair, exact.  bf16: the code's bits shifted
// into place make the value times 2^-120 (NaN codes: see where they are found).
template <bool F16>
CC_DEV uint32_t widen2(uint32_t two) {
  uint32_t r;
  if constexpr (F16) {
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(r) : "h"((unsigned short)two));
  } else {
    const uint32_t x = __byte_perm(two, 0, 0x1404);   // a byte at the top of each half
    const uint32_t y = (x & 0x80008000u) | ((x >> 4) & 0x07F007F0u);
    const uint32_t scale = 0x7B807B80u;               // 2^120, twice
    const __nv_bfloat162 z = __hmul2(*reinterpret_cast<const __nv_bfloat162 *>(&y),
                                     *reinterpret_cast<const __nv_bfloat162 *>(&scale));
    r = *reinterpret_cast<const uint32_t *>(&z);
  }
  return r;
}

template <int DH, bool F16>
__global__ void __launch_bounds__(kThreads, 1)
    received_tiles_kernel(const __grid_constant__ KvReceivedParams p, const __grid_constant__ CUtensorMap tq) {
  using L = RtSmem<DH>;
  extern __shared__ uint8_t smem_raw[];
  uint8_t *smem = reinterpret_cast<uint8_t *>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  float4 *term_sh = reinterpret_cast<float4 *>(smem + L::OFF_TERM);
  volatile uint32_t *live_sh = reinterpret_cast<volatile uint32_t *>(smem + L::OFF_LIVE);
  uint64_t *q_full = reinterpret_cast<uint64_t *>(smem + L::OFF_BAR);   // [kStages]
  uint64_t *q_empty = q_full + kStages;                                 // [kStages]
  uint64_t *s_full = q_empty + kStages;                                 // [2 slot tiles][2]
  uint64_t *s_empty = s_full + 4;                                       // [2][2]
  uint64_t *a_full = s_empty + 4;                                       // [2]
  uint32_t *tmem_slot = reinterpret_cast<uint32_t *>(a_full + 2);
  __shared__ Pieces walk_sh[16];
  __shared__ float f_sh[2][2][2][KT];   // [piece's parity][slot tile][half of the codes][slot]
  volatile int *abort_flag = reinterpret_cast<volatile int *>(tmem_slot + 1);

  pdl_trigger();   // the finish may launch: it waits for this grid
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const long long total = line_length(p);
  const int n = line_shares(p.shares, total), share = blockIdx.x;
  if (share == 0)   // reported once: sequences whose rows or lengths are bad
    for (int b = threadIdx.x; b < p.rows.batch; b += kThreads)
      if (!seq_rows(p.rows, b, !p.memory_only).ok) set_status(p.status, CC_ERR_DEVICE_ARG);
  if (share >= n) return;

  if (threadIdx.x == 0) {
    for (int s = 0; s < kStages; ++s) {
      mbar_init(&q_full[s], 2);   // the copies, the terms
      mbar_init(&q_empty[s], 16);   // the slots' warps: they have seen the products' end and read the terms
    }
    for (int i = 0; i < 4; ++i) {
      mbar_init(&s_full[i], 1);
      mbar_init(&s_empty[i], 8);
    }
    for (int i = 0; i < 2; ++i) mbar_init(&a_full[i], 8);
    *abort_flag = 0;
    fence_barrier_init();
  }
  const int G = p.hq / p.hkv;
  {   // rows of a tile that hold no query: zeros, so that their scores are numbers
    const int pad = (QT - p.P * G) * 8;   // 16-byte pieces
    for (int i = threadIdx.x; i < pad * L::NH * kStages; i += kThreads)
      *reinterpret_cast<uint4 *>(smem + L::OFF_Q + (i / pad) * (QT * 128) + p.P * G * 128 + i % pad * 16) = make_uint4(0, 0, 0, 0);
    fence_proxy_async_smem();
  }
  if (warp == 17) tmem_alloc(tmem_slot, 512);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = *tmem_slot;
  Pieces u;
  u.start(p, total, n, share);

  if (warp >= 16) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kRegsOthers));
  if (warp == 18) {
    // ----------------------------------------------------------- query tiles
    if (lane == 0) tma_prefetch_desc(&tq);
    int it = 0;
    bool ok = true;
    while (ok && u.next(p)) {
      if (lane == 0)
        for (int t = u.t0; ok && t < u.t1; ++t, ++it) {
          const int s = it % kStages;
          if (!(ok = mbar_wait_short(&q_empty[s], ((it / kStages) & 1) ^ 1, abort_flag, p.status))) break;
          mbar_arrive_expect_tx(&q_full[s], (uint32_t)(L::NH * p.P * G * 128));
          for (int h = 0; h < L::NH; ++h)
            tma_load_3d(smem + L::OFF_Q + s * L::TILE + h * QT * 128, &tq, &q_full[s], h * 64, u.g * G,
                        u.q.s.r0 + t * p.P);
        }
      ok = __shfl_sync(0xFFFFFFFFu, ok ? 1 : 0, 0) != 0;
    }
  } else if (warp == 19) {
    // ------------------------------------ the rows' terms, their loads a tile ahead
    int pos[QT / 32], at[QT / 32];
#pragma unroll
    for (int i = 0; i < QT / 32; ++i) {
      const int col = lane + 32 * i;
      pos[i] = col / G;
      at[i] = pos[i] * p.hq + col - pos[i] * G;
      if (pos[i] >= p.P) pos[i] = 0x40000000;   // no row
    }
    int it = 0;
    bool ok = true;
    while (ok && u.next(p)) {
      const float *src = p.lse + (long long)u.q.s.r0 * p.hq + u.g * G;
      float next[QT / 32];
      auto load = [&](int t) {
        const int left = u.q.s.count - t * p.P;   // rows of the tile and on
#pragma unroll
        for (int i = 0; i < QT / 32; ++i)
          next[i] = t < u.t1 && pos[i] < left ? __ldg(src + (long long)t * p.P * p.hq + at[i]) : INFINITY;
      };
      load(u.t0);
      for (int t = u.t0; t < u.t1; ++t, ++it) {
        const int s = it % kStages;
        RowLse y[QT / 32];
        uint32_t dead = 0;   // bit h: a row of columns 48 h ... adds nothing
#pragma unroll
        for (int i = 0; i < QT / 32; ++i) {
          y[i] = row_lse(p, next[i]);
          // (or holds no query)
          const uint32_t adds = __ballot_sync(0xFFFFFFFFu, y[i].y < INFINITY || pos[i] >= p.P);
          const int c = 32 * i / CH;
          if (i % 3 == 1)
            dead |= ((adds & 0xFFFFu) != 0xFFFFu ? 1u << c : 0u) | (adds >> 16 != 0xFFFFu ? 2u << c : 0u);
          else
            dead |= adds != ~0u ? 1u << c : 0u;
        }
        load(t + 1);
        if (!(ok = mbar_wait_short(&q_empty[s], ((it / kStages) & 1) ^ 1, abort_flag, p.status))) break;
#pragma unroll
        for (int i = 0; i < QT / 32; ++i) {
          const int col = lane + 32 * i;
          float *term = reinterpret_cast<float *>(term_sh + s * (QT / 2) + col / 2) + (col & 1);
          term[0] = -y[i].y;
          term[2] = 1.f - y[i].rest + 0.5f * y[i].rest * y[i].rest;   // e^-rest, a small one
        }
        if (lane == 0) live_sh[s] = ~dead;
        __syncwarp();
        if (lane == 0) mbar_arrive(&q_full[s]);
      }
    }
  } else {
    // ------- products: a warp per slot tile, so that one's run while the other waits and starts
    constexpr uint32_t idesc = F16 ? make_idesc_f16(128, QT, 0, 0) : make_idesc_bf16(128, QT, 0, 0);
    const int w = warp - 16;
    int it = 0;
    unsigned job = 0, filled = 0;   // of this slot tile: products, times that its operand was
    bool ok = true;
    while (ok && u.next(p)) {
      const int n = u.t1 - u.t0;
      if (w == 1 && u.q.keys - u.kt * kUnitSlots <= KT) {   // no second tile of slots
        it += n;
        continue;
      }
      if (lane == 0) {
        ok = mbar_wait_short(&a_full[w], filled++ & 1, abort_flag, p.status);
        for (int i = 0; ok && i < n; ++i, ++it, ++job) {
          if (!(ok = mbar_wait_short(&q_full[it % kStages], (it / kStages) & 1, abort_flag, p.status) &&
                     mbar_wait_short(&s_empty[2 * w + (job & 1)], ((job >> 1) & 1) ^ 1, abort_flag, p.status)))
            break;
          tc_fence_after();
          const uint64_t qd = make_sdesc_sw128(smem_u32(smem + L::OFF_Q + it % kStages * L::TILE), 16, 1024);
          const uint32_t d = tmem + 128 + (2 * w + (job & 1)) * QT, a = tmem + w * 64;
#pragma unroll
          for (int kk = 0; kk < DH / 16; ++kk)
            umma_ts(d, a + kk * 8, qd + (uint64_t)((((kk >> 2) * QT * 128) >> 4) + (kk & 3) * 2), idesc, kk > 0);
          umma_commit(&s_full[2 * w + (job & 1)]);
        }
      }
      ok = __shfl_sync(0xFFFFFFFFu, ok ? 1 : 0, 0) != 0;
      it = __shfl_sync(0xFFFFFFFFu, it, 0);
    }
  }
  } else {
    // ------------------------------------------------------ slots and their weights
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kRegsSlots));
    const int w = warp >> 3, half = (warp >> 2) & 1;   // slot tile of the unit; which columns of its scores
    const int r = (warp & 3) * 32 + lane;              // slot whose codes this thread widens, half of them
    const uint32_t lanes = uint32_t((warp & 3) * 32) << 16;
    const int hs = p.pg.head_major ? 1 : p.hkv, log_block = 31 - __clz(p.block);
    const int mine = lane >> 2, quad = lane & 3;
    int it = 0;
    unsigned job = 0, filled = 0;
    bool ok = true;
    // positions in the tile of the first and last of the warp's columns
    const int col0 = half * CH, first_pos = col0 / G, last_pos = min(p.P - 1, (col0 + CH - 1) / G);
    // (between pieces the walk waits in shared memory: its registers are needed)
    if (lane == 0) walk_sh[warp] = u;
    while (ok) {
      __syncwarp();
      Pieces u = walk_sh[warp];
      if (!u.next(p)) break;
      __syncwarp();
      if (lane == 0) walk_sh[warp] = u;
      if (w == 1 && u.q.keys - u.kt * kUnitSlots <= KT) {
        // no second tile of slots: an arrival for each query tile all the same
        for (int t = u.t0; ok && t < u.t1; ++t, ++it) {
          ok = mbar_wait_short(&q_full[it % kStages], (it / kStages) & 1, abort_flag, p.status);
          __syncwarp();
          if (lane == 0) mbar_arrive(&q_empty[it % kStages]);
        }
        continue;
      }
      const int slot0 = u.kt * kUnitSlots + w * KT, warp_slot0 = slot0 + (warp & 3) * 32;
      // ---- the slots' codes, a slot's scale a factor of its scores (-1: there is no such page)
      {
        const int slot = slot0 + r;
        float f = 0.f;
        uint32_t code[DH / 8];
#pragma unroll
        for (int i = 0; i < DH / 8; ++i) code[i] = 0;
        if (slot < u.q.keys) {
          const long long row = p.pg.head_major ? ((long long)u.b * p.hkv + u.g) * p.rows.cap + slot
                                                : kv_row(p.pg, p.rows.cap, u.b, slot);
          if (row >= 0) {
            const int gs = p.pg.head_major ? 0 : u.g;
            const uint4 *src = reinterpret_cast<const uint4 *>(p.k + (row * hs + gs) * DH + half * (DH / 2));
#pragma unroll
            for (int i = 0; i < DH / 32; ++i) *reinterpret_cast<uint4 *>(&code[4 * i]) = __ldg(src + i);
            const float scale = __uint_as_float((uint32_t)p.ke[(row >> log_block) * hs + gs] << 23);
            f = p.scale_log2 * fmaf(scale, 0.f, scale);   // (e = 255: NaN)
          } else {
            f = -1.f;
            set_status(p.status, CC_ERR_DEVICE_ARG);
          }
        }
        if constexpr (!F16) {   // a NaN code: every score of the slot is none
          uint32_t any = 0;
#pragma unroll
          for (int i = 0; i < DH / 8; ++i) any |= __vcmpeq4(code[i] & 0x7F7F7F7Fu, 0x7F7F7F7Fu);
          if (any) f = NAN;
        }
        f_sh[filled & 1][w][half][r] = f;
        uint32_t a[DH / 4];
#pragma unroll
        for (int i = 0; i < DH / 8; ++i) {
          a[2 * i] = widen2<F16>(code[i] & 0xFFFFu);
          a[2 * i + 1] = widen2<F16>(code[i] >> 16);
        }
        const uint32_t a_t = tmem + lanes + w * 64 + half * (DH / 4);
        if constexpr (DH == 128) tmem_st32(a_t, a);
        else tmem_st16(a_t, a);
        tmem_st_wait();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(&a_full[w]);
      }
      // ---- a lane has the weights of four slots (8 apart) and every fourth pair of rows, so that a
      // row's terms are read once for four
      if (!(ok = mbar_wait_short(&a_full[w], filled & 1, abort_flag, p.status))) break;
      float2 fs[4], acc[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int row = (warp & 3) * 32 + mine + 8 * i;
        const float f0 = f_sh[filled & 1][w][0][row], f1 = f_sh[filled & 1][w][1][row];
        fs[i].x = fs[i].y = f0 == f0 ? f1 : f0;   // NaN where either half is
        acc[i] = make_float2(0.f, 0.f);
      }
      ++filled;
      for (int t = u.t0; t < u.t1; ++t, ++it, ++job) {
        const int s = it % kStages;
        const unsigned buf = 2 * w + (job & 1);
        if (!(ok = mbar_wait_short(&q_full[s], (it / kStages) & 1, abort_flag, p.status) &&
                   mbar_wait_short(&s_full[buf], (job >> 1) & 1, abort_flag, p.status)))
          break;
        tc_fence_after();
        {
          uint32_t sr[2][CH / 2];   // slots 0 - 15 and 16 - 31 of the warp's
          const uint32_t at = tmem + lanes + 128 + buf * QT + col0;
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            tmem_ld_rows16(at + ((uint32_t)i << 20), *reinterpret_cast<uint32_t(*)[16]>(&sr[i][0]));
            tmem_ld_rows16(at + ((uint32_t)i << 20) + 32, *reinterpret_cast<uint32_t(*)[8]>(&sr[i][16]));
          }
          const bool live = (live_sh[s] >> half) & 1u;   // every row of the columns adds
          const float4 *terms = term_sh + s * (QT / 2) + col0 / 2 + quad;
          // the last slots that the first and the last row of the columns see
          const int pos = u.q.s.seq + t * p.P;
          const int seen_first = p.memory_only ? 0x7FFFFFFF : pos + first_pos;
          const int seen_last = p.memory_only ? 0x7FFFFFFF : pos + last_pos;
          const float4 y0 = terms[0];   // (while the scores come; there are no registers for more)
          tmem_ld_wait();
          tc_fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive(&s_empty[buf]);   // copied out: the buffer may be refilled
          if (live && warp_slot0 + 31 <= seen_first) {
#pragma unroll
            for (int k = 0; k < CH / 8; ++k) {
              const float4 y = k == 0 ? y0 : terms[4 * k];   // of two columns -y and e^-rest
              float2 x[4];
#pragma unroll
              for (int i = 0; i < 4; ++i) {
                const uint32_t *x2 = &sr[i >> 1][4 * k + 2 * (i & 1)];
                x[i] = __ffma2_rn(make_float2(__uint_as_float(x2[0]), __uint_as_float(x2[1])), fs[i], make_float2(y.x, y.y));
              }
#pragma unroll
              for (int i = 0; i < 4; ++i) x[i] = make_float2(ex2(x[i].x), ex2(x[i].y));
#pragma unroll
              for (int i = 0; i < 4; ++i) acc[i] = __ffma2_rn(x[i], make_float2(y.z, y.w), acc[i]);
            }
          } else if (warp_slot0 <= seen_last) {   // (some row sees some slot)
            // of the lane's columns (8 k, and 8 k + 1), the first that sees the slot; none where no row of the
            // tile does: the columns that hold no query come behind the rows, and 0 times no number is none
            int from[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const int after = warp_slot0 + mine + 8 * i - pos;   // (at most P + 31)
              from[i] = p.memory_only ? -1 : after >= p.P ? QT : max(after, 0) * G - col0 - 2 * quad;
            }
            // (chosen, not multiplied by 0: what a row does not see, or one that adds nothing, may be no number)
            auto weigh = [&](auto some_dead) {
              constexpr bool dead = decltype(some_dead)::value;
#pragma unroll
              for (int k = 0; k < CH / 8; ++k) {
                const float4 y = terms[4 * k];
                const bool some0 = !dead || y.x > -INFINITY, some1 = !dead || y.y > -INFINITY;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                  const uint32_t *x2 = &sr[i >> 1][4 * k + 2 * (i & 1)];
                  float2 x = __ffma2_rn(make_float2(__uint_as_float(x2[0]), __uint_as_float(x2[1])), fs[i], make_float2(y.x, y.y));
                  x.x = some0 && 8 * k >= from[i] ? x.x : -INFINITY;
                  x.y = some1 && 8 * k + 1 >= from[i] ? x.y : -INFINITY;
                  acc[i] = __ffma2_rn(make_float2(ex2(x.x), ex2(x.y)), make_float2(y.z, y.w), acc[i]);
                }
              }
            };
            if (live) weigh(std::false_type());
            else weigh(std::true_type());
          }
        }
        __syncwarp();
        if (lane == 0) mbar_arrive(&q_empty[s]);   // the terms are read
      }
      if (!ok) break;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        float x = acc[i].x + acc[i].y;
        x += __shfl_xor_sync(0xFFFFFFFFu, x, 1);
        x += __shfl_xor_sync(0xFFFFFFFFu, x, 2);
        const int row = (warp & 3) * 32 + mine + 8 * i;
        if (quad != i || slot0 + row >= u.q.keys) continue;
        if (fs[i].x == -1.f) x = 0.f;
        if (u.whole)
          p.part[(((long long)u.g * p.rows.batch + u.b) * p.rows.cap + slot0 + row) * 2 + half] = x;
        else
          p.cut[((2 * share + (u.begins ? 1 : 0)) * kUnitSlots + w * KT + row) * 2 + half] = x;
      }
    }
  }

  tc_fence_before();
  __syncthreads();
  if (*abort_flag) __nanosleep(1000000);   // let copies still in flight land
  if (warp == 17) {
    tc_fence_after();
    tmem_dealloc(tmem, 512);
  }
}

// acc[b][j] += the heads' sums in order; a unit that spans shares is the sum of its pieces.
__global__ void __launch_bounds__(kUnitSlots) finish_kernel(const __grid_constant__ KvReceivedParams p) {
  // of each KV head's unit: the first share with query tiles of it (-1: it lies in one), the last
  __shared__ int first_sh[kUnitSlots], last_sh[kUnitSlots];
  const int per_seq = (p.rows.cap + kUnitSlots - 1) / kUnitSlots, tid = threadIdx.x;
  const int b = blockIdx.x / per_seq, kt = blockIdx.x - b * per_seq;
  const SeqLine q = seq_line(p, b);
  if (kt >= q.nk) {
    pdl_wait();
    return;
  }
  const long long total = line_length(p), before = length_before(p, b);
  const int n = line_shares(p.shares, total);
  const int slot = kt * kUnitSlots + tid;
  float *dst = p.acc + (long long)b * p.rows.cap + slot;
  // (the other kernel leaves the accumulators alone: only its sums are waited for)
  const float old = slot < q.keys && !(p.first && slot >= q.s.seq) ? *dst : 0.f;
  float sum = 0.f;
  for (int g0 = 0; g0 < p.hkv; g0 += kUnitSlots) {
    __syncthreads();
    if (g0 + tid < p.hkv) {
      const int g = g0 + tid;
      const int span0 = q.tiles + kUnitCost;
      int span = span0, cost = kUnitCost;
      long long at = before;
      if (kt < q.nfull) {
        at += ((long long)kt * p.hkv + g) * span0;
      } else {
        at += (long long)q.nfull * p.hkv * span0;
        for (int k = q.nfull; k < kt; ++k) at += (long long)(q.tiles - first_tile(p, q, k) + kEdgeCost) * p.hkv;
        cost = kEdgeCost;
        span = q.tiles - first_tile(p, q, kt) + kEdgeCost;
        at += (long long)g * span;
      }
      const int c0 = share_at(at, total, n);
      int lo = c0;
      const int c1 = share_at(at + span - 1, total, n);
      // (shares that end before the first query tile have no sums)
      while (lo < c1 && total * (lo + 1) / n - at <= cost) ++lo;
      first_sh[tid] = c0 == c1 ? -1 : lo * 2 + (lo == c0 ? 1 : 0);
      last_sh[tid] = c1;
    }
    __syncthreads();
    if (g0 == 0) pdl_wait();
    if (slot >= q.keys) continue;
    const float2 *cut = reinterpret_cast<const float2 *>(p.cut) + tid;
    const float2 *part = reinterpret_cast<const float2 *>(p.part) + (long long)b * p.rows.cap + slot;
    const int heads = min(kUnitSlots, p.hkv - g0);
    for (int i0 = 0; i0 < heads; i0 += 4) {   // (the loads of four heads together)
      float2 x[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        if (i0 + j >= heads) break;
        const int first = first_sh[i0 + j];   // share, and whether the unit begins there
        x[j] = first < 0 ? part[(long long)(g0 + i0 + j) * p.rows.batch * p.rows.cap] : cut[first * kUnitSlots];
      }
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        if (i0 + j >= heads) break;
        const int first = first_sh[i0 + j];
        if (first >= 0)
          for (int c = first / 2 + 1; c <= last_sh[i0 + j]; ++c) {
            const float2 y = cut[2 * c * kUnitSlots];
            x[j] = make_float2(x[j].x + y.x, x[j].y + y.y);
          }
        sum += x[j].x + x[j].y;
      }
    }
  }
  if (slot < q.keys) *dst = old + sum;
}

template <int DH, bool F16>
cudaError_t launch(const KvReceivedParams &p, const CUtensorMap &tq, cudaStream_t st) {
  static bool attr_set[64] = {};
  int dev = 0;
  cudaGetDevice(&dev);
  if (dev < 64 && !attr_set[dev]) {
    const cudaError_t e = cudaFuncSetAttribute(received_tiles_kernel<DH, F16>,
                                               cudaFuncAttributeMaxDynamicSharedMemorySize, RtSmem<DH>::BYTES);
    if (e != cudaSuccess) return e;
    attr_set[dev] = true;
  }
  received_tiles_kernel<DH, F16><<<p.shares, kThreads, RtSmem<DH>::BYTES, st>>>(p, tq);
  const cudaError_t e = cudaGetLastError();
  if (e != cudaSuccess) return e;
  const unsigned blocks = (unsigned)((p.rows.cap + kUnitSlots - 1) / kUnitSlots) * (unsigned)p.rows.batch;
  return launch_pdl(finish_kernel, dim3(blocks), dim3(kUnitSlots), 0, st, p);
}

}  // namespace

int kv_received_positions(int group) { return QT / group; }

size_t kv_received_part_bytes(const KvReceivedParams &p, int sms) {
  return (size_t)p.hkv * p.rows.batch * p.rows.cap * 8 + (size_t)sms * 2 * kUnitSlots * 8;
}

cudaError_t launch_kv_received_tiles(KvReceivedParams p, const CUtensorMap &tq, void *ws, int sms, cudaStream_t st) {
  p.P = kv_received_positions(p.hq / p.hkv);
  p.shares = sms;
  p.cut = reinterpret_cast<float *>(ws);
  p.part = p.cut + (size_t)sms * 4 * kUnitSlots;
  if (p.head_dim == 128) return p.f16 ? launch<128, true>(p, tq, st) : launch<128, false>(p, tq, st);
  return p.f16 ? launch<64, true>(p, tq, st) : launch<64, false>(p, tq, st);
}

}  // namespace cc
