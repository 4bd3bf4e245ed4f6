// kvappend.cu -- new tokens' keys (rotated) and values into one layer of the
// cache, their queries rotated on the way, and the bookkeeping that ends a
// step.
//
// A unit of work is a block of `block` cache slots of one sequence that new
// rows fall into (block format: the slots that share a scale), a CTA's is a unit
// and a share of the heads.  Block format: first the warps, shared evenly among the KV
// heads' keys and values, bound the unit's magnitudes, and a warp settles each scale
// and rescales what the block held.  For keys it bounds the radius of each rotated pair, sqrt(a^2 + b^2) <= max + min / 2, so that
// the scale needs no angle and is the same bits however cos and sin are rounded;
// it is at most 1.12 times the largest magnitude that any rotation gives.  Then
// teams of head_dim / 16 lanes take a row each, or where there are few rows some of
// its heads: a lane holds 8 elements of a head and the 8 that they rotate with, and
// cos and sin of its angles stay in registers from head to head.
//
// Bound by HBM; keys and values are read twice, the second time from L2.  A lane
// copies what it will read a few heads (rows, for the bound) ahead into slots of its
// own (cp.async, no barrier): loops unrolled over loads instead held as much in
// flight but half of the time nothing, and their code was a single token's latency.
// Four chunks of 4096 tokens, 32/8 heads of 128, bf16: 369 MB in 71 us (5.2 TB/s); 2957
// tokens of five ragged sequences, 28/4 heads, fp32: 100 MB in 16.7 us (6.0 TB/s); a
// token each of 64 sequences: 6.6 us, latency (launch, bound, rows one after another).
#include "kvappend.cuh"

#include <algorithm>
#include <atomic>
#include <type_traits>

namespace cc {

namespace {

constexpr int kThreads = 256;
// CTAs per SM to split the heads for, and where there are heads for so many (three are
// resident: the last wave is a smaller part; four chunks of 4096 tokens, 32/8 heads, in
// blocks of 128, 64 and 32 slots: 76.9 -> 71.1, 77.2 -> 70.8, 72.5 -> 67.6 us).  Short of
// that one wave is better: 28/4 heads, three shares 58, four 63.
constexpr int kSplitCtas = 2;
constexpr int kManyCtas = 6;
constexpr int kLeastExp = 10, kMostExp = 247, kUnitExp = 127;   // scale exponents written

// The 8 elements of half a head that a lane holds: pieces of 16 bytes which lie side
// by side across the team's lanes, so that a load or store takes whole sectors.
template <typename T, int DH>
struct Lane {
  static constexpr int GRP = 16 / sizeof(T), PIECES = 8 / GRP, APART = DH / 2 / PIECES;
  int first;   // of piece 0
  CC_DEV explicit Lane(int lane) : first(lane % (DH / 16) * GRP) {}
  CC_DEV int element(int i) const { return first + i / GRP * APART + i % GRP; }
  CC_DEV void store(T *dst, const float (&x)[8]) const {   // dst: the half's first element
#pragma unroll
    for (int j = 0; j < PIECES; ++j) {
      if constexpr (sizeof(T) == 4) {
        *reinterpret_cast<float4 *>(dst + first + j * APART) =
            make_float4(x[4 * j], x[4 * j + 1], x[4 * j + 2], x[4 * j + 3]);
      } else {
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i)
          w[i] = std::is_same_v<T, __half> ? pack_f16x2(x[2 * i], x[2 * i + 1])
                                           : pack_bf16x2(x[2 * i], x[2 * i + 1]);
        *reinterpret_cast<uint4 *>(dst + first) = make_uint4(w[0], w[1], w[2], w[3]);
      }
    }
  }
  CC_DEV void store_bf16(__nv_bfloat16 *dst, const float (&x)[8]) const {
#pragma unroll
    for (int i = 0; i < 8; i += 4)
      *reinterpret_cast<uint2 *>(dst + element(i)) =
          make_uint2(pack_bf16x2(x[i], x[i + 1]), pack_bf16x2(x[i + 2], x[i + 3]));
  }
  CC_DEV void store_codes(uint8_t *dst, const float (&x)[8]) const {
    const uint32_t lo = pack_e4m3x2(x[0], x[1]) | (pack_e4m3x2(x[2], x[3]) << 16);
    const uint32_t hi = pack_e4m3x2(x[4], x[5]) | (pack_e4m3x2(x[6], x[7]) << 16);
    if constexpr (PIECES == 1) {
      *reinterpret_cast<uint2 *>(dst + first) = make_uint2(lo, hi);
    } else {
      *reinterpret_cast<uint32_t *>(dst + element(0)) = lo;
      *reinterpret_cast<uint32_t *>(dst + element(4)) = hi;
    }
  }
};

// 8 elements as they lie in memory, in words.
template <typename T>
struct Raw8 {
  uint32_t w[2 * sizeof(T)];
  CC_DEV void widen(float (&x)[8]) const {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      if constexpr (sizeof(T) == 4) x[i] = __uint_as_float(w[i]);
      else if constexpr (std::is_same_v<T, __half>)
        x[i] = i & 1 ? __high2float(*reinterpret_cast<const __half2 *>(&w[i / 2]))
                     : __low2float(*reinterpret_cast<const __half2 *>(&w[i / 2]));
      else x[i] = i & 1 ? bf16_hi(w[i / 2]) : bf16_lo(w[i / 2]);
    }
  }
};

CC_DEV float finite_abs(float x) {
  const float a = fabsf(x);
  return a < INFINITY ? a : 0.f;   // infinities and NaN: 0
}
// The least exponent e with bound <= 448 * 2^(e - 127), in the written range
// (448 = 1.75 * 2^8: a mantissa past .75 takes the next power); 0 for a bound
// of 0, which any scale holds.
CC_DEV int scale_exp(float bound) {
  if (!(bound > 0.f)) return 0;
  const int e = (int)((__float_as_uint(bound) + 0x1FFFFFu) >> 23) - 8;
  return min(max(e, kLeastExp), kMostExp);
}
CC_DEV float pow2_biased(int e) { return e > 0 ? __uint_as_float((uint32_t)e << 23) : 0.f; }
// 1 / 2^(e - 127), e from 1 on (of 2^127 a subnormal).
CC_DEV float inverse_pow2(int e) { return e == 254 ? __uint_as_float(1u << 22) : pow2_biased(254 - e); }

// 8 pairs: cos, sin, and minus sin, two to a register pair.
struct Turn {
  float2 c[4], s[4], n[4];
};
CC_DEV void rotate8(float (&a)[8], float (&b)[8], const Turn &t) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float2 x = make_float2(a[2 * i], a[2 * i + 1]), y = make_float2(b[2 * i], b[2 * i + 1]);
    const float2 u = __ffma2_rn(y, t.n[i], __fmul2_rn(x, t.c[i]));
    const float2 v = __ffma2_rn(x, t.s[i], __fmul2_rn(y, t.c[i]));
    a[2 * i] = u.x, a[2 * i + 1] = u.y;
    b[2 * i] = v.x, b[2 * i + 1] = v.y;
  }
}

// cos and sin of a fraction of a turn: those of the nearest 256th from a table,
// turned by what is left (|d| <= pi / 256: the Taylor series to d^4 and d^3 are good to
// 2^-40 and 2^-38), an eighth of the instructions of sincospif.
constexpr int kTable = 256;
CC_DEV void table_entry(float2 *table, int i) {
  float sn, cs;
  sincospif((float)i * (2.f / kTable), &sn, &cs);
  table[i] = make_float2(cs, sn);
}
CC_DEV void turn_cs(const float2 *table, uint32_t frac, float &c, float &s) {   // frac / 2^32 of a turn
  const uint32_t at = frac + (1u << 23);   // to the nearest entry
  const float2 t = table[at >> 24];
  const float d = (float)((int)(at & 0xFFFFFFu) - (1 << 23)) * 1.4629180792671596e-09f;   // 2 pi / 2^32
  const float d2 = d * d;
  const float cd1 = d2 * fmaf(d2, 1.f / 24.f, -0.5f), sd = fmaf(d * d2, -1.f / 6.f, d);   // cos d - 1, sin d
  c = t.x + fmaf(t.x, cd1, -t.y * sd);   // (the small terms' roundings do not count)
  s = t.y + fmaf(t.y, cd1, t.x * sd);
}

// What magnitudes a lane has seen of one head's keys or values.
template <typename T>
struct Bound {
  float top = 0.f;     // keys: of max + min / 2; fp32 values too
  uint32_t seen = 0;   // 16-bit types: the largest magnitudes' bits, two at a time
  CC_DEV static float of(uint32_t bits) {
    return std::is_same_v<T, __half> ? __half2float(__ushort_as_half((unsigned short)bits))
                                     : __uint_as_float(bits << 16);
  }
  // Infinities and NaN take no part: with `careful` one by one, else they are seen
  // and `odd` tells.
  CC_DEV void add(const Raw8<T> &ra, const Raw8<T> &rc, bool is_k, bool careful) {
    if (sizeof(T) == 4 || careful) {
      float a[8], c[8];
      ra.widen(a);
      rc.widen(c);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float u = finite_abs(a[i]), w = finite_abs(c[i]), hi = fmaxf(u, w);
        top = fmaxf(top, is_k ? __fadd_rn(hi, 0.5f * fminf(u, w)) : hi);
      }
    } else {
      float2 m = make_float2(0.f, 0.f);
#pragma unroll
      for (int i = 0; i < 4; ++i) {   // magnitudes order as their bits do
        const uint32_t u = ra.w[i] & 0x7FFF7FFFu, w = rc.w[i] & 0x7FFF7FFFu, hi = __vmaxu2(u, w);
        seen = __vmaxu2(seen, hi);
        if (is_k) {
          const uint32_t lo = __vminu2(u, w);
          m.x = fmaxf(m.x, __fadd_rn(of(hi & 0xFFFFu), 0.5f * of(lo & 0xFFFFu)));
          m.y = fmaxf(m.y, __fadd_rn(of(hi >> 16), 0.5f * of(lo >> 16)));
        }
      }
      top = fmaxf(top, fmaxf(m.x, m.y));
    }
  }
  CC_DEV bool odd() const {
    const uint32_t inf = std::is_same_v<T, __half> ? 0x7C00u : 0x7F80u;
    return max(seen & 0xFFFFu, seen >> 16) >= inf;
  }
  CC_DEV float get(bool is_k) const { return is_k ? top : fmaxf(top, of(max(seen & 0xFFFFu, seen >> 16))); }
};

// A lane's items ahead: 8 + 8 elements each.
template <typename T, int DH>
struct Ahead {
  using L = Lane<T, DH>;
  static constexpr int SLOTS = 256 / (2 * L::PIECES * 16);   // 256 bytes a lane
  static constexpr int BYTES = kThreads * 256;
  uint8_t *mem;   // of the lane
  CC_DEV void issue(int slot, const T *half0) {   // this lane's first element of the head
    const uint32_t to = smem_u32(mem) + slot * (2 * L::PIECES * 16 * kThreads);
#pragma unroll
    for (int i = 0; i < 2 * L::PIECES; ++i)
      asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(to + i * 16 * kThreads),
                   "l"(half0 + i * L::APART) : "memory");
  }
  CC_DEV void get(int slot, Raw8<T> &a, Raw8<T> &c) const {
    const uint4 *from = reinterpret_cast<const uint4 *>(mem + slot * (2 * L::PIECES * 16 * kThreads));
#pragma unroll
    for (int i = 0; i < L::PIECES; ++i) {
      *reinterpret_cast<uint4 *>(&a.w[4 * i]) = from[i * kThreads];
      *reinterpret_cast<uint4 *>(&c.w[4 * i]) = from[(L::PIECES + i) * kThreads];
    }
  }
  CC_DEV static void commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
  CC_DEV static void wait_oldest() {   // of SLOTS - 1 in flight before the last one was issued
    asm volatile("cp.async.wait_group %0;" ::"n"(SLOTS - 1) : "memory");
  }
};

template <typename T, int DH>
__global__ void __launch_bounds__(kThreads, 3)
    kv_append_kernel(const __grid_constant__ KvAppendParams p) {
  constexpr int HALF = DH / 2, TPR = DH / 16, RPI = 32 / TPR;   // lanes per row, rows per warp
  constexpr int TEAMS = kThreads / TPR, SLOTS = Ahead<T, DH>::SLOTS;
  extern __shared__ __align__(16) uint8_t smem[];
  const int B = p.block, per_seq = (p.rows.max_rows + B - 2) / B + 1;
  const int b = blockIdx.x / per_seq;
  const SeqRows s = seq_rows(p.rows, b, true);
  if (!s.ok) {
    if (threadIdx.x == 0) set_status(p.status, CC_ERR_DEVICE_ARG);
    return;
  }
  // the unit's slots [base, base + B): older ones [base, base + old), new ones
  // [base + old, base + old + n), rows from r0
  const int base = (s.seq / B + (blockIdx.x - b * per_seq)) * B;
  const int old = max(s.seq - base, 0);
  const int r0 = s.r0 + base + old - s.seq;
  const int n = min(base + B, s.seq + s.count) - (base + old);
  if (n <= 0) return;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const Lane<T, DH> mine(lane);
  Ahead<T, DH> ahead{smem + tid * 16};
  float2 *table = reinterpret_cast<float2 *>(smem + Ahead<T, DH>::BYTES);
  // of K heads, then of V heads: the bound, then 1 / scale
  float *scale = reinterpret_cast<float *>(table + kTable);
  // this CTA's heads
  const int ny = gridDim.y, y = blockIdx.y;
  const int k0 = p.hkv * y / ny, nk = p.hkv * (y + 1) / ny - k0;
  const int q0 = p.hq * y / ny, nq = p.q ? p.hq * (y + 1) / ny - q0 : 0;
  const bool by_block = p.format == CC_KV_E4M3_BLOCK;
  // the unit lies in one page: vector of KV head g and slot base + i
  const long long row0 = p.pg.head_major ? 0 : kv_row(p.pg, p.rows.cap, b, base);
  const int vstep = p.pg.head_major ? 1 : p.hkv;
  const long long head_step = (p.pg.head_major ? (long long)p.rows.cap : 1) * DH;   // elements
  auto vec_at = [&](int g) {
    return p.pg.head_major ? ((long long)b * p.hkv + g) * p.rows.cap + base : row0 * p.hkv + g;
  };
  if (row0 < 0 && tid == 0) set_status(p.status, CC_ERR_DEVICE_ARG);

  if (p.rotate) table_entry(table, tid);
  static_assert(kTable == kThreads, "a thread an entry");
  if (by_block && row0 >= 0) {
    constexpr int kWarps = kThreads / 32;
    // bounds: a job (K or V of a head) to as many warps as there are for it
    const int jobs = 2 * nk;
    int parts = 1;
    while (parts * 2 * jobs <= kWarps) parts *= 2;
    for (int i = tid; i < jobs; i += kThreads) scale[i] = 0.f;
    __syncthreads();
    const int team = lane / TPR + warp % parts * RPI;
    for (int job = warp / parts; job < jobs; job += kWarps / parts) {
      const bool is_k = job < nk;
      const long long ld = is_k ? p.k_ld : p.v_ld;
      const T *src = reinterpret_cast<const T *>(is_k ? p.k : p.v) + r0 * ld +
                     (k0 + (is_k ? job : job - nk)) * DH + mine.first;
      Bound<T> bound;
      auto sweep = [&](bool careful) {
        auto issue = [&](int r, int slot) {
          if (r < n) ahead.issue(slot, src + r * ld);
          ahead.commit();
        };
#pragma unroll 1
        for (int i = 0; i < SLOTS - 1; ++i) issue(team + i * RPI * parts, i);
        int slot = 0;
#pragma unroll 1
        for (int r = team; r < n; r += RPI * parts) {
          issue(r + (SLOTS - 1) * RPI * parts, slot == 0 ? SLOTS - 1 : slot - 1);
          ahead.wait_oldest();
          Raw8<T> a, c;
          ahead.get(slot, a, c);
          slot = slot + 1 == SLOTS ? 0 : slot + 1;
          bound.add(a, c, is_k, careful);
        }
      };
      sweep(false);
      if (__any_sync(0xFFFFFFFFu, bound.odd())) {
        bound = Bound<T>();
        sweep(true);
      }
      const float top = warp_max(bound.get(is_k));
      // (magnitudes order as their bits do)
      if (lane == 0) atomicMax(reinterpret_cast<int *>(scale) + job, __float_as_int(top));
    }
    __syncthreads();
    for (int job = warp; job < jobs; job += kWarps) {
      const bool is_k = job < nk;
      const int g = k0 + (is_k ? job : job - nk);
      const long long vec0 = vec_at(g);
      const long long ei = p.pg.head_major ? vec0 / B : row0 / B * p.hkv + g;
      uint8_t *ep = (is_k ? p.ke : p.ve) + ei;
      const int e_old = old ? *ep : 0;
      int e = max(scale_exp(scale[job]), e_old);
      if (e == 0) e = kUnitExp;   // zeros alone
      if (old && e > e_old) {     // the older codes by a power of two
        const float f = e_old > 0 ? pow2_biased(127 + e_old - e) : 0.f;   // (a scale of 0)
        uint8_t *codes = reinterpret_cast<uint8_t *>(is_k ? p.kc : p.vc);
#pragma unroll 1
        for (int r = lane / TPR; r < old; r += RPI) {
          uint4 *at = reinterpret_cast<uint4 *>(codes + (vec0 + (long long)r * vstep) * DH + lane % TPR * 16);
          const uint4 u = *at;
          uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            uint32_t r2[2];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
              uint32_t h2;
              asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h2) : "h"((unsigned short)(w[i] >> (16 * h))));
              const float2 x = __half22float2(*reinterpret_cast<const __half2 *>(&h2));
              r2[h] = pack_e4m3x2(x.x * f, x.y * f);
            }
            w[i] = r2[0] | (r2[1] << 16);
          }
          *at = make_uint4(w[0], w[1], w[2], w[3]);
        }
      }
      __syncwarp();   // every lane has read the bound and the older exponent
      if (lane == 0) {
        *ep = (uint8_t)e;
        scale[job] = inverse_pow2(e);
      }
    }
  }
  __syncthreads();

  // ---- rows by heads: rt rows at a time, TEAMS / rt teams to a row, each taking
  // every ht-th of the row's K, V and Q heads
  int rt = 1;
  while (rt < TEAMS && rt < n) rt *= 2;
  const int team = tid / TPR, ht = TEAMS / rt, h0 = team / rt, heads = 2 * nk + nq;
  if (h0 >= heads || team % rt >= n) return;
  const int follow = !p.rotate || p.pos || s.seq == 0
                         ? 0 : p.cache_pos[(size_t)b * p.rows.cap + s.seq - 1] + 1;
  auto position = [&](int r) {
    return !p.rotate ? 0 : p.pos ? (r < n ? p.pos[r0 + r] : 0) : follow + (base + old - s.seq) + r;
  };
  int ri = team % rt, hi = h0;   // the next item to copy, and its row's K, V and Q
  const T *ki, *vi, *qi;
  auto enter = [&]() {
    const long long r = r0 + ri;
    ki = reinterpret_cast<const T *>(p.k) + r * p.k_ld + k0 * DH + mine.first;
    vi = reinterpret_cast<const T *>(p.v) + r * p.v_ld + (k0 - nk) * DH + mine.first;
    qi = reinterpret_cast<const T *>(p.q) + r * p.q_ld + (q0 - 2 * nk) * DH + mine.first;
  };
  enter();
  auto issue = [&](int slot) {
    if (ri < n) {
      const T *src = (hi < nk ? ki : hi < 2 * nk ? vi : qi) + hi * DH;
      ahead.issue(slot, src);
      hi += ht;
      if (hi >= heads) {
        hi = h0;
        ri += rt;
        enter();
      }
    }
    ahead.commit();
  };
#pragma unroll 1
  for (int i = 0; i < SLOTS - 1; ++i) issue(i);
  int slot = 0, next_pos = position(team % rt);
#pragma unroll 1
  for (int r = team % rt; r < n; r += rt) {
    Turn t;
    if (p.rotate) {
      int at = next_pos;
      next_pos = position(r + rt);
      if (at < 0) {
        set_status(p.status, CC_ERR_DEVICE_ARG);
        at = 0;
      }
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        // pos * turns mod 2^64 is a fraction of a turn
        float sn, cs;
        turn_cs(table, (uint32_t)(((unsigned long long)at * p.turns[mine.element(i)]) >> 32), cs, sn);
        (i & 1 ? t.c[i / 2].y : t.c[i / 2].x) = cs;
        (i & 1 ? t.s[i / 2].y : t.s[i / 2].x) = sn;
        (i & 1 ? t.n[i / 2].y : t.n[i / 2].x) = -sn;
      }
    }
    // where the row's K and V of head k0 go, and its Q of head q0
    const long long el0 = row0 < 0 ? 0 : (vec_at(k0) + (long long)(old + r) * vstep) * DH;
    T *out = reinterpret_cast<T *>(p.q_out) + (r0 + r) * p.q_out_ld + q0 * DH;
#pragma unroll 1
    for (int h = h0; h < heads; h += ht) {
      issue(slot == 0 ? SLOTS - 1 : slot - 1);
      ahead.wait_oldest();
      Raw8<T> ra, rc;
      ahead.get(slot, ra, rc);
      float a[8], c[8];
      ra.widen(a);
      rc.widen(c);
      slot = slot + 1 == SLOTS ? 0 : slot + 1;
      const bool is_k = h < nk, is_q = h >= 2 * nk;
      if (p.rotate && (is_k || is_q)) rotate8(a, c, t);
      if (is_q) {
        mine.store(out + (h - 2 * nk) * DH, a);
        mine.store(out + (h - 2 * nk) * DH + HALF, c);
        continue;
      }
      if (row0 < 0) continue;
      const long long el = el0 + (is_k ? h : h - nk) * head_step;
      void *buf = is_k ? p.kc : p.vc;
      if (p.format == CC_KV_BF16) {
        mine.store_bf16(reinterpret_cast<__nv_bfloat16 *>(buf) + el, a);
        mine.store_bf16(reinterpret_cast<__nv_bfloat16 *>(buf) + el + HALF, c);
        continue;
      }
      const float inv = by_block ? scale[h] : is_k ? p.k_qscale : p.v_qscale;
      // 0 times an infinity: NaN (one scale a layer saturates it, as the appends do)
      const float2 inv2 = make_float2(inv, inv), zero = make_float2(0.f, 0.f);
#pragma unroll
      for (int i = 0; i < 8; i += 2) {
        float2 x = make_float2(a[i], a[i + 1]), z = make_float2(c[i], c[i + 1]);
        const float2 xs = __fmul2_rn(x, inv2), zs = __fmul2_rn(z, inv2);
        x = by_block ? __ffma2_rn(x, zero, xs) : xs;
        z = by_block ? __ffma2_rn(z, zero, zs) : zs;
        a[i] = x.x, a[i + 1] = x.y, c[i] = z.x, c[i + 1] = z.y;
      }
      mine.store_codes(reinterpret_cast<uint8_t *>(buf) + el, a);
      mine.store_codes(reinterpret_cast<uint8_t *>(buf) + el + HALF, c);
    }
  }
}

__global__ void __launch_bounds__(kThreads)
    kv_advance_kernel(StepRows rows, const int32_t *pos, const int32_t *tokens, int32_t *seq_len,
                      int32_t *cache_tokens, int32_t *cache_pos, unsigned *status) {
  const int b = blockIdx.x;
  const SeqRows s = seq_rows(rows, b, true);
  if (!s.ok) {
    if (threadIdx.x == 0) set_status(status, CC_ERR_DEVICE_ARG);
    return;
  }
  const size_t at = (size_t)b * rows.cap + s.seq;
  const int follow = pos || s.seq == 0 ? 0 : cache_pos[at - 1] + 1;
  for (int i = threadIdx.x; i < s.count; i += kThreads) {
    const int at_pos = pos ? pos[s.r0 + i] : follow + i;
    if (at_pos < 0) set_status(status, CC_ERR_DEVICE_ARG);
    cache_pos[at + i] = max(at_pos, 0);
    if (tokens) cache_tokens[at + i] = tokens[s.r0 + i];
  }
  __syncthreads();   // every thread has read seq_len
  if (threadIdx.x == 0) seq_len[b] = s.seq + s.count;
}

template <typename T, int DH>
cudaError_t launch_append_as(const KvAppendParams &p, int sms, cudaStream_t st) {
  const int per_seq = (p.rows.max_rows + p.block - 2) / p.block + 1;
  const long long units = (long long)p.rows.batch * per_seq;
  if (units > 0x7FFFFFFFll) return cudaErrorInvalidValue;
  auto kern = kv_append_kernel<T, DH>;
  // a unit's heads over several CTAs until they fill the SMs
  const long long busy = std::min(units, (long long)p.rows.n_rows / p.block + p.rows.batch);   // (about)
  const long long ctas = (long long)sms * (busy * p.hkv >= kManyCtas * sms ? kManyCtas : kSplitCtas);
  const int split = (int)std::min<long long>(p.hkv, std::max<long long>(1, (ctas + busy - 1) / busy));
  const size_t smem = Ahead<T, DH>::BYTES + kTable * sizeof(float2) + 2 * ((size_t)p.hkv / split + 1) * sizeof(float);
  // one limit for every head count: a call must not lower what another thread's needs
  constexpr size_t kMostSmem = 200 * 1024;
  if (smem > kMostSmem) return cudaErrorInvalidValue;
  static std::atomic<bool> attr_set[64] = {};
  int dev = 0;
  cudaGetDevice(&dev);
  if (dev >= 64 || !attr_set[dev]) {
    const cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kMostSmem);
    if (e != cudaSuccess) return e;
    if (dev < 64) attr_set[dev] = true;
  }
  kern<<<dim3((unsigned)units, (unsigned)split), kThreads, smem, st>>>(p);
  return cudaGetLastError();
}

template <typename T>
cudaError_t launch_append_dh(const KvAppendParams &p, int sms, cudaStream_t st) {
  return p.head_dim == 128 ? launch_append_as<T, 128>(p, sms, st) : launch_append_as<T, 64>(p, sms, st);
}

}  // namespace

cudaError_t launch_kv_append(const KvAppendParams &p, int sms, cudaStream_t st) {
  if (p.head_dim != 64 && p.head_dim != 128) return cudaErrorInvalidValue;
  switch (p.dtype) {
    case CC_BF16: return launch_append_dh<__nv_bfloat16>(p, sms, st);
    case CC_F16: return launch_append_dh<__half>(p, sms, st);
    case CC_F32: return launch_append_dh<float>(p, sms, st);
    default: return cudaErrorInvalidValue;
  }
}

cudaError_t launch_kv_advance(const StepRows &rows, const int32_t *pos, const int32_t *tokens,
                              int32_t *seq_len, int32_t *cache_tokens, int32_t *cache_pos,
                              unsigned *status, cudaStream_t st) {
  kv_advance_kernel<<<rows.batch, kThreads, 0, st>>>(rows, pos, tokens, seq_len, cache_tokens,
                                                      cache_pos, status);
  return cudaGetLastError();
}

}  // namespace cc
