// kvappend.cu -- new tokens' keys (rotated) and values into one layer of the
// cache, their queries rotated on the way, and the bookkeeping that ends a
// step.
//
// A unit of work is a block of `block` cache slots of one sequence that new
// rows fall into (block format: the slots that share a scale).  A CTA takes one
// unit, or with few units a share of its heads: it tabulates cos and sin of its
// rows' angles once for all heads; then a warp takes one KV head's keys or
// values of the unit, and teams of head_dim / 16 lanes take one query head of
// one row.  A lane holds 8 elements and the 8 that they rotate with.
//
// Block format: a KV head's warp reads its rows twice, first for the bound of
// their magnitudes.  For keys it bounds the radius of each rotated pair,
// sqrt(a^2 + b^2) <= max + min / 2, so that the scale needs no angle and is the
// same bits however cos and sin are rounded; it is at most 1.12 times the
// largest magnitude that any rotation gives.  The second read hits L1.
#include "kvappend.cuh"

#include <algorithm>

namespace cc {

namespace {

constexpr int kThreads = 256;
constexpr int kLeastExp = 10, kMostExp = 247, kUnitExp = 127;   // scale exponents written

template <typename T>
CC_DEV void load8(const T *src, float (&x)[8]) {
  if constexpr (sizeof(T) == 4) {
    const float4 a = reinterpret_cast<const float4 *>(src)[0], b = reinterpret_cast<const float4 *>(src)[1];
    x[0] = a.x, x[1] = a.y, x[2] = a.z, x[3] = a.w, x[4] = b.x, x[5] = b.y, x[6] = b.z, x[7] = b.w;
  } else {
    const uint4 u = *reinterpret_cast<const uint4 *>(src);
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if constexpr (std::is_same_v<T, __half>) {
        const float2 f = __half22float2(*reinterpret_cast<const __half2 *>(&w[i]));
        x[2 * i] = f.x, x[2 * i + 1] = f.y;
      } else {
        x[2 * i] = bf16_lo(w[i]), x[2 * i + 1] = bf16_hi(w[i]);
      }
    }
  }
}
template <typename T>
CC_DEV void store8(T *dst, const float (&x)[8]) {
  if constexpr (sizeof(T) == 4) {
    reinterpret_cast<float4 *>(dst)[0] = make_float4(x[0], x[1], x[2], x[3]);
    reinterpret_cast<float4 *>(dst)[1] = make_float4(x[4], x[5], x[6], x[7]);
  } else {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i)
      w[i] = std::is_same_v<T, __half> ? pack_f16x2(x[2 * i], x[2 * i + 1])
                                       : pack_bf16x2(x[2 * i], x[2 * i + 1]);
    *reinterpret_cast<uint4 *>(dst) = make_uint4(w[0], w[1], w[2], w[3]);
  }
}
CC_DEV void store_codes8(uint8_t *dst, const float (&x)[8]) {
  *reinterpret_cast<uint2 *>(dst) =
      make_uint2(pack_e4m3x2(x[0], x[1]) | (pack_e4m3x2(x[2], x[3]) << 16),
                 pack_e4m3x2(x[4], x[5]) | (pack_e4m3x2(x[6], x[7]) << 16));
}

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

// (a, b) of 8 rotated pairs with their (cos, sin)
CC_DEV void rotate8(float (&a)[8], float (&b)[8], const float2 *cs) {
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float2 t = cs[i];
    const float x = a[i], y = b[i];
    a[i] = x * t.x - y * t.y;
    b[i] = y * t.x + x * t.y;
  }
}

template <typename T, int DH>
__global__ void __launch_bounds__(kThreads)
    kv_append_kernel(const __grid_constant__ KvAppendParams p) {
  constexpr int HALF = DH / 2, TPR = DH / 16, RPI = 32 / TPR;   // lanes per row, rows per warp
  extern __shared__ float2 trig[];   // [rows of the unit][HALF]
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

  if (p.rotate) {
    const int follow = p.pos || s.seq == 0
                           ? 0 : p.cache_pos[(size_t)b * p.rows.cap + s.seq - 1] + 1;
    for (int i = tid; i < n * HALF; i += kThreads) {
      const int r = i / HALF, k = i - r * HALF;
      int at = p.pos ? p.pos[r0 + r] : follow + (base + old - s.seq) + r;
      if (at < 0) {
        if (k == 0) set_status(p.status, CC_ERR_DEVICE_ARG);
        at = 0;
      }
      // pos * turns mod 2^64 is a fraction of a turn; its top 32 bits as a
      // signed fraction times 2 are the angle in units of pi
      const int32_t frac = (int32_t)(((unsigned long long)at * p.turns[k]) >> 32);
      float sn, cs;
      sincospif((float)frac * 0x1p-31f, &sn, &cs);
      trig[i] = make_float2(cs, sn);
    }
    __syncthreads();
  }

  const int stride = gridDim.y * (kThreads / 32);
  const int team = lane / TPR, at8 = (lane % TPR) * 8;
  for (int job = blockIdx.y * (kThreads / 32) + warp; job < 2 * p.hkv; job += stride) {
    const bool is_k = job < p.hkv;
    const int g = is_k ? job : job - p.hkv;
    const long long vec0 = kv_vec(p.pg, p.rows.cap, b, g, base);
    if (vec0 < 0) {
      if (lane == 0) set_status(p.status, CC_ERR_DEVICE_ARG);
      continue;
    }
    const int vstep = p.pg.head_major ? 1 : p.hkv;
    const long long ld = is_k ? p.k_ld : p.v_ld;
    const T *src = reinterpret_cast<const T *>(is_k ? p.k : p.v) + r0 * ld + g * DH + at8;
    const bool turn = is_k && p.rotate;
    float inv = is_k ? p.k_qscale : p.v_qscale;
    const bool by_block = p.format == CC_KV_E4M3_BLOCK;
    uint8_t *codes = reinterpret_cast<uint8_t *>(is_k ? p.kc : p.vc);
    if (by_block) {
      // a block lies in one page: its scale is the one of its first slot
      const long long ei = p.pg.head_major ? vec0 / B : (vec0 / p.hkv) / B * p.hkv + g;
      uint8_t *ep = (is_k ? p.ke : p.ve) + ei;
      const int e_old = old ? *ep : 0;
      float bound = 0.f;
#pragma unroll 2
      for (int r = team; r < n; r += RPI) {
        float a[8], c[8];
        load8(src + r * ld, a);
        load8(src + r * ld + HALF, c);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const float x = finite_abs(a[i]), y = finite_abs(c[i]);
          const float hi = fmaxf(x, y);
          bound = fmaxf(bound, is_k ? __fadd_rn(hi, 0.5f * fminf(x, y)) : hi);
        }
      }
      int e = max(scale_exp(warp_max(bound)), e_old);
      if (e == 0) e = kUnitExp;   // zeros alone
      if (old && e > e_old) {
        const float f = pow2_biased(127 + e_old - e);
        for (int r = team; r < old; r += RPI) {
          uint8_t *at = codes + (vec0 + (long long)r * vstep) * DH + at8 * 2;
          uint4 u = *reinterpret_cast<const uint4 *>(at);
          uint32_t *w = &u.x;
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
          *reinterpret_cast<uint4 *>(at) = u;
        }
      }
      if (lane == 0) *ep = (uint8_t)e;
      inv = pow2_biased(254 - e);
    }
#pragma unroll 2
    for (int r = team; r < n; r += RPI) {
      float a[8], c[8];
      load8(src + r * ld, a);
      load8(src + r * ld + HALF, c);
      if (turn) rotate8(a, c, trig + r * HALF + at8);
      const long long el = (vec0 + (long long)(old + r) * vstep) * DH + at8;
      if (p.format == CC_KV_BF16) {
        __nv_bfloat16 *dst = reinterpret_cast<__nv_bfloat16 *>(codes) + el;
        store8(dst, a);
        store8(dst + HALF, c);
      } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          // one scale a layer saturates infinities, as the appends do
          a[i] = by_block && fabsf(a[i]) == INFINITY ? NAN : a[i] * inv;
          c[i] = by_block && fabsf(c[i]) == INFINITY ? NAN : c[i] * inv;
        }
        store_codes8(codes + el, a);
        store_codes8(codes + el + HALF, c);
      }
    }
  }
  if (!p.q) return;
  const int teams = gridDim.y * (kThreads / TPR);
#pragma unroll 2
  for (int i = blockIdx.y * (kThreads / TPR) + tid / TPR; i < n * p.hq; i += teams) {
    const int r = i / p.hq, h = i - r * p.hq;
    const T *src = reinterpret_cast<const T *>(p.q) + (r0 + r) * p.q_ld + h * DH + at8;
    T *dst = reinterpret_cast<T *>(p.q_out) + (r0 + r) * p.q_out_ld + h * DH + at8;
    float a[8], c[8];
    load8(src, a);
    load8(src + HALF, c);
    if (p.rotate) rotate8(a, c, trig + r * HALF + at8);
    store8(dst, a);
    store8(dst + HALF, c);
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
    cache_pos[at + i] = pos ? max(pos[s.r0 + i], 0) : follow + i;
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
  const size_t smem = p.rotate ? (size_t)std::min(p.block, p.rows.max_rows) * (DH / 2) * sizeof(float2) : 0;
  auto kern = kv_append_kernel<T, DH>;
  if (smem > 48 * 1024) {   // (a block of 128 rows of 128: 64 KB)
    const cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
    if (e != cudaSuccess) return e;
  }
  // a unit's heads over several CTAs until they fill the SMs
  const int most = std::max(1, (2 * p.hkv + p.hq) / 8);
  const int split = (int)std::min<long long>(most, std::max<long long>(1, 6LL * sms / units));
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
