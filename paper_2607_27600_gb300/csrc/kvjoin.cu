// kvjoin.cu -- attention over disjoint slots joined by the parts' log-sum-exp.
//
// With parts (o_i, s_i) of one row and head, m = max s_i and w_i = e^(s_i - m):
//   out = sum_i w_i o_i / sum_i w_i,   lse = m + ln sum_i w_i.
// A part that saw no slot (s_i = -inf) has weight 0 and is not looked at.  Weights and
// sums are fp32, one rounding at the end.
//
// Bound by HBM: each part is read once, out written once.  A head's elements are
// 16 bytes a thread, all of them in one warp, so that each lane computes the weights for
// itself (the loads of a head's s_i are one sector) and out or lse may lie where a part
// does: a thread reads its own elements, and a warp its heads' s_i, before either is written.
// 8192 rows of 32 heads of 128, two bf16 parts: 43 us, 4.8 TB/s, in 16384 CTAs of which a thread's
// life is its addresses (with a division), one round of loads and one store; up to 300 rows the launch
// and the call bound it (12 - 16 us).
#include "kvjoin.cuh"

#include <type_traits>

namespace cc {

namespace {

constexpr int kThreads = 256;
constexpr float kLog2e = 1.44269504088896341f;

template <typename T>
CC_DEV void unpack(const uint4 &u, float (&x)[16 / sizeof(T)]) {
  const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if constexpr (std::is_same_v<T, float>) {
      x[i] = __uint_as_float(w[i]);
    } else if constexpr (std::is_same_v<T, __half>) {
      const float2 f = __half22float2(*reinterpret_cast<const __half2 *>(&w[i]));
      x[2 * i] = f.x;
      x[2 * i + 1] = f.y;
    } else {
      x[2 * i] = bf16_lo(w[i]);
      x[2 * i + 1] = bf16_hi(w[i]);
    }
  }
}
template <typename T>
CC_DEV uint4 pack(const float (&x)[16 / sizeof(T)]) {
  uint32_t w[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if constexpr (std::is_same_v<T, float>) w[i] = __float_as_uint(x[i]);
    else if constexpr (std::is_same_v<T, __half>) w[i] = pack_f16x2(x[2 * i], x[2 * i + 1]);
    else w[i] = pack_bf16x2(x[2 * i], x[2 * i + 1]);
  }
  return make_uint4(w[0], w[1], w[2], w[3]);
}

// PARTS: their number where there are few, all of whose loads then start at once; 0: any
// number, four at a time after all of their s_i.
template <typename T, int PARTS>
__global__ void __launch_bounds__(kThreads) kv_join_kernel(const __grid_constant__ KvJoinParams p) {
  constexpr int E = 16 / sizeof(T), CHUNK = PARTS > 0 ? PARTS : 4;
  const int n_parts = PARTS > 0 ? PARTS : p.n_parts;
  const int per_head = p.head_dim / E, per_row = p.hq * per_head;   // threads
  const long long at = (long long)blockIdx.x * kThreads + threadIdx.x, end = (long long)p.n_rows * per_row;
  // (a warp's threads past the end, whole heads of them, leave together)
  if (at >= end) return;
  const long long stay = end - (at - (threadIdx.x & 31));
  const unsigned team = stay < 32 ? (1u << stay) - 1u : ~0u;
  const int row = end < (1ll << 32) ? (int)((unsigned)at / (unsigned)per_row) : (int)(at / per_row);
  const int in_row = (int)(at - (long long)row * per_row);
  const int head = in_row / per_head;
  const long long rh = (long long)row * p.hq + head, elem = (long long)in_row * E;
  uint4 u[CHUNK];
  float s[CHUNK];
  // (what a part that saw no slot holds is loaded with the others, and left out)
  auto load = [&](int i0) {
#pragma unroll
    for (int i = 0; i < CHUNK; ++i)
      if (PARTS > 0 || i0 + i < n_parts) {
        u[i] = __ldcs(reinterpret_cast<const uint4 *>(reinterpret_cast<const T *>(p.part[i0 + i]) +
                                                      row * p.part_ld[i0 + i] + elem));
        s[i] = p.part_lse[i0 + i][rh];
      }
  };
  float m = -INFINITY;
  bool bad = false;   // a row that failed in a part
  load(0);
  if constexpr (PARTS > 0) {
#pragma unroll
    for (int i = 0; i < PARTS; ++i) {
      bad |= !(s[i] < INFINITY);
      m = fmaxf(m, s[i]);
    }
  } else {
    for (int i = 0; i < n_parts; ++i) {
      const float si = p.part_lse[i][rh];
      bad |= !(si < INFINITY);
      m = fmaxf(m, si);
    }
  }
  float total = 0.f, y[E];
#pragma unroll
  for (int e = 0; e < E; ++e) y[e] = 0.f;
  for (int i0 = 0; i0 < n_parts; i0 += CHUNK) {
    if (i0 > 0) load(i0);
#pragma unroll
    for (int i = 0; i < CHUNK; ++i) {
      if (PARTS == 0 && i0 + i >= n_parts) break;
      const float w = bad || s[i] == -INFINITY ? 0.f : exp2f((s[i] - m) * kLog2e);
      if (w == 0.f) continue;
      total += w;
      float x[E];
      unpack<T>(u[i], x);
#pragma unroll
      for (int e = 0; e < E; ++e) y[e] = fmaf(w, x[e], y[e]);
    }
  }
  const float inv = total > 0.f ? 1.f / total : 0.f;
#pragma unroll
  for (int e = 0; e < E; ++e) y[e] *= inv;
  *reinterpret_cast<uint4 *>(reinterpret_cast<T *>(p.out) + row * p.out_ld + elem) = pack<T>(y);
  __syncwarp(team);   // (lse may be one of the parts')
  if (p.lse && in_row % per_head == 0) p.lse[rh] = bad ? NAN : total > 0.f ? m + logf(total) : -INFINITY;
}

template <typename T>
void launch(const KvJoinParams &p, unsigned grid, cudaStream_t st) {
  switch (p.n_parts) {
    case 1: kv_join_kernel<T, 1><<<grid, kThreads, 0, st>>>(p); break;
    case 2: kv_join_kernel<T, 2><<<grid, kThreads, 0, st>>>(p); break;
    case 3: kv_join_kernel<T, 3><<<grid, kThreads, 0, st>>>(p); break;
    case 4: kv_join_kernel<T, 4><<<grid, kThreads, 0, st>>>(p); break;
    default: kv_join_kernel<T, 0><<<grid, kThreads, 0, st>>>(p);
  }
}

}  // namespace

cudaError_t launch_kv_join(const KvJoinParams &p, cudaStream_t st) {
  const int e = p.dtype == CC_F32 ? 4 : 8;
  const long long threads = (long long)p.n_rows * p.hq * p.head_dim / e;
  const unsigned grid = (unsigned)((threads + kThreads - 1) / kThreads);
  if (p.dtype == CC_F32) launch<float>(p, grid, st);
  else if (p.dtype == CC_F16) launch<__half>(p, grid, st);
  else launch<__nv_bfloat16>(p, grid, st);
  return cudaGetLastError();
}

}  // namespace cc
