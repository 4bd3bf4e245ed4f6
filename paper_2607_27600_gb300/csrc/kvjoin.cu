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

template <typename T>
__global__ void __launch_bounds__(kThreads) kv_join_kernel(const __grid_constant__ KvJoinParams p) {
  constexpr int E = 16 / sizeof(T);
  const int per_head = p.head_dim / E, per_row = p.hq * per_head;   // threads
  const long long at = (long long)blockIdx.x * kThreads + threadIdx.x;
  // (a warp's threads past the end, whole heads of them, leave together)
  if (at >= (long long)p.n_rows * per_row) return;
  const unsigned team = __activemask();
  const int row = (int)(at / per_row), in_row = (int)(at - (long long)row * per_row);
  const int head = in_row / per_head;
  const long long rh = (long long)row * p.hq + head;
  float m = -INFINITY;
  bool bad = false;   // a row that failed in a part
  for (int i = 0; i < p.n_parts; ++i) {
    const float s = p.part_lse[i][rh];
    bad |= !(s < INFINITY);
    m = fmaxf(m, s);
  }
  float total = 0.f, y[E];
#pragma unroll
  for (int e = 0; e < E; ++e) y[e] = 0.f;
  if (!bad && m > -INFINITY)
    for (int i = 0; i < p.n_parts; ++i) {
      const float w = exp2f((p.part_lse[i][rh] - m) * kLog2e);
      if (w == 0.f) continue;
      total += w;
      float x[E];
      unpack<T>(*reinterpret_cast<const uint4 *>(reinterpret_cast<const T *>(p.part[i]) + row * p.part_ld[i] +
                                                 (long long)in_row * E), x);
#pragma unroll
      for (int e = 0; e < E; ++e) y[e] = fmaf(w, x[e], y[e]);
    }
  if (total > 0.f) {
#pragma unroll
    for (int e = 0; e < E; ++e) y[e] = y[e] / total;
  }
  *reinterpret_cast<uint4 *>(reinterpret_cast<T *>(p.out) + row * p.out_ld + (long long)in_row * E) = pack<T>(y);
  __syncwarp(team);   // (lse may be one of the parts')
  if (p.lse && in_row % per_head == 0) p.lse[rh] = bad ? NAN : total > 0.f ? m + logf(total) : -INFINITY;
}

}  // namespace

cudaError_t launch_kv_join(const KvJoinParams &p, cudaStream_t st) {
  const int e = p.dtype == CC_F32 ? 4 : 8;
  const long long threads = (long long)p.n_rows * p.hq * p.head_dim / e;
  const unsigned grid = (unsigned)((threads + kThreads - 1) / kThreads);
  if (p.dtype == CC_F32) kv_join_kernel<float><<<grid, kThreads, 0, st>>>(p);
  else if (p.dtype == CC_F16) kv_join_kernel<__half><<<grid, kThreads, 0, st>>>(p);
  else kv_join_kernel<__nv_bfloat16><<<grid, kThreads, 0, st>>>(p);
  return cudaGetLastError();
}

}  // namespace cc
