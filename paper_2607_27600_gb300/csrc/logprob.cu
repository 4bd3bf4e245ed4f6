// logprob.cu -- log-probability of a given token, entropy and the largest
// alternatives of each row of logits, in one pass over the logits.
//
//   S = sum e^(z - m), W = sum e^(z - m) (z - m) with a running maximum m;
//   ln p_t = (z_t - m) - ln S,  H = ln S - W / S.
// m is kept exact (every 2 vectors), not raised lazily: with a reference well
// below the maximum the two terms of H would cancel.
//
// Alternatives without a second pass: each thread keeps its largest logit and
// where that is.  The top-th largest of the CTA's thread maxima is a lower bound
// of the top-th largest logit, so only the `top` threads at or above it hold
// candidates, and their few dozen vectors are read again (from L2).  Keys
// of (value, lower position first) are all distinct, so ties change nothing.
//
// Bound by HBM.  A CTA takes a row; with few rows a cluster of up to 8 CTAs
// does, a contiguous segment each, and rank 0 joins their sums and sorted lists
// through distributed shared memory.
#include "logprob.cuh"

#include <float.h>

#include <type_traits>

namespace cc {

namespace {

constexpr int kThreads = 512, kWarps = kThreads / 32;
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kFar = -200.f;   // e^x is 0 in fp32 below

CC_DEV float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
CC_DEV uint4 load_once(const void *p) {
  uint4 v;
  asm volatile("ld.global.nc.L1::no_allocate.v4.u32 {%0,%1,%2,%3}, [%4];"
               : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p));
  return v;
}

template <typename T>
CC_DEV float to_float(T x) {
  if constexpr (std::is_same_v<T, float>) return x;
  else if constexpr (std::is_same_v<T, __half>) return __half2float(x);
  else return __bfloat162float(x);
}

// One row as 16-byte vectors: vector v holds elements v * N - skip + [0, N), of
// which those outside [0, vocab) do not exist.
template <typename T>
struct Row {
  static constexpr int N = 16 / sizeof(T);
  const T *base;   // 16-byte aligned, `skip` elements before the row
  int skip, vocab;
  CC_DEV Row(const T *row, int n) : vocab(n) {
    skip = (int)((reinterpret_cast<uintptr_t>(row) & 15) / sizeof(T));
    base = row - skip;
  }
  CC_DEV int vectors() const { return (int)(((long long)vocab + skip + N - 1) / N); }
  CC_DEV int first(int v) const { return v * N - skip; }
  CC_DEV bool whole(int v) const { return first(v) >= 0 && (long long)first(v) + N <= vocab; }
  CC_DEV void widen(uint4 u, float (&x)[N]) const {
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if constexpr (std::is_same_v<T, float>) {
        x[i] = __uint_as_float(w[i]);
      } else if constexpr (std::is_same_v<T, __half>) {
        const float2 f = __half22float2(*reinterpret_cast<const __half2 *>(&w[i]));
        x[2 * i] = f.x, x[2 * i + 1] = f.y;
      } else {
        x[2 * i] = bf16_lo(w[i]), x[2 * i + 1] = bf16_hi(w[i]);
      }
    }
  }
  // (a vector at the row's ends: what lies outside reads as -inf)
  CC_DEV void load(int v, float (&x)[N]) const {
    if (whole(v)) {
      widen(load_once(base + (long long)v * N), x);
    } else {
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const int e = first(v) + i;
        x[i] = e >= 0 && e < vocab ? to_float(base[(long long)v * N + i]) : -INFINITY;
      }
    }
  }
};

// Order of alternatives as one whole number, larger first: the value (NaN as
// -inf, -0 as 0), then the lower position.  0 is below every key.
CC_DEV uint32_t ordered(float z) {
  const float y = z != z ? -INFINITY : z + 0.f;
  const uint32_t u = __float_as_uint(y);
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}
CC_DEV float from_ordered(uint32_t o) {
  return __uint_as_float(o & 0x80000000u ? o & 0x7FFFFFFFu : ~o);
}
typedef unsigned long long Key;
CC_DEV Key make_key(uint32_t order, uint32_t at) { return ((Key)order << 32) | (0xFFFFFFFFu - at); }
CC_DEV uint32_t key_at(Key k) { return 0xFFFFFFFFu - (uint32_t)k; }

// Lists of a warp: lane i holds the i-th largest of 32 keys.
CC_DEV Key sort_step(Key k, int step, bool descending) {
  const Key o = __shfl_xor_sync(0xFFFFFFFFu, k, step);
  const bool low = (threadIdx.x & step) == 0;
  return (low == descending) == (k > o) ? k : o;
}
CC_DEV Key sort_list(Key k) {
#pragma unroll
  for (int size = 2; size <= 32; size <<= 1)
#pragma unroll
    for (int step = size >> 1; step > 0; step >>= 1)
      k = sort_step(k, step, (threadIdx.x & size & 31) == 0);
  return k;
}
CC_DEV Key merge_lists(Key a, Key b) {   // the 32 largest of both
  const Key r = __shfl_xor_sync(0xFFFFFFFFu, b, 31);
  Key k = a > r ? a : r;
#pragma unroll
  for (int step = 16; step > 0; step >>= 1) k = sort_step(k, step, true);
  return k;
}
CC_DEV Key insert_key(Key list, Key k) {
  const int at = __popc(__ballot_sync(0xFFFFFFFFu, list > k)), lane = threadIdx.x & 31;
  const Key up = __shfl_up_sync(0xFFFFFFFFu, list, 1);
  return lane < at ? list : lane == at ? k : up;
}

struct Sums {
  float m, s, w;
};
CC_DEV Sums join(Sums a, Sums b) {
  const float m = fmaxf(a.m, b.m);
  const float da = fmaxf(a.m - m, kFar), db = fmaxf(b.m - m, kFar);
  // a maximum of +inf: its own sum is NaN already
  const float fa = ex2(da * kLog2e), fb = ex2(db * kLog2e);
  return {m, a.s * fa + b.s * fb, fa * (a.w + a.s * da) + fb * (b.w + b.s * db)};
}
CC_DEV Sums warp_join(Sums x) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1)
    x = join(x, {__shfl_xor_sync(0xFFFFFFFFu, x.m, o), __shfl_xor_sync(0xFFFFFFFFu, x.s, o),
                 __shfl_xor_sync(0xFFFFFFFFu, x.w, o)});
  return x;
}

template <typename T>
__global__ void __launch_bounds__(kThreads, 2)
    token_logprob_kernel(const __grid_constant__ LogprobParams p) {
  constexpr int N = Row<T>::N;
  __shared__ Key lists[kWarps][32];
  __shared__ float sums[kWarps][3];
  __shared__ Key part_list[8][32];   // rank 0: the cluster's
  __shared__ float part_sums[8][3];
  __shared__ int marked[kMaxTop], n_marked;
  const int cl = (int)cluster_nctarank(), rank = (int)cluster_ctarank();
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int r = blockIdx.x / cl;
  if (cl > 1)   // the other CTAs of the cluster have started before their memory is written
    asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
  const T *row_ptr = reinterpret_cast<const T *>(p.logits) + (long long)r * p.ld;
  const Row<T> row(row_ptr, p.vocab);
  const int nv = row.vectors();
  const int v0 = (int)((long long)nv * rank / cl), v1 = (int)((long long)nv * (rank + 1) / cl);

  // ---- one pass: sums, and the thread's largest logit
  Sums a{-FLT_MAX, 0.f, 0.f};
  float best = -INFINITY;
  int best_v = -1;
  auto add = [&](const float (&x)[N], const float (&y)[N], int vx, int vy) {
    float mx = -INFINITY, my = -INFINITY;   // (NaN drops out)
#pragma unroll
    for (int i = 0; i < N; ++i) mx = fmaxf(mx, x[i]), my = fmaxf(my, y[i]);
    if (mx > best || best_v < 0) best = mx, best_v = vx;
    if (my > best) best = my, best_v = vy;
    const float m = fmaxf(a.m, fmaxf(mx, my));
    const float d = fmaxf(a.m - m, kFar), f = ex2(d * kLog2e);
    float s = 0.f, w = 0.f;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const float dx = x[i] - m, dy = y[i] - m;
      const float ex = ex2(dx * kLog2e), ey = ex2(dy * kLog2e);
      s += ex + ey;
      w = fmaf(ex, fmaxf(dx, kFar), w);   // (0 times -inf would be NaN)
      w = fmaf(ey, fmaxf(dy, kFar), w);
    }
    a.w = fmaf(f, fmaf(a.s, d, a.w), w);
    a.s = fmaf(a.s, f, s);
    a.m = m;
  };
  int v = v0 + tid;
  for (; v + 3 * kThreads < v1; v += 4 * kThreads) {
    uint4 u[4];
    if (row.whole(v) && row.whole(v + 3 * kThreads)) {
#pragma unroll
      for (int k = 0; k < 4; ++k) u[k] = load_once(row.base + (long long)(v + k * kThreads) * N);
      float x[N], y[N];
      row.widen(u[0], x);
      row.widen(u[1], y);
      add(x, y, v, v + kThreads);
      row.widen(u[2], x);
      row.widen(u[3], y);
      add(x, y, v + 2 * kThreads, v + 3 * kThreads);
    } else {
#pragma unroll 1
      for (int k = 0; k < 4; k += 2) {
        float x[N], y[N];
        row.load(v + k * kThreads, x);
        row.load(v + (k + 1) * kThreads, y);
        add(x, y, v + k * kThreads, v + (k + 1) * kThreads);
      }
    }
  }
#pragma unroll 1
  for (; v < v1; v += 2 * kThreads) {
    float x[N], y[N];
    row.load(v, x);
    const bool two = v + kThreads < v1;
    if (two) {
      row.load(v + kThreads, y);
    } else {
#pragma unroll
      for (int i = 0; i < N; ++i) y[i] = -INFINITY;
    }
    add(x, y, v, v + kThreads);
  }
  a = warp_join(a);
  if (lane == 0) sums[warp][0] = a.m, sums[warp][1] = a.s, sums[warp][2] = a.w;

  // ---- the segment's largest `top` as a sorted list in warp 0
  Key list = 0;
  if (p.top > 0) {
    if (tid == 0) n_marked = 0;
    const Key mine = best_v < 0 ? 0 : make_key(ordered(best), (uint32_t)best_v);
    lists[warp][lane] = sort_list(mine);
    __syncthreads();
#pragma unroll 1
    for (int w = kWarps / 2; w > 0; w >>= 1) {
      if (warp < w) lists[warp][lane] = merge_lists(lists[warp][lane], lists[warp + w][lane]);
      __syncthreads();
    }
    const Key least = lists[0][p.top - 1];   // the top-th largest thread maximum
    if (mine != 0 && mine >= least) marked[atomicAdd(&n_marked, 1)] = tid;
    __syncthreads();
    // the marked threads' vectors again, a warp at a time
#pragma unroll 1
    for (int k = warp; k < n_marked; k += kWarps) {
#pragma unroll 1
      for (int u0 = v0 + marked[k]; u0 < v1; u0 += 32 * kThreads) {
        const int u = u0 + lane * kThreads;
        float x[N];
        if (u < v1) row.load(u, x);
#pragma unroll
        for (int i = 0; i < N; ++i) {
          const int e = row.first(u) + i;
          const bool in = u < v1 && e >= 0 && e < p.vocab;
          const uint32_t o = in ? ordered(x[i]) : 0u;
          unsigned cand = __ballot_sync(0xFFFFFFFFu, in && make_key(o, (uint32_t)u) >= least);
          while (cand) {
            const int src = __ffs(cand) - 1;
            cand &= cand - 1;
            list = insert_key(list, __shfl_sync(0xFFFFFFFFu, make_key(o, (uint32_t)e), src));
          }
        }
      }
    }
    __syncthreads();   // every thread has read `least`
    lists[warp][lane] = list;
  }
  __syncthreads();
  if (warp == 0) {
    if (p.top > 0) {
      const int used = min(kWarps, max(n_marked, 1));
      list = lists[0][lane];
      for (int w = 1; w < used; ++w) list = merge_lists(list, lists[w][lane]);
    }
    a = lane < kWarps ? Sums{sums[lane][0], sums[lane][1], sums[lane][2]} : Sums{-FLT_MAX, 0.f, 0.f};
    a = warp_join(a);
  }

  // ---- the cluster's segments
  if (cl > 1) {
    asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
    if (warp == 0) {
      const uint32_t to = cluster_addr(&part_list[rank][lane], 0);
      asm volatile("st.shared::cluster.u64 [%0], %1;" ::"r"(to), "l"(list) : "memory");
      if (lane < 3) {
        const uint32_t ts = cluster_addr(&part_sums[rank][lane], 0);
        asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(ts),
                     "f"(lane == 0 ? a.m : lane == 1 ? a.s : a.w) : "memory");
      }
    }
    cluster_sync();
    if (rank != 0 || warp != 0) return;
    for (int c = 1; c < cl; ++c) {
      if (p.top > 0) list = merge_lists(list, part_list[c][lane]);
      a = join(a, {part_sums[c][0], part_sums[c][1], part_sums[c][2]});
    }
  }
  if (warp != 0) return;
  const float ln_s = logf(a.s);
  if (lane == 0) {
    // a row that allows nothing has no distribution
    const float none = a.s > 0.f ? 0.f : NAN;
    if (p.logprob) {
      const int t = p.targets[r];
      float lp = 0.f;
      if (t >= 0 && t < p.vocab) lp = to_float(row_ptr[t]) - a.m - ln_s + none;
      else if (t != -1) set_status(p.status, CC_ERR_DEVICE_ARG);
      p.logprob[r] = lp;
    }
    if (p.entropy) p.entropy[r] = ln_s - a.w / a.s;
  }
  if (lane < p.top) {
    if (p.top_ids) p.top_ids[(long long)r * p.top + lane] = (int32_t)key_at(list);
    if (p.top_logprob)
      p.top_logprob[(long long)r * p.top + lane] =
          from_ordered((uint32_t)(list >> 32)) - a.m - ln_s + (a.s > 0.f ? 0.f : NAN);
  }
}

template <typename T>
cudaError_t launch_as(const LogprobParams &p, int sms, cudaStream_t st) {
  // CTAs of a row: until two waves of the SMs' CTAs are in flight, each with a
  // few vectors per thread
  int cl = 1;
  while (cl < 8 && (long long)p.rows * cl * 2 <= 2 * sms &&
         (long long)p.vocab >= 4LL * cl * kThreads * (16 / (int)sizeof(T)))
    cl *= 2;
  if ((long long)p.rows * cl > 0x7FFFFFFFll) return cudaErrorInvalidValue;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(p.rows * cl));
  cfg.blockDim = dim3(kThreads);
  cfg.stream = st;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = cl;
  attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, token_logprob_kernel<T>, p);
}

}  // namespace

cudaError_t launch_token_logprobs(const LogprobParams &p, int sms, cudaStream_t st) {
  switch (p.dtype) {
    case CC_BF16: return launch_as<__nv_bfloat16>(p, sms, st);
    case CC_F16: return launch_as<__half>(p, sms, st);
    case CC_F32: return launch_as<float>(p, sms, st);
    default: return cudaErrorInvalidValue;
  }
}

}  // namespace cc
