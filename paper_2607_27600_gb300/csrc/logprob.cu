// logprob.cu -- log-probability of a given token, entropy and the largest
// alternatives of each row of logits, in one pass over the logits.
//
// With c = log2(e) and a running maximum m, t = z c - m c:
//   S = sum 2^t, W = sum 2^t t;  ln p_k = (z_k c - m c - log2 S) / c,
//   H = (log2 S - W / S) / c.
// m is exact after every four vectors, not raised lazily: with a reference well
// below the maximum the two terms of H would cancel.  A forbidden logit (-inf, or
// any below -2^20) is raised to -2^20, whose term is 0 in both sums; a row whose
// maximum lies near there or past 2^20 (nothing allowed, the type's lowest value
// everywhere) is done again from t = (z - m) c.
//
// Alternatives without a second pass: each thread keeps its largest logit and
// where that is.  The top-th largest maximum of 64 groups of threads is a lower
// bound of the top-th largest logit, so only the threads that reach it (hardly more
// than `top`) hold candidates, and their few dozen vectors are read again (from L2).
// Keys of (value, lower position first) are all distinct, so ties change nothing.
//
// Bound by HBM, and close behind by issue slots: 16-bit maxima and fp32 sums in pairs
// keep it under 6 instructions per logit.  A CTA takes a row; with few rows a
// cluster of up to 8 CTAs does, a contiguous segment each, and rank 0 joins their
// sums and sorted lists through distributed shared memory.
//
// 4096 rows of 128256 bf16 logits, 8 alternatives: 1.05 GB in 187 us (5.6 TB/s); 64 rows
// of 152064: 12.3 us a call, 10 of them in the kernel; one fp32 row: 10.2 us, 7.3 in the
// kernel, cluster and sort one after another.
// One of the 64 rows done again (nothing allowed, or the lowest value everywhere): 156 us,
// of one warp that reads it twice.
#include "logprob.cuh"

#include <type_traits>

namespace cc {

namespace {

constexpr float kC = 1.4426950408889634f, kLn2 = 0.69314718055994531f;
// A forbidden logit.  A power of two, so that kLow c is no rounding away from itself
// (at the maxima that the sums take, up to 2^20, z c and m c are 0.1 apart at most).
constexpr float kLow = -0x1p20f;
constexpr float kFar = -200.f;   // 2^x is 0 in fp32 below
constexpr int kManyRows = 2;     // per SM, past which a row has 256 threads
constexpr int kCand = 256;       // candidates of a segment that are sorted at once

CC_DEV float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
CC_DEV float max_nan(float a, float b) {   // NaN if either is
  float y;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(y) : "f"(a), "f"(b));
  return y;
}
CC_DEV uint4 load_once(const void *p) {
  uint4 v;
  asm volatile("ld.global.nc.L1::no_allocate.v4.u32 {%0,%1,%2,%3}, [%4];"
               : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p));
  return v;
}

CC_DEV void copy16(uint32_t dst, const void *src) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}

template <typename T>
CC_DEV float to_float(T x) {
  if constexpr (std::is_same_v<T, float>) return x;
  else if constexpr (std::is_same_v<T, __half>) return __half2float(x);
  else return __bfloat162float(x);
}

// Two logits of a vector's word (one, fp32) as fp32.
template <typename T>
CC_DEV float2 widen_word(uint32_t w) {
  if constexpr (std::is_same_v<T, __half>) return __half22float2(*reinterpret_cast<const __half2 *>(&w));
  else return make_float2(bf16_lo(w), bf16_hi(w));
}
// Larger of the logits, word by word (NaN drops out).
template <typename T>
CC_DEV uint32_t max_word(uint32_t a, uint32_t b) {
  if constexpr (std::is_same_v<T, float>) {
    return __float_as_uint(fmaxf(__uint_as_float(a), __uint_as_float(b)));
  } else {
    using V = std::conditional_t<std::is_same_v<T, __half>, __half2, __nv_bfloat162>;
    const V r = __hmax2(*reinterpret_cast<const V *>(&a), *reinterpret_cast<const V *>(&b));
    return *reinterpret_cast<const uint32_t *>(&r);
  }
}
template <typename T>
CC_DEV uint32_t max_vec(uint4 u) {
  return max_word<T>(max_word<T>(u.x, u.y), max_word<T>(u.z, u.w));
}
template <typename T>
CC_DEV float max_of_word(uint32_t w) {
  if constexpr (std::is_same_v<T, float>) {
    return __uint_as_float(w);
  } else {
    const float2 f = widen_word<T>(w);
    return fmaxf(f.x, f.y);
  }
}

// One row as 16-byte vectors: vector v holds elements v * N - skip + [0, N).
// Vectors [lo, hi) lie in the row as a whole; the few elements before and after
// them are its edges.
template <typename T>
struct Row {
  static constexpr int N = 16 / sizeof(T);
  const T *base;   // 16-byte aligned, `skip` elements before the row
  int skip, vocab, lo, hi;
  CC_DEV Row(const T *row, int n) : vocab(n) {
    skip = (int)((reinterpret_cast<uintptr_t>(row) & 15) / sizeof(T));
    base = row - skip;
    lo = skip ? 1 : 0;
    hi = max(lo, (int)(((long long)vocab + skip) / N));
  }
  CC_DEV int first(int v) const { return v * N - skip; }
  CC_DEV const T *at(int v) const { return base + (long long)v * N; }
  // Edge element i, in ascending position (or -1).
  CC_DEV int edge(int i) const {
    const int before = min(vocab, lo * N - skip);
    const int e = i < before ? i : max(first(hi), before) + i - before;
    return e < vocab ? e : -1;
  }
  CC_DEV void widen(uint4 u, float (&x)[N]) const {
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if constexpr (std::is_same_v<T, float>) {
        x[i] = __uint_as_float(w[i]);
      } else {
        const float2 f = widen_word<T>(w[i]);
        x[2 * i] = f.x, x[2 * i + 1] = f.y;
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

CC_DEV float scaled(float m) { return __fmul_rn(m, kC); }   // (rounded, whatever it is added to)

// Merges the first n lists into lists[0].  The whole CTA calls; they are written
// and every thread has seen it.
CC_DEV void merge_tree(Key (*lists)[32], int n, int warp, int lane) {
#pragma unroll 1
  while (n > 1) {
    const int half = (n + 1) / 2;
    if (warp + half < n) lists[warp][lane] = merge_lists(lists[warp][lane], lists[warp + half][lane]);
    __syncthreads();
    n = half;
  }
}

// m: the maximum, at least kLow; s, w: the sums against scaled(m).
struct Sums {
  float m, s, w;
};
CC_DEV Sums join(Sums a, Sums b) {
  const float m = fmaxf(a.m, b.m);
  // (a maximum of +inf: the sums are NaN already)
  const float mc = scaled(m), da = fmaxf(scaled(a.m) - mc, kFar), db = fmaxf(scaled(b.m) - mc, kFar);
  const float fa = ex2(da), fb = ex2(db);
  return {m, a.s * fa + b.s * fb, fa * (a.w + a.s * da) + fb * (b.w + b.s * db)};
}
CC_DEV Sums warp_join(Sums x) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1)
    x = join(x, {__shfl_xor_sync(0xFFFFFFFFu, x.m, o), __shfl_xor_sync(0xFFFFFFFFu, x.s, o),
                 __shfl_xor_sync(0xFFFFFFFFu, x.w, o)});
  return x;
}

// The sums of a word's one or two logits against mc (pairs where there are two).
template <typename T>
CC_DEV void add_word(uint32_t w, float2 mc, float2 &s, float2 &ws) {
  float2 z;
  if constexpr (std::is_same_v<T, float>) {
    z = make_float2(__uint_as_float(w), 0.f);
    const float t = fmaf(max_nan(z.x, kLow), kC, mc.x), e = ex2(t);
    s.x += e;
    ws.x = fmaf(e, t, ws.x);
  } else {
    if constexpr (std::is_same_v<T, __half>) {
      z = widen_word<T>(w);
      z = make_float2(max_nan(z.x, kLow), max_nan(z.y, kLow));
    } else {   // both at once
      const __nv_bfloat162 low = __floats2bfloat162_rn(kLow, kLow);
      const __nv_bfloat162 r = __hmax2_nan(*reinterpret_cast<const __nv_bfloat162 *>(&w), low);
      z = widen_word<T>(*reinterpret_cast<const uint32_t *>(&r));
    }
    const float2 t = __ffma2_rn(z, make_float2(kC, kC), mc), e = make_float2(ex2(t.x), ex2(t.y));
    s = __fadd2_rn(s, e);
    ws = __ffma2_rn(e, t, ws);
  }
}

template <typename T, int THREADS>
__global__ void __launch_bounds__(THREADS, 1024 / THREADS)
    token_logprob_kernel(const __grid_constant__ LogprobParams p) {
  constexpr int N = Row<T>::N, kWarps = THREADS / 32;
  extern __shared__ __align__(16) uint8_t stage_mem[];   // two batches: [2][4][THREADS] vectors
  __shared__ Key lists[kWarps][32];
  __shared__ float sums[kWarps][3];
  __shared__ Key part_list[8][32];   // rank 0: the cluster's
  __shared__ float part_sums[8][3];
  __shared__ Key groups[64], cand[kCand];
  __shared__ int marked[THREADS], n_marked, n_cand;
  const int cl = (int)cluster_nctarank(), rank = (int)cluster_ctarank();
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int r = blockIdx.x / cl;
  if (cl > 1)   // the other CTAs of the cluster have started before their memory is written
    asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
  const T *row_ptr = reinterpret_cast<const T *>(p.logits) + (long long)r * p.ld;
  const Row<T> row(row_ptr, p.vocab);
  const int nv = row.hi - row.lo;
  const int v0 = row.lo + (int)((long long)nv * rank / cl), v1 = row.lo + (int)((long long)nv * (rank + 1) / cl);

  // ---- one pass: sums, and the thread's largest logit.  Batches of four vectors
  // (the last one of fewer); a thread copies ahead what it will read itself: no barrier
  Sums a{kLow, 0.f, 0.f};
  float best = -INFINITY;
  const int mine_n = max(0, (v1 - v0 - tid + THREADS - 1) / THREADS);   // this thread's vectors
  const int full = mine_n / 4, rest = mine_n % 4;
  int best_v = mine_n > 0 ? v0 + tid : -1, v = v0 + tid;
  const uint8_t *src = reinterpret_cast<const uint8_t *>(row.at(v));
  const uint32_t ring = smem_u32(stage_mem) + tid * 16;
  auto issue = [&](int i, int st) {   // batch i
    const uint32_t to = ring + st * (4 * THREADS * 16);
    if (i < full) {
#pragma unroll
      for (int k = 0; k < 4; ++k) copy16(to + k * THREADS * 16, src + k * THREADS * 16);
      src += 4 * THREADS * 16;
    } else if (i == full) {
      for (int k = 0; k < rest; ++k) copy16(to + k * THREADS * 16, src + k * THREADS * 16);
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
  };
  issue(0, 0);
#pragma unroll 1
  for (int i = 0; i < full + (rest ? 1 : 0); ++i, v += 4 * THREADS) {
    issue(i + 1, (i + 1) & 1);
    asm volatile("cp.async.wait_group 1;" ::: "memory");
    const uint4 *here = reinterpret_cast<const uint4 *>(stage_mem) + (i & 1) * 4 * THREADS + tid;
    uint4 u[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) u[k] = here[k * THREADS];
    if (i == full) {
      constexpr uint32_t kInf = std::is_same_v<T, float> ? 0xFF800000u
                                : std::is_same_v<T, __half> ? 0xFC00FC00u : 0xFF80FF80u;
#pragma unroll
      for (int k = 1; k < 4; ++k)
        if (k >= rest) u[k] = make_uint4(kInf, kInf, kInf, kInf);
    }
    uint32_t mw[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) mw[k] = max_vec<T>(u[k]);
    const float top = max_of_word<T>(max_word<T>(max_word<T>(mw[0], mw[1]), max_word<T>(mw[2], mw[3])));
    if (top > best) {
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const float x = max_of_word<T>(mw[k]);
        if (x > best) best = x, best_v = v + k * THREADS;
      }
    }
    const float m = fmaxf(a.m, top), mc = scaled(m);
    const float d = fmaxf(scaled(a.m) - mc, kFar), f = ex2(d);
    const float2 nmc = make_float2(-mc, -mc);
    float2 s = make_float2(0.f, 0.f), ws = make_float2(0.f, 0.f);
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      add_word<T>(u[k].x, nmc, s, ws);
      add_word<T>(u[k].y, nmc, s, ws);
      add_word<T>(u[k].z, nmc, s, ws);
      add_word<T>(u[k].w, nmc, s, ws);
    }
    a.w = fmaf(f, fmaf(a.s, d, a.w), ws.x + ws.y);
    a.s = fmaf(a.s, f, s.x + s.y);
    a.m = m;
  }
  // the edges: up to 2 N - 2 elements, a lane each
  int edge = -1;
  if (rank == 0 && warp == 0) {
    edge = row.edge(lane);
    if (edge >= 0) {
      const float z = to_float(row_ptr[edge]), m = fmaxf(z, kLow);
      const float t = fmaf(max_nan(z, kLow), kC, -scaled(m)), e = ex2(t);
      a = join(a, {m, e, e * t});
    }
  }
  a = warp_join(a);
  if (lane == 0) sums[warp][0] = a.m, sums[warp][1] = a.s, sums[warp][2] = a.w;

  // ---- the segment's largest `top` as a sorted list in warp 0
  Key list = 0;
  if (p.top > 0) {
    if (tid == 0) n_marked = n_cand = 0;
    const Key mine = best_v < 0 ? 0 : make_key(ordered(best), (uint32_t)best_v);
    // the top-th largest of 64 groups' maxima bounds the top-th largest logit from
    // below, and hardly more threads than `top` reach it
    Key group = mine;
#pragma unroll
    for (int o = 1; o < THREADS / 64; o <<= 1) {
      const Key k = __shfl_xor_sync(0xFFFFFFFFu, group, o);
      group = k > group ? k : group;
    }
    if (tid % (THREADS / 64) == 0) groups[tid / (THREADS / 64)] = group;
    __syncthreads();
    const Key least = __shfl_sync(
        0xFFFFFFFFu, merge_lists(sort_list(groups[lane]), sort_list(groups[32 + lane])), p.top - 1);
    if (mine != 0 && mine >= least) marked[atomicAdd(&n_marked, 1)] = tid;
    __syncthreads();
    // their vectors again, a warp per thread; `take` gets the elements that reach the bound
    auto scan = [&](auto &&take) {
#pragma unroll 1
      for (int k = warp; k < n_marked; k += kWarps) {
#pragma unroll 1
        for (int u0 = v0 + marked[k]; u0 < v1; u0 += 32 * THREADS) {
          const int u = u0 + lane * THREADS;
          float x[N];
          row.widen(u < v1 ? load_once(row.at(u)) : make_uint4(0, 0, 0, 0), x);
#pragma unroll
          for (int i = 0; i < N; ++i) {
            const uint32_t o = ordered(x[i]);
            take(u < v1 && make_key(o, (uint32_t)u) >= least, make_key(o, (uint32_t)(row.first(u) + i)));
          }
        }
      }
      if (warp == 0)
        take(edge >= 0, edge >= 0 ? make_key(ordered(to_float(row_ptr[edge])), (uint32_t)edge) : 0);
    };
    scan([&](bool in, Key k) {
      if (!in) return;
      const int at = atomicAdd(&n_cand, 1);
      if (at < kCand) cand[at] = k;
    });
    __syncthreads();
    if (n_cand <= kCand) {
      if (warp == 0)
        for (int c = 0; c < n_cand; c += 32) {
          const Key k = sort_list(c + lane < n_cand ? cand[c + lane] : 0);
          list = c ? merge_lists(list, k) : k;
        }
    } else {   // many equal logits at the bound: each warp's largest, then all warps'
      scan([&](bool in, Key k) {
        for (unsigned some = __ballot_sync(0xFFFFFFFFu, in); some; some &= some - 1)
          list = insert_key(list, __shfl_sync(0xFFFFFFFFu, k, __ffs(some) - 1));
      });
      lists[warp][lane] = list;
      __syncthreads();
      merge_tree(lists, kWarps, warp, lane);
      list = lists[0][lane];
    }
  }
  __syncthreads();
  if (warp == 0) {
    a = lane < kWarps ? Sums{sums[lane][0], sums[lane][1], sums[lane][2]} : Sums{kLow, 0.f, 0.f};
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
    if (rank != 0) return;
    if (p.top > 0) {
      merge_tree(part_list, cl, warp, lane);
      list = part_list[0][lane];
    }
    if (warp == 0) {
      a = lane < cl ? Sums{part_sums[lane][0], part_sums[lane][1], part_sums[lane][2]} : Sums{kLow, 0.f, 0.f};
      a = warp_join(a);
    }
  }
  if (warp != 0) return;
  // ---- a row without a maximum that the sums can stand on: again, from differences
  float largest = a.m;
  const bool odd = a.m <= 0.5f * kLow || a.m >= -kLow;
  if (odd) {
    largest = -INFINITY;
    for (int e = lane; e < p.vocab; e += 32) largest = fmaxf(largest, to_float(row_ptr[e]));
    largest = warp_max(largest);
    float s = 0.f, w = 0.f;
    for (int e = lane; e < p.vocab; e += 32) {
      const float z = to_float(row_ptr[e]);
      if (z == -INFINITY) continue;
      const float t = (z - largest) * kC, x = ex2(t);
      s += x;
      w = fmaf(x, max_nan(t, kFar), w);
    }
    a.s = warp_sum(s);
    a.w = warp_sum(w);
  }
  // a row that allows nothing has no distribution
  const float log_s = a.s > 0.f ? log2f(a.s) : NAN;
  auto log_prob = [&](float z) {
    // (z c of a logit far below would be coarse, or infinite)
    return odd || fabsf(z) >= -kLow ? (z - largest) - log_s * kLn2
                                    : (fmaf(z, kC, -scaled(a.m)) - log_s) * kLn2;
  };
  if (lane == 0) {
    if (p.logprob) {
      const int t = p.targets[r];
      const bool in = t >= 0 && t < p.vocab;
      if (!in && t != -1) set_status(p.status, CC_ERR_DEVICE_ARG);
      p.logprob[r] = in ? log_prob(to_float(row_ptr[t])) : 0.f;
    }
    if (p.entropy) p.entropy[r] = (log_s - a.w / a.s) * kLn2;
  }
  if (lane < p.top) {
    if (p.top_ids) p.top_ids[(long long)r * p.top + lane] = (int32_t)key_at(list);
    if (p.top_logprob)
      p.top_logprob[(long long)r * p.top + lane] = log_prob(from_ordered((uint32_t)(list >> 32)));
  }
}

template <typename T, int THREADS>
cudaError_t launch_as(const LogprobParams &p, int cl, cudaStream_t st) {
  if ((long long)p.rows * cl > 0x7FFFFFFFll) return cudaErrorInvalidValue;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(p.rows * cl));
  cfg.blockDim = dim3(THREADS);
  cfg.dynamicSmemBytes = 2 * 4 * THREADS * 16;
  cfg.stream = st;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = cl;
  attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  static bool attr_set[64] = {};
  int dev = 0;
  cudaGetDevice(&dev);
  if (dev < 64 && !attr_set[dev]) {
    const cudaError_t e = cudaFuncSetAttribute(token_logprob_kernel<T, THREADS>,
                                               cudaFuncAttributeMaxDynamicSharedMemorySize,
                                               (int)cfg.dynamicSmemBytes);
    if (e != cudaSuccess) return e;
    attr_set[dev] = true;
  }
  return cudaLaunchKernelEx(&cfg, token_logprob_kernel<T, THREADS>, p);
}

template <typename T>
cudaError_t launch_rows(const LogprobParams &p, int sms, cudaStream_t st) {
  // Few rows: the largest clusters of which all rows' are resident at one CTA of 512
  // threads per SM (152 SMs hold 15 clusters of 8, 36 of 4 and 76 of 2), each thread
  // with a few vectors: 64 rows of 152064 bf16 logits in pairs 10.4 us, in fours 12.8.
  // Many: CTAs of 256 threads, so that the rows on an SM are at different points of
  // their work.
  if (p.rows > kManyRows * sms) return launch_as<T, 256>(p, 1, st);
  int cl = 8;
  const int hold[9] = {0, 0, sms / 2, 0, sms * 36 / 152, 0, 0, 0, sms * 15 / 152};
  while (cl > 1 && (p.rows > hold[cl] ||
                    (long long)p.vocab < 2LL * cl * 512 * (16 / (int)sizeof(T))))
    cl /= 2;
  return launch_as<T, 512>(p, cl, st);
}

}  // namespace

cudaError_t launch_token_logprobs(const LogprobParams &p, int sms, cudaStream_t st) {
  switch (p.dtype) {
    case CC_BF16: return launch_rows<__nv_bfloat16>(p, sms, st);
    case CC_F16: return launch_rows<__half>(p, sms, st);
    case CC_F32: return launch_rows<float>(p, sms, st);
    default: return cudaErrorInvalidValue;
  }
}

}  // namespace cc
