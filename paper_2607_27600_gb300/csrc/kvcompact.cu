// kvcompact.cu -- in-place compaction of a block-scaled cache: slot k of every
// sequence receives old slot keep_idx[k], and the codes that come to share a block come
// to share its scale.
//
// A block's new exponent is the largest of its slots' old ones, e' = max e, so that no
// value outgrows it; the codes of the others become round(code * 2^(e - e')), one
// rounding to nearest (ties to even) of what is a shift of the exponent but near the
// format's least values.  Slots whose block's elements are no numbers (e = 255) take no part
// in e' and become NaN codes; where there are only such, the block stays one.
//
// keep_idx ascends, so a destination never lies above its source, but its write may
// clobber the source of a lower destination.  A unit is 128 destination slots (whole
// blocks) of 128 bytes of one array's slots: a head or two, which have their own scales
// and depend on nothing else.  It
//   1. copies its sources to shared memory (cp.async) with their exponents,
//   2. publishes that they are read (release),
//   3. waits (acquire, bounded) for the lower units of its array and heads that read from its
//      destinations, which a pre-pass finds from keep_idx, and
//   4. rescales and writes.
// Units are numbered sequence by sequence, slots ascending, the arrays and heads of
// the same slots side by side; a CTA takes every n-th, all CTAs are resident
// (cooperative launch), and a unit waits only on lower ones after publishing its own, so
// that nothing can deadlock.  A slot that stays where it is and keeps its scale is not written.
//
// Bound by HBM: kept codes are read once and written once.  Eight small CTAs an SM hide
// a unit's chain of loads (indices, exponents and codes, flags).
#include "kvcompact.cuh"

#include <algorithm>

namespace cc {

namespace {

constexpr int kThreads = 256;
constexpr int kPlanThreads = 256;
constexpr int kNoNumbers = 255;      // a scale exponent
constexpr uint32_t kNanCodes = 0x7F7F7F7Fu;
constexpr int kSharedBatch = 1024;   // sequences whose first chunks fit in shared memory

CC_DEV void st_release(unsigned *p, unsigned v) {
  asm volatile("st.release.gpu.global.u32 [%0], %1;" ::"l"(p), "r"(v) : "memory");
}
CC_DEV unsigned ld_acquire(const unsigned *p) {
  unsigned v;
  asm volatile("ld.acquire.gpu.global.u32 %0, [%1];" : "=r"(v) : "l"(p) : "memory");
  return v;
}
CC_DEV bool wait_flag(const unsigned *flag, unsigned *status) {
  if (ld_acquire(flag)) return true;
  const uint64_t t0 = globaltimer();
  for (uint32_t it = 1;; ++it) {
    if (ld_acquire(flag)) return true;
    __nanosleep(32);
    if ((it & 255u) == 0 && globaltimer() - t0 > kWaitLimitNs) {
      set_status(status, CC_ERR_TIMEOUT);
      return false;
    }
  }
}
CC_DEV void copy16(uint32_t dst, const void *src) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}
CC_DEV void copy_wait_all() { asm volatile("cp.async.wait_all;" ::: "memory"); }

// Kept slots of sequence b (0 and reported by the pre-pass: a count outside [0, cap]).
CC_DEV int kept_of(const KvCompactParams &p, int b) {
  const int j = p.keep_count[b];
  return j < 0 || j > p.cap ? 0 : j;
}
// Source of destination k: an entry below it or past the buffer stands for k itself
// (reported by the pre-pass).
CC_DEV int source_of(const KvCompactParams &p, const int32_t *idx, int k) {
  const int s = idx[k];
  return s < k || s >= p.cap ? k : s;
}

// Pre-pass.  Blocks of y = batch: the sequences' first chunks.  Else, for sequence y: of
// each chunk of slots the first kept slot whose source lies in it or past it (entry k
// fills the chunks between its source's and the one before), and a check of the entries.
// All clear a share of the flags.
__global__ void __launch_bounds__(kPlanThreads) plan_kernel(const __grid_constant__ KvCompactParams p) {
  const int b = blockIdx.y;
  const size_t blocks = (size_t)gridDim.x * gridDim.y, block = (size_t)blockIdx.y * gridDim.x + blockIdx.x;
  for (size_t i = block * kPlanThreads + threadIdx.x; i < p.flag_count / 4; i += blocks * kPlanThreads)
    reinterpret_cast<uint4 *>(p.flags)[i] = make_uint4(0u, 0u, 0u, 0u);
  if (b == p.batch) {
    if (blockIdx.x > 0) return;
    __shared__ int warp_sums[kPlanThreads / 32];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    int carry = 0;
    for (int b0 = 0; b0 < p.batch; b0 += kPlanThreads) {
      const int t = b0 + threadIdx.x;
      int n = 0;
      if (t < p.batch) {
        if (p.keep_count[t] != kept_of(p, t)) set_status(p.status, CC_ERR_DEVICE_ARG);
        n = (kept_of(p, t) + kCompactChunk - 1) / kCompactChunk;
      }
      int incl = n;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const int v = __shfl_up_sync(0xFFFFFFFFu, incl, o);
        if (lane >= o) incl += v;
      }
      if (lane == 31) warp_sums[warp] = incl;
      __syncthreads();
      int add = carry;
      for (int w = 0; w < kPlanThreads / 32; ++w) {
        if (w < warp) add += warp_sums[w];
        carry += warp_sums[w];
      }
      if (t < p.batch) p.first_chunk[t] = add + incl - n;
      __syncthreads();
    }
    if (threadIdx.x == 0) p.first_chunk[p.batch] = carry;
    return;
  }
  const int J = kept_of(p, b), n = p.seq_len[b];
  const int32_t *idx = p.keep_idx + (size_t)b * p.cap;
  int *reader = p.reader + (size_t)b * p.reader_ld;
  for (int k = blockIdx.x * kPlanThreads + threadIdx.x; k < J; k += gridDim.x * kPlanThreads) {
    const int s = idx[k], before = k > 0 ? idx[k - 1] : -1;
    if (s < k || s >= n || s <= before || n > p.cap) set_status(p.status, CC_ERR_DEVICE_ARG);
    const int c = source_of(p, idx, k) / kCompactChunk;
    for (int u = k > 0 ? source_of(p, idx, k - 1) / kCompactChunk + 1 : 0; u <= c; ++u) reader[u] = k;
    if (k == J - 1)
      for (int u = c + 1; u < p.reader_ld; ++u) reader[u] = J;
  }
}

// 16 codes times 2^-fall (fall = 0 .. 255), rounded to nearest even.  Through fp16, which
// holds code * 2^-fall exactly down to 2^-14 and else on a grid of 2^-24, fine enough that what
// rounds to a code of 0 (up to 2^-10) stays on its side.
CC_DEV uint4 rescale(uint4 v, int fall) {
  const int e = 15 - fall;   // of 2^-fall as fp16
  const uint32_t bits = e > 0 ? (uint32_t)e << 10 : e > -10 ? 1u << (9 + e) : 0u;
  const uint32_t f2 = bits | (bits << 16);
  const __half2 f = *reinterpret_cast<const __half2 *>(&f2);
  uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    unsigned short half[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      uint32_t x;
      asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(x) : "h"((unsigned short)(w[i] >> (16 * h))));
      const __half2 y = __hmul2(*reinterpret_cast<const __half2 *>(&x), f);
      asm("cvt.rn.satfinite.e4m3x2.f16x2 %0, %1;" : "=h"(half[h]) : "r"(*reinterpret_cast<const uint32_t *>(&y)));
    }
    w[i] = (uint32_t)half[0] | ((uint32_t)half[1] << 16);
  }
  return make_uint4(w[0], w[1], w[2], w[3]);
}

__global__ void __launch_bounds__(kThreads, 8) compact_kernel(const __grid_constant__ KvCompactParams p) {
  constexpr int C = kCompactChunk;
  __shared__ __align__(16) uint8_t st[C * kCompactWidth];
  __shared__ int base_sh[kSharedBatch + 1];
  __shared__ long long from_sh[C], to_sh[C];   // vectors of 16 bytes in the array (-1: not moved)
  __shared__ int e_sh[2][C], new_sh[2][C];     // exponents of the slots, and of their new blocks
  __shared__ int go_sh;
  const int tid = threadIdx.x;
  const bool cached = p.batch <= kSharedBatch;
  if (cached)
    for (int i = tid; i <= p.batch; i += kThreads) base_sh[i] = p.first_chunk[i];
  if (blockIdx.x == 0)   // the new lengths; no unit reads seq_len
    for (int b = tid; b < p.batch; b += kThreads) p.seq_len[b] = kept_of(p, b);
  __syncthreads();
  const int *base = cached ? base_sh : p.first_chunk;
  const long long total = (long long)base[p.batch] * p.planes;
  const int log_block = 31 - __clz(p.block);
  for (long long u = blockIdx.x; u < total; u += gridDim.x) {
    const int chunk = (int)(u / p.planes), plane = (int)(u - (long long)chunk * p.planes);
    int lo = 0, hi = p.batch - 1;
    while (lo < hi) {   // the last sequence whose first chunk is at or before it
      const int mid = (lo + hi + 1) >> 1;
      if (base[mid] <= chunk) lo = mid; else hi = mid - 1;
    }
    const int b = lo, c = chunk - base[b], k0 = c * C;
    const int J = kept_of(p, b), rows = min(C, J - k0);
    const int32_t *idx = p.keep_idx + (size_t)b * p.cap;
    // which chunks of the sequence read from this one's slots
    int r_lo = 0, r_hi = -1;
    if (tid < 32) {
      const int *reader = p.reader + (size_t)b * p.reader_ld;
      const int k_lo = reader[c], k_hi = reader[c + 1] - 1;
      r_lo = max(0, k_lo / C);
      r_hi = k_hi >= k_lo ? min(c - 1, k_hi / C) : -1;
    }
    unsigned *flags = p.flags + (u - (long long)c * p.planes);   // of the sequence's first chunk
    // ---- what the plane is: heads of an array of codes, columns of h, or the small arrays
    const bool codes = plane < p.n_arrays * p.array_planes;
    const bool small = plane == p.planes - 1;
    const int array = codes ? plane / p.array_planes : 0, part = codes ? plane - array * p.array_planes
                                                              : plane - p.n_arrays * p.array_planes;
    uint8_t *buf;
    long long row_bytes, column;   // bytes between slots, and of the plane's first byte in one
    int width, heads = 0, g = 0;
    if (codes) {
      buf = p.codes[array];
      if (p.pg.head_major) {
        g = part;
        heads = 1;
        row_bytes = p.head_dim;
        column = (long long)g * p.cap * p.head_dim;
      } else {
        const int each = kCompactWidth / p.head_dim;
        g = part * each;
        heads = min(each, p.hkv - g);
        row_bytes = (long long)p.hkv * p.head_dim;
        column = (long long)g * p.head_dim;
      }
      width = heads * p.head_dim;
    } else {
      buf = p.h;
      row_bytes = p.h_bytes;
      column = (long long)part * kCompactWidth;
      width = small ? 0 : min(kCompactWidth, p.h_bytes - part * kCompactWidth);
    }
    // ---- the slots' places and exponents
    if (tid < C) {
      const int k = k0 + tid;
      long long from = -1, to = -1;
      int e0 = -1, e1 = -1;
      if (tid < rows) {
        const int s = source_of(p, idx, k);
        if (codes) {
          long long sr, dr;
          if (p.pg.head_major) {
            sr = (long long)b * p.hkv * p.cap + s;
            dr = (long long)b * p.hkv * p.cap + k;
          } else {
            sr = kv_row(p.pg, p.cap, b, s);
            dr = kv_row(p.pg, p.cap, b, k);
          }
          if (sr < 0 || dr < 0) {
            set_status(p.status, CC_ERR_DEVICE_ARG);   // no such page: the slot stays
          } else {
            from = sr * row_bytes + column;
            to = dr * row_bytes + column;
            const uint8_t *ex = p.exps[array];
            if (p.pg.head_major) {
              e0 = ex[(((long long)b * p.hkv + g) * p.cap + s) >> log_block];
            } else {
              const long long at = (sr >> log_block) * p.hkv + g;
              e0 = ex[at];
              if (heads > 1) e1 = ex[at + 1];
            }
          }
        } else {
          from = ((long long)b * p.cap + s) * row_bytes + column;
          to = ((long long)b * p.cap + k) * row_bytes + column;
        }
        if (small) {
          from = (long long)b * p.cap + s;
          to = (long long)b * p.cap + k;
        }
      }
      from_sh[tid] = from;
      to_sh[tid] = to;
      e_sh[0][tid] = e0;
      e_sh[1][tid] = e1;
    }
    __syncthreads();
    // ---- 1. the sources
    const int pieces = width / 16;
    uint32_t small_v[3] = {0, 0, 0};
    if (small) {
      if (tid < C && from_sh[tid] >= 0) {
        const long long at = from_sh[tid];
        small_v[0] = p.tokens[at];
        small_v[1] = p.pos[at];
        if (p.acc) small_v[2] = __float_as_uint(p.acc[at]);
        uint32_t *v = reinterpret_cast<uint32_t *>(st);
#pragma unroll
        for (int i = 0; i < 3; ++i) v[i * C + tid] = small_v[i];
      }
    } else {
      const uint32_t dst = smem_u32(st);
      for (int i = tid; i < C * pieces; i += kThreads) {
        const int r = i / pieces, q = i - r * pieces;
        if (from_sh[r] >= 0) copy16(dst + r * kCompactWidth + q * 16, buf + from_sh[r] + q * 16);
      }
    }
    // ---- the blocks' new exponents
    if (tid < 2 * C) {
      const int h = tid / C, r = tid - h * C;
      const int first = r & ~(p.block - 1);
      int top = -1, any = -1;
      if (h < heads)
        for (int i = 0; i < p.block; ++i) {
          const int e = e_sh[h][first + i];
          any = max(any, e);
          if (e != kNoNumbers) top = max(top, e);
        }
      new_sh[h][r] = top >= 0 ? top : any;   // (none a number: stays 255; no slot: -1)
    }
    copy_wait_all();
    __syncthreads();
    // ---- 2. published; 3. the units that read from the destinations
    if (tid < 32) {
      if (tid == 0) st_release(&flags[(long long)c * p.planes], 1u);
      bool go = true;
      for (int r = r_lo + tid; r <= r_hi; r += 32) go &= wait_flag(&flags[(long long)r * p.planes], p.status);
      go = __all_sync(0xFFFFFFFFu, go);
      if (tid == 0) go_sh = go;
    }
    __syncthreads();
    // ---- 4. the destinations
    if (go_sh) {
      if (small) {
        if (tid < C && to_sh[tid] >= 0 && to_sh[tid] != from_sh[tid]) {
          const uint32_t *v = reinterpret_cast<const uint32_t *>(st);
          const long long at = to_sh[tid];
          p.tokens[at] = v[tid];
          p.pos[at] = v[C + tid];
          if (p.acc) p.acc[at] = __uint_as_float(v[2 * C + tid]);
        }
      } else {
        for (int i = tid; i < C * pieces; i += kThreads) {
          const int r = i / pieces, q = i - r * pieces;
          if (to_sh[r] < 0) continue;
          uint4 v = *reinterpret_cast<const uint4 *>(st + r * kCompactWidth + q * 16);
          bool same = to_sh[r] == from_sh[r];
          if (codes) {
            const int h = q * 16 / p.head_dim, e = e_sh[h][r], e1 = new_sh[h][r];
            if (e != e1) {
              same = false;
              v = e == kNoNumbers ? make_uint4(kNanCodes, kNanCodes, kNanCodes, kNanCodes)
                                  : rescale(v, e == 0 ? 255 : e1 - e);
            }
          }
          if (!same) *reinterpret_cast<uint4 *>(buf + to_sh[r] + q * 16) = v;
        }
        if (codes && tid < 2 * C) {   // a block's first slot writes its exponent
          const int h = tid / C, r = tid - h * C;
          if (h < heads && r < rows && (r & (p.block - 1)) == 0 && new_sh[h][r] >= 0) {
            // (the first slot's page, or that of the slots of its block: one page)
            long long at;
            if (p.pg.head_major) {
              at = (((long long)b * p.hkv + g) * p.cap + k0 + r) >> log_block;
            } else {
              const long long dr = kv_row(p.pg, p.cap, b, k0 + r);
              at = dr < 0 ? -1 : (dr >> log_block) * p.hkv + g + h;
            }
            if (at >= 0) p.exps[array][at] = (uint8_t)new_sh[h][r];
          }
        }
      }
    }
    __syncthreads();   // shared memory is read
  }
}

}  // namespace

void kv_compact_plan(KvCompactParams &p) {
  const int each = p.pg.head_major ? 1 : kCompactWidth / p.head_dim;
  p.array_planes = (p.hkv + each - 1) / each;
  p.h_planes = p.h ? (p.h_bytes + kCompactWidth - 1) / kCompactWidth : 0;
  p.planes = p.n_arrays * p.array_planes + p.h_planes + 1;
  const int chunks = (p.cap + kCompactChunk - 1) / kCompactChunk;
  p.reader_ld = chunks + 1;
  p.flag_count = ((size_t)p.batch * chunks * p.planes + 3) & ~size_t(3);
}

namespace {
size_t align256(size_t x) { return (x + 255) & ~size_t(255); }
}

size_t kv_compact_bytes(const KvCompactParams &p) {
  return align256((size_t)(p.batch + 1) * 4) + align256((size_t)p.batch * p.reader_ld * 4) + align256(p.flag_count * 4);
}

void kv_compact_bind(KvCompactParams &p, void *ws) {
  uint8_t *w = reinterpret_cast<uint8_t *>(ws);
  p.first_chunk = reinterpret_cast<int *>(w);
  w += align256((size_t)(p.batch + 1) * 4);
  p.reader = reinterpret_cast<int *>(w);
  w += align256((size_t)p.batch * p.reader_ld * 4);
  p.flags = reinterpret_cast<unsigned *>(w);
}

cudaError_t launch_kv_compact(const KvCompactParams &p, int sms, cudaStream_t st) {
  static int resident[64] = {};
  int dev = 0;
  cudaGetDevice(&dev);
  if (dev < 0 || dev >= 64) return cudaErrorInvalidDevice;
  if (!resident[dev]) {
    int n = 0;
    const cudaError_t e = cudaOccupancyMaxActiveBlocksPerMultiprocessor(&n, compact_kernel, kThreads, 0);
    if (e != cudaSuccess) return e;
    if (n < 1) return cudaErrorLaunchOutOfResources;
    resident[dev] = n;
  }
  const int blocks = std::max(1, std::min((p.cap + kPlanThreads - 1) / kPlanThreads, 4096 / (p.batch + 1)));
  plan_kernel<<<dim3(blocks, p.batch + 1), kPlanThreads, 0, st>>>(p);
  cudaError_t e = cudaGetLastError();
  if (e != cudaSuccess) return e;
  const long long most = (long long)p.batch * ((p.cap + kCompactChunk - 1) / kCompactChunk) * p.planes;
  const int grid = (int)std::min<long long>((long long)sms * resident[dev], most);
  void *args[] = {const_cast<KvCompactParams *>(&p)};
  return cudaLaunchCooperativeKernel((const void *)compact_kernel, dim3(grid), dim3(kThreads), args, 0, st);
}

}  // namespace cc
