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
// Bound by HBM: kept codes are read once and written once.  Ten small CTAs an SM hide
// a unit's chain of loads (indices, exponents and codes, flags).  32 layers of 16384 slots to
// 4096, 8 heads of 128: 108 us, 5.0 TB/s; six ragged sequences that keep nearly all, 4 layers:
// 155 us, 3.6 TB/s: each unit waits for the one before and its release (20 us of it), of which few layers
// leave little else to do; 4 layers of 131072 slots to 8192: 32 us, 2.1 TB/s: a chain of the pre-pass
// and one or two units a CTA.  Measured slower: a second buffer, so that the next unit's codes come
// during a unit's waits (fewer CTAs fit); the release by another warp than the one that waits (the same).
#include "kvcompact.cuh"

#include <algorithm>

namespace cc {

namespace {

constexpr int kThreads = 128;
constexpr int kResident = 10;        // CTAs per SM
constexpr int kRows = kThreads / 8;  // slots of eight pieces of 16 bytes that the CTA moves at a time
static_assert(kThreads == kCompactChunk && kCompactWidth == 128, "a thread per slot, eight pieces of a slot");
constexpr int kPlanThreads = 256;
constexpr int kNoNumbers = 255;      // a scale exponent
constexpr int kStays = -1, kNoFall = 256;   // falls of a slot that is not written, and of one whose codes become NaN
constexpr uint32_t kNanCodes = 0x7F7F7F7Fu;
constexpr int kSharedBatch = 512;    // sequences whose first chunks fit in shared memory

// A unit's reads of its sources come before the writes of the units that wait for its flag by
// release and acquire.  A release waits for the stores of the CTA's last unit too, so that a
// unit none of whose sources can be overwritten stores its flag relaxed: there is nothing to
// order.  Released and always relaxed: 32 layers of 16384 slots to 4096 108 and 105 us (always
// released 115), six ragged sequences that keep nearly all 154 and 135.
CC_DEV void st_flag(unsigned *p, bool release) {
  if (release) asm volatile("st.release.gpu.global.u32 [%0], %1;" ::"l"(p), "r"(1u) : "memory");
  else asm volatile("st.relaxed.gpu.global.u32 [%0], %1;" ::"l"(p), "r"(1u) : "memory");
}
CC_DEV unsigned ld_flag(const unsigned *p) {
  unsigned v;
  asm volatile("ld.acquire.gpu.global.u32 %0, [%1];" : "=r"(v) : "l"(p) : "memory");
  return v;
}
CC_DEV bool wait_flag(const unsigned *flag, unsigned *status) {
  if (ld_flag(flag)) return true;
  const uint64_t t0 = globaltimer();
  for (uint32_t it = 1;; ++it) {
    if (ld_flag(flag)) return true;
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
  // (unsigned: the last steps pass 2^31)
  for (unsigned at = blockIdx.x * kPlanThreads + threadIdx.x; at < (unsigned)J; at += gridDim.x * kPlanThreads) {
    const int k = (int)at, s = idx[k], before = k > 0 ? idx[k - 1] : -1;
    if (s < k || s >= n || s <= before || n > p.cap) set_status(p.status, CC_ERR_DEVICE_ARG);
    const int c = source_of(p, idx, k) / kCompactChunk;
    for (int u = k > 0 ? source_of(p, idx, k - 1) / kCompactChunk + 1 : 0; u <= c; ++u) reader[u] = k;
    if (k == J - 1)
      for (int u = c + 1; u < p.reader_ld; ++u) reader[u] = J;
  }
}

// 16 codes times 2^-fall (fall = 1 .. 255), rounded to nearest even.  Where all of them are normal
// numbers and stay so, their exponent fields fall.  Else through fp16, which holds code * 2^-fall
// exactly down to 2^-14 and else on a grid of 2^-24, fine enough that what rounds to a code of
// 0 (up to 2^-10) stays on its side.
CC_DEV uint4 rescale(uint4 v, int fall) {
  if (fall < 14) {
    const uint32_t ones = 0x01010101u, tops = 0x80808080u, least = (uint32_t)(fall + 1) * 8 * ones, by = (uint32_t)fall * 8 * ones;
    uint32_t fine = tops, none = 0;   // bytes of at least the least magnitude, and those that are no numbers
    const uint32_t x[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t size = x[i] & ~tops;
      fine &= (size | tops) - least;
      none |= size + ones;
    }
    if ((fine & ~none & tops) == tops) return make_uint4(v.x - by, v.y - by, v.z - by, v.w - by);
  }
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

// A block's new exponent from its slots' old ones by one maximum: 255 (no number) ranks below
// 0, and a slot that is not moved (-1) below that.
CC_DEV int rank_of(int e) { return e == kNoNumbers ? 0 : e + 1; }
CC_DEV int exponent_of(int rank) { return rank == 0 ? kNoNumbers : rank - 1; }

__global__ void __launch_bounds__(kThreads, kResident) compact_kernel(const __grid_constant__ KvCompactParams p) {
  constexpr int C = kCompactChunk;
  __shared__ __align__(16) uint8_t st[C * kCompactWidth];
  __shared__ int base_sh[kSharedBatch + 1];
  __shared__ int src_sh[C];        // row of each slot's source in the array (-1: not moved)
  __shared__ int top_sh[2][8];     // for each head of the plane: ranks of the maxima over 16 slots
  // what becomes of each slot's codes: kStays, or they fall by so many steps of the exponent
  __shared__ int fall_sh[2][C];
  __shared__ int go_sh;
  const int tid = threadIdx.x, lane = tid & 31;
  const bool cached = p.batch <= kSharedBatch;
  if (cached)
    for (int i = tid; i <= p.batch; i += kThreads) base_sh[i] = p.first_chunk[i];
  if (blockIdx.x == 0)   // the new lengths; no unit reads seq_len
    for (int b = tid; b < p.batch; b += kThreads) p.seq_len[b] = kept_of(p, b);
  __syncthreads();
  const int *base = cached ? base_sh : p.first_chunk;
  const int chunks = base[p.batch];
  const int log_block = 31 - __clz(p.block), each = kCompactWidth / p.head_dim;
  // this CTA's units: chunk and plane step by step (units lie plane by plane within a chunk)
  const int chunk_step = gridDim.x / p.planes, plane_step = gridDim.x - chunk_step * p.planes;
  int chunk = blockIdx.x / p.planes, plane = blockIdx.x - chunk * p.planes;
  int b = 0, J = 0, next_s = 0;   // next_s: of this thread's slot, the coming unit's entry of keep_idx
  // The sequence of `chunk`, and its entries on their way.
  auto enter = [&]() {
    if (chunk >= chunks) return;
    bool moved = J == 0;
    while (base[b + 1] <= chunk) {
      ++b;
      moved = true;
    }
    if (moved) J = kept_of(p, b);
    const int k = (chunk - base[b]) * C + tid;
    if (k < J) next_s = p.keep_idx[(size_t)b * p.cap + k];
  };
  enter();
  while (chunk < chunks) {
    const int c = chunk - base[b], k0 = c * C, rows = min(C, J - k0);
    unsigned *flags = p.flags + ((size_t)base[b] * p.planes + plane);   // of the sequence's first chunk
    // ---- what the plane is: heads of an array of codes, columns of h, or the small arrays
    const bool codes = plane < p.n_arrays * p.array_planes, small = plane == p.planes - 1;
    const int array = codes ? plane / p.array_planes : 0;
    const int part = codes ? plane - array * p.array_planes : plane - p.n_arrays * p.array_planes;
    uint8_t *buf = codes ? p.codes[array] : p.h;
    const uint8_t *exps = codes ? p.exps[array] : nullptr;
    // a slot's row starts at (first + row) * row_bytes + column of the array
    long long first = 0;
    int row_bytes = p.h_bytes, column = part * kCompactWidth, pieces = min(kCompactWidth, p.h_bytes - column) / 16;
    int heads = 0, g = 0;
    if (codes) {
      g = p.pg.head_major ? part : part * each;
      heads = p.pg.head_major ? 1 : min(each, p.hkv - g);
      row_bytes = p.pg.head_major ? p.head_dim : p.hkv * p.head_dim;
      column = p.pg.head_major ? 0 : g * p.head_dim;
      pieces = heads * p.head_dim / 16;
      if (p.pg.head_major) first = (long long)(b * p.hkv + g) * p.cap;
    }
    // row of the chunk's first slot (a chunk lies in one page; -1: none)
    const bool paged = codes && p.pg.table && !p.pg.head_major;
    const int seq_row = codes && p.pg.head_major ? 0 : b * p.cap;
    const int to = paged ? (int)kv_row(p.pg, p.cap, b, k0) : seq_row + k0;
    // ---- the slots' rows
    int row = -1;
    bool later = false;   // the source, or its block's exponent, is a later chunk's to write
    if (tid < rows) {
      const int s = next_s < k0 + tid || next_s >= p.cap ? k0 + tid : next_s;   // (as source_of)
      later = s >= k0 + C && s < (J + C - 1) / C * C;
      row = paged ? (int)kv_row(p.pg, p.cap, b, s) : seq_row + s;
      if (row < 0 || to < 0) {
        // no such page: the destination's is not written; without the source's the slot is its own
        // source, whose codes come to its block's new scale as the others' do
        set_status(p.status, CC_ERR_DEVICE_ARG);
        row = to < 0 ? -1 : to + tid;
      }
    }
    src_sh[tid] = row;
    __syncthreads();
    // ---- 1. the sources, and meanwhile their exponents
    const int q = tid & 7, r0 = tid >> 3;   // this thread's piece of 16 bytes, and first slot
    if (small) {
      if (row >= 0) {
        uint32_t *v = reinterpret_cast<uint32_t *>(st) + tid;
        v[0] = p.tokens[row];
        v[C] = p.pos[row];
        if (p.acc) v[2 * C] = __float_as_uint(p.acc[row]);
      }
    } else if (q < pieces) {
      const uint32_t dst = smem_u32(st) + tid * 16;
      const uint8_t *src = buf + first * row_bytes + column + q * 16;
#pragma unroll
      for (int i = 0; i < C / kRows; ++i) {
        const int from = src_sh[r0 + kRows * i];
        if (from >= 0) copy16(dst + i * kRows * kCompactWidth, src + (long long)from * row_bytes);
      }
    }
    int e[2] = {-1, -1};
    if (codes) {   // the maxima over 16 slots; a block is 1, 2, 4 or 8 of them
      if (row >= 0) {
        const uint8_t *at = exps + (p.pg.head_major ? (first + row) >> log_block : (long long)(row >> log_block) * p.hkv + g);
        e[0] = at[0];
        if (heads > 1) e[1] = at[1];
      }
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        int m = row < 0 ? -1 : rank_of(e[h]);
#pragma unroll
        for (int o = 1; o < 16; o <<= 1) m = max(m, __shfl_xor_sync(0xFFFFFFFFu, m, o));
        if ((lane & 15) == 0) top_sh[h][tid >> 4] = m;
      }
    }
    // which chunks of the sequence read from this one's slots
    int r_lo = 0, r_hi = -1;
    if (tid < 32) {
      const int *reader = p.reader + (size_t)b * p.reader_ld + c;
      const int k_lo = reader[0], k_hi = reader[1] - 1;
      r_lo = max(0, k_lo / C);
      r_hi = k_hi >= k_lo ? min(c - 1, k_hi / C) : -1;
    }
    chunk += chunk_step;
    plane += plane_step;
    if (plane >= p.planes) {
      plane -= p.planes;
      ++chunk;
    }
    enter();
    copy_wait_all();
    const bool awaited = __syncthreads_or(later);
    // ---- 2. published; 3. the units that read from the destinations, and meanwhile the falls
    if (tid < 32) {
      if (tid == 0) st_flag(flags + (size_t)c * p.planes, awaited);
      bool go = true;
      for (int r = r_lo + lane; r <= r_hi; r += 32) go &= wait_flag(flags + (size_t)r * p.planes, p.status);
      go = __all_sync(0xFFFFFFFFu, go);
      if (tid == 0) go_sh = go;
    }
    const bool stays = row < 0 || row == to + tid;
    int top[2] = {-1, -1};   // ranks of the slot's blocks
    if (codes) {
      const int i0 = (tid >> 4) & ~((p.block >> 4) - 1);
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        for (int i = 0; i < p.block >> 4; ++i) top[h] = max(top[h], top_sh[h][i0 + i]);
        int fall = stays ? kStays : 0;
        if (row >= 0 && rank_of(e[h]) != top[h]) fall = e[h] == kNoNumbers ? kNoFall : e[h] == 0 ? 255 : exponent_of(top[h]) - e[h];
        fall_sh[h][tid] = fall;
      }
    } else {
      fall_sh[0][tid] = stays ? kStays : 0;
    }
    __syncthreads();
    // ---- 4. the destinations
    if (go_sh) {
      if (small) {
        if (!stays) {
          const uint32_t *v = reinterpret_cast<const uint32_t *>(st) + tid;
          p.tokens[to + tid] = v[0];
          p.pos[to + tid] = v[C];
          if (p.acc) p.acc[to + tid] = __uint_as_float(v[2 * C]);
        }
      } else if (q < pieces) {
        uint8_t *dst = buf + (first + to + r0) * row_bytes + column + q * 16;
        const int *falls = fall_sh[codes ? q * 16 / p.head_dim : 0] + r0;
        const uint4 *src = reinterpret_cast<const uint4 *>(st) + tid;
#pragma unroll
        for (int i = 0; i < C / kRows; ++i, dst += kRows * row_bytes) {
          const int fall = falls[kRows * i];
          if (fall < 0) continue;
          uint4 v = src[kThreads * i];
          if (fall > 0) v = fall == kNoFall ? make_uint4(kNanCodes, kNanCodes, kNanCodes, kNanCodes) : rescale(v, fall);
          *reinterpret_cast<uint4 *>(dst) = v;
        }
      }
      if (codes && tid < rows && (tid & (p.block - 1)) == 0 && to >= 0) {   // the blocks' exponents, by their first slots
        uint8_t *at = p.exps[array] + (p.pg.head_major ? (first + to + tid) >> log_block
                                                      : (long long)((to + tid) >> log_block) * p.hkv + g);
#pragma unroll
        for (int h = 0; h < 2; ++h)
          if (h < heads && top[h] >= 0) at[h] = (uint8_t)exponent_of(top[h]);
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
