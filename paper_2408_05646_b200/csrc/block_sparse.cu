// Which blocks of the cache a token attends (decode over a selection of blocks):
//   block_bounds_kernel  per-channel minima and maxima of the keys of every complete block of rows
//   block_scores_kernel  an upper bound on the scores of a block's rows, sum_c max(q'_c lo_c, q'_c hi_c) / sqrt(d_head),
//                        the largest over the group's query heads
//   block_select_kernel  the blocks with the highest bounds, besides the first and the newest ones
// Bounds are exact (minima and maxima of stored numbers); scores are taken in 64 bits, so that two blocks are told apart
// wherever their scores differ and a selection does not depend on the order of a sum.  Equal scores go to the lower block.
#include <cuda_bf16.h>

#include "internal.h"
#include "tc_common.cuh"

namespace ea {
namespace {

constexpr unsigned kFull = 0xffffffffu;

template <typename T> struct Vec;            // 16 bytes of a row and their minimum / maximum
template <> struct Vec<__nv_bfloat16> {
  static __device__ __forceinline__ uint32_t mn(uint32_t a, uint32_t b) {
    __nv_bfloat162 r = __hmin2(*reinterpret_cast<__nv_bfloat162*>(&a), *reinterpret_cast<__nv_bfloat162*>(&b));
    return *reinterpret_cast<uint32_t*>(&r);
  }
  static __device__ __forceinline__ uint32_t mx(uint32_t a, uint32_t b) {
    __nv_bfloat162 r = __hmax2(*reinterpret_cast<__nv_bfloat162*>(&a), *reinterpret_cast<__nv_bfloat162*>(&b));
    return *reinterpret_cast<uint32_t*>(&r);
  }
};
template <> struct Vec<float> {
  static __device__ __forceinline__ uint32_t mn(uint32_t a, uint32_t b) { return __float_as_uint(fminf(__uint_as_float(a), __uint_as_float(b))); }
  static __device__ __forceinline__ uint32_t mx(uint32_t a, uint32_t b) { return __float_as_uint(fmaxf(__uint_as_float(a), __uint_as_float(b))); }
};

// Thread = (block, 16-byte column of the key rows): consecutive threads read consecutive pieces of a row.
template <typename T>
__global__ void __launch_bounds__(256) block_bounds_kernel(const SparseParams p) {
  const int unit = blockIdx.x, h = unit / p.B, b = unit - h * p.B;
  const HeadInfo hd = p.heads[h];
  const int nc = hd.rp_k * static_cast<int>(sizeof(T)) / 16;
  const int idx = blockIdx.y * 256 + threadIdx.x;
  const int blk = p.block0 + idx / nc, c = idx % nc;
  const int n_b = p.deficit != nullptr ? p.n - __ldg(p.deficit + b) : p.n;
  const int G = 1 << p.block_shift;
  if (blk >= p.block1 || blk >= (n_b >> p.block_shift)) return;     // complete blocks only
  const int64_t row0 = physical_row(p.pages, b, p.n_max, blk << p.block_shift);
  const uint4* src = reinterpret_cast<const uint4*>(p.cache + hd.k_off) + row0 * nc + c;
  uint4 lo, hi;
  constexpr int kAhead = 16;                 // loads of a thread under way together (the shortest block)
  for (int r0 = 0; r0 < G; r0 += kAhead) {
    uint4 x[kAhead];
#pragma unroll
    for (int r = 0; r < kAhead; ++r) x[r] = __ldg(src + static_cast<int64_t>(r0 + r) * nc);
    if (r0 == 0) lo = hi = x[0];
#pragma unroll
    for (int r = 0; r < kAhead; ++r) {
      lo.x = Vec<T>::mn(lo.x, x[r].x); lo.y = Vec<T>::mn(lo.y, x[r].y); lo.z = Vec<T>::mn(lo.z, x[r].z); lo.w = Vec<T>::mn(lo.w, x[r].w);
      hi.x = Vec<T>::mx(hi.x, x[r].x); hi.y = Vec<T>::mx(hi.y, x[r].y); hi.z = Vec<T>::mx(hi.z, x[r].z); hi.w = Vec<T>::mx(hi.w, x[r].w);
    }
  }
  uint4* dst = reinterpret_cast<uint4*>(p.bounds + p.slab[h]) + physical_block(p, b, blk) * 2 * nc + c;
  dst[0] = lo;
  dst[nc] = hi;
}

// The two 16-bit numbers of a word as doubles, times 2^-896: exponent and mantissa bits moved into place (zeros and
// subnormal numbers come out right too).  The factor is taken out of the query.
__device__ __forceinline__ double tiny_high(uint32_t w) { return __hiloint2double((static_cast<int>(w) >> 3) & 0x8fffe000, 0); }
__device__ __forceinline__ double tiny_low(uint32_t w) { return __hiloint2double((static_cast<int>(w << 16) >> 3) & 0x8fffffff, 0); }

// 16 bytes of lo and hi (eight 16-bit channels, or four of 32 bits) against the same channels of a query: a channel
// contributes q hi where q > 0 and q lo where q < 0.  `neg` has ones in the place of the channels whose q is negative.
// Even and odd channels have sums of their own.
__device__ __forceinline__ uint32_t pick(uint32_t neg, uint32_t lo, uint32_t hi) { return (lo & neg) | (hi & ~neg); }
__device__ __forceinline__ void add_bounds(const uint4& lo, const uint4& hi, const uint4& neg, const double* q, double (&acc)[2], __nv_bfloat16) {
  const uint32_t w[4] = {pick(neg.x, lo.x, hi.x), pick(neg.y, lo.y, hi.y), pick(neg.z, lo.z, hi.z), pick(neg.w, lo.w, hi.w)};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const double2 x = *reinterpret_cast<const double2*>(q + 2 * i);
    acc[0] = fma(x.x, tiny_low(w[i]), acc[0]);
    acc[1] = fma(x.y, tiny_high(w[i]), acc[1]);
  }
}
__device__ __forceinline__ void add_bounds(const uint4& lo, const uint4& hi, const uint4& neg, const double* q, double (&acc)[2], float) {
  const uint32_t w[4] = {pick(neg.x, lo.x, hi.x), pick(neg.y, lo.y, hi.y), pick(neg.z, lo.z, hi.z), pick(neg.w, lo.w, hi.w)};
#pragma unroll
  for (int i = 0; i < 4; i += 2) {
    const double2 x = *reinterpret_cast<const double2*>(q + i);
    acc[0] = fma(x.x, static_cast<double>(__uint_as_float(w[i])), acc[0]);
    acc[1] = fma(x.y, static_cast<double>(__uint_as_float(w[i + 1])), acc[1]);
  }
}
template <typename T> __device__ __forceinline__ double query_factor();
template <> __device__ __forceinline__ double query_factor<__nv_bfloat16>() { return __hiloint2double((1023 + 896) << 20, 0); }   // 2^896
template <> __device__ __forceinline__ double query_factor<float>() { return 1.0; }

// A CTA takes a run of blocks of a unit, 64 at a time: the bounds of the next 64 come in by coalesced 16-byte copies while
// two threads score a block, half of its channels each (in shared memory a block's bounds sit at an odd multiple of 16 bytes,
// so that the threads' reads meet all banks).
constexpr int kScoreBlocks = 64, kScoreThreads = 2 * kScoreBlocks;
template <typename T>
__global__ void __launch_bounds__(kScoreThreads) block_scores_kernel(const SparseParams p, int max_steps) {
  chain_go();
  extern __shared__ __align__(16) unsigned char sm[];
  const int unit = blockIdx.x, h = unit / p.B, b = unit - h * p.B, tid = threadIdx.x;
  const int n_b = p.deficit != nullptr ? p.n - __ldg(p.deficit + b) : p.n;
  const int have = (n_b + (1 << p.block_shift) - 1) >> p.block_shift;
  const int first = p.sink + blockIdx.y * kScoreBlocks * max_steps, last = min(have - p.recent, first + kScoreBlocks * max_steps);
  if (have <= p.list_len || first >= last) {                 // nothing to choose
    chain_wait();
    return;
  }
  const HeadInfo& hd = p.heads[h];
  const int rp_k = hd.rp_k;
  constexpr int kPer = 16 / sizeof(T);       // channels of a 16-byte piece
  const int nc = rp_k / kPer, per = 2 * nc, pitch = (per + 1) * 16;
  double* qs = reinterpret_cast<double*>(sm);                // [group][rp_k]
  T* neg = reinterpret_cast<T*>(qs + p.group * rp_k);        // [group][rp_k]: all ones where q is negative
  unsigned char* ring = reinterpret_cast<unsigned char*>(neg + p.group * rp_k);    // [2][64][pitch]
  const char* slab = p.bounds + p.slab[h];
  const int steps = (last - first + kScoreBlocks - 1) / kScoreBlocks;
  // piece c of block j, stepped through in place of a division per piece
  const int j_first = tid / per, c_first = tid % per, j_step = kScoreThreads / per, c_step = kScoreThreads % per;
  const bool paged = p.pages.table != nullptr;
  auto load = [&](int step) {
    const int blk0 = first + step * kScoreBlocks, count = min(kScoreBlocks, last - blk0);
    unsigned char* dst = ring + (step & 1) * kScoreBlocks * pitch + j_first * pitch + c_first * 16;
    const char* src = slab + (static_cast<int64_t>(b) * p.seq_blocks + blk0) * per * 16 + tid * 16;
    int j = j_first, c = c_first;
    while (j < count) {
      tc::cp_async16(dst, paged ? slab + (physical_block(p, b, blk0 + j) * per + c) * 16 : src, 16);
      src += kScoreThreads * 16;
      dst += j_step * pitch + c_step * 16;
      j += j_step;
      c += c_step;
      if (c >= per) { c -= per; ++j; dst += pitch - per * 16; }
    }
    tc::cp_async_commit();
  };
  load(0);                                   // (the bounds are older than the chain, the queries are not)
  chain_wait();
  for (int i = tid; i < p.group * rp_k; i += kScoreThreads) {
    const int g = i / rp_k, c = i - g * rp_k;
    const double x = p.q64[(static_cast<int64_t>(unit) * p.group + g) * p.q_stride + c];
    qs[i] = x * query_factor<T>();
    if constexpr (sizeof(T) == 2) reinterpret_cast<uint16_t*>(neg)[i] = x < 0 ? 0xffffu : 0u;
    else reinterpret_cast<uint32_t*>(neg)[i] = x < 0 ? 0xffffffffu : 0u;
  }
  const int mine = tid >> 1, half = tid & 1;
  const int c_lo = half ? nc / 2 : 0, c_hi = half ? nc : nc / 2;
  for (int step = 0; step < steps; ++step) {
    if (step + 1 < steps) {
      load(step + 1);
      tc::cp_async_wait<1>();
    } else {
      tc::cp_async_wait<0>();
    }
    __syncthreads();
    const int blk = first + step * kScoreBlocks + mine;
    const uint4* lo = reinterpret_cast<const uint4*>(ring + ((step & 1) * kScoreBlocks + mine) * pitch);
    double best = 0;
    for (int g = 0; g < p.group; ++g) {
      double acc[2] = {0, 0};                // even and odd channels
      if (blk < last) {
        const double* q = qs + g * rp_k;
        const uint4* n4 = reinterpret_cast<const uint4*>(neg + g * rp_k);
#pragma unroll 5
        for (int c = c_lo; c < c_hi; ++c) add_bounds(lo[c], lo[nc + c], n4[c], q + c * kPer, acc, T());
      }
      const double part = acc[0] + acc[1];
      const double other = __shfl_xor_sync(kFull, part, 1);
      const double s = half ? other + part : part + other;                   // the same for both threads
      if (g == 0 || s > best) best = s;
    }
    // the position bias of the block's last row, the one it takes least from
    if (hd.alibi_slope != 0.f)
      best -= static_cast<double>(hd.alibi_slope) * (n_b - 1 - (((blk + 1) << p.block_shift) - 1));
    if (!half && blk < last) p.scores[static_cast<int64_t>(unit) * p.score_stride + blk] = best;
    __syncthreads();
  }
}

// Doubles as integers in the same order (a zero of either sign is one number).
__device__ __forceinline__ uint64_t order_key(double x) {
  const uint64_t b = static_cast<uint64_t>(__double_as_longlong(x + 0.0));
  return b >> 63 ? ~b : b | (1ull << 63);
}

// One CTA per unit: the k-th highest key by counting digits of 11 bits, then one ordered pass that writes the chosen
// blocks in ascending order (sorted lists read the cache front to back, and equal scores go to the lower block).  Keys are
// taken relative to the lowest one and digits start at the highest bit of the range: scores share their leading bits, and
// counting those would send every key to one counter.
constexpr int kSelThreads = 256, kDigit = 11, kBins = 1 << kDigit, kKeep = 4, kSegment = kSelThreads * kKeep;
__global__ void __launch_bounds__(kSelThreads) block_select_kernel(const SparseParams p) {
  chain_go();
  chain_wait();
  __shared__ int hist[kBins];
  __shared__ int warp_sum[kSelThreads / 32];
  __shared__ int s_digit, s_above, s_count;
  __shared__ uint64_t s_low[kSelThreads / 32], s_high[kSelThreads / 32];
  const int unit = blockIdx.x, h = unit / p.B, b = unit - h * p.B;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int n_b = p.deficit != nullptr ? p.n - __ldg(p.deficit + b) : p.n;
  const int have = (n_b + (1 << p.block_shift) - 1) >> p.block_shift;
  const int M = p.list_len;
  int32_t* list = p.list + static_cast<int64_t>(unit) * M;
  int32_t* index = p.index ? p.index + (static_cast<int64_t>(b) * p.H + h) * p.index_len : nullptr;
  auto put = [&](int at, int blk) {
    list[at] = blk;
    if (index) index[at] = blk;
  };
  if (have <= M) {                           // all of them
    for (int i = tid; i < M; i += kSelThreads) put(i, i < have ? i : -1);
    for (int i = M + tid; index && i < p.index_len; i += kSelThreads) index[i] = -1;
    return;
  }
  const int first = p.sink, last = have - p.recent, want = M - p.sink - p.recent;
  for (int i = tid; i < p.sink; i += kSelThreads) put(i, i);
  for (int i = tid; i < p.recent; i += kSelThreads) put(M - p.recent + i, last + i);
  if (want == 0) return;
  const double* scores = p.scores + static_cast<int64_t>(unit) * p.score_stride;

  // Segments of 1024 keys, four neighbours per thread; those of the first segment stay in registers, later ones (long
  // sequences of short blocks) are read again.
  const int count = last - first, segments = (count + kSegment - 1) / kSegment;
  uint64_t keep[kKeep];
  auto read = [&](int segment, uint64_t (&k)[kKeep]) {
#pragma unroll
    for (int j = 0; j < kKeep; ++j) {
      const int i = segment * kSegment + tid * kKeep + j;
      k[j] = i < count ? order_key(scores[first + i]) : 0;
    }
  };
  // f(key) for every key of this thread
  auto each = [&](auto f) {
#pragma unroll
    for (int j = 0; j < kKeep; ++j)
      if (tid * kKeep + j < count) f(keep[j]);
    for (int s = 1; s < segments; ++s) {
      uint64_t k[kKeep];
      read(s, k);
#pragma unroll
      for (int j = 0; j < kKeep; ++j)
        if (s * kSegment + tid * kKeep + j < count) f(k[j]);
    }
  };
  read(0, keep);
  uint64_t lowest = ~0ull, highest = 0;
  each([&](uint64_t k) {
    lowest = k < lowest ? k : lowest;
    highest = k > highest ? k : highest;
  });
#pragma unroll
  for (int d = 16; d; d >>= 1) {
    const uint64_t a = __shfl_xor_sync(kFull, lowest, d), c = __shfl_xor_sync(kFull, highest, d);
    lowest = a < lowest ? a : lowest;
    highest = c > highest ? c : highest;
  }
  if (lane == 0) { s_low[warp] = lowest; s_high[warp] = highest; }
  for (int i = tid; i < kBins; i += kSelThreads) hist[i] = 0;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < kSelThreads / 32; ++w) {
    lowest = s_low[w] < lowest ? s_low[w] : lowest;
    highest = s_high[w] > highest ? s_high[w] : highest;
  }
  uint64_t prefix = 0;       // the digits found so far; keys above it (compared on their top bits) are chosen
  int shift = 64 - __clzll(static_cast<long long>((highest - lowest) | 1)), need = want;   // no key has a bit from here on
  bool again = false;
  while (shift > 0) {
    const int bits = shift >= kDigit ? kDigit : shift;
    const int next = shift - bits;
    if (again) {
      for (int i = tid; i < kBins; i += kSelThreads) hist[i] = 0;
      __syncthreads();
    }
    again = true;
    each([&](uint64_t absolute) {
      const uint64_t k = absolute - lowest;
      if (shift >= 64 || (k >> shift) == prefix) atomicAdd(&hist[(k >> next) & ((1 << bits) - 1)], 1);
    });
    __syncthreads();
    // counts from the highest digit down: thread i holds the bins 2047 - 8i .. 2040 - 8i
    int mine[8], sum = 0;
#pragma unroll
    for (int j = 0; j < 8; ++j) { mine[j] = hist[kBins - 1 - 8 * tid - j]; sum += mine[j]; }
    int scan = sum;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
      const int y = __shfl_up_sync(kFull, scan, d);
      if (lane >= d) scan += y;
    }
    if (lane == 31) warp_sum[warp] = scan;
    __syncthreads();
    int above = scan - sum;
    for (int w = 0; w < warp; ++w) above += warp_sum[w];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      if (above < need && above + mine[j] >= need) {          // one thread, one bin
        s_digit = kBins - 1 - 8 * tid - j;
        s_above = above;
        s_count = mine[j];
      }
      above += mine[j];
    }
    __syncthreads();
    prefix = prefix << bits | static_cast<uint64_t>(s_digit);
    need -= s_above;
    shift = next;
    if (s_count == need) break;              // every key of this digit is chosen
    __syncthreads();
  }
  // keys with (key >> shift) above the prefix are in; of those equal to it the first `need`
  int done = 0, ties = 0;
  for (int seg = 0; seg < segments; ++seg) {
    uint64_t k[kKeep];
    if (seg == 0) {
#pragma unroll
      for (int j = 0; j < kKeep; ++j) k[j] = keep[j];
    } else {
      read(seg, k);
    }
    int eq = 0, gt = 0;                      // of this thread
    bool is_eq[kKeep], is_gt[kKeep];
#pragma unroll
    for (int j = 0; j < kKeep; ++j) {
      const bool there = seg * kSegment + tid * kKeep + j < count;
      const uint64_t d = (k[j] - lowest) >> shift;
      is_eq[j] = there && d == prefix;
      is_gt[j] = there && d > prefix;
      eq += is_eq[j];
      gt += is_gt[j];
    }
    int scan = eq << 16 | gt;                // both counts of a segment fit 16 bits
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
      const int y = __shfl_up_sync(kFull, scan, d);
      if (lane >= d) scan += y;
    }
    __syncthreads();
    if (lane == 31) warp_sum[warp] = scan;
    __syncthreads();
    int before = scan - (eq << 16 | gt), total = 0;
#pragma unroll
    for (int w = 0; w < kSelThreads / 32; ++w) {
      if (w < warp) before += warp_sum[w];
      total += warp_sum[w];
    }
    int e = ties + (before >> 16);           // ties before the thread's first key, in the whole range
    int at = p.sink + done + (before & 0xffff) + min(e, need) - min(ties, need);
#pragma unroll
    for (int j = 0; j < kKeep; ++j) {
      if (is_gt[j] || (is_eq[j] && e < need)) put(at++, first + seg * kSegment + tid * kKeep + j);
      e += is_eq[j];
    }
    done += (total & 0xffff) + min(ties + (total >> 16), need) - min(ties, need);
    ties += total >> 16;
  }
}

}  // namespace

cudaError_t launch_block_bounds(const SparseParams& p, int dtype, cudaStream_t s, uint64_t* launches) {
  // the widest key row a head can have: 128 channels
  const int64_t pieces = static_cast<int64_t>(p.block1 - p.block0) * 128 * (dtype == 0 ? 2 : 4) / 16;
  const dim3 grid(p.B * p.H, static_cast<unsigned>((pieces + 255) / 256));
  if (dtype == 0) block_bounds_kernel<__nv_bfloat16><<<grid, 256, 0, s>>>(p);
  else block_bounds_kernel<float><<<grid, 256, 0, s>>>(p);
  ++*launches;
  return cudaGetLastError();
}

template <typename T>
static cudaError_t launch_scores_t(const SparseParams& p, int max_rp_k, cudaStream_t s) {
  const size_t smem = (sizeof(double) + sizeof(T)) * p.group * max_rp_k +
                      2 * static_cast<size_t>(kScoreBlocks) * (2 * max_rp_k * sizeof(T) + 16);
  static size_t configured[kMaxDevices] = {};
  const cudaError_t e = ensure_dynamic_smem(block_scores_kernel<T>, smem, configured);
  if (e != cudaSuccess) return e;
  // runs of up to three steps, as long as there are CTAs for five on every SM (16 x 1024 blocks of 32 heads: 42 us with one
  // step, 35 with three, 39 with sixteen)
  const int64_t chunks = (p.max_blocks - p.sink - p.recent + kScoreBlocks - 1) / kScoreBlocks, units = static_cast<int64_t>(p.B) * p.H;
  int64_t steps = units * chunks / (5 * 148);
  steps = steps < 1 ? 1 : steps > 3 ? 3 : steps;
  if (chunks > 65535 * steps) steps = (chunks + 65534) / 65535;              // (the second grid dimension)
  return launch_chained(true, block_scores_kernel<T>, dim3(static_cast<unsigned>(units), static_cast<unsigned>((chunks + steps - 1) / steps)),
                        kScoreThreads, smem, s, p, static_cast<int>(steps));
}

cudaError_t launch_block_scores(const SparseParams& p, int dtype, int max_rp_k, cudaStream_t s, uint64_t* launches) {
  ++*launches;
  return dtype == 0 ? launch_scores_t<__nv_bfloat16>(p, max_rp_k, s) : launch_scores_t<float>(p, max_rp_k, s);
}

cudaError_t launch_block_select(const SparseParams& p, cudaStream_t s, uint64_t* launches) {
  ++*launches;
  return launch_chained(true, block_select_kernel, p.B * p.H, kSelThreads, 0, s, p);
}

}  // namespace ea
