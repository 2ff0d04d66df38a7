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
  uint4 lo = __ldg(src), hi = lo;
#pragma unroll 8
  for (int r = 1; r < G; ++r) {
    const uint4 x = __ldg(src + static_cast<int64_t>(r) * nc);
    lo.x = Vec<T>::mn(lo.x, x.x); lo.y = Vec<T>::mn(lo.y, x.y); lo.z = Vec<T>::mn(lo.z, x.z); lo.w = Vec<T>::mn(lo.w, x.w);
    hi.x = Vec<T>::mx(hi.x, x.x); hi.y = Vec<T>::mx(hi.y, x.y); hi.z = Vec<T>::mx(hi.z, x.z); hi.w = Vec<T>::mx(hi.w, x.w);
  }
  uint4* dst = reinterpret_cast<uint4*>(p.bounds + p.slab[h]) + physical_block(p, b, blk) * 2 * nc + c;
  dst[0] = lo;
  dst[nc] = hi;
}

// The two 16-bit numbers of a word as doubles, times 2^-896: exponent and mantissa bits moved into place (zeros and
// subnormal numbers come out right too).  The factor is taken out of the query.
__device__ __forceinline__ double tiny_high(uint32_t w) { return __hiloint2double((static_cast<int>(w) >> 3) & 0x8fffe000, 0); }
__device__ __forceinline__ double tiny_low(uint32_t w) { return __hiloint2double((static_cast<int>(w << 16) >> 3) & 0x8fffffff, 0); }

// 16 bytes of lo and hi (eight 16-bit channels, or four of 32 bits) against the same channels of GQ queries: a channel
// contributes q hi where q > 0 and q lo where q < 0.  Even and odd channels have sums of their own.
__device__ __forceinline__ bool negative(double x) { return __double2hiint(x) < 0; }
template <int GQ>
__device__ __forceinline__ void add_bounds(const uint4& lo, const uint4& hi, const double* q, int q_stride, double (&acc)[2 * GQ], __nv_bfloat16) {
  const uint32_t l[4] = {lo.x, lo.y, lo.z, lo.w}, u[4] = {hi.x, hi.y, hi.z, hi.w};
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int g = 0; g < GQ; ++g) {
      const double2 x = *reinterpret_cast<const double2*>(q + g * q_stride + 2 * i);
      acc[2 * g] = fma(x.x, tiny_low(negative(x.x) ? l[i] : u[i]), acc[2 * g]);
      acc[2 * g + 1] = fma(x.y, tiny_high(negative(x.y) ? l[i] : u[i]), acc[2 * g + 1]);
    }
}
template <int GQ>
__device__ __forceinline__ void add_bounds(const uint4& lo, const uint4& hi, const double* q, int q_stride, double (&acc)[2 * GQ], float) {
  const uint32_t l[4] = {lo.x, lo.y, lo.z, lo.w}, u[4] = {hi.x, hi.y, hi.z, hi.w};
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int g = 0; g < GQ; ++g) {
      const double x = q[g * q_stride + i];
      acc[2 * g + (i & 1)] = fma(x, static_cast<double>(__uint_as_float(negative(x) ? l[i] : u[i])), acc[2 * g + (i & 1)]);
    }
}
template <typename T> __device__ __forceinline__ double query_factor();
template <> __device__ __forceinline__ double query_factor<__nv_bfloat16>() { return __hiloint2double((1023 + 896) << 20, 0); }   // 2^896
template <> __device__ __forceinline__ double query_factor<float>() { return 1.0; }

// A CTA takes 128 blocks of a unit: their bounds come in by coalesced 16-byte copies (in shared memory a block's bounds sit
// at an odd multiple of 16 bytes, so that 128 threads read one each without bank conflicts), then one thread scores one
// block for the group's queries, GQ at a time.
constexpr int kScoreBlocks = 128;
template <typename T, int GQ>
__global__ void __launch_bounds__(kScoreBlocks) block_scores_kernel(const SparseParams p) {
  extern __shared__ __align__(16) unsigned char sm[];
  __shared__ int64_t phys[kScoreBlocks];
  const int unit = blockIdx.x, h = unit / p.B, b = unit - h * p.B, tid = threadIdx.x;
  const int n_b = p.deficit != nullptr ? p.n - __ldg(p.deficit + b) : p.n;
  const int have = (n_b + (1 << p.block_shift) - 1) >> p.block_shift;
  const int first = p.sink + blockIdx.y * kScoreBlocks, last = have - p.recent;
  if (have <= p.list_len || first >= last) return;           // nothing to choose
  const HeadInfo hd = p.heads[h];
  constexpr int kPer = 16 / sizeof(T);       // channels of a 16-byte piece
  const int nc = hd.rp_k / kPer, pitch = (2 * nc + 1) * 16;
  const int groups = (p.group + GQ - 1) / GQ * GQ;
  double* qs = reinterpret_cast<double*>(sm);                // [groups][rp_k]
  unsigned char* bounds = sm + sizeof(double) * groups * hd.rp_k;
  const int blk = first + tid;
  phys[tid] = blk < last ? physical_block(p, b, blk) : -1;
  __syncthreads();
  const char* slab = p.bounds + p.slab[h];
  const int per = 2 * nc;
  for (int i = tid; i < kScoreBlocks * per; i += kScoreBlocks) {
    const int j = i / per, c = i - j * per;
    const int64_t at = phys[j];
    if (at >= 0) tc::cp_async16(bounds + j * pitch + c * 16, slab + (at * per + c) * 16, 16);
  }
  tc::cp_async_commit();
  for (int i = tid; i < groups * hd.rp_k; i += kScoreBlocks) {
    const int g = i / hd.rp_k, c = i - g * hd.rp_k;
    qs[i] = g < p.group ? p.q64[(static_cast<int64_t>(unit) * p.group + g) * p.q_stride + c] * query_factor<T>() : 0.0;
  }
  tc::cp_async_wait<0>();
  __syncthreads();
  if (blk >= last) return;
  const uint4* lo = reinterpret_cast<const uint4*>(bounds + tid * pitch);
  double best = 0;
  for (int g0 = 0; g0 < p.group; g0 += GQ) {
    double acc[2 * GQ];                      // even and odd channels
#pragma unroll
    for (int g = 0; g < 2 * GQ; ++g) acc[g] = 0;
#pragma unroll 2
    for (int c = 0; c < nc; ++c) add_bounds<GQ>(lo[c], lo[nc + c], qs + g0 * hd.rp_k + c * kPer, hd.rp_k, acc, T());
#pragma unroll
    for (int g = 0; g < GQ; ++g) {
      const double s = acc[2 * g] + acc[2 * g + 1];
      if (g0 + g < p.group && (g0 + g == 0 || s > best)) best = s;
    }
  }
  // the position bias of the block's last row, the one it takes least from
  if (hd.alibi_slope != 0.f)
    best -= static_cast<double>(hd.alibi_slope) * (n_b - 1 - (((blk + 1) << p.block_shift) - 1));
  p.scores[static_cast<int64_t>(unit) * p.score_stride + blk] = best;
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
constexpr int kSelThreads = 256, kDigit = 11, kBins = 1 << kDigit, kKeep = 4;
__global__ void __launch_bounds__(kSelThreads) block_select_kernel(const SparseParams p) {
  __shared__ int hist[kBins];
  __shared__ int warp_sum[8], warp_sum2[8];
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

  // the first kKeep keys of a thread stay in its registers, the rest (long sequences of short blocks) are read again
  uint64_t keep[kKeep];
#pragma unroll
  for (int j = 0; j < kKeep; ++j) {
    const int i = first + j * kSelThreads + tid;
    keep[j] = i < last ? order_key(scores[i]) : 0;
  }
  auto key = [&](int j) { return order_key(scores[first + j * kSelThreads + tid]); };
  const int mine_n = (last - first - tid + kSelThreads - 1) / kSelThreads;        // keys of this thread
  uint64_t lowest = ~0ull, highest = 0;
  auto extend = [&](uint64_t k) {
    lowest = k < lowest ? k : lowest;
    highest = k > highest ? k : highest;
  };
#pragma unroll
  for (int j = 0; j < kKeep; ++j)
    if (j < mine_n) extend(keep[j]);
  for (int j = kKeep; j < mine_n; ++j) extend(key(j));
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
    auto count = [&](uint64_t absolute) {
      const uint64_t k = absolute - lowest;
      if (shift >= 64 || (k >> shift) == prefix) atomicAdd(&hist[(k >> next) & ((1 << bits) - 1)], 1);
    };
#pragma unroll
    for (int j = 0; j < kKeep; ++j)
      if (j < mine_n) count(keep[j]);
    for (int j = kKeep; j < mine_n; ++j) count(key(j));
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
  auto emit = [&](int i, uint64_t absolute) {
    const uint64_t k = (absolute - lowest) >> shift;
    const bool eq = i < last && k == prefix, gt = i < last && k > prefix;
    const unsigned beq = __ballot_sync(kFull, eq), bgt = __ballot_sync(kFull, gt);
    if (lane == 0) { warp_sum[warp] = __popc(beq); warp_sum2[warp] = __popc(bgt); }
    __syncthreads();
    int e0 = ties, g0 = 0, e_all = 0, g_all = 0;
#pragma unroll
    for (int w = 0; w < 8; ++w) {
      if (w < warp) { e0 += warp_sum[w]; g0 += warp_sum2[w]; }
      e_all += warp_sum[w];
      g_all += warp_sum2[w];
    }
    const unsigned below = (1u << lane) - 1;
    const int my_e = e0 + __popc(beq & below);               // ties before this block, in the whole range
    const int taken_e = min(my_e, need) - min(ties, need);   // of them chosen, within this round
    if (gt || (eq && my_e < need)) put(p.sink + done + g0 + __popc(bgt & below) + taken_e, i);
    done += g_all + min(ties + e_all, need) - min(ties, need);
    ties += e_all;
    __syncthreads();
  };
  __syncthreads();
  const int rounds = (last - first + kSelThreads - 1) / kSelThreads;
#pragma unroll
  for (int j = 0; j < kKeep; ++j)
    if (j < rounds) emit(first + j * kSelThreads + tid, keep[j]);
  for (int j = kKeep; j < rounds; ++j) emit(first + j * kSelThreads + tid, j < mine_n ? key(j) : 0);
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

template <typename T, int GQ>
static cudaError_t launch_scores_t(const SparseParams& p, int max_rp_k, cudaStream_t s) {
  const int groups = (p.group + GQ - 1) / GQ * GQ;
  const size_t smem = sizeof(double) * groups * max_rp_k + static_cast<size_t>(kScoreBlocks) * (2 * max_rp_k * sizeof(T) + 16);
  static size_t configured[kMaxDevices] = {};
  const cudaError_t e = ensure_dynamic_smem(block_scores_kernel<T, GQ>, smem, configured);
  if (e != cudaSuccess) return e;
  const int middle = p.max_blocks - p.sink - p.recent;
  block_scores_kernel<T, GQ><<<dim3(p.B * p.H, (middle + kScoreBlocks - 1) / kScoreBlocks), kScoreBlocks, smem, s>>>(p);
  return cudaGetLastError();
}

cudaError_t launch_block_scores(const SparseParams& p, int dtype, int max_rp_k, cudaStream_t s, uint64_t* launches) {
  ++*launches;
  if (p.group == 1) return dtype == 0 ? launch_scores_t<__nv_bfloat16, 1>(p, max_rp_k, s) : launch_scores_t<float, 1>(p, max_rp_k, s);
  return dtype == 0 ? launch_scores_t<__nv_bfloat16, 4>(p, max_rp_k, s) : launch_scores_t<float, 4>(p, max_rp_k, s);
}

cudaError_t launch_block_select(const SparseParams& p, cudaStream_t s, uint64_t* launches) {
  block_select_kernel<<<p.B * p.H, kSelThreads, 0, s>>>(p);
  ++*launches;
  return cudaGetLastError();
}

}  // namespace ea
