// Which blocks of the cache a token attends (decode over a selection of blocks):
//   block_bounds_kernel  per-channel minima and maxima of the keys of every complete block of rows
//   block_scores_kernel  an upper bound on the scores of a block's rows, sum_c max(q'_c lo_c, q'_c hi_c) / sqrt(d_head),
//                        the largest over the group's query heads
//   block_select_kernel  the blocks with the highest bounds, besides the first and the newest ones
// Bounds are exact (minima and maxima of stored numbers); scores are taken in 64 bits, so that two blocks are told apart
// wherever their scores differ and a selection does not depend on the order of a sum.  Equal scores go to the lower block.
#include <cuda_bf16.h>

#include "internal.h"

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

// A 16-bit number as a double, times 2^-896: its exponent and mantissa bits moved into place (zero and subnormal numbers
// come out right too).  The factor is taken out of the query.
__device__ __forceinline__ double tiny_double(uint32_t bits16) {
  return __hiloint2double(static_cast<int>(((bits16 & 0x8000u) << 16) | ((bits16 & 0x7fffu) << 13)), 0);
}

// Eight 16-bit channels (or four of 32 bits) of lo and hi against the same channels of the query.
__device__ __forceinline__ void add_bounds(const uint4& lo, const uint4& hi, const double* q, double (&acc)[2], __nv_bfloat16) {
  const uint32_t l[4] = {lo.x, lo.y, lo.z, lo.w}, u[4] = {hi.x, hi.y, hi.z, hi.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const double q0 = q[2 * i], q1 = q[2 * i + 1];
    acc[0] = fma(q0, tiny_double((q0 < 0 ? l[i] : u[i]) & 0xffffu), acc[0]);
    acc[1] = fma(q1, tiny_double((q1 < 0 ? l[i] : u[i]) >> 16), acc[1]);
  }
}
__device__ __forceinline__ void add_bounds(const uint4& lo, const uint4& hi, const double* q, double (&acc)[2], float) {
  const uint32_t l[4] = {lo.x, lo.y, lo.z, lo.w}, u[4] = {hi.x, hi.y, hi.z, hi.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) acc[i & 1] = fma(q[i], static_cast<double>(__uint_as_float(q[i] < 0 ? l[i] : u[i])), acc[i & 1]);
}
template <typename T> __device__ __forceinline__ double query_factor();
template <> __device__ __forceinline__ double query_factor<__nv_bfloat16>() { return __hiloint2double((1023 + 896) << 20, 0); }   // 2^896
template <> __device__ __forceinline__ double query_factor<float>() { return 1.0; }

// One thread per block; the queries of the group sit in shared memory.
template <typename T>
__global__ void __launch_bounds__(128) block_scores_kernel(const SparseParams p) {
  extern __shared__ double qs[];             // [group][rp_k]
  const int unit = blockIdx.x, h = unit / p.B, b = unit - h * p.B;
  const int n_b = p.deficit != nullptr ? p.n - __ldg(p.deficit + b) : p.n;
  const int have = (n_b + (1 << p.block_shift) - 1) >> p.block_shift;
  const int first = p.sink + blockIdx.y * 128, last = have - p.recent;
  if (have <= p.list_len || first >= last) return;           // nothing to choose
  const HeadInfo hd = p.heads[h];
  for (int i = threadIdx.x; i < p.group * hd.rp_k; i += 128) {
    const int g = i / hd.rp_k, c = i - g * hd.rp_k;
    qs[i] = p.q64[(static_cast<int64_t>(unit) * p.group + g) * p.q_stride + c] * query_factor<T>();
  }
  __syncthreads();
  const int blk = first + threadIdx.x;
  if (blk >= last) return;
  constexpr int kPer = 16 / sizeof(T);       // channels of a 16-byte piece
  const int nc = hd.rp_k / kPer;
  const uint4* lo = reinterpret_cast<const uint4*>(p.bounds + p.slab[h]) + physical_block(p, b, blk) * 2 * nc;
  double best = 0;
  for (int g = 0; g < p.group; ++g) {
    double acc[2] = {0, 0};
    for (int c = 0; c < nc; ++c) add_bounds(__ldg(lo + c), __ldg(lo + nc + c), qs + g * hd.rp_k + c * kPer, acc, T());
    const double s = acc[0] + acc[1];
    best = g == 0 || s > best ? s : best;
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

// One CTA per unit: the k-th highest key by counting digits of 11 bits from the top, then one ordered pass that writes
// the chosen blocks in ascending order (sorted lists read the cache front to back, and equal scores go to the lower block).
constexpr int kSelThreads = 256, kDigit = 11, kBins = 1 << kDigit;
__global__ void __launch_bounds__(kSelThreads) block_select_kernel(const SparseParams p) {
  __shared__ int hist[kBins];
  __shared__ int warp_sum[8], warp_sum2[8];
  __shared__ int s_digit, s_above, s_count;
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

  uint64_t prefix = 0;       // the digits found so far; keys above it (compared on their top bits) are chosen
  int shift = 64, need = want;
  while (shift > 0) {
    const int bits = shift >= kDigit ? kDigit : shift;
    const int next = shift - bits;
    for (int i = tid; i < kBins; i += kSelThreads) hist[i] = 0;
    __syncthreads();
    for (int i = first + tid; i < last; i += kSelThreads) {
      const uint64_t k = order_key(scores[i]);
      if (shift == 64 || (k >> shift) == prefix) atomicAdd(&hist[(k >> next) & ((1 << bits) - 1)], 1);
    }
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
    prefix = (shift == 64 ? 0 : prefix << bits) | static_cast<uint64_t>(s_digit);
    need -= s_above;
    shift = next;
    if (s_count == need) break;              // every key of this digit is chosen
    __syncthreads();
  }
  // keys with (key >> shift) above the prefix are in; of those equal to it the first `need`
  int done = 0, ties = 0;
  for (int i0 = first; i0 < last; i0 += kSelThreads) {
    __syncthreads();
    const int i = i0 + tid;
    const uint64_t k = i < last ? order_key(scores[i]) >> shift : 0;
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

cudaError_t launch_block_scores(const SparseParams& p, int dtype, int max_rp_k, cudaStream_t s, uint64_t* launches) {
  const dim3 grid(p.B * p.H, (p.max_blocks + 127) / 128);
  const size_t smem = sizeof(double) * p.group * max_rp_k;
  if (dtype == 0) block_scores_kernel<__nv_bfloat16><<<grid, 128, smem, s>>>(p);
  else block_scores_kernel<float><<<grid, 128, smem, s>>>(p);
  ++*launches;
  return cudaGetLastError();
}

cudaError_t launch_block_select(const SparseParams& p, cudaStream_t s, uint64_t* launches) {
  block_select_kernel<<<p.B * p.H, kSelThreads, 0, s>>>(p);
  ++*launches;
  return cudaGetLastError();
}

}  // namespace ea
