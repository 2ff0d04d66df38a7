// Several query rows per K/V head over one sequence's rows: the drafted tokens of a tree (each with its group of query
// heads), or one token over a list of blocks.  This file holds the parts that are the same for every layer type:
//   mq_query_kernel    Q' = Q U^K of every query row (and in 64 bits for the block scores)
//   mq_simt_kernel     attention on the CUDA cores, any dtype (single-precision layers run on it)
//   mq_combine_kernel  merges the pieces of a query row and lifts o' through (U^V)^T
//   tree_commit_kernel moves the rows of an accepted path together
#include <cuda_bf16.h>

#include "internal.h"
#include "tc_common.cuh"

namespace ea {
namespace {

using tc::ex2;

template <typename T> __device__ __forceinline__ float to_f(T v);
template <> __device__ __forceinline__ float to_f<float>(float v) { return v; }
template <> __device__ __forceinline__ float to_f<__nv_bfloat16>(__nv_bfloat16 v) { return __bfloat162float(v); }
template <typename T> __device__ __forceinline__ T from_f(float v);
template <> __device__ __forceinline__ float from_f<float>(float v) { return v; }
template <> __device__ __forceinline__ __nv_bfloat16 from_f<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }

constexpr unsigned kFull = 0xffffffffu;
constexpr double kLog2e = 1.4426950408889634;

// A drafted token's mask with the bits that name no token of the tree cleared.
__device__ __forceinline__ uint64_t tree_mask(uint64_t m, int tokens) { return tokens < 64 ? m & ((1ull << tokens) - 1) : m; }
// How far behind the cached rows token t sits: the number of the other tokens it sees.
__device__ __forceinline__ int tree_depth(uint64_t m, int t) { return __popcll(m & ~(1ull << t)); }

// ---------------------------------------------------------------- Q'

// One CTA per (unit, run of kQueryRows query rows): thread c owns column c of Q'.  With q64 the sums are taken in 64
// bits (products of a 16-bit and a 32-bit number are exact there, so the order of the sum moves a block score by
// 1e-16 of its terms, far below any two scores that are not equal).
constexpr int kQueryRows = 8;
template <typename T, typename Acc>
__global__ void __launch_bounds__(128) mq_query_kernel(const MqQueryParams p) {
  __shared__ float x[kQueryRows][128];
  const int unit = blockIdx.x, h = unit / p.B, b = unit - h * p.B;
  const int r0 = blockIdx.y * kQueryRows, nr = min(kQueryRows, p.rows - r0);
  const HeadInfo hd = p.heads[h];
  const T* q = static_cast<const T*>(p.q);
  const int c = threadIdx.x;
  Acc acc[kQueryRows];
  if (p.flags & 0x1u) {                      // EA_Q_PREPROJECTED: the rows are rank-r already
    for (int r = 0; r < nr; ++r) {
      const int t = (r0 + r) / p.group, i = (r0 + r) - t * p.group;
      const T* src = q + (static_cast<int64_t>(b) * p.tokens + t) * p.group * p.lr_k_width +
                     static_cast<int64_t>(p.group) * hd.lr_k_off + static_cast<int64_t>(i) * hd.rp_k;
      acc[r] = c < hd.r_k ? static_cast<Acc>(to_f<T>(src[c])) : Acc(0);
    }
  } else {
    for (int idx = threadIdx.x; idx < nr * p.d_head; idx += 128) {
      const int r = idx / p.d_head, d = idx - r * p.d_head;
      const int t = (r0 + r) / p.group, i = (r0 + r) - t * p.group;
      x[r][d] = to_f<T>(q[b * p.q_stride_b + t * p.q_stride_t + (static_cast<int64_t>(h) * p.group + i) * p.d_head + d]);
    }
    __syncthreads();
#pragma unroll
    for (int r = 0; r < kQueryRows; ++r) acc[r] = Acc(0);
    if (c < hd.rp_k) {
      const float* U = p.basis + hd.uk_off + c;
#pragma unroll 8
      for (int d = 0; d < p.d_head; ++d) {
        const Acc u = static_cast<Acc>(__ldg(U + d * hd.rp_k));
#pragma unroll
        for (int r = 0; r < kQueryRows; ++r)
          if (r < nr) acc[r] += static_cast<Acc>(x[r][d]) * u;
      }
    }
  }
  if (c >= hd.rp_k) return;
  const int64_t row0 = static_cast<int64_t>(unit) * p.rows + r0;
#pragma unroll
  for (int r = 0; r < kQueryRows; ++r)
    if (r < nr) {
      p.qp[(row0 + r) * p.q_stride + c] = static_cast<float>(acc[r] * static_cast<Acc>(kLog2e * p.scale));
      if (p.q64) p.q64[(row0 + r) * p.q_stride + c] = static_cast<double>(acc[r]) * p.scale;
    }
}

// ---------------------------------------------------------------- attention on the CUDA cores

// 8 warps, one query row each, over tiles of 32 cached rows staged in shared memory as fp32: lane = cached row for the
// scores, lane = channel (up to four) for the weighted sum.  Sums and the softmax state are fp32.
constexpr int kSimtRows = 8, kSimtTile = 32;
template <typename T>
__global__ void __launch_bounds__(256) mq_simt_kernel(const MqDecodeParams p) {
  extern __shared__ float sm[];
  __shared__ int64_t phys[kSimtTile];
  __shared__ int logical[kSimtTile];         // logical row, -1 = nothing there
  const int chunks = (p.rows + kSimtRows - 1) / kSimtRows;
  const int unit = blockIdx.x / chunks, chunk = blockIdx.x - unit * chunks, split = blockIdx.y;
  const int h = unit / p.B, b = unit - h * p.B;
  const HeadInfo hd = p.heads[h];
  const int rp_k = hd.rp_k, rp_v = hd.rp_v, kp = rp_k + 1;
  float* qs = sm;                            // [8][rp_k]
  float* ks = qs + kSimtRows * rp_k;         // [32][rp_k + 1]
  float* vs = ks + kSimtTile * kp;           // [32][rp_v]
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int row = chunk * kSimtRows + warp;
  const bool live = row < p.rows;
  const int t = live ? row / p.group : 0;

  const int n_b = p.deficit != nullptr ? p.n - __ldg(p.deficit + b) : p.n;
  const int64_t end = p.list ? static_cast<int64_t>(p.list_len) << p.block_shift : static_cast<int64_t>(n_b) + p.tail;
  const int per = (p.tiles + p.splits - 1) / p.splits;
  const int64_t lo = min(end, static_cast<int64_t>(split) * per * 128);
  const int64_t hi = min(end, lo + static_cast<int64_t>(per) * 128);
  const uint64_t* masks = p.mask + static_cast<int64_t>(b) * p.tokens;
  const uint64_t seen = p.tail && live ? tree_mask(masks[t], p.tokens) : 0;
  const int pos = p.tail ? n_b + tree_depth(seen, t) : n_b - 1;        // position of the query
  const int32_t* list = p.list ? p.list + static_cast<int64_t>(unit) * p.list_len : nullptr;

  for (int i = tid; i < kSimtRows * rp_k; i += 256) {
    const int r = i / rp_k, c = i - r * rp_k;
    const int row_i = chunk * kSimtRows + r;
    qs[i] = row_i < p.rows ? p.qp[(static_cast<int64_t>(unit) * p.rows + row_i) * p.q_stride + c] : 0.f;
  }
  float m = -INFINITY, l = 0.f, o[4] = {0.f, 0.f, 0.f, 0.f};
  for (int64_t j0 = lo; j0 < hi; j0 += kSimtTile) {
    if (tid < kSimtTile) {
      int r = -1;
      if (j0 + tid < hi) {
        if (list) {
          const int blk = list[(j0 + tid) >> p.block_shift];
          r = blk < 0 ? -1 : (blk << p.block_shift) + static_cast<int>((j0 + tid) & ((1 << p.block_shift) - 1));
          if (r >= n_b) r = -1;
        } else {
          r = static_cast<int>(j0) + tid;
        }
      }
      logical[tid] = r;
      phys[tid] = r >= 0 ? physical_row(p.pages, b, p.n_max, r) : 0;
    }
    __syncthreads();                         // (first round: qs too)
    for (int i = tid; i < kSimtTile * rp_k; i += 256) {
      const int r = i / rp_k, c = i - r * rp_k;
      ks[r * kp + c] = logical[r] >= 0 ? to_f<T>(reinterpret_cast<const T*>(p.cache + hd.k_off)[phys[r] * rp_k + c]) : 0.f;
    }
    for (int i = tid; i < kSimtTile * rp_v; i += 256) {
      const int r = i / rp_v, c = i - r * rp_v;
      vs[i] = logical[r] >= 0 ? to_f<T>(reinterpret_cast<const T*>(p.cache + hd.v_off)[phys[r] * rp_v + c]) : 0.f;
    }
    __syncthreads();
    if (live) {
      const float* kr = ks + lane * kp;
      const float* qr = qs + warp * rp_k;
      float s = 0.f;
#pragma unroll 8
      for (int c = 0; c < rp_k; ++c) s = fmaf(qr[c], kr[c], s);
      const int r = logical[lane];
      int at = r;                            // position of the cached row
      bool open = r >= 0;
      if (p.tail && r >= n_b) {
        const int d = r - n_b;
        open = (seen >> d) & 1;
        at = n_b + tree_depth(tree_mask(masks[d], p.tokens), d);
      }
      if (hd.alibi_slope2 != 0.f) s = fmaf(hd.alibi_slope2, static_cast<float>(at - pos), s);
      s = open ? s : -INFINITY;
      float mt = s;
#pragma unroll
      for (int d = 16; d; d >>= 1) mt = fmaxf(mt, __shfl_xor_sync(kFull, mt, d));
      const float m2 = fmaxf(m, mt);
      const float base = m2 == -INFINITY ? 0.f : m2;      // nothing seen yet: every weight below is 2^-inf = 0
      const float f = ex2(m - base);
      const float w = ex2(s - base);
      m = m2;
      l = fmaf(l, f, w);                     // this lane's share; summed over the lanes at the end
#pragma unroll
      for (int i = 0; i < 4; ++i) o[i] *= f;
      const unsigned used = __ballot_sync(kFull, open);
      for (int jj = 0; jj < kSimtTile; ++jj) {
        if (!((used >> jj) & 1)) continue;   // a masked row takes no part, whatever its value row holds
        const float wj = __shfl_sync(kFull, w, jj);
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (lane + 32 * i < rp_v) o[i] = fmaf(wj, vs[jj * rp_v + lane + 32 * i], o[i]);
      }
    }
    __syncthreads();
  }
  if (!live) return;
#pragma unroll
  for (int d = 16; d; d >>= 1) l += __shfl_xor_sync(kFull, l, d);
  float* part = p.partials + ((static_cast<int64_t>(unit) * p.rows + row) * p.splits + split) * p.part_stride;
  if (lane == 0) { part[0] = m; part[1] = l; }
#pragma unroll
  for (int i = 0; i < 4; ++i)
    if (lane + 32 * i < rp_v) part[4 + lane + 32 * i] = o[i];
}

// ---------------------------------------------------------------- merge and lift

// One CTA per run of RB query rows of a unit: a row of (U^V)^T is read once for the RB rows.
template <typename T, int RB>
__global__ void __launch_bounds__(128) mq_combine_kernel(const MqDecodeParams p) {
  __shared__ float os[RB][128];
  const int runs = (p.rows + RB - 1) / RB;
  const int unit = blockIdx.x / runs, r0 = (blockIdx.x - unit * runs) * RB, tid = threadIdx.x;
  const int h = unit / p.B, b = unit - h * p.B;
  const HeadInfo hd = p.heads[h];
  const int nr = min(RB, p.rows - r0);
  for (int r = 0; r < nr; ++r) {
    const float* part = p.partials + (static_cast<int64_t>(unit) * p.rows + r0 + r) * p.splits * p.part_stride;
    float M = -INFINITY;
    for (int s = 0; s < p.splits; ++s) M = fmaxf(M, part[s * p.part_stride]);
    const float base = M == -INFINITY ? 0.f : M;
    float L = 0.f, acc = 0.f;
    for (int s = 0; s < p.splits; ++s) {
      const float* x = part + s * p.part_stride;
      const float f = ex2(x[0] - base);      // 0 for a piece without rows
      L = fmaf(x[1], f, L);
      if (tid < hd.rp_v) acc = fmaf(x[4 + tid], f, acc);
    }
    // a query row that sees nothing returns zeros
    os[r][tid] = tid < hd.rp_v ? (L == 0.f ? 0.f : acc / L) : 0.f;
  }
  __syncthreads();
  T* out = static_cast<T*>(p.out);
  if (p.flags & 0x2u) {                      // EA_OUT_LOWRANK
    for (int r = 0; r < nr; ++r) {
      const int t = (r0 + r) / p.group, i = (r0 + r) - t * p.group;
      T* dst = out + (static_cast<int64_t>(b) * p.tokens + t) * p.group * p.lr_v_width +
               static_cast<int64_t>(p.group) * hd.lr_v_off + static_cast<int64_t>(i) * hd.rp_v;
      if (tid < hd.rp_v) dst[tid] = from_f<T>(os[r][tid]);
    }
    return;
  }
  if (tid >= p.d_head) return;
  const float* Ut = p.basis + hd.uvt_off + tid;
  float y[RB];
#pragma unroll
  for (int r = 0; r < RB; ++r) y[r] = 0.f;
#pragma unroll 8
  for (int c = 0; c < hd.rp_v; ++c) {
    const float u = __ldg(Ut + c * p.d_head);
#pragma unroll
    for (int r = 0; r < RB; ++r)
      if (r < nr) y[r] = fmaf(os[r][c], u, y[r]);
  }
#pragma unroll
  for (int r = 0; r < RB; ++r)
    if (r < nr) {
      const int t = (r0 + r) / p.group, i = (r0 + r) - t * p.group;
      out[b * p.out_stride_b + t * p.out_stride_t + (static_cast<int64_t>(h) * p.group + i) * p.d_head + tid] = from_f<T>(y[r]);
    }
}

// ---------------------------------------------------------------- acceptance of a path

// Rows n_b + path[i] move to n_b + i.  One CTA per unit walks the 16-byte pieces of the rows in ascending order, a
// batch at a time: all loads of a batch before its stores.  path is strictly increasing, so path[i] >= i: a batch
// never overwrites a row that a later one reads.
__global__ void __launch_bounds__(256) tree_commit_kernel(const __grid_constant__ TreeCommitParams p) {
  const int bi = blockIdx.x / p.H, h = blockIdx.x - bi * p.H, b = p.b0 + bi;
  const int count = p.count[bi];
  if (count == 0) return;
  const HeadInfo hd = p.heads[h];
  const int n_b = p.deficit != nullptr ? p.n - p.deficit[b] : p.n;
  const int kc = hd.rp_k * p.es / 16, vc = hd.rp_v * p.es / 16, per = kc + vc;
  constexpr int kBatch = 4;
  for (int i0 = 0; i0 < count * per; i0 += 256 * kBatch) {
    uint4 x[kBatch];
    uint4* dst[kBatch];
#pragma unroll
    for (int k = 0; k < kBatch; ++k) {
      const int idx = i0 + k * 256 + threadIdx.x;
      dst[k] = nullptr;
      if (idx < count * per) {
        const int i = idx / per, c = idx - i * per, from = p.path[bi][i];
        if (from != i) {
          const int64_t src = physical_row(p.pages, b, p.n_max, n_b + from), to = physical_row(p.pages, b, p.n_max, n_b + i);
          uint4* slab = reinterpret_cast<uint4*>(p.cache + (c < kc ? hd.k_off : hd.v_off));
          const int w = c < kc ? kc : vc, cc = c < kc ? c : c - kc;
          x[k] = slab[src * w + cc];
          dst[k] = slab + to * w + cc;
        }
      }
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < kBatch; ++k)
      if (dst[k]) *dst[k] = x[k];
    __syncthreads();
  }
}

}  // namespace

cudaError_t launch_mq_query(const MqQueryParams& p, int dtype, cudaStream_t s, uint64_t* launches) {
  const dim3 grid(p.B * p.H, (p.rows + kQueryRows - 1) / kQueryRows);
  if (dtype == 0) {
    if (p.q64) mq_query_kernel<__nv_bfloat16, double><<<grid, 128, 0, s>>>(p);
    else mq_query_kernel<__nv_bfloat16, float><<<grid, 128, 0, s>>>(p);
  } else {
    if (p.q64) mq_query_kernel<float, double><<<grid, 128, 0, s>>>(p);
    else mq_query_kernel<float, float><<<grid, 128, 0, s>>>(p);
  }
  ++*launches;
  return cudaGetLastError();
}

cudaError_t launch_mq_simt(const MqDecodeParams& p, int dtype, cudaStream_t s, uint64_t* launches) {
  const int chunks = (p.rows + kSimtRows - 1) / kSimtRows;
  const dim3 grid(p.B * p.H * chunks, p.splits);
  const size_t smem = sizeof(float) * (kSimtRows * 128 + kSimtTile * 129 + kSimtTile * 128);
  if (dtype == 0) mq_simt_kernel<__nv_bfloat16><<<grid, 256, smem, s>>>(p);
  else mq_simt_kernel<float><<<grid, 256, smem, s>>>(p);
  ++*launches;
  return cudaGetLastError();
}

cudaError_t launch_mq_combine(const MqDecodeParams& p, int dtype, cudaStream_t s, uint64_t* launches) {
  const int64_t units = static_cast<int64_t>(p.B) * p.H;
  const bool many = units * p.rows >= 2048;                   // enough rows to fill the chip eight at a time
  const int rb = many ? 8 : 1;
  const unsigned grid = static_cast<unsigned>(units * ((p.rows + rb - 1) / rb));
  if (dtype == 0) {
    if (many) mq_combine_kernel<__nv_bfloat16, 8><<<grid, 128, 0, s>>>(p);
    else mq_combine_kernel<__nv_bfloat16, 1><<<grid, 128, 0, s>>>(p);
  } else {
    if (many) mq_combine_kernel<float, 8><<<grid, 128, 0, s>>>(p);
    else mq_combine_kernel<float, 1><<<grid, 128, 0, s>>>(p);
  }
  ++*launches;
  return cudaGetLastError();
}

cudaError_t launch_tree_commit(const TreeCommitParams& p, int sequences, cudaStream_t s, uint64_t* launches) {
  tree_commit_kernel<<<sequences * p.H, 256, 0, s>>>(p);
  ++*launches;
  return cudaGetLastError();
}

}  // namespace ea
