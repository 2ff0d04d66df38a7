// Several query rows per K/V head over one sequence's rows: the drafted tokens of a tree (each with its group of query
// heads), or one token over a list of blocks.  This file holds the parts that are the same for every layer type:
//   mq_project_*, mq_query64, mq_copy_query: Q' of every query row, K' and V' of drafted tokens
//   mq_simt_kernel     attention on the CUDA cores, any dtype (single-precision layers run on it)
//   mq_combine_*       merge the pieces of a query row and lift o' through (U^V)^T
//   tree_commit_kernel moves the rows of an accepted path together
//   write_lens_kernel  the lengths of a captured call
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

// ---------------------------------------------------------------- projections

// Packed pairs of fp32: each half is the ordinary fused multiply-add.
__device__ __forceinline__ uint64_t pack2(float a, float b) {
  uint64_t r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
  return r;
}
__device__ __forceinline__ float2 unpack2(uint64_t v) {
  float2 r;
  asm("mov.b64 {%0, %1}, %2;" : "=f"(r.x), "=f"(r.y) : "l"(v));
  return r;
}
__device__ __forceinline__ void ffma2(uint64_t& d, uint64_t a, uint64_t b) {
  asm("fma.rn.f32x2 %0, %1, %2, %0;" : "+l"(d) : "l"(a), "l"(b));
}

// Token rows of one head and kind (0: queries, 1: keys, 2: values) and where their rank-r form goes.
struct Rows {
  int kind, h, count;      // count: rows of this head and kind
  int rp;
  const float* U;          // [d_head][rp]
};
__device__ __forceinline__ Rows rows_of(const MqProjectParams& p, int kind, int h) {
  Rows r;
  const HeadInfo& hd = p.heads[h];
  r.kind = kind; r.h = h;
  r.count = p.B * p.tokens * (kind == 0 ? p.group : 1);
  r.rp = kind == 2 ? hd.rp_v : hd.rp_k;
  r.U = p.basis + (kind == 2 ? hd.uv_off : hd.uk_off);
  return r;
}
template <typename T>
__device__ __forceinline__ const T* row_source(const MqProjectParams& p, const Rows& w, int row) {
  if (w.kind == 0) {
    const int bt = row / p.group, i = row - bt * p.group, b = bt / p.tokens, t = bt - b * p.tokens;
    return static_cast<const T*>(p.q) + b * p.q_stride_b + t * p.q_stride_t + (static_cast<int64_t>(w.h) * p.group + i) * p.d_head;
  }
  const int b = row / p.tokens, t = row - b * p.tokens;
  return static_cast<const T*>(w.kind == 1 ? p.k : p.v) + b * p.kv_stride_b + t * p.kv_stride_t + static_cast<int64_t>(w.h) * p.d_head;
}
// Where a projected row goes (its first column): the scratch for queries, the cache for keys and values.
template <typename T>
__device__ __forceinline__ char* row_target(const MqProjectParams& p, const Rows& w, int row) {
  if (w.kind == 0) {
    const int bt = row / p.group, i = row - bt * p.group, b = bt / p.tokens, t = bt - b * p.tokens;
    return reinterpret_cast<char*>(p.qp + ((static_cast<int64_t>(w.h) * p.B + b) * p.tokens * p.group + t * p.group + i) * p.q_stride);
  }
  const int b = row / p.tokens, t = row - b * p.tokens;
  const HeadInfo& hd = p.heads[w.h];
  const int64_t crow = physical_row(p.pages, b, p.n_max, p.row0 - (p.deficit ? __ldg(p.deficit + b) : 0) + t);
  return p.cache + (w.kind == 1 ? hd.k_off : hd.v_off) + crow * w.rp * static_cast<int64_t>(sizeof(T));
}
// Columns c..c+N-1: scaled into the scratch, or rounded into the cache.
template <typename T, int N>
__device__ __forceinline__ void store_row(const MqProjectParams& p, const Rows& w, char* row, int c, const float (&x)[N]) {
  if (w.kind == 0 || sizeof(T) == 4) {
    const float f = w.kind == 0 ? p.q_scale : 1.f;
    float* dst = reinterpret_cast<float*>(row) + c;
#pragma unroll
    for (int j = 0; j < N; j += 2) *reinterpret_cast<float2*>(dst + j) = make_float2(x[j] * f, x[j + 1] * f);
  } else {
    uint32_t* dst = reinterpret_cast<uint32_t*>(row) + c / 2;
#pragma unroll
    for (int j = 0; j < N; j += 2) dst[j / 2] = tc::pack_bf16(x[j], x[j + 1]);
  }
}

// Every output is one chain of fused multiply-adds over d_head in ascending order, as in the append kernel: a drafted row
// that is accepted is bit for bit the row that appending its token would have stored.
//
// Many rows: a CTA takes 64 rows of one head and kind against its basis.  A lane has two rows, a warp a quarter of the
// columns: the columns' numbers are the same for all lanes, so a 16-byte load from shared memory feeds eight multiply-adds of
// every lane (and still takes two turns: the loads are the bound).  Five CTAs per SM hold the instance for rank 80 to 96
// registers, 24 bytes of them spilled for 16-bit layers and 204 for fp32 ones (four CTAs: 136 and 140 at rank 128).  Four
// rows per lane halve the loads but leave three CTAs per SM, and a CTA's first loads, past an L2 that the last pass over a long cache has emptied, are a third
// of its time: 504 tokens of 32 heads 37 us against 36.  Tiles of 8 x 4 and 8 x 8 with both operands spread over the lanes
// were bound by their loads too.
constexpr int kPrThreads = 128, kPrRows = 64, kPrPad = 64;

// acc[r][c]: row 2 lane + r, column c0 + c.  a: [k][a_pitch], b: [k][width] with kPrPad floats to spare behind it (the last
// columns of the last warp can lie past the width; they are not stored).
template <int C>
struct RegTile {
  float acc[2][C];
  int lane, c0;
  __device__ __forceinline__ RegTile(int tid) : lane(tid & 31), c0((tid >> 5) * C) {
#pragma unroll
    for (int r = 0; r < 2; ++r)
#pragma unroll
      for (int c = 0; c < C; ++c) acc[r][c] = 0.f;
  }
  __device__ __forceinline__ void multiply(const float* a, const float* b, int k_count, int width, int a_pitch) {
    const float* ar = a + 2 * lane;
    const float* br = b + c0;
    if (c0 >= width) return;
#pragma unroll 4
    for (int k = 0; k < k_count; ++k) {
      const float2 x = *reinterpret_cast<const float2*>(ar + k * a_pitch);
#pragma unroll
      for (int c = 0; c < C; c += 4) {
        const float4 u = *reinterpret_cast<const float4*>(br + c);
        acc[0][c] = fmaf(x.x, u.x, acc[0][c]); acc[0][c + 1] = fmaf(x.x, u.y, acc[0][c + 1]);
        acc[0][c + 2] = fmaf(x.x, u.z, acc[0][c + 2]); acc[0][c + 3] = fmaf(x.x, u.w, acc[0][c + 3]);
        acc[1][c] = fmaf(x.y, u.x, acc[1][c]); acc[1][c + 1] = fmaf(x.y, u.y, acc[1][c + 1]);
        acc[1][c + 2] = fmaf(x.y, u.z, acc[1][c + 2]); acc[1][c + 3] = fmaf(x.y, u.w, acc[1][c + 3]);
      }
      br += width;
    }
  }
};
// Four values of a row at a time, as T or (wide) as fp32.
template <typename T>
__device__ __forceinline__ void put4(T* dst, float a, float b, float c, float d, bool whole) {
  if (whole) {
    if constexpr (sizeof(T) == 2) *reinterpret_cast<uint2*>(dst) = make_uint2(tc::pack_bf16(a, b), tc::pack_bf16(c, d));
    else *reinterpret_cast<float4*>(dst) = make_float4(a, b, c, d);
  } else {
    dst[0] = from_f<T>(a); dst[1] = from_f<T>(b); dst[2] = from_f<T>(c); dst[3] = from_f<T>(d);
  }
}

// Warp-level products for 16-bit layers.  A 32-bit factor enters as two 16-bit parts (the rounded number and its rounded
// remainder, together off by 2^-18 of it).
__device__ __forceinline__ void mma16(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void split_pair(float x0, float x1, uint32_t& hi, uint32_t& lo) {
  hi = tc::pack_bf16(x0, x1);
  lo = tc::pack_bf16(x0 - __uint_as_float(hi << 16), x1 - __uint_as_float(hi & 0xffff0000u));
}
// An image of a basis (leading parts, then remainders; blocks of 8 x 8 numbers, eight columns of the product by eight of its
// inner dimension) into shared memory.  Word `lane` of a block is the lane's half of a B fragment.
__device__ __forceinline__ void copy_image(const float* image, int words, uint32_t* to, int tid, int threads) {
  for (int i = tid; i < words / 4; i += threads) tc::cp_async16(to + 4 * i, image + 4 * i, 16);
  tc::cp_async_commit();
}

// Q' of 64 token rows of a 16-bit layer: a warp's 16 rows are A fragments straight from global memory, exact; the basis is
// split.  (K' and V' rows keep their chains of 32-bit multiply-adds.)
__device__ __forceinline__ void project_queries(const MqProjectParams& p, const Rows& w, int tile, uint32_t* image) {
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, gid = lane >> 2, tig = lane & 3;
  uint32_t a[8][4] = {};
  char* to[2];
#pragma unroll
  for (int i = 0; i < 2; ++i) {              // rows gid and gid + 8
    const int row = tile * kPrRows + warp * 16 + gid + 8 * i;
    to[i] = nullptr;
    if (row >= w.count) continue;
    const __nv_bfloat16* src = row_source<__nv_bfloat16>(p, w, row);
    to[i] = row_target<__nv_bfloat16>(p, w, row);
    if (p.aligned) {
      const uint32_t* x = reinterpret_cast<const uint32_t*>(src) + tig;
#pragma unroll
      for (int k = 0; k < 16; ++k)
        if (8 * k < p.d_head) a[k >> 1][2 * (k & 1) + i] = __ldg(x + 4 * k);
    } else {
      const uint16_t* x = reinterpret_cast<const uint16_t*>(src) + 2 * tig;
#pragma unroll
      for (int k = 0; k < 16; ++k)
        if (8 * k < p.d_head) a[k >> 1][2 * (k & 1) + i] = static_cast<uint32_t>(x[8 * k]) | static_cast<uint32_t>(x[8 * k + 1]) << 16;
    }
  }
  const int steps = p.d_head >> 4, tiles = w.rp >> 3, part = ((w.rp + 15) & ~15) * p.d_head / 2;      // words of one image
  copy_image(p.basis + p.heads[w.h].ukt16_off, 2 * part, image, tid, kPrThreads);
  tc::cp_async_wait<0>();
  __syncthreads();
#pragma unroll 2
  for (int nt = 0; nt < tiles; ++nt) {
    float acc[2][4] = {};                    // leading parts and remainders apart: twice as many chains
#pragma unroll
    for (int s = 0; s < 8; ++s) {
      if (s >= steps) break;
      const uint32_t* b = image + (nt * 2 * steps + 2 * s) * 32 + lane;
      mma16(acc[0], a[s], b[0], b[32]);
      mma16(acc[1], a[s], b[part], b[part + 32]);
    }
#pragma unroll
    for (int i = 0; i < 2; ++i)
      if (to[i] != nullptr)
        *reinterpret_cast<float2*>(reinterpret_cast<float*>(to[i]) + 8 * nt + 2 * tig) =
            make_float2((acc[0][2 * i] + acc[1][2 * i]) * p.q_scale, (acc[0][2 * i + 1] + acc[1][2 * i + 1]) * p.q_scale);
  }
}

// d_head in steps of 32: while a step is multiplied, the next one's rows are on their way into registers and its part of the
// basis into shared memory.
constexpr int kPrStep = 32;
template <typename T, int C>
__global__ void __launch_bounds__(kPrThreads, C <= 20 ? 5 : 4) mq_project_many_kernel(const __grid_constant__ MqProjectParams p) {
  chain_go();
  extern __shared__ __align__(16) float sm[];
  constexpr int kPer = kPrThreads / kPrRows;                 // threads that load a row
  const int tiles_q = (p.B * p.tokens * p.group + kPrRows - 1) / kPrRows, tiles_kv = (p.B * p.tokens + kPrRows - 1) / kPrRows;
  const int nq = p.with_q ? tiles_q : 0;
  int tile = blockIdx.x;
  const int kind = tile < nq ? 0 : tile - nq < tiles_kv ? 1 : 2;
  tile -= kind == 0 ? 0 : kind == 1 ? nq : nq + tiles_kv;
  const Rows w = rows_of(p, kind, blockIdx.y);
  if constexpr (sizeof(T) == 2) {
    if (kind == 0 && p.d_head % 16 == 0) {
      project_queries(p, w, tile, reinterpret_cast<uint32_t*>(sm));
      return;
    }
  }
  const int tid = threadIdx.x, mine = tid % kPrRows, part = tid / kPrRows, row = tile * kPrRows + mine;
  float* xt = sm;                            // [2][32][rows]: a step of the rows, transposed
  float* us = sm + 2 * kPrStep * kPrRows;    // [2][32][rp], kPrPad to spare
  __shared__ char* target[kPrRows];
  constexpr int kVec = 16 / sizeof(T), kLoads = kPrStep / kVec / kPer;
  const T* src = row < w.count ? row_source<T>(p, w, row) : nullptr;
  uint4 raw[kLoads];
  auto fetch = [&](int d0) {                 // this thread's row, its pieces of columns d0 .. d0 + 31
    const int nd = min(kPrStep, p.d_head - d0);
#pragma unroll
    for (int j = 0; j < kLoads; ++j) {
      const int d = (j * kPer + part) * kVec;
      raw[j] = make_uint4(0u, 0u, 0u, 0u);
      if (src != nullptr && d < nd) {
        if (p.aligned) {
          raw[j] = __ldg(reinterpret_cast<const uint4*>(src + d0 + d));
        } else {
          T* e = reinterpret_cast<T*>(&raw[j]);
#pragma unroll
          for (int i = 0; i < kVec; ++i) e[i] = src[d0 + d + i];
        }
      }
    }
  };
  auto basis = [&](int d0, int buf) {
    const int nd = min(kPrStep, p.d_head - d0);
    for (int i = tid; i < nd * w.rp / 4; i += kPrThreads) tc::cp_async16(us + buf * kPrStep * w.rp + 4 * i, w.U + d0 * w.rp + 4 * i, 16);
    tc::cp_async_commit();
  };
  auto put = [&](int buf) {
#pragma unroll
    for (int j = 0; j < kLoads; ++j) {
      const T* e = reinterpret_cast<const T*>(&raw[j]);
#pragma unroll
      for (int i = 0; i < kVec; ++i) xt[(buf * kPrStep + (j * kPer + part) * kVec + i) * kPrRows + mine] = to_f<T>(e[i]);
    }
  };
  basis(0, 0);
  fetch(0);
  if (part == 0) target[mine] = src ? row_target<T>(p, w, row) : nullptr;
  put(0);
  RegTile<C> t(tid);
  for (int d0 = 0, buf = 0; d0 < p.d_head; d0 += kPrStep, buf ^= 1) {
    tc::cp_async_wait<0>();
    __syncthreads();                         // step d0 is there, the other buffers are free
    const bool more = d0 + kPrStep < p.d_head;
    if (more) {
      basis(d0 + kPrStep, buf ^ 1);
      fetch(d0 + kPrStep);
    }
    t.multiply(xt + buf * kPrStep * kPrRows, us + buf * kPrStep * w.rp, min(kPrStep, p.d_head - d0), w.rp, kPrRows);
    if (more) put(buf ^ 1);
  }
  const float f = w.kind == 0 ? p.q_scale : 1.f;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    char* at = target[2 * t.lane + i];
    if (at == nullptr) continue;
#pragma unroll
    for (int c = 0; c < C; c += 4) {
      if (t.c0 + c >= w.rp) break;           // (whole pieces: the rank is a multiple of 8)
      if (w.kind == 0) put4(reinterpret_cast<float*>(at) + t.c0 + c, t.acc[i][c] * f, t.acc[i][c + 1] * f, t.acc[i][c + 2] * f, t.acc[i][c + 3] * f, true);
      else put4(reinterpret_cast<T*>(at) + t.c0 + c, t.acc[i][c], t.acc[i][c + 1], t.acc[i][c + 2], t.acc[i][c + 3], true);
    }
  }
}

// Few rows (a batch of one, short trees): latency is all.  A CTA takes 8 rows x 32 columns, a thread one row and a pair of
// columns; the rows and the 16 KB of the basis arrive together.
constexpr int kPfRows = 8, kPfCols = 32;
template <typename T>
__global__ void __launch_bounds__(128) mq_project_few_kernel(const __grid_constant__ MqProjectParams p) {
  chain_go();
  __shared__ __align__(16) float us[128 * kPfCols];
  __shared__ float xs[kPfRows][128 + 1];
  const int tiles_q = (p.B * p.tokens * p.group + kPfRows - 1) / kPfRows, tiles_kv = (p.B * p.tokens + kPfRows - 1) / kPfRows;
  const int nq = p.with_q ? tiles_q : 0;
  int tile = blockIdx.x;
  const int kind = tile < nq ? 0 : tile - nq < tiles_kv ? 1 : 2;
  tile -= kind == 0 ? 0 : kind == 1 ? nq : nq + tiles_kv;
  const Rows w = rows_of(p, kind, blockIdx.y);
  const int c0 = blockIdx.z * kPfCols, r0 = tile * kPfRows, tid = threadIdx.x;
  if (c0 >= w.rp) return;
  const int nc = min(kPfCols, w.rp - c0);    // a multiple of 8
  for (int i = tid; i < p.d_head * (kPfCols / 4); i += 128) {
    const int d = i / (kPfCols / 4), c = i % (kPfCols / 4) * 4;
    if (c < nc) tc::cp_async16(us + d * kPfCols + c, w.U + d * w.rp + c0 + c, 16);
  }
  tc::cp_async_commit();
  const int nr = min(kPfRows, w.count - r0);
  for (int i = tid; i < nr * p.d_head; i += 128) {
    const int r = i / p.d_head, d = i - r * p.d_head;
    xs[r][d] = to_f<T>(row_source<T>(p, w, r0 + r)[d]);
  }
  tc::cp_async_wait<0>();
  __syncthreads();
  const int r = tid >> 4, c = 2 * (tid & 15);
  if (r >= nr || c >= nc) return;
  uint64_t acc = 0;
#pragma unroll 16
  for (int d = 0; d < p.d_head; ++d)
    ffma2(acc, pack2(xs[r][d], xs[r][d]), *reinterpret_cast<const uint64_t*>(us + d * kPfCols + c));
  const float2 v = unpack2(acc);
  const float x[2] = {v.x, v.y};
  store_row<T, 2>(p, w, row_target<T>(p, w, r0 + r), c0 + c, x);
}

// Queries that are rank-r already: into the scratch.
template <typename T>
__global__ void __launch_bounds__(128) mq_copy_query_kernel(const MqQueryParams p) {
  chain_go();
  const int unit = blockIdx.x, h = unit / p.B, b = unit - h * p.B, row = blockIdx.y, c = threadIdx.x;
  const HeadInfo hd = p.heads[h];
  if (c >= hd.rp_k) return;
  const int t = row / p.group, i = row - t * p.group;
  const T* src = static_cast<const T*>(p.q) + (static_cast<int64_t>(b) * p.tokens + t) * p.group * p.lr_k_width +
                 static_cast<int64_t>(p.group) * hd.lr_k_off + static_cast<int64_t>(i) * hd.rp_k;
  const double x = c < hd.r_k ? static_cast<double>(to_f<T>(src[c])) : 0.0;
  const int64_t at = (static_cast<int64_t>(unit) * p.rows + row) * p.q_stride + c;
  p.qp[at] = static_cast<float>(x * (kLog2e * p.scale));
  if (p.q64) p.q64[at] = x * p.scale;
}

// Q' of one token in 64 bits, for the block scores (and rounded once for the attention): products of a 16-bit and a 32-bit
// number are exact there, so the order of the sum moves a score by 1e-16 of its terms, far below any two scores that are
// not equal.  One CTA per four rows (sequences and query heads) of a head: threads (column, share of d_head); the shares are
// added in a fixed order.
constexpr int kQ64Threads = 512, kQ64Rows = 4, kQ64Ahead = 16;
template <typename T>
__global__ void __launch_bounds__(kQ64Threads) mq_query64_kernel(const MqQueryParams p) {
  chain_go();
  __shared__ double x[kQ64Rows][128];
  __shared__ double part[kQ64Threads][kQ64Rows];
  const int h = blockIdx.y, tid = threadIdx.x;
  const int rp_k = p.heads[h].rp_k;
  const float* U = p.basis + p.heads[h].uk_off;
  // rows of a head: query head g of sequence b is row b * group + g; this CTA's four
  const int r0 = blockIdx.x * kQ64Rows, nr = min(kQ64Rows, p.B * p.group - r0);
  const int shares = kQ64Threads / rp_k;                     // at least four
  const int share = tid / rp_k, c = tid - share * rp_k;
  const int each = (p.d_head + shares - 1) / shares, d0 = share * each, d1 = min(p.d_head, d0 + each);
  float u[kQ64Ahead];                        // on their way while the queries arrive
#pragma unroll
  for (int j = 0; j < kQ64Ahead; ++j) u[j] = share < shares && d0 + j < d1 ? __ldg(U + (d0 + j) * rp_k + c) : 0.f;
  for (int i = tid; i < kQ64Rows * p.d_head; i += kQ64Threads) {
    const int r = i / p.d_head, d = i - r * p.d_head, b = (r0 + r) / p.group, g = (r0 + r) - b * p.group;
    x[r][d] = r < nr ? static_cast<double>(to_f<T>(static_cast<const T*>(p.q)[b * p.q_stride_b + (static_cast<int64_t>(h) * p.group + g) * p.d_head + d])) : 0.0;
  }
  __syncthreads();
  double acc[kQ64Rows] = {0, 0, 0, 0};
  if (share < shares) {
#pragma unroll
    for (int j = 0; j < kQ64Ahead; ++j)
      if (d0 + j < d1) {
        const double uu = u[j];
#pragma unroll
        for (int r = 0; r < kQ64Rows; ++r) acc[r] = fma(x[r][d0 + j], uu, acc[r]);
      }
    for (int d = d0 + kQ64Ahead; d < d1; ++d) {
      const double uu = __ldg(U + d * rp_k + c);
#pragma unroll
      for (int r = 0; r < kQ64Rows; ++r) acc[r] = fma(x[r][d], uu, acc[r]);
    }
#pragma unroll
    for (int r = 0; r < kQ64Rows; ++r) part[tid][r] = acc[r];
  }
  __syncthreads();
  for (int i = tid; i < nr * rp_k; i += kQ64Threads) {
    const int r = i / rp_k, cc = i - r * rp_k, b = (r0 + r) / p.group, g = (r0 + r) - b * p.group;
    double s = 0;
    for (int k = 0; k < shares; ++k) s += part[k * rp_k + cc][r];
    const int64_t at = ((static_cast<int64_t>(h) * p.B + b) * p.group + g) * p.q_stride + cc;
    p.qp[at] = static_cast<float>(s * (kLog2e * p.scale));
    p.q64[at] = s * p.scale;
  }
}

// ---------------------------------------------------------------- attention on the CUDA cores

// 8 warps, one query row each, over tiles of 32 cached rows staged in shared memory as fp32: lane = cached row for the
// scores, lane = channel (up to four) for the weighted sum.  Sums and the softmax state are fp32.
// This is the simple form, right for every layer; it suits few query rows over short contexts (4 heads, 512 rows, 5 tokens:
// 28 us a call).  Every 8 query rows read all cached rows again, and a multiply-add of a score costs two loads from shared
// memory: 4 x 8192 rows, 32 heads of rank 80, fp32: 16 tokens 1618 us and 64 tokens 6138 us, where the bytes are 105 us and
// elementary torch operations take 1324 and 2058; 64 blocks of 64 rows of 4 x 32768: 1007 us, bytes 59.
constexpr int kSimtRows = 8, kSimtTile = 32;
template <typename T>
__global__ void __launch_bounds__(256) mq_simt_kernel(const MqDecodeParams p) {
  chain_go();
  chain_wait();
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
  const int64_t lo = (static_cast<int64_t>(split) * p.per) << p.tile_shift;
  if (split > 0 && lo >= end) return;        // a shorter sequence: nothing left (its first piece always reports)
  const int64_t hi = min(end, lo + (static_cast<int64_t>(p.per) << p.tile_shift));
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

// The pieces of a query row: `count` partials; 2^fold of them `step` floats apart from `first` on, then the same `stride` on.
struct Pieces {
  const float* first;
  int64_t step, stride;
  int count, fold;
  __device__ __forceinline__ const float* at(int s) const { return first + (s >> fold) * stride + (s & ((1 << fold) - 1)) * step; }
};
// The CTA whose range has tile x: the first cta_extra CTAs have a tile more.
__device__ __forceinline__ int cta_of_tile(const MqDecodeParams& p, int x) {
  const int cut = p.cta_extra * (p.cta_tiles + 1);
  return x < cut ? x / (p.cta_tiles + 1) : p.cta_extra + (x - cut) / p.cta_tiles;
}
// Equal pieces of an item: [unit * rows + row][splits].  Ranges over all items (grid > 0): the CTAs whose ranges meet the
// item; `before` = tiles of the sequences in front of b (one run of query rows).
__device__ __forceinline__ Pieces pieces_of(const MqDecodeParams& p, int unit, int row, int64_t before) {
  const int h = unit / p.B, b = unit - h * p.B;
  const int tiles = p.list != nullptr ? p.tiles
                                      : (p.n - (p.deficit != nullptr ? __ldg(p.deficit + b) : 0) + p.tail + (1 << p.tile_shift) - 1) >> p.tile_shift;
  if (p.grid == 0)
    return {p.partials + (static_cast<int64_t>(unit) * p.rows + row) * p.splits * p.part_stride, 0, p.part_stride, max(1, (tiles + p.per - 1) / p.per), 0};
  const int chunks = (p.rows + p.item_rows - 1) / p.item_rows, chunk = row / p.item_rows;
  const int64_t x = (h * p.head_tiles + before) * chunks + static_cast<int64_t>(chunk) * tiles;
  const int c0 = cta_of_tile(p, static_cast<int>(x)), c1 = cta_of_tile(p, static_cast<int>(x) + tiles - 1);
  const int64_t slot = static_cast<int64_t>(unit) * chunks + chunk + c0;
  const int fold = p.copies >> 1;            // (1, 2 or 4 copies)
  return {p.partials + (slot * p.slot_rows + (row - chunk * p.item_rows)) * p.part_stride, static_cast<int64_t>(p.slot_rows >> fold) * p.part_stride,
          static_cast<int64_t>(p.slot_rows) * p.part_stride, (c1 - c0 + 1) << fold, fold};
}
// Tiles of the sequences in front of b, by a whole warp.
__device__ __forceinline__ int64_t tiles_before(const MqDecodeParams& p, int b) {
  if (p.grid == 0) return 0;
  if (p.list != nullptr) return static_cast<int64_t>(b) * p.tiles;
  if (p.deficit == nullptr) return static_cast<int64_t>(b) * ((p.n + p.tail + (1 << p.tile_shift) - 1) >> p.tile_shift);
  int64_t sum = 0;
  for (int i = threadIdx.x & 31; i < b; i += 32) sum += (p.n - __ldg(p.deficit + i) + p.tail + (1 << p.tile_shift) - 1) >> p.tile_shift;
#pragma unroll
  for (int d = 16; d; d >>= 1) sum += __shfl_xor_sync(kFull, sum, d);
  return sum;
}
// o' of one query row from its pieces (0 for a row that sees nothing), column c of this thread where `has`; by whole warps.
// Few pieces: everything is read at once.  Many: the lanes read a piece's maximum and sum each, so that the chain of
// dependent reads is two long.
__device__ __forceinline__ float merged(const Pieces& w, int c, bool has) {
  const int lane = threadIdx.x & 31;
  constexpr int kFew = 4;
  if (w.count <= kFew) {
    float m[kFew], l[kFew], a[kFew], top = -INFINITY, sum = 0.f, o = 0.f;
#pragma unroll
    for (int s = 0; s < kFew; ++s) {
      const float* x = w.at(s);
      m[s] = s < w.count ? x[0] : -INFINITY;
      l[s] = s < w.count ? x[1] : 0.f;
      a[s] = s < w.count && has ? x[4 + c] : 0.f;
    }
#pragma unroll
    for (int s = 0; s < kFew; ++s) top = fmaxf(top, m[s]);
    if (top == -INFINITY) top = 0.f;
#pragma unroll
    for (int s = 0; s < kFew; ++s) {
      const float f = ex2(m[s] - top);       // 0 for a piece without rows
      sum = fmaf(l[s], f, sum);
      o = fmaf(a[s], f, o);
    }
    return sum == 0.f ? 0.f : o / sum;
  }
  float M = -INFINITY;
  for (int s = lane; s < w.count; s += 32) M = fmaxf(M, w.at(s)[0]);
#pragma unroll
  for (int d = 16; d; d >>= 1) M = fmaxf(M, __shfl_xor_sync(kFull, M, d));
  const float base = M == -INFINITY ? 0.f : M;
  float L = 0.f, acc = 0.f;
  for (int s0 = 0; s0 < w.count; s0 += 32) {
    const int n = min(32, w.count - s0);
    const float* x = w.at(s0 + lane);
    const float f = lane < n ? ex2(x[0] - base) : 0.f;       // 0 for a piece without rows
    L = lane < n ? fmaf(x[1], f, L) : L;
#pragma unroll 8
    for (int s = 0; s < n; ++s) {
      const float fs = __shfl_sync(kFull, f, s);
      if (has) acc = fmaf(w.at(s0 + s)[4 + c], fs, acc);
    }
  }
#pragma unroll
  for (int d = 16; d; d >>= 1) L += __shfl_xor_sync(kFull, L, d);
  return L == 0.f ? 0.f : acc / L;
}

// Packed rank-r output.
template <typename T>
__global__ void __launch_bounds__(128) mq_combine_lowrank_kernel(const MqDecodeParams p) {
  chain_wait();
  const int unit = blockIdx.x / p.rows, row = blockIdx.x - unit * p.rows, c = threadIdx.x;
  const int h = unit / p.B, b = unit - h * p.B;
  const HeadInfo hd = p.heads[h];
  const Pieces w = pieces_of(p, unit, row, tiles_before(p, b));
  const float x = merged(w, c, c < hd.rp_v);
  if (c >= hd.rp_v) return;
  const int t = row / p.group, i = row - t * p.group;
  static_cast<T*>(p.out)[(static_cast<int64_t>(b) * p.tokens + t) * p.group * p.lr_v_width + static_cast<int64_t>(p.group) * hd.lr_v_off +
                         static_cast<int64_t>(i) * hd.rp_v + c] = from_f<T>(x);
}

template <typename T>
__device__ __forceinline__ T* out_row(const MqDecodeParams& p, int h, int b, int row) {
  const int t = row / p.group, i = row - t * p.group;
  return static_cast<T*>(p.out) + b * p.out_stride_b + t * p.out_stride_t + (static_cast<int64_t>(h) * p.group + i) * p.d_head;
}

// Few rows: one CTA per query row, thread = output column and half of the rank.
template <typename T>
__global__ void __launch_bounds__(256) mq_combine_few_kernel(const MqDecodeParams p) {
  __shared__ float os[128], ys[128];
  const int unit = blockIdx.x / p.rows, row = blockIdx.x - unit * p.rows, tid = threadIdx.x;
  const int h = unit / p.B, b = unit - h * p.B;
  const HeadInfo hd = p.heads[h];
  const int d = tid & 127, half = tid >> 7;
  const int cut = hd.rp_v >> 1, c0 = half ? cut : 0, nc = half ? hd.rp_v - cut : cut;
  // the basis is on its way while the pieces are merged
  constexpr int kAhead = 32;
  const float* Ut = p.basis + hd.uvt_off + c0 * p.d_head + d;
  float u[kAhead];
#pragma unroll
  for (int j = 0; j < kAhead; ++j) u[j] = j < nc && d < p.d_head ? __ldg(Ut + j * p.d_head) : 0.f;
  const Pieces w = pieces_of(p, unit, row, tiles_before(p, b));
  chain_wait();
  if (tid < 128) {
    const float x = merged(w, tid, tid < hd.rp_v);
    if (tid < hd.rp_v) os[tid] = x;
  }
  __syncthreads();
  float y = 0.f;
#pragma unroll
  for (int j = 0; j < kAhead; ++j)
    if (j < nc) y = fmaf(os[c0 + j], u[j], y);
  if (d < p.d_head)
    for (int j = kAhead; j < nc; ++j) y = fmaf(os[c0 + j], __ldg(Ut + j * p.d_head), y);
  if (half) ys[d] = y;
  __syncthreads();
  if (!half && d < p.d_head) out_row<T>(p, h, b, row)[d] = from_f<T>(y + ys[d]);
}

// Many rows: 64 query rows of one head (of one sequence after the other) against (U^V)^T.
constexpr int kCbRows = 64, kCbPitch = kCbRows + 4;
// o' of the CTA's rows, transposed: [rp_v][kCbPitch].  Two threads merge a row, half of its columns each.
template <typename T>
__device__ __forceinline__ void merge_rows(const MqDecodeParams& p, const HeadInfo& hd, int h, int tid, float* ot, T** target) {
  const int total = p.B * p.rows;
  const int r = tid & (kCbRows - 1), g = blockIdx.x * kCbRows + r;
  const bool there = g < total;
  const int b = there ? g / p.rows : 0;
  // tiles in front of the first sequence here, then of each of those up to this row's own
  const int b0 = blockIdx.x * kCbRows / p.rows;
  int64_t before = tiles_before(p, b0);
  if (p.grid > 0)
    for (int i = b0; i < b; ++i) before += p.list != nullptr ? p.tiles : (p.n - (p.deficit != nullptr ? __ldg(p.deficit + i) : 0) + p.tail + (1 << p.tile_shift) - 1) >> p.tile_shift;
  Pieces w{nullptr, 0, 0, 0, 0};
  if (there) w = pieces_of(p, h * p.B + b, g - b * p.rows, before);
  if (tid < kCbRows) target[r] = there ? out_row<T>(p, h, b, g - b * p.rows) : nullptr;
  chain_wait();
  float M = -INFINITY, L = 0.f;
#pragma unroll 2
  for (int s = 0; s < w.count; ++s) M = fmaxf(M, w.at(s)[0]);
  const float base = M == -INFINITY ? 0.f : M;
#pragma unroll 2
  for (int s = 0; s < w.count; ++s) L = fmaf(w.at(s)[1], ex2(w.at(s)[0] - base), L);
  const float inv = L == 0.f ? 0.f : 1.f / L;                // (a row that sees nothing: its sums are zeros)
  const int half = hd.rp_v / 2, c_lo = (tid / kCbRows) * half;           // half is a multiple of 4
  constexpr int kPieces = 8;                                 // 16-byte pieces of the row that are read together
  for (int c0 = 0; c0 < half; c0 += 4 * kPieces) {
    float4 o[kPieces];
#pragma unroll
    for (int j = 0; j < kPieces; ++j) o[j] = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 1
    for (int s = 0; s < w.count; ++s) {
      const float* x = w.at(s);
      const float f = ex2(x[0] - base) * inv;
#pragma unroll
      for (int j = 0; j < kPieces; ++j) {
        if (c0 + 4 * j >= half) continue;
        const float4 v = *reinterpret_cast<const float4*>(x + 4 + c_lo + c0 + 4 * j);
        o[j].x = fmaf(v.x, f, o[j].x); o[j].y = fmaf(v.y, f, o[j].y); o[j].z = fmaf(v.z, f, o[j].z); o[j].w = fmaf(v.w, f, o[j].w);
      }
    }
#pragma unroll
    for (int j = 0; j < kPieces; ++j) {
      if (c0 + 4 * j >= half) continue;
      float* at = ot + (c_lo + c0 + 4 * j) * kCbPitch + r;
      at[0] = o[j].x; at[kCbPitch] = o[j].y; at[2 * kCbPitch] = o[j].z; at[3 * kCbPitch] = o[j].w;
    }
  }
}

// fp32 layers, and head widths that are no multiple of 16: the register tiles of the projection.
template <typename T, int C>
__global__ void __launch_bounds__(kPrThreads) mq_combine_many_kernel(const __grid_constant__ MqDecodeParams p) {
  extern __shared__ __align__(16) float sm[];
  const int h = blockIdx.y, tid = threadIdx.x;
  const HeadInfo hd = p.heads[h];
  float* ot = sm;
  float* us = sm + hd.rp_v * kCbPitch;      // [rp_v][d_head]
  __shared__ T* target[kCbRows];
  const float* Ut = p.basis + hd.uvt_off;
  for (int i = tid; i < hd.rp_v * p.d_head / 4; i += kPrThreads) tc::cp_async16(us + 4 * i, Ut + 4 * i, 16);
  tc::cp_async_commit();
  merge_rows<T>(p, hd, h, tid, ot, target);
  tc::cp_async_wait<0>();
  __syncthreads();
  RegTile<C> t(tid);
  t.multiply(ot, us, hd.rp_v, p.d_head, kCbPitch);
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    T* dst = target[2 * t.lane + i];
    if (dst == nullptr) continue;
    const bool whole = reinterpret_cast<uintptr_t>(dst) % (4 * sizeof(T)) == 0;
#pragma unroll
    for (int c = 0; c < C; c += 4)
      if (t.c0 + c < p.d_head) put4(dst + t.c0 + c, t.acc[i][c], t.acc[i][c + 1], t.acc[i][c + 2], t.acc[i][c + 3], whole);
  }
}

// 16-bit layers: a warp lifts 16 rows with warp-level products, both factors in two parts (three products: what is left out,
// remainder times remainder, is 2^-18 of the terms).  NT: runs of 8 output columns.
template <int NT>
__global__ void __launch_bounds__(kPrThreads) mq_combine_mma_kernel(const __grid_constant__ MqDecodeParams p) {
  extern __shared__ __align__(16) float sm[];
  const int h = blockIdx.y, tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, gid = lane >> 2, tig = lane & 3;
  const HeadInfo hd = p.heads[h];
  const int steps = (hd.rp_v + 15) >> 4, tiles = p.d_head >> 3, part = 16 * steps * p.d_head / 2;     // words of one image
  uint32_t* image = reinterpret_cast<uint32_t*>(sm);
  float* ot = sm + 2 * part;                                 // [16 steps][kCbPitch]
  __shared__ __nv_bfloat16* target[kCbRows];
  copy_image(p.basis + hd.uvl16_off, 2 * part, image, tid, kPrThreads);
  for (int i = hd.rp_v * kCbPitch + tid; i < 16 * steps * kCbPitch; i += kPrThreads) ot[i] = 0.f;
  merge_rows<__nv_bfloat16>(p, hd, h, tid, ot, target);
  tc::cp_async_wait<0>();
  __syncthreads();
  float acc[NT][4] = {};
  for (int s = 0; s < steps; ++s) {
    const float* x = ot + (16 * s + 2 * tig) * kCbPitch + 16 * warp + gid;
    uint32_t hi[4], lo[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {            // rows gid, gid + 8 of columns 2 tig, 2 tig + 1, then of the eight columns behind
      const float* y = x + (i >> 1) * 8 * kCbPitch + (i & 1) * 8;
      split_pair(y[0], y[kCbPitch], hi[i], lo[i]);
    }
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      if (nt >= tiles) break;
      const uint32_t* b = image + (nt * 2 * steps + 2 * s) * 32 + lane;
      mma16(acc[nt], hi, b[0], b[32]);
      mma16(acc[nt], lo, b[0], b[32]);
      mma16(acc[nt], hi, b[part], b[part + 32]);
    }
  }
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    __nv_bfloat16* dst = target[16 * warp + gid + 8 * i];
    if (dst == nullptr) continue;
    dst += 2 * tig;
    const bool whole = reinterpret_cast<uintptr_t>(dst) % 4 == 0;
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      if (nt >= tiles) break;
      if (whole) {
        *reinterpret_cast<uint32_t*>(dst + 8 * nt) = tc::pack_bf16(acc[nt][2 * i], acc[nt][2 * i + 1]);
      } else {
        dst[8 * nt] = __float2bfloat16_rn(acc[nt][2 * i]);
        dst[8 * nt + 1] = __float2bfloat16_rn(acc[nt][2 * i + 1]);
      }
    }
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
  const int n_b = (p.deficit != nullptr ? p.n - p.deficit[b] : p.n) - (p.grown ? count : 0);
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

__global__ void __launch_bounds__(128) write_lens_kernel(const __grid_constant__ LensParams p) {
  for (int i = threadIdx.x; i < p.count; i += 128) p.to[i] = p.value[i];
}

}  // namespace

cudaError_t launch_write_lens(const LensParams& p, cudaStream_t s, uint64_t* launches) {
  write_lens_kernel<<<1, 128, 0, s>>>(p);
  ++*launches;
  return cudaGetLastError();
}

cudaError_t launch_mq_query(const MqQueryParams& p, int dtype, cudaStream_t s, uint64_t* launches) {
  if (p.flags & 0x1u) {                      // EA_Q_PREPROJECTED
    const dim3 grid(p.B * p.H, p.rows);
    if (dtype == 0) mq_copy_query_kernel<__nv_bfloat16><<<grid, 128, 0, s>>>(p);
    else mq_copy_query_kernel<float><<<grid, 128, 0, s>>>(p);
  } else {
    const dim3 grid((p.B * p.group + kQ64Rows - 1) / kQ64Rows, p.H);
    if (dtype == 0) mq_query64_kernel<__nv_bfloat16><<<grid, kQ64Threads, 0, s>>>(p);
    else mq_query64_kernel<float><<<grid, kQ64Threads, 0, s>>>(p);
  }
  ++*launches;
  return cudaGetLastError();
}

template <typename T, int C>
static cudaError_t launch_project_many(const MqProjectParams& p, int tiles, int max_rp, cudaStream_t s) {
  size_t smem = sizeof(float) * (2 * kPrStep * (kPrRows + max_rp) + kPrPad);
  const size_t image = static_cast<size_t>((max_rp + 15) & ~15) * p.d_head * 4;
  if (sizeof(T) == 2 && p.with_q && image > smem) smem = image;
  static size_t configured[kMaxDevices] = {};
  const cudaError_t e = ensure_dynamic_smem(mq_project_many_kernel<T, C>, smem, configured);
  if (e != cudaSuccess) return e;
  mq_project_many_kernel<T, C><<<dim3(tiles, p.H), kPrThreads, smem, s>>>(p);
  return cudaGetLastError();
}
template <typename T>
static cudaError_t launch_project_t(const MqProjectParams& p, int max_rp, cudaStream_t s) {
  const int rows_kv = p.B * p.tokens, rows_q = rows_kv * p.group;
  auto tiles = [&](int rows) {
    return (p.with_q ? (rows_q + rows - 1) / rows : 0) + (p.k != nullptr ? 2 * ((rows_kv + rows - 1) / rows) : 0);
  };
  if (rows_kv < 48) {                        // too few rows to fill a tile
    mq_project_few_kernel<T><<<dim3(tiles(kPfRows), p.H, (max_rp + kPfCols - 1) / kPfCols), 128, 0, s>>>(p);
    return cudaGetLastError();
  }
  const int n = tiles(kPrRows);
  switch ((max_rp + 15) / 16) {              // columns of a warp: a quarter of the widest rank, in fours
    case 1: case 2: return launch_project_many<T, 8>(p, n, max_rp, s);
    case 3: return launch_project_many<T, 12>(p, n, max_rp, s);
    case 4: return launch_project_many<T, 16>(p, n, max_rp, s);
    case 5: return launch_project_many<T, 20>(p, n, max_rp, s);
    case 6: return launch_project_many<T, 24>(p, n, max_rp, s);
    case 7: return launch_project_many<T, 28>(p, n, max_rp, s);
    default: return launch_project_many<T, 32>(p, n, max_rp, s);
  }
}

cudaError_t launch_mq_project(const MqProjectParams& p, int dtype, int max_rp, cudaStream_t s, uint64_t* launches) {
  ++*launches;
  return dtype == 0 ? launch_project_t<__nv_bfloat16>(p, max_rp, s) : launch_project_t<float>(p, max_rp, s);
}

cudaError_t launch_mq_simt(const MqDecodeParams& p, int dtype, cudaStream_t s, uint64_t* launches) {
  const int chunks = (p.rows + kSimtRows - 1) / kSimtRows;
  const dim3 grid(p.B * p.H * chunks, p.splits);
  const size_t smem = sizeof(float) * (kSimtRows * 128 + kSimtTile * 129 + kSimtTile * 128);
  ++*launches;
  return dtype == 0 ? launch_chained(p.chained != 0, mq_simt_kernel<__nv_bfloat16>, grid, 256, smem, s, p) : launch_chained(p.chained != 0, mq_simt_kernel<float>, grid, 256, smem, s, p);
}

template <typename Kernel>
static cudaError_t launch_combine_many(const MqDecodeParams& p, Kernel kernel, size_t smem, size_t (&configured)[kMaxDevices], cudaStream_t s) {
  const cudaError_t e = ensure_dynamic_smem(kernel, smem, configured);
  if (e != cudaSuccess) return e;
  return launch_chained(p.chained != 0, kernel, dim3((p.B * p.rows + kCbRows - 1) / kCbRows, p.H), kPrThreads, smem, s, p);
}
template <typename T>
static cudaError_t launch_combine_t(const MqDecodeParams& p, int max_rp_v, cudaStream_t s) {
  const int64_t units = static_cast<int64_t>(p.B) * p.H, rows = units * p.rows;
  if (p.flags & 0x2u) {                      // EA_OUT_LOWRANK
    return launch_chained(p.chained != 0, mq_combine_lowrank_kernel<T>, static_cast<unsigned>(rows), 128, 0, s, p);
  } else if (p.B * p.rows >= 64 && rows >= 2048) {
    static size_t configured[4][kMaxDevices] = {};
    if (sizeof(T) == 2 && p.d_head % 16 == 0) {
      const size_t smem = static_cast<size_t>((max_rp_v + 15) & ~15) * (p.d_head + kCbPitch) * sizeof(float);
      return p.d_head <= 64 ? launch_combine_many(p, mq_combine_mma_kernel<8>, smem, configured[0], s)
                            : launch_combine_many(p, mq_combine_mma_kernel<16>, smem, configured[1], s);
    }
    const size_t smem = sizeof(float) * (max_rp_v * (kCbPitch + p.d_head) + kPrPad);
    return p.d_head <= 64 ? launch_combine_many(p, mq_combine_many_kernel<T, 16>, smem, configured[2], s)
                          : launch_combine_many(p, mq_combine_many_kernel<T, 32>, smem, configured[3], s);
  } else {
    return launch_chained(p.chained != 0, mq_combine_few_kernel<T>, static_cast<unsigned>(rows), 256, 0, s, p);
  }
}

cudaError_t launch_mq_combine(const MqDecodeParams& p, int dtype, int max_rp_v, cudaStream_t s, uint64_t* launches) {
  ++*launches;
  return dtype == 0 ? launch_combine_t<__nv_bfloat16>(p, max_rp_v, s) : launch_combine_t<float>(p, max_rp_v, s);
}

cudaError_t launch_tree_commit(const TreeCommitParams& p, int sequences, cudaStream_t s, uint64_t* launches) {
  tree_commit_kernel<<<sequences * p.H, 256, 0, s>>>(p);
  ++*launches;
  return cudaGetLastError();
}

}  // namespace ea
