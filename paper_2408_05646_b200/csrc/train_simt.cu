// Causal attention over rank-space rows and its backward pass on the CUDA cores, for fp32 layers.
//   S_ij = scale q'_i k'_j + b(i - j)  (j <= i < length),  P = softmax(S),  o'_i = sum_j P_ij v'_j
//   delta_i = do'_i o'_i,  dS_ij = P_ij (do'_i v'_j - delta_i),
//   dq'_i = scale sum_j dS_ij k'_j,  dk'_j = scale sum_i dS_ij q'_i,  dv'_j = sum_i P_ij do'_i,  db_u = sum dS_ij over the
//   distances of bucket u
// P is recomputed from the row's maximum and the reciprocal of its sum, which the forward pass leaves: their logarithm, one
// number, would cost the exponent's last bits.  A CTA has a tile of 32 query (or key) rows and walks the other axis in tiles
// of 64, fetched one ahead; a thread has 2 x 4 scores and 2 rows x 2 to 8 columns of the sums.  dq' and dk', dv' are two
// kernels, so that nothing is added up by atomics.  A tile's products are summed apart and then added, which keeps the rounding
// errors of long sums down.  Bound by the latency of the shared-memory reads in front of the multiply-adds (2 x 500 tokens,
// 8 heads of rank 40: forward 45, dq' 56, dk' and dv' 53 us; own tiles of 64 rows, half as many CTAs, took 95, 128 and 136).
// The loops are unrolled for registers, not for CTAs: with the compiler's own choice, 128 registers and two CTAs per SM, the
// three took 188 us, with one CTA and its loads four steps ahead 159.  Every thread fetches pieces of one row, without a division:
// 159 to 151.
#include "internal.h"
#include "tc_common.cuh"

namespace ea {
namespace {

constexpr int kOwn = 32;                  // rows of a CTA's own tile
constexpr int kWalk = 64;                 // rows of a tile of the walked axis
constexpr int kThreads = 256;
constexpr int kPitchP = kWalk + 4;
constexpr int RI = kOwn / 16;             // own rows of a thread
template <int NC> constexpr int kPitch = 16 * NC + 4;        // of rows in shared memory, for NC columns a thread

__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// Packed rows on their way into shared memory, zeros behind `rows`; columns from `live` on are the rank's
// padding: zeros, whatever the caller left there.  wide: the rows lie on 16-byte boundaries.
template <int COUNT, int PITCH>
__device__ __forceinline__ void fetch_rows(float* dst, const float* src, int64_t stride, int rows, int width, int live, bool wide, int tid) {
  constexpr int kLanes = kThreads / COUNT;                   // threads of a row
  const int r = tid / kLanes, first = tid % kLanes;
  const uint32_t to = tc::smem_u32(dst + r * PITCH);
  const float* from = r < rows ? src + r * stride : src;
  const int have = r < rows ? live : 0;                      // numbers of the row
  if (wide) {
    for (int c = 4 * first; c < width; c += 4 * kLanes) {
      const int bytes = 4 * min(max(have - c, 0), 4);
      asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(to + 4 * c), "l"(bytes > 0 ? from + c : src), "r"(bytes) : "memory");
    }
  } else {
    for (int c = first; c < width; c += kLanes) {
      const int bytes = c < have ? 4 : 0;
      asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(to + 4 * c), "l"(bytes > 0 ? from + c : src), "r"(bytes) : "memory");
    }
  }
}
// The rows of this CTA's own tile, kept for the backward pass.
template <int PITCH>
__device__ __forceinline__ void keep_rows(float* dst, const float* src, int64_t stride, int rows, int width, int tid) {
  const int quads = width >> 2;
  for (int idx = tid; idx < rows * quads; idx += kThreads) {
    const int r = idx / quads, c = 4 * (idx - r * quads);
    *reinterpret_cast<float4*>(dst + r * stride + c) = *reinterpret_cast<const float4*>(src + r * PITCH + c);
  }
}
__device__ __forceinline__ bool on16(const void* x) { return (reinterpret_cast<uintptr_t>(x) & 15) == 0; }

// s[i][j] = sum_c a[ty + 16 i][c] b[tx + 16 j][c]
template <int PITCH>
__device__ __forceinline__ void product_nt(float (&s)[RI][4], const float* a, const float* b, int width, int ty, int tx) {
#pragma unroll
  for (int i = 0; i < RI; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j) s[i][j] = 0.f;
#pragma unroll 4
  for (int c = 0; c < width; c += 4) {
    float4 x[RI], y[4];
#pragma unroll
    for (int i = 0; i < RI; ++i) x[i] = *reinterpret_cast<const float4*>(a + (ty + 16 * i) * PITCH + c);
#pragma unroll
    for (int j = 0; j < 4; ++j) y[j] = *reinterpret_cast<const float4*>(b + (tx + 16 * j) * PITCH + c);
#pragma unroll
    for (int i = 0; i < RI; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        s[i][j] = fmaf(x[i].x, y[j].x, s[i][j]);
        s[i][j] = fmaf(x[i].y, y[j].y, s[i][j]);
        s[i][j] = fmaf(x[i].z, y[j].z, s[i][j]);
        s[i][j] = fmaf(x[i].w, y[j].w, s[i][j]);
      }
  }
}

// Column pairs of a thread: 2 tx and 2 tx + 1 of every 32.
__device__ __forceinline__ int column(int c, int tx) { return 32 * (c >> 1) + 2 * tx + (c & 1); }

// sum[i][c] += sum_k w[ty + 16 i][k] x[k][column(c)], k = 0 .. 63
template <int NC, int PITCH>
__device__ __forceinline__ void product_nn(float (&sum)[RI][NC], const float* w, const float* x, int ty, int tx) {
  float part[RI][NC];
#pragma unroll
  for (int i = 0; i < RI; ++i)
#pragma unroll
    for (int c = 0; c < NC; ++c) part[i][c] = 0.f;
#pragma unroll 4
  for (int k = 0; k < kWalk; k += 4) {
    float4 a[RI];
#pragma unroll
    for (int i = 0; i < RI; ++i) a[i] = *reinterpret_cast<const float4*>(w + (ty + 16 * i) * kPitchP + k);
#pragma unroll
    for (int c = 0; c < NC; c += 2) {
      const float* at = x + k * PITCH + column(c, tx);         // (columns past the width hold anything and are not stored)
      const float2 x0 = *reinterpret_cast<const float2*>(at), x1 = *reinterpret_cast<const float2*>(at + PITCH);
      const float2 x2 = *reinterpret_cast<const float2*>(at + 2 * PITCH), x3 = *reinterpret_cast<const float2*>(at + 3 * PITCH);
#pragma unroll
      for (int i = 0; i < RI; ++i) {
        part[i][c] = fmaf(a[i].w, x3.x, fmaf(a[i].z, x2.x, fmaf(a[i].y, x1.x, fmaf(a[i].x, x0.x, part[i][c]))));
        part[i][c + 1] = fmaf(a[i].w, x3.y, fmaf(a[i].z, x2.y, fmaf(a[i].y, x1.y, fmaf(a[i].x, x0.y, part[i][c + 1]))));
      }
    }
  }
#pragma unroll
  for (int i = 0; i < RI; ++i)
#pragma unroll
    for (int c = 0; c < NC; ++c) sum[i][c] += part[i][c];
}

// Bias in the base-2 domain (ALiBi's slope or the table's entry) of the kOwn + kWalk - 1 distances of a pair of tiles, from
// `first` on; -infinity where the key comes after the query.
__device__ __forceinline__ void fetch_bias(float* dst, const TrainParams& p, const HeadInfo& hd, int h, int first, int tid) {
  const int x = first + tid;
  if (tid < kOwn + kWalk)
    dst[tid] = x < 0 ? -INFINITY
               : p.bias != nullptr ? __ldg(p.bias + static_cast<int64_t>(h) * p.bias_len + min(x, p.bias_len - 1))
                                   : -hd.alibi_slope2 * static_cast<float>(x);
}
// 2^(s scale + bias - m).  The maximum comes off inside the multiply-add: what is rounded is the difference, which is small
// where the weight counts.
__device__ __forceinline__ float weight(float s, float scale, float bias, float m) { return ex2(fmaf(s, scale, -m) + bias); }
__device__ __forceinline__ int tokens_of(const TrainParams& p, int b) {
  return p.lens_in != nullptr ? min(max(__ldg(p.lens_in + b), 0), p.T) : p.T;
}

struct Unit { int h, i, b; };
__device__ __forceinline__ Unit query_unit(const TrainParams& p, int u) {
  Unit x;
  const int hq = u / p.B;
  x.b = u - hq * p.B;
  x.h = hq / p.group;
  x.i = hq - x.h * p.group;
  return x;
}
// element of the packed rows where head h, query head i, token t of sequence b starts
__device__ __forceinline__ int64_t q_at(const TrainParams& p, const HeadInfo& hd, const Unit& u, int t) {
  return (static_cast<int64_t>(u.b) * p.T + t) * (static_cast<int64_t>(p.group) * p.lr_k_width) + p.group * hd.lr_k_off + u.i * hd.rp_k;
}
__device__ __forceinline__ int64_t o_at(const TrainParams& p, const HeadInfo& hd, const Unit& u, int t) {
  return (static_cast<int64_t>(u.b) * p.T + t) * (static_cast<int64_t>(p.group) * p.lr_v_width) + p.group * hd.lr_v_off + u.i * hd.rp_v;
}
__device__ __forceinline__ int64_t k_at(const TrainParams& p, const HeadInfo& hd, int b, int t) {
  return (static_cast<int64_t>(b) * p.T + t) * p.lr_k_width + hd.lr_k_off;
}
__device__ __forceinline__ int64_t v_at(const TrainParams& p, const HeadInfo& hd, int b, int t) {
  return (static_cast<int64_t>(b) * p.T + t) * p.lr_v_width + hd.lr_v_off;
}

template <int NC>
__global__ void __launch_bounds__(kThreads, 2) train_simt_forward_kernel(const TrainParams p) {
  extern __shared__ __align__(16) float sm[];
  __shared__ float bias_of[2][kOwn + kWalk];
  const Unit u = query_unit(p, blockIdx.x);
  const HeadInfo hd = p.heads[u.h];
  const int tile = gridDim.y - 1 - blockIdx.y, i0 = tile * kOwn;         // long rows first
  const int tid = threadIdx.x, ty = tid >> 4, tx = tid & 15;
  const int rk = hd.rp_k, rv = hd.rp_v, n = tokens_of(p, u.b), rows = max(0, min(kOwn, n - i0)), end = rows > 0 ? i0 + rows : 0;
  if (blockIdx.x == 0 && blockIdx.y == 0)
    for (int b = tid; b < p.B; b += kThreads) p.lens[b] = tokens_of(p, b);
  constexpr int kTile = kWalk * kPitch<NC>, kOwnTile = kOwn * kPitch<NC>;
  float* Qs = sm;
  float* Ks = Qs + kOwnTile;
  float* Vs = Ks + 2 * kTile;
  float* Ps = Vs + 2 * kTile;
  const int64_t q_stride = static_cast<int64_t>(p.group) * p.lr_k_width;
  const float *q = static_cast<const float*>(p.q), *k = static_cast<const float*>(p.k), *v = static_cast<const float*>(p.v);
  const bool wide_k = on16(k), wide_v = on16(v);
  auto fetch = [&](int j0) {
    const int buf = (j0 / kWalk) & 1;
    fetch_rows<kWalk, kPitch<NC>>(Ks + buf * kTile, k + k_at(p, hd, u.b, j0), p.lr_k_width, n - j0, rk, hd.r_k, wide_k, tid);
    fetch_rows<kWalk, kPitch<NC>>(Vs + buf * kTile, v + v_at(p, hd, u.b, j0), p.lr_v_width, n - j0, rv, hd.r_v, wide_v, tid);
    fetch_bias(bias_of[buf], p, hd, u.h, i0 - j0 - (kWalk - 1), tid);
  };
  if (rows > 0) {
    fetch_rows<kOwn, kPitch<NC>>(Qs, q + q_at(p, hd, u, i0), q_stride, rows, rk, hd.r_k, on16(q), tid);
    if (u.i == 0) {                                          // one query head of the group keeps the keys and values
      fetch_rows<kOwn, kPitch<NC>>(Ks + kTile, k + k_at(p, hd, u.b, i0), p.lr_k_width, rows, rk, hd.r_k, wide_k, tid);
      fetch_rows<kOwn, kPitch<NC>>(Vs + kTile, v + v_at(p, hd, u.b, i0), p.lr_v_width, rows, rv, hd.r_v, wide_v, tid);
    }
    fetch(0);
    tc::cp_async_commit();
    tc::cp_async_wait<0>();
    __syncthreads();
    keep_rows<kPitch<NC>>(p.q_copy + q_at(p, hd, u, i0), Qs, q_stride, rows, rk, tid);
    if (u.i == 0) {
      keep_rows<kPitch<NC>>(p.k_copy + k_at(p, hd, u.b, i0), Ks + kTile, p.lr_k_width, rows, rk, tid);
      keep_rows<kPitch<NC>>(p.v_copy + v_at(p, hd, u.b, i0), Vs + kTile, p.lr_v_width, rows, rv, tid);
    }
  }
  float m[RI], l[RI], o[RI][NC];
#pragma unroll
  for (int i = 0; i < RI; ++i) {
    m[i] = -INFINITY;
    l[i] = 0.f;
#pragma unroll
    for (int c = 0; c < NC; ++c) o[i][c] = 0.f;
  }
  for (int j0 = 0; j0 < end; j0 += kWalk) {
    const int buf = (j0 / kWalk) & 1;
    tc::cp_async_wait<0>();
    __syncthreads();                                         // this tile is there, the one before is done with
    if (j0 + kWalk < end) fetch(j0 + kWalk);
    tc::cp_async_commit();
    float s[RI][4];
    product_nt<kPitch<NC>>(s, Qs, Ks + buf * kTile, rk, ty, tx);
#pragma unroll
    for (int i = 0; i < RI; ++i) {
      float top = m[i], bias[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        bias[j] = bias_of[buf][ty + 16 * i - tx - 16 * j + kWalk - 1];
        if (bias[j] != -INFINITY) top = fmaxf(top, fmaf(s[i][j], p.scale_log2, bias[j]));
        else s[i][j] = 0.f;
      }
#pragma unroll
      for (int d = 8; d >= 1; d >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, d));
      const float keep = top == -INFINITY ? 1.f : ex2(m[i] - top);
      float sum = 0.f;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const float e = top == -INFINITY ? 0.f : weight(s[i][j], p.scale_log2, bias[j], top);
        sum += e;
        Ps[(ty + 16 * i) * kPitchP + tx + 16 * j] = e;
      }
#pragma unroll
      for (int d = 8; d >= 1; d >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
      l[i] = fmaf(l[i], keep, sum);
      m[i] = top;
#pragma unroll
      for (int c = 0; c < NC; ++c) o[i][c] *= keep;
    }
    __syncwarp();                                            // (a warp reads the rows that it wrote)
    product_nn<NC, kPitch<NC>>(o, Ps, Vs + buf * kTile, ty, tx);
  }
  float* out = static_cast<float*>(p.out);
  const int64_t stat = static_cast<int64_t>(blockIdx.x) * p.pad, all = static_cast<int64_t>(gridDim.x) * p.pad;
#pragma unroll
  for (int i = 0; i < RI; ++i) {
    const int row = i0 + ty + 16 * i;
    if (row >= p.T) continue;
    const float inv = row < n ? 1.f / l[i] : 0.f;
    if (tx == 0) {
      p.lse[stat + row] = row < n ? m[i] : INFINITY;
      p.lse[all + stat + row] = inv;
    }
#pragma unroll
    for (int c = 0; c < NC; ++c) {
      const int col = column(c, tx);
      if (col >= rv) continue;
      const float x = row < n ? o[i][c] * inv : 0.f;
      out[o_at(p, hd, u, row) + col] = x;
      p.o[(static_cast<int64_t>(blockIdx.x) * p.T + row) * p.o_stride + col] = x;
    }
  }
}

// P of a score, from the statistics of its row
__device__ __forceinline__ float probability(float s, float scale, float bias, float m, float inv) {
  return bias != -INFINITY ? weight(s, scale, bias, m) * inv : 0.f;
}

// dq' of a tile of query rows; also their delta, and this tile's share of the bias gradient.
template <int NC>
__global__ void __launch_bounds__(kThreads, 1) train_simt_dq_kernel(const TrainParams p) {
  extern __shared__ __align__(16) float sm[];
  __shared__ float stats[3][kOwn];                           // maximum, reciprocal sum, delta
  __shared__ float bias_of[2][kOwn + kWalk], diagonal[kOwn + kWalk];
  __shared__ double by_bucket[kMaxBuckets];
  __shared__ int starts[kMaxBuckets + 1];
  const Unit u = query_unit(p, blockIdx.x);
  const HeadInfo hd = p.heads[u.h];
  const int tile = gridDim.y - 1 - blockIdx.y, i0 = tile * kOwn;
  const int tid = threadIdx.x, ty = tid >> 4, tx = tid & 15;
  const int rk = hd.rp_k, rv = hd.rp_v, n = kept_tokens(p, u.b), rows = max(0, min(kOwn, n - i0)), end = rows > 0 ? i0 + rows : 0;
  constexpr int kTile = kWalk * kPitch<NC>, kOwnTile = kOwn * kPitch<NC>;
  float* Qs = sm;
  float* Gs = Qs + kOwnTile;
  float* Ks = Gs + kOwnTile;
  float* Vs = Ks + 2 * kTile;
  float* Ps = Vs + 2 * kTile;
  const int64_t stat = static_cast<int64_t>(blockIdx.x) * p.pad, all = static_cast<int64_t>(gridDim.x) * p.pad;
  auto fetch = [&](int j0) {
    const int buf = (j0 / kWalk) & 1;
    fetch_rows<kWalk, kPitch<NC>>(Ks + buf * kTile, p.k_copy + k_at(p, hd, u.b, j0), p.lr_k_width, n - j0, rk, hd.r_k, true, tid);
    fetch_rows<kWalk, kPitch<NC>>(Vs + buf * kTile, p.v_copy + v_at(p, hd, u.b, j0), p.lr_v_width, n - j0, rv, hd.r_v, true, tid);
    fetch_bias(bias_of[buf], p, hd, u.h, i0 - j0 - (kWalk - 1), tid);
  };
  if (rows > 0) {
    fetch_rows<kOwn, kPitch<NC>>(Qs, p.q_copy + q_at(p, hd, u, i0), static_cast<int64_t>(p.group) * p.lr_k_width, rows, rk, hd.r_k, true, tid);
    fetch_rows<kOwn, kPitch<NC>>(Gs, static_cast<const float*>(p.d_out) + o_at(p, hd, u, i0), static_cast<int64_t>(p.group) * p.lr_v_width, rows, rv, hd.r_v,
                     on16(p.d_out), tid);
    fetch(0);
    tc::cp_async_commit();
    tc::cp_async_wait<0>();
  }
  if (p.dtable != nullptr) {
    if (tid < p.buckets) by_bucket[tid] = 0;
    for (int b = tid; b <= p.buckets; b += kThreads) starts[b] = __ldg(p.starts + b);
  }
  __syncthreads();
  {
    const int r = tid >> 3;                                  // eight threads for a row of do' o'
    float sum = 0.f;
    if (r < rows) {
      const float* o = p.o + (static_cast<int64_t>(blockIdx.x) * p.T + i0 + r) * p.o_stride;
      for (int c = tid & 7; c < hd.r_v; c += 8) sum = fmaf(Gs[r * kPitch<NC> + c], o[c], sum);
    }
    sum += __shfl_xor_sync(0xffffffffu, sum, 1);
    sum += __shfl_xor_sync(0xffffffffu, sum, 2);
    sum += __shfl_xor_sync(0xffffffffu, sum, 4);
    if ((tid & 7) == 0) {
      stats[0][r] = r < rows ? p.lse[stat + i0 + r] : INFINITY;
      stats[1][r] = r < rows ? p.lse[all + stat + i0 + r] : 0.f;
      stats[2][r] = sum;
      if (i0 + r < p.T) p.delta[stat + i0 + r] = sum;
    }
  }
  float dq[RI][NC];
#pragma unroll
  for (int i = 0; i < RI; ++i)
#pragma unroll
    for (int c = 0; c < NC; ++c) dq[i][c] = 0.f;
  for (int j0 = 0; j0 < end; j0 += kWalk) {
    const int buf = (j0 / kWalk) & 1;
    tc::cp_async_wait<0>();
    __syncthreads();                                         // this tile is there, the one before is done with
    if (j0 + kWalk < end) fetch(j0 + kWalk);
    tc::cp_async_commit();
    float s[RI][4], g[RI][4];
    product_nt<kPitch<NC>>(s, Qs, Ks + buf * kTile, rk, ty, tx);
    product_nt<kPitch<NC>>(g, Gs, Vs + buf * kTile, rv, ty, tx);
#pragma unroll
    for (int i = 0; i < RI; ++i) {
      const int r = ty + 16 * i;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const float pr = probability(s[i][j], p.scale_log2, bias_of[buf][r - tx - 16 * j + kWalk - 1], stats[0][r], stats[1][r]);
        Ps[r * kPitchP + tx + 16 * j] = pr * (g[i][j] - stats[2][r]);
      }
    }
    __syncwarp();                                            // (a warp reads the rows that it wrote)
    product_nn<NC, kPitch<NC>>(dq, Ps, Ks + buf * kTile, ty, tx);
    if (p.dtable != nullptr) {
      // sums along the diagonals, i.e. over equal distances; then each bucket's distances by a warp, in a fixed order
      __syncthreads();
      if (tid < kOwn + kWalk - 1) {
        float sum = 0.f;
        const int d = tid - (kWalk - 1);                     // row - column
#pragma unroll 4
        for (int r = max(0, d); r < min(kOwn, kWalk + d); ++r) sum += Ps[r * kPitchP + r - d];
        diagonal[tid] = sum;
      }
      __syncthreads();
      const int shift = i0 - j0 - (kWalk - 1), lane = tid & 31;          // distance of diagonal[0]
      for (int b = tid >> 5; b < p.buckets; b += kThreads / 32) {
        const int first = starts[b], behind = starts[b + 1];
        if (first > shift + kOwn + kWalk - 2 || behind <= shift) continue;
        const int from = max(first - shift, 0), to = behind > shift + kOwn + kWalk - 1 ? kOwn + kWalk - 1 : behind - shift;
        double sum = 0;
        for (int d = from + lane; d < to; d += 32) sum += diagonal[d];
#pragma unroll
        for (int x = 16; x >= 1; x >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, x);
        if (lane == 0) by_bucket[b] += sum;
      }
    }
  }
  float* out = static_cast<float*>(p.dq);
#pragma unroll
  for (int i = 0; i < RI; ++i) {
    const int row = i0 + ty + 16 * i;
    if (row >= p.T) continue;
#pragma unroll
    for (int c = 0; c < NC; ++c)
      if (column(c, tx) < rk) out[q_at(p, hd, u, row) + column(c, tx)] = dq[i][c] * p.scale;
  }
  __syncthreads();
  if (p.dtable != nullptr && tid < p.buckets)                // (group 1: a head's units are its sequences)
    p.bias_part[(static_cast<int64_t>(blockIdx.x) * gridDim.y + tile) * p.buckets + tid] = static_cast<float>(by_bucket[tid]);
}

// dk', dv' of a tile of keys: the query rows of every query head of the group.
template <int NC>
__global__ void __launch_bounds__(kThreads, 1) train_simt_dkv_kernel(const TrainParams p) {
  extern __shared__ __align__(16) float sm[];
  __shared__ float stats[2][3][kWalk], bias_of[2][kOwn + kWalk];
  const int h = blockIdx.x / p.B, b = blockIdx.x - h * p.B;
  const HeadInfo hd = p.heads[h];
  const int j0 = blockIdx.y * kOwn;                          // the first keys have the most queries
  const int tid = threadIdx.x, ty = tid >> 4, tx = tid & 15;
  const int rk = hd.rp_k, rv = hd.rp_v, n = kept_tokens(p, b), rows = max(0, min(kOwn, n - j0));
  constexpr int kTile = kWalk * kPitch<NC>, kOwnTile = kOwn * kPitch<NC>;
  float* Ks = sm;
  float* Vs = Ks + kOwnTile;
  float* Qs = Vs + kOwnTile;
  float* Gs = Qs + 2 * kTile;
  float* Ps = Gs + 2 * kTile;
  const int64_t all = static_cast<int64_t>(p.H) * p.group * p.B * p.pad;
  const int per_head = (n - j0 + kWalk - 1) / kWalk, total = rows > 0 ? p.group * per_head : 0;
  const bool wide_g = on16(p.d_out);
  auto fetch = [&](int t) {                                  // tile t of all the group's
    const int buf = t & 1, i = t / per_head, i0 = j0 + (t - i * per_head) * kWalk;
    const Unit u = {h, i, b};
    const int64_t stat = (static_cast<int64_t>(h * p.group + i) * p.B + b) * p.pad;
    fetch_rows<kWalk, kPitch<NC>>(Qs + buf * kTile, p.q_copy + q_at(p, hd, u, i0), static_cast<int64_t>(p.group) * p.lr_k_width, n - i0, rk, hd.r_k, true, tid);
    fetch_rows<kWalk, kPitch<NC>>(Gs + buf * kTile, static_cast<const float*>(p.d_out) + o_at(p, hd, u, i0), static_cast<int64_t>(p.group) * p.lr_v_width, n - i0, rv,
                      hd.r_v, wide_g, tid);
    if (tid < kWalk) {
      const bool there = i0 + tid < n;
      stats[buf][0][tid] = there ? p.lse[stat + i0 + tid] : INFINITY;
      stats[buf][1][tid] = there ? p.lse[all + stat + i0 + tid] : 0.f;
      stats[buf][2][tid] = there ? p.delta[stat + i0 + tid] : 0.f;
    }
    fetch_bias(bias_of[buf], p, hd, h, i0 - j0 - (kOwn - 1), tid);
  };
  float dk[RI][NC], dv[RI][NC];
#pragma unroll
  for (int i = 0; i < RI; ++i)
#pragma unroll
    for (int c = 0; c < NC; ++c) dk[i][c] = dv[i][c] = 0.f;
  if (total > 0) {
    fetch_rows<kOwn, kPitch<NC>>(Ks, p.k_copy + k_at(p, hd, b, j0), p.lr_k_width, rows, rk, hd.r_k, true, tid);
    fetch_rows<kOwn, kPitch<NC>>(Vs, p.v_copy + v_at(p, hd, b, j0), p.lr_v_width, rows, rv, hd.r_v, true, tid);
    fetch(0);
    tc::cp_async_commit();
  }
  for (int t = 0; t < total; ++t) {
    const int buf = t & 1;
    tc::cp_async_wait<0>();
    __syncthreads();                                         // this tile is there, the one before is done with
    if (t + 1 < total) fetch(t + 1);
    tc::cp_async_commit();
    float s[RI][4], g[RI][4];
    product_nt<kPitch<NC>>(s, Ks, Qs + buf * kTile, rk, ty, tx);
#pragma unroll
    for (int a = 0; a < RI; ++a)
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        const int r = tx + 16 * c, key = ty + 16 * a;
        s[a][c] = probability(s[a][c], p.scale_log2, bias_of[buf][r - key + kOwn - 1], stats[buf][0][r], stats[buf][1][r]);
        Ps[key * kPitchP + r] = s[a][c];
      }
    product_nt<kPitch<NC>>(g, Vs, Gs + buf * kTile, rv, ty, tx);
    __syncwarp();                                            // (a warp reads the rows that it wrote)
    product_nn<NC, kPitch<NC>>(dv, Ps, Gs + buf * kTile, ty, tx);
    __syncwarp();
#pragma unroll
    for (int a = 0; a < RI; ++a)
#pragma unroll
      for (int c = 0; c < 4; ++c)
        Ps[(ty + 16 * a) * kPitchP + tx + 16 * c] = s[a][c] * (g[a][c] - stats[buf][2][tx + 16 * c]);
    __syncwarp();
    product_nn<NC, kPitch<NC>>(dk, Ps, Qs + buf * kTile, ty, tx);
  }
  float *out_k = static_cast<float*>(p.dk), *out_v = static_cast<float*>(p.dv);
#pragma unroll
  for (int a = 0; a < RI; ++a) {
    const int key = j0 + ty + 16 * a;
    if (key >= p.T) continue;
#pragma unroll
    for (int c = 0; c < NC; ++c) {
      const int col = column(c, tx);
      if (col < rk) out_k[k_at(p, hd, b, key) + col] = dk[a][c] * p.scale;
      if (col < rv) out_v[v_at(p, hd, b, key) + col] = dv[a][c];
    }
  }
}

constexpr size_t smem_bytes(int pitch, int own) {
  return (static_cast<size_t>(pitch) * (own * kOwn + 4 * kWalk) + kOwn * kPitchP) * sizeof(float);
}

template <int NC>
cudaError_t forward_t(const TrainParams& p, cudaStream_t s) {
  static size_t done[kMaxDevices] = {};
  const size_t smem = smem_bytes(kPitch<NC>, 1);
  const cudaError_t e = ensure_dynamic_smem(train_simt_forward_kernel<NC>, smem, done);
  if (e != cudaSuccess) return e;
  train_simt_forward_kernel<NC><<<dim3(p.H * p.group * p.B, train_simt_tiles(p.T)), kThreads, smem, s>>>(p);
  return cudaGetLastError();
}
template <int NC>
cudaError_t backward_t(const TrainParams& p, cudaStream_t s) {
  static size_t done_q[kMaxDevices] = {}, done_kv[kMaxDevices] = {};
  const size_t smem = smem_bytes(kPitch<NC>, 2);
  cudaError_t e = ensure_dynamic_smem(train_simt_dq_kernel<NC>, smem, done_q);
  if (e == cudaSuccess) e = ensure_dynamic_smem(train_simt_dkv_kernel<NC>, smem, done_kv);
  if (e != cudaSuccess) return e;
  train_simt_dq_kernel<NC><<<dim3(p.H * p.group * p.B, train_simt_tiles(p.T)), kThreads, smem, s>>>(p);
  e = cudaGetLastError();
  if (e != cudaSuccess) return e;
  train_simt_dkv_kernel<NC><<<dim3(p.H * p.B, train_simt_tiles(p.T)), kThreads, smem, s>>>(p);
  return cudaGetLastError();
}

}  // namespace

int train_simt_tiles(int T) { return (T + kOwn - 1) / kOwn; }

// Columns of a thread by the widest rank: 32, 64, 96 or 128 columns over 16 threads (a rank of 40 in the widest instance would
// spend two thirds of its multiply-adds on columns that are not there).
cudaError_t launch_train_simt_forward(const TrainParams& p, cudaStream_t s, uint64_t* launches) {
  ++*launches;
  const int widest = p.max_rp_k > p.max_rp_v ? p.max_rp_k : p.max_rp_v;
  return widest <= 32 ? forward_t<2>(p, s) : widest <= 64 ? forward_t<4>(p, s) : widest <= 96 ? forward_t<6>(p, s) : forward_t<8>(p, s);
}
cudaError_t launch_train_simt_backward(const TrainParams& p, cudaStream_t s, uint64_t* launches) {
  *launches += 2;
  const int widest = p.max_rp_k > p.max_rp_v ? p.max_rp_k : p.max_rp_v;
  return widest <= 32 ? backward_t<2>(p, s) : widest <= 64 ? backward_t<4>(p, s) : widest <= 96 ? backward_t<6>(p, s) : backward_t<8>(p, s);
}

}  // namespace ea
