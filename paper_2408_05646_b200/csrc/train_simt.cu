// Causal attention over rank-space rows and its backward pass on the CUDA cores, for fp32 layers.
//   S_ij = scale q'_i k'_j + b(i - j)  (j <= i < length),  P = softmax(S),  o'_i = sum_j P_ij v'_j
//   delta_i = do'_i o'_i,  dS_ij = P_ij (do'_i v'_j - delta_i),
//   dq'_i = scale sum_j dS_ij k'_j,  dk'_j = scale sum_i dS_ij q'_i,  dv'_j = sum_i P_ij do'_i,  db_u = sum dS_ij over the
//   distances of bucket u
// P is recomputed from the row's maximum and the reciprocal of its sum, which the forward pass leaves: their logarithm, one
// number, would cost the exponent's last bits.  A CTA has a tile of 64 query (or key) rows and walks the other axis in tiles
// of 64; a thread has 4 x 4 scores and 4 rows x 8 columns of the sums.  dq' and dk', dv' are two kernels, so that nothing is
// added up by atomics.  A tile's products are summed apart and then added, which keeps the rounding errors of long sums down.
// Bound by the loads from shared memory (two for eight multiply-adds in the score products): figures in the table of cases.
#include "internal.h"

namespace ea {
namespace {

constexpr int kRows = 64;
constexpr int kThreads = 256;
constexpr int kPitchP = kRows + 4;

__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// rows x width numbers of packed rows into shared memory (pitch = width + 4), zeros behind `rows`; columns from `live` on are
// the rank's padding: zeros, whatever the caller left there.  copy: the same numbers kept for the backward pass.
__device__ __forceinline__ void load_rows(float* dst, const float* src, int64_t stride, int rows, int width, int live, int tid,
                                          float* copy = nullptr) {
  for (int idx = tid; idx < kRows * width; idx += kThreads) {
    const int r = idx / width, c = idx - r * width;
    float x = 0.f;
    if (r < rows) {
      if (c < live) x = src[r * stride + c];
      if (copy != nullptr) copy[r * stride + c] = x;
    }
    dst[r * (width + 4) + c] = x;
  }
}

// s[i][j] = sum_c a[ty + 16 i][c] b[tx + 16 j][c]
__device__ __forceinline__ void product_nt(float (&s)[4][4], const float* a, const float* b, int width, int ty, int tx) {
  const int pitch = width + 4;
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j) s[i][j] = 0.f;
#pragma unroll 2
  for (int c = 0; c < width; c += 4) {
    float4 x[4], y[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = *reinterpret_cast<const float4*>(a + (ty + 16 * i) * pitch + c);
#pragma unroll
    for (int j = 0; j < 4; ++j) y[j] = *reinterpret_cast<const float4*>(b + (tx + 16 * j) * pitch + c);
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        s[i][j] = fmaf(x[i].x, y[j].x, s[i][j]);
        s[i][j] = fmaf(x[i].y, y[j].y, s[i][j]);
        s[i][j] = fmaf(x[i].z, y[j].z, s[i][j]);
        s[i][j] = fmaf(x[i].w, y[j].w, s[i][j]);
      }
  }
}

// sum[i][c] += sum_k w[ty + 16 i][k] x[k][tx + 16 c], k = 0 .. 63
template <int NC>
__device__ __forceinline__ void product_nn(float (&sum)[4][NC], const float* w, const float* x, int width, int ty, int tx) {
  const int pitch = width + 4;
  float part[4][NC];
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int c = 0; c < NC; ++c) part[i][c] = 0.f;
#pragma unroll 2
  for (int k = 0; k < kRows; k += 4) {
    float4 a[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) a[i] = *reinterpret_cast<const float4*>(w + (ty + 16 * i) * kPitchP + k);
#pragma unroll
    for (int c = 0; c < NC; ++c) {
      const int col = min(tx + 16 * c, width - 1);           // (columns past the width repeat the last one and are not stored)
      const float x0 = x[k * pitch + col], x1 = x[(k + 1) * pitch + col];
      const float x2 = x[(k + 2) * pitch + col], x3 = x[(k + 3) * pitch + col];
#pragma unroll
      for (int i = 0; i < 4; ++i)
        part[i][c] = fmaf(a[i].w, x3, fmaf(a[i].z, x2, fmaf(a[i].y, x1, fmaf(a[i].x, x0, part[i][c]))));
    }
  }
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int c = 0; c < NC; ++c) sum[i][c] += part[i][c];
}

// Bias of a distance >= 0 in the base-2 domain: ALiBi's slope or the table's entry.
__device__ __forceinline__ float bias_of(const TrainParams& p, const HeadInfo& hd, int h, int distance) {
  if (p.bias != nullptr) return __ldg(p.bias + static_cast<int64_t>(h) * p.bias_len + min(max(distance, 0), p.bias_len - 1));
  return -hd.alibi_slope2 * static_cast<float>(distance);
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
__global__ void __launch_bounds__(kThreads) train_simt_forward_kernel(const TrainParams p) {
  extern __shared__ __align__(16) float sm[];
  const Unit u = query_unit(p, blockIdx.x);
  const HeadInfo hd = p.heads[u.h];
  const int tile = gridDim.y - 1 - blockIdx.y, i0 = tile * kRows;        // long rows first
  const int tid = threadIdx.x, ty = tid >> 4, tx = tid & 15;
  const int rk = hd.rp_k, rv = hd.rp_v, n = tokens_of(p, u.b);
  if (blockIdx.x == 0 && blockIdx.y == 0)
    for (int b = tid; b < p.B; b += kThreads) p.lens[b] = tokens_of(p, b);
  float* Qs = sm;
  float* Ks = Qs + kRows * (rk + 4);
  float* Vs = Ks + kRows * (rk + 4);
  float* Ps = Vs + kRows * (rv + 4);
  const int64_t q_stride = static_cast<int64_t>(p.group) * p.lr_k_width, o_stride = static_cast<int64_t>(p.group) * p.lr_v_width;
  const float *q = static_cast<const float*>(p.q), *k = static_cast<const float*>(p.k), *v = static_cast<const float*>(p.v);
  load_rows(Qs, q + q_at(p, hd, u, i0), q_stride, max(0, min(kRows, n - i0)), rk, hd.r_k, tid, p.q_copy + q_at(p, hd, u, i0));
  if (u.i == 0) {                                            // one query head of the group keeps the keys and values
    load_rows(Ks, k + k_at(p, hd, u.b, i0), p.lr_k_width, max(0, min(kRows, n - i0)), rk, hd.r_k, tid, p.k_copy + k_at(p, hd, u.b, i0));
    load_rows(Vs, v + v_at(p, hd, u.b, i0), p.lr_v_width, max(0, min(kRows, n - i0)), rv, hd.r_v, tid, p.v_copy + v_at(p, hd, u.b, i0));
  }
  float m[4], l[4], o[4][NC];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    m[i] = -INFINITY;
    l[i] = 0.f;
#pragma unroll
    for (int c = 0; c < NC; ++c) o[i][c] = 0.f;
  }
  for (int j0 = 0; j0 <= i0 && i0 < n; j0 += kRows) {
    __syncthreads();
    load_rows(Ks, k + k_at(p, hd, u.b, j0), p.lr_k_width, min(kRows, n - j0), rk, hd.r_k, tid);
    load_rows(Vs, v + v_at(p, hd, u.b, j0), p.lr_v_width, min(kRows, n - j0), rv, hd.r_v, tid);
    __syncthreads();
    float s[4][4];
    product_nt(s, Qs, Ks, rk, ty, tx);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int row = i0 + ty + 16 * i;
      float top = m[i], bias[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int key = j0 + tx + 16 * j;
        const bool open = row < n && key <= row;
        bias[j] = open ? bias_of(p, hd, u.h, row - key) : -INFINITY;
        if (open) top = fmaxf(top, fmaf(s[i][j], p.scale_log2, bias[j]));
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
    __syncthreads();
    product_nn<NC>(o, Ps, Vs, rv, ty, tx);
  }
  float* out = static_cast<float*>(p.out);
  const int64_t stat = static_cast<int64_t>(blockIdx.x) * p.pad, all = static_cast<int64_t>(gridDim.x) * p.pad;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int row = i0 + ty + 16 * i;
    if (row >= p.T) continue;
    const float inv = row < n ? 1.f / l[i] : 0.f;
    if (tx == 0) {
      p.lse[stat + row] = row < n ? m[i] : INFINITY;
      p.lse[all + stat + row] = inv;
    }
#pragma unroll
    for (int c = 0; c < NC; ++c) {
      const int col = tx + 16 * c;
      if (col >= rv) continue;
      const float x = row < n ? o[i][c] * inv : 0.f;
      out[o_at(p, hd, u, row) + col] = x;
      p.o[(static_cast<int64_t>(blockIdx.x) * p.T + row) * p.o_stride + col] = x;
    }
  }
}

// P (or its transpose) of a score tile, from the statistics of its rows
__device__ __forceinline__ float probability(const TrainParams& p, const HeadInfo& hd, int h, float s, int row, int key, int n,
                                             float m, float inv) {
  return row < n && key <= row ? weight(s, p.scale_log2, bias_of(p, hd, h, row - key), m) * inv : 0.f;
}

// dq' of a tile of query rows; also their delta, and this tile's share of the bias gradient.
template <int NC>
__global__ void __launch_bounds__(kThreads) train_simt_dq_kernel(const TrainParams p) {
  extern __shared__ __align__(16) float sm[];
  __shared__ float stats[3][kRows];                          // maximum, reciprocal sum, delta
  __shared__ float diagonal[2 * kRows];
  const Unit u = query_unit(p, blockIdx.x);
  const HeadInfo hd = p.heads[u.h];
  const int tile = gridDim.y - 1 - blockIdx.y, i0 = tile * kRows;
  const int tid = threadIdx.x, ty = tid >> 4, tx = tid & 15;
  const int rk = hd.rp_k, rv = hd.rp_v, n = __ldg(p.lens + u.b), rows = max(0, min(kRows, n - i0));
  float* Qs = sm;
  float* Gs = Qs + kRows * (rk + 4);
  float* Ks = Gs + kRows * (rv + 4);
  float* Vs = Ks + kRows * (rk + 4);
  float* Ps = Vs + kRows * (rv + 4);
  const int64_t stat = static_cast<int64_t>(blockIdx.x) * p.pad, all = static_cast<int64_t>(gridDim.x) * p.pad;
  load_rows(Qs, p.q_copy + q_at(p, hd, u, i0), static_cast<int64_t>(p.group) * p.lr_k_width, rows, rk, hd.r_k, tid);
  load_rows(Gs, static_cast<const float*>(p.d_out) + o_at(p, hd, u, i0), static_cast<int64_t>(p.group) * p.lr_v_width, rows, rv, hd.r_v, tid);
  __syncthreads();
  for (int r = tid >> 2; r < kRows; r += kThreads / 4) {     // four threads for a row of do' o'
    float sum = 0.f;
    if (r < rows) {
      const float* o = p.o + (static_cast<int64_t>(blockIdx.x) * p.T + i0 + r) * p.o_stride;
      for (int c = tid & 3; c < hd.r_v; c += 4) sum = fmaf(Gs[r * (rv + 4) + c], o[c], sum);
    }
    sum += __shfl_xor_sync(0xffffffffu, sum, 1);
    sum += __shfl_xor_sync(0xffffffffu, sum, 2);
    if ((tid & 3) == 0) {
      stats[0][r] = r < rows ? p.lse[stat + i0 + r] : INFINITY;
      stats[1][r] = r < rows ? p.lse[all + stat + i0 + r] : 0.f;
      stats[2][r] = sum;
      if (i0 + r < p.T) p.delta[stat + i0 + r] = sum;
    }
  }
  float dq[4][NC];
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int c = 0; c < NC; ++c) dq[i][c] = 0.f;
  double by_bucket = 0;                                      // thread u < buckets: bucket u
  for (int j0 = 0; j0 <= i0 && i0 < n; j0 += kRows) {
    __syncthreads();
    load_rows(Ks, p.k_copy + k_at(p, hd, u.b, j0), p.lr_k_width, min(kRows, n - j0), rk, hd.r_k, tid);
    load_rows(Vs, p.v_copy + v_at(p, hd, u.b, j0), p.lr_v_width, min(kRows, n - j0), rv, hd.r_v, tid);
    __syncthreads();
    float s[4][4], g[4][4];
    product_nt(s, Qs, Ks, rk, ty, tx);
    product_nt(g, Gs, Vs, rv, ty, tx);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int r = ty + 16 * i;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const float pr = probability(p, hd, u.h, s[i][j], i0 + r, j0 + tx + 16 * j, n, stats[0][r], stats[1][r]);
        Ps[r * kPitchP + tx + 16 * j] = pr * (g[i][j] - stats[2][r]);
      }
    }
    __syncthreads();
    product_nn<NC>(dq, Ps, Ks, rk, ty, tx);
    if (p.dtable != nullptr) {
      // sums along the diagonals, i.e. over equal distances; then each bucket's distances, in their order
      if (tid < 2 * kRows - 1) {
        float sum = 0.f;
        const int d = tid - (kRows - 1);                     // row - column
        for (int r = max(0, d); r < min(kRows, kRows + d); ++r) sum += Ps[r * kPitchP + r - d];
        diagonal[tid] = sum;
      }
      __syncthreads();
      if (tid < p.buckets) {
        const int shift = i0 - j0 - (kRows - 1);             // distance of diagonal[0]
        const int64_t from = static_cast<int64_t>(__ldg(p.starts + tid)) - shift, to = static_cast<int64_t>(__ldg(p.starts + tid + 1)) - shift;
        for (int d = static_cast<int>(max(static_cast<long long>(from), 0ll)); d < min(static_cast<long long>(to), 2ll * kRows - 1); ++d)
          by_bucket += diagonal[d];
      }
    }
  }
  float* out = static_cast<float*>(p.dq);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int row = i0 + ty + 16 * i;
    if (row >= p.T) continue;
#pragma unroll
    for (int c = 0; c < NC; ++c)
      if (tx + 16 * c < rk) out[q_at(p, hd, u, row) + tx + 16 * c] = dq[i][c] * p.scale;
  }
  if (p.dtable != nullptr && tid < p.buckets)                // (group 1: a head's units are its sequences)
    p.bias_part[(static_cast<int64_t>(blockIdx.x) * gridDim.y + tile) * p.buckets + tid] = static_cast<float>(by_bucket);
}

// dk', dv' of a tile of keys: the query rows of every query head of the group.
template <int NC>
__global__ void __launch_bounds__(kThreads) train_simt_dkv_kernel(const TrainParams p) {
  extern __shared__ __align__(16) float sm[];
  __shared__ float stats[3][kRows];
  const int h = blockIdx.x / p.B, b = blockIdx.x - h * p.B;
  const HeadInfo hd = p.heads[h];
  const int j0 = blockIdx.y * kRows;                         // the first keys have the most queries
  const int tid = threadIdx.x, ty = tid >> 4, tx = tid & 15;
  const int rk = hd.rp_k, rv = hd.rp_v, n = __ldg(p.lens + b);
  float* Ks = sm;
  float* Vs = Ks + kRows * (rk + 4);
  float* Qs = Vs + kRows * (rv + 4);
  float* Gs = Qs + kRows * (rk + 4);
  float* Ps = Gs + kRows * (rv + 4);
  load_rows(Ks, p.k_copy + k_at(p, hd, b, j0), p.lr_k_width, max(0, min(kRows, n - j0)), rk, hd.r_k, tid);
  load_rows(Vs, p.v_copy + v_at(p, hd, b, j0), p.lr_v_width, max(0, min(kRows, n - j0)), rv, hd.r_v, tid);
  float dk[4][NC], dv[4][NC];
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int c = 0; c < NC; ++c) dk[i][c] = dv[i][c] = 0.f;
  const int64_t all = static_cast<int64_t>(p.H) * p.group * p.B * p.pad;
  for (int i = 0; i < p.group; ++i) {
    const Unit u = {h, i, b};
    const int64_t stat = (static_cast<int64_t>(h * p.group + i) * p.B + b) * p.pad;
    for (int i0 = j0; i0 < n; i0 += kRows) {
      const int rows = min(kRows, n - i0);
      __syncthreads();
      load_rows(Qs, p.q_copy + q_at(p, hd, u, i0), static_cast<int64_t>(p.group) * p.lr_k_width, rows, rk, hd.r_k, tid);
      load_rows(Gs, static_cast<const float*>(p.d_out) + o_at(p, hd, u, i0), static_cast<int64_t>(p.group) * p.lr_v_width, rows, rv, hd.r_v, tid);
      if (tid < kRows) {
        stats[0][tid] = tid < rows ? p.lse[stat + i0 + tid] : INFINITY;
        stats[1][tid] = tid < rows ? p.lse[all + stat + i0 + tid] : 0.f;
        stats[2][tid] = tid < rows ? p.delta[stat + i0 + tid] : 0.f;
      }
      __syncthreads();
      float s[4][4], g[4][4];
      product_nt(s, Ks, Qs, rk, ty, tx);
#pragma unroll
      for (int a = 0; a < 4; ++a)
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          const int r = tx + 16 * c;
          s[a][c] = probability(p, hd, h, s[a][c], i0 + r, j0 + ty + 16 * a, n, stats[0][r], stats[1][r]);
          Ps[(ty + 16 * a) * kPitchP + r] = s[a][c];
        }
      product_nt(g, Vs, Gs, rv, ty, tx);
      __syncthreads();
      product_nn<NC>(dv, Ps, Gs, rv, ty, tx);
      __syncthreads();
#pragma unroll
      for (int a = 0; a < 4; ++a)
#pragma unroll
        for (int c = 0; c < 4; ++c)
          Ps[(ty + 16 * a) * kPitchP + tx + 16 * c] = s[a][c] * (g[a][c] - stats[2][tx + 16 * c]);
      __syncthreads();
      product_nn<NC>(dk, Ps, Qs, rk, ty, tx);
    }
  }
  float *out_k = static_cast<float*>(p.dk), *out_v = static_cast<float*>(p.dv);
#pragma unroll
  for (int a = 0; a < 4; ++a) {
    const int key = j0 + ty + 16 * a;
    if (key >= p.T) continue;
#pragma unroll
    for (int c = 0; c < NC; ++c) {
      const int col = tx + 16 * c;
      if (col < rk) out_k[k_at(p, hd, b, key) + col] = dk[a][c] * p.scale;
      if (col < rv) out_v[v_at(p, hd, b, key) + col] = dv[a][c];
    }
  }
}

size_t smem_bytes(const TrainParams& p, int key_tiles, int value_tiles) {
  return (static_cast<size_t>(kRows) * (key_tiles * (p.max_rp_k + 4) + value_tiles * (p.max_rp_v + 4)) + kRows * kPitchP) * sizeof(float);
}

template <int NC>
cudaError_t forward_t(const TrainParams& p, cudaStream_t s) {
  static size_t done[kMaxDevices] = {};
  const size_t smem = smem_bytes(p, 2, 1);
  const cudaError_t e = ensure_dynamic_smem(train_simt_forward_kernel<NC>, smem, done);
  if (e != cudaSuccess) return e;
  train_simt_forward_kernel<NC><<<dim3(p.H * p.group * p.B, train_simt_tiles(p.T)), kThreads, smem, s>>>(p);
  return cudaGetLastError();
}
template <int NC>
cudaError_t backward_t(const TrainParams& p, cudaStream_t s) {
  static size_t done_q[kMaxDevices] = {}, done_kv[kMaxDevices] = {};
  const size_t smem = smem_bytes(p, 2, 2);
  cudaError_t e = ensure_dynamic_smem(train_simt_dq_kernel<NC>, smem, done_q);
  if (e == cudaSuccess) e = ensure_dynamic_smem(train_simt_dkv_kernel<NC>, smem, done_kv);
  if (e != cudaSuccess) return e;
  train_simt_dq_kernel<NC><<<dim3(p.H * p.group * p.B, train_simt_tiles(p.T)), kThreads, smem, s>>>(p);
  train_simt_dkv_kernel<NC><<<dim3(p.H * p.B, train_simt_tiles(p.T)), kThreads, smem, s>>>(p);
  return cudaGetLastError();
}

}  // namespace

int train_simt_tiles(int T) { return (T + kRows - 1) / kRows; }

// Columns of a thread by the widest rank: 32, 64 or 128 columns over 16 threads (a rank of 40 in the widest instance would
// spend three quarters of its multiply-adds on columns that are not there).
cudaError_t launch_train_simt_forward(const TrainParams& p, cudaStream_t s, uint64_t* launches) {
  ++*launches;
  const int widest = p.max_rp_k > p.max_rp_v ? p.max_rp_k : p.max_rp_v;
  return widest <= 32 ? forward_t<2>(p, s) : widest <= 64 ? forward_t<4>(p, s) : forward_t<8>(p, s);
}
cudaError_t launch_train_simt_backward(const TrainParams& p, cudaStream_t s, uint64_t* launches) {
  *launches += 2;
  const int widest = p.max_rp_k > p.max_rp_v ? p.max_rp_k : p.max_rp_v;
  return widest <= 32 ? backward_t<2>(p, s) : widest <= 64 ? backward_t<4>(p, s) : backward_t<8>(p, s);
}

}  // namespace ea
