// Rows of a training call as operand tiles of the tensor-core kernels (16-bit layers).
// A tile is 128 rows of one (head, sequence) in the core-matrix order of the products: 16-byte chunk (row, c) at (row / 8) *
// group + 128 c + 16 (row % 8).  One order serves a product that contracts over the rank and one that contracts over the rows,
// so a tile is one contiguous copy into shared memory.  The numbers become fp16: P and dS, which the products take from
// registers, keep 11 significant bits instead of bf16's 8 that way (both operands of a product have one type; with bf16 their
// rounding alone would be as large as that of the output).  bf16 values have 8 bits and fit; what fp16 lacks is range.  Every
// tile is therefore multiplied by the power of two that brings its largest number into [2^7, 2^8): a number keeps all its
// bits down to 2^-22 of the tile's largest, and what is below is off by at most 2^-32 of it (half of fp16's last step is 2^-25, the
// largest at least 2^7; powers end at 2^119).  The consumers take the powers out of the scales that they multiply by anyway.
// (Numbers that are not finite take no part in the choice and stay what they are.)
// The gradient's tiles also get delta = do' o' here, the dot product of a row with the o' that the forward pass kept in 32 bits
// (from the rounded output it would be off by a rounding of o', once per row and the same for all its keys).
// Bound by bytes: rows in, tiles out (4 x 4096 tokens, 32 heads, rank 80: q', k', v' 503 MB in 109 us, do' and o' 336 MB in 74,
// 4.6 TB/s).
#include <cuda_bf16.h>

#include "internal.h"
#include "tc_common.cuh"

namespace ea {
namespace {

using namespace tc;

constexpr int kPackThreads = 256;

__device__ __forceinline__ float2 pair_of(uint32_t w) {
  return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u));
}
// largest finite magnitude (bf16 bits) of a pair against m
__device__ __forceinline__ uint32_t take_max(uint32_t m, uint32_t w) {
  const uint32_t a = w & 0x7fffu, b = (w >> 16) & 0x7fffu;
  if (a < 0x7f80u) m = max(m, a);
  if (b < 0x7f80u) m = max(m, b);
  return m;
}

// GRAD: do' (with delta); otherwise q', k' and v' of the call, units of all three one after the other.
template <bool GRAD>
__global__ void __launch_bounds__(kPackThreads) train_pack_kernel(const TrainParams p, int aligned) {
  __shared__ uint32_t tops[kPackThreads / 32];
  chain_go();
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  if (blockIdx.x == 0 && tid == 0) p.next[GRAD ? 1 : 0] = 0;
  const int tile = blockIdx.x % p.tiles;
  int unit = blockIdx.x / p.tiles;
  const int q_units = p.H * p.group * p.B, units = p.H * p.B;
  int which = GRAD ? 3 : 0;                                  // 0: q', 1: k', 2: v', 3: do'
  if (!GRAD && unit >= q_units) {
    unit -= q_units;
    which = unit < units ? 1 : 2;
    if (which == 2) unit -= units;
  }
  const bool shared_head = which == 1 || which == 2, key_side = which == 0 || which == 1;
  const int hq = unit / p.B, b = unit - hq * p.B, group = shared_head ? 1 : p.group;
  const int h = hq / group, i = hq - h * group;
  const HeadInfo hd = p.heads[h];
  const int r = key_side ? hd.r_k : hd.r_v, rp = key_side ? hd.rp_k : hd.rp_v, nch = ((rp + 15) & ~15) >> 3;
  const int64_t width = static_cast<int64_t>(group) * (key_side ? p.lr_k_width : p.lr_v_width);
  const __nv_bfloat16* src = static_cast<const __nv_bfloat16*>(which == 0 ? p.q : which == 1 ? p.k : which == 2 ? p.v : p.d_out) +
                             static_cast<int64_t>(b) * p.T * width + group * (key_side ? hd.lr_k_off : hd.lr_v_off) + i * rp;
  int n;
  if (GRAD) {
    n = kept_tokens(p, b);
  } else {
    n = p.lens_in != nullptr ? min(max(__ldg(p.lens_in + b), 0), p.T) : p.T;
    if (blockIdx.x == 0)                                     // the lengths, kept for the launches behind
      for (int x = tid; x < p.B; x += kPackThreads)
        p.lens[x] = p.lens_in != nullptr ? min(max(__ldg(p.lens_in + x), 0), p.T) : p.T;
  }
  const int64_t at = static_cast<int64_t>(unit) * p.tiles + tile;
  int32_t* e_of = which == 0 ? p.q_exp : which == 1 ? p.k_exp : which == 2 ? p.v_exp : p.g_exp;
  if (tile * kTile >= n) {                                   // behind the text: nobody takes the tile
    if (tid == 0) e_of[at] = kTrainNoNumber;
    return;
  }
  const bool wide = (aligned >> which) & 1;                  // rows start on 16-byte boundaries

  // A warp has the row groups `warp` and `warp + 8`; an instruction takes 8 rows x 4 chunks, so that both the rows' reads and
  // the tile's writes are whole sectors.
  const int r8 = lane & 7, c4 = lane >> 3;
  uint4 x[2][4];
  uint32_t top = 0;
#pragma unroll
  for (int g = 0; g < 2; ++g) {
    const int row = (warp + 8 * g) * 8 + r8, t = tile * kTile + row;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const int c = 4 * k + c4;
      uint4 w = make_uint4(0u, 0u, 0u, 0u);
      if (t < n && c * 8 < rp) {
        const __nv_bfloat16* at = src + t * width + c * 8;
        if (wide) {
          w = __ldg(reinterpret_cast<const uint4*>(at));
        } else {
          const unsigned short* v = reinterpret_cast<const unsigned short*>(at);
          w.x = __ldg(v) | static_cast<uint32_t>(__ldg(v + 1)) << 16;
          w.y = __ldg(v + 2) | static_cast<uint32_t>(__ldg(v + 3)) << 16;
          w.z = __ldg(v + 4) | static_cast<uint32_t>(__ldg(v + 5)) << 16;
          w.w = __ldg(v + 6) | static_cast<uint32_t>(__ldg(v + 7)) << 16;
        }
        if (c * 8 + 8 > r) {                                 // padding columns of the rank
          uint32_t* e = reinterpret_cast<uint32_t*>(&w);
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            if (c * 8 + 2 * j + 1 >= r) e[j] &= 0xffffu;
            if (c * 8 + 2 * j >= r) e[j] = 0u;
          }
        }
      }
      x[g][k] = w;
      top = take_max(take_max(take_max(take_max(top, w.x), w.y), w.z), w.w);
    }
  }
  top = __reduce_max_sync(0xffffffffu, top);
  if (lane == 0) tops[warp] = top;
  __syncthreads();
  top = __reduce_max_sync(0xffffffffu, tops[lane & (kPackThreads / 32 - 1)]);
  const int e = top == 0 ? kTrainNoNumber : min(7 - (max(static_cast<int>(top >> 7), 1) - 127), kTrainNoNumber - 1);
  const float scale = __int_as_float((e + 127) << 23);
  if (tid == 0) e_of[at] = e;
  char* dst = (which == 0 ? p.q_tiles : which == 1 ? p.k_tiles : which == 2 ? p.v_tiles : p.g_tiles) + at * (key_side ? p.tile_k : p.tile_v);
#pragma unroll
  for (int g = 0; g < 2; ++g) {
    const int row = (warp + 8 * g) * 8 + r8, t = tile * kTile + row;
    float sum = 0.f;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const int c = 4 * k + c4;
      if (c >= nch) continue;
      const float2 a = pair_of(x[g][k].x), bb = pair_of(x[g][k].y), cc = pair_of(x[g][k].z), dd = pair_of(x[g][k].w);
      if (GRAD && t < n && c * 8 < rp) {
        const float4* o = reinterpret_cast<const float4*>(p.o + (static_cast<int64_t>(unit) * p.T + t) * p.o_stride + c * 8);
        const float4 o0 = __ldg(o), o1 = __ldg(o + 1);
        sum = fmaf(a.x, o0.x, fmaf(a.y, o0.y, fmaf(bb.x, o0.z, fmaf(bb.y, o0.w, sum))));
        sum = fmaf(cc.x, o1.x, fmaf(cc.y, o1.y, fmaf(dd.x, o1.z, fmaf(dd.y, o1.w, sum))));
      }
      uint4 w;
      w.x = pack_f16(a.x * scale, a.y * scale);
      w.y = pack_f16(bb.x * scale, bb.y * scale);
      w.z = pack_f16(cc.x * scale, cc.y * scale);
      w.w = pack_f16(dd.x * scale, dd.y * scale);
      *reinterpret_cast<uint4*>(dst + chunk_off(row, c, nch << 7)) = w;
    }
    if (GRAD) {
      sum += __shfl_xor_sync(0xffffffffu, sum, 8);
      sum += __shfl_xor_sync(0xffffffffu, sum, 16);
      if (c4 == 0) p.delta[static_cast<int64_t>(unit) * p.pad + t] = sum;
    }
  }
}

}  // namespace

cudaError_t launch_train_pack(const TrainParams& p, bool gradient, cudaStream_t s, uint64_t* launches) {
  auto bit = [](const void* x, int k) { return reinterpret_cast<uintptr_t>(x) % 16 == 0 ? 1 << k : 0; };
  const int64_t units = static_cast<int64_t>(p.H) * p.B;
  if (gradient) {
    train_pack_kernel<true><<<static_cast<unsigned>(units * p.group * p.tiles), kPackThreads, 0, s>>>(p, bit(p.d_out, 3));
  } else {
    train_pack_kernel<false><<<static_cast<unsigned>(units * (p.group + 2) * p.tiles), kPackThreads, 0, s>>>(
        p, bit(p.q, 0) | bit(p.k, 1) | bit(p.v, 2));
  }
  ++*launches;
  return cudaGetLastError();
}

}  // namespace ea
