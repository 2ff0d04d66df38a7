// Causal attention over rank-space rows and its backward pass on the fifth-generation tensor cores (16-bit layers): tcgen05
// products of fp16 tiles (see train_pack.cu), accumulators in TMEM.
//   S_ij = scale q'_i k'_j + b(i - j)  (j <= i < length),  P = softmax(S),  o'_i = sum_j P_ij v'_j
//   delta_i = do'_i o'_i,  dS_ij = P_ij (do'_i v'_j - delta_i),
//   dq'_i = scale sum_j dS_ij k'_j,  dk'_j = scale sum_i dS_ij q'_i,  dv'_j = sum_i P_ij do'_i
// Scores are kept in the base-2 domain.  The forward pass leaves L_i = log2 sum_j 2^S_ij per row; the backward pass recomputes
// P_ij = 2^(S_ij - L_i) from one product, without a maximum or a sum.
//
// A tile is 128 rows.  Every CTA is one thread that copies tiles (one bulk copy each, into a ring), one warp that issues the
// products, and eight softmax warps; one CTA per SM, whose 512 TMEM columns it takes.  P and dS go back to TMEM in the place of
// the scores they came from, as the A operand of the next product, and never touch shared memory.  The backward pass is two
// kernels, one that owns a tile of keys (dk', dv': four products per pair of tiles) and one that owns a tile of queries (dq':
// three, S and do' v' a second time): the alternative, dq' added up in memory by every tile of keys, moves 512 r bytes of
// fp32 additions per pair of tiles through L2 and leaves sums whose order changes from run to run.
//
// Tiles carry a power of two each (2^e).  What is accumulated over tiles needs one scale: the tile's deviation from the
// smallest exponent of all goes into the factors that P and dS are formed with, where it costs nothing.
// Every wait is bounded; one that runs out ends every other one of the launch through the status word.
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "internal.h"
#include "tc_common.cuh"

namespace ea {
namespace {

using namespace tc;

constexpr int kNone = 0, kAlibi = 1, kTable = 2;             // position bias
constexpr int kSoftmaxWarps = 8, kCopyWarp = 8, kIssueWarp = 9;
constexpr int kTrThreads = 10 * 32;
constexpr int kMaxRing = 8;
constexpr int kHeaderBytes = 1024;
constexpr int kForwardShift = 7;          // P of the forward pass times 2^7: its reference lags behind the maximum by up to 2^8
constexpr int kBackwardShift = 14;        // P of the backward pass, at most 1, times 2^14: fp16 keeps all bits down to 2^-28

struct __align__(16) TrHeader {
  unsigned long long full[kMaxRing], empty[kMaxRing];        // ring of tiles
  unsigned long long own;                                    // the CTA's own tiles
  unsigned long long s_full[2], p_full[2], g_full, g_read, done;
  uint32_t tmem_base;
  int smallest[4];                                           // smallest exponents of q', k', v', do'
};
static_assert(sizeof(TrHeader) <= kHeaderBytes, "header outgrew its area");

__device__ __forceinline__ bool elect_one() {
  uint32_t p;
  asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(p));
  return p != 0;
}
__device__ __forceinline__ bool wait_all(unsigned long long* bar, uint32_t parity, int* status) {
  return __all_sync(0xffffffffu, mbar_wait(bar, parity, status)) != 0;
}
// 2^e; exponents that no pair of ordinary tiles has end at the ends of the range
__device__ __forceinline__ float pow2(int e) { return __int_as_float((min(max(e, -126), 127) + 127) << 23); }
__device__ __forceinline__ void arrive_warp(unsigned long long* bar, int lane) {
  __syncwarp();
  if (lane == 0) mbar_arrive(bar);
}
__device__ __forceinline__ void tmem_ld32(uint32_t taddr, uint32_t (&r)[32]) {
  tmem_ld16(taddr, *reinterpret_cast<uint32_t(*)[16]>(&r[0]));
  tmem_ld16(taddr + 16, *reinterpret_cast<uint32_t(*)[16]>(&r[16]));
}
// tcgen05.wait::ld that the registers of the loads under way depend on
__device__ __forceinline__ void tmem_wait_ld_of(uint32_t (&r)[16]) {
  asm volatile("tcgen05.wait::ld.sync.aligned;"
               : "+r"(r[0]), "+r"(r[1]), "+r"(r[2]), "+r"(r[3]), "+r"(r[4]), "+r"(r[5]), "+r"(r[6]), "+r"(r[7]), "+r"(r[8]), "+r"(r[9]),
                 "+r"(r[10]), "+r"(r[11]), "+r"(r[12]), "+r"(r[13]), "+r"(r[14]), "+r"(r[15])
               :
               : "memory");
}
__device__ __forceinline__ void tmem_wait_ld_of(uint32_t (&r)[32]) {
  tmem_wait_ld_of(*reinterpret_cast<uint32_t(*)[16]>(&r[0]));
  tmem_wait_ld_of(*reinterpret_cast<uint32_t(*)[16]>(&r[16]));
}
constexpr uint32_t kMnMajorB = 1u << 16;

// A product over the rank: D[128][128] = A B^T, both tiles K-major; KS steps of 16 columns.
template <int KS>
__device__ __forceinline__ void issue_rank_steps(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc) {
#pragma unroll
  for (int s = 0; s < KS; ++s) mma_ss(d, a + 16 * s, b + 16 * s, idesc, s > 0);
}
__device__ __forceinline__ void issue_rank(int steps, uint32_t d, uint64_t a, uint64_t b) {
  const uint32_t idesc = instr_desc_f16(kTile);
  switch (steps) {
    case 1: issue_rank_steps<1>(d, a, b, idesc); break;
    case 2: issue_rank_steps<2>(d, a, b, idesc); break;
    case 3: issue_rank_steps<3>(d, a, b, idesc); break;
    case 4: issue_rank_steps<4>(d, a, b, idesc); break;
    case 5: issue_rank_steps<5>(d, a, b, idesc); break;
    case 6: issue_rank_steps<6>(d, a, b, idesc); break;
    case 7: issue_rank_steps<7>(d, a, b, idesc); break;
    default: issue_rank_steps<8>(d, a, b, idesc); break;
  }
}
// A product over 128 rows: D[128][r16] (+)= A B with A (P or dS) in TMEM, its second half `half` columns behind the first,
// and B a tile taken MN-major (`group`: bytes of 8 of its rows).
__device__ __forceinline__ void issue_rows(uint32_t d, uint32_t a, uint32_t half, uint64_t b, int group, uint32_t idesc, bool add) {
  const uint64_t step = static_cast<uint64_t>(group) >> 3;   // 16 rows = two groups, in units of 16 bytes
#pragma unroll
  for (int s = 0; s < kTile / 16; ++s) mma_ts(d, a + (s >> 2) * half + (s & 3) * 8, b + s * step, idesc, add || s > 0);
}

// One query row's (or key row's) numbers of the packed gradients: 8 columns from `c`, rounded to bf16, `live` columns exist.
__device__ __forceinline__ void store8(__nv_bfloat16* dst, const float* x, bool aligned) {
  uint4 w;
  w.x = pack_bf16(x[0], x[1]); w.y = pack_bf16(x[2], x[3]); w.z = pack_bf16(x[4], x[5]); w.w = pack_bf16(x[6], x[7]);
  if (aligned) {
    *reinterpret_cast<uint4*>(dst) = w;
  } else {
    unsigned short* u = reinterpret_cast<unsigned short*>(dst);
    const uint32_t e[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      u[2 * j] = static_cast<unsigned short>(e[j]);
      u[2 * j + 1] = static_cast<unsigned short>(e[j] >> 16);
    }
  }
}
// Columns [lo, hi) (multiples of 16) of this thread's accumulator row times `scale` into a packed row; zeros where `live` is false.
__device__ __forceinline__ void store_row(uint32_t acc, int lo, int hi, int rp, float scale, __nv_bfloat16* dst, bool in_range,
                                          bool live, bool aligned) {
#pragma unroll 1
  for (int c = lo; c < hi; c += 16) {
    uint32_t r[16];
    tmem_ld16(acc + c, r);
    tmem_wait_ld_of(r);
    float x[16];
#pragma unroll
    for (int j = 0; j < 16; ++j) x[j] = live ? __uint_as_float(r[j]) * scale : 0.f;
    if (in_range) {
      store8(dst + c, x, aligned);
      if (c + 8 < rp) store8(dst + c + 8, x + 8, aligned);
    }
  }
}
__device__ __forceinline__ void zero_row(int lo, int hi, int rp, __nv_bfloat16* dst, bool aligned) {
  const float x[8] = {};
  for (int c = lo; c < min(hi, rp); c += 8) store8(dst + c, x, aligned);
}

// smallest of `count` exponents, by one warp
__device__ __forceinline__ int smallest_of(const int32_t* e, int count, int lane, int m = kTrainNoNumber) {
  for (int i = lane; i < count; i += 32) m = min(m, __ldg(e + i));
  return __reduce_min_sync(0xffffffffu, m);
}

// Bias of a tile of queries i0 .. against a tile of keys j0 ..: one number for all (`far`), unless some distance lies in front of the last entry.
__device__ __forceinline__ bool near_tile(const TrainParams& p, int i0, int j0) { return i0 - j0 - (kTile - 1) < p.bias_len - 1; }

// ---------------------------------------------------------------- forward

// A CTA has two tiles of queries, each with four softmax warps (a thread per query row, all 128 keys of a tile), so that the
// products of one run under the softmax of the other.  Per tile of keys: S, the row's maximum, 2^(S - reference) and their
// sum, P in the place of S, o' += P v'.  The reference is a lazy one: it moves, and o' is rescaled, only when a score exceeds
// it by 8.  TMEM: S of both tiles (128 columns each, P in the first 64 of them), o' of both.
// Bound by the exponentials (16 a clock: 2048 clocks for two pairs of tiles; their products take 1280 at rank 80).
template <int BIAS>
__global__ void __launch_bounds__(kTrThreads, 1) train_forward_kernel(const TrainParams p, int stages, int aligned) {
  extern __shared__ __align__(1024) unsigned char smem[];
  TrHeader* hdr = reinterpret_cast<TrHeader*>(smem);
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int unit = blockIdx.x, hq = unit / p.B, b = unit - hq * p.B, h = hq / p.group, ih = hq - h * p.group;
  const int key_unit = h * p.B + b;
  const HeadInfo hd = p.heads[h];
  const int pair = gridDim.y - 1 - blockIdx.y;               // long rows first
  const int n = __ldg(p.lens + b);
  const int rk16 = (hd.rp_k + 15) & ~15, rv16 = (hd.rp_v + 15) & ~15;
  const int q_bytes = kTile * rk16 * 2, v_bytes = kTile * rv16 * 2, stage_bytes = q_bytes + v_bytes;
  unsigned char* own = smem + kHeaderBytes;
  unsigned char* ring = own + 2 * q_bytes;
  int nt[2];                                                 // tiles of keys that a tile of queries sees
  for (int x = 0; x < 2; ++x) nt[x] = (2 * pair + x) * kTile < n ? 2 * pair + x + 1 : 0;
  const int most = max(nt[0], nt[1]);

  if (warp == 0) tmem_alloc(&hdr->tmem_base, 512);
  if (tid == 0) {
    for (int s = 0; s < kMaxRing; ++s) {
      mbar_init(&hdr->full[s], 1);
      mbar_init(&hdr->empty[s], 1);
    }
    mbar_init(&hdr->own, 1);
    for (int x = 0; x < 2; ++x) {
      mbar_init(&hdr->s_full[x], 1);
      mbar_init(&hdr->p_full[x], 4);
    }
    mbar_init(&hdr->done, 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == kIssueWarp) {
    const int m = smallest_of(p.v_exp + static_cast<int64_t>(key_unit) * p.tiles, p.tiles, lane);
    if (lane == 0) hdr->smallest[2] = m;
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = hdr->tmem_base;

  if (warp == kCopyWarp) {
    if (lane == 0 && most > 0) {
      const uint64_t keep = policy_evict_normal();
      const char* q = p.q_tiles + (static_cast<int64_t>(unit) * p.tiles + 2 * pair) * p.tile_k;
      mbar_arrive_expect_tx(&hdr->own, (nt[1] > 0 ? 2 : 1) * q_bytes);
      bulk_load(own, q, q_bytes, &hdr->own, keep);
      if (nt[1] > 0) bulk_load(own + q_bytes, q + p.tile_k, q_bytes, &hdr->own, keep);
      const char* k = p.k_tiles + static_cast<int64_t>(key_unit) * p.tiles * p.tile_k;
      const char* v = p.v_tiles + static_cast<int64_t>(key_unit) * p.tiles * p.tile_v;
      int issued = 0;
      for (int j = 0; j < most; ++j, ++issued) {
        const int st = j % stages;
        if (j >= stages && !mbar_wait(&hdr->empty[st], (j / stages - 1) & 1u, p.status)) break;
        mbar_arrive_expect_tx(&hdr->full[st], stage_bytes);
        bulk_load(ring + st * stage_bytes, k + static_cast<int64_t>(j) * p.tile_k, q_bytes, &hdr->full[st], keep);
        bulk_load(ring + st * stage_bytes + q_bytes, v + static_cast<int64_t>(j) * p.tile_v, v_bytes, &hdr->full[st], keep);
      }
      // copies in flight must land before the CTA leaves; normally their consumers have waited for them
      mbar_wait(&hdr->own, 0, p.status);
      for (int s = 0; s < stages && s < issued; ++s) mbar_wait(&hdr->full[s], ((issued - 1 - s) / stages) & 1u, p.status);
    }
  } else if (warp == kIssueWarp) {
    if (most > 0) {
      const bool lead = elect_one();
      const uint32_t idesc_o = instr_desc_f16(rv16) | kMnMajorB;
      const uint64_t dq = smem_desc(smem_u32(own), 128, rk16 << 4);
      const uint64_t dk = smem_desc(smem_u32(ring), 128, rk16 << 4);
      const uint64_t dv = smem_desc(smem_u32(ring) + q_bytes, rv16 << 4, 128);
      const uint64_t stage = stage_bytes >> 4;
      auto score = [&](int x, int st) {                      // S of tile x against the keys of a stage
        if (lead) {
          issue_rank(rk16 >> 4, tmem + x * kTile, dq + x * (q_bytes >> 4), dk + st * stage);
          mma_commit(&hdr->s_full[x]);
        }
        __syncwarp();
      };
      bool ok = wait_all(&hdr->own, 0, p.status) && wait_all(&hdr->full[0], 0, p.status);
      if (ok) {
        tc_fence_after();
        for (int x = 0; x < 2; ++x)
          if (nt[x] > 0) score(x, 0);
      }
      for (int j = 0; j < most && ok; ++j) {
        const int st = j % stages, next = (j + 1) % stages;
        bool ready = false;
        for (int x = 0; x < 2 && ok; ++x) {
          if (j >= nt[x]) continue;
          ok = wait_all(&hdr->p_full[x], j & 1u, p.status);
          if (!ok) break;
          tc_fence_after();
          if (lead) issue_rows(tmem + 256 + x * kTile, tmem + x * kTile, 32, dv + st * stage, rv16 << 4, idesc_o, j > 0);
          __syncwarp();
          if (j + 1 < nt[x]) {
            if (!ready) ok = wait_all(&hdr->full[next], ((j + 1) / stages) & 1u, p.status);
            ready = true;
            if (!ok) break;
            tc_fence_after();
            score(x, next);
          } else if (x == (nt[1] > 0 ? 1 : 0)) {             // (the longer tile ends last)
            if (lead) mma_commit(&hdr->done);
            __syncwarp();
          }
        }
        if (ok && lead) mma_commit(&hdr->empty[st]);
        __syncwarp();
      }
      if (!ok && lead) mma_commit(&hdr->done);               // (the softmax leaves by the status word)
      wait_all(&hdr->done, 0, p.status);                     // nothing is under way when the CTA leaves
      if (ok) wait_all(&hdr->empty[(most - 1) % stages], ((most - 1) / stages) & 1u, p.status);
    }
  } else {
    const int x = warp >> 2, row = (warp & 3) * 32 + lane, tile = 2 * pair + x, i0 = tile * kTile, i = i0 + row;
    const uint32_t lanes = static_cast<uint32_t>((warp & 3) * 32) << 16;
    const uint32_t tS = tmem + lanes + x * kTile, tO = tmem + lanes + 256 + x * kTile;
    const int64_t tiles_at = static_cast<int64_t>(key_unit) * p.tiles;
    const int g_v = hdr->smallest[2];
    const float* table = BIAS == kTable ? p.bias + static_cast<int64_t>(h) * p.bias_len : nullptr;
    const float slope2 = BIAS == kAlibi ? hd.alibi_slope2 : 0.f;
    float m = -INFINITY, l = 0.f;
    bool ok = true;
    const int q_e = nt[x] > 0 ? __ldg(p.q_exp + static_cast<int64_t>(unit) * p.tiles + tile) : 0;
    for (int j = 0; j < nt[x]; ++j) {
      const int j0 = j * kTile;
      float c = p.scale_log2 * pow2(-q_e - __ldg(p.k_exp + tiles_at + j));
      const float f = pow2(g_v - __ldg(p.v_exp + tiles_at + j));
      const bool diag = j0 == i0, near = BIAS == kTable && near_tile(p, i0, j0);
      float base = BIAS == kTable && !near ? __ldg(table + p.bias_len - 1) : BIAS == kAlibi ? slope2 * static_cast<float>(j0 - i) : 0.f;
      ok = wait_all(&hdr->s_full[x], j & 1u, p.status);
      if (!ok) break;
      tc_fence_after();
      // S of a tile with masked keys or distances of their own goes back scaled, biased and masked
      if (diag || near) {
#pragma unroll 1
        for (int k = 0; k < kTile; k += 32) {
          uint32_t r[32];
          tmem_ld32(tS + k, r);
          tmem_wait_ld_of(r);
#pragma unroll
          for (int e = 0; e < 32; ++e) {
            float y = __uint_as_float(r[e]) * c;
            if (near) y += __ldg(table + min(max(i - j0 - k - e, 0), p.bias_len - 1));
            if (BIAS == kAlibi) y += base + slope2 * static_cast<float>(k + e);
            if (diag && k + e > row) y = -INFINITY;
            r[e] = __float_as_uint(y);
          }
          tmem_st16(tS + k, *reinterpret_cast<uint32_t(*)[16]>(&r[0]));
          tmem_st16(tS + k + 16, *reinterpret_cast<uint32_t(*)[16]>(&r[16]));
        }
        tmem_wait_st();
        c = 1.f;
        base = 0.f;
      }
      const bool slanted = BIAS == kAlibi && !diag;          // the bias grows along the keys
      float top = -INFINITY;
      {
        float mx[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll 1
        for (int k = 0; k < kTile; k += 32) {
          uint32_t r[32];
          tmem_ld32(tS + k, r);
          tmem_wait_ld_of(r);
          if (slanted) {
#pragma unroll
            for (int e = 0; e < 32; ++e) r[e] = __float_as_uint(fmaf(__uint_as_float(r[e]), c, slope2 * static_cast<float>(k + e)));
          }
#pragma unroll
          for (int e = 0; e < 32; e += 8)
#pragma unroll
            for (int w = 0; w < 4; ++w) mx[w] = max3(mx[w], __uint_as_float(r[e + 2 * w]), __uint_as_float(r[e + 2 * w + 1]));
        }
        top = fmaxf(fmaxf(mx[0], mx[1]), fmaxf(mx[2], mx[3]));
        top = (slanted ? top : top * c) + base;              // (the scale is positive)
      }
      const bool raise = top > m + 8.f;
      const float now = raise ? top : m;
      if (__any_sync(0xffffffffu, raise)) {
        const float alpha = raise ? ex2(m - now) : 1.f;      // (0 at the first tile)
        l *= alpha;
        if (j > 0) {                                         // (S(j) came behind the product that last added to o')
#pragma unroll 1
          for (int k = 0; k < rv16; k += 16) {
            uint32_t o[16];
            tmem_ld16(tO + k, o);
            tmem_wait_ld_of(o);
#pragma unroll
            for (int e = 0; e < 16; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * alpha);
            tmem_st16(tO + k, o);
          }
        }
        m = now;
      }
      const float add = m == -INFINITY ? 0.f : base - m + kForwardShift;
      float sum0 = 0.f, sum1 = 0.f;
      uint32_t r[32];
      tmem_ld32(tS, r);
      tmem_wait_ld_of(r);
#pragma unroll 1
      for (int k = 0; k < kTile; k += 32) {
        float y[32];
#pragma unroll
        for (int e = 0; e < 32; e += 2) {
          if (slanted) {
            y[e] = fmaf(__uint_as_float(r[e]), c, fmaf(slope2, static_cast<float>(k + e), add));
            y[e + 1] = fmaf(__uint_as_float(r[e + 1]), c, fmaf(slope2, static_cast<float>(k + e + 1), add));
          } else {
            fma2(y[e], y[e + 1], __uint_as_float(r[e]), __uint_as_float(r[e + 1]), c, add);
          }
        }
        if (k + 32 < kTile) tmem_ld32(tS + k + 32, r);
        uint32_t w[16];
#pragma unroll
        for (int e = 0; e < 32; e += 2) {
          float e0 = ex2(y[e]), e1 = ex2(y[e + 1]);
          add2(sum0, sum1, e0, e1);
          if (f != 1.f) { e0 *= f; e1 *= f; }
          w[e / 2] = pack_f16(e0, e1);
        }
        tmem_wait_ld_of(r);                                      // (the columns behind are read before P reaches them)
        tmem_st16(tS + k / 2, w);
      }
      l += sum0 + sum1;
      tmem_wait_st();
      tc_fence_before();
      arrive_warp(&hdr->p_full[x], lane);
    }
    if (most > 0 && ok) ok = wait_all(&hdr->done, 0, p.status);
    tc_fence_after();
    if (ok && tile < p.tiles) {
      const bool live = nt[x] > 0 && i < n;
      const float inv = live ? 1.f / l : 0.f, back = pow2(-g_v);
      p.lse[static_cast<int64_t>(unit) * p.pad + i] = live ? kForwardShift - m - log2f(l) : -INFINITY;
      __nv_bfloat16* out = static_cast<__nv_bfloat16*>(p.out) +
                           (static_cast<int64_t>(b) * p.T + i) * (static_cast<int64_t>(p.group) * p.lr_v_width) + p.group * hd.lr_v_off + ih * hd.rp_v;
      float* o32 = p.o + (static_cast<int64_t>(unit) * p.T + i) * p.o_stride;
      if (nt[x] == 0) {
        if (i < p.T) zero_row(0, rv16, hd.rp_v, out, aligned);
      } else {
#pragma unroll 1
        for (int k = 0; k < rv16; k += 16) {
          uint32_t o[16];
          tmem_ld16(tO + k, o);
          tmem_wait_ld_of(o);
          float y[16];
#pragma unroll
          for (int e = 0; e < 16; ++e) y[e] = live ? __uint_as_float(o[e]) * inv * back : 0.f;
          if (i < p.T) {
#pragma unroll
            for (int half = 0; half < 2; ++half) {
              if (k + 8 * half >= hd.rp_v) continue;
              store8(out + k + 8 * half, y + 8 * half, aligned);
              *reinterpret_cast<float4*>(o32 + k + 8 * half) = make_float4(y[8 * half], y[8 * half + 1], y[8 * half + 2], y[8 * half + 3]);
              *reinterpret_cast<float4*>(o32 + k + 8 * half + 4) = make_float4(y[8 * half + 4], y[8 * half + 5], y[8 * half + 6], y[8 * half + 7]);
            }
          }
        }
      }
    }
  }
  tc_fence_before();
  __syncthreads();
  if (warp == 0) tmem_dealloc(tmem, 512);
}

// ---------------------------------------------------------------- dk', dv'

// A CTA owns a tile of keys and walks the tiles of queries that see it, of every query head of the group.  Per pair of tiles:
//   S^T = k' q'^T,  P^T = 2^(S^T - L);   dv' += P^T do';   G^T = v' do'^T,  dS^T = P^T (G^T - delta);   dk' += dS^T q'
// A thread has a key row (one TMEM lane) and half of the tile's queries; L and delta lie along its columns and come with the
// tile's ring stage.  While the softmax forms dS^T, the products run dv' and the next S^T; while it forms P^T, dk' and the next
// G^T.  TMEM: S^T, G^T (P^T and dS^T in their place, a half in each half's first 32 columns), dv', dk'.
// Bound by the two phases' chains: 1024 clocks of exponentials and some 500 of arithmetic a pair, 1280 of products at rank 80.
template <int BIAS>
__global__ void __launch_bounds__(kTrThreads, 1) train_dkv_kernel(const TrainParams p, int stages, int aligned) {
  extern __shared__ __align__(1024) unsigned char smem[];
  TrHeader* hdr = reinterpret_cast<TrHeader*>(smem);
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int key_unit = blockIdx.x, h = key_unit / p.B, b = key_unit - h * p.B;
  const HeadInfo hd = p.heads[h];
  const int tile = blockIdx.y, j0 = tile * kTile;            // the first keys have the most queries
  const int n = __ldg(p.lens + b);
  const int rk16 = (hd.rp_k + 15) & ~15, rv16 = (hd.rp_v + 15) & ~15;
  const int k_bytes = kTile * rk16 * 2, v_bytes = kTile * rv16 * 2, stage_bytes = k_bytes + v_bytes + 1024;
  unsigned char* own = smem + kHeaderBytes;
  unsigned char* ring = own + k_bytes + v_bytes;
  const int per_head = (n + kTile - 1) / kTile - tile;       // tiles of queries of one head
  const int total = per_head > 0 ? per_head * p.group : 0;

  if (warp == 0) tmem_alloc(&hdr->tmem_base, 512);
  if (tid == 0) {
    for (int s = 0; s < kMaxRing; ++s) {
      mbar_init(&hdr->full[s], 1);
      mbar_init(&hdr->empty[s], 1);
    }
    mbar_init(&hdr->own, 1);
    mbar_init(&hdr->s_full[0], 1);
    mbar_init(&hdr->g_full, 1);
    for (int x = 0; x < 2; ++x) mbar_init(&hdr->p_full[x], kSoftmaxWarps);      // P^T, dS^T
    mbar_init(&hdr->done, 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == kIssueWarp) {
    const int v = smallest_of(p.v_exp + static_cast<int64_t>(key_unit) * p.tiles, p.tiles, lane);
    int q = kTrainNoNumber, g = kTrainNoNumber;
    for (int i = 0; i < p.group; ++i) {
      const int64_t at = (static_cast<int64_t>(h * p.group + i) * p.B + b) * p.tiles;
      q = smallest_of(p.q_exp + at, p.tiles, lane, q);
      g = smallest_of(p.g_exp + at, p.tiles, lane, g);
    }
    if (lane == 0) {
      hdr->smallest[0] = q;
      hdr->smallest[2] = v;
      hdr->smallest[3] = g;
    }
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = hdr->tmem_base;

  if (warp == kCopyWarp) {
    if (lane == 0 && total > 0) {
      const uint64_t keep = policy_evict_normal();
      mbar_arrive_expect_tx(&hdr->own, k_bytes + v_bytes);
      bulk_load(own, p.k_tiles + (static_cast<int64_t>(key_unit) * p.tiles + tile) * p.tile_k, k_bytes, &hdr->own, keep);
      bulk_load(own + k_bytes, p.v_tiles + (static_cast<int64_t>(key_unit) * p.tiles + tile) * p.tile_v, v_bytes, &hdr->own, keep);
      int g = 0;
      bool ok = true;
      for (int i = 0; i < p.group && ok; ++i) {
        const int64_t unit = static_cast<int64_t>(h * p.group + i) * p.B + b;
        for (int t = 0; t < per_head; ++t, ++g) {
          const int st = g % stages;
          if (g >= stages && !(ok = mbar_wait(&hdr->empty[st], (g / stages - 1) & 1u, p.status))) break;
          unsigned char* to = ring + st * stage_bytes;
          unsigned long long* full = &hdr->full[st];
          const int64_t at = unit * p.tiles + tile + t;
          mbar_arrive_expect_tx(full, stage_bytes);
          bulk_load(to, p.q_tiles + at * p.tile_k, k_bytes, full, keep);
          bulk_load(to + k_bytes, p.g_tiles + at * p.tile_v, v_bytes, full, keep);
          bulk_load(to + k_bytes + v_bytes, p.lse + unit * p.pad + (tile + t) * kTile, 512, full, keep);
          bulk_load(to + k_bytes + v_bytes + 512, p.delta + unit * p.pad + (tile + t) * kTile, 512, full, keep);
        }
      }
      mbar_wait(&hdr->own, 0, p.status);
      for (int s = 0; s < stages && s < g; ++s) mbar_wait(&hdr->full[s], ((g - 1 - s) / stages) & 1u, p.status);
    }
  } else if (warp == kIssueWarp) {
    if (total > 0) {
      const bool lead = elect_one();
      const uint32_t idesc_k = instr_desc_f16(rk16) | kMnMajorB, idesc_v = instr_desc_f16(rv16) | kMnMajorB;
      const uint64_t dk = smem_desc(smem_u32(own), 128, rk16 << 4), dv = smem_desc(smem_u32(own) + k_bytes, 128, rv16 << 4);
      const uint64_t q_rank = smem_desc(smem_u32(ring), 128, rk16 << 4), g_rank = smem_desc(smem_u32(ring) + k_bytes, 128, rv16 << 4);
      const uint64_t q_rows = smem_desc(smem_u32(ring), rk16 << 4, 128), g_rows = smem_desc(smem_u32(ring) + k_bytes, rv16 << 4, 128);
      const uint64_t stage = stage_bytes >> 4;
      const uint32_t tS = tmem, tG = tmem + 128, tV = tmem + 256, tK = tmem + 384;
      bool ok = wait_all(&hdr->own, 0, p.status) && wait_all(&hdr->full[0], 0, p.status);
      if (ok) {
        tc_fence_after();
        if (lead) {
          issue_rank(rk16 >> 4, tS, dk, q_rank);
          mma_commit(&hdr->s_full[0]);
          issue_rank(rv16 >> 4, tG, dv, g_rank);
          mma_commit(&hdr->g_full);
        }
        __syncwarp();
      }
      for (int g = 0; g < total && ok; ++g) {
        const uint64_t at = static_cast<uint64_t>(g % stages) * stage, next = static_cast<uint64_t>((g + 1) % stages) * stage;
        const bool more = g + 1 < total;
        ok = wait_all(&hdr->p_full[0], g & 1u, p.status);
        if (ok && more) ok = wait_all(&hdr->full[(g + 1) % stages], ((g + 1) / stages) & 1u, p.status);
        if (!ok) break;
        tc_fence_after();
        if (lead) {
          issue_rows(tV, tS, 64, g_rows + at, rv16 << 4, idesc_v, g > 0);
          if (more) {
            issue_rank(rk16 >> 4, tS, dk, q_rank + next);
            mma_commit(&hdr->s_full[0]);
          }
        }
        __syncwarp();
        ok = wait_all(&hdr->p_full[1], g & 1u, p.status);
        if (!ok) break;
        tc_fence_after();
        if (lead) {
          issue_rows(tK, tG, 64, q_rows + at, rk16 << 4, idesc_k, g > 0);
          mma_commit(&hdr->empty[g % stages]);
          if (more) {
            issue_rank(rv16 >> 4, tG, dv, g_rank + next);
            mma_commit(&hdr->g_full);
          }
        }
        __syncwarp();
      }
      if (lead) mma_commit(&hdr->done);
      __syncwarp();
      wait_all(&hdr->done, 0, p.status);
    }
  } else {
    const int hf = warp >> 2, row = (warp & 3) * 32 + lane, key = j0 + row;
    const uint32_t lanes = static_cast<uint32_t>((warp & 3) * 32) << 16;
    const uint32_t tS = tmem + lanes + hf * 64, tG = tmem + lanes + 128 + hf * 64;
    const float* table = BIAS == kTable ? p.bias + static_cast<int64_t>(h) * p.bias_len : nullptr;
    const float slope2 = BIAS == kAlibi ? hd.alibi_slope2 : 0.f;
    const int g_q = hdr->smallest[0], g_v = hdr->smallest[2], g_g = hdr->smallest[3];
    const int k_e = __ldg(p.k_exp + static_cast<int64_t>(key_unit) * p.tiles + tile), v_e = __ldg(p.v_exp + static_cast<int64_t>(key_unit) * p.tiles + tile);
    bool ok = true;
    int64_t exps = (static_cast<int64_t>(h * p.group) * p.B + b) * p.tiles + tile;
    int t = 0;
    for (int g = 0; g < total; ++g) {
      const int st = g % stages, i0 = j0 + t * kTile;
      const int q_e = __ldg(p.q_exp + exps + t), g_e = __ldg(p.g_exp + exps + t);
      // P^T = 2^(S c + add - L), times 2^14 and the tile's share of do''s scale;  dS^T = P^T (G^T a - delta d), at most 2^15:
      // |do' v'| and |delta| are below r 2^(16 - e - e'), e and e' the smallest exponents of do' and v'
      const float c = p.scale_log2 * pow2(-q_e - k_e);
      const int lift = kBackwardShift + g_g - g_e;
      const int d_e = -9 + g_g + g_v + g_q - q_e - lift;
      const float d = pow2(d_e), a = pow2(d_e - g_e - v_e);
      const bool near = BIAS == kTable && near_tile(p, i0, j0);
      float add = static_cast<float>(max(lift, -2000));
      if (BIAS == kTable && !near) add += __ldg(table + p.bias_len - 1);
      if (BIAS == kAlibi) add += slope2 * static_cast<float>(key - i0 - hf * 64);
      if (++t == per_head) { t = 0; exps += static_cast<int64_t>(p.B) * p.tiles; }
      ok = wait_all(&hdr->full[st], (g / stages) & 1u, p.status) && wait_all(&hdr->s_full[0], g & 1u, p.status);
      if (!ok) break;
      tc_fence_after();
      const float* lse = reinterpret_cast<const float*>(ring + st * stage_bytes + k_bytes + v_bytes) + hf * 64;
      const float* delta = lse + 128;
      const bool diag = i0 == j0;
      float e[64];
#pragma unroll
      for (int k = 0; k < 64; k += 32) {
        uint32_t r[32];
        tmem_ld32(tS + k, r);
        tmem_wait_ld_of(r);
#pragma unroll
        for (int x = 0; x < 32; x += 4) {
          const float4 ls = *reinterpret_cast<const float4*>(lse + k + x);
          const float l4[4] = {ls.x, ls.y, ls.z, ls.w};
#pragma unroll
          for (int y = 0; y < 4; y += 2) {
            float a0 = add, a1 = add;
            if (BIAS == kAlibi) { a0 = fmaf(-slope2, static_cast<float>(k + x + y), add); a1 = fmaf(-slope2, static_cast<float>(k + x + y + 1), add); }
            a0 += l4[y];
            a1 += l4[y + 1];
            e[k + x + y] = fmaf(__uint_as_float(r[x + y]), c, a0);
            e[k + x + y + 1] = fmaf(__uint_as_float(r[x + y + 1]), c, a1);
          }
        }
      }
      if (near) {
#pragma unroll
        for (int k = 0; k < 64; ++k) e[k] += __ldg(table + min(max(i0 + hf * 64 + k - key, 0), p.bias_len - 1));
      }
#pragma unroll
      for (int k = 0; k < 64; ++k) e[k] = ex2(e[k]);
      if (diag) {
#pragma unroll
        for (int k = 0; k < 64; ++k)
          if (hf * 64 + k < row) e[k] = 0.f;
      }
#pragma unroll
      for (int k = 0; k < 64; k += 32) {
        uint32_t w[16];
#pragma unroll
        for (int x = 0; x < 16; ++x) w[x] = pack_f16(e[k + 2 * x], e[k + 2 * x + 1]);
        tmem_st16(tS + k / 2, w);
      }
      tmem_wait_st();
      tc_fence_before();
      arrive_warp(&hdr->p_full[0], lane);
      ok = wait_all(&hdr->g_full, g & 1u, p.status);
      if (!ok) break;
      tc_fence_after();
#pragma unroll
      for (int k = 0; k < 64; k += 32) {
        uint32_t r[32], w[16];
        tmem_ld32(tG + k, r);
        tmem_wait_ld_of(r);
#pragma unroll
        for (int x = 0; x < 32; x += 4) {
          const float4 dl = *reinterpret_cast<const float4*>(delta + k + x);
          const float d4[4] = {dl.x, dl.y, dl.z, dl.w};
#pragma unroll
          for (int y = 0; y < 4; y += 2) {
            const float x0 = e[k + x + y] * fmaf(__uint_as_float(r[x + y]), a, -d * d4[y]);
            const float x1 = e[k + x + y + 1] * fmaf(__uint_as_float(r[x + y + 1]), a, -d * d4[y + 1]);
            w[(x + y) / 2] = pack_f16(x0, x1);
          }
        }
        tmem_st16(tG + k / 2, w);
      }
      tmem_wait_st();
      tc_fence_before();
      arrive_warp(&hdr->p_full[1], lane);
    }
    if (total > 0 && ok) ok = wait_all(&hdr->done, 0, p.status);
    tc_fence_after();
    if (ok) {
      const bool in_range = key < p.T, live = key < n;
      const int k_split = ((rk16 >> 4) + 1) / 2 * 16, v_split = ((rv16 >> 4) + 1) / 2 * 16;
      const int k_lo = hf ? k_split : 0, k_hi = hf ? rk16 : k_split, v_lo = hf ? v_split : 0, v_hi = hf ? rv16 : v_split;
      __nv_bfloat16* to_k = static_cast<__nv_bfloat16*>(p.dk) + (static_cast<int64_t>(b) * p.T + key) * p.lr_k_width + hd.lr_k_off;
      __nv_bfloat16* to_v = static_cast<__nv_bfloat16*>(p.dv) + (static_cast<int64_t>(b) * p.T + key) * p.lr_v_width + hd.lr_v_off;
      if (total == 0) {
        if (in_range) {
          zero_row(k_lo, k_hi, hd.rp_k, to_k, aligned & 1);
          zero_row(v_lo, v_hi, hd.rp_v, to_v, aligned & 2);
        }
      } else {
        store_row(tmem + lanes + 384, k_lo, k_hi, hd.rp_k, p.scale * pow2(9 - g_g - g_v - g_q), to_k, in_range, live, aligned & 1);
        store_row(tmem + lanes + 256, v_lo, v_hi, hd.rp_v, pow2(-kBackwardShift - g_g), to_v, in_range, live, aligned & 2);
      }
    }
  }
  tc_fence_before();
  __syncthreads();
  if (warp == 0) tmem_dealloc(tmem, 512);
}

// ---------------------------------------------------------------- dq'

// A CTA owns a tile of queries and walks the tiles of keys that it sees: S = q' k'^T, G = do' v'^T, dS = P (G - delta),
// dq' += dS k'.  A thread has a query row and half of the tile's keys.  S has two buffers, so that the softmax finds the next
// scores when it has done a tile; dS takes the place of S, and G is free again as soon as it has been read.
// TMEM: S[2], G, dq'.  Bound by the softmax warps: 1024 clocks of exponentials and some 500 of arithmetic a pair.
// The gradient of a learned bias is a sum over dS of equal distance: over diagonals.  Far tiles, whose distances share the last
// bucket, are added up whole; in the others a sum moves one lane up with every column, so that it follows its diagonal, and
// leaves the warp complete.  All of it in a fixed order, without atomics.
template <int BIAS>
__global__ void __launch_bounds__(kTrThreads, 1) train_dq_kernel(const TrainParams p, int stages, int aligned) {
  extern __shared__ __align__(1024) unsigned char smem[];
  TrHeader* hdr = reinterpret_cast<TrHeader*>(smem);
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int unit = blockIdx.x, hq = unit / p.B, b = unit - hq * p.B, h = hq / p.group, ih = hq - h * p.group;
  const int key_unit = h * p.B + b;
  const HeadInfo hd = p.heads[h];
  const int tile = gridDim.y - 1 - blockIdx.y, i0 = tile * kTile;
  const int n = __ldg(p.lens + b);
  const int rk16 = (hd.rp_k + 15) & ~15, rv16 = (hd.rp_v + 15) & ~15;
  const int k_bytes = kTile * rk16 * 2, v_bytes = kTile * rv16 * 2, stage_bytes = k_bytes + v_bytes;
  unsigned char* own = smem + kHeaderBytes;
  unsigned char* ring = own + k_bytes + v_bytes;
  float* diagonals = reinterpret_cast<float*>(ring + stages * stage_bytes);      // [softmax warps][96], then [warps][buckets]
  const int nt = i0 < n ? tile + 1 : 0;

  if (warp == 0) tmem_alloc(&hdr->tmem_base, 512);
  if (tid == 0) {
    for (int s = 0; s < kMaxRing; ++s) {
      mbar_init(&hdr->full[s], 1);
      mbar_init(&hdr->empty[s], 1);
    }
    mbar_init(&hdr->own, 1);
    for (int x = 0; x < 2; ++x) {
      mbar_init(&hdr->s_full[x], 1);
      mbar_init(&hdr->p_full[x], kSoftmaxWarps);             // dS in S's buffer
    }
    mbar_init(&hdr->g_full, 1);
    mbar_init(&hdr->g_read, kSoftmaxWarps);
    mbar_init(&hdr->done, 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == kIssueWarp) {
    const int k = smallest_of(p.k_exp + static_cast<int64_t>(key_unit) * p.tiles, p.tiles, lane);
    const int v = smallest_of(p.v_exp + static_cast<int64_t>(key_unit) * p.tiles, p.tiles, lane);
    if (lane == 0) {
      hdr->smallest[1] = k;
      hdr->smallest[2] = v;
    }
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = hdr->tmem_base;

  if (warp == kCopyWarp) {
    if (lane == 0 && nt > 0) {
      const uint64_t keep = policy_evict_normal();
      const int64_t at = static_cast<int64_t>(unit) * p.tiles + tile, keys = static_cast<int64_t>(key_unit) * p.tiles;
      mbar_arrive_expect_tx(&hdr->own, k_bytes + v_bytes);
      bulk_load(own, p.q_tiles + at * p.tile_k, k_bytes, &hdr->own, keep);
      bulk_load(own + k_bytes, p.g_tiles + at * p.tile_v, v_bytes, &hdr->own, keep);
      int issued = 0;
      for (int j = 0; j < nt; ++j, ++issued) {
        const int st = j % stages;
        if (j >= stages && !mbar_wait(&hdr->empty[st], (j / stages - 1) & 1u, p.status)) break;
        unsigned char* to = ring + st * stage_bytes;
        mbar_arrive_expect_tx(&hdr->full[st], stage_bytes);
        bulk_load(to, p.k_tiles + (keys + j) * p.tile_k, k_bytes, &hdr->full[st], keep);
        bulk_load(to + k_bytes, p.v_tiles + (keys + j) * p.tile_v, v_bytes, &hdr->full[st], keep);
      }
      mbar_wait(&hdr->own, 0, p.status);
      for (int s = 0; s < stages && s < issued; ++s) mbar_wait(&hdr->full[s], ((issued - 1 - s) / stages) & 1u, p.status);
    }
  } else if (warp == kIssueWarp) {
    if (nt > 0) {
      const bool lead = elect_one();
      const uint32_t idesc = instr_desc_f16(rk16) | kMnMajorB;
      const uint64_t dq = smem_desc(smem_u32(own), 128, rk16 << 4), dg = smem_desc(smem_u32(own) + k_bytes, 128, rv16 << 4);
      const uint64_t k_rank = smem_desc(smem_u32(ring), 128, rk16 << 4), v_rank = smem_desc(smem_u32(ring) + k_bytes, 128, rv16 << 4);
      const uint64_t k_rows = smem_desc(smem_u32(ring), rk16 << 4, 128);
      const uint64_t stage = stage_bytes >> 4;
      const uint32_t tG = tmem + 256, tQ = tmem + 384;
      bool ok = wait_all(&hdr->own, 0, p.status);
      // S(j) into buffer j & 1 and, for the first tile, G(0)
      auto score = [&](int j) {
        ok = wait_all(&hdr->full[j % stages], (j / stages) & 1u, p.status);
        if (!ok) return;
        tc_fence_after();
        if (lead) {
          issue_rank(rk16 >> 4, tmem + (j & 1) * kTile, dq, k_rank + static_cast<uint64_t>(j % stages) * stage);
          mma_commit(&hdr->s_full[j & 1]);
        }
        __syncwarp();
      };
      auto second = [&](int j) {
        if (lead) {
          issue_rank(rv16 >> 4, tG, dg, v_rank + static_cast<uint64_t>(j % stages) * stage);
          mma_commit(&hdr->g_full);
        }
        __syncwarp();
      };
      if (ok) score(0);
      if (ok) second(0);
      if (ok && nt > 1) score(1);
      for (int j = 0; j < nt && ok; ++j) {
        if (j + 1 < nt) {                                    // G(j) has been read: G(j + 1)
          ok = wait_all(&hdr->g_read, j & 1u, p.status);
          if (!ok) break;
          tc_fence_after();
          second(j + 1);
        }
        ok = wait_all(&hdr->p_full[j & 1], (j >> 1) & 1u, p.status);
        if (!ok) break;
        tc_fence_after();
        if (lead) {
          issue_rows(tQ, tmem + (j & 1) * kTile, 64, k_rows + static_cast<uint64_t>(j % stages) * stage, rk16 << 4, idesc, j > 0);
          mma_commit(&hdr->empty[j % stages]);
        }
        __syncwarp();
        if (j + 2 < nt) score(j + 2);
      }
      if (lead) mma_commit(&hdr->done);
      __syncwarp();
      wait_all(&hdr->done, 0, p.status);
    }
  } else {
    const int hf = warp >> 2, row = (warp & 3) * 32 + lane, i = i0 + row;
    const uint32_t lanes = static_cast<uint32_t>((warp & 3) * 32) << 16;
    const uint32_t tG = tmem + lanes + 256 + hf * 64;
    const float* table = BIAS == kTable ? p.bias + static_cast<int64_t>(h) * p.bias_len : nullptr;
    const float slope2 = BIAS == kAlibi ? hd.alibi_slope2 : 0.f;
    const int g_k = hdr->smallest[1], g_v = hdr->smallest[2];
    const int64_t keys = static_cast<int64_t>(key_unit) * p.tiles;
    const int64_t stat = static_cast<int64_t>(unit) * p.pad + i;
    const float lse = nt > 0 ? __ldg(p.lse + stat) : 0.f, delta = nt > 0 ? __ldg(p.delta + stat) : 0.f;
    const int q_e = nt > 0 ? __ldg(p.q_exp + static_cast<int64_t>(unit) * p.tiles + tile) : 0;
    const int g_e = nt > 0 ? __ldg(p.g_exp + static_cast<int64_t>(unit) * p.tiles + tile) : 0;
    const bool sums = BIAS == kTable && p.dtable != nullptr;
    float* my_diagonals = diagonals + warp * 96;
    float far_sum = 0.f;                                     // dS of far tiles, this thread's
    float by_bucket[8] = {};                                 // buckets lane, lane + 32, ...: this warp's
    bool ok = true;
    for (int j = 0; j < nt; ++j) {
      const int j0 = j * kTile;
      const int k_e = __ldg(p.k_exp + keys + j), v_e = __ldg(p.v_exp + keys + j);
      // dS at most 2^15 (see above), times the tile's share of the scale of k'
      const float c = p.scale_log2 * pow2(-q_e - k_e);
      const int d_e = -9 + g_e + g_v + g_k - k_e;
      const float a = pow2(d_e - g_e - v_e), d = pow2(d_e) * delta;
      const bool near = BIAS == kTable && near_tile(p, i0, j0), diag = j0 == i0;
      float add = lse;
      if (BIAS == kTable && !near) add += __ldg(table + p.bias_len - 1);
      if (BIAS == kAlibi) add += slope2 * static_cast<float>(j0 + hf * 64 - i);
      const uint32_t tS = tmem + lanes + (j & 1) * kTile + hf * 64;
      ok = wait_all(&hdr->s_full[j & 1], (j >> 1) & 1u, p.status);
      if (!ok) break;
      tc_fence_after();
      float e[64];
#pragma unroll
      for (int k = 0; k < 64; k += 32) {
        uint32_t r[32];
        tmem_ld32(tS + k, r);
        tmem_wait_ld_of(r);
#pragma unroll
        for (int x = 0; x < 32; x += 2) {
          if (BIAS == kAlibi) {
            e[k + x] = fmaf(__uint_as_float(r[x]), c, fmaf(slope2, static_cast<float>(k + x), add));
            e[k + x + 1] = fmaf(__uint_as_float(r[x + 1]), c, fmaf(slope2, static_cast<float>(k + x + 1), add));
          } else {
            fma2(e[k + x], e[k + x + 1], __uint_as_float(r[x]), __uint_as_float(r[x + 1]), c, add);
          }
        }
      }
      if (near) {
#pragma unroll
        for (int k = 0; k < 64; ++k) e[k] += __ldg(table + min(max(i - j0 - hf * 64 - k, 0), p.bias_len - 1));
      }
#pragma unroll
      for (int k = 0; k < 64; ++k) e[k] = ex2(e[k]);
      if (diag) {
#pragma unroll
        for (int k = 0; k < 64; ++k)
          if (hf * 64 + k > row) e[k] = 0.f;
      }
      ok = wait_all(&hdr->g_full, j & 1u, p.status);
      if (!ok) break;
      tc_fence_after();
#pragma unroll
      for (int k = 0; k < 64; k += 32) {
        uint32_t r[32];
        tmem_ld32(tG + k, r);
        tmem_wait_ld_of(r);
#pragma unroll
        for (int x = 0; x < 32; x += 2) {
          float y0, y1;
          fma2(y0, y1, __uint_as_float(r[x]), __uint_as_float(r[x + 1]), a, -d);
          e[k + x] *= y0;
          e[k + x + 1] *= y1;
        }
      }
      tc_fence_before();
      arrive_warp(&hdr->g_read, lane);
#pragma unroll
      for (int k = 0; k < 64; k += 32) {
        uint32_t w[16];
#pragma unroll
        for (int x = 0; x < 16; ++x) w[x] = pack_f16(e[k + 2 * x], e[k + 2 * x + 1]);
        tmem_st16(tS + k / 2, w);
      }
      tmem_wait_st();
      tc_fence_before();
      arrive_warp(&hdr->p_full[j & 1], lane);
      if (sums) {
        const float back = pow2(-d_e);
        if (!near) {
          float s = 0.f;
#pragma unroll
          for (int k = 0; k < 64; ++k) s += e[k];
          far_sum = fmaf(s, back, far_sum);
        } else {
          // slot 63 + (row in the warp) - column
          float s = 0.f;
#pragma unroll
          for (int k = 0; k < 64; ++k) {
            s = __shfl_up_sync(0xffffffffu, s, 1);
            s = (lane == 0 ? 0.f : s) + e[k];
            if (lane == 31) my_diagonals[94 - k] = s;
          }
          if (lane < 31) my_diagonals[lane] = s;
          __syncwarp();
          const int first = i0 + (warp & 3) * 32 - j0 - hf * 64 - 63;      // distance of slot 0
#pragma unroll
          for (int u = 0; u < 8; ++u) {
            const int bucket = lane + 32 * u;
            if (bucket < p.buckets) {
              const int from = max(__ldg(p.starts + bucket) - first, 0);
              const int next = __ldg(p.starts + bucket + 1), to = next > first + 95 ? 95 : next - first;
              float sum = 0.f;
              for (int x = from; x < to; ++x) sum += my_diagonals[x];
              by_bucket[u] = fmaf(sum, back, by_bucket[u]);
            }
          }
          __syncwarp();
        }
      }
    }
    if (nt > 0 && ok) ok = wait_all(&hdr->done, 0, p.status);
    tc_fence_after();
    if (ok) {
      const int split = ((rk16 >> 4) + 1) / 2 * 16, lo = hf ? split : 0, hi = hf ? rk16 : split;
      __nv_bfloat16* to = static_cast<__nv_bfloat16*>(p.dq) +
                          (static_cast<int64_t>(b) * p.T + i) * (static_cast<int64_t>(p.group) * p.lr_k_width) + p.group * hd.lr_k_off + ih * hd.rp_k;
      if (nt == 0) {
        if (i < p.T) zero_row(lo, hi, hd.rp_k, to, aligned);
      } else {
        store_row(tmem + lanes + 384, lo, hi, hd.rp_k, p.scale * pow2(9 - g_e - g_v - g_k), to, i < p.T, i < n, aligned);
      }
    }
    if (sums) {
#pragma unroll
      for (int d = 16; d >= 1; d >>= 1) far_sum += __shfl_xor_sync(0xffffffffu, far_sum, d);
      float* mine = diagonals + kSoftmaxWarps * 96 + warp * p.buckets;
#pragma unroll
      for (int u = 0; u < 8; ++u) {
        const int bucket = lane + 32 * u;
        if (bucket < p.buckets) mine[bucket] = by_bucket[u] + (bucket == p.buckets - 1 ? far_sum : 0.f);
      }
    }
  }
  tc_fence_before();
  __syncthreads();
  if (BIAS == kTable && p.dtable != nullptr && tid < p.buckets) {        // (group 1: a head's units are its sequences)
    float sum = 0.f;
#pragma unroll
    for (int w = 0; w < kSoftmaxWarps; ++w) sum += diagonals[kSoftmaxWarps * 96 + w * p.buckets + tid];
    p.bias_part[(static_cast<int64_t>(unit) * p.tiles + tile) * p.buckets + tid] = sum;
  }
  if (warp == 0) tmem_dealloc(tmem, 512);
}

// Ring stages that fit beside the CTA's own tiles.
int ring_stages(size_t fixed, size_t stage, size_t* smem) {
  int stages = static_cast<int>((227 * 1024 - fixed) / stage);
  if (stages > kMaxRing) stages = kMaxRing;
  *smem = fixed + stages * stage;
  if (*smem < 120 * 1024) *smem = 120 * 1024;                // one CTA per SM: it takes all of the SM's TMEM
  return stages;
}
template <typename Kernel>
cudaError_t run(Kernel kernel, size_t (&done)[kMaxDevices], dim3 grid, size_t smem, const TrainParams& p, int stages, int aligned, cudaStream_t s) {
  const cudaError_t e = ensure_dynamic_smem(kernel, smem, done);
  if (e != cudaSuccess) return e;
  kernel<<<grid, kTrThreads, smem, s>>>(p, stages, aligned);
  return cudaGetLastError();
}
int bias_of(const TrainParams& p) { return p.bias != nullptr ? kTable : p.alibi ? kAlibi : kNone; }
bool on16(const void* x) { return reinterpret_cast<uintptr_t>(x) % 16 == 0; }

}  // namespace

cudaError_t launch_train_tc_forward(const TrainParams& p, cudaStream_t s, uint64_t* launches) {
  static size_t done[3][kMaxDevices] = {};
  const size_t k = p.tile_k, v = p.tile_v;
  size_t smem = 0;
  const int stages = ring_stages(kHeaderBytes + 2 * k, k + v, &smem), bias = bias_of(p);
  const dim3 grid(p.H * p.group * p.B, (p.tiles + 1) / 2);
  ++*launches;
  const int aligned = on16(p.out);
  if (bias == kTable) return run(train_forward_kernel<kTable>, done[2], grid, smem, p, stages, aligned, s);
  if (bias == kAlibi) return run(train_forward_kernel<kAlibi>, done[1], grid, smem, p, stages, aligned, s);
  return run(train_forward_kernel<kNone>, done[0], grid, smem, p, stages, aligned, s);
}

cudaError_t launch_train_tc_backward(const TrainParams& p, cudaStream_t s, uint64_t* launches) {
  static size_t done_kv[3][kMaxDevices] = {}, done_q[3][kMaxDevices] = {};
  const size_t k = p.tile_k, v = p.tile_v;
  const int bias = bias_of(p);
  size_t smem = 0;
  int stages = ring_stages(kHeaderBytes + k + v, k + v + 1024, &smem);
  const dim3 grid_kv(p.H * p.B, p.tiles), grid_q(p.H * p.group * p.B, p.tiles);
  const int aligned = on16(p.dk) | on16(p.dv) << 1;
  cudaError_t e = bias == kTable   ? run(train_dkv_kernel<kTable>, done_kv[2], grid_kv, smem, p, stages, aligned, s)
                  : bias == kAlibi ? run(train_dkv_kernel<kAlibi>, done_kv[1], grid_kv, smem, p, stages, aligned, s)
                                   : run(train_dkv_kernel<kNone>, done_kv[0], grid_kv, smem, p, stages, aligned, s);
  if (e != cudaSuccess) return e;
  ++*launches;
  const size_t sums = p.dtable != nullptr ? kSoftmaxWarps * (96 + static_cast<size_t>(p.buckets)) * sizeof(float) : 0;
  stages = ring_stages(kHeaderBytes + k + v + sums, k + v, &smem);
  const bool q16 = on16(p.dq);
  e = bias == kTable   ? run(train_dq_kernel<kTable>, done_q[2], grid_q, smem, p, stages, q16, s)
      : bias == kAlibi ? run(train_dq_kernel<kAlibi>, done_q[1], grid_q, smem, p, stages, q16, s)
                       : run(train_dq_kernel<kNone>, done_q[0], grid_q, smem, p, stages, q16, s);
  ++*launches;
  return e;
}

}  // namespace ea
