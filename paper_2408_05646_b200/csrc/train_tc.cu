// Causal attention over rank-space rows and its backward pass on the fifth-generation tensor cores (16-bit layers): tcgen05
// products of fp16 tiles (see train_pack.cu), accumulators in TMEM.
//   S_ij = scale q'_i k'_j + b(i - j)  (j <= i < length),  P = softmax(S),  o'_i = sum_j P_ij v'_j
//   delta_i = do'_i o'_i,  dS_ij = P_ij (do'_i v'_j - delta_i),
//   dq'_i = scale sum_j dS_ij k'_j,  dk'_j = scale sum_i dS_ij q'_i,  dv'_j = sum_i P_ij do'_i
// Scores are kept in the base-2 domain.  The forward pass leaves L_i = log2 sum_j 2^S_ij per row; the backward pass recomputes
// P_ij = 2^(S_ij - L_i) from one product, without a maximum or a sum.
//
// A tile is 128 rows.  A persistent CTA per SM (it takes the SM's 512 TMEM columns) works through items: a tile (or two) of one
// axis, which it keeps in shared memory, against the tiles of the other axis, which stream through a ring in halves of 64 rows
// with score buffers of their own: while the softmax works on one half, the products of the other run.  Roles:
//   * a copying warp: a bulk copy per operand tile.  It alone reads the item list, lengths and exponents; what the others need to know
//     of an item goes with the item's own tiles, of which there are two sets where they fit, so that an item starts with its
//     tiles at hand (a CTA per item spent some 7000 clocks on its start and end: a fifth of the time at 4096 tokens);
//   * issuing warps, two or three.  (With one, the products were late: it shares its scheduler with softmax warps, which leave
//     it an instruction every 10 to 20 clocks.)  Products of one accumulator have one issuer, so that their order is fixed;
//   * eight softmax warps.  P and dS go back to TMEM as the A operand of the next product and never touch shared memory.
// The backward pass has two kinds of items, one that owns a tile of keys (dk', dv': four products per pair of tiles) and one that
// owns a tile of queries (dq': three, S and do' v' a second time): the alternative, dq' added up in memory by every tile of keys,
// moves 512 r bytes of fp32 additions per pair of tiles through L2 and needs turns for sums whose order does not change from run to run (not
// built).
// 4 x 4096 tokens, 32 heads, rank 80: forward 514 us, a backward call 1257 in a burst and 1425 under the power limit, 74 of them
// packing (684 and 603 TFLOP/s of the five products that the formulas need); tensor pipe busy 34 and 48 % of the time, exponentials
// 55 and 44 %, an instruction issued in 0.40 and
// 0.37 of the clocks.  What is left is the chain of a half tile, product, load, exponentials, store, product, of which two
// run at a time (some 4700 clocks for a pair of tiles, its key item and its query item together, against 2640 of their products).
// Tried and slower: three chains (a third fewer registers for each), sixteen softmax warps with half the columns, turns between
// the halves' exponentials, a part of the exponentials as polynomials on the multiply-add units.  No difference: 216 registers
// for the softmax warps and 56 for the others.
//
// Tiles carry a power of two each (2^e).  What is accumulated over tiles needs one scale: the tile's deviation from the
// smallest exponent of all goes into the factors that P and dS are formed with, where it costs nothing.
// Every wait is bounded; one that runs out ends every other one of the launch through the status word, but for those that see
// products and copies under way to their end.
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "internal.h"
#include "tc_common.cuh"

namespace ea {
namespace {

using namespace tc;

constexpr int kNone = 0, kAlibi = 1, kTable = 2;             // position bias
constexpr int kSoftmaxWarps = 8, kCopyWarp = 8, kIssueWarp = 9;
constexpr int kTrThreads = 12 * 32;       // softmax, copies, up to three issuing warps
constexpr int kHalf = 64;                 // rows of the walked axis that share a score buffer
constexpr int kMaxRing = 8;
constexpr int kHeaderBytes = 960;
constexpr int kScaleBytes = 16;           // behind a stage's tiles: the scales of the pair of tiles, worked out by the copying warp
constexpr int kForwardShift = 7;          // P of the forward pass times 2^7: its reference lags behind the maximum by up to 2^8
constexpr int kBackwardShift = 14;        // P of the backward pass, at most 1, times 2^14: fp16 keeps all bits down to 2^-28
constexpr int kLeastDeviation = -60;      // of a tile from the smallest exponent: with it P and dS are zero in fp16 (a tile of zeros has
                                          //   any), and what is summed in 32 bits, the rows' sums and dS of a learned bias, stays in range

// What a launch decides for all its CTAs.
struct Plan {
  int stages, sets;         // of the ring; sets of own tiles (1 or 2)
  int items, per_unit;      // items of the launch, and of a unit
  int units, chunk;         // units; as many as follow one another in the list with all their items (see item_of)
  int aligned;              // outputs on 16-byte boundaries: bit 0, bit 1
  int apart;                // dk', dv': P has TMEM columns of its own
};

// An item, as the copying warp passes it on.
struct Item {
  int unit, h, b, i;        // unit of the owned axis, its K/V head, sequence, query head of the group
  int tile, n;              // first tile of the owned axis, tokens of the sequence
  int rp_k, rp_v;
  int tiles[2];             // tiles that it walks (forward: for either of its two tiles of queries); tiles[0] < 0: no more items
  int small[4];             // smallest exponents of q', k', v', do'
};

struct __align__(16) TrHeader {
  unsigned long long full[kMaxRing], empty[kMaxRing];        // ring of tiles
  unsigned long long own_full[2], own_empty[2];              // the item's own tiles and its description
  unsigned long long s_full[2][2], p_full[2][2];             // forward: [tile of queries][half]
  unsigned long long g_full[2], g_read[2], s_read[2], p_used[2][2];
  unsigned long long acc_full[2], acc_free[2];               // sums complete; read
  unsigned long long drain[3];                               // an issuing warp's last products
  uint32_t tmem_base;
  Item item[2];
};
static_assert(2 * sizeof(TrHeader) <= kHeaderBytes, "header outgrew its area");

__device__ __forceinline__ bool elect_one() {
  uint32_t p;
  asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(p));
  return p != 0;
}
// A wait of a whole warp, in one short loop.  (Waits that leave the loop lane by lane, in a function of their own, cost the softmax
// warps issue slots and registers: 4 x 4096 tokens 1376 us, so 1258.)
__device__ __forceinline__ bool wait_all(unsigned long long* bar, uint32_t parity, int* status) {
  if (__all_sync(0xffffffffu, mbar_try_wait(bar, parity))) return true;
  uint64_t t0 = 0;
  for (uint32_t i = 1;; ++i) {
    if (__all_sync(0xffffffffu, mbar_try_wait(bar, parity))) return true;
    if ((i & 255u) == 0) {                                   // (as mbar_wait: a bound, and an end when another wait gave up)
      const uint64_t now = global_ns();
      if (t0 == 0) t0 = now;
      bool over = *reinterpret_cast<volatile int*>(status) == kStatusTimeout;
      if (now - t0 > kWaitBoundNs) {
        atomicExch(status, kStatusTimeout);
        over = true;
      }
      if (__any_sync(0xffffffffu, over)) return false;
    }
  }
}
// The same with the loop in a function of its own, lane by lane: the forward pass, whose softmax is longer, is better off with it
// (514 us, so 538).
__device__ __noinline__ bool wait_long(unsigned long long* bar, uint32_t parity, int* status) { return mbar_wait(bar, parity, status); }
__device__ __forceinline__ bool wait_called(unsigned long long* bar, uint32_t parity, int* status) {
  if (__all_sync(0xffffffffu, mbar_try_wait(bar, parity))) return true;
  return __all_sync(0xffffffffu, wait_long(bar, parity, status)) != 0;
}
// 2^e; exponents that no pair of ordinary tiles has end at the ends of the range
__device__ __forceinline__ float pow2(int e) { return __int_as_float((min(max(e, -126), 127) + 127) << 23); }
// 2^e in two factors, for results: their exponents are sums of three tiles' and reach over both ends of the range
__device__ __forceinline__ float2 halves_of(int e) { return make_float2(pow2(e >> 1), pow2(e - (e >> 1))); }
// Exponent of dS for the smallest exponents of do' and v': |do' v'| and |delta| are below r 2^(16 - g_e - v_e), and with it dS at
// most 2^15, the end of fp16.  (Gradients too small for that get as much of it as there is.)
__device__ __forceinline__ int gradient_exponent(int g_e, int v_e) { return min(g_e + v_e - 9, 126); }
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

// A product over the rank: D[128][64] = A B^T, both K-major, B the half of a tile; KS steps of 16 columns.
template <int KS>
__device__ __forceinline__ void issue_rank_steps(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc) {
#pragma unroll
  for (int s = 0; s < KS; ++s) mma_ss(d, a + 16 * s, b + 16 * s, idesc, s > 0);
}
__device__ __forceinline__ void issue_rank(int steps, uint32_t d, uint64_t a, uint64_t b) {
  const uint32_t idesc = instr_desc_f16(kHalf);
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
// A product over the 64 rows of a half: D[128][r16] (+)= A B with A (P or dS) in 32 columns of TMEM and B the half of a tile,
// taken MN-major (`group`: bytes of 8 of its rows).
__device__ __forceinline__ void issue_rows(uint32_t d, uint32_t a, uint64_t b, int group, uint32_t idesc, bool add) {
  const uint64_t step = static_cast<uint64_t>(group) >> 3;   // 16 rows = two groups, in units of 16 bytes
#pragma unroll
  for (int s = 0; s < kHalf / 16; ++s) mma_ts(d, a + 8 * s, b + s * step, idesc, add || s > 0);
}
// second half of a tile, in a descriptor: 64 rows = 8 groups
__device__ __forceinline__ uint64_t half_of(int half, int group) { return static_cast<uint64_t>(half) * (group >> 1); }
// A place in the ring and the phase of its barriers.
struct Place {
  int stage = 0;
  uint32_t phase = 0;
  __device__ __forceinline__ void next(int stages) {
    if (++stage == stages) { stage = 0; phase ^= 1u; }
  }
};
// Pairs of fp32 numbers in 64-bit registers.
__device__ __forceinline__ unsigned long long both(float x) { return pack2(x, x); }
__device__ __forceinline__ unsigned long long pair_at(const uint32_t (&r)[32], int k) {
  return pack2(__uint_as_float(r[2 * k]), __uint_as_float(r[2 * k + 1]));
}

// Entry `index` of the list of items.  The items of `chunk` units follow one another, the longest (slot 0) first: those that run
// at a time then stream tiles of a few units, which stay in L2 (all units at once are 168 MB for 4 x 4096 tokens of 32 heads),
// and the longest of many units together leave short ones for the end.  (Chunks of 32, 48, 80, 110 MB: 1398, 1378, 1380, 1390 us.)
__device__ __forceinline__ void item_of(const Plan& plan, int index, int& unit, int& slot) {
  const int per_chunk = plan.chunk * plan.per_unit, first = index / per_chunk * plan.chunk, rest = index % per_chunk;
  const int width = min(plan.chunk, plan.units - first);
  slot = rest / width;
  unit = first + rest - slot * width;
}
// The next entry for this CTA: lists are worked through in their order, by whichever CTA is free (texts of unequal lengths, dealt
// out beforehand, left the last CTA with 1.2 to 1.9 times the average work).  The first entries go by the CTA's number; the
// counter is zeroed by the packing in front.  Which CTA has an item does not change the item's result.
__device__ __forceinline__ int next_entry(int32_t* counter, int lane) {
  int x = 0;
  if (lane == 0) x = atomicAdd(counter, 1);
  return gridDim.x + __shfl_sync(0xffffffffu, x, 0);
}
// Set of own tiles of a CTA's item and the phase of its barriers.
__device__ __forceinline__ int set_of(const Plan& plan, int it) { return plan.sets == 2 ? it & 1 : 0; }
__device__ __forceinline__ uint32_t set_phase(const Plan& plan, int it) { return (plan.sets == 2 ? it >> 1 : it) & 1u; }

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
// Columns [lo, hi) (multiples of 16) of this thread's accumulator row times `scale` 2^e into a packed row; zeros where `live` is false.
__device__ __forceinline__ void store_row(uint32_t acc, int lo, int hi, int rp, float scale, int e, __nv_bfloat16* dst, bool in_range,
                                          bool live, bool aligned) {
  const float2 power = halves_of(e);
  scale *= power.x;
#pragma unroll 1
  for (int c = lo; c < hi; c += 16) {
    uint32_t r[16];
    tmem_ld16(acc + c, r);
    tmem_wait_ld_of(r);
    float x[16];
#pragma unroll
    for (int j = 0; j < 16; ++j) x[j] = live ? __uint_as_float(r[j]) * scale * power.y : 0.f;
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

// Bias of a half tile of queries i0 .. against keys j0 ..: one number for all, unless some distance lies in front of the last entry.
__device__ __forceinline__ bool near_tile(const TrainParams& p, int i0, int j0) { return i0 - j0 - (kTile - 1) < p.bias_len - 1; }

// Barriers of a run through a list of items.
__device__ __forceinline__ void set_up(TrHeader* hdr, int empty, int own_empty, int p_full, int acc_full, int acc_free) {
  for (int s = 0; s < kMaxRing; ++s) {
    mbar_init(&hdr->full[s], 1);
    mbar_init(&hdr->empty[s], empty);
  }
  for (int x = 0; x < 2; ++x) {
    mbar_init(&hdr->own_full[x], 1);
    mbar_init(&hdr->own_empty[x], own_empty);
    for (int y = 0; y < 2; ++y) {
      mbar_init(&hdr->s_full[x][y], 1);
      mbar_init(&hdr->p_full[x][y], p_full);
      mbar_init(&hdr->p_used[x][y], 1);
    }
    mbar_init(&hdr->g_full[x], 1);
    mbar_init(&hdr->g_read[x], kSoftmaxWarps / 2);
    mbar_init(&hdr->s_read[x], kSoftmaxWarps / 2);
    mbar_init(&hdr->acc_full[x], acc_full);
    mbar_init(&hdr->acc_free[x], acc_free);
  }
  for (int x = 0; x < 3; ++x) mbar_init(&hdr->drain[x], 1);
}
// All of a CTA's threads behind the set-up; returns the TMEM base.  What the launch before this one wrote is there afterwards.
__device__ __forceinline__ uint32_t begin(TrHeader* hdr, int warp, int tid) {
  if (warp == 0) tmem_alloc(&hdr->tmem_base, 512);
  if (tid == 0) asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  chain_go();
  chain_wait();
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  return __shfl_sync(0xffffffffu, hdr->tmem_base, 0);
}
__device__ __forceinline__ void end(uint32_t tmem, int warp) {
  tc_fence_before();
  __syncthreads();
  if (warp == 0) tmem_dealloc(tmem, 512);
}
// A wait for products or copies under way, which come to an end by themselves.  It has the bound of every wait, but does not end
// when another one gave up: that is when it is needed.
__device__ __noinline__ void wait_landed(unsigned long long* bar, uint32_t parity) {
  if (mbar_try_wait(bar, parity)) return;
  const uint64_t t0 = global_ns();
  while (!mbar_try_wait(bar, parity))
    if (global_ns() - t0 > kWaitBoundNs) return;
}
// The end of an issuing warp: nothing of it is under way when the CTA leaves.
__device__ __forceinline__ void drain(TrHeader* hdr, int which, bool lead) {
  if (lead) mma_commit(&hdr->drain[which]);
  __syncwarp();
  wait_landed(&hdr->drain[which], 0);
  __syncwarp();
}
// The end of a copying warp: all of its copies have landed before the CTA leaves, or goes over to the other kind of items.  (Their
// consumers wait for them too, but not those that gave up.)  `items`: phases of own_full that were begun.
__device__ __forceinline__ void drain_copies(TrHeader* hdr, const Plan& plan, int items, int issued, int lane) {
  if (lane == 0) {
    for (int s = 0; s < plan.sets && s < items; ++s) wait_landed(&hdr->own_full[s], set_phase(plan, items - 1 - ((items - 1 - s) % plan.sets)));
    for (int s = 0; s < plan.stages && s < issued; ++s) wait_landed(&hdr->full[s], ((issued - 1 - s) / plan.stages) & 1u);
  }
  __syncwarp();
}
// Test hook: a softmax warp gives up at its first item, as if that wait had run out.
__device__ __forceinline__ bool gives_up(const TrainParams& p, bool here, int it, int lane) {
  if (p.give_up_once == 0 || !here || it > 0) return false;
  if (lane == 0) atomicExch(p.status, kStatusTimeout);
  return true;
}

// ---------------------------------------------------------------- forward

// An item is two tiles of queries, each with four softmax warps (a thread per query row) and an issuing warp.  Per half tile of
// keys: S, the row's maximum, 2^(S - reference) and their sum, P in the place of S, o' += P v'.  The reference is a lazy one:
// it moves, and o' is rescaled, only when a score exceeds it by 8.  TMEM: two halves of S for both tiles (64 columns each, P in
// the first 32 of them), o' of both.
// Least clocks for two pairs of tiles at rank 80: exponentials 2048 (16 a clock), products 1630.
template <int BIAS>
__global__ void __launch_bounds__(kTrThreads, 1) train_forward_kernel(const __grid_constant__ TrainParams p, const __grid_constant__ Plan plan) {
  extern __shared__ __align__(1024) unsigned char smem[];
  TrHeader* hdr = reinterpret_cast<TrHeader*>(smem);
  const int tid = threadIdx.x, warp = __shfl_sync(0xffffffffu, tid >> 5, 0), lane = tid & 31;
  unsigned char* own = smem + kHeaderBytes;                  // sets of two tiles of q'
  unsigned char* ring = own + plan.sets * 2 * p.tile_k;
  const int stage_bytes = p.tile_k + p.tile_v + kScaleBytes; // (tiles of narrower heads fill a part)
  if (tid == 0) set_up(hdr, 2, 2 + kSoftmaxWarps, 4, 1, 4);
  const uint32_t tmem = begin(hdr, warp, tid);

  if (warp == kCopyWarp) {
    const uint64_t keep = policy_evict_normal();
    bool ok = true;
    Place at;
    int issued = 0, it = 0, index = blockIdx.x;
    for (;; ++it) {
      const int set = set_of(plan, it);
      if (it >= plan.sets) ok = wait_called(&hdr->own_empty[set], set_phase(plan, it) ^ 1u, p.status);
      if (!ok) break;
      Item* item = &hdr->item[set];
      if (it > 0) index = next_entry(p.next, lane);
      if (index >= plan.items) {
        if (lane == 0) {
          item->tiles[0] = -1;
          mbar_arrive(&hdr->own_full[set]);
        }
        break;
      }
      int unit, slot;
      item_of(plan, index, unit, slot);
      const int hq = unit / p.B, b = unit - hq * p.B, h = hq / p.group, key_unit = h * p.B + b;
      const int tile = 2 * (plan.per_unit - 1 - slot);
      const int n = kept_tokens(p, b), rp_k = __ldg(&p.heads[h].rp_k), rp_v = __ldg(&p.heads[h].rp_v);
      const int q_bytes = kTile * ((rp_k + 15) & ~15) * 2, v_bytes = kTile * ((rp_v + 15) & ~15) * 2;
      const int nt0 = tile * kTile < n ? tile + 1 : 0, nt1 = (tile + 1) * kTile < n ? tile + 2 : 0, most = max(nt0, nt1);
      const int32_t *k_exp = p.k_exp + static_cast<int64_t>(key_unit) * p.tiles, *v_exp = p.v_exp + static_cast<int64_t>(key_unit) * p.tiles;
      const int g_v = smallest_of(v_exp, most, lane);                                      // (of the tiles it walks)
      const int64_t q_at = static_cast<int64_t>(unit) * p.tiles + tile;
      const int q_e0 = __ldg(p.q_exp + q_at), q_e1 = nt1 > 0 ? __ldg(p.q_exp + q_at + 1) : 0;
      if (lane == 0) {
        item->unit = unit; item->h = h; item->b = b; item->i = hq - h * p.group;
        item->tile = tile; item->n = n; item->rp_k = rp_k; item->rp_v = rp_v;
        item->tiles[0] = nt0; item->tiles[1] = nt1;
        item->small[2] = g_v;
        unsigned char* to = own + set * 2 * p.tile_k;
        const char* q = p.q_tiles + q_at * p.tile_k;
        if (most > 0) {
          mbar_arrive_expect_tx(&hdr->own_full[set], (nt1 > 0 ? 2 : 1) * q_bytes);
          bulk_load(to, q, q_bytes, &hdr->own_full[set], keep);
          if (nt1 > 0) bulk_load(to + p.tile_k, q + p.tile_k, q_bytes, &hdr->own_full[set], keep);
        } else {
          mbar_arrive(&hdr->own_full[set]);
        }
        const char* k = p.k_tiles + static_cast<int64_t>(key_unit) * p.tiles * p.tile_k;
        const char* v = p.v_tiles + static_cast<int64_t>(key_unit) * p.tiles * p.tile_v;
        for (int j = 0; j < most; ++j, ++issued, at.next(plan.stages)) {
          // the tile's deviation from the largest v'
          const int k_e = __ldg(k_exp + j), f = max(g_v - __ldg(v_exp + j), kLeastDeviation);
          unsigned long long* full = &hdr->full[at.stage];
          if (issued >= plan.stages && !(ok = mbar_wait(&hdr->empty[at.stage], at.phase ^ 1u, p.status))) break;
          unsigned char* st = ring + at.stage * stage_bytes;
          *reinterpret_cast<float4*>(st + p.tile_k + p.tile_v) =
              make_float4(p.scale_log2 * pow2(-q_e0 - k_e), p.scale_log2 * pow2(-q_e1 - k_e), static_cast<float>(f), pow2(-f));
          mbar_arrive_expect_tx(full, q_bytes + v_bytes);
          bulk_load(st, k + static_cast<int64_t>(j) * p.tile_k, q_bytes, full, keep);
          bulk_load(st + p.tile_k, v + static_cast<int64_t>(j) * p.tile_v, v_bytes, full, keep);
        }
      }
      ok = __all_sync(0xffffffffu, ok);
      if (!ok) { ++it; break; }
    }
    drain_copies(hdr, plan, ok ? it + 1 : it, issued, lane);  // (the last phase ended the list)
  } else if (warp >= kIssueWarp && warp < kIssueWarp + 2) {
    const int x = warp - kIssueWarp;                         // the products of one tile of queries
    const bool lead = elect_one();
    const uint64_t stage = stage_bytes >> 4;
    const uint32_t tS = tmem + x * kTile, tO = tmem + 256 + x * kTile;
    bool ok = true;
    int done = 0, sums = 0;                                  // tiles and items behind this warp
    Place at, next;                                          // of P v' and of S
    for (int it = 0; ok; ++it) {
      const int set = set_of(plan, it);
      ok = wait_called(&hdr->own_full[set], set_phase(plan, it), p.status);
      if (!ok || hdr->item[set].tiles[0] < 0) break;
      const int nt = hdr->item[set].tiles[x], most = max(hdr->item[set].tiles[0], hdr->item[set].tiles[1]);
      const int rk16 = (hdr->item[set].rp_k + 15) & ~15, rv16 = (hdr->item[set].rp_v + 15) & ~15;
      const uint32_t idesc_o = instr_desc_f16(rv16) | kMnMajorB;
      const uint64_t dq = smem_desc(smem_u32(own) + (set * 2 + x) * p.tile_k, 128, rk16 << 4);
      const uint64_t dk = smem_desc(smem_u32(ring), 128, rk16 << 4), dv = smem_desc(smem_u32(ring) + p.tile_k, rv16 << 4, 128);
      if (nt > 0 && sums > 0) ok = wait_called(&hdr->acc_free[x], (sums - 1) & 1u, p.status);
      for (int j = 0; nt > 0 && j < 2 * nt + 2 && ok; ++j) { // S of half j, two halves ahead of P
        const int half = j & 1;
        if (j >= 2) {
          ok = wait_called(&hdr->p_full[x][half], (done + ((j - 2) >> 1)) & 1u, p.status);
          if (!ok) break;
          tc_fence_after();
          if (lead) {
            issue_rows(tO, tS + half * kHalf, dv + stage * at.stage + half_of(half, rv16 << 4), rv16 << 4, idesc_o, j > 2);
            mma_commit(&hdr->p_used[x][half]);
            if (half) mma_commit(&hdr->empty[at.stage]);
          }
          __syncwarp();
          if (half) at.next(plan.stages);
        }
        if (j < 2 * nt) {                                    // (in P's place: behind the product that takes it)
          if (!half) ok = wait_called(&hdr->full[next.stage], next.phase, p.status);
          if (!ok) break;
          tc_fence_after();
          if (lead) {
            issue_rank(rk16 >> 4, tS + half * kHalf, dq, dk + stage * next.stage + half_of(half, rk16 << 4));
            mma_commit(&hdr->s_full[x][half]);
          }
          __syncwarp();
          if (half) next.next(plan.stages);
        }
      }
      if (ok && lead) {
        if (nt > 0) mma_commit(&hdr->acc_full[x]);
        mma_commit(&hdr->own_empty[set]);
      }
      __syncwarp();
      done += nt;
      sums += nt > 0;
      for (int j = nt; j < most && ok; ++j) {                // tiles that only the other tile of queries sees
        ok = wait_called(&hdr->full[at.stage], at.phase, p.status);
        if (ok && lead) mbar_arrive(&hdr->empty[at.stage]);
        at.next(plan.stages);
        next.next(plan.stages);
      }
    }
    drain(hdr, x, lead);
  } else if (warp < kSoftmaxWarps) {
    const int x = warp >> 2, row = (warp & 3) * 32 + lane;
    const uint32_t lanes = static_cast<uint32_t>((warp & 3) * 32) << 16;
    const uint32_t tS = tmem + lanes + x * kTile, tO = tmem + lanes + 256 + x * kTile;
    bool ok = true;
    int done = 0, sums = 0;
    Place at;
    for (int it = 0; ok; ++it) {
      const int set = set_of(plan, it);
      ok = wait_called(&hdr->own_full[set], set_phase(plan, it), p.status);
      if (gives_up(p, blockIdx.x == 0 && warp == 0, it, lane)) ok = false;
      if (!ok) break;
      const Item item = hdr->item[set];
      if (item.tiles[0] < 0) break;
      const int nt = x ? item.tiles[1] : item.tiles[0], most = max(item.tiles[0], item.tiles[1]);
      const int tile = item.tile + x, i0 = tile * kTile, i = i0 + row, n = item.n, rv16 = (item.rp_v + 15) & ~15, g_v = item.small[2];
      const float* table = BIAS == kTable ? p.bias + static_cast<int64_t>(item.h) * p.bias_len : nullptr;
      const float far_bias = BIAS == kTable ? __ldg(table + p.bias_len - 1) : 0.f;
      const float slope2 = BIAS == kAlibi ? __ldg(&p.heads[item.h].alibi_slope2) : 0.f;
      float m = -INFINITY, l = 0.f;
      for (int j = 0; j < 2 * nt; ++j) {
        const int half = j & 1, j0 = j * kHalf;
        const bool diag = j >= 2 * nt - 2, near = BIAS == kTable && near_tile(p, i0, j0);
        float base = BIAS == kTable && !near ? far_bias : BIAS == kAlibi ? slope2 * static_cast<float>(j0 - i) : 0.f;
        const uint32_t tSh = tS + half * kHalf;
        ok = (half || wait_called(&hdr->full[at.stage], at.phase, p.status)) && wait_called(&hdr->s_full[x][half], (done + (j >> 1)) & 1u, p.status);
        if (!ok) break;
        tc_fence_after();
        const float4 scales = *reinterpret_cast<const float4*>(ring + at.stage * stage_bytes + p.tile_k + p.tile_v);
        float c = x ? scales.y : scales.x;
        // S of a tile with masked keys or distances of their own goes back scaled, biased and masked
        if (diag || near) {
#pragma unroll 1
          for (int k = 0; k < kHalf; k += 32) {
            uint32_t r[32];
            tmem_ld32(tSh + k, r);
            tmem_wait_ld_of(r);
#pragma unroll
            for (int e = 0; e < 32; ++e) {
              float y = __uint_as_float(r[e]) * c;
              if (near) y += __ldg(table + min(max(i - j0 - k - e, 0), p.bias_len - 1));
              if (BIAS == kAlibi) y += base + slope2 * static_cast<float>(k + e);
              if (diag && half * kHalf + k + e > row) y = -INFINITY;
              r[e] = __float_as_uint(y);
            }
            tmem_st16(tSh + k, *reinterpret_cast<uint32_t(*)[16]>(&r[0]));
            tmem_st16(tSh + k + 16, *reinterpret_cast<uint32_t(*)[16]>(&r[16]));
          }
          tmem_wait_st();
          c = 1.f;
          base = 0.f;
        }
        const bool slanted = BIAS == kAlibi && !diag;        // the bias grows along the keys
        uint32_t r[2][32];
        tmem_ld32(tSh, r[0]);
        tmem_ld32(tSh + 32, r[1]);
        tmem_wait_ld_of(r[0]);
        tmem_wait_ld_of(r[1]);
        float mx[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          if (slanted) {
#pragma unroll
            for (int e = 0; e < 32; ++e) r[k][e] = __float_as_uint(fmaf(__uint_as_float(r[k][e]), c, slope2 * static_cast<float>(32 * k + e)));
          }
#pragma unroll
          for (int e = 0; e < 32; e += 8)
#pragma unroll
            for (int w = 0; w < 4; ++w) mx[w] = max3(mx[w], __uint_as_float(r[k][e + 2 * w]), __uint_as_float(r[k][e + 2 * w + 1]));
        }
        if (slanted) c = 1.f;
        const float top = fmaf(fmaxf(fmaxf(mx[0], mx[1]), fmaxf(mx[2], mx[3])), c, base);         // (the scale is positive)
        const bool raise = top > m + 8.f;
        const float now = raise ? top : m;
        if (__any_sync(0xffffffffu, raise)) {
          const float alpha = raise ? ex2(m - now) : 1.f;    // (0 at the first keys)
          l *= alpha;
          if (j > 0) {                                       // the half before has been added to o'
            ok = wait_called(&hdr->p_used[x][half ^ 1], (done + ((j - 1) >> 1)) & 1u, p.status);
            if (!ok) break;
            tc_fence_after();
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
        const float add = m == -INFINITY ? 0.f : base - m + kForwardShift + scales.z;
        float sum0 = 0.f, sum1 = 0.f;
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          uint32_t w[16];
#pragma unroll
          for (int e = 0; e < 32; e += 2) {
            float y0, y1;
            fma2(y0, y1, __uint_as_float(r[k][e]), __uint_as_float(r[k][e + 1]), c, add);
            y0 = ex2(y0);
            y1 = ex2(y1);
            add2(sum0, sum1, y0, y1);
            w[e / 2] = pack_f16(y0, y1);
          }
          tmem_st16(tSh + 16 * k, w);
        }
        l = fmaf(sum0 + sum1, scales.w, l);
        tmem_wait_st();
        tc_fence_before();
        arrive_warp(&hdr->p_full[x][half], lane);
        if (half) at.next(plan.stages);
      }
      if (!ok) break;
      for (int j = nt; j < most; ++j) at.next(plan.stages);
      done += nt;
      if (nt > 0) ok = wait_called(&hdr->acc_full[x], sums & 1u, p.status);
      if (!ok) break;
      tc_fence_after();
      if (tile < p.tiles) {
        const bool live = nt > 0 && i < n, there = i < p.T;
        const float inv = live ? 1.f / l : 0.f, back = pow2(-g_v);
        p.lse[static_cast<int64_t>(item.unit) * p.pad + i] = live ? kForwardShift - m - log2f(l) : -INFINITY;
        __nv_bfloat16* out = static_cast<__nv_bfloat16*>(p.out) + (static_cast<int64_t>(item.b) * p.T + i) * (static_cast<int64_t>(p.group) * p.lr_v_width) +
                             p.group * __ldg(&p.heads[item.h].lr_v_off) + item.i * item.rp_v;
        float* o32 = p.o + (static_cast<int64_t>(item.unit) * p.T + i) * p.o_stride;
        if (nt == 0) {
          if (there) zero_row(0, rv16, item.rp_v, out, plan.aligned & 1);
        } else {
#pragma unroll 1
          for (int k = 0; k < rv16; k += 16) {
            uint32_t o[16];
            tmem_ld16(tO + k, o);
            tmem_wait_ld_of(o);
            float y[16];
#pragma unroll
            for (int e = 0; e < 16; ++e) y[e] = live ? __uint_as_float(o[e]) * inv * back : 0.f;
            if (there) {
#pragma unroll
              for (int part = 0; part < 2; ++part) {
                if (k + 8 * part >= item.rp_v) continue;
                store8(out + k + 8 * part, y + 8 * part, plan.aligned & 1);
                *reinterpret_cast<float4*>(o32 + k + 8 * part) = make_float4(y[8 * part], y[8 * part + 1], y[8 * part + 2], y[8 * part + 3]);
                *reinterpret_cast<float4*>(o32 + k + 8 * part + 4) = make_float4(y[8 * part + 4], y[8 * part + 5], y[8 * part + 6], y[8 * part + 7]);
              }
            }
          }
        }
      }
      if (nt > 0) {
        tc_fence_before();
        arrive_warp(&hdr->acc_free[x], lane);
        ++sums;
      }
      arrive_warp(&hdr->own_empty[set], lane);
    }
  }
  end(tmem, warp);
}

// ---------------------------------------------------------------- dk', dv'

// An item is a tile of keys; it walks the tiles of queries that see it, of every query head of the group.  Per half:
//   S^T = k' q'^T,  P^T = 2^(S^T - L);   dv' += P^T do';   G^T = v' do'^T,  dS^T = P^T (G^T - delta);   dk' += dS^T q'
// Each half has four softmax warps of its own; a thread has a key row (one TMEM lane).  L and delta lie along its columns and
// come with the tile's ring stage.  One issuing warp has S^T, one dv', one G^T and dk'.
// TMEM: S^T and G^T of both halves (dS^T in G^T's place), dv', dk'.  P^T has columns of its own where the ranks leave 64 of
// them (their sum at most 192, each in steps of 32): the next S^T then starts when this one has been read.  Otherwise it takes
// S^T's place.
template <int BIAS>
__device__ __forceinline__ void dkv_items(const TrainParams& p, const Plan& plan, TrHeader* hdr, unsigned char* smem, uint32_t tmem, int warp, int lane, int& index) {
  unsigned char* own = smem;                                 // sets of a tile of k' and one of v'
  unsigned char* ring = own + plan.sets * (p.tile_k + p.tile_v);
  const int rows_at = p.tile_k + p.tile_v, stage_bytes = rows_at + 1024 + kScaleBytes;      // q', do', then L and delta
  const bool apart = plan.apart != 0;
  // TMEM columns of S^T, G^T, dv', dk', and of P^T
  constexpr uint32_t cS = 0, cG = 128;
  const uint32_t cP = apart ? 256 : cS, p_step = apart ? 32 : kHalf, cV = apart ? 320 : 256;
  const uint32_t cK = cV + (apart ? (((p.max_rp_v + 15) & ~15) + 31) & ~31 : 128);
  if (warp == kCopyWarp) {
    const uint64_t keep = policy_evict_normal();
    bool ok = true;
    Place at;
    int issued = 0, it = 0;
    for (;; ++it) {
      const int set = set_of(plan, it);
      if (it >= plan.sets) ok = wait_all(&hdr->own_empty[set], set_phase(plan, it) ^ 1u, p.status);
      if (!ok) break;
      Item* item = &hdr->item[set];
      if (it > 0) index = next_entry(p.next + 1, lane);
      if (index >= plan.items) {
        if (lane == 0) {
          item->tiles[0] = -1;
          mbar_arrive(&hdr->own_full[set]);
        }
        break;
      }
      int unit, tile;                                        // (the first keys have the most queries)
      item_of(plan, index, unit, tile);
      const int h = unit / p.B, b = unit - h * p.B;
      const int n = kept_tokens(p, b), rp_k = __ldg(&p.heads[h].rp_k), rp_v = __ldg(&p.heads[h].rp_v);
      const int k_bytes = kTile * ((rp_k + 15) & ~15) * 2, v_bytes = kTile * ((rp_v + 15) & ~15) * 2;
      const int per_head = max((n + kTile - 1) / kTile - tile, 0);                          // tiles of queries of one head
      const int64_t own_at = static_cast<int64_t>(unit) * p.tiles + tile;
      const int k_e = __ldg(p.k_exp + own_at), v_e = __ldg(p.v_exp + own_at);
      const int g_v = smallest_of(p.v_exp + static_cast<int64_t>(unit) * p.tiles, p.tiles, lane);   // (delta knows every key)
      int g_q = kTrainNoNumber, g_g = kTrainNoNumber;
      for (int i = 0; i < p.group; ++i) {
        const int64_t at_q = (static_cast<int64_t>(h * p.group + i) * p.B + b) * p.tiles + tile;          // (of the tiles it walks)
        g_q = smallest_of(p.q_exp + at_q, p.tiles - tile, lane, g_q);
        g_g = smallest_of(p.g_exp + at_q, p.tiles - tile, lane, g_g);
      }
      if (lane == 0) {
        item->unit = unit; item->h = h; item->b = b; item->i = 0;
        item->tile = tile; item->n = n; item->rp_k = rp_k; item->rp_v = rp_v;
        item->tiles[0] = per_head * p.group; item->tiles[1] = per_head;
        item->small[0] = g_q; item->small[2] = g_v; item->small[3] = g_g;
        unsigned char* to = own + set * (p.tile_k + p.tile_v);
        if (per_head > 0) {
          mbar_arrive_expect_tx(&hdr->own_full[set], k_bytes + v_bytes);
          bulk_load(to, p.k_tiles + own_at * p.tile_k, k_bytes, &hdr->own_full[set], keep);
          bulk_load(to + p.tile_k, p.v_tiles + own_at * p.tile_v, v_bytes, &hdr->own_full[set], keep);
        } else {
          mbar_arrive(&hdr->own_full[set]);
        }
      }
      const float* table = BIAS == kTable ? p.bias + static_cast<int64_t>(h) * p.bias_len : nullptr;
      const float far_bias = BIAS == kTable ? __ldg(table + p.bias_len - 1) : 0.f;
      const float slope2 = BIAS == kAlibi ? __ldg(&p.heads[h].alibi_slope2) : 0.f;
      for (int i = 0; i < p.group && ok; ++i) {
        const int64_t q_unit = static_cast<int64_t>(h * p.group + i) * p.B + b;
        for (int t = 0; t < per_head; ++t, ++issued, at.next(plan.stages)) {
          // P^T = 2^(S c + lift - L), times 2^14 and the tile's share of do''s scale;  dS^T = P^T (G^T a - delta d), with the
          // tile's share of q''s.  The rows' own numbers, lift - L and delta d, are worked out here, four a lane.
          const int64_t from = q_unit * p.tiles + tile + t, row_at = q_unit * p.pad + (tile + t) * kTile + 4 * lane;
          const int q_e = __ldg(p.q_exp + from), g_e = __ldg(p.g_exp + from);
          float4 l = __ldg(reinterpret_cast<const float4*>(p.lse + row_at)), dl = __ldg(reinterpret_cast<const float4*>(p.delta + row_at));
          const int lift = kBackwardShift + g_g - g_e;
          const int d_e = max(gradient_exponent(g_g, g_v) + max(g_q - q_e, kLeastDeviation) - lift, -126);
          float add = static_cast<float>(lift);
          if (BIAS == kTable && !near_tile(p, t * kTile, 0)) add += far_bias;
          if (BIAS == kAlibi) add -= slope2 * static_cast<float>(t * kTile + 4 * lane);
          l.x += add; l.y += add - slope2; l.z += add - 2.f * slope2; l.w += add - 3.f * slope2;
          const float d = -pow2(d_e);
          dl.x *= d; dl.y *= d; dl.z *= d; dl.w *= d;
          unsigned long long* full = &hdr->full[at.stage];
          if (issued >= plan.stages && !(ok = wait_all(&hdr->empty[at.stage], at.phase ^ 1u, p.status))) break;
          unsigned char* st = ring + at.stage * stage_bytes;
          *reinterpret_cast<float4*>(st + rows_at + 16 * lane) = l;
          *reinterpret_cast<float4*>(st + rows_at + 512 + 16 * lane) = dl;
          if (lane == 0)
            *reinterpret_cast<float2*>(st + rows_at + 1024) = make_float2(p.scale_log2 * pow2(-q_e - k_e), pow2(d_e - g_e - v_e));
          __syncwarp();
          if (lane == 0) {
            mbar_arrive_expect_tx(full, k_bytes + v_bytes);
            bulk_load(st, p.q_tiles + from * p.tile_k, k_bytes, full, keep);
            bulk_load(st + p.tile_k, p.g_tiles + from * p.tile_v, v_bytes, full, keep);
          }
        }
      }
      ok = __all_sync(0xffffffffu, ok);
      if (!ok) { ++it; break; }
    }
    if (!ok) index = 0x7fffffff;                             // (and none of the other kind)
    drain_copies(hdr, plan, ok ? it + 1 : it, issued, lane);  // (the last phase ended the list)
  } else if (warp >= kIssueWarp) {
    const int role = warp - kIssueWarp;                      // S^T; dv'; G^T and dk'
    const bool lead = elect_one();
    const uint64_t stage = stage_bytes >> 4;
    bool ok = true;
    int done = 0, sums = 0;                                  // tiles and items behind this warp
    Place at, next;
    for (int it = 0; ok; ++it) {
      const int set = set_of(plan, it);
      ok = wait_all(&hdr->own_full[set], set_phase(plan, it), p.status);
      if (!ok || hdr->item[set].tiles[0] < 0) break;
      const int total = hdr->item[set].tiles[0];
      const int rk16 = (hdr->item[set].rp_k + 15) & ~15, rv16 = (hdr->item[set].rp_v + 15) & ~15;
      const uint32_t own_at = smem_u32(own) + set * (p.tile_k + p.tile_v), ring_at = smem_u32(ring);
      if (role == 0) {
        const uint64_t dk = smem_desc(own_at, 128, rk16 << 4), q_rank = smem_desc(ring_at, 128, rk16 << 4);
        for (int g = 0; g < 2 * total && ok; ++g) {
          const int half = g & 1, behind = done + (g >> 1);  // tiles before this one
          if (!half) ok = wait_all(&hdr->full[at.stage], at.phase, p.status);
          // the buffer is free when its S^T has been read, or the P^T in its place taken in
          if (ok && behind > 0) ok = wait_all(apart ? &hdr->s_read[half] : &hdr->p_used[0][half], (behind - 1) & 1u, p.status);
          if (!ok) break;
          tc_fence_after();
          if (lead) {
            issue_rank(rk16 >> 4, tmem + cS + half * kHalf, dk, q_rank + stage * at.stage + half_of(half, rk16 << 4));
            mma_commit(&hdr->s_full[0][half]);
          }
          __syncwarp();
          if (half) at.next(plan.stages);
        }
      } else if (role == 1) {
        const uint32_t idesc = instr_desc_f16(rv16) | kMnMajorB;
        const uint64_t g_rows = smem_desc(ring_at + p.tile_k, rv16 << 4, 128);
        if (total > 0 && sums > 0) ok = wait_all(&hdr->acc_free[0], (sums - 1) & 1u, p.status);
        for (int g = 0; g < 2 * total && ok; ++g) {
          const int half = g & 1;
          if (!half) ok = wait_all(&hdr->full[at.stage], at.phase, p.status);
          if (ok) ok = wait_all(&hdr->p_full[0][half], (done + (g >> 1)) & 1u, p.status);
          if (!ok) break;
          tc_fence_after();
          if (lead) {
            issue_rows(tmem + cV, tmem + cP + half * p_step, g_rows + stage * at.stage + half_of(half, rv16 << 4), rv16 << 4, idesc, g > 0);
            mma_commit(&hdr->p_used[0][half]);
            if (half) mma_commit(&hdr->empty[at.stage]);
          }
          __syncwarp();
          if (half) at.next(plan.stages);
        }
        if (ok && lead && total > 0) mma_commit(&hdr->acc_full[0]);
        __syncwarp();
      } else {
        const uint32_t idesc = instr_desc_f16(rk16) | kMnMajorB;
        const uint64_t dv = smem_desc(own_at + p.tile_k, 128, rv16 << 4), g_rank = smem_desc(ring_at + p.tile_k, 128, rv16 << 4);
        const uint64_t q_rows = smem_desc(ring_at, rk16 << 4, 128);
        for (int g = 0; total > 0 && g < 2 * total + 2 && ok; ++g) {
          const int half = g & 1;
          if (g >= 2) {
            if (g == 2 && sums > 0) ok = wait_all(&hdr->acc_free[0], (sums - 1) & 1u, p.status);
            if (ok) ok = wait_all(&hdr->p_full[1][half], (done + ((g - 2) >> 1)) & 1u, p.status);
            if (!ok) break;
            tc_fence_after();
            if (lead) {
              issue_rows(tmem + cK, tmem + cG + half * kHalf, q_rows + stage * at.stage + half_of(half, rk16 << 4), rk16 << 4, idesc, g > 2);
              if (half) mma_commit(&hdr->empty[at.stage]);
            }
            __syncwarp();
            if (half) at.next(plan.stages);
          }
          if (g < 2 * total) {                               // (in dS^T's place: behind the product that takes it)
            if (!half) ok = wait_all(&hdr->full[next.stage], next.phase, p.status);
            if (!ok) break;
            tc_fence_after();
            if (lead) {
              issue_rank(rv16 >> 4, tmem + cG + half * kHalf, dv, g_rank + stage * next.stage + half_of(half, rv16 << 4));
              mma_commit(&hdr->g_full[half]);
            }
            __syncwarp();
            if (half) next.next(plan.stages);
          }
        }
        if (ok && lead && total > 0) mma_commit(&hdr->acc_full[0]);
        __syncwarp();
      }
      if (ok && lead) mma_commit(&hdr->own_empty[set]);
      __syncwarp();
      done += total;
      sums += total > 0;
    }
    drain(hdr, role, lead);
  } else {
    const int half = warp >> 2, row = (warp & 3) * 32 + lane;
    const uint32_t lanes = static_cast<uint32_t>((warp & 3) * 32) << 16;
    const uint32_t tS = tmem + lanes + cS + half * kHalf, tG = tmem + lanes + cG + half * kHalf, tP = tmem + lanes + cP + half * p_step;
    bool ok = true;
    int done = 0, sums = 0;
    Place at;
    for (int it = 0; ok; ++it) {
      const int set = set_of(plan, it);
      ok = wait_all(&hdr->own_full[set], set_phase(plan, it), p.status);
      if (gives_up(p, blockIdx.x == 0 && warp == 0, it, lane)) ok = false;
      if (!ok) break;
      const int total = hdr->item[set].tiles[0], per_head = hdr->item[set].tiles[1], h = hdr->item[set].h;
      if (total < 0) break;
      const int j0 = hdr->item[set].tile * kTile, key = j0 + row;
      const float* table = BIAS == kTable ? p.bias + static_cast<int64_t>(h) * p.bias_len : nullptr;
      const float slope2 = BIAS == kAlibi ? __ldg(&p.heads[h].alibi_slope2) : 0.f;
      int t = 0;
      for (int g = 0; g < total; ++g) {
        const uint32_t phase = (done + g) & 1u;
        const int far0 = t * kTile + half * kHalf - row;     // distance of the thread's first pair
        // (near: by whole tiles, as the copying warp has it)
        const bool near = BIAS == kTable && near_tile(p, t * kTile, 0), diag = t == 0;
        if (++t == per_head) t = 0;
        ok = wait_all(&hdr->full[at.stage], at.phase, p.status) && wait_all(&hdr->s_full[0][half], phase, p.status);
        if (!ok) break;
        tc_fence_after();
        const float* lse = reinterpret_cast<const float*>(ring + at.stage * stage_bytes + rows_at) + half * kHalf;
        const float2 scales = *reinterpret_cast<const float2*>(ring + at.stage * stage_bytes + rows_at + 1024);
        float c = scales.x;
        uint32_t r[2][32];
        // S of a tile with masked queries or distances of their own goes back scaled, biased and masked
        if (diag || near) {
#pragma unroll 1
          for (int k0 = 0; k0 < kHalf; k0 += 32) {
            tmem_ld32(tS + k0, r[0]);
            tmem_wait_ld_of(r[0]);
#pragma unroll
            for (int k = 0; k < 32; ++k) {
              float y = __uint_as_float(r[0][k]) * c;
              if (near) y += __ldg(table + min(max(far0 + k0 + k, 0), p.bias_len - 1));
              if (diag && half * kHalf + k0 + k < row) y = -INFINITY;
              r[0][k] = __float_as_uint(y);
            }
            tmem_st16(tS + k0, *reinterpret_cast<uint32_t(*)[16]>(&r[0][0]));
            tmem_st16(tS + k0 + 16, *reinterpret_cast<uint32_t(*)[16]>(&r[0][16]));
          }
          tmem_wait_st();
          c = 1.f;
        }
        tmem_ld32(tS, r[0]);
        tmem_ld32(tS + 32, r[1]);
        unsigned long long e[32];                            // pairs of queries
        const unsigned long long c_2 = both(c), slant = both(slope2 * static_cast<float>(row));
#pragma unroll
        for (int k = 0; k < 32; k += 2) {
          const ulonglong2 l = *reinterpret_cast<const ulonglong2*>(lse + 2 * k);
          e[k] = BIAS == kAlibi ? add2p(l.x, slant) : l.x;
          e[k + 1] = BIAS == kAlibi ? add2p(l.y, slant) : l.y;
        }
        tmem_wait_ld_of(r[0]);
        tmem_wait_ld_of(r[1]);
        tc_fence_before();
        arrive_warp(&hdr->s_read[half], lane);
        uint32_t w[2][16];
#pragma unroll
        for (int k = 0; k < 32; ++k) {
          float x, y;
          unpack2(fma2p(pair_at(r[k >> 4], k & 15), c_2, e[k]), x, y);
          x = ex2(x);
          y = ex2(y);
          w[k >> 4][k & 15] = pack_f16(x, y);
          e[k] = pack2(x, y);
        }
        if (apart && done + g > 0) {                         // dv' has taken in the P^T of the tile before
          ok = wait_all(&hdr->p_used[0][half], phase ^ 1u, p.status);
          if (!ok) break;
          tc_fence_after();
        }
        tmem_st16(tP, w[0]);
        tmem_st16(tP + 16, w[1]);
        ok = wait_all(&hdr->g_full[half], phase, p.status);
        if (!ok) {
          tmem_wait_st();
          break;
        }
        tc_fence_after();
        tmem_ld32(tG, r[0]);
        tmem_ld32(tG + 32, r[1]);
        tmem_wait_st();
        tc_fence_before();
        arrive_warp(&hdr->p_full[0][half], lane);
        tmem_wait_ld_of(r[0]);
        tmem_wait_ld_of(r[1]);
        const unsigned long long a = both(scales.y);
#pragma unroll
        for (int k = 0; k < 32; k += 2) {
          const ulonglong2 dl = *reinterpret_cast<const ulonglong2*>(lse + 128 + 2 * k);
          float x, y;
          unpack2(mul2p(e[k], fma2p(pair_at(r[k >> 4], k & 15), a, dl.x)), x, y);
          w[k >> 4][k & 15] = pack_f16(x, y);
          unpack2(mul2p(e[k + 1], fma2p(pair_at(r[k >> 4], (k & 15) + 1), a, dl.y)), x, y);
          w[k >> 4][(k & 15) + 1] = pack_f16(x, y);
        }
        tmem_st16(tG, w[0]);
        tmem_st16(tG + 16, w[1]);
        tmem_wait_st();
        tc_fence_before();
        arrive_warp(&hdr->p_full[1][half], lane);
        at.next(plan.stages);
      }
      if (!ok) break;
      done += total;
      if (total > 0) ok = wait_all(&hdr->acc_full[0], sums & 1u, p.status);
      if (!ok) break;
      tc_fence_after();
      {
        // a half's warps have half of the columns of their rows
        const Item item = hdr->item[set];
        const bool there = key < p.T, live = key < item.n;
        const int rk16 = (item.rp_k + 15) & ~15, rv16 = (item.rp_v + 15) & ~15;
        const int k_split = ((rk16 >> 4) + 1) / 2 * 16, v_split = ((rv16 >> 4) + 1) / 2 * 16;
        const int k_lo = half ? k_split : 0, k_hi = half ? rk16 : k_split, v_lo = half ? v_split : 0, v_hi = half ? rv16 : v_split;
        const int64_t at_row = static_cast<int64_t>(item.b) * p.T + key;
        __nv_bfloat16* to_k = static_cast<__nv_bfloat16*>(p.dk) + at_row * p.lr_k_width + __ldg(&p.heads[h].lr_k_off);
        __nv_bfloat16* to_v = static_cast<__nv_bfloat16*>(p.dv) + at_row * p.lr_v_width + __ldg(&p.heads[h].lr_v_off);
        if (total == 0) {
          if (there) {
            zero_row(k_lo, k_hi, item.rp_k, to_k, plan.aligned & 1);
            zero_row(v_lo, v_hi, item.rp_v, to_v, plan.aligned & 2);
          }
        } else {
          store_row(tmem + lanes + cK, k_lo, k_hi, item.rp_k, p.scale, -gradient_exponent(item.small[3], item.small[2]) - item.small[0], to_k, there, live, plan.aligned & 1);
          store_row(tmem + lanes + cV, v_lo, v_hi, item.rp_v, 1.f, -kBackwardShift - item.small[3], to_v, there, live, plan.aligned & 2);
          tc_fence_before();
          arrive_warp(&hdr->acc_free[0], lane);
          ++sums;
        }
      }
      arrive_warp(&hdr->own_empty[set], lane);
    }
  }
}

// ---------------------------------------------------------------- dq'

// An item is a tile of queries; it walks the tiles of keys that it sees: S = q' k'^T, G = do' v'^T, dS = P (G - delta),
// dq' += dS k'.  Each half tile of keys has four softmax warps of its own; a thread has a query row.  dS takes the place of S,
// which has two buffers for each half, so that the next S is there when dS is done; G is free again as soon as it has been read.
// One issuing warp has S, one dq', one G.  TMEM: S (four buffers) and G of both halves, dq'.
// The gradient of a learned bias is a sum over dS of equal distance: over diagonals.  Far tiles, whose distances share the last
// bucket, are added up whole; in the others a sum moves one lane up with every column, so that it follows its diagonal, and
// leaves the warp complete.  All of it in a fixed order, without atomics.
template <int BIAS>
__device__ __forceinline__ void dq_items(const TrainParams& p, const Plan& plan, TrHeader* hdr, unsigned char* smem, uint32_t tmem, int warp, int lane, int index, int first) {
  unsigned char* own = smem;                                 // sets of a tile of q' and one of do'
  unsigned char* ring = own + plan.sets * (p.tile_k + p.tile_v);
  const int scales_at = p.tile_k + p.tile_v, stage_bytes = scales_at + kScaleBytes;
  float* diagonals = reinterpret_cast<float*>(ring + plan.stages * stage_bytes);           // [softmax warps][96]
  constexpr uint32_t cS = 0, cG = 256, cQ = 384;             // TMEM columns of S ([half][tile & 1]), G ([half]), dq'
  if (warp == kCopyWarp) {
    const uint64_t keep = policy_evict_normal();
    bool ok = true;
    Place at;
    int issued = 0, it = 0;
    for (;; ++it) {
      const int set = set_of(plan, it);
      if (it >= plan.sets) ok = wait_all(&hdr->own_empty[set], set_phase(plan, it) ^ 1u, p.status);
      if (!ok) break;
      Item* item = &hdr->item[set];
      if (it > 0) index = next_entry(p.next + 1, lane) - first;
      if (index >= plan.items) {
        if (lane == 0) {
          item->tiles[0] = -1;
          mbar_arrive(&hdr->own_full[set]);
        }
        break;
      }
      int unit, slot;
      item_of(plan, index, unit, slot);
      const int tile = p.tiles - 1 - slot;
      const int hq = unit / p.B, b = unit - hq * p.B, h = hq / p.group, key_unit = h * p.B + b;
      const int n = kept_tokens(p, b), rp_k = __ldg(&p.heads[h].rp_k), rp_v = __ldg(&p.heads[h].rp_v);
      const int k_bytes = kTile * ((rp_k + 15) & ~15) * 2, v_bytes = kTile * ((rp_v + 15) & ~15) * 2;
      const int nt = tile * kTile < n ? tile + 1 : 0;
      const int64_t own_at = static_cast<int64_t>(unit) * p.tiles + tile, keys = static_cast<int64_t>(key_unit) * p.tiles;
      const int q_e = __ldg(p.q_exp + own_at), g_e = __ldg(p.g_exp + own_at);
      const int g_k = smallest_of(p.k_exp + keys, nt, lane), g_v = smallest_of(p.v_exp + keys, nt, lane);         // (of the tiles it walks)
      if (lane == 0) {
        item->unit = unit; item->h = h; item->b = b; item->i = hq - h * p.group;
        item->tile = tile; item->n = n; item->rp_k = rp_k; item->rp_v = rp_v;
        item->tiles[0] = nt;
        item->small[1] = g_k; item->small[2] = g_v; item->small[3] = g_e;
        unsigned char* to = own + set * (p.tile_k + p.tile_v);
        if (nt > 0) {
          mbar_arrive_expect_tx(&hdr->own_full[set], k_bytes + v_bytes);
          bulk_load(to, p.q_tiles + own_at * p.tile_k, k_bytes, &hdr->own_full[set], keep);
          bulk_load(to + p.tile_k, p.g_tiles + own_at * p.tile_v, v_bytes, &hdr->own_full[set], keep);
        } else {
          mbar_arrive(&hdr->own_full[set]);
        }
        for (int j = 0; j < nt; ++j, ++issued, at.next(plan.stages)) {
          // P = 2^(S c - L);  dS = P (G a - delta d), with the tile's share of the scale of k'.  The
          // gradient of a learned bias takes dS back to its own size, so a, d and 1 / d are powers of one exponent in range.
          const int k_e = __ldg(p.k_exp + keys + j), v_e = __ldg(p.v_exp + keys + j);
          const int d_e = max(gradient_exponent(g_e, g_v) + max(g_k - k_e, kLeastDeviation), -126);
          unsigned long long* full = &hdr->full[at.stage];
          if (issued >= plan.stages && !(ok = mbar_wait(&hdr->empty[at.stage], at.phase ^ 1u, p.status))) break;
          unsigned char* st = ring + at.stage * stage_bytes;
          *reinterpret_cast<float4*>(st + scales_at) =
              make_float4(p.scale_log2 * pow2(-q_e - k_e), pow2(d_e), pow2(d_e - g_e - v_e), pow2(-d_e));
          mbar_arrive_expect_tx(full, k_bytes + v_bytes);
          bulk_load(st, p.k_tiles + (keys + j) * p.tile_k, k_bytes, full, keep);
          bulk_load(st + p.tile_k, p.v_tiles + (keys + j) * p.tile_v, v_bytes, full, keep);
        }
      }
      ok = __all_sync(0xffffffffu, ok);
      if (!ok) { ++it; break; }
    }
    drain_copies(hdr, plan, ok ? it + 1 : it, issued, lane);  // (the last phase ended the list)
  } else if (warp >= kIssueWarp) {
    const int role = warp - kIssueWarp;                      // S; dq'; G
    const bool lead = elect_one();
    const uint64_t stage = stage_bytes >> 4;
    bool ok = true;
    int done = 0, sums = 0;                                  // tiles and items behind this warp
    Place at;
    for (int it = 0; ok; ++it) {
      const int set = set_of(plan, it);
      ok = wait_all(&hdr->own_full[set], set_phase(plan, it), p.status);
      if (!ok || hdr->item[set].tiles[0] < 0) break;
      const int nt = hdr->item[set].tiles[0];
      const int rk16 = (hdr->item[set].rp_k + 15) & ~15, rv16 = (hdr->item[set].rp_v + 15) & ~15;
      const uint32_t own_at = smem_u32(own) + set * (p.tile_k + p.tile_v), ring_at = smem_u32(ring);
      const uint64_t dq = smem_desc(own_at, 128, rk16 << 4), dg = smem_desc(own_at + p.tile_k, 128, rv16 << 4);
      const uint64_t k_rank = smem_desc(ring_at, 128, rk16 << 4), v_rank = smem_desc(ring_at + p.tile_k, 128, rv16 << 4);
      const uint64_t k_rows = smem_desc(ring_at, rk16 << 4, 128);
      const uint32_t idesc = instr_desc_f16(rk16) | kMnMajorB;
      if (role == 1 && nt > 0 && sums > 0) ok = wait_all(&hdr->acc_free[0], (sums - 1) & 1u, p.status);
      for (int j = 0; j < 2 * nt && ok; ++j) {
        const int half = j & 1, behind = done + (j >> 1), buf = behind & 1;                // tiles before this one; buffer of S
        const uint32_t tS = tmem + cS + half * 128 + buf * kHalf;
        if (!half) ok = wait_all(&hdr->full[at.stage], at.phase, p.status);
        if (role == 0) {
          if (ok && behind >= 2) ok = wait_all(&hdr->p_used[buf][half], ((behind - 2) >> 1) & 1u, p.status);     // dS taken in
          if (!ok) break;
          tc_fence_after();
          if (lead) {
            issue_rank(rk16 >> 4, tS, dq, k_rank + stage * at.stage + half_of(half, rk16 << 4));
            mma_commit(&hdr->s_full[buf][half]);
          }
        } else if (role == 1) {
          if (ok) ok = wait_all(&hdr->p_full[buf][half], (behind >> 1) & 1u, p.status);
          if (!ok) break;
          tc_fence_after();
          if (lead) {
            issue_rows(tmem + cQ, tS, k_rows + stage * at.stage + half_of(half, rk16 << 4), rk16 << 4, idesc, j > 0);
            mma_commit(&hdr->p_used[buf][half]);
            if (half) mma_commit(&hdr->empty[at.stage]);
          }
        } else {
          if (ok && behind > 0) ok = wait_all(&hdr->g_read[half], (behind - 1) & 1u, p.status);
          if (!ok) break;
          tc_fence_after();
          if (lead) {
            issue_rank(rv16 >> 4, tmem + cG + half * kHalf, dg, v_rank + stage * at.stage + half_of(half, rv16 << 4));
            mma_commit(&hdr->g_full[half]);
            if (half) mma_commit(&hdr->empty[at.stage]);
          }
        }
        __syncwarp();
        if (half) at.next(plan.stages);
      }
      if (ok && lead) {
        if (role == 1 && nt > 0) mma_commit(&hdr->acc_full[0]);
        mma_commit(&hdr->own_empty[set]);
      }
      __syncwarp();
      done += nt;
      sums += nt > 0;
    }
    drain(hdr, role, lead);
  } else {
    const int half = warp >> 2, row = (warp & 3) * 32 + lane;
    const uint32_t lanes = static_cast<uint32_t>((warp & 3) * 32) << 16;
    const uint32_t tG = tmem + lanes + cG + half * kHalf;
    const bool want = BIAS == kTable && p.dtable != nullptr;
    float* my_diagonals = diagonals + warp * 96;
    bool ok = true;
    int done = 0, sums = 0;
    Place at;
    for (int it = 0; ok; ++it) {
      const int set = set_of(plan, it);
      ok = wait_all(&hdr->own_full[set], set_phase(plan, it), p.status);
      if (gives_up(p, blockIdx.x == gridDim.x - 1 && warp == 0, it, lane)) ok = false;
      if (!ok) break;
      const int nt = hdr->item[set].tiles[0], h = hdr->item[set].h, unit = hdr->item[set].unit, tile = hdr->item[set].tile;
      if (nt < 0) break;
      const int i0 = tile * kTile, i = i0 + row;
      const float* table = BIAS == kTable ? p.bias + static_cast<int64_t>(h) * p.bias_len : nullptr;
      const float far_bias = BIAS == kTable ? __ldg(table + p.bias_len - 1) : 0.f;
      const float slope2 = BIAS == kAlibi ? __ldg(&p.heads[h].alibi_slope2) : 0.f;
      const int64_t stat = static_cast<int64_t>(unit) * p.pad + i;
      const float lse = nt > 0 ? __ldg(p.lse + stat) : 0.f, delta = nt > 0 ? __ldg(p.delta + stat) : 0.f;
      float far_sum = 0.f;                                   // dS of far tiles, this thread's
      float by_bucket[8] = {};                               // buckets lane, lane + 32, ...: this warp's
      for (int j = 0; j < nt; ++j, at.next(plan.stages)) {
        const int behind = done + j, buf = behind & 1, j0 = j * kTile + half * kHalf;
        const bool near = BIAS == kTable && near_tile(p, i0, j0), diag = j == nt - 1;
        const uint32_t tS = tmem + lanes + cS + half * 128 + buf * kHalf;
        float add = lse;
        if (BIAS == kTable && !near) add += far_bias;
        if (BIAS == kAlibi) add += slope2 * static_cast<float>(j0 - i);
        ok = wait_all(&hdr->full[at.stage], at.phase, p.status) && wait_all(&hdr->s_full[buf][half], (behind >> 1) & 1u, p.status);
        if (!ok) break;
        tc_fence_after();
        const float4 scales = *reinterpret_cast<const float4*>(ring + at.stage * stage_bytes + scales_at);
        float c = scales.x;
        uint32_t r[2][32];
        // S of a tile with masked keys or distances of their own goes back scaled, biased and masked
        if (diag || near) {
#pragma unroll 1
          for (int k0 = 0; k0 < kHalf; k0 += 32) {
            tmem_ld32(tS + k0, r[0]);
            tmem_wait_ld_of(r[0]);
#pragma unroll
            for (int k = 0; k < 32; ++k) {
              float y = __uint_as_float(r[0][k]) * c;
              if (near) y += __ldg(table + min(max(i - j0 - k0 - k, 0), p.bias_len - 1));
              if (diag && half * kHalf + k0 + k > row) y = -INFINITY;
              r[0][k] = __float_as_uint(y);
            }
            tmem_st16(tS + k0, *reinterpret_cast<uint32_t(*)[16]>(&r[0][0]));
            tmem_st16(tS + k0 + 16, *reinterpret_cast<uint32_t(*)[16]>(&r[0][16]));
          }
          tmem_wait_st();
          c = 1.f;
        }
        tmem_ld32(tS, r[0]);
        tmem_ld32(tS + 32, r[1]);
        tmem_wait_ld_of(r[0]);
        tmem_wait_ld_of(r[1]);
        uint32_t gr[2][32];                                  // G, on its way beside the exponentials (it is there before S as a rule)
        ok = wait_all(&hdr->g_full[half], behind & 1u, p.status);
        if (!ok) break;
        tc_fence_after();
        tmem_ld32(tG, gr[0]);
        tmem_ld32(tG + 32, gr[1]);
        unsigned long long e[32];                            // pairs of keys
        const unsigned long long c_2 = both(c), add_2 = both(add);
#pragma unroll
        for (int k = 0; k < 32; ++k) {
          float x, y;
          unpack2(fma2p(pair_at(r[k >> 4], k & 15), c_2, BIAS == kAlibi ? fma2p(both(slope2), pack2(2 * k, 2 * k + 1), add_2) : add_2), x, y);
          e[k] = pack2(ex2(x), ex2(y));
        }
        tmem_wait_ld_of(gr[0]);
        tmem_wait_ld_of(gr[1]);
        tc_fence_before();
        arrive_warp(&hdr->g_read[half], lane);
        const unsigned long long a_2 = both(scales.z), d_2 = both(-scales.y * delta);
        uint32_t w[2][16];
#pragma unroll
        for (int k = 0; k < 32; ++k) {
          e[k] = mul2p(e[k], fma2p(pair_at(gr[k >> 4], k & 15), a_2, d_2));
          float x, y;
          unpack2(e[k], x, y);
          w[k >> 4][k & 15] = pack_f16(x, y);
        }
        tmem_st16(tS, w[0]);
        tmem_st16(tS + 16, w[1]);
        tmem_wait_st();
        tc_fence_before();
        arrive_warp(&hdr->p_full[buf][half], lane);
        if (want) {
          const float back = scales.w;
          if (!near) {
            unsigned long long s = e[0];
#pragma unroll
            for (int k = 1; k < 32; ++k) s = add2p(s, e[k]);
            float x, y;
            unpack2(s, x, y);
            far_sum = fmaf(x + y, back, far_sum);
          } else {
            // slot 63 + (row in the warp) - column
            float s = 0.f;
#pragma unroll
            for (int k = 0; k < kHalf; ++k) {
              float x, y;
              unpack2(e[k / 2], x, y);
              s = __shfl_up_sync(0xffffffffu, s, 1);
              s = (lane == 0 ? 0.f : s) + (k & 1 ? y : x);
              if (lane == 31) my_diagonals[94 - k] = s;
            }
            if (lane < 31) my_diagonals[lane] = s;
            __syncwarp();
            const int first = i0 + (warp & 3) * 32 - j0 - 63;                              // distance of slot 0
            float last = 0.f;                                // the last bucket's, which can be most of them
            for (int x = max(p.bias_len - 1 - first, 0) + lane; x < 95; x += 32) last += my_diagonals[x];
            far_sum = fmaf(last, back, far_sum);
#pragma unroll
            for (int u = 0; u < 8; ++u) {
              const int bucket = lane + 32 * u;
              if (bucket < p.buckets - 1) {
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
      if (!ok) break;
      done += nt;
      if (want) {
#pragma unroll
        for (int d = 16; d >= 1; d >>= 1) far_sum += __shfl_xor_sync(0xffffffffu, far_sum, d);
        // (group 1: a head's units are its sequences)
        float* part = p.bias_part + ((static_cast<int64_t>(unit) * p.tiles + tile) * kSoftmaxWarps + warp) * p.buckets;
#pragma unroll
        for (int u = 0; u < 8; ++u) {
          const int bucket = lane + 32 * u;
          if (bucket < p.buckets) part[bucket] = by_bucket[u] + (bucket == p.buckets - 1 ? far_sum : 0.f);
        }
      }
      if (nt > 0) ok = wait_all(&hdr->acc_full[0], sums & 1u, p.status);
      if (!ok) break;
      tc_fence_after();
      {
        const Item item = hdr->item[set];
        const int rk16 = (item.rp_k + 15) & ~15, split = ((rk16 >> 4) + 1) / 2 * 16, lo = half ? split : 0, hi = half ? rk16 : split;
        __nv_bfloat16* to = static_cast<__nv_bfloat16*>(p.dq) + (static_cast<int64_t>(item.b) * p.T + i) * (static_cast<int64_t>(p.group) * p.lr_k_width) +
                            p.group * __ldg(&p.heads[h].lr_k_off) + item.i * item.rp_k;
        if (nt == 0) {
          if (i < p.T) zero_row(lo, hi, item.rp_k, to, plan.aligned & 1);
        } else {
          store_row(tmem + lanes + cQ, lo, hi, item.rp_k, p.scale, -gradient_exponent(item.small[3], item.small[2]) - item.small[1], to, i < p.T, i < item.n, plan.aligned & 1);
          tc_fence_before();
          arrive_warp(&hdr->acc_free[0], lane);
          ++sums;
        }
      }
      arrive_warp(&hdr->own_empty[set], lane);
    }
  }
}

// ---------------------------------------------------------------- both in one launch

// One list: the tiles of keys, then the tiles of queries.  A CTA goes over to the latter when the former are all taken, so that
// a small call has all its items running at a time (a text of 129 tokens through 32 heads: 64 and 64 items; two launches
// 30.7 us, one 24.0) and a large one does not wait for the last of the first kind.
template <int BIAS>
__global__ void __launch_bounds__(kTrThreads, 1) train_backward_kernel(const __grid_constant__ TrainParams p, const __grid_constant__ Plan plan_kv, const __grid_constant__ Plan plan_q) {
  extern __shared__ __align__(1024) unsigned char smem[];
  TrHeader* hdr = reinterpret_cast<TrHeader*>(smem);         // one for each kind of items
  const int tid = threadIdx.x, warp = __shfl_sync(0xffffffffu, tid >> 5, 0), lane = tid & 31;
  if (tid == 0) {
    set_up(hdr, 2, 3 + kSoftmaxWarps, kSoftmaxWarps / 2, 2, kSoftmaxWarps);
    set_up(hdr + 1, 2, 3 + kSoftmaxWarps, kSoftmaxWarps / 2, 1, kSoftmaxWarps);
  }
  const uint32_t tmem = begin(hdr, warp, tid);
  int index = blockIdx.x;                                    // (the copying warp's)
  dkv_items<BIAS>(p, plan_kv, hdr, smem + kHeaderBytes, tmem, warp, lane, index);
  fence_async_smem();                                        // (copies follow on plain writes)
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  dq_items<BIAS>(p, plan_q, hdr + 1, smem + kHeaderBytes, tmem, warp, lane, index - plan_kv.items, plan_kv.items);
  end(tmem, warp);
}

// Sets of own tiles and ring stages: two sets where two stages fit beside them (ranks up to 112), else one.  Rank 80, 4 x 4096
// tokens: two sets and three stages 1510 us, one set and four 1612; rank 96, 4 x 2048: two and two 512, one and three 567; a step
// of 2 x 1111 tokens with ranks 48 to 112 161 and 182.
Plan plan_of(const TrainParams& p, int units, int per_unit, size_t own, size_t stage, size_t behind, size_t* smem) {
  Plan plan{};
  const size_t room = 227 * 1024 - kHeaderBytes - behind;
  const size_t one = (room - own) / stage, two = room > 2 * own ? (room - 2 * own) / stage : 0;
  plan.sets = two >= 2 ? 2 : 1;
  plan.stages = static_cast<int>(plan.sets == 2 ? two : one);
  if (plan.stages > kMaxRing) plan.stages = kMaxRing;
  *smem = kHeaderBytes + behind + plan.sets * own + plan.stages * stage;
  if (*smem < 120 * 1024) *smem = 120 * 1024;                // one CTA per SM: it takes all of the SM's TMEM
  plan.units = units;
  plan.per_unit = per_unit;
  plan.items = units * per_unit;
  const size_t walked = static_cast<size_t>(p.tiles) * (p.tile_k + p.tile_v);               // of a unit
  const size_t chunk = (size_t(48) << 20) / walked;          // (some 50 of the 126 MB of L2)
  plan.chunk = chunk < 1 ? 1 : chunk > static_cast<size_t>(units) ? units : static_cast<int>(chunk);
  return plan;
}
int bias_of(const TrainParams& p) { return p.bias != nullptr ? kTable : p.alibi ? kAlibi : kNone; }
int on16(const void* x) { return reinterpret_cast<uintptr_t>(x) % 16 == 0 ? 1 : 0; }

}  // namespace

// (chained to the launch before it, which packs the tiles: its set-up runs beside that one's end)
cudaError_t launch_train_tc_forward(const TrainParams& p, cudaStream_t s, uint64_t* launches) {
  static size_t done[3][kMaxDevices] = {};
  const size_t k = p.tile_k, v = p.tile_v;
  size_t smem = 0;
  Plan plan = plan_of(p, p.H * p.group * p.B, (p.tiles + 1) / 2, 2 * k, k + v + kScaleBytes, 0, &smem);
  plan.aligned = on16(p.out);
  const int grid = plan.items < p.sm_count ? plan.items : p.sm_count;
  auto run = [&](auto kernel, size_t (&table)[kMaxDevices]) -> cudaError_t {
    const cudaError_t e = ensure_dynamic_smem(kernel, smem, table);
    if (e != cudaSuccess) return e;
    ++*launches;
    return launch_chained(true, kernel, dim3(grid), dim3(kTrThreads), smem, s, p, plan);
  };
  const int bias = bias_of(p);
  if (bias == kTable) return run(train_forward_kernel<kTable>, done[2]);
  if (bias == kAlibi) return run(train_forward_kernel<kAlibi>, done[1]);
  return run(train_forward_kernel<kNone>, done[0]);
}

cudaError_t launch_train_tc_backward(const TrainParams& p, cudaStream_t s, uint64_t* launches) {
  static size_t done[3][kMaxDevices] = {};
  const size_t k = p.tile_k, v = p.tile_v;
  size_t smem = 0, smem_q = 0;
  Plan plan_kv = plan_of(p, p.H * p.B, p.tiles, k + v, k + v + 1024 + kScaleBytes, 0, &smem);
  plan_kv.aligned = on16(p.dk) | on16(p.dv) << 1;
  auto in_32 = [](int rp) { return (((rp + 15) & ~15) + 31) & ~31; };
  plan_kv.apart = in_32(p.max_rp_k) + in_32(p.max_rp_v) <= 192;
  const size_t diagonals = p.dtable != nullptr ? kSoftmaxWarps * 96 * sizeof(float) : 0;
  Plan plan_q = plan_of(p, p.H * p.group * p.B, p.tiles, k + v, k + v + kScaleBytes, diagonals, &smem_q);
  plan_q.aligned = on16(p.dq);
  if (smem_q > smem) smem = smem_q;
  const int64_t items = static_cast<int64_t>(plan_kv.items) + plan_q.items;
  const int grid = items < p.sm_count ? static_cast<int>(items) : p.sm_count;
  auto run = [&](auto kernel, size_t (&table)[kMaxDevices]) -> cudaError_t {
    const cudaError_t e = ensure_dynamic_smem(kernel, smem, table);
    if (e != cudaSuccess) return e;
    ++*launches;
    return launch_chained(true, kernel, dim3(grid), dim3(kTrThreads), smem, s, p, plan_kv, plan_q);
  };
  const int bias = bias_of(p);
  if (bias == kTable) return run(train_backward_kernel<kTable>, done[2]);
  if (bias == kAlibi) return run(train_backward_kernel<kAlibi>, done[1]);
  return run(train_backward_kernel<kNone>, done[0]);
}

}  // namespace ea
