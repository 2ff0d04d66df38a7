// Attention of many query rows per K/V head (a large tree of drafted tokens, or a smaller one times its group of query
// heads) over one sequence's rows on the fifth-generation tensor cores: tcgen05 products, accumulators in TMEM.
//
// With more than 16 query rows a tile of cached rows carries more arithmetic than warp-level products deliver while it
// streams; a tcgen05 product has 128 rows of queries.  An item is a run of 128 query rows of a unit with all its cached
// rows, in tiles of 128.  The tiles of all items, laid end to end, are cut into one equal range per CTA, one CTA per SM:
// sequences of any lengths keep every SM busy to the end (with one CTA per piece of an item the last wave and the CTAs'
// starts, five tiles' worth each, cost a third).  A piece of an item that a CTA works through leaves a partial.  Roles:
//   * two threads stream K' and V' tiles by TMA (64 x 64 boxes of the cache slabs' tensor maps, 128-byte swizzle), each
//     into a ring of its own: a K' stage is free again when S(t) has read it, two products before the V' stage of the same
//     tile.  Boxes without a row of the sequence, and columns past the rank, arrive as zeros;
//   * one warp issues S(t) = Q' K'^T, another O' += P V'.  Q' (in shared memory) and P (in TMEM) enter as two 16-bit
//     parts each (leading part and remainder, 16 significant bits together), so every product is issued twice over; the
//     result carries no more than the rounding of the output.  P(t) takes the place of S(t), 16 rows at a time, so that no
//     thread overwrites what another still reads;
//   * three softmax groups of four warps, one per S buffer, a thread per query row: S(t), its softmax, P(t) V' and S(t + 3)
//     into the same columns are a chain of some 6000 cycles, of which three run at a time.  What the groups share is the
//     reference of a row, a lazy one that moves only when a score exceeds it by 8: it is handed from tile to tile once a
//     tile's maximum is known, before its exponentials.  At the end of a piece the group of its last tile writes the
//     partial, the other two load the next piece's Q' and go on.
// At most 64 (32) query rows: Q' is in the operand two (four) times, each copy takes a half (quarter) of every tile's rows
// and leaves a partial of its own; the products cost the same, a softmax thread has half (a quarter) of the work.
//
// Bound by the chain of a buffer and, where three overlap, by the products: 1330 cycles a tile of rank 80 by the tensor
// core's own rate, 1900 to 2050 measured.  16 sequences of 256 to 8192 rows, 8 heads, 128 query rows: 71 us (189 MB: 30 us of
// copy rate); 8 x 4160 rows, 32 heads, 63 query rows: 90 us.  Before: sixteen softmax warps on one tile with a block-wide
// maximum, 2700 cycles (88 and 119 us).  Not better: P and V' in halves with barriers of their own (2750 cycles: the issuing
// warps share their schedulers with the softmax, and every instruction of theirs is fetched anew); boxes of 16 columns for
// the last part of K', which leave room for more stages; L2 prefetches two tiles ahead.
// The tiles that hold drafted rows are masked per query; there the softmax warps also clear rows behind the sequence's end
// and the non-finite values of drafted rows in the V' tile (a product with a zero weight would still carry them): the
// latter are added at the end to the query rows that do see them.
// TMEM (512 columns): S[3] (128 each), O' (128).  Every wait is bounded; one that runs out ends every other one of the
// launch through the status word.
#include <cuda_bf16.h>

#include "internal.h"
#include "tc_common.cuh"

namespace ea {
namespace {

using namespace tc;

constexpr int kKeys = 128;                    // cached rows of a tile
constexpr int kAtom = kKeys * 128;            // one swizzled atom column of a tile: 128 rows x 64 elements
constexpr int kBox = 64 * 128;                // bytes of one TMA box
constexpr int kBufs = 3;                      // S buffers, each with a softmax group of its own: a thread per query row
constexpr int kSoftmax = kBufs * kTile;       // softmax threads
constexpr int kSWarp = kSoftmax / 32, kLoadWarp = kSWarp + 2;       // S, O'; K' tiles, V' tiles
constexpr int kTcThreads = kSoftmax + 128;
constexpr int kMaxStages = 6;

// A walk over the items of a CTA's range: head, sequence, run of query rows, and the tiles of it that the CTA has.
struct Walk {
  int h, b, chunk, chunks;
  int rp_k, rp_v;            // of the head
  int n_b, tiles;            // cached rows and tiles of the item
  int t, nt;                 // first tile and number of tiles of the piece
  int left;                  // tiles of the CTA's range behind this piece
  __device__ __forceinline__ void sequence(const MqDecodeParams& p) {
    n_b = p.deficit != nullptr ? p.n - __ldg(p.deficit + b) : p.n;
    tiles = (n_b + p.tail + kKeys - 1) / kKeys;
  }
  __device__ __forceinline__ void head(const MqDecodeParams& p) {
    rp_k = p.heads[h].rp_k;
    rp_v = p.heads[h].rp_v;
  }
  __device__ __forceinline__ void piece() {
    nt = min(left, tiles - t);
    left -= nt;
  }
  __device__ __forceinline__ bool next(const MqDecodeParams& p) {
    if (left == 0) return false;
    t = 0;
    if (++chunk == chunks) {
      chunk = 0;
      if (++b == p.B) {
        b = 0;
        ++h;
        head(p);
      }
      sequence(p);
    }
    piece();
    return true;
  }
};
struct __align__(16) TcHeader {
  // one arrival each
  unsigned long long k_full[kMaxStages], k_empty[kMaxStages], v_full[kMaxStages], v_empty[kMaxStages];
  unsigned long long s_full[kBufs], o_done[kBufs];                      // per S buffer
  unsigned long long ref_ready[kBufs][4];     // per S buffer and 32 query rows: the row references behind its tile
  unsigned long long p_full[kBufs], o_free, q_full, sums_ready;         // arrivals of one group, of two
  unsigned long long odd[3];                  // drafted tokens with a value that is not finite; pieces take turns
  uint32_t tmem_base;
  float ref[kTile];                           // reference of every query row behind the newest tile
  float sums[2][kBufs - 1][kTile];            // row sums of the other groups at a piece's end; pieces take turns
};
constexpr int kSingles = 4 * kMaxStages + 6 * kBufs;         // barriers with one arrival
constexpr int kHeaderBytes = 3 * 1024;
static_assert(sizeof(TcHeader) <= kHeaderBytes, "header outgrew its area");

__device__ __forceinline__ void split_pair(float x0, float x1, uint32_t& hi, uint32_t& lo) {
  hi = pack_bf16(x0, x1);
  lo = pack_bf16(x0 - __uint_as_float(hi << 16), x1 - __uint_as_float(hi & 0xffff0000u));
}
// tcgen05.wait::ld that the registers of a load under way depend on
__device__ __forceinline__ void tmem_wait_ld_of(uint32_t (&r)[16]) {
  asm volatile("tcgen05.wait::ld.sync.aligned;"
               : "+r"(r[0]), "+r"(r[1]), "+r"(r[2]), "+r"(r[3]), "+r"(r[4]), "+r"(r[5]), "+r"(r[6]), "+r"(r[7]), "+r"(r[8]), "+r"(r[9]),
                 "+r"(r[10]), "+r"(r[11]), "+r"(r[12]), "+r"(r[13]), "+r"(r[14]), "+r"(r[15])
               :
               : "memory");
}
__device__ __forceinline__ bool finite16(uint32_t bits16) { return (bits16 & 0x7f80u) != 0x7f80u; }

// One lane of the warp.  A warp that issues tcgen05 products stays together and lets this lane do it, so that descriptors live
// in uniform registers: 42 and 66 cycles for a product of 80 and 128 columns (40 and 64 are the tensor core's own), where a
// branch on the lane number, with a move into a uniform register per operand, takes 83 and 92.
__device__ __forceinline__ bool elect_one() {
  uint32_t p;
  asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(p));
  return p != 0;
}
template <int KS>
__device__ __forceinline__ void issue_s(uint32_t d, uint64_t dq, uint64_t q_part, uint64_t dk, uint32_t idesc) {
#pragma unroll
  for (int s = 0; s < KS; ++s)
#pragma unroll
    for (int part = 0; part < 2; ++part)
      mma_ss(d, dq + part * q_part + 16 * s, dk + (s >> 2) * (kAtom >> 4) + (s & 3) * 2, idesc, part > 0 || s > 0);
}

struct Ring { int q_bytes, k_stages, k_stage, v_stages, v_stage; };      // shared memory behind the header

// The walk of CTA c.  Called by whole warps (sequences of unequal lengths are searched 32 at a time).
__device__ Walk start_walk(const MqDecodeParams& p, int c, int lane) {
  Walk w;
  w.chunks = (p.rows + kTile - 1) / kTile;
  const int x = c * p.cta_tiles + min(c, p.cta_extra);
  const int per_head = static_cast<int>(p.head_tiles) * w.chunks;      // head_tiles: tiles of all sequences
  w.h = x / per_head;
  w.head(p);
  int rest = x - w.h * per_head;
  w.b = 0;
  if (p.deficit == nullptr) {
    w.sequence(p);
    const int each = w.tiles * w.chunks;
    w.b = rest / each;
    rest -= w.b * each;
  } else {
    for (int b0 = 0; b0 < p.B; b0 += 32) {
      const int tiles = b0 + lane < p.B ? (p.n - __ldg(p.deficit + b0 + lane) + p.tail + kKeys - 1) / kKeys : 0;
      int scan = tiles * w.chunks;
#pragma unroll
      for (int d = 1; d < 32; d <<= 1) {
        const int y = __shfl_up_sync(0xffffffffu, scan, d);
        if (lane >= d) scan += y;
      }
      const unsigned past = __ballot_sync(0xffffffffu, rest < scan);      // sequences that end behind the place
      if (past) {
        const int k = __ffs(past) - 1;
        if (k > 0) rest -= __shfl_sync(0xffffffffu, scan, k - 1);
        w.b = b0 + k;
        break;
      }
      rest -= __shfl_sync(0xffffffffu, scan, 31);
    }
    w.sequence(p);
  }
  w.chunk = rest / w.tiles;
  w.t = rest - w.chunk * w.tiles;
  w.left = p.cta_tiles + (c < p.cta_extra ? 1 : 0);
  w.piece();
  return w;
}

__global__ void __launch_bounds__(kTcThreads, 1) mq_tc_kernel(const __grid_constant__ MqDecodeParams p, Ring rings) {
  extern __shared__ __align__(1024) unsigned char smem[];
  TcHeader* hdr = reinterpret_cast<TcHeader*>(smem);
  unsigned char* q_tile = smem + kHeaderBytes;               // Q': leading parts, remainders; then K' stages, V' stages
  unsigned char* ring = q_tile + rings.q_bytes;
  unsigned char* v_ring = ring + rings.k_stages * rings.k_stage;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;

  if (warp == 0) tmem_alloc(&hdr->tmem_base, 512);
  if (tid < kSingles + kBufs + 3) mbar_init(&hdr->k_full[0] + tid, tid < kSingles ? 1 : tid <= kSingles + kBufs ? kTile : 2 * kTile);
  else if (tid >= 64 && tid < 64 + 3) hdr->odd[tid - 64] = 0;
  asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  chain_go();
  Walk w = start_walk(p, blockIdx.x, lane);
  chain_wait();                               // drafted rows and queries: from the kernels before
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = hdr->tmem_base;

  // Every role counts the CTA's tiles through (g): ring stages, S buffers and the phases of their barriers go on over the
  // borders of the pieces.
  if (warp >= kLoadWarp) {
    if (lane == 0) {
      const bool v_side = warp > kLoadWarp;
      unsigned char* tiles = v_side ? v_ring : ring;
      unsigned long long* full = v_side ? hdr->v_full : hdr->k_full;
      unsigned long long* empty = v_side ? hdr->v_empty : hdr->k_empty;
      const int stage = v_side ? rings.v_stage : rings.k_stage, stages = v_side ? rings.v_stages : rings.k_stages;
      const bool paged = p.pages.table != nullptr;
      const int slab_pages = paged ? p.n_max >> p.pages.shift : 1;        // (pages lie inside one slab of the pool)
      bool ok = true;
      int g = 0;
      do {
        const unsigned char* map = static_cast<const unsigned char*>(p.tmaps) + static_cast<size_t>(w.h) * 256 + (v_side ? 128 : 0);
        tensormap_acquire(map);
        const int atoms = ((v_side ? w.rp_v : w.rp_k) + 63) >> 6;
        const int row_end = w.n_b + p.tail;
        const int32_t* table = p.pages.table + static_cast<int64_t>(w.b) * p.pages.width;
        int page[2] = {0, 0};
        auto fetch = [&](int i) {             // a tile's pages, one tile ahead of their use
          for (int box = 0; paged && i < w.nt && box < 2; ++box) {
            const int r = (w.t + i) * kKeys + 64 * box;
            if (r < row_end) page[box] = __ldg(table + (r >> p.pages.shift));
          }
        };
        fetch(0);
        for (int i = 0; i < w.nt; ++i, ++g) {
          const int st = g % stages;
          if (g >= stages) ok = mbar_wait(&empty[st], (g / stages - 1) & 1u, p.status);
          if (!ok) break;
          mbar_arrive_expect_tx(&full[st], static_cast<uint32_t>(atoms * kAtom));
#pragma unroll
          for (int box = 0; box < 2; ++box) {
            const int r = (w.t + i) * kKeys + 64 * box;
            int y = 0, z = p.B;               // no row of the sequence here: outside the map, zeros
            if (r < row_end) {
              y = r; z = w.b;
              if (paged) {
                z = page[box] / slab_pages;
                y = ((page[box] - z * slab_pages) << p.pages.shift) + (r & ((1 << p.pages.shift) - 1));
              }
            }
            for (int a = 0; a < atoms; ++a) tma_load_3d(tiles + st * stage + a * kAtom + box * kBox, map, a * 64, y, z, &full[st]);
          }
          fetch(i + 1);
        }
      } while (ok && w.next(p));
      // copies in flight must land before the CTA leaves; normally their consumers have waited for them
      for (int s = 0; s < stages && s < g; ++s) mbar_wait(&full[s], ((g - 1 - s) / stages) & 1u, p.status);
    }
  } else if (warp >= kSWarp) {
    const bool lead = elect_one();
    auto wait = [&](unsigned long long* bar, uint32_t parity) { return __all_sync(0xffffffffu, mbar_wait(bar, parity, p.status)) != 0; };
    bool ok = true;
    int g = 0, piece = 0;
    if (warp == kSWarp) {
      const uint32_t idesc = instr_desc(kKeys, false);
      const uint64_t dk0 = smem_desc_sw128(smem_u32(ring), 16, 1024);
      const int stages = rings.k_stages;
      do {
        const int rpk16 = (w.rp_k + 15) & ~15;
        const uint64_t dq = smem_desc(smem_u32(q_tile), 128, (rpk16 >> 3) << 7);    // canonical tiles of 128 rows
        const uint64_t q_part = static_cast<uint64_t>(kTile * rpk16 * 2 >> 4);
        ok = wait(&hdr->q_full, piece & 1u);   // (the piece behind is announced after products that this warp issues below)
        for (int i = 0; i < w.nt && ok; ++i, ++g) {
          const int st = g % stages, buf = g % kBufs;
          ok = wait(&hdr->k_full[st], (g / stages) & 1u);    // (a stage is refilled after k_empty, which this warp commits below)
          if (ok && g >= kBufs) ok = wait(&hdr->o_done[buf], (g / kBufs - 1) & 1u);       // P(g - 3) has been read
          if (!ok) break;
          tc_fence_after();
          const uint64_t dk = dk0 + static_cast<uint64_t>(st) * (rings.k_stage >> 4);
          const uint32_t d = tmem + buf * 128;
          if (lead) {
            switch (rpk16 >> 4) {
              case 1: issue_s<1>(d, dq, q_part, dk, idesc); break;
              case 2: issue_s<2>(d, dq, q_part, dk, idesc); break;
              case 3: issue_s<3>(d, dq, q_part, dk, idesc); break;
              case 4: issue_s<4>(d, dq, q_part, dk, idesc); break;
              case 5: issue_s<5>(d, dq, q_part, dk, idesc); break;
              case 6: issue_s<6>(d, dq, q_part, dk, idesc); break;
              case 7: issue_s<7>(d, dq, q_part, dk, idesc); break;
              default: issue_s<8>(d, dq, q_part, dk, idesc); break;
            }
            mma_commit(&hdr->s_full[buf]);
            mma_commit(&hdr->k_empty[st]);
          }
          __syncwarp();
        }
        ++piece;
      } while (ok && w.next(p));
      // the last commits' arrivals must have landed before the CTA may leave
      if (ok) ok = wait(&hdr->k_empty[(g - 1) % stages], ((g - 1) / stages) & 1u);
    } else {
      const uint64_t dv0 = smem_desc_sw128(smem_u32(v_ring), kAtom, 1024);
      const int stages = rings.v_stages;
      do {
        const uint32_t idesc = instr_desc((w.rp_v + 15) & ~15, true);
        // the piece before has read O' (and the phase behind needs products that this warp issues below)
        if (piece > 0) ok = wait(&hdr->o_free, (piece - 1) & 1u);
        ++piece;
        for (int i = 0; i < w.nt && ok; ++i, ++g) {
          const int st = g % stages, buf = g % kBufs;
          // (both are filled again only after the commits below)
          ok = wait(&hdr->v_full[st], (g / stages) & 1u) && wait(&hdr->p_full[buf], (g / kBufs) & 1u);
          if (!ok) break;
          tc_fence_after();
          const uint64_t dv = dv0 + static_cast<uint64_t>(st) * (rings.v_stage >> 4);
          const uint32_t pa = tmem + buf * 128;
          if (lead) {
#pragma unroll
            for (int s = 0; s < kKeys / 16; ++s)
#pragma unroll
              for (int part = 0; part < 2; ++part)
                mma_ts(tmem + kBufs * 128, pa + 16 * s + 8 * part, dv + s * (2048 >> 4), idesc, i > 0 || part > 0 || s > 0);
            mma_commit(&hdr->o_done[buf]);
            mma_commit(&hdr->v_empty[st]);
          }
          __syncwarp();
        }
      } while (ok && w.next(p));
      if (ok) ok = wait(&hdr->v_empty[(g - 1) % stages], ((g - 1) / stages) & 1u);
    }
  } else {
    // ------------------------------------------------------------------ softmax: a group per S buffer, a thread per query row
    const int mine = warp >> 2, quad = warp & 3, row = quad * 32 + lane, prev = mine == 0 ? kBufs - 1 : mine - 1;
    const uint32_t lane_base = static_cast<uint32_t>(quad * 32) << 16;
    const uint32_t tS = tmem + lane_base + mine * 128, tO = tmem + lane_base + kBufs * 128;
    // At most 64 (32) query rows: the operand holds them two (four) times, and a copy looks after a half (quarter) of every
    // tile's rows, with a reference, a sum and a partial of its own.
    const int span = kKeys / p.copies, copy = row / span, c_lo = copy * span, c_hi = c_lo + span;       // (span: rows of a copy too)
    const int q_row = p.copies > 1 ? row - copy * span : row;
    auto wait = [&](unsigned long long* bar, uint32_t parity) { return __all_sync(0xffffffffu, mbar_wait(bar, parity, p.status)) != 0; };
    // the drafted tokens that this thread's row sees
    auto load_mask = [&](const Walk& w) -> uint64_t {
      const int my_row = w.chunk * kTile + q_row;
      const uint64_t seen = my_row < p.rows ? __ldg(p.mask + static_cast<int64_t>(w.b) * p.tokens + my_row / p.group) : 0;
      return p.tokens < 64 ? seen & ((1ull << p.tokens) - 1) : seen;
    };
    // Q' of a piece as canonical tiles, 16 channels at a time, by two of the groups (slots 0 and 1); they announce it
    auto load_q = [&](const Walk& w, int slot) {
      const int rp_k = w.rp_k, rpk16 = (rp_k + 15) & ~15, group = (rpk16 >> 3) << 7;
      const int my_row = w.chunk * kTile + q_row;
      const float* src = p.qp + ((static_cast<int64_t>(w.h) * p.B + w.b) * p.rows + my_row) * p.q_stride;
#pragma unroll 1
      for (int c0 = 16 * slot; c0 < rpk16; c0 += 32) {
        float4 x[4];
#pragma unroll
        for (int j = 0; j < 4; ++j)
          x[j] = my_row < p.rows && c0 + 8 * (j >> 1) < rp_k ? __ldg(reinterpret_cast<const float4*>(src + c0) + j) : make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
        for (int half = 0; half < 2; ++half) {
          uint4 hi, lo;
          split_pair(x[2 * half].x, x[2 * half].y, hi.x, lo.x);
          split_pair(x[2 * half].z, x[2 * half].w, hi.y, lo.y);
          split_pair(x[2 * half + 1].x, x[2 * half + 1].y, hi.z, lo.z);
          split_pair(x[2 * half + 1].z, x[2 * half + 1].w, hi.w, lo.w);
          unsigned char* at = q_tile + chunk_off(row, (c0 >> 3) + half, group);
          *reinterpret_cast<uint4*>(at) = hi;
          *reinterpret_cast<uint4*>(at + kTile * rpk16 * 2) = lo;
        }
      }
      fence_async_smem();
    };
    bool ok = true;
    int g0 = 0;                                              // the CTA's tiles in front of this piece
    uint64_t seen = load_mask(w);
    if (mine < 2) {
      load_q(w, mine);
      mbar_arrive(&hdr->q_full);
    }
    for (int piece = 0;; ++piece) {
      const int nt = w.nt, n_b = w.n_b, rp_v = w.rp_v, rpv16 = (rp_v + 15) & ~15;
      const int live = min(kTile, p.rows - w.chunk * kTile);
      const bool idle = (q_row & ~31) >= live;               // no query in these 32 rows
      float m = -INFINITY, l = 0.f;                          // reference at this thread's newest tile, sum against it
      for (int i = (mine + kBufs - g0 % kBufs) % kBufs; i < nt; i += kBufs) {
        const int g = g0 + i;
        ok = wait(&hdr->s_full[mine], (g / kBufs) & 1u);
        if (!ok) break;
        tc_fence_after();
        const int key0 = (w.t + i) * kKeys;                  // first row of the tile
        const bool special = key0 + kKeys > n_b;
        // the rows of columns j .. j + 31 that this query sees, one bit each
        auto open = [&](int j) -> uint32_t {
          const int s0 = key0 + j - n_b;                    // drafted token of the first one; cached rows lie below 0
          if (s0 >= 0) return s0 < 64 ? static_cast<uint32_t>(seen >> s0) : 0u;
          return s0 <= -32 ? ~0u : ((1u << -s0) - 1) | static_cast<uint32_t>(seen << -s0);
        };
        float top = -INFINITY;
        if (special && !idle) {                              // masked scores become -inf
#pragma unroll 1
          for (int j = c_lo; j < c_hi; j += 32) {
            const uint32_t bits = open(j);
            if (!__any_sync(0xffffffffu, bits != ~0u)) continue;
            uint32_t r[32];
            tmem_ld16(tS + j, *reinterpret_cast<uint32_t(*)[16]>(&r[0]));
            tmem_ld16(tS + j + 16, *reinterpret_cast<uint32_t(*)[16]>(&r[16]));
            tmem_wait_ld();
#pragma unroll
            for (int c = 0; c < 32; ++c)
              if (!((bits >> c) & 1)) r[c] = 0xff800000u;
            tmem_st16(tS + j, *reinterpret_cast<uint32_t(*)[16]>(&r[0]));
            tmem_st16(tS + j + 16, *reinterpret_cast<uint32_t(*)[16]>(&r[16]));
          }
          tmem_wait_st();
        }
        if (!idle) {
          float mx[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll 1
          for (int j = c_lo; j < c_hi; j += 32) {
            uint32_t r[32];
            tmem_ld16(tS + j, *reinterpret_cast<uint32_t(*)[16]>(&r[0]));
            tmem_ld16(tS + j + 16, *reinterpret_cast<uint32_t(*)[16]>(&r[16]));
            tmem_wait_ld();
#pragma unroll
            for (int c = 0; c < 32; c += 8)
#pragma unroll
              for (int k = 0; k < 4; ++k) mx[k] = max3(mx[k], __uint_as_float(r[c + 2 * k]), __uint_as_float(r[c + 2 * k + 1]));
          }
          top = fmaxf(fmaxf(mx[0], mx[1]), fmaxf(mx[2], mx[3]));
        }
        // The reference of the row: from the tile before, raised here, handed on to the tile behind.
        if (g > 0) ok = wait(&hdr->ref_ready[prev][quad], ((g - 1) / kBufs) & 1u);
        if (!ok) break;
        if (i == 0 && row == 0) hdr->odd[(piece + 1) % 3] = 0;                // (last read two pieces ago)
        const float before = i > 0 ? hdr->ref[row] : -INFINITY;
        const bool raise = top > before + 8.f;
        const float now = raise ? top : before;
        hdr->ref[row] = now;
        __syncwarp();
        if (lane == 0) mbar_arrive(&hdr->ref_ready[mine][quad]);
        if (now != m) {
          l *= ex2(m - now);                                 // (0 before the first row)
          m = now;
        }
        if (i > 0 && __any_sync(0xffffffffu, raise)) {       // rescale O'
          ok = wait(&hdr->o_done[prev], ((g - 1) / kBufs) & 1u);
          if (!ok) break;
          tc_fence_after();
          const float alpha = raise ? ex2(before - now) : 1.f;
#pragma unroll 1
          for (int c0 = 0; c0 < rpv16; c0 += 16) {
            uint32_t o[16];
            tmem_ld16(tO + c0, o);
            tmem_wait_ld();
#pragma unroll
            for (int j = 0; j < 16; ++j) o[j] = __float_as_uint(__uint_as_float(o[j]) * alpha);
            tmem_st16(tO + c0, o);
          }
        }
        // Exponentials against the reference and their sum.  P takes S's place 16 rows at a time: the leading parts go into
        // the first eight of their columns, the remainders into the other eight.
        if (!idle) {
          float sum0 = 0.f, sum1 = 0.f;
          const float neg = m == -INFINITY ? 0.f : -m;
          // Loops small enough to stay at hand: an instruction that has to be fetched costs some 25 cycles.  The next 16
          // columns come in once these are in other registers.
          uint32_t r[16], x[16];
          tmem_ld16(tS + c_lo, r);
          tmem_wait_ld();
#pragma unroll 1
          for (int j = c_lo; j < c_hi; j += 16) {
            float y[16];
#pragma unroll
            for (int c = 0; c < 16; c += 2) fma2(y[c], y[c + 1], __uint_as_float(r[c]), __uint_as_float(r[c + 1]), 1.f, neg);
            if (j + 16 < c_hi) tmem_ld16(tS + j + 16, r);
#pragma unroll
            for (int c = 0; c < 16; c += 2) {
              const float e0 = ex2(y[c]), e1 = ex2(y[c + 1]);
              add2(sum0, sum1, e0, e1);
              split_pair(e0, e1, x[c / 2], x[8 + c / 2]);
            }
            tmem_st16(tS + j, x);
            tmem_wait_ld_of(r);
          }
          l += sum0 + sum1;
          if (p.copies > 1) {                                // the other copies' rows of the tile
#pragma unroll
            for (int c = 0; c < 16; ++c) x[c] = 0u;
#pragma unroll 1
            for (int j = 0; j < kKeys; j += 16)
              if (j < c_lo || j >= c_hi) tmem_st16(tS + j, x);
          }
        }
        if (special) {
          // the V' tile: rows behind the end cleared, values of drafted rows that are not finite cleared and noted
          // (A wait tells a phase from its neighbours only.  S(g) says that tile g - 3 has been used up; with two stages the
          // one that this stage held before, g - 2, may still be on its way.)
          const int st = g % rings.v_stages, held = g - rings.v_stages;
          if (held >= 0 && rings.v_stages < kBufs) ok = wait(&hdr->o_done[held % kBufs], (held / kBufs) & 1u);
          if (ok) ok = wait(&hdr->v_full[st], (g / rings.v_stages) & 1u);
          if (!ok) break;
          const int r_log = key0 + row, row_end = n_b + p.tail;
          if (r_log >= n_b) {
            unsigned char* v_row = v_ring + st * rings.v_stage;
            const int pieces16 = 8 * ((rpv16 + 63) >> 6);
            auto piece_at = [&](int c) { return reinterpret_cast<uint4*>(v_row + (c >> 3) * kAtom + sw128_off(row, c & 7)); };
            if (r_log >= row_end) {
#pragma unroll 1
              for (int c = 0; c < pieces16; ++c) *piece_at(c) = make_uint4(0u, 0u, 0u, 0u);
            } else {
              uint32_t odd = 0;                              // bits 15 and 31: an exponent of ones
#pragma unroll 1
              for (int c = 0; c < pieces16; ++c) {
                const uint4 v = *piece_at(c);
                odd |= ((v.x & 0x7f807f80u) + 0x00800080u) | ((v.y & 0x7f807f80u) + 0x00800080u) | ((v.z & 0x7f807f80u) + 0x00800080u) |
                       ((v.w & 0x7f807f80u) + 0x00800080u);
              }
              if (odd & 0x80008000u) {
#pragma unroll 1
                for (int c = 0; c < 4 * pieces16; ++c) {
                  uint32_t* at = reinterpret_cast<uint32_t*>(piece_at(c >> 2)) + (c & 3);
                  uint32_t u = *at;
                  if (!finite16(u)) u &= 0xffff0000u;
                  if (!finite16(u >> 16)) u &= 0x0000ffffu;
                  *at = u;
                }
                atomicOr(&hdr->odd[piece % 3], 1ull << (r_log - n_b));
              }
            }
          }
          fence_async_smem();
        }
        tmem_wait_st();
        tc_fence_before();
        mbar_arrive(&hdr->p_full[mine]);
      }
      if (!ok) break;
      // ---- the piece's end.  The group of the last tile writes the partial; the other two load the next piece's Q' and go on.
      // (They have handed over their sums and read the reference before they announce Q', and no product of the next piece
      // comes before that: sums and references are not overwritten too early, and no barrier is two phases ahead of a waiter.)
      const int last = g0 + nt - 1, last_buf = last % kBufs;
      const uint32_t last_phase = (last / kBufs) & 1u;
      g0 += nt;
      Walk next = w;
      const bool more = next.next(p);
      if (mine != last_buf) {
        const int slot = (mine - last_buf + 2) % kBufs;
        ok = wait(&hdr->s_full[last_buf], last_phase);       // the last product that reads this piece's Q'
        if (!ok) break;
        if (more) load_q(next, slot);
        ok = wait(&hdr->ref_ready[last_buf][quad], last_phase);
        if (!ok) break;
        const float top = hdr->ref[row];
        hdr->sums[piece & 1][slot][row] = top == m ? l : l * ex2(m - top);
        mbar_arrive(&hdr->sums_ready);
        if (more) mbar_arrive(&hdr->q_full);
      } else {
        // (The next piece's sums cannot complete before this: either this group hands over some of them itself, or it has
        // that piece's last tile, whose reference the others wait for before they hand over theirs.)
        ok = wait(&hdr->sums_ready, piece & 1u) && wait(&hdr->o_done[last_buf], last_phase);
        if (!ok) break;
        tc_fence_after();
        const uint64_t odd = hdr->odd[piece % 3] & seen;
        const int64_t item = (static_cast<int64_t>(w.h) * p.B + w.b) * w.chunks + w.chunk;
        float* part = p.partials + ((item + blockIdx.x) * p.slot_rows + row) * p.part_stride;
        if (q_row < live) {
          part[0] = m;
          part[1] = l + (hdr->sums[piece & 1][0][row] + hdr->sums[piece & 1][1][row]);
        }
#pragma unroll 1
        for (int c0 = 0; c0 < rpv16; c0 += 16) {
          uint32_t o[16];
          tmem_ld16(tO + c0, o);
          tmem_wait_ld();
          if (q_row >= live) continue;
#pragma unroll
          for (int j = 0; j < 16; j += 4)
            if (c0 + j < rp_v)
              *reinterpret_cast<uint4*>(part + 4 + c0 + j) = make_uint4(o[j], o[j + 1], o[j + 2], o[j + 3]);
          for (uint64_t rest = odd; rest; rest &= rest - 1) {              // (rare) values that are not finite, of rows this query sees
            const int r_log = n_b + __ffsll(static_cast<long long>(rest)) - 1, column = r_log & (kKeys - 1);
            if (column < c_lo || column >= c_hi) continue;               // another copy's
            const int64_t at = physical_row(p.pages, w.b, p.n_max, r_log);
            const uint16_t* v = reinterpret_cast<const uint16_t*>(p.cache + p.heads[w.h].v_off) + at * rp_v;
#pragma unroll 1
            for (int c = c0; c < min(c0 + 16, rp_v); ++c)
              if (!finite16(v[c])) part[4 + c] += __uint_as_float(static_cast<uint32_t>(v[c]) << 16);
          }
        }
        tc_fence_before();
        mbar_arrive(&hdr->o_free);                           // the next piece's products may overwrite O'
      }
      if (!more) break;
      w = next;
      seen = load_mask(w);
    }
  }
  tc_fence_before();
  __syncthreads();
  if (warp == 0) tmem_dealloc(tmem, 512);
}

}  // namespace

cudaError_t launch_mq_tc(const MqDecodeParams& p, int max_rp_k, int max_rp_v, cudaStream_t s, uint64_t* launches) {
  // three K' stages and two V' stages always fit (Q' 64 KB and 16 KB atoms at full rank); narrower ranks have more
  Ring r{2 * kTile * ((max_rp_k + 15) & ~15) * 2, 3, ((max_rp_k + 63) >> 6) * kAtom, 2, ((max_rp_v + 63) >> 6) * kAtom};
  const int room = 227 * 1024 - kHeaderBytes - r.q_bytes;
  for (bool more = true; more;) {
    more = false;
    if (r.v_stages < r.k_stages && r.k_stages * r.k_stage + (r.v_stages + 1) * r.v_stage <= room) { ++r.v_stages; more = true; }
    else if (r.k_stages < kMaxStages && (r.k_stages + 1) * r.k_stage + r.v_stages * r.v_stage <= room) { ++r.k_stages; more = true; }
  }
  const size_t smem = kHeaderBytes + r.q_bytes + static_cast<size_t>(r.k_stages) * r.k_stage + static_cast<size_t>(r.v_stages) * r.v_stage;
  static size_t configured[kMaxDevices] = {};
  const cudaError_t e = ensure_dynamic_smem(mq_tc_kernel, smem, configured);
  if (e != cudaSuccess) return e;
  ++*launches;
  return launch_chained(p.chained != 0, mq_tc_kernel, p.grid, kTcThreads, smem, s, p, r);
}

}  // namespace ea
