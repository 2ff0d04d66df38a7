// Attention of many query rows per K/V head (a large tree of drafted tokens, or a smaller one times its group of query
// heads) over one sequence's rows on the fifth-generation tensor cores: tcgen05 products, accumulators in TMEM.
//
// With more than 16 query rows a tile of cached rows carries more arithmetic than warp-level products deliver while it
// streams; a tcgen05 product has 128 rows of queries.  An item is a run of 128 query rows of a unit with all its cached
// rows, in tiles of 128.  The tiles of all items, laid end to end, are cut into one equal range per CTA, one CTA per SM:
// sequences of any lengths keep every SM busy to the end (with one CTA per piece of an item the last wave and the CTAs'
// starts, five tiles' worth each, cost a third).  A piece of an item that a CTA works through leaves a partial; the loaders
// and the issuer of S run on into the next piece while the softmax warps finish the last one.  Roles:
//   * two threads stream K' and V' tiles by TMA (64 x 64 boxes of the cache slabs' tensor maps, 128-byte swizzle), each
//     into a ring of its own: a K' stage is free again when S(t) has read it, two products before the V' stage of the same
//     tile (with one ring for both the issuer of S waited 1400 cycles a tile for the copies).  Boxes without a row of the sequence, and columns past the rank, arrive as zeros;
//   * one thread issues S(t) = Q' K'^T, another O' += P V'.  Q' (in shared memory) and P (in TMEM) enter as two 16-bit
//     parts each (leading part and remainder, 16 significant bits together), so every product is issued twice over; the
//     result carries no more than the rounding of the output.  P(t) takes the place of S(t): its leading part the first 64
//     columns, the remainder the other 64.  S has three buffers: S(t), its softmax, P(t) V' and S(t + 3) into the same
//     columns are a chain of some 5900 cycles, of which two tiles at a time left the products idle a third of the time;
//   * sixteen softmax warps, four threads per query row (32 rows of the tile each): a lazy reference that moves only when a
//     score exceeds it by 8, agreed through one reducing barrier that also orders the loads of S before the stores of P.
//     (Eight warps were the bound: 2600 cycles a tile against 2300 of the products.)
// The tiles that hold drafted rows are masked per query; there the softmax warps also clear rows behind the sequence's end
// and the non-finite values of drafted rows in the V' tile (a product with a zero weight would still carry them): the
// latter are added at the end to the query rows that do see them.
// TMEM (512 columns): S[3] (128 each), O' (128).  Every wait is bounded.
#include <cuda_bf16.h>

#include "internal.h"
#include "tc_common.cuh"

namespace ea {
namespace {

using namespace tc;

constexpr int kKeys = 128;                    // cached rows of a tile
constexpr int kAtom = kKeys * 128;            // one swizzled atom column of a tile: 128 rows x 64 elements
constexpr int kBox = 64 * 128;                // bytes of one TMA box
constexpr int kParts = 4, kPart = kKeys / kParts;            // threads per query row, rows of a tile each looks after
constexpr int kSoftmax = kParts * kTile;      // softmax threads
constexpr int kSWarp = kSoftmax / 32, kPvWarp = kSWarp + 1, kLoadWarp = kSWarp + 2;   // ... and the last: K' tiles, V' tiles
constexpr int kTcThreads = kSoftmax + 128;
constexpr int kMaxStages = 6;
constexpr int kBufs = 3;                      // S buffers

// A walk over the items of a CTA's range: head, sequence, run of query rows, and the tiles of it that the CTA has.
struct Walk {
  int h, b, chunk, chunks;
  int rp_k, rp_v;            // of the head
  int n_b, tiles;            // cached rows and tiles of the item
  int t, nt;                 // first tile and number of tiles of the piece
  int64_t left;              // tiles of the CTA's range behind this piece
  __device__ __forceinline__ void sequence(const MqDecodeParams& p) {
    n_b = p.deficit != nullptr ? p.n - __ldg(p.deficit + b) : p.n;
    tiles = (n_b + p.tail + kKeys - 1) / kKeys;
  }
  __device__ __forceinline__ void head(const MqDecodeParams& p) {
    rp_k = p.heads[h].rp_k;
    rp_v = p.heads[h].rp_v;
  }
  __device__ __forceinline__ void piece() {
    nt = static_cast<int>(left < tiles - t ? left : tiles - t);
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
  unsigned long long k_full[kMaxStages], k_empty[kMaxStages], v_full[kMaxStages], v_empty[kMaxStages];
  unsigned long long q_full;
  unsigned long long s_full[kBufs], p_full[kBufs], o_done[kBufs];       // per S buffer
  unsigned long long odd[2];                  // drafted tokens with a value that is not finite; pieces take turns
  uint32_t tmem_base;
  int abort_flag;
  Walk walk[3];                               // the softmax warps' walk (they have no registers to spare for it): the piece
  int more[3];                                //   before, which some still finish, this one and the next
  float exch[kParts][kTile];                  // row maxima (main loop), row sums (epilogue)
};
constexpr int kHeaderBytes = 3072;
static_assert(sizeof(TcHeader) <= kHeaderBytes, "header outgrew its area");

__device__ __forceinline__ bool softmax_barrier_or(bool pred) {    // the softmax threads
  uint32_t out;
  asm volatile(
      "{\n\t.reg .pred p, q;\n\t"
      "setp.ne.u32 q, %1, 0;\n\t"
      "bar.red.or.pred p, 1, %2, q;\n\t"
      "selp.u32 %0, 1, 0, p;\n\t}"
      : "=r"(out)
      : "r"(pred ? 1u : 0u), "n"(kSoftmax)
      : "memory");
  return out != 0;
}
__device__ __forceinline__ void tmem_st8(uint32_t taddr, const uint32_t (&r)[8]) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%8], {%0, %1, %2, %3, %4, %5, %6, %7};" ::"r"(r[0]), "r"(r[1]), "r"(r[2]),
               "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(taddr)
               : "memory");
}
__device__ __forceinline__ void split_pair(float x0, float x1, uint32_t& hi, uint32_t& lo) {
  hi = pack_bf16(x0, x1);
  lo = pack_bf16(x0 - __uint_as_float(hi << 16), x1 - __uint_as_float(hi & 0xffff0000u));
}
__device__ __forceinline__ bool finite16(uint32_t bits16) { return (bits16 & 0x7f80u) != 0x7f80u; }

template <int KS>
__device__ __forceinline__ void issue_s(uint32_t d, uint64_t dq, uint64_t q_part, uint64_t dk, uint32_t idesc) {
#pragma unroll
  for (int part = 0; part < 2; ++part)
#pragma unroll
    for (int s = 0; s < KS; ++s)
      mma_ss(d, dq + part * q_part + 16 * s, dk + (s >> 2) * (kAtom >> 4) + (s & 3) * 2, idesc, part > 0 || s > 0);
}

struct Ring { int q_bytes, k_stages, k_stage, v_stages, v_stage; };      // shared memory behind the header

// The walk of CTA c.  Called by whole warps (sequences of unequal lengths are searched 32 at a time).
__device__ Walk start_walk(const MqDecodeParams& p, int c, int lane) {
  Walk w;
  w.chunks = (p.rows + kTile - 1) / kTile;
  const int64_t x = c * p.total_tiles / p.grid, end = (c + 1) * p.total_tiles / p.grid;
  const int64_t per_head = p.head_tiles * w.chunks;          // head_tiles: tiles of all sequences
  w.h = static_cast<int>(x / per_head);
  w.head(p);
  int64_t rest = x - w.h * per_head;
  w.b = 0;
  if (p.deficit == nullptr) {
    w.sequence(p);
    const int64_t each = static_cast<int64_t>(w.tiles) * w.chunks;
    w.b = static_cast<int>(rest / each);
    rest -= w.b * each;
  } else {
    for (int b0 = 0; b0 < p.B; b0 += 32) {
      const int tiles = b0 + lane < p.B ? (p.n - __ldg(p.deficit + b0 + lane) + p.tail + kKeys - 1) / kKeys : 0;
      int64_t scan = static_cast<int64_t>(tiles) * w.chunks;
#pragma unroll
      for (int d = 1; d < 32; d <<= 1) {
        const int64_t y = __shfl_up_sync(0xffffffffu, scan, d);
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
  w.chunk = static_cast<int>(rest / w.tiles);
  w.t = static_cast<int>(rest - static_cast<int64_t>(w.chunk) * w.tiles);
  w.left = end - x;
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
  if (tid == 0) {
    for (int s = 0; s < kMaxStages; ++s) {
      mbar_init(&hdr->k_full[s], 1);
      mbar_init(&hdr->k_empty[s], 1);
      mbar_init(&hdr->v_full[s], 1);
      mbar_init(&hdr->v_empty[s], 1);
    }
    mbar_init(&hdr->q_full, kSoftmax);
    for (int i = 0; i < kBufs; ++i) {
      mbar_init(&hdr->s_full[i], 1);
      mbar_init(&hdr->p_full[i], kSoftmax);
      mbar_init(&hdr->o_done[i], 1);
    }
    hdr->odd[0] = hdr->odd[1] = 0;
    hdr->abort_flag = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  chain_go();
  Walk w = start_walk(p, blockIdx.x, lane);
  chain_wait();                               // drafted rows and queries: from the kernels before
  if (tid == 0) {
    hdr->walk[0] = w;
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = hdr->tmem_base;
  volatile int* abort_flag = &hdr->abort_flag;

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
          if (g >= stages) ok = mbar_wait(&empty[st], (g / stages - 1) & 1u, p.status) && !*abort_flag;
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
      if (!ok) *abort_flag = 1;
      // copies in flight must land before the CTA leaves; normally their consumers have waited for them
      for (int s = 0; s < stages && s < g; ++s) mbar_wait(&full[s], ((g - 1 - s) / stages) & 1u, p.status);
    }
  } else if (warp == kSWarp) {
    if (lane == 0) {
      const uint32_t idesc = instr_desc(kKeys, false);
      const uint64_t dk0 = smem_desc_sw128(smem_u32(ring), 16, 1024);
      const int stages = rings.k_stages;
      bool ok = true;
      int g = 0, piece = 0;
      do {
        const int rpk16 = (w.rp_k + 15) & ~15;
        const uint64_t dq = smem_desc(smem_u32(q_tile), 128, (rpk16 >> 3) << 7);    // canonical tiles of 128 rows
        const uint64_t q_part = static_cast<uint64_t>(kTile * rpk16 * 2 >> 4);
        ok = mbar_wait(&hdr->q_full, piece & 1u, p.status);
        for (int i = 0; i < w.nt && ok; ++i, ++g) {
          const int st = g % stages, buf = g % kBufs;
          ok = mbar_wait(&hdr->k_full[st], (g / stages) & 1u, p.status);
          if (ok && g >= kBufs) ok = mbar_wait(&hdr->o_done[buf], (g / kBufs - 1) & 1u, p.status);    // P(g - 3) has been read
          ok = ok && !*abort_flag;
          if (!ok) break;
          tc_fence_after();
          const uint64_t dk = dk0 + static_cast<uint64_t>(st) * (rings.k_stage >> 4);
          const uint32_t d = tmem + buf * 128;
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
        ++piece;
      } while (ok && w.next(p));
      // the last commits' arrivals must have landed before the CTA may leave
      if (ok) ok = mbar_wait(&hdr->k_empty[(g - 1) % stages], ((g - 1) / stages) & 1u, p.status);
      if (!ok) *abort_flag = 1;
    }
  } else if (warp == kPvWarp) {
    if (lane == 0) {
      const uint64_t dv0 = smem_desc_sw128(smem_u32(v_ring), kAtom, 1024);
      const int stages = rings.v_stages;
      bool ok = true;
      int g = 0;
      do {
        const uint32_t idesc = instr_desc((w.rp_v + 15) & ~15, true);
        for (int i = 0; i < w.nt && ok; ++i, ++g) {
          const int st = g % stages, buf = g % kBufs;
          ok = mbar_wait(&hdr->p_full[buf], (g / kBufs) & 1u, p.status) && mbar_wait(&hdr->v_full[st], (g / stages) & 1u, p.status) &&
               !*abort_flag;
          if (!ok) break;
          tc_fence_after();
          const uint64_t dv = dv0 + static_cast<uint64_t>(st) * (rings.v_stage >> 4);
          const uint32_t pa = tmem + buf * 128;
#pragma unroll
          for (int part = 0; part < 2; ++part)
#pragma unroll
            for (int s = 0; s < kKeys / 16; ++s)
              mma_ts(tmem + kBufs * 128, pa + 64 * part + 8 * s, dv + s * (2048 >> 4), idesc, i > 0 || part > 0 || s > 0);
          mma_commit(&hdr->o_done[buf]);
          mma_commit(&hdr->v_empty[st]);
        }
      } while (ok && w.next(p));
      if (ok) ok = mbar_wait(&hdr->v_empty[(g - 1) % stages], ((g - 1) / stages) & 1u, p.status);
      if (!ok) *abort_flag = 1;
    }
  } else {
    // ------------------------------------------------------------------ softmax: four threads per query row
    const int part_id = warp >> 2, row = (warp & 3) * 32 + lane;
    const uint32_t lane_base = static_cast<uint32_t>((warp & 3) * 32) << 16;
    const uint32_t tO = tmem + lane_base + kBufs * 128;
    bool ok = true;
    // Q' of a piece as canonical tiles, a step of 16 channels at a time; returns the drafted tokens this thread's row sees
    auto load_q = [&](const Walk& w) -> uint64_t {
      const int rp_k = w.rp_k, rpk16 = (rp_k + 15) & ~15, group = (rpk16 >> 3) << 7;
      const int my_row = w.chunk * kTile + row;
      const bool there = my_row < p.rows;
      const float* src = p.qp + ((static_cast<int64_t>(w.h) * p.B + w.b) * p.rows + my_row) * p.q_stride;
      uint64_t seen = there ? __ldg(p.mask + static_cast<int64_t>(w.b) * p.tokens + my_row / p.group) : 0;
      float4 x[2][4];
#pragma unroll
      for (int k = 0; k < 2; ++k)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const int c = 16 * (part_id + kParts * k) + 4 * j;
          x[k][j] = there && c < rp_k ? __ldg(reinterpret_cast<const float4*>(src + c)) : make_float4(0.f, 0.f, 0.f, 0.f);
        }
      if (p.tokens < 64) seen &= (1ull << p.tokens) - 1;
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        const int c0 = 16 * (part_id + kParts * k);
        if (c0 < rpk16) {
#pragma unroll
          for (int half = 0; half < 2; ++half) {
            uint4 hi, lo;
            split_pair(x[k][2 * half].x, x[k][2 * half].y, hi.x, lo.x);
            split_pair(x[k][2 * half].z, x[k][2 * half].w, hi.y, lo.y);
            split_pair(x[k][2 * half + 1].x, x[k][2 * half + 1].y, hi.z, lo.z);
            split_pair(x[k][2 * half + 1].z, x[k][2 * half + 1].w, hi.w, lo.w);
            unsigned char* at = q_tile + chunk_off(row, (c0 >> 3) + half, group);
            *reinterpret_cast<uint4*>(at) = hi;
            *reinterpret_cast<uint4*>(at + kTile * rpk16 * 2) = lo;
          }
        }
      }
      fence_async_smem();
      mbar_arrive(&hdr->q_full);
      return seen;
    };
    int g = 0, now = 0;                                      // now: this piece's place in hdr->walk
    uint64_t seen = load_q(hdr->walk[0]);
    for (int piece = 0; ok; ++piece) {
      const Walk& w = hdr->walk[now];
      const int ahead = now == 2 ? 0 : now + 1;
      if (tid == 0) {                                        // the next piece, known behind the barriers of this one
        Walk next = w;
        hdr->more[ahead] = next.next(p) ? 1 : 0;
        hdr->walk[ahead] = next;
      }
      const int nt = w.nt, first_special = max(0, w.n_b / kKeys - w.t);    // tiles with a row that is not a cached one
      const int rpv16 = (w.rp_v + 15) & ~15;
      float m_run = -INFINITY, base = 0.f, l_run = 0.f;
      // Named barriers have no time limit: every decision to leave the loop is taken through one of them.
      for (int i = 0; i < nt; ++i, ++g) {
        const int buf = g % kBufs;
        const uint32_t tS = tmem + lane_base + buf * 128;
        const bool waited = mbar_wait(&hdr->s_full[buf], (g / kBufs) & 1u, p.status);
        const bool special = i >= first_special;
        uint32_t r[kPart];
        float cand = -INFINITY;
        if (waited) {
          tc_fence_after();
          tmem_ld16(tS + kPart * part_id, *reinterpret_cast<uint32_t(*)[16]>(&r[0]));
          tmem_ld16(tS + kPart * part_id + 16, *reinterpret_cast<uint32_t(*)[16]>(&r[16]));
          tmem_wait_ld();
          if (special) {
            const int s0 = (w.t + i) * kKeys + kPart * part_id - w.n_b;        // drafted token of the first row; cached rows lie below 0
            uint32_t open = s0 >= 0 ? 0u : s0 <= -kPart ? ~0u : (1u << -s0) - 1;
            if (s0 >= 0) open |= s0 < 64 ? static_cast<uint32_t>(seen >> s0) : 0u;
            else if (s0 > -kPart) open |= static_cast<uint32_t>(seen << -s0);
#pragma unroll
            for (int c = 0; c < kPart; ++c)
              if (!((open >> c) & 1)) r[c] = 0xff800000u;    // -inf
          }
          float mx0 = -INFINITY, mx1 = -INFINITY;
#pragma unroll
          for (int c = 0; c < kPart; c += 4) {
            mx0 = max3(mx0, __uint_as_float(r[c]), __uint_as_float(r[c + 1]));
            mx1 = max3(mx1, __uint_as_float(r[c + 2]), __uint_as_float(r[c + 3]));
          }
          cand = fmaxf(mx0, mx1);
        }
        float alpha = 1.f;
        if (softmax_barrier_or(!waited || cand > m_run + 8.f || *abort_flag != 0)) {
          hdr->exch[part_id][row] = cand;
          if (softmax_barrier_or(!waited || *abort_flag != 0)) {      // a wait gave up somewhere: all of them leave here
            ok = false;
            break;
          }
          const float top = fmaxf(fmaxf(hdr->exch[0][row], hdr->exch[1][row]), fmaxf(hdr->exch[2][row], hdr->exch[3][row]));
          if (top > m_run + 8.f) {                           // the same decision in all four threads of the row
            alpha = ex2(m_run - top);
            m_run = base = top;
          }
          l_run *= alpha;
          if (i > 0 && __any_sync(0xffffffffu, alpha != 1.f)) {       // rescale this thread's columns of the row of O'
            const bool got = mbar_wait(&hdr->o_done[(g - 1) % kBufs], ((g - 1) / kBufs) & 1u, p.status);
            if (__all_sync(0xffffffffu, got)) {
              tc_fence_after();
#pragma unroll 1
              for (int c0 = 16 * part_id; c0 < rpv16; c0 += 16 * kParts) {
                uint32_t o[16];
                tmem_ld16(tO + c0, o);
                tmem_wait_ld();
#pragma unroll
                for (int j = 0; j < 16; ++j) o[j] = __float_as_uint(__uint_as_float(o[j]) * alpha);
                tmem_st16(tO + c0, o);
              }
            } else {
              *abort_flag = 1;                               // seen by every softmax thread at the next barrier
            }
          }
        }
        if (special) {
          // the V' tile: rows behind the end cleared, values of drafted rows that are not finite cleared and noted
          const int st = g % rings.v_stages;
          const bool landed = mbar_wait(&hdr->v_full[st], (g / rings.v_stages) & 1u, p.status);
          const int r_log = (w.t + i) * kKeys + row, n_b = w.n_b, row_end = n_b + p.tail;
          if (landed && r_log >= n_b) {
            unsigned char* v_tile = v_ring + st * rings.v_stage;
            const int pieces16 = 8 * ((rpv16 + 63) >> 6);
            bool odd = false;
#pragma unroll 1
            for (int c = part_id; c < pieces16; c += kParts) {
              uint4* at = reinterpret_cast<uint4*>(v_tile + (c >> 3) * kAtom + sw128_off(row, c & 7));
              uint4 v = *at;
              uint32_t* u = reinterpret_cast<uint32_t*>(&v);
              bool touched = false;
#pragma unroll
              for (int j = 0; j < 4; ++j) {
                if (r_log >= row_end) { touched = touched || u[j] != 0; u[j] = 0; continue; }
                if (!finite16(u[j])) { u[j] &= 0xffff0000u; touched = odd = true; }
                if (!finite16(u[j] >> 16)) { u[j] &= 0x0000ffffu; touched = odd = true; }
              }
              if (touched) *at = v;
            }
            if (odd) atomicOr(&hdr->odd[piece & 1], 1ull << (r_log - n_b));
          }
          fence_async_smem();
        }
        // exponentials against the reference, their sum, P as two 16-bit parts over S
        float sum0 = 0.f, sum1 = 0.f;
        const float neg = -base;
#pragma unroll
        for (int j0 = 0; j0 < kPart / 2; j0 += 8) {
          uint32_t hi[8], lo[8];
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            float y0, y1;
            fma2(y0, y1, __uint_as_float(r[2 * (j0 + j)]), __uint_as_float(r[2 * (j0 + j) + 1]), 1.f, neg);
            const float e0 = ex2(y0), e1 = ex2(y1);
            add2(sum0, sum1, e0, e1);
            split_pair(e0, e1, hi[j], lo[j]);
          }
          tmem_st8(tS + kPart / 2 * part_id + j0, hi);
          tmem_st8(tS + 64 + kPart / 2 * part_id + j0, lo);
        }
        l_run += sum0 + sum1;
        tmem_wait_st();
        tc_fence_before();
        mbar_arrive(&hdr->p_full[buf]);
      }
      // ---- the next piece's Q' (this one's last S product has read its own), so that its products go on meanwhile
      uint64_t seen_next = 0;
      const bool more = ok && hdr->more[ahead] != 0;
      if (more) seen_next = load_q(hdr->walk[ahead]);
      // ---- the piece's partial
      if (ok) {
        const bool done = mbar_wait(&hdr->o_done[(g - 1) % kBufs], ((g - 1) / kBufs) & 1u, p.status);
        if (!done) *abort_flag = 1;
        tc_fence_after();
      }
      hdr->exch[part_id][row] = l_run;                       // the four sums share the reference
      const bool fine = !softmax_barrier_or(!ok || *abort_flag != 0);
      ok = fine;
      const uint64_t odd = hdr->odd[piece & 1] & seen;
      if (tid == 0) hdr->odd[(piece + 1) & 1] = 0;           // (read by everyone before this barrier, next written behind another)
      const int rp_v = w.rp_v, n_b = w.n_b, live = min(kTile, p.rows - w.chunk * kTile);
      const int64_t item = (static_cast<int64_t>(w.h) * p.B + w.b) * w.chunks + w.chunk;
      float* part = p.partials + ((item + blockIdx.x) * p.slot_rows + row) * p.part_stride;
      if (part_id == 0 && row < live) {
        part[0] = fine ? m_run : -INFINITY;
        part[1] = fine ? (hdr->exch[0][row] + hdr->exch[1][row]) + (hdr->exch[2][row] + hdr->exch[3][row]) : 0.f;
      }
#pragma unroll 1
      for (int c0 = 16 * part_id; c0 < rpv16; c0 += 16 * kParts) {
        uint32_t o[16];
        tmem_ld16(tO + c0, o);
        tmem_wait_ld();
        if (row >= live) continue;
#pragma unroll
        for (int j = 0; j < 16; j += 4) {
          if (c0 + j >= rp_v) break;
          float4 v = make_float4(__uint_as_float(o[j]), __uint_as_float(o[j + 1]), __uint_as_float(o[j + 2]), __uint_as_float(o[j + 3]));
          if (!fine) v = make_float4(0.f, 0.f, 0.f, 0.f);
          for (uint64_t rest = odd; rest; rest &= rest - 1) {          // (rare) values that are not finite, of rows this query sees
            const int64_t at = physical_row(p.pages, w.b, p.n_max, n_b + __ffsll(static_cast<long long>(rest)) - 1);
            const uint2 u = *reinterpret_cast<const uint2*>(p.cache + p.heads[w.h].v_off + (at * rp_v + c0 + j) * 2);
            if (!finite16(u.x)) v.x += __uint_as_float(u.x << 16);
            if (!finite16(u.x >> 16)) v.y += __uint_as_float(u.x & 0xffff0000u);
            if (!finite16(u.y)) v.z += __uint_as_float(u.y << 16);
            if (!finite16(u.y >> 16)) v.w += __uint_as_float(u.y & 0xffff0000u);
          }
          *reinterpret_cast<float4*>(part + 4 + c0 + j) = v;
        }
      }
      tc_fence_before();                                     // (the next piece's products overwrite O' once P is announced)
      if (!more) break;
      seen = seen_next;
      now = ahead;
    }
    if (!ok) *abort_flag = 1;
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
