// Attention of several query rows per K/V head over one sequence's rows (a tree of drafted tokens, or one token over a
// list of blocks) with warp-level tensor-core products, for 16-bit layers.
//
// A warp takes 32 cached rows of every tile of 128 (16 of 64 for wide ranks) and 8 or 16 query rows: S = Q' K'^T and O' += P V' with mma.sync
// m16n8k16, the softmax in between on the accumulator fragments, which are at the same time the A fragments of the second
// product.  The 16 rows of an A operand hold 8 queries twice: rows 0-7 the leading 16-bit part of Q' (or of P), rows 8-15
// what it leaves.  A thread of the fragment layout owns rows g and g + 8, the two halves of one query, so adding them is
// one addition in the same thread; Q' and P enter the products with 16 significant bits and the result carries no more
// than the rounding of the output.  With at most 8 query rows the second half of the operand would be empty anyway.
//
// Rows travel by 16-byte asynchronous copies into a ring that belongs to the warps that read it (one warp, or two that
// share the rows and split the queries): no block-wide barrier and no wait that could fail to end.  In shared memory a row
// sits at an odd multiple of 16 bytes, so that the eight rows of an ldmatrix meet all banks once, whatever the rank.
// Heads narrower than the instance keep zeros in the rest of their rows: the products run over the instance's width
// without a branch (guards per piece of a row cut the code into short blocks that cannot overlap: twice the time).
//
// Bound by the bytes of K' and V' where rows are long: 16 sequences of 32k rows with 16 drafted tokens, 32 heads of rank 80,
// 5.37 GB in 847 us.  Three CTAs per SM for rank 80 (tiles of 64 rows) read no faster: 992 us for the whole call against 918.
#include <cuda_bf16.h>

#include "internal.h"
#include "tc_common.cuh"

namespace ea {
namespace {

using namespace tc;

constexpr unsigned kFull = 0xffffffffu;
constexpr float kRaise = 8.f;              // a running maximum is raised when a score exceeds it by this much
constexpr int kGroups = 4;                 // key groups of a tile

__device__ __forceinline__ void mma16(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void ldsm4(uint32_t (&r)[4], uint32_t addr) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void ldsm2(uint32_t (&r)[4], uint32_t addr) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x2.shared.b16 {%0,%1}, [%2];" : "=r"(r[0]), "=r"(r[1]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void ldsm2_t(uint32_t (&r)[4], uint32_t addr) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x2.trans.shared.b16 {%0,%1}, [%2];" : "=r"(r[0]), "=r"(r[1]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void ldsm4_t(uint32_t (&r)[4], uint32_t addr) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void cp_async16_to(uint32_t dst, const void* src, uint64_t policy) {
  asm volatile("cp.async.cg.shared.global.L2::cache_hint [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "l"(policy) : "memory");
}
__device__ __forceinline__ void cp_async16_fill(uint32_t dst, const void* src, uint32_t bytes) {   // 0 bytes: zeros
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(bytes) : "memory");
}
__device__ __forceinline__ float quad_max(float v) {
  v = fmaxf(v, __shfl_xor_sync(kFull, v, 1));
  return fmaxf(v, __shfl_xor_sync(kFull, v, 2));
}
// (x0, x1) as two pairs of 16-bit numbers: hi = the rounded values, lo = the rounded remainders
__device__ __forceinline__ void split_pair(float x0, float x1, uint32_t& hi, uint32_t& lo) {
  hi = pack_bf16(x0, x1);
  lo = pack_bf16(x0 - __uint_as_float(hi << 16), x1 - __uint_as_float(hi & 0xffff0000u));
}
__device__ __forceinline__ uint64_t tree_mask(uint64_t m, int tokens) { return tokens < 64 ? m & ((1ull << tokens) - 1) : m; }
__device__ __forceinline__ int tree_depth(uint64_t m, int t) { return __popcll(m & ~(1ull << t)); }

// The 16-byte pieces of a row, and the distance of two rows in shared memory in such pieces.
__host__ __device__ constexpr int odd_pieces(int pieces) { return pieces | 1; }

// Shape of an instance: NC = 8-channel pieces of a row (even); MT = tiles of 8 queries per warp; WG = warps that share a
// key group's rows.  Wide rows come 16 at a time, so that two CTAs with two or three stages each still fit an SM.
template <int NC, int MT, int WG>
struct Shape {
  static constexpr int kRows = NC > 12 ? 16 : 32;                         // rows of a key group
  static constexpr int kHalves = kRows / 16, kJ = kRows / 8;
  static constexpr int kTile = kGroups * kRows, kTileShift = kTile == 64 ? 6 : 7;
  static constexpr int kThreads = kGroups * WG * 32;
  static constexpr int kQueries = 8 * MT * WG;
  static constexpr int kPitch = odd_pieces(NC) * 16;
  static constexpr int kSlot = kRows * 2 * kPitch;                        // one key group's rows of a tile
  static constexpr int kCtas = WG == 2 ? 1 : NC <= 8 && MT == 1 ? 3 : 2;  // resident CTAs per SM
  static constexpr bool kQReg = MT * NC * 2 <= 40;                        // Q' fragments in registers, else in shared memory
  static constexpr int kQBytes = kQReg ? 0 : WG * MT * (NC / 2) * 32 * 16;
  static constexpr int kHead = 32 * 8 + 64 * 4;                           // masks of the queries, positions of the drafted rows
  static constexpr int kRoom = (kCtas == 3 ? 75 : kCtas == 2 ? 113 : 226) * 1024 - kHead - kQBytes;
  static constexpr int kStages = kRoom / (kGroups * kSlot) < 4 ? kRoom / (kGroups * kSlot) : 4;
  static constexpr int kMerge = kGroups * kQueries * (2 + 8 * NC + 1) * 4;
  static constexpr int kRing = kGroups * kSlot * kStages > kMerge ? kGroups * kSlot * kStages : kMerge;
  static constexpr size_t kSmem = kHead + kQBytes + kRing;
  static_assert(NC % 2 == 0 && kStages >= 2, "instance does not fit");
};

// What a CTA works on: a piece of one item (unit, run of query rows), or, in ranges, one piece after the other.
struct Item {
  int h, b, chunk, t;        // first tile of the piece
  int tiles;                 // of the item
};
__device__ __forceinline__ int item_tiles(const MqDecodeParams& p, int b) {
  if (p.list != nullptr) return p.tiles;
  return (p.n - (p.deficit != nullptr ? __ldg(p.deficit + b) : 0) + p.tail + (1 << p.tile_shift) - 1) >> p.tile_shift;
}
// The item that tile x of all of them belongs to.  By whole warps (sequences of unequal lengths are searched 32 at a time).
__device__ __forceinline__ Item item_of(const MqDecodeParams& p, int x, int chunks, int lane) {
  Item w;
  const int per_head = static_cast<int>(p.head_tiles) * chunks;
  w.h = x / per_head;
  int rest = x - w.h * per_head;
  w.b = 0;
  if (p.deficit == nullptr || p.list != nullptr) {
    w.tiles = p.tiles;
    w.b = rest / (p.tiles * chunks);
    rest -= w.b * p.tiles * chunks;
  } else {
    for (int b0 = 0; b0 < p.B; b0 += 32) {
      int scan = b0 + lane < p.B ? item_tiles(p, b0 + lane) * chunks : 0;
#pragma unroll
      for (int d = 1; d < 32; d <<= 1) {
        const int y = __shfl_up_sync(kFull, scan, d);
        if (lane >= d) scan += y;
      }
      const unsigned past = __ballot_sync(kFull, rest < scan);            // sequences that end behind the place
      if (past) {
        const int k = __ffs(past) - 1;
        if (k > 0) rest -= __shfl_sync(kFull, scan, k - 1);
        w.b = b0 + k;
        break;
      }
      rest -= __shfl_sync(kFull, scan, 31);
    }
    w.tiles = item_tiles(p, w.b);
  }
  w.chunk = rest / w.tiles;
  w.t = rest - w.chunk * w.tiles;
  return w;
}

// Where the rows of a key group come from: runs of 16 neighbouring rows (a block can be 16 rows long).
struct Source {
  int64_t row[2];          // physical first row of each half
  int valid[2];            // rows of each half that exist
  int first[2];            // logical first row of each half (-1: nothing there)
};

template <int NC, int MT, int WG>
__global__ void __launch_bounds__(Shape<NC, MT, WG>::kThreads, Shape<NC, MT, WG>::kCtas)
    mq_mma_kernel(const MqDecodeParams p) {
  using S = Shape<NC, MT, WG>;
  constexpr int NKS = NC / 2, kRows = S::kRows, HV = S::kHalves, NJ = S::kJ;
  chain_go();
  extern __shared__ __align__(1024) unsigned char smem[];
  uint64_t* q_mask = reinterpret_cast<uint64_t*>(smem);                   // [32]
  float* draft_pos = reinterpret_cast<float*>(smem + 32 * 8);             // [64]
  uint4* q_img = reinterpret_cast<uint4*>(smem + S::kHead);               // [WG][MT][NKS][32 lanes]
  unsigned char* ring = smem + S::kHead + S::kQBytes;

  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, gid = lane >> 2, tig = lane & 3;
  const int kg = warp & 3, rg = warp >> 2;                                // key group, share of the queries
  const int chunks = (p.rows + S::kQueries - 1) / S::kQueries;
  Item item;
  int left = 0;                                                           // tiles of the CTA's range from here on
  if (p.grid > 0) {
    const int c = blockIdx.x;
    item = item_of(p, c * p.cta_tiles + min(c, p.cta_extra), chunks, lane);
    left = p.cta_tiles + (c < p.cta_extra ? 1 : 0);
  } else {
    const int unit = blockIdx.x / chunks;
    item.h = unit / p.B; item.b = unit - item.h * p.B; item.chunk = blockIdx.x - unit * chunks;
    item.t = blockIdx.y * p.per;
    item.tiles = item_tiles(p, item.b);
  }
  chain_wait();                        // drafted rows, queries, the list: from the kernels before
  if (p.grid == 0 && item.t > 0 && item.t >= item.tiles) return;          // a shorter sequence: nothing left (its first piece always reports)
  for (;;) {                           // the pieces
    const int h = item.h, b = item.b, unit = h * p.B + b, chunk = item.chunk;
    const HeadInfo hd = p.heads[h];
    const int nck = hd.rp_k >> 3, ncv = hd.rp_v >> 3;                       // pieces of this head's rows
    constexpr int kpitch = S::kPitch, vpitch = S::kPitch;
    const int row0 = chunk * S::kQueries;                                   // first query row of the CTA

    const int n_b = p.deficit != nullptr ? p.n - __ldg(p.deficit + b) : p.n;
    const int t_lo = item.t, t_hi = min(item.tiles, t_lo + (p.grid > 0 ? left : p.per));
    const int32_t* list = p.list ? p.list + static_cast<int64_t>(unit) * p.list_len : nullptr;
    const char* k_slab = p.cache + hd.k_off;
    const char* v_slab = p.cache + hd.v_off;
    const bool bias = hd.alibi_slope2 != 0.f;

    // ---- rows: the copies of one key group, by its own warps.  What the address of a tile needs (the block's number, its
    // page) is loaded one and two tiles ahead of its use.
    const int64_t pos0 = static_cast<int64_t>(kg) * kRows;                  // of the key group inside a tile
    int blk_next[2] = {-1, -1}, blk_now[2] = {-1, -1}, page_now[2] = {0, 0};   // per half
    auto fetch_block = [&](int t, int (&blk)[2]) {                          // list entries of tile t
      if (list == nullptr || t >= t_hi) return;
#pragma unroll
      for (int i = 0; i < HV; ++i) {
        const int64_t at = ((static_cast<int64_t>(t) << S::kTileShift) + pos0 + 16 * i) >> p.block_shift;
        blk[i] = at < p.list_len ? __ldg(list + at) : -1;
      }
    };
    auto logical = [&](int t, int i, int blk) -> int {                      // first logical row of a half
      const int64_t at = (static_cast<int64_t>(t) << S::kTileShift) + pos0 + 16 * i;
      if (list == nullptr) return static_cast<int>(at);
      return blk < 0 ? -1 : (blk << p.block_shift) + static_cast<int>(at & ((1 << p.block_shift) - 1));
    };
    const int row_end = n_b + p.tail;
    auto fetch_page = [&](int t, const int (&blk)[2], int (&page)[2]) {
      if (p.pages.table == nullptr || t >= t_hi) return;
#pragma unroll
      for (int i = 0; i < HV; ++i) {
        const int r = logical(t, i, blk[i]);
        page[i] = r >= 0 && r < row_end ? __ldg(p.pages.table + static_cast<int64_t>(b) * p.pages.width + (r >> p.pages.shift)) : 0;
      }
    };
    auto source = [&](int t, const int (&blk)[2], const int (&page)[2]) {
      Source s;
      s.row[1] = 0; s.valid[1] = 0; s.first[1] = 0;
#pragma unroll
      for (int i = 0; i < HV; ++i) {
        const int r = logical(t, i, blk[i]);
        const bool there = r >= 0 && r < row_end;
        s.first[i] = r;
        s.valid[i] = there ? min(16, row_end - r) : 0;
        s.row[i] = !there ? 0
                   : p.pages.table == nullptr ? static_cast<int64_t>(b) * p.n_max + r
                                              : (static_cast<int64_t>(page[i]) << p.pages.shift) + (r & ((1 << p.pages.shift) - 1));
      }
      return s;
    };
    const int cl = lane + 32 * rg;                                          // this thread among the copiers of the group
    constexpr int kStep = 32 * WG;
    // Piece i = cl, cl + kStep, ... of the rows, row after row: its row and place are stepped, not divided out (with a
    // division and the row's checks for every piece the copies were most of the kernel's instructions).
    struct Walk { int row, c, d_row, d_c; };
    auto walk = [&](int nc) { return Walk{cl / nc, cl % nc, kStep / nc, kStep % nc}; };
    const Walk wk = walk(nck), wv = walk(ncv);
    // Rows that one CTA reads are not kept in L2 (16 x 32k rows 970 -> 918 us, 64 x 777 150 -> 144); with more query rows
    // than a CTA takes the CTAs next to it read them too.
    const uint64_t policy = chunks == 1 ? policy_evict_first() : policy_evict_normal();
    auto copy_rows = [&](unsigned char* dst, const char* slab, int nc, const Walk& w0, const Source& s) {
      const char* src = slab + s.row[0] * (nc * 16) + cl * 16;
      Walk w = w0;
      uint32_t to = smem_u32(dst) + w.row * kpitch + w.c * 16;
      const uint32_t step = w.d_row * kpitch + w.d_c * 16, wrap = kpitch - nc * 16;
      const int total = kRows * nc;
      if (s.valid[0] == 16 && (HV == 1 || (s.valid[1] == 16 && s.row[1] == s.row[0] + 16))) {    // whole, and neighbours
#pragma unroll
        for (int i0 = 0; i0 < kRows * NC; i0 += kStep) {
          if (i0 + cl < total) cp_async16_to(to, src + i0 * 16, policy);
          to += step;
          w.c += w.d_c;
          if (w.c >= nc) { w.c -= nc; to += wrap; }
        }
      } else {
        const int64_t skip = HV == 2 ? (s.row[1] - s.row[0] - 16) * (nc * 16) : 0;
#pragma unroll 1
        for (int i = cl; i < total; i += kStep) {
          const bool late = HV == 2 && w.row >= 16;
          const bool there = late ? w.row - 16 < s.valid[1] : w.row < s.valid[0];
          cp_async16_fill(to, there ? src + (late ? skip : 0) : slab, there ? 16u : 0u);
          src += kStep * 16;
          to += step;
          w.row += w.d_row;
          w.c += w.d_c;
          if (w.c >= nc) { w.c -= nc; ++w.row; to += wrap; }
        }
      }
    };
    auto slot_of = [&](int it) { return ring + ((it % S::kStages) * kGroups + kg) * S::kSlot; };
    int ahead[S::kStages - 1][2];                                           // logical first rows of the tiles under way
    auto issue = [&](int t) {
#pragma unroll
      for (int i = 0; i + 1 < S::kStages - 1; ++i) { ahead[i][0] = ahead[i + 1][0]; ahead[i][1] = ahead[i + 1][1]; }
      if (t < t_hi) {
        const Source s = source(t, blk_now, page_now);
        ahead[S::kStages - 2][0] = s.first[0]; ahead[S::kStages - 2][1] = s.first[1];
        unsigned char* dst = slot_of(t - t_lo);
        copy_rows(dst, k_slab, nck, wk, s);
        copy_rows(dst + kRows * kpitch, v_slab, ncv, wv, s);
      }
      cp_async_commit();
      blk_now[0] = blk_next[0]; blk_now[1] = blk_next[1];
      fetch_page(t + 1, blk_now, page_now);
      fetch_block(t + 2, blk_next);
    };
    if (nck < NC || ncv < NC)            // the rest of a narrow head's rows: zeros that no copy touches
      for (int i = tid; i < kGroups * S::kStages * kRows * 2; i += S::kThreads) {
        uint4* row = reinterpret_cast<uint4*>(ring + i * kpitch);
        for (int c = (i / kRows) & 1 ? ncv : nck; c < NC; ++c) row[c] = make_uint4(0u, 0u, 0u, 0u);
      }
    fetch_block(t_lo, blk_now);
    fetch_page(t_lo, blk_now, page_now);
    fetch_block(t_lo + 1, blk_next);
#pragma unroll
    for (int i = 0; i < S::kStages - 1; ++i) issue(t_lo + i);

    // ---- queries: fragments of Q' (leading parts in rows 0-7 of the operand, remainders in rows 8-15)
    const uint64_t* masks = p.mask + static_cast<int64_t>(b) * p.tokens;
    if (p.tail) {
      if (tid < S::kQueries) {
        const int r = row0 + tid;
        q_mask[tid] = r < p.rows ? tree_mask(masks[r / p.group], p.tokens) : 0;
      }
      if (bias && tid < p.tokens) draft_pos[tid] = static_cast<float>(tree_depth(tree_mask(masks[tid], p.tokens), tid));
    }
    uint32_t qa[S::kQReg ? MT : 1][S::kQReg ? NKS : 1][4];
    // Positions count from the first row behind the cached ones: they are small where a bias lets a row weigh anything, and
    // exact in single precision there (counted from the front, neighbours past 2^24 rows would become one number).
    float q_pos[MT];
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) {
      const int r = row0 + (rg * MT + mt) * 8 + gid;
      const float* src = p.qp + (static_cast<int64_t>(unit) * p.rows + r) * p.q_stride;
#pragma unroll
      for (int ks = 0; ks < NKS; ++ks) {
        uint32_t f[4];
#pragma unroll
        for (int half = 0; half < 2; ++half) {
          const int c = 16 * ks + 8 * half + 2 * tig;
          const bool in = r < p.rows && c < 8 * nck;
          const float2 x = in ? *reinterpret_cast<const float2*>(src + c) : make_float2(0.f, 0.f);
          split_pair(x.x, x.y, f[2 * half], f[2 * half + 1]);
        }
        if constexpr (S::kQReg) {
#pragma unroll
          for (int i = 0; i < 4; ++i) qa[mt][ks][i] = f[i];
        } else if (kg == 0) {
          q_img[((rg * MT + mt) * NKS + ks) * 32 + lane] = make_uint4(f[0], f[1], f[2], f[3]);
        }
      }
      q_pos[mt] = -1.f;
      if (p.tail && bias && r < p.rows) {
        const int t = r / p.group;
        q_pos[mt] = static_cast<float>(tree_depth(tree_mask(masks[t], p.tokens), t));
      }
    }
    __syncthreads();

    float o[MT][NC][4];
    float m[MT], base[MT], l[MT];
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) {
      m[mt] = -INFINITY; base[mt] = 0.f; l[mt] = 0.f;
#pragma unroll
      for (int c = 0; c < NC; ++c)
#pragma unroll
        for (int i = 0; i < 4; ++i) o[mt][c][i] = 0.f;
    }
    auto group_sync = [&]() {
      if constexpr (WG == 1) __syncwarp();
      else asm volatile("bar.sync %0, %1;" ::"r"(1 + kg), "n"(32 * WG) : "memory");
    };
    const uint32_t k_lane = static_cast<uint32_t>((lane & 7) * kpitch + (lane >> 3) * 16);
    const uint32_t v_lane = static_cast<uint32_t>(kRows * kpitch + (lane & (kRows - 1)) * vpitch);

    for (int t = t_lo; t < t_hi; ++t) {
      cp_async_wait<S::kStages - 2>();
      group_sync();                      // the tile is there for every warp of the group, and the tile before it is read
      const int first[2] = {ahead[0][0], ahead[0][1]};
      issue(t + S::kStages - 1);
      unsigned char* st = slot_of(t - t_lo);
      const uint32_t k_addr = smem_u32(st) + k_lane, v_addr = smem_u32(st) + v_lane;

      float s[MT][NJ][4];
#pragma unroll
      for (int mt = 0; mt < MT; ++mt)
#pragma unroll
        for (int j = 0; j < NJ; ++j)
#pragma unroll
          for (int i = 0; i < 4; ++i) s[mt][j][i] = 0.f;
#pragma unroll
      for (int c4 = 0; c4 < NC; c4 += 4) {
        uint32_t kf[NJ][4];
#pragma unroll
        for (int j = 0; j < NJ; ++j) {
          if (c4 + 2 < NC) ldsm4(kf[j], k_addr + j * 8 * kpitch + c4 * 16);
          else ldsm2(kf[j], k_addr + j * 8 * kpitch + c4 * 16);
        }
#pragma unroll
        for (int half = 0; half < 2; ++half) {
          const int ks = c4 / 2 + half;
          if (ks < NKS) {
#pragma unroll
            for (int mt = 0; mt < MT; ++mt) {
              uint32_t a[4];
              if constexpr (S::kQReg) {
#pragma unroll
                for (int i = 0; i < 4; ++i) a[i] = qa[mt][ks < NKS ? ks : 0][i];
              } else {
                const uint4 f = q_img[((rg * MT + mt) * NKS + ks) * 32 + lane];
                a[0] = f.x; a[1] = f.y; a[2] = f.z; a[3] = f.w;
              }
#pragma unroll
              for (int j = 0; j < NJ; ++j) mma16(s[mt][j], a, kf[j][2 * half], kf[j][2 * half + 1]);
            }
          }
        }
      }
      // ---- scores: the two halves of a query, the bias, the mask.  sc[mt][j][e]: row 8 j + 2 tig + e of the group
      float sc[MT][NJ][2];
#pragma unroll
      for (int mt = 0; mt < MT; ++mt)
#pragma unroll
        for (int j = 0; j < NJ; ++j) {
          sc[mt][j][0] = s[mt][j][0] + s[mt][j][2];
          sc[mt][j][1] = s[mt][j][1] + s[mt][j][3];
        }
      // the end of the sequence, drafted rows, a list entry that is not there (they come last, as the incomplete block does)
      const bool special = first[0] < 0 || (HV == 2 && first[1] < 0) || (HV == 2 ? max(first[0], first[1]) : first[0]) + 16 > n_b;
      unsigned odd_rows = 0;             // drafted rows whose values are not finite
      if (bias && !special) {
#pragma unroll
        for (int j = 0; j < NJ; ++j)
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            const float place = static_cast<float>(first[j >> 1] - n_b + 8 * (j & 1) + 2 * tig + e);
#pragma unroll
            for (int mt = 0; mt < MT; ++mt) sc[mt][j][e] = fmaf(hd.alibi_slope2, place - q_pos[mt], sc[mt][j][e]);
          }
      }
      if (special) {
#pragma unroll
        for (int j = 0; j < NJ; ++j)
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            const int kk = 8 * (j & 1) + 2 * tig + e;                       // inside its half
            const int r = first[j >> 1] < 0 ? row_end : first[j >> 1] + kk;
            const bool drafted = r >= n_b && r < row_end;
            const float place = bias ? (drafted ? draft_pos[r - n_b] : static_cast<float>(r - n_b)) : 0.f;
#pragma unroll
            for (int mt = 0; mt < MT; ++mt) {
              bool open = r < n_b;
              if (drafted) open = (q_mask[(rg * MT + mt) * 8 + gid] >> (r - n_b)) & 1;
              if (bias) sc[mt][j][e] = fmaf(hd.alibi_slope2, place - q_pos[mt], sc[mt][j][e]);
              if (!open) sc[mt][j][e] = -INFINITY;
            }
          }
        if (p.tail && first[0] + kRows > n_b) {          // (the whole sequence: the two halves are neighbours)
          const int r = first[0] + lane;
          bool bad = false;
          if (lane < kRows && r >= n_b && r < row_end) {
            const uint4* x = reinterpret_cast<const uint4*>(st + kRows * kpitch + lane * vpitch);
            for (int c = 0; c < ncv; ++c) {
              const uint4 w = x[c];
              const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
              for (int i = 0; i < 4; ++i)
                bad = bad || (u[i] & 0x7f80u) == 0x7f80u || (u[i] & 0x7f800000u) == 0x7f800000u;
            }
          }
          odd_rows = __ballot_sync(kFull, bad);
        }
      }
      // ---- online softmax on the fragments
      bool raise = false;
      float mx[MT];
#pragma unroll
      for (int mt = 0; mt < MT; ++mt) {
        mx[mt] = fmaxf(max3(sc[mt][0][0], sc[mt][0][1], sc[mt][1][0]), sc[mt][1][1]);
#pragma unroll
        for (int j = 2; j < NJ; ++j) mx[mt] = max3(mx[mt], sc[mt][j][0], sc[mt][j][1]);
        raise = raise || mx[mt] > m[mt] + kRaise;
      }
      if (__any_sync(kFull, raise)) {
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) {
          const float top = fmaxf(m[mt], quad_max(mx[mt]));
          base[mt] = top == -INFINITY ? 0.f : top;
          const float f = ex2(m[mt] - base[mt]);                            // 0 before the first row
          m[mt] = top;
          l[mt] *= f;
#pragma unroll
          for (int c = 0; c < NC; ++c)
#pragma unroll
            for (int i = 0; i < 4; ++i) o[mt][c][i] *= f;
        }
      }
      uint32_t pa[MT][HV][4];            // A fragments of P for the steps of 16 rows: leading parts and remainders
#pragma unroll
      for (int mt = 0; mt < MT; ++mt)
#pragma unroll
        for (int j = 0; j < NJ; ++j) {
          sc[mt][j][0] = ex2(sc[mt][j][0] - base[mt]);
          sc[mt][j][1] = ex2(sc[mt][j][1] - base[mt]);
          l[mt] += sc[mt][j][0] + sc[mt][j][1];
          split_pair(sc[mt][j][0], sc[mt][j][1], pa[mt][j >> 1][(j & 1) * 2], pa[mt][j >> 1][(j & 1) * 2 + 1]);
        }
      if (odd_rows) {
        // A product with a zero weight would still carry an infinity or NaN of a row that the query does not see: such rows
        // are added one by one where their weight is not zero, and then cleared for the products.
#pragma unroll
        for (int j = 0; j < NJ; ++j)
#pragma unroll
          for (int e = 0; e < 2; ++e)
            for (int src = 0; src < 4; ++src) {
              const int key = 8 * j + 2 * src + e;
              if (!((odd_rows >> key) & 1)) continue;
              const __nv_bfloat16* v = reinterpret_cast<const __nv_bfloat16*>(st + kRows * kpitch + key * vpitch);
#pragma unroll
              for (int mt = 0; mt < MT; ++mt) {
                const float w = __shfl_sync(kFull, sc[mt][j][e], (lane & ~3) | src);
                if (w != 0.f) {
#pragma unroll
                  for (int c = 0; c < NC; ++c) {
                    o[mt][c][0] = fmaf(w, __bfloat162float(v[8 * c + 2 * tig]), o[mt][c][0]);
                    o[mt][c][1] = fmaf(w, __bfloat162float(v[8 * c + 2 * tig + 1]), o[mt][c][1]);
                  }
                }
              }
            }
        group_sync();
        if ((odd_rows >> lane) & 1) {
          uint4* x = reinterpret_cast<uint4*>(st + kRows * kpitch + lane * vpitch);
          for (int c = 0; c < ncv; ++c) x[c] = make_uint4(0u, 0u, 0u, 0u);
        }
        group_sync();
      }
      // ---- O' += P V'
#pragma unroll
      for (int c = 0; c < NC; ++c) {
        uint32_t vf[4];
        if (HV == 2) ldsm4_t(vf, v_addr + c * 16);
        else ldsm2_t(vf, v_addr + c * 16);
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) {
          mma16(o[mt][c], pa[mt][0], vf[0], vf[1]);
          if (HV == 2) mma16(o[mt][c], pa[mt][HV - 1], vf[2], vf[3]);
        }
      }
    }
    cp_async_wait<0>();
    __syncthreads();

    // ---- merge the key groups (the ring is idle): per query the maximum, then sums and O' scaled to it
    constexpr int Q = S::kQueries, OS = 8 * NC + 1;
    float* wm = reinterpret_cast<float*>(ring);                // [4][Q]
    float* wl = wm + kGroups * Q;                              // [4][Q]
    float* wo = wl + kGroups * Q;                              // [4][Q][OS]
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) {
      l[mt] += __shfl_xor_sync(kFull, l[mt], 1);
      l[mt] += __shfl_xor_sync(kFull, l[mt], 2);
      const int q = kg * Q + (rg * MT + mt) * 8 + gid;
      if (tig == 0) { wm[q] = m[mt]; wl[q] = l[mt]; }
#pragma unroll
      for (int c = 0; c < NC; ++c)
        if (c < ncv) {
          wo[q * OS + 8 * c + 2 * tig] = o[mt][c][0] + o[mt][c][2];
          wo[q * OS + 8 * c + 2 * tig + 1] = o[mt][c][1] + o[mt][c][3];
        }
    }
    __syncthreads();
    const int rp_v = 8 * ncv;
    const int nq = min(Q, p.rows - row0);
    for (int i = tid; i < nq * (rp_v + 2); i += S::kThreads) {
      const int q = i / (rp_v + 2), c = i - q * (rp_v + 2);
      const float M = fmaxf(fmaxf(wm[q], wm[Q + q]), fmaxf(wm[2 * Q + q], wm[3 * Q + q]));
      const float mb = M == -INFINITY ? 0.f : M;
      float acc = 0.f;
#pragma unroll
      for (int w = 0; w < kGroups; ++w)
        acc = fmaf(c < rp_v ? wo[(w * Q + q) * OS + c] : wl[w * Q + q], ex2(wm[w * Q + q] - mb), acc);
      float* part = p.partials + (p.grid > 0 ? (static_cast<int64_t>(unit) * chunks + chunk + blockIdx.x) * p.slot_rows + q
                                             : (static_cast<int64_t>(unit) * p.rows + row0 + q) * p.splits + blockIdx.y) * p.part_stride;
      if (c < rp_v) part[4 + c] = acc;
      else if (c == rp_v) part[1] = acc;
      else part[0] = M;
    }
    left -= t_hi - t_lo;
    if (left <= 0) break;                // (one piece per CTA: left is 0)
    item.t = 0;
    if (++item.chunk == chunks) {
      item.chunk = 0;
      if (++item.b == p.B) {
        item.b = 0;
        ++item.h;
      }
      item.tiles = item_tiles(p, item.b);
    }
    __syncthreads();                     // the ring and the masks are the next piece's
  }
}

template <int NC, int MT, int WG>
cudaError_t launch_instance(const MqDecodeParams& p, cudaStream_t s) {
  using S = Shape<NC, MT, WG>;
  static size_t configured[kMaxDevices] = {};
  const cudaError_t e = ensure_dynamic_smem(mq_mma_kernel<NC, MT, WG>, S::kSmem, configured);
  if (e != cudaSuccess) return e;
  const int chunks = (p.rows + S::kQueries - 1) / S::kQueries;
  return launch_chained(p.chained != 0, mq_mma_kernel<NC, MT, WG>, p.grid > 0 ? dim3(p.grid) : dim3(p.B * p.H * chunks, p.splits), S::kThreads, S::kSmem, s, p);
}
template <int NC>
cudaError_t launch_rank(const MqDecodeParams& p, cudaStream_t s) {
  if (p.rows <= 8) return launch_instance<NC, 1, 1>(p, s);
  if (p.rows <= 16) return launch_instance<NC, 2, 1>(p, s);
  return launch_instance<NC, 2, 2>(p, s);
}

}  // namespace

MqShape mq_mma_shape(int rows, int max_rp) {
  const int shift = max_rp > 96 ? 6 : 7;
  if (rows <= 8) return {8, max_rp <= 64 ? 3 : 2, shift};
  if (rows <= 16) return {16, 2, shift};
  return {32, 1, shift};
}

cudaError_t launch_mq_mma(const MqDecodeParams& p, int max_rp, cudaStream_t s, uint64_t* launches) {
  ++*launches;
  if (max_rp <= 48) return launch_rank<6>(p, s);
  if (max_rp <= 64) return launch_rank<8>(p, s);
  if (max_rp <= 80) return launch_rank<10>(p, s);
  if (max_rp <= 96) return launch_rank<12>(p, s);
  if (max_rp <= 112) return launch_rank<14>(p, s);
  return launch_rank<16>(p, s);
}

}  // namespace ea
