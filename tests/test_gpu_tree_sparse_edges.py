"""Rows at the edges of tiles, pieces, pages and blocks inside long sequences: some thirty rows of a unit carry all of the
weight, and they sit on such edges.  Bases are unit vectors, so that nothing but the kernels' own arithmetic stands between a
row and the output, and the bound (mq_helpers) is tight: every case checks that the expected value without any single one of
those rows would lie outside it."""
import math

import numpy as np
import pytest
import torch

from mq_helpers import BF16, FP32, HALF_STEP, Case, check, mask_tensor, np64, randn, sparse_expected, tree_expected, trees

pytestmark = pytest.mark.gpu

SCORE = 22.0                   # of a row that counts; all others score 0: e^-22 each


@pytest.fixture(scope="module")
def B():
    from paper_2408_05646_b200 import build
    build.build_library()
    from paper_2408_05646_b200 import binding
    return binding


class Edges(Case):
    def __init__(self, B, dtype, batch, H, group, d, ranks, lens, n_max, seed, page_rows=0):
        self.dtype, self.batch, self.H, self.group, self.d = dtype, batch, H, group, d
        self.rk = self.rv = ranks
        self.lens, self.slopes = list(lens), None
        self.U_k = self.U_v = [np.eye(d, dtype=np.float32)[:, :r] for r in ranks]
        self.lay = lay = B.EigenAttnLayer(batch, H, d, n_max, dtype, self.U_k, self.U_v)
        self.page_rows, self.table = page_rows, None
        if page_rows:
            perm = np.random.default_rng(seed).permutation(batch * n_max // page_rows)
            per = len(perm) // batch
            self.table = [[int(x) for x in perm[b * per:(b + 1) * per]] for b in range(batch)]
            lay.set_page_table(self.table, page_rows)
        self.sign = [torch.tensor(np.random.default_rng(seed + h).choice([-1.0, 1.0], r), device="cuda").to(dtype) for h, r in enumerate(ranks)]
        for h in range(H):
            slab = lay.cache_rows(h, "v")
            slab[..., :ranks[h]] = randn(slab.shape[:-1] + (ranks[h],), seed + h, dtype)
        if len(set(lens)) > 1:
            lay.set_lens(lens)
        else:
            lay.set_len(lens[0])

    def place(self, seed, near=(16, 32, 64, 128), count=30):
        """Fresh rows that count, on edges; returns their places per unit."""
        g = np.random.default_rng(seed)
        places = {}
        for h in range(self.H):
            slab = self.lay.cache_rows(h, "k")
            slab.zero_()
            flat = slab.view(-1, slab.shape[-1])
            for b, n in enumerate(self.lens):
                steps = g.choice(near, 4 * count)
                at = steps * g.integers(0, max(n, 1) // steps + 1) - g.integers(0, 2, 4 * count)
                at = sorted({0, n - 1} | set(int(x) for x in at[(at >= 0) & (at < n)][:count - 2])) if n else []
                places[b, h] = at
                if not at:
                    continue
                rows = torch.tensor(at, device="cuda")
                if self.table is not None:
                    rows = torch.tensor([self.table[b][j // self.page_rows] * self.page_rows + j % self.page_rows for j in at], device="cuda")
                else:
                    rows = rows + b * slab.shape[1]
                flat[rows, :self.rk[h]] = self.sign[h]
        return places

    def tokens(self, T, heads, kind, seed):
        """Queries along the rows' direction (score SCORE), drafted keys like the rows that count."""
        x = randn((self.batch, T, heads, self.d), seed, self.dtype)
        if kind == "v":
            return x
        group = heads // self.H
        for h in range(self.H):
            r = self.rk[h]
            scale = SCORE * math.sqrt(self.d) / r if kind == "q" else 1.0
            x[:, :, h * group:(h + 1) * group] = 0
            x[:, :, h * group:(h + 1) * group, :r] = (self.sign[h].float() * scale).to(self.dtype)
        return x


def would_notice(want, slack, V, weight, dtype):
    """Leaving out any one of rows V (weight each, all alike) changes `want` by more than the bound allows somewhere."""
    without = (want - weight * V) / (1 - weight)
    over = np.abs(without - want) - 2 * (HALF_STEP[dtype] * np.maximum(np.abs(want), np.abs(without)) + slack)
    assert (over.max(1) > 0).all()


SHAPES = [
    # dtype, batch, H, group, d, ranks, lens, T, page, impl
    (BF16, 3, 2, 1, 128, [80, 80], [6020, 1053, 333], 4, 0, 0),        # warp level, 8 query rows
    (BF16, 2, 2, 1, 64, [48, 64], [4099, 2048], 7, 0, 0),
    (BF16, 2, 2, 2, 128, [112, 128], [3000, 1666], 6, 0, 0),           # 16 query rows, tiles of 64
    (BF16, 2, 2, 1, 96, [96, 96], [2300, 5000], 13, 0, 0),
    (BF16, 2, 2, 1, 128, [80, 24], [2999, 1000], 30, 0, 1),            # 32 query rows, warp level
    (BF16, 2, 1, 3, 128, [128], [1500, 2111], 20, 0, 1),
    (BF16, 2, 2, 1, 128, [80, 80], [4222, 1777], 20, 0, 0),            # tcgen05: four copies of the rows
    (BF16, 2, 2, 1, 128, [80, 48], [4200, 1900], 50, 0, 0),            # two copies
    (BF16, 3, 1, 4, 128, [80], [3010, 0, 5555], 32, 0, 0),             # 128 query rows
    (BF16, 2, 1, 4, 128, [128], [2500, 2222], 63, 0, 0),               # two runs of query rows, two V' stages
    (BF16, 3, 2, 1, 128, [80, 64], [3111, 900, 257], 5, 128, 0),       # pages, warp level
    (BF16, 3, 2, 1, 128, [80, 64], [3111, 900, 257], 40, 256, 0),      # pages, tcgen05
    (FP32, 2, 2, 1, 64, [64, 32], [1900, 700], 5, 0, 0),
    (FP32, 2, 1, 3, 80, [80], [1500, 400], 9, 128, 0),
]


@pytest.mark.parametrize("dtype,batch,H,group,d,ranks,lens,T,page,impl", SHAPES)
def test_tree(B, dtype, batch, H, group, d, ranks, lens, T, page, impl):
    c = Edges(B, dtype, batch, H, group, d, ranks, lens, -(-(max(lens) + T) // 256) * 256, 211, page)
    c.lay.set_option(B.EA_OPT_TREE_IMPL, impl)
    c.lay.tree_attach(T, group)
    q, k, v = c.tokens(T, H * group, "q", 213), c.tokens(T, H, "k", 215), c.tokens(T, H, "v", 217)
    masks, _ = trees(batch, T, 9)
    m = mask_tensor(masks)
    for seed, ctas in ((0, 0), (1, 0), (2, 3), (3, 11), (4, 300)):
        places = c.place(seed)
        c.lay.set_option(B.EA_OPT_DECODE_CTAS, ctas)
        out = c.lay.decode_tree(q, k, v, m, group=group)
        want, slack = tree_expected(c, q, masks, T)
        check(out, want, slack, dtype, f"tree {seed}")
        for (b, h), at in places.items():
            K, V = c.rows(b, h, lens[b] + T, "k"), c.rows(b, h, lens[b] + T, "v")
            for t in (0, T - 1):
                rows = at + [lens[b] + s for s in range(T) if masks[b][t] >> s & 1]
                pad = np.zeros((len(rows), d))
                pad[:, :ranks[h]] = V[rows]
                if len(rows) > 1:
                    would_notice(want[b, t, h * group], slack[b, t, h * group], pad, 1.0 / len(rows), dtype)
    c.lay.poll_status()


BLOCKS = [
    # dtype, batch, H, group, d, ranks, lens, block, n_blocks, page
    (BF16, 2, 2, 1, 128, [80, 80], [6020, 3333], 16, 60, 0),
    (BF16, 2, 2, 1, 128, [64, 48], [6000, 1053], 32, 50, 0),
    (BF16, 2, 1, 4, 128, [112], [5000, 4097], 64, 30, 0),
    (BF16, 2, 1, 16, 128, [128], [5555, 2000], 128, 20, 0),
    (BF16, 2, 2, 2, 96, [96, 40], [3000, 3001], 32, 60, 128),
    (FP32, 2, 1, 1, 64, [64], [2500, 1111], 32, 40, 0),
]


@pytest.mark.parametrize("dtype,batch,H,group,d,ranks,lens,block,n_blocks,page", BLOCKS)
def test_blocks(B, dtype, batch, H, group, d, ranks, lens, block, n_blocks, page):
    c = Edges(B, dtype, batch, H, group, d, ranks, lens, -(-max(lens) // 256) * 256, 311, page)
    c.lay.sparse_attach(block)
    q = c.tokens(1, H * group, "q", 313)
    for seed, ctas in ((0, 0), (1, 0), (2, 3), (3, 11), (4, 300)):
        places = c.place(seed, near=(16, block, 2 * block), count=min(n_blocks - 2, 30))
        c.lay.set_len(0)                               # other keys: forget the bounds
        c.lay.set_lens(lens)
        c.lay.sparse_sync()
        c.lay.set_option(B.EA_OPT_DECODE_CTAS, ctas)
        out, index = c.lay.decode_sparse(q, n_blocks, group=group, return_index=True)
        want, slack, idx = sparse_expected(c, q, block, n_blocks, 1, 1)
        assert np.array_equal(index.cpu().numpy(), idx)
        check(out, want, slack, dtype, f"blocks {seed}")
        for (b, h), at in places.items():
            assert set(j // block for j in at) <= set(idx[b, h].tolist())
            pad = np.zeros((len(at), d))
            pad[:, :ranks[h]] = c.rows(b, h, lens[b], "v")[at]
            would_notice(want[b, 0, h * group], slack[b, 0, h * group], pad, 1.0 / len(at), dtype)
    c.lay.poll_status()
