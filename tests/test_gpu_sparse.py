"""Decode over selected blocks on the GPU against the 64-bit definition: block bounds, the choice, the attention."""
import numpy as np
import pytest
import torch

from mq_helpers import BF16, FP32, Case, check, mask_tensor, np64, randn, sparse_expected, tree_expected, trees
from oracle import tree_sparse as ts

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    from paper_2408_05646_b200 import build
    build.build_library()
    from paper_2408_05646_b200 import binding
    return binding


def bounds_of(c, b, h, block, count):
    """Bounds of a unit's first `count` blocks, wherever its rows live."""
    x = c.lay.sparse_bounds(h)
    r = c.rk[h]
    if c.table is None:
        x = x[b, :count]
    else:
        per = c.page_rows // block
        x = x.reshape(-1, 2, x.shape[-1])[[c.table[b][j // per] * per + j % per for j in range(count)]]
    return np64(x[:, 0])[:, :r], np64(x[:, 1])[:, :r]


SHAPES = [
    # dtype, batch, H, group, d, rk, rv, lens, block, n_blocks, sink, recent, page
    (BF16, 1, 2, 1, 128, [80, 80], [80, 80], [1000], 64, 6, 1, 1, 0),
    (BF16, 2, 2, 1, 128, [64, 64], [64, 64], [1024, 1024], 32, 9, 1, 1, 0),          # the last block is complete
    (BF16, 3, 2, 4, 128, [80, 48], [64, 112], [2000, 1, 333], 16, 20, 1, 1, 0),      # a sequence of one row, grouped queries
    (BF16, 2, 1, 16, 128, [128], [128], [700, 699], 128, 3, 0, 2, 0),                # the largest group, no first block
    (BF16, 1, 2, 1, 128, [80, 80], [80, 80], [1500], 16, 2, 1, 1, 0),                # nothing left to choose
    (BF16, 1, 3, 3, 96, [33, 96, 8], [90, 7, 64], [777], 32, 7, 2, 3, 0),            # odd ranks
    (BF16, 2, 2, 5, 40, [40, 17], [24, 40], [900, 450], 64, 5, 1, 1, 0),
    (BF16, 2, 2, 1, 128, [80, 64], [64, 80], [1023, 512], 64, 5, 1, 1, 128),         # pages of 128 rows, shuffled
    (BF16, 1, 1, 2, 128, [80], [80], [5000], 16, 100, 4, 8, 256),                    # more blocks than a CTA's threads
    (BF16, 2, 1, 1, 64, [32], [32], [40000, 17000], 16, 1500, 3, 2, 0),              # several segments of keys, many of them chosen
    (BF16, 5, 30, 1, 16, [8] * 30, [16] * 30, [10240] * 5, 16, 40, 1, 1, 0),         # several steps of scores per CTA
    (BF16, 64, 33, 1, 16, [16] * 33, [8] * 33, [96 - i for i in range(64)], 16, 4, 1, 1, 0),      # many query rows in the merge
    (FP32, 1, 4, 1, 64, [32] * 4, [32] * 4, [500], 16, 8, 1, 1, 0),
    (FP32, 2, 2, 2, 80, [33, 80], [80, 12], [640, 200], 32, 6, 1, 2, 128),
    (BF16, 1, 1, 1, 64, [32], [32], [40], 64, 50, 3, 4, 0),                          # a budget beyond the cache
]


@pytest.mark.parametrize("dtype,batch,H,group,d,rk,rv,lens,block,n_blocks,sink,recent,page", SHAPES)
def test_sparse_decode_matches_the_definition(B, dtype, batch, H, group, d, rk, rv, lens, block, n_blocks, sink, recent, page):
    n_max = -(-(max(lens) + 8) // 256) * 256
    c = Case(B, dtype, batch, H, group, d, rk, rv, lens, n_max, seed=53, page_rows=page)
    c.lay.sparse_attach(block)
    assert c.lay.sparse_lens() == [0] * batch
    c.lay.sparse_sync()
    assert c.lay.sparse_lens() == [n // block * block for n in lens]
    for b in range(batch):
        for h in range(H):
            lo, hi = ts.block_bounds(c.rows(b, h, lens[b], "k"), block)
            got = bounds_of(c, b, h, block, lens[b] // block)
            assert np.array_equal(got[0], lo) and np.array_equal(got[1], hi), (b, h)
    q = randn((batch, 1, H * group, d), 61, dtype, 2.0)
    out, index = c.lay.decode_sparse(q, n_blocks, group=group, sink=sink, recent=recent, return_index=True)
    want, slack, idx = sparse_expected(c, q, block, n_blocks, sink, recent)
    assert np.array_equal(index.cpu().numpy(), idx)
    check(out, want, slack, dtype, "sparse")
    for ctas in (1, 7, 300):
        c.lay.set_option(B.EA_OPT_DECODE_CTAS, ctas)
        check(c.lay.decode_sparse(q, n_blocks, group=group, sink=sink, recent=recent), want, slack, dtype, f"sparse, {ctas} CTAs")
    c.lay.set_option(B.EA_OPT_DECODE_CTAS, 0)
    assert torch.equal(c.lay.decode_sparse(q, n_blocks, group=group, sink=sink, recent=recent), out)
    c.lay.poll_status()


@pytest.mark.parametrize("dtype", [BF16, FP32])
def test_alibi_takes_part_in_the_choice(B, dtype):
    c = Case(B, dtype, 2, 3, 1, 128, [80, 64, 48], [80, 64, 128], [1500, 900], 1536, seed=59, slopes=[0.05, 0.004, 0.0])
    c.lay.sparse_attach(32)
    c.lay.sparse_sync()
    q = randn((2, 1, 3, 128), 63, dtype, 2.0)
    out, index = c.lay.decode_sparse(q, 8, return_index=True)
    want, slack, idx = sparse_expected(c, q, 32, 8, 1, 1)
    assert np.array_equal(index.cpu().numpy(), idx)
    assert not np.array_equal(idx[:, 0], idx[:, 2])
    check(out, want, slack, dtype, "sparse with ALiBi")


def test_equal_scores_go_to_the_lower_block_and_zero_queries_choose_in_order(B):
    """Blocks that hold the same rows have the same score to the last bit; a zero query has no preference at all."""
    c = Case(B, BF16, 1, 2, 1, 128, [80, 80], [80, 80], [64], 1024, seed=67)
    k, v = c.k, c.v
    for _ in range(14):
        c.lay.append_kv(k, v)                          # fifteen times the same 64 rows
    c.lens = [960]
    c.lay.sparse_attach(64)
    c.lay.sparse_sync()
    for q in (randn((1, 1, 2, 128), 69, BF16), torch.zeros((1, 1, 2, 128), dtype=BF16, device="cuda")):
        _, index = c.lay.decode_sparse(q, 6, return_index=True)
        assert index.tolist() == [[[0, 1, 2, 3, 4, 14]] * 2]


def test_equal_scores_across_segments(B):
    """One block's rows over and over, 2500 blocks of them, with a few others in between: those are chosen, and of the equal
    ones the first, wherever in the list they lie."""
    c = Case(B, BF16, 1, 1, 1, 64, [32], [32], [16], 40064, seed=68)
    k, v = c.k[:, :, :, :], c.v[:, :, :, :]
    c.lay.append_kv(k.repeat(1, 2499, 1, 1), v.repeat(1, 2499, 1, 1))
    slab = c.lay.cache_rows(0, "k")
    q = randn((1, 1, 1, 64), 70, BF16)
    rank_q = np64(q)[0, 0, 0] @ np.float64(c.U_k[0])
    big = torch.tensor(np.sign(rank_q) * 9.0, device="cuda").to(BF16)
    high = [700, 1500, 2400]
    for j in high:
        slab[0, 16 * j + 5, :32] = big
    c.lens = [40000]
    c.lay.sparse_attach(16)
    c.lay.sparse_sync()
    for n_blocks in (6, 1200, 2300):
        out, index = c.lay.decode_sparse(q, n_blocks, return_index=True)
        middle = [j for j in range(1, 2499) if j not in high]
        want = sorted([0, 2499] + high + middle[:n_blocks - 5])
        assert index[0, 0].tolist() == want
        e, slack, idx = sparse_expected(c, q, 16, n_blocks, 1, 1)
        assert idx[0, 0].tolist() == want
        check(out, e, slack, BF16, f"{n_blocks} blocks")


def test_side_stream_and_two_layers_at_once(B):
    """Two layers with buffers of their own on two streams: each call's launches depend on their own stream alone."""
    cs = [Case(B, BF16, 2, 4, 2, 128, [80] * 4, [80] * 4, [6000, 3000], 6144, seed=s) for s in (105, 107)]
    qs = [randn((2, 1, 8, 128), 109 + i, BF16, 2.0) for i in range(2)]
    for c in cs:
        c.lay.sparse_attach(32)
        c.lay.sparse_sync()
    want = [c.lay.decode_sparse(q, 12, group=2) for c, q in zip(cs, qs)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    outs = [[torch.zeros_like(w) for _ in range(30)] for w in want]
    for i in range(30):
        for c, q, s, o in zip(cs, qs, streams, outs):
            c.lay.decode_sparse(q, 12, group=2, out=o[i], stream=s)
    torch.cuda.synchronize()
    for w, o in zip(want, outs):
        assert all(torch.equal(w, x) for x in o)


def test_blocks_beyond_32_bit_offsets(B):
    """A key slab of 2 GiB per sequence; a handful of blocks near the end of the second sequence score highest."""
    n_max, d, n, block = 2 ** 23 + 128, 128, 2 ** 23 + 90, 128
    U = np.eye(d, dtype=np.float32)
    lay = B.EigenAttnLayer(2, 1, d, n_max, BF16, [U], [U])
    for which in "kv":
        lay.cache_rows(0, which).zero_()
    lay.set_lens([1, n])
    lay.sparse_attach(block)
    far = [n // block - 3, n // block - 1000, 40000]
    rows = randn((2, 3, d), 3, BF16)
    rows[0, :, 0] = 32.0
    for i, j in enumerate(far):
        lay.cache_rows(0, "k")[1, block * j + 17 * i] = rows[0, i]
        lay.cache_rows(0, "v")[1, block * j + 17 * i] = rows[1, i]
    lay.sparse_sync()
    q = randn((2, 1, 1, d), 5, BF16)
    q[:, :, :, 0] = 32.0
    out, index = lay.decode_sparse(q, 5, return_index=True)
    last = (n + block - 1) // block - 1
    assert index[:, 0].tolist() == [[0, -1, -1, -1, -1], sorted([0, last] + far)]
    s = np64(rows[0]) @ np64(q[1, 0, 0]) / np.sqrt(d)
    w = np.exp(s - s.max())
    w /= w.sum()
    e_s = (2.0 ** -16 + (2 * d + 4) * 2.0 ** -23) * (np.abs(np64(rows[0])) @ np.abs(np64(q[1, 0, 0]))).max() / np.sqrt(d)
    assert s.min() > 60                                # the zero rows beside them: 640 times e^-60
    e_w = 2.2 * e_s + 2.0 ** -15 + 1000 * 2.0 ** -24
    check(out[1, 0, 0], w @ np64(rows[1]), (2 * e_w + (d + 2) * 2.0 ** -22) * (w @ np.abs(np64(rows[1]))), BF16, "far blocks")


def test_a_budget_that_covers_everything_is_ordinary_decode(B):
    c = Case(B, BF16, 2, 2, 1, 128, [80, 64], [64, 80], [700, 450], 1024, seed=71)
    c.lay.sparse_attach(32)                            # (no bounds needed when nothing is left out)
    q = randn((2, 1, 2, 128), 73, BF16, 2.0)
    out, index = c.lay.decode_sparse(q, 22, return_index=True)
    want, slack, idx = sparse_expected(c, q, 32, 22, 1, 1)
    assert np.array_equal(index.cpu().numpy(), idx) and idx[0, 0, -1] == 21 and idx[1, 0, -1] == -1
    check(out, want, slack, BF16, "all blocks")
    diff = (out.float() - c.lay.decode(q).float()).abs()
    assert bool((diff <= 2 * 2.0 ** -8 * out.float().abs() + 1e-4).all())     # two roundings of nearly one number


def test_bounds_follow_the_cache(B):
    """Appending, rewinding, unequal lengths, a new page table: a call never uses bounds of rows that have changed."""
    c = Case(B, BF16, 2, 2, 1, 64, [32, 48], [48, 32], [600, 600], 1024, seed=79)
    lay = c.lay
    lay.sparse_attach(32)
    q = randn((2, 1, 2, 64), 83, BF16, 2.0)

    def refused():
        with pytest.raises(B.EigenAttnError) as e:
            lay.decode_sparse(q, 5)
        assert e.value.status == B.EA_ERR_INVALID_ARG and "sparse_sync" in str(e.value)

    def agrees():
        out, index = lay.decode_sparse(q, 5, return_index=True)
        want, slack, idx = sparse_expected(c, q, 32, 5, 1, 1)
        assert np.array_equal(index.cpu().numpy(), idx)
        check(out, want, slack, BF16, "after a change")
    refused()
    lay.sparse_sync()
    agrees()
    for i in range(40):                                # one token at a time; the newest block needs no bounds
        k, v = randn((2, 1, 2, 64), 900 + i, BF16), randn((2, 1, 2, 64), 990 + i, BF16)
        lay.decode_step(q, k, v)
        c.lens = [n + 1 for n in c.lens]
        if i == 7:
            agrees()                                   # 608 rows: 19 complete blocks, 18 with bounds, the newest one open
    refused()                                          # 640 rows: block 18 has filled and is not the newest any more
    lay.sparse_sync()
    agrees()
    lay.set_lens([500, 641 - 1])                       # one sequence rewound, then other rows in its place
    assert lay.sparse_lens() == [480, 640]
    lay.append_kv(randn((2, 100, 2, 64), 5, BF16, 3.0), randn((2, 100, 2, 64), 6, BF16))
    c.lens = [600, 740]
    refused()
    lay.sparse_sync()
    assert lay.sparse_lens() == [576, 736]
    agrees()
    # a drafted tree does not touch the bounds; what it accepts does
    lay.tree_attach(40)
    masks, _ = trees(2, 40, 3, "chain")
    qt, kt, vt = randn((2, 40, 2, 64), 7, BF16), randn((2, 40, 2, 64), 8, BF16), randn((2, 40, 2, 64), 9, BF16)
    out = lay.decode_tree(qt, kt, vt, mask_tensor(masks))
    check(out, *tree_expected(c, qt, masks, 40), BF16, "tree")
    agrees()
    lay.tree_commit([list(range(36)), [0, 3, 5]], 40)
    c.lens = [636, 743]
    lay.sparse_sync()
    agrees()
    lay.set_len(636)
    c.lens = [636, 636]
    agrees()
    lay.set_page_table([[0, 1, 2, 3, 4, 5, 6, 7], [8, 9, 10, 11, 12, 13, 14, 15]], 128)     # the same rows, but who knows
    c.table, c.page_rows = [[0, 1, 2, 3, 4, 5, 6, 7], [8, 9, 10, 11, 12, 13, 14, 15]], 128
    refused()
    lay.sparse_sync()
    agrees()


def test_captured_call_replays_with_new_queries(B):
    c = Case(B, BF16, 2, 2, 2, 128, [80, 80], [80, 80], [900, 900], 1024, seed=89)
    c.lay.sparse_attach(32)
    c.lay.sparse_sync()
    q = randn((2, 1, 4, 128), 91, BF16, 2.0)
    out = torch.zeros((2, 1, 4, 128), dtype=BF16, device="cuda")
    c.lay.decode_sparse(q, 6, group=2, out=out)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        c.lay.decode_sparse(q, 6, group=2, out=out)
    for seed in (93, 95):
        q.copy_(randn((2, 1, 4, 128), seed, BF16, 2.0))
        g.replay()
        torch.cuda.synchronize()
        want, slack, _ = sparse_expected(c, q, 32, 6, 1, 1)
        check(out, want, slack, BF16, "replayed")


def test_rank_space_forms(B):
    """Merged weights: packed rank-space queries in, packed o' out."""
    group = 2
    c = Case(B, BF16, 2, 2, group, 64, [40, 24], [16, 56], [600, 333], 1024, seed=97)
    c.lay.sparse_attach(16)
    c.lay.sparse_sync()
    offs_k, offs_v = c.lay.offs_k, c.lay.offs_v
    qp = randn((2, 1, group * offs_k[-1]), 99, BF16, 2.0)
    low = c.lay.decode_sparse(qp, 7, group=group, q_preprojected=True, out_lowrank=True)
    for b in range(2):
        for h in range(2):
            K, V = c.rows(b, h, c.lens[b], "k"), c.rows(b, h, c.lens[b], "v")
            qh = np64(qp[b, 0, group * offs_k[h]:group * offs_k[h + 1]]).reshape(group, -1)[:, :c.rk[h]]
            blocks = ts.choose_blocks(qh, K, 16, 7, 1, 1, c.d)
            rows = [j for j in range(c.lens[b]) if j // 16 in set(blocks)]
            got = np64(low[b, 0, group * offs_v[h]:group * offs_v[h + 1]]).reshape(group, -1)
            for i in range(group):
                want = ts.blocks_head(qh[i], K, V, blocks, 16, np.float64(c.U_v[h]), lowrank_out=True)
                s = K[rows] @ qh[i] / 8.0
                w = np.exp(s - s.max()) / np.exp(s - s.max()).sum()
                e_s = c.score_error(qh[i] @ np.float64(c.U_k[h]).T, K[rows], h, 0.0, 0)
                check(got[i, :c.rv[h]], want, c.bound(w, V[rows], e_s, h, lowrank=True), BF16, f"o' of unit {b, h}")


def test_refusals(B):
    c = Case(B, BF16, 1, 2, 1, 64, [32, 32], [32, 32], [300], 512, seed=103)
    lay = c.lay
    q = randn((1, 1, 2, 64), 1, BF16)

    def refused(status, fn):
        with pytest.raises(B.EigenAttnError) as e:
            fn()
        assert e.value.status == status, e.value
    refused(B.EA_ERR_INVALID_ARG, lambda: lay.decode_sparse(q, 4))
    refused(B.EA_ERR_INVALID_ARG, lay.sparse_sync)
    refused(B.EA_ERR_INVALID_ARG, lay.sparse_lens)
    for rows in (0, 8, 48, 256):
        refused(B.EA_ERR_SHAPE, lambda: lay.sparse_attach(rows))
    buf = lay.sparse_attach(32)
    raw = B.lib.eigen_attn_sparse_attach
    assert raw(lay.handle, 32, buf.data_ptr() + 16, 1 << 30, None) == B.EA_ERR_INVALID_ARG
    assert raw(lay.handle, 32, buf.data_ptr(), 64, None) == B.EA_ERR_CAPACITY
    lay.sparse_sync()
    for args in ((1, 1, 1), (4, -1, 1), (4, 1, 0), (0, 0, 1)):
        refused(B.EA_ERR_SHAPE, lambda: lay.decode_sparse(q, args[0] if args[0] > 0 else 0, sink=args[1], recent=args[2]))
    call = [lay.handle, q.data_ptr(), 0, 1, 4, 1, 1, q.data_ptr(), 0, None, 0, None]
    for at, value, status in ((1, None, -1), (7, None, -1), (3, 0, -2), (3, 17, -2), (10, 4, -1)):
        bad = list(call)
        bad[at] = value
        assert B.lib.eigen_attn_decode_sparse(*bad) == status, (at, value)
    lay.set_alibi([0.5, 0.25])
    refused(B.EA_ERR_UNSUPPORTED, lambda: lay.decode_sparse(randn((1, 1, 4, 64), 1, BF16), 4, group=2))
    lay.set_alibi(None)
    lay.set_rope(10000.0)
    refused(B.EA_ERR_UNSUPPORTED, lambda: lay.decode_sparse(q, 4))
    lay.set_rope(0.0)
    lay.set_len(0)
    refused(B.EA_ERR_SHAPE, lambda: lay.decode_sparse(q, 4))
    lay.sparse_detach()
    refused(B.EA_ERR_INVALID_ARG, lambda: lay.decode_sparse(q, 4))
    lay.poll_status()
