"""Tree attention on the GPU against the 64-bit definition: drafted tokens over the cached rows and their ancestors, and
the acceptance of a path."""
import numpy as np
import pytest
import torch

from mq_helpers import BF16, FP32, Case, check, mask_tensor, np64, randn, tree_expected, trees

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    from paper_2408_05646_b200 import build
    build.build_library()
    from paper_2408_05646_b200 import binding
    return binding


def drafted(c, T, seed, peak=1.5):
    return (randn((c.batch, T, c.H * c.group, c.d), seed, c.dtype, peak), randn((c.batch, T, c.H, c.d), seed + 1, c.dtype),
            randn((c.batch, T, c.H, c.d), seed + 2, c.dtype))


def check_stored(c, k, v, T):
    """The drafted rows behind each sequence's own: projections rounded once (sum of d products in single precision)."""
    for b in range(c.batch):
        for h in range(c.H):
            for which, x, U in (("k", k, c.U_k[h]), ("v", v, c.U_v[h])):
                x, U = np64(x)[b, :, h], np.float64(U)
                got = c.rows(b, h, c.lens[b] + T, which)[c.lens[b]:]
                check(got, x @ U, c.d * 2.0 ** -24 * (np.abs(x) @ np.abs(U)), c.dtype, f"{which} rows of unit {b, h}")


SHAPES = [
    # dtype, batch, H, group, d, rk, rv, lens, T, kind, page
    (BF16, 1, 2, 1, 128, [80, 80], [80, 80], [300], 4, "chain", 0),              # one user, a short chain
    (BF16, 1, 1, 1, 128, [80], [80], [0], 1, "chain", 0),                        # nothing cached, one token
    (BF16, 1, 1, 1, 64, [32], [32], [1], 2, "tree", 0),
    (BF16, 2, 2, 1, 128, [80, 80], [80, 80], [127, 128], 8, "tree", 0),          # the drafted rows start at / before a tile's end
    (BF16, 2, 2, 1, 128, [64, 64], [64, 64], [129, 0], 9, "tree", 0),            # a sequence without rows beside another
    (BF16, 2, 2, 4, 128, [80, 80], [80, 80], [1037, 640], 16, "tree", 0),        # grouped queries: 64 query rows
    (BF16, 1, 2, 4, 128, [128, 128], [128, 128], [515], 13, "tree", 0),          # full rank, 52 query rows
    (BF16, 1, 1, 16, 128, [80], [80], [200], 64, "tree", 0),                     # the most query rows a call can have
    (BF16, 2, 3, 2, 128, [24, 40, 128], [8, 72, 56], [333, 90], 63, "tree", 0),  # ranks that differ, odd multiples of 8
    (BF16, 2, 3, 1, 96, [48, 96, 33], [90, 7, 64], [257, 700], 5, "any", 0),     # ranks that are no multiples of 8, any mask
    (BF16, 1, 2, 3, 40, [40, 17], [24, 40], [65], 7, "any", 0),                  # d_head that is no multiple of 16
    (BF16, 3, 2, 1, 128, [80, 64], [64, 80], [500, 256, 130], 31, "tree", 128),  # pages of 128 rows, shuffled
    (BF16, 2, 1, 8, 128, [112], [96], [900, 3], 3, "any", 256),
    (BF16, 2, 1, 2, 128, [80], [80], [6000, 5000], 20, "tree", 0),               # many tiles for one unit
    (BF16, 1, 2, 3, 128, [64, 48], [64, 40], [1500], 60, "any", 0),              # 180 query rows, narrow heads
    (BF16, 2, 1, 1, 128, [80], [80], [200, 100], 40, "tree", 256),               # pages that do not divide n_max (384 rows)
    (BF16, 2, 1, 3, 128, [80], [80], [300, 0], 20, "any", 0),                    # empty masks beside no cached row, 60 query rows
    (BF16, 40, 1, 4, 64, [32], [32], [37 * i % 290 for i in range(40)], 8, "tree", 0),     # more sequences than a warp has lanes
    (FP32, 1, 4, 1, 64, [32] * 4, [32] * 4, [512], 5, "tree", 0),
    (FP32, 2, 2, 2, 80, [33, 80], [80, 12], [100, 0], 17, "any", 0),
    (FP32, 2, 2, 1, 128, [128, 64], [128, 32], [260, 131], 64, "tree", 128),
]


@pytest.mark.parametrize("impl", [0, 1])               # 0: tcgen05 products from 17 query rows on, 1: warp-level products
@pytest.mark.parametrize("dtype,batch,H,group,d,rk,rv,lens,T,kind,page", SHAPES)
def test_tree_matches_the_definition(B, dtype, batch, H, group, d, rk, rv, lens, T, kind, page, impl):
    if impl == 1 and (dtype == FP32 or T * group <= 16):
        pytest.skip("one kernel serves this case")
    n_max = 384 if (page, T) == (256, 40) else -(-(max(lens) + T + 5) // 256) * 256
    c = Case(B, dtype, batch, H, group, d, rk, rv, lens, n_max, seed=11, page_rows=page)
    c.lay.set_option(B.EA_OPT_TREE_IMPL, impl)
    q, k, v = drafted(c, T, 31)
    masks, _ = trees(batch, T, 7, kind)
    c.lay.tree_attach(T, group)
    before = c.lay.lens()
    out = c.lay.decode_tree(q, k, v, mask_tensor(masks), group=group)
    assert c.lay.lens() == before == lens
    check_stored(c, k, v, T)
    want, slack = tree_expected(c, q, masks, T)
    check(out, want, slack, dtype, "tree")
    for ctas in (1, 7, 300):                           # CTAs per unit must not matter
        c.lay.set_option(B.EA_OPT_DECODE_CTAS, ctas)
        check(c.lay.decode_tree(q, k, v, mask_tensor(masks), group=group), want, slack, dtype, f"tree, {ctas} CTAs")
    c.lay.set_option(B.EA_OPT_DECODE_CTAS, 0)
    assert torch.equal(c.lay.decode_tree(q, k, v, mask_tensor(masks), group=group), out)      # the same again, bit for bit
    c.lay.poll_status()


@pytest.mark.parametrize("dtype,batch,H,group,d,r,T,off", [
    (BF16, 8, 25, 1, 64, 32, 64, 0),                   # 128 rows per CTA in the projection, 64 in the merge
    (BF16, 8, 25, 1, 64, 32, 64, 1),                   # tensors that begin one element behind a 16-byte boundary
    (BF16, 3, 14, 4, 128, 72, 24, 1),                  # 64 rows per CTA in the projection, d_head 128
    (FP32, 8, 25, 1, 40, 24, 64, 1),
    (FP32, 2, 2, 1, 64, 32, 3, 1),                     # few rows
    (BF16, 2, 2, 1, 64, 32, 3, 1),
])
def test_many_rows_and_unaligned_tensors(B, dtype, batch, H, group, d, r, T, off):
    """Every shape of the projection and the merge: stored rows are bit for bit those of append_kv, whatever the alignment."""
    lens = [(29 * i) % 41 for i in range(batch)]
    rk, rv = [r - 3 * (h % 4) for h in range(H)], [r - 5 * (h % 3) for h in range(H)]
    a = Case(B, dtype, batch, H, group, d, rk, rv, lens, 128, seed=47)
    ref = Case(B, dtype, batch, H, group, d, rk, rv, lens, 128, seed=47)
    q, k, v = drafted(a, T, 141)
    masks, _ = trees(batch, T, 17)
    m = mask_tensor(masks)
    a.lay.tree_attach(T, group)

    def moved(x):                                      # the same numbers, `off` elements further
        flat = torch.full((x.numel() + 8,), 3.0, dtype=dtype, device="cuda")
        flat[off:off + x.numel()] = x.reshape(-1)
        return flat, flat[off:off + x.numel()].view(x.shape)
    flat, out = moved(torch.full_like(q, -7.0))
    a.lay.decode_tree(moved(q)[1], moved(k)[1], moved(v)[1], m, group=group, out=out)
    assert (flat[:off] == 3.0).all() and (flat[off + q.numel():] == 3.0).all()
    units = {(b, h) for b in range(batch) for h in range(H) if (b * H + h) % (batch * H // 4) == 0 or (b, h) == (batch - 1, H - 1)}
    want, slack = tree_expected(a, q, masks, T, units=units)
    for b, h in units:
        at = slice(h * group, (h + 1) * group)
        check(out[b:b + 1, :, at], want[b:b + 1, :, at], slack[b:b + 1, :, at], dtype, f"unit {b, h}")
    assert torch.isfinite(out).all()
    ref.lay.append_kv(k, v)                            # the same rows by the ordinary way
    a.lay.tree_commit([list(range(T))] * batch, T)
    assert a.lay.lens() == ref.lay.lens()
    for h in range(H):
        for which in "kv":
            x, y = a.lay.cache_rows(h, which), ref.lay.cache_rows(h, which)
            for b in range(batch):
                assert torch.equal(x[b, :lens[b] + T], y[b, :lens[b] + T]), (b, h, which)


def test_commit_of_more_sequences_than_one_launch_takes(B):
    batch, T = 150, 6
    lens = [(7 * i) % 50 for i in range(batch)]
    c = Case(B, BF16, batch, 1, 1, 16, [8], [16], lens, 64, seed=61)
    q, k, v = drafted(c, T, 161)
    masks, _ = trees(batch, T, 21)
    c.lay.tree_attach(T)
    c.lay.decode_tree(q, k, v, mask_tensor(masks))
    g = np.random.default_rng(5)
    paths = [sorted(int(x) for x in g.permutation(T)[:g.integers(0, T + 1)]) for _ in range(batch)]
    slabs = {w: np64(c.lay.cache_rows(0, w)) for w in "kv"}
    c.lay.tree_commit(paths, T)
    assert c.lay.lens() == [n + len(p) for n, p in zip(lens, paths)]
    for w in "kv":
        got = np64(c.lay.cache_rows(0, w))
        for b in range(batch):
            want = slabs[w][b].copy()
            want[lens[b]:lens[b] + len(paths[b])] = slabs[w][b][[lens[b] + s for s in paths[b]]]
            assert np.array_equal(got[b], want), (b, w)


@pytest.mark.parametrize("T", [4, 24])                 # warp-level products, tcgen05 products
def test_rows_beyond_32_bit_offsets(B, T):
    """A head's slab of 4 GiB: rows of the second sequence lie at byte offsets past 2^31 and 2^32.  All rows are zero but the
    last 50, whose scores are some 60 above: the 8.4 million others together weigh e^-60 * 2^23 of them."""
    n_max, d, n = 2 ** 23 + 256, 128, 2 ** 23 + 100
    U = np.eye(d, dtype=np.float32)
    lay = B.EigenAttnLayer(2, 1, d, n_max, BF16, [U], [U])
    for which in "kv":
        lay.cache_rows(0, which).zero_()
    lay.set_lens([40, n])
    rows = randn((2, 50, d), 3, BF16)
    rows[0, :, 0] = 32.0                               # times the query's 32 / sqrt(128): a score of 90, the rest moves it by ~3
    lay.cache_rows(0, "k")[1, n - 50:n] = rows[0]
    lay.cache_rows(0, "v")[1, n - 50:n] = rows[1]
    q, k, v = (randn((2, T, 1, d), 5 + i, BF16) for i in range(3))
    q[:, :, :, 0] = 32.0
    k[:, :, :, 0] = 32.0
    masks, _ = trees(2, T, 1)
    lay.tree_attach(T)
    out = lay.decode_tree(q, k, v, mask_tensor(masks))
    lay.poll_status()
    assert torch.equal(lay.cache_rows(0, "k")[1, n:n + T], k[1, :, 0]) and torch.equal(lay.cache_rows(0, "v")[1, n:n + T], v[1, :, 0])
    K, V = np.concatenate([np64(rows[0]), np64(k[1, :, 0])]), np.concatenate([np64(rows[1]), np64(v[1, :, 0])])
    for t in range(T):
        keep = [j for j in range(50 + T) if j < 50 or masks[1][t] >> (j - 50) & 1]
        s = K[keep] @ np64(q[1, t, 0]) / np.sqrt(d)
        assert s.min() > 60
        w = np.exp(s - s.max())
        w /= w.sum()
        e_s = (2.0 ** -16 + (2 * d + 4) * 2.0 ** -23) * (np.abs(K[keep]) @ np.abs(np64(q[1, t, 0]))).max() / np.sqrt(d)
        e_w = 2.2 * e_s + 2.0 ** -15 + 2 ** 23 * np.exp(-60.0) + 200 * 2.0 ** -24
        slack = (2 * e_w + (d + 2) * 2.0 ** -22) * (w @ np.abs(V[keep]))
        check(out[1, t, 0], w @ V[keep], slack, BF16, f"token {t}")


@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("lens", [[400, 400], [300, 0]])
def test_alibi_positions_count_ancestors(B, dtype, lens):
    c = Case(B, dtype, 2, 3, 1, 128, [80, 64, 48], [80, 64, 128], lens, 512, seed=13, slopes=[0.5, 0.0625, 0.0])
    q, k, v = drafted(c, 12, 41, peak=3.0)
    masks, _ = trees(2, 12, 9)
    c.lay.tree_attach(12)
    out = c.lay.decode_tree(q, k, v, mask_tensor(masks))
    check(out, *tree_expected(c, q, masks, 12), dtype, "tree with ALiBi")


@pytest.mark.parametrize("dtype", [BF16, FP32])
def test_strided_tensors_and_rank_space_forms(B, dtype):
    """Token tensors that are slices of larger ones; merged weights in (packed q', k', v') and out (packed o')."""
    T, group = 6, 2
    c = Case(B, dtype, 2, 2, group, 64, [40, 24], [16, 56], [70, 33], 256, seed=17)
    q, k, v = drafted(c, T, 51)
    masks, _ = trees(2, T, 3)
    m = mask_tensor(masks)
    c.lay.tree_attach(T, group)
    plain = c.lay.decode_tree(q, k, v, m, group=group)

    def inside(x, fill):
        big = torch.full((x.shape[0] + 1, 2 * x.shape[1] + 1) + x.shape[2:], fill, dtype=dtype, device=x.device)
        view = big[1:, 1::2]
        view.copy_(x)
        return big, view
    kv = torch.full((2, T, 2) + k.shape[2:], 9.0, dtype=dtype, device="cuda")
    kv[:, :, 0], kv[:, :, 1] = k, v                    # k and v interleaved by token: one stride for both
    big, out = inside(torch.zeros_like(plain), -7.0)
    c.lay.decode_tree(inside(q, 5.0)[1], kv[:, :, 0], kv[:, :, 1], m, group=group, out=out)
    assert torch.equal(out, plain)
    rest = big.clone()
    rest[1:, 1::2] = -7.0
    assert (rest == -7.0).all()                        # nothing beside the output rows was written
    # rank-space output
    low = c.lay.decode_tree(q, k, v, m, group=group, out_lowrank=True)
    want, slack = tree_expected(c, q, masks, T, lowrank=True)
    for h in range(2):
        at = group * c.lay.offs_v[h]
        rp = c.lay.offs_v[h + 1] - c.lay.offs_v[h]
        got = low[:, :, at:at + group * rp].reshape(2, T, group, rp)
        check(got[..., :c.rv[h]], want[h], slack[h], dtype, f"o' of head {h}")
        assert not got[..., c.rv[h]:].any()
    # rank-space input: rows of the packed width, padding columns holding anything
    offs_k, offs_v = c.lay.offs_k, c.lay.offs_v
    qp, kp, vp = (randn((2, T, w), 61 + i, dtype) for i, w in enumerate((group * offs_k[-1], offs_k[-1], offs_v[-1])))
    out = c.lay.decode_tree(qp, kp, vp, m, group=group, q_preprojected=True, kv_preprojected=True)
    for b in range(2):
        for h in range(2):
            rows = c.rows(b, h, c.lens[b] + T, "k")[c.lens[b]:]
            assert np.array_equal(rows, np64(kp[b, :, offs_k[h]:offs_k[h] + c.rk[h]]))
    low = [np64(qp[:, :, group * offs_k[h]:group * offs_k[h + 1]].reshape(2, T, group, -1)) for h in range(2)]
    want, slack = tree_expected(c, None, masks, T, rank_q=lambda b, h, i: low[h][b, :, i, :c.rk[h]])
    check(out, want, slack, dtype, "rank-space input")


@pytest.mark.parametrize("dtype,group", [(BF16, 1), (BF16, 4), (FP32, 1)])
@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_what_a_masked_token_holds_does_not_matter(B, dtype, group, bad):
    """A sibling branch whose rows are infinities or NaN, and such rows behind the sequence: the tokens that do not see
    them return what they return with ordinary numbers there."""
    T, poison = 20, 7
    c = Case(B, dtype, 2, 2, group, 128, [80, 64], [80, 96], [200, 140], 512, seed=19)
    for h in range(2):
        for which in "kv":                             # rows nobody has written yet
            c.lay.cache_rows(h, which)[:, 240:].fill_(bad)
    q, k, v = drafted(c, T, 71)
    masks, _ = trees(2, T, 5)
    masks = [[m if t == poison else m & ~(1 << poison) for t, m in enumerate(row)] for row in masks]
    c.lay.tree_attach(T, group)
    want = c.lay.decode_tree(q, k, v, mask_tensor(masks), group=group)
    k, v = k.clone(), v.clone()
    k[:, poison], v[:, poison] = bad, bad
    out = c.lay.decode_tree(q, k, v, mask_tensor(masks), group=group)
    others = [t for t in range(T) if t != poison]
    assert torch.isfinite(want[:, others]).all()
    w, s = np64(want[:, others]), np.abs(np64(want[:, others]))
    # the same rows with the same weights: at most the order of a few sums differs
    check(out[:, others], w, 2.0 ** -14 * (s + 1.0), dtype, "tokens beside a poisoned one")
    assert not torch.isfinite(out[:, poison]).any()    # the token that sees itself is what its rows make it


@pytest.mark.parametrize("dtype,page", [(BF16, 0), (BF16, 128), (FP32, 0)])
def test_commit_moves_the_accepted_rows_and_nothing_else(B, dtype, page):
    T, lens = 64, [130, 0, 77]
    c = Case(B, dtype, 3, 2, 1, 64, [40, 64], [64, 16], lens, 256, seed=23, page_rows=page)
    q, k, v = drafted(c, T, 81)
    masks, _ = trees(3, T, 15)
    c.lay.tree_attach(T)
    c.lay.decode_tree(q, k, v, mask_tensor(masks))
    paths = [[0, 2, 3, 9, 40, 63], [], list(range(1, 64))]
    cap = 256
    before = [[[c.rows(b, h, cap, w) for w in "kv"] for h in range(2)] for b in range(3)]
    c.lay.tree_commit(paths, T)
    assert c.lay.lens() == [n + len(p) for n, p in zip(lens, paths)]
    for b in range(3):
        for h in range(2):
            for i, w in enumerate("kv"):
                want = before[b][h][i].copy()
                want[lens[b]:lens[b] + len(paths[b])] = before[b][h][i][[lens[b] + s for s in paths[b]]]
                assert np.array_equal(c.rows(b, h, cap, w), want), (b, h, w)


@pytest.mark.parametrize("dtype,group", [(BF16, 1), (BF16, 2), (FP32, 1)])
def test_speculative_steps_equal_one_token_at_a_time(B, dtype, group):
    """Draft, verify, accept, three times over; then the cache is what appending the accepted tokens one by one gives, and
    the next ordinary decode agrees with the layer that was filled that way."""
    lens, T = [60, 131], 10
    a = Case(B, dtype, 2, 2, group, 128, [80, 48], [80, 64], lens, 256, seed=29)
    b = Case(B, dtype, 2, 2, group, 128, [80, 48], [80, 64], lens, 256, seed=29)
    a.lay.tree_attach(T, group)
    g = np.random.default_rng(3)
    for step in range(3):
        q, k, v = drafted(a, T, 100 + 10 * step)
        masks, parents = trees(2, T, step)
        out = a.lay.decode_tree(q, k, v, mask_tensor(masks), group=group)
        check(out, *tree_expected(a, q, masks, T), dtype, f"step {step}")
        paths = []
        for s in range(2):
            p = [int(g.integers(0, T))]
            while parents[s][p[0]] >= 0:
                p.insert(0, parents[s][p[0]])
            paths.append(p[:max(0, len(p) - s * step)])
        a.lay.tree_commit(paths, T)
        longest = max(len(p) for p in paths)
        if longest:                                     # the accepted tokens, appended (and cut to each sequence's count)
            idx = torch.tensor([p + [0] * (longest - len(p)) for p in paths], device="cuda")
            take = lambda x: torch.stack([x[s][idx[s]] for s in range(2)])
            b.lay.append_kv(take(k), take(v))
        b.lay.set_lens([n + len(p) for n, p in zip(b.lens, paths)])
        a.lens = b.lens = [n + len(p) for n, p in zip(b.lens, paths)]
        assert a.lay.lens() == b.lay.lens() == a.lens
    for s in range(2):
        for h in range(2):
            for w in "kv":
                assert np.array_equal(a.rows(s, h, a.lens[s], w), b.rows(s, h, b.lens[s], w))
    q = randn((2, 1, 2, 128), 7, dtype)
    assert torch.equal(a.lay.decode(q), b.lay.decode(q))
    # equal counts keep the differences between the lengths: no upload, the same state
    q, k, v = drafted(a, T, 400)
    a.lay.decode_tree(q, k, v, mask_tensor(trees(2, T, 1, "chain")[0]), group=group)
    a.lay.tree_commit([[0, 1, 2], [0, 1, 2]], T)
    assert a.lay.lens() == [n + 3 for n in a.lens]


def test_captured_call_replays_with_new_contents(B):
    """A captured call reads the tensors as they are at replay: queries, drafted rows and masks may change."""
    T, group = 8, 2
    c = Case(B, BF16, 2, 2, group, 128, [80, 80], [80, 80], [300, 300], 512, seed=37)
    c.lay.tree_attach(T, group)
    q, k, v = drafted(c, T, 91)
    m = mask_tensor(trees(2, T, 1)[0])
    out = torch.zeros((2, T, 2 * group, 128), dtype=BF16, device="cuda")
    c.lay.decode_tree(q, k, v, m, group=group, out=out)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        c.lay.decode_tree(q, k, v, m, group=group, out=out)
        with pytest.raises(B.EigenAttnError) as e:
            c.lay.tree_commit([[0], [0]], T)
        assert e.value.status == B.EA_ERR_UNSUPPORTED
    for seed in (200, 300):
        for dst, src in zip((q, k, v), drafted(c, T, seed)):
            dst.copy_(src)
        masks = trees(2, T, seed)[0]
        m.copy_(mask_tensor(masks))
        g.replay()
        torch.cuda.synchronize()
        check(out, *tree_expected(c, q, masks, T), BF16, "replayed")
    s = torch.cuda.Stream()                            # another stream, ordered by the caller
    s.wait_stream(torch.cuda.current_stream())
    again = c.lay.decode_tree(q, k, v, m, group=group, stream=s)
    torch.cuda.current_stream().wait_stream(s)
    assert torch.equal(again, out)


def test_refusals(B):
    c = Case(B, BF16, 2, 2, 1, 64, [32, 32], [32, 32], [10, 10], 64, seed=43)
    lay = c.lay
    q, k, v = drafted(c, 4, 1)
    m = mask_tensor(trees(2, 4, 1)[0])

    def refused(status, fn):
        with pytest.raises(B.EigenAttnError) as e:
            fn()
        assert e.value.status == status, e.value
        assert lay.lens() == [10, 10]
    refused(B.EA_ERR_INVALID_ARG, lambda: lay.decode_tree(q, k, v, m))                       # no scratch
    for bad in ((0, 1), (65, 1), (4, 0), (4, 17)):
        refused(B.EA_ERR_SHAPE, lambda: lay.tree_attach(*bad))
    buf = lay.tree_attach(2)
    refused(B.EA_ERR_CAPACITY, lambda: lay.decode_tree(q, k, v, m))                          # scratch for fewer tokens
    raw = B.lib.eigen_attn_tree_attach
    assert raw(lay.handle, 4, 1, buf.data_ptr() + 16, 1 << 30) == B.EA_ERR_INVALID_ARG
    assert raw(lay.handle, 4, 1, buf.data_ptr(), 1) == B.EA_ERR_CAPACITY
    lay.tree_attach(4)
    lay.decode_tree(q, k, v, m)
    args = [lay.handle, q.data_ptr(), 0, 0, 1, k.data_ptr(), v.data_ptr(), 0, 0, 4, m.data_ptr(), q.data_ptr(), 0, 0, 0, None]
    for at, value, status in ((1, None, -1), (5, None, -1), (6, None, -1), (10, None, -1), (11, None, -1), (4, 0, -2), (4, 17, -2),
                              (9, 0, -2), (9, 65, -2), (14, 8, -1), (10, m.data_ptr() + 4, -1)):
        call = list(args)
        call[at] = value
        assert B.lib.eigen_attn_decode_tree(*call) == status, (at, value)
    for paths, status in (([[0, 0], []], -1), ([[2, 1], []], -1), ([[4], []], -1), ([[-1], []], -1)):
        refused(status, lambda: lay.tree_commit(paths, 4))
    refused(B.EA_ERR_SHAPE, lambda: lay.tree_commit([[], []], 65))
    lay.set_len(61)                                    # three rows of room
    with pytest.raises(B.EigenAttnError) as e:
        lay.decode_tree(q, k, v, m)
    assert e.value.status == B.EA_ERR_CAPACITY
    with pytest.raises(B.EigenAttnError) as e:
        lay.tree_commit([[0], [0]], 4)
    assert e.value.status == B.EA_ERR_CAPACITY
    lay.set_len(10)
    lay.set_alibi([0.5, 0.25])
    q2 = randn((2, 2, 4, 64), 5, BF16)
    refused(B.EA_ERR_UNSUPPORTED, lambda: lay.decode_tree(q2, k[:, :2], v[:, :2], m[:, :2].contiguous(), group=2))
    lay.set_alibi(None)
    lay.set_rope(10000.0)
    refused(B.EA_ERR_UNSUPPORTED, lambda: lay.decode_tree(q, k, v, m))
    lay.set_rope(0.0)
    lay.tree_detach()
    refused(B.EA_ERR_INVALID_ARG, lambda: lay.decode_tree(q, k, v, m))
    lay.poll_status()
