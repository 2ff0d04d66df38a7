"""What a stream capture may hold of tree attention and of decode over selected blocks, and what replays then see."""
import numpy as np
import pytest
import torch

from mq_helpers import BF16, FP32, Case, check, mask_tensor, randn, sparse_expected, tree_expected, trees

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    from paper_2408_05646_b200 import build
    build.build_library()
    from paper_2408_05646_b200 import binding
    return binding


def test_bounds_are_not_taken_for_there_during_a_capture(B):
    c = Case(B, BF16, 2, 2, 1, 128, [80, 48], [80, 64], [900, 900], 1024, seed=11)
    lay = c.lay
    lay.sparse_attach(32)
    q = randn((2, 1, 2, 128), 13, BF16, 2.0)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        with pytest.raises(B.EigenAttnError) as e:
            lay.sparse_sync()
        assert e.value.status == B.EA_ERR_UNSUPPORTED
        q.mul_(1.0)                                    # (a graph of its own is no empty one)
    assert lay.sparse_lens() == [0, 0]
    with pytest.raises(B.EigenAttnError) as e:         # no bounds yet
        lay.decode_sparse(q, 5)
    assert e.value.status == B.EA_ERR_INVALID_ARG
    lay.sparse_sync()
    want, slack, idx = sparse_expected(c, q, 32, 5, 1, 1)
    out = torch.zeros_like(q)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        lay.sparse_sync()                              # nothing to do: nothing is taken for done
        lay.decode_sparse(q, 5, out=out)
    g.replay()
    torch.cuda.synchronize()
    check(out, want, slack, BF16, "replayed")


def test_a_refused_attach_leaves_the_buffer_that_was_there(B, monkeypatch):
    """sparse_attach waits for the stream, which a capture does not allow: it refuses before it touches the capture, and the
    layer keeps the buffer that the library still uses."""
    c = Case(B, BF16, 1, 2, 1, 128, [80, 48], [80, 64], [900], 1024, seed=17)
    lay = c.lay
    buf = lay.sparse_attach(32)
    lay.sparse_sync()
    q = randn((1, 1, 2, 128), 19, BF16, 2.0)
    want = lay.decode_sparse(q, 5)
    spare = torch.empty(2 * buf.numel(), dtype=torch.uint8, device="cuda")
    monkeypatch.setattr(B, "device_alloc", lambda n, device: spare[:n])    # (the guarded one fills what it hands out)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        with pytest.raises(B.EigenAttnError) as e:
            lay.sparse_attach(64)
        assert e.value.status == B.EA_ERR_UNSUPPORTED
        q.mul_(1.0)
    assert lay.sparse_buf is buf and lay.sparse_block == 32 and lay.sparse_lens() == [896]
    assert torch.equal(lay.decode_sparse(q, 5), want)


@pytest.mark.parametrize("dtype,T,slopes", [(BF16, 4, None), (BF16, 24, None), (BF16, 20, [0.25, 0.0]), (FP32, 5, None)])
@pytest.mark.parametrize("preprojected", [False, True])
def test_a_captured_tree_keeps_its_lengths(B, dtype, T, slopes, preprojected):
    """Lengths that differ, a captured call, other lengths: a replay returns what the call returned with its own."""
    lens = [700, 130, 405]
    c = Case(B, dtype, 3, 2, 1, 64, [32, 24], [24, 32], lens, 1024, seed=23, slopes=slopes)
    lay = c.lay
    lay.tree_attach(T)
    q = randn((3, T, 2, 64), 29, dtype)
    k, v = ((randn((3, T, w[-1]), 31 + i, dtype) for i, w in enumerate((lay.offs_k, lay.offs_v))) if preprojected else
            (randn((3, T, 2, 64), 31 + i, dtype) for i in range(2)))
    masks, _ = trees(3, T, 7)
    m = mask_tensor(masks)
    want = lay.decode_tree(q, k, v, m, kv_preprojected=preprojected)
    check(want, *tree_expected(c, q, masks, T), dtype, "tree")
    out = torch.zeros_like(want)
    lay.decode_tree(q, k, v, m, kv_preprojected=preprojected, out=out)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        lay.decode_tree(q, k, v, m, kv_preprojected=preprojected, out=out)
    before = [lay.cache_rows(h, w).clone() for h in range(2) for w in "kv"]
    for now in (lens, [10, 700, 20], [1, 2, 699], [700, 700, 699], [0, 0, 1]):
        lay.set_lens(now)
        out.zero_()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want), now
        assert all(torch.equal(a, b) for a, b in zip(before, [lay.cache_rows(h, w) for h in range(2) for w in "kv"]))
    lay.set_len(5)
    g.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, want)
    lay.poll_status()


@pytest.mark.parametrize("dtype,group", [(BF16, 1), (BF16, 4), (FP32, 1)])
def test_a_captured_choice_of_blocks_keeps_its_lengths(B, dtype, group):
    lens = [700, 130, 405]
    c = Case(B, dtype, 3, 2, group, 64, [32, 24], [24, 32], lens, 1024, seed=37)
    lay = c.lay
    lay.sparse_attach(16)
    lay.sparse_sync()
    q = randn((3, 1, 2 * group, 64), 41, dtype, 2.0)
    want, slack, idx = sparse_expected(c, q, 16, 9, 1, 1)
    out = torch.zeros_like(q)
    first = lay.decode_sparse(q, 9, group=group, out=out).clone()
    check(first, want, slack, dtype, "sparse")
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        lay.decode_sparse(q, 9, group=group, out=out)
    for now in (lens, [10, 700, 20], [1, 2, 699], [700, 700, 699]):
        lay.set_lens(now)
        out.zero_()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, first), now
    lay.poll_status()


def test_lengths_of_a_large_captured_batch(B):
    """More sequences than one launch's parameters carry."""
    batch, T = 1000, 3
    lens = [(7 * i) % 50 for i in range(batch)]
    c = Case(B, BF16, batch, 1, 1, 16, [8], [16], lens, 64, seed=43)
    lay = c.lay
    lay.tree_attach(T)
    q, k, v = (randn((batch, T, 1, 16), 47 + i, BF16) for i in range(3))
    m = mask_tensor(trees(batch, T, 3)[0])
    want = lay.decode_tree(q, k, v, m)
    out = torch.zeros_like(want)
    lay.decode_tree(q, k, v, m, out=out)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        lay.decode_tree(q, k, v, m, out=out)
    lay.set_lens([49 - n for n in lens])
    out.zero_()
    g.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, want)
