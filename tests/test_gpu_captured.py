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
