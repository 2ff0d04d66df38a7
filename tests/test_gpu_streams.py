"""Calls on another stream than the current one, while that is busy: nothing a call needs may run on the current stream."""
import pytest
import torch

from mq_helpers import BF16, FP32, Case, mask_tensor, randn, trees

pytestmark = pytest.mark.gpu

BUSY = 400_000_000             # cycles: some 0.2 s


@pytest.fixture(scope="module")
def B():
    from paper_2408_05646_b200 import build
    build.build_library()
    from paper_2408_05646_b200 import binding
    return binding


def two_strides(shape, seed, dtype):
    """k contiguous, v a slice of a wider tensor (a fused projection's, say)."""
    B, T, H, d = shape
    k = randn(shape, seed, dtype)
    wide = randn((B, T, 3 * H, d), seed + 1, dtype)
    return k, wide[:, :, 2 * H:]


def busy(stream):
    with torch.cuda.stream(stream):
        torch.cuda._sleep(BUSY)


@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("call", ["decode_tree", "decode_step"])
@pytest.mark.parametrize("delayed", ["current", "call"])
def test_keys_and_values_of_different_strides(B, dtype, call, delayed):
    """The copies that bring k and v into one layout run on the call's stream (delayed: what the current stream still has to
    do does not matter) and stay there (delayed: memory handed out on the current stream is not theirs)."""
    T = 8 if call == "decode_tree" else 1
    c = Case(B, dtype, 2, 4, 1, 64, [32] * 4, [32] * 4, [100, 60], 256, seed=3)
    ref = Case(B, dtype, 2, 4, 1, 64, [32] * 4, [32] * 4, [100, 60], 256, seed=3)
    q = randn((2, T, 4, 64), 5, dtype)
    k, v = two_strides((2, T, 4, 64), 7, dtype)
    mask = mask_tensor(trees(2, T, 3)[0])
    outs = [torch.zeros_like(q) for _ in range(2)]
    for x in (c, ref):
        x.lay.tree_attach(T)
    s = torch.cuda.Stream()

    def run(x, k, v, out, stream=None):
        if call == "decode_tree":
            return x.lay.decode_tree(q, k, v, mask, out=out, stream=stream)
        return x.lay.decode_step(q, k, v, out=out, stream=stream)
    run(ref, k.contiguous(), v.contiguous(), outs[0])
    torch.cuda.synchronize()
    busy(torch.cuda.current_stream() if delayed == "current" else s)
    run(c, k, v, outs[1], stream=s)
    trash = [torch.full_like(t, float("nan")) for t in (k, k, k, k)]       # where a freed copy of the current stream would be
    if delayed == "current":
        s.synchronize()
    else:
        torch.cuda.current_stream().synchronize()
        s.synchronize()
    got = [outs[1].clone()] + [c.lay.cache_rows(h, w).clone() for h in range(4) for w in "kv"]
    want = [outs[0]] + [ref.lay.cache_rows(h, w) for h in range(4) for w in "kv"]
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    del trash
