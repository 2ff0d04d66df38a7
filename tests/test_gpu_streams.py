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


def test_what_a_call_allocates_belongs_to_its_stream(B, monkeypatch):
    """Every result (and buffer) that a call on another stream creates comes from that stream's memory: from the current
    stream's it could still be in use there."""
    guarded, seen = B.device_alloc, []

    def alloc(nbytes, device):
        seen.append(torch.cuda.current_stream())
        return guarded(nbytes, device)
    c = Case(B, BF16, 2, 2, 1, 64, [32, 48], [48, 32], [300, 300], 512, seed=9)
    pre = B.EigenAttnLayer(2, 2, 64, 512, BF16, c.U_k, c.U_v, max_prefill_tokens=64)
    lay = c.lay
    lay.tree_attach(6, 2)
    s = torch.cuda.Stream()
    q1, q2, qt = randn((2, 1, 2, 64), 1, BF16), randn((2, 1, 4, 64), 2, BF16), randn((2, 6, 4, 64), 3, BF16)
    k, v = randn((2, 6, 2, 64), 4, BF16), randn((2, 6, 2, 64), 5, BF16)
    mask = mask_tensor(trees(2, 6, 1)[0])
    torch.cuda.synchronize()
    monkeypatch.setattr(B, "device_alloc", alloc)
    calls = [
        (1, lambda: lay.decode(q1, stream=s)), (1, lambda: lay.decode(q1, out_lowrank=True, stream=s)),
        (1, lambda: lay.decode_static(q1, stream=s)), (1, lambda: lay.decode_step(q1, k[:, :1], v[:, :1], stream=s)),
        (1, lambda: lay.decode_step(q1, k[:, :1], v[:, :1], out_lowrank=True, stream=s)),
        (1, lambda: lay.decode_gqa(q2, 2, stream=s)),
        (1, lambda: pre.prefill(k, k, v, stream=s)), (1, lambda: pre.prefill(k, k, v, out_lowrank=True, stream=s)),
        (1, lambda: lay.decode_tree(qt, k, v, mask, group=2, stream=s)),
        (1, lambda: lay.decode_tree(qt, k, v, mask, group=2, out_lowrank=True, stream=s)),
        (1, lambda: lay.sparse_attach(32, stream=s)), (0, lambda: lay.sparse_sync(stream=s)),
        (2, lambda: lay.decode_sparse(q2, 3, group=2, return_index=True, stream=s)),
        (1, lambda: lay.decode_sparse(q2, 3, group=2, out_lowrank=True, stream=s)),
        (1, lambda: lay.quant_attach(4, 32, stream=s)), (0, lambda: lay.quant_sync(stream=s)),
        (1, lambda: lay.decode_quant(q1, stream=s)),
    ]
    current = torch.cuda.current_stream()
    for i, (count, call) in enumerate(calls):
        seen.clear()
        keep = call()
        assert len(seen) == count and all(x == s for x in seen), i
        assert torch.cuda.current_stream() == current
        torch.cuda.synchronize()
        del keep
    seen.clear()
    lay.decode(q1)
    assert seen == [current]
    torch.cuda.synchronize()
