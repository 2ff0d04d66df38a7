"""Training calls of 16-bit layers whose tiles carry powers of two far apart, or whose results lie at the ends of the range,
against the fp64 definitions."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
from oracle import training as oracle
from test_gpu_train import BF, F32, layer, rows

pytestmark = pytest.mark.gpu


def step(q, k, v, g, r, d_head, buckets=None, table=None):
    """Outputs of a step over packed rows, and the definition's: {"out", "dq", "dk", "dv"} (and "table" for buckets)."""
    lay = layer(q.shape[0], r, r, d_head, q.dtype)
    bias = None
    if buckets is not None:
        lay.bias_attach(*buckets)
        lay.set_bias(table.cuda())
        bias = oracle.bias_by_distance(table.double().numpy(), buckets[1], q.shape[1])
    lay.train_attach(q.shape[1])
    out = lay.train_forward(q.cuda(), k.cuda(), v.cuda())
    res = lay.train_backward(g.cuda(), bias_grad=buckets is not None)
    lay.poll_status()
    got = {name: x.double().cpu().numpy() for name, x in zip(("out", "dq", "dk", "dv", "table"), (out,) + tuple(res))}
    want = oracle.train(*[x.double().numpy() for x in (q, k, v, g)], r, r, d_head, 1, None, bias)
    if buckets is not None:
        for name in ("by_distance", "by_distance_size"):
            by = np.zeros((len(r), buckets[0]))
            for d in range(q.shape[1]):
                by[:, oracle.bucket_of(d, *buckets)] += want[name][:, d]
            want["table" + name[len("by_distance"):]] = by
    return got, want


def within(got, want, names, dtype, part):
    """Half a step of the type (below the smallest normal number: half of its last bit), and `part` of the terms' sizes."""
    half, least = torch.finfo(dtype).eps / 2, torch.finfo(dtype).tiny * torch.finfo(dtype).eps / 2
    for name in names:
        assert np.isfinite(got[name]).all(), name
        over = np.abs(got[name] - want[name]) - half * np.abs(want[name]) - least - part * want[name + "_size"]
        worst = np.argmax(over)
        assert over.max() <= 0, (name, got[name].flat[worst], want[name].flat[worst], want[name + "_size"].flat[worst])


@pytest.mark.parametrize("grad_scale", [1.0, 2.0 ** 16, 2.0 ** 30])
@pytest.mark.parametrize("key_scale", [0.0, 2.0 ** -100])
def test_the_table_gradient_counts_blocks_of_tiny_keys(key_scale, grad_scale):
    """128 keys that are zero (padding in front of a text, say) still take part in the softmax: their dS belongs to the buckets.
    Tolerance: dS goes into these sums in 32 bits; its delta has the o' of P's 11 significant bits (2^-12 of the terms)."""
    T, r, buckets = 400, [32, 24], (16, 64)
    gen = torch.Generator().manual_seed(5)
    q, k, v, g = (rows(gen, 2, T, r, 1, BF, s, 0.0) for s in (1.5, 1.0, 1.0, grad_scale))
    k[:, 128:256] *= key_scale
    table = torch.randn(2, buckets[0], generator=gen).to(BF)
    got, want = step(q, k, v, g, r, 64, buckets, table)
    within(got, want, ["table"], BF, 2.0 ** -12)
    within(got, want, ["out", "dq", "dk", "dv"], BF, 2.0 ** -11)
