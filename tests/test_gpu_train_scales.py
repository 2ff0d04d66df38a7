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


def within(got, want, names, dtype, part, floor={}):
    """Half a step of the type (below the smallest normal number: half of its last bit), `part` of the terms' sizes, and an
    absolute `floor` where one is given."""
    half, least = torch.finfo(dtype).eps / 2, torch.finfo(dtype).tiny * torch.finfo(dtype).eps / 2
    for name in names:
        assert np.isfinite(got[name]).all(), name
        over = np.abs(got[name] - want[name]) - half * np.abs(want[name]) - least - part * want[name + "_size"] - floor.get(name, 0)
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


@pytest.mark.parametrize("q_e,k_e,v_e,g_e", [(0, 0, 0, -110), (-24, -24, -8, -90), (40, -40, -64, -64), (-40, 40, -64, -64), (30, -30, 20, 60)])
def test_results_near_the_ends_of_the_range(q_e, k_e, v_e, g_e):
    """Tensors of very small or large numbers: the powers of two of three tiles add up to more than one factor can hold.  Least
    products that count: delta = do' o' of 2^-128 in the third and fourth case, kept to 2^-149 or 2^-21 of it."""
    T, r = 140, [32, 24]
    gen = torch.Generator().manual_seed(6)
    x = [rows(gen, 1, T, r, 1, BF, s * 2.0 ** e, 0.0) for s, e in zip((1.5, 1.0, 1.0, 1.0), (q_e, k_e, v_e, g_e))]
    got, want = step(*x, r, 64)
    within(got, want, ["out", "dq", "dk", "dv"], BF, 2.0 ** -11)


def test_large_results_of_which_the_largest_numbers_are_no_part():
    """A column of v' (2^42) that do' (2^66) does not ask for sets the exponents; dk' is of the others' (2^26), times q' (2^32).
    dS is then small in fp16: 2^24 2^(-e-e') becomes 2^15 there (e, e' the smallest exponents of do' and v'; 2^-e <= 2^-7
    max|do'|, 2^-e' <= 2^-7 max|v'|), so that the smallest half step, 2^-25, is 2^-30 max|do'| max|v'| of dS, and with the tile's deviation, at
    most a factor of two more, dk' is off by up to 2^-29 max|do'| max|v'| max|q'| scale for every query, dq' by the same with k' for
    every key (scale 1 / 8).  Here that is 2^121.6 in the sum of all 140; the largest dk' is 2^125.5, and a power of two left out of the
    results takes nearly all of it away."""
    T, r = 140, [32, 24]
    gen = torch.Generator().manual_seed(7)
    q, k, v, g = (rows(gen, 1, T, r, 1, BF, s, 0.0) for s in (1.5 * 2.0 ** 32, 2.0 ** -32, 2.0 ** 26, 2.0 ** 66))
    for first in (0, 32):
        v[:, :, first] *= 2.0 ** 16
        g[:, :, first] = 0
    got, want = step(q, k, v, g, r, 64)
    assert np.abs(want["dk"]).max() > 2.0 ** 118
    mq, mk, mv, mg = (x.abs().max().item() for x in (q, k, v, g))
    floor = {"dk": T * 2.0 ** -29 * mg * mv * mq / 8, "dq": T * 2.0 ** -29 * mg * mv * mk / 8}
    within(got, want, ["out", "dq", "dk", "dv"], BF, 2.0 ** -11, floor)


@pytest.mark.parametrize("largest", [1.0, 1.9921875, -1.5])
@pytest.mark.parametrize("side", [1.0, -1.0])
def test_numbers_far_below_the_largest_of_their_block(largest, side):
    """One token, whose o' is its v' and whose dv' is its do': what an operand's conversion leaves is seen as it is.  From 2^-22 of the
    largest on a number is kept; below, it is off by up to 2^-32 of the largest (half of fp16's last step, 2^-25, where the largest
    is at least 2^7), and one of 2^-32 can be off by just that."""
    r = 64
    x = torch.zeros(1, 1, 2 * r, dtype=BF)
    x[0, 0, 0] = x[0, 0, r] = largest
    e = torch.arange(1, r)
    x[0, 0, 1:r] = (side * 1.6953125 * 2.0 ** -(e.double() * 0.75).floor()).to(BF)          # eight bits each
    x[0, 0, r + 1:] = (side * 2.0 ** -e.double()).to(BF)
    one = torch.ones(1, 1, 2 * r, dtype=BF)
    lay = layer(1, [r, r], [r, r], r, BF)
    lay.train_attach(1)
    out = lay.train_forward(one.cuda(), one.cuda(), x.cuda())
    _, _, dv = lay.train_backward(x.cuda())
    top = abs(largest)
    for got in (out, dv):
        err = (got.cpu().double() - x.double()).abs()
        assert (err[x.double().abs() >= top * 2.0 ** -22] == 0).all()
        assert err.max() <= top * 2.0 ** -32
    if largest == 1.0:                                       # the bound is reached: 2^-32 lies between 0 and fp16's 2^-24 / 2^7
        assert (out.cpu().double() - x.double())[0, 0, r + 32].abs() == 2.0 ** -32
