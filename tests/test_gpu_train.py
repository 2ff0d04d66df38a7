"""Training calls (attention over rank-space rows, its backward pass, the learned bias) against the fp64 definitions."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
from oracle import training as oracle

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32


def layer(B, r_k, r_v, d_head, dtype, n_max=8):
    from paper_2408_05646_b200 import binding
    eye = np.eye(d_head, dtype=np.float32)
    return binding.EigenAttnLayer(B, len(r_k), d_head, n_max, dtype, [eye[:, :r] for r in r_k], [eye[:, :r] for r in r_v])


def rows(gen, B, T, r, group, dtype, scale, junk):
    """Packed rows; padding columns hold `junk`."""
    cols, width = oracle.packed_columns(r, group)
    x = torch.full((B, T, width), junk, dtype=dtype)
    for c in cols:
        x[:, :, torch.as_tensor(c)] = (torch.randn(B, T, len(c), generator=gen) * scale).to(dtype)
    return x


def close(got, want, size, dtype, what):
    """Element by element: half a step of the type for the rounding, and the errors of P, dS and the products, relative to
    `size`, the sum of the absolute terms.  16-bit layers: P and dS enter the products with 11 significant bits (2^-12), and
    what is worked out in 32 bits in front of them adds less than that again.  fp32 layers, in units of 2^-24: a score is a
    32-bit sum of products, off by a few |S| (|S| reaches 1.5 sqrt(r / d_head) times 5, at most 7.5: three times that), a
    product do' v' by some sqrt(128), a sum over T terms in tiles by some sqrt(64) + sqrt(T / 64): 45 together.
    Root mean square: a rounding is 0.43 half steps, and the errors of many terms do not line up: half of that again in
    16-bit layers, and in fp32 layers sqrt(T) half steps and what a score's error brings (22)."""
    got = got.double().cpu().numpy()
    assert np.isfinite(got).all(), what
    half = torch.finfo(dtype).eps / 2
    err = np.abs(got - want)
    over = err - half * np.abs(want) - (2.0 ** -11 if dtype == BF else 45 * half) * size
    assert over.max() <= 0, (what, err.max(), over.max())
    rms, rms_size = np.sqrt(np.mean(want ** 2)), np.sqrt(np.mean(size ** 2))
    steps, tiny = (0.65, 2.0 ** -21) if dtype == BF else (2 * np.sqrt(max(16, want.shape[1])) + 22, 2.0 ** -22)
    # (tiny: where the terms cancel, as the first token's dS does exactly, 32-bit sums of them are left)
    assert np.sqrt(np.mean(err ** 2)) <= steps * half * rms + tiny * rms_size, (what, np.sqrt(np.mean(err ** 2)) / max(rms, 1e-300) / half)


def run_case(B, T, r_k, r_v, d_head, dtype, group=1, lens=None, alibi=None, buckets=None, seed=0, grad_scale=1.0, junk=3.0):
    gen = torch.Generator().manual_seed(seed)
    q = rows(gen, B, T, r_k, group, dtype, 1.5, junk)
    k, v = rows(gen, B, T, r_k, 1, dtype, 1.0, junk), rows(gen, B, T, r_v, 1, dtype, 1.0, junk)
    g = rows(gen, B, T, r_v, group, dtype, grad_scale, junk)
    lay = layer(B, r_k, r_v, d_head, dtype)
    bias = table = None
    if alibi is not None:
        lay.set_alibi(alibi)
        bias = -np.float64(np.float32(alibi))[:, None] * np.arange(T)
    if buckets is not None:
        table = torch.randn(len(r_k), buckets[0], generator=gen).to(dtype)
        lay.bias_attach(*buckets)
        lay.set_bias(table.cuda())
        bias = oracle.bias_by_distance(table.double().numpy(), buckets[1], T)
    lay.train_attach(T, group)
    dev_lens = None if lens is None else torch.tensor(lens, dtype=torch.int32, device="cuda")
    qd, kd, vd = q.cuda(), k.cuda(), v.cuda()
    if lens is not None:                        # what lies behind a sequence's end is not read
        for b, n in enumerate(lens):
            for x in (qd, kd, vd):
                x[b, max(0, n):] = float("nan")
    out = lay.train_forward(qd, kd, vd, lens=dev_lens, group=group)
    for x in (qd, kd, vd):
        x.fill_(float("nan"))                   # the layer has kept what it needs
    if lens is not None:
        dev_lens.fill_(0)
    gd = g.cuda()
    if lens is not None:
        for b, n in enumerate(lens):
            gd[b, max(0, n):] = float("nan")
    res = lay.train_backward(gd, bias_grad=buckets is not None)
    lay.poll_status()
    want = oracle.train(q.double().numpy(), k.double().numpy(), v.double().numpy(), g.double().numpy(), r_k, r_v, d_head, group,
                        lens, bias)
    for name, x in zip(("out", "dq", "dk", "dv"), (out,) + tuple(res[:3])):
        close(x, want[name], want[name + "_size"], dtype, name)
        outside = np.ones(x.shape[-1], bool)    # padding columns, and rows behind the end, are zero
        r, gr = {"out": (r_v, group), "dq": (r_k, group), "dk": (r_k, 1), "dv": (r_v, 1)}[name]
        for c in oracle.packed_columns(r, gr)[0]:
            outside[c] = False
        assert (x.float().cpu().numpy()[:, :, outside] == 0).all(), name
        if lens is not None:
            for b, n in enumerate(lens):
                assert (x[b, max(0, n):] == 0).all(), (name, b)
    if buckets is not None:
        by, size = np.zeros((len(r_k), buckets[0])), np.zeros((len(r_k), buckets[0]))
        for d in range(T):
            by[:, oracle.bucket_of(d, *buckets)] += want["by_distance"][:, d]
            size[:, oracle.bucket_of(d, *buckets)] += want["by_distance_size"][:, d]
        got = res[3].double().cpu().numpy()
        assert np.isfinite(got).all()
        half = torch.finfo(dtype).eps / 2
        # fp32 layers as above.  16-bit layers: dS goes into these sums in 32 bits, but its delta = do' o' has the o' of P's
        # 11 significant bits: off by up to 2^-12 of sum_j P_ij |do'_i| |v'_j|, which `size` contains
        part = 2.0 ** -12 if dtype == BF else 45 * half
        over = np.abs(got - by) - half * np.abs(by)
        worst = np.argmax(over - part * size)
        assert (over <= part * size).all(), [float(x.flat[worst]) for x in (got, by, size, over)]
    return lay


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("T", [1, 2, 63, 64, 65, 127, 128, 129, 300])
def test_lengths_round_tile_borders(dtype, T):
    run_case(2, T, [32, 32], [32, 32], 64, dtype, seed=T)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("r_k,r_v,d_head", [([8], [8], 8), ([1, 5], [3, 8], 16), ([80, 20], [80, 44], 128), ([128], [128], 128),
                                            ([128, 16], [24, 112], 128), ([96, 64, 48], [64, 96, 40], 96)])
def test_ranks(dtype, r_k, r_v, d_head):
    run_case(1, 200, r_k, r_v, d_head, dtype, seed=len(r_k))


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("group", [2, 3, 16])
def test_gradients_of_shared_heads(dtype, group):
    run_case(2, 150, [24, 32], [32, 24], 64, dtype, group=group, lens=[150, 77])


@pytest.mark.parametrize("dtype", [BF, F32])
def test_unequal_lengths_and_empty_sequences(dtype):
    run_case(6, 260, [40], [40], 64, dtype, lens=[260, 0, 1, 128, 129, 400])


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("T", [100, 400])
def test_alibi(dtype, T):
    run_case(2, T, [32, 48], [48, 32], 64, dtype, alibi=[0.25, 0.0078125], lens=[T, T // 3])


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("buckets", [(32, 128), (2, 2), (3, 7), (21, 64), (64, 1024), (256, 300)])
@pytest.mark.parametrize("T", [1, 50, 390])
def test_learned_bias_and_its_gradient(dtype, buckets, T):
    run_case(2, T, [32, 40], [40, 32], 64, dtype, buckets=buckets, lens=[T, max(0, T - 30)])


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("grad_scale", [2.0 ** -40, 2.0 ** 30])
def test_gradients_of_any_size(dtype, grad_scale):
    run_case(1, 140, [32], [32], 64, dtype, grad_scale=grad_scale)
