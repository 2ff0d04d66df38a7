"""The learned bias of relative positions where the cache is attended: decode, decode_step, decode_static, prefill."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
from oracle import training as oracle
import helpers

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32
BUCKETS = (32, 128)


def make(B, r_k, r_v, d, dtype, n_max, max_prefill=0, buckets=BUCKETS, seed=0):
    from paper_2408_05646_b200 import binding
    rng = np.random.default_rng(seed)
    U_k = [np.linalg.qr(rng.standard_normal((d, d)))[0][:, :r].astype(np.float32) for r in r_k]
    U_v = [np.linalg.qr(rng.standard_normal((d, d)))[0][:, :r].astype(np.float32) for r in r_v]
    lay = binding.EigenAttnLayer(B, len(r_k), d, n_max, dtype, U_k, U_v, max_prefill_tokens=max_prefill)
    table = torch.from_numpy(rng.standard_normal((len(r_k), buckets[0]))).to(dtype)
    lay.bias_attach(*buckets)
    lay.set_bias(table.cuda())
    bias = oracle.bias_by_distance(table.double().numpy(), buckets[1], n_max)
    return lay, U_k, U_v, bias, rng


def draw(rng, dtype, *shape, scale=1.0):
    return torch.from_numpy(rng.standard_normal(shape) * scale).to(dtype)


def attend(q, K, V, U_k, U_v, d, bias, last):
    """One query at position `last` over rows 0 .. last."""
    s = K[:last + 1] @ (q @ U_k.astype(np.float64)) / np.sqrt(d) + bias[last::-1]
    w = np.exp(s - s.max())
    return (w / w.sum()) @ V[:last + 1] @ U_v.astype(np.float64).T


def project(x, U, dtype):
    """Rows as the cache keeps them."""
    return torch.from_numpy(x.double().numpy() @ U.astype(np.float64)).to(dtype).double().numpy()


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("n,lens,page", [(1, None, 0), (130, None, 0), (1000, [1000, 17, 512], 0), (700, [700, 1, 399], 128)])
def test_decode(dtype, n, lens, page):
    B, d, r_k, r_v = 3, 64, [32, 40], [24, 64]
    lay, U_k, U_v, bias, rng = make(B, r_k, r_v, d, dtype, 1024, seed=n)
    if page:
        order = rng.permutation(B * 1024 // page).reshape(B, -1).tolist()
        lay.set_page_table(order, page)
    k, v = draw(rng, dtype, B, n, 2, d), draw(rng, dtype, B, n, 2, d)
    lay.append_kv(k.cuda(), v.cuda())
    if lens:
        lay.set_lens(lens)
    q = draw(rng, dtype, B, 1, 2, d, scale=2.0)
    k1, v1 = draw(rng, dtype, B, 1, 2, d), draw(rng, dtype, B, 1, 2, d)
    outs = [lay.decode(q.cuda()), lay.decode_static(q.cuda())]
    step = lay.decode_step(q.cuda(), k1.cuda(), v1.cuda())
    want, want_step = np.zeros((B, 1, 2, d)), np.zeros((B, 1, 2, d))
    for b in range(B):
        m = lens[b] if lens else n
        for h in range(2):
            K, V = (project(torch.cat([x[b, :m, h], y[b, :, h]]), U[h], dtype) for x, y, U in ((k, k1, U_k), (v, v1, U_v)))
            qh = q[b, 0, h].double().numpy()
            want[b, 0, h] = attend(qh, K, V, U_k[h], U_v[h], d, bias[h], m - 1)
            want_step[b, 0, h] = attend(qh, K, V, U_k[h], U_v[h], d, bias[h], m)
    for got in outs:
        helpers.assert_close(got, want, dtype, "decode")
    helpers.assert_close(step, want_step, dtype, "decode_step")
    lay.poll_status()


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("impl", [0, 1, 3])
@pytest.mark.parametrize("T,first", [(1, 0), (200, 0), (300, 77)])
def test_prefill(dtype, impl, T, first):
    B, d, r_k, r_v = 2, 64, [32, 40], [24, 64]
    lay, U_k, U_v, bias, rng = make(B, r_k, r_v, d, dtype, 512, max_prefill=T, seed=T)
    from paper_2408_05646_b200 import binding
    lay.set_option(binding.EA_OPT_PREFILL_IMPL, impl)
    k, v = draw(rng, dtype, B, first + T, 2, d), draw(rng, dtype, B, first + T, 2, d)
    if first:
        lay.append_kv(k[:, :first].contiguous().cuda(), v[:, :first].contiguous().cuda())
    q = draw(rng, dtype, B, T, 2, d)
    got = lay.prefill(q.cuda(), k[:, first:].contiguous().cuda(), v[:, first:].contiguous().cuda())
    want = np.zeros((B, T, 2, d))
    for b in range(B):
        for h in range(2):
            K, V = project(k[b, :, h], U_k[h], dtype), project(v[b, :, h], U_v[h], dtype)
            for t in range(T):
                want[b, t, h] = attend(q[b, t, h].double().numpy(), K, V, U_k[h], U_v[h], d, bias[h], first + t)
    helpers.assert_close(got, want, dtype, "prefill")


@pytest.mark.parametrize("buckets", [(32, 128), (2, 2), (64, 1024)])
@pytest.mark.parametrize("impl", [0, 3])
@pytest.mark.parametrize("T,lens", [(640, [0, 64]), (530, [130, 77])])
def test_long_prompts_behind_unequal_lengths(T, lens, impl, buckets):
    """Tiles near the diagonal, and tiles whose distances all share the last bucket."""
    from paper_2408_05646_b200 import binding
    d, r_k, r_v = 64, [32, 64], [40, 24]
    lay, U_k, U_v, bias, rng = make(2, r_k, r_v, d, BF, 768, max_prefill=T, buckets=buckets, seed=T)
    lay.set_option(binding.EA_OPT_PREFILL_IMPL, impl)
    k0, v0 = draw(rng, BF, 2, 130, 2, d), draw(rng, BF, 2, 130, 2, d)
    lay.append_kv(k0.cuda(), v0.cuda())
    lay.set_lens(lens)
    q, k, v = (draw(rng, BF, 2, T, 2, d) for _ in range(3))
    got = lay.prefill(q.cuda(), k.cuda(), v.cuda())
    want = np.zeros((2, T, 2, d))
    for b, n in enumerate(lens):
        for h in range(2):
            K = np.concatenate([project(k0[b, :n, h], U_k[h], BF), project(k[b, :, h], U_k[h], BF)])
            V = np.concatenate([project(v0[b, :n, h], U_v[h], BF), project(v[b, :, h], U_v[h], BF)])
            for t in range(T):
                want[b, t, h] = attend(q[b, t, h].double().numpy(), K, V, U_k[h], U_v[h], d, bias[h], n + t)
    helpers.assert_close(got, want, BF, "prefill")
    lay.poll_status()


@pytest.mark.parametrize("dtype", [BF, F32])
def test_a_prompt_in_pages(dtype):
    """A page table changes addresses and nothing else."""
    from paper_2408_05646_b200 import binding
    d, r_k, r_v, T = 64, [32, 40], [24, 64], 300
    outs = []
    for paged in (False, True):
        lay, _, _, _, rng = make(2, r_k, r_v, d, dtype, 512, max_prefill=T)
        lay.set_option(binding.EA_OPT_PREFILL_IMPL, 1)
        if paged:
            lay.set_page_table([[5, 0, 3, 6], [1, 7, 2, 4]], 128)
        q, k, v = (draw(rng, dtype, 2, T, 2, d).cuda() for _ in range(3))
        outs.append((lay.prefill(q, k, v), lay.decode(q[:, -1:].contiguous())))
    assert torch.equal(outs[0][0], outs[1][0])
    helpers.assert_close(outs[1][1], outs[0][1].double().cpu().numpy(), dtype, "decode")


def test_a_bias_can_be_changed_and_taken_away():
    B, d, r = 1, 64, [32]
    lay, U_k, U_v, bias, rng = make(B, r, r, d, F32, 256)
    k, v, q = draw(rng, F32, B, 200, 1, d).cuda(), draw(rng, F32, B, 200, 1, d).cuda(), draw(rng, F32, B, 1, 1, d).cuda()
    lay.append_kv(k, v)
    first = lay.decode(q)
    table = torch.zeros(1, 32, device="cuda")
    lay.set_bias(table)
    none = lay.decode(q)
    lay.bias_detach()
    assert not torch.equal(first, none)
    assert torch.allclose(none, lay.decode(q), rtol=0, atol=1e-6)
    lay.set_alibi([0.5])
    assert not torch.allclose(none, lay.decode(q), atol=1e-3)
