"""What the cache holds behind a sequence's end (rejected drafted tokens, a rewound sequence) has no weight in any result,
even where it is an infinity or NaN: a product of such a row with a zero weight would not be zero."""
import pytest
import torch

from mq_helpers import BF16, FP32, bases, mask_tensor, randn, trees

pytestmark = pytest.mark.gpu

BAD = [float("nan"), float("-inf")]


@pytest.fixture(scope="module")
def B():
    from paper_2408_05646_b200 import build
    build.build_library()
    from paper_2408_05646_b200 import binding
    return binding


def layer(B, dtype, batch, H, d, r, n_max, n, **more):
    U_k, U_v = bases(H, d, r, r, 5)
    lay = B.EigenAttnLayer(batch, H, d, n_max, dtype, U_k, U_v, **more)
    if n:
        lay.append_kv(randn((batch, n, H, d), 1, dtype), randn((batch, n, H, d), 2, dtype))
    return lay


def same_with_bad_rows(lay, lens, call):
    """call() from the state of `lens` rows, with zeros and then with infinities or NaN behind every sequence's end."""
    def state(fill):
        for h in range(lay.H):
            for which in "kv":
                rows = lay.cache_rows(h, which)
                for b, n in enumerate(lens):
                    rows[b, n:] = fill
        if len(set(lens)) > 1:
            lay.set_lens(lens)
        else:
            lay.set_len(lens[0])
        out = call()
        lay.poll_status()
        return out.clone()
    want = state(0.0)
    assert torch.isfinite(want).all()
    for bad in BAD:
        assert torch.equal(state(bad), want), bad


@pytest.mark.parametrize("impl", [0, 1, 3])            # warp-specialised tcgen05, CUDA cores, single-tile tcgen05
@pytest.mark.parametrize("lens,T", [([0], 1), ([5, 5], 3), ([130, 130], 63), ([7, 7], 57), ([64, 64], 64), ([130, 70], 131),
                                    ([3, 3], 255), ([20, 20], 257), ([100, 31], 300), ([61, 61], 259), ([0, 0], 512)])
@pytest.mark.parametrize("r,alibi", [(80, False), (128, False), (64, True)])
def test_prompt(B, impl, lens, T, r, alibi):
    batch, H, d = len(lens), 2, 128
    lay = layer(B, BF16, batch, H, d, [r, 48], 1024, max(lens), max_prefill_tokens=512)
    lay.set_option(B.EA_OPT_PREFILL_IMPL, impl)
    if alibi:
        lay.set_alibi([0.25, 0.01])
    q, k, v = (randn((batch, T, H, d), 11 + i, BF16) for i in range(3))
    same_with_bad_rows(lay, lens, lambda: lay.prefill(q, k, v))


@pytest.mark.parametrize("scratch", [0, 1])            # CUDA cores, tensor cores
@pytest.mark.parametrize("lens,T", [([0, 0], 5), ([130, 130], 70), ([17, 17], 300)])
def test_prompt_with_a_rotary_embedding(B, scratch, lens, T):
    lay = layer(B, BF16, 2, 2, 128, [80, 64], 1024, max(lens), max_prefill_tokens=512, rope_prompt_scratch=bool(scratch))
    lay.set_rope(10000.0)
    q, k, v = (randn((2, T, 2, 128), 21 + i, BF16) for i in range(3))
    same_with_bad_rows(lay, lens, lambda: lay.prefill(q, k, v))


@pytest.mark.parametrize("impl", [0, 1])               # warp-level products, tcgen05
@pytest.mark.parametrize("r", [[80, 80], [64, 48], [40, 128]])
@pytest.mark.parametrize("lens", [[1, 1], [129, 640], [300, 5], [1000, 1000]])
@pytest.mark.parametrize("rope", [False, True])
def test_grouped_decode(B, impl, r, lens, rope):
    lay = layer(B, BF16, 2, 2, 128, r, 1024, max(lens))
    lay.set_option(B.EA_OPT_GQA_IMPL, impl)
    if rope:
        lay.set_rope(10000.0)
    q = randn((2, 1, 8, 128), 31, BF16)
    same_with_bad_rows(lay, lens, lambda: lay.decode_gqa(q, 4))


@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("lens", [[1, 1], [129, 640], [300, 5], [1000, 1000]])
@pytest.mark.parametrize("rope", [False, True])
def test_decode_and_step(B, dtype, lens, rope):
    if rope and dtype == FP32:
        pytest.skip("rotary embedding: 16-bit layers")
    lay = layer(B, dtype, 2, 2, 64, [48, 33], 1024, max(lens))
    if rope:
        lay.set_rope(10000.0)
    q, k, v = (randn((2, 1, 2, 64), 41 + i, dtype) for i in range(3))
    same_with_bad_rows(lay, lens, lambda: lay.decode(q))
    same_with_bad_rows(lay, lens, lambda: lay.decode_step(q, k, v))


@pytest.mark.parametrize("lens", [[129, 640], [1000, 1000]])
@pytest.mark.parametrize("group", [16, 32])
def test_quantised_decode(B, lens, group):
    lay = layer(B, BF16, 2, 2, 128, [80, 64], 1024, max(lens))
    q = randn((2, 1, 2, 128), 51, BF16)

    def call():
        lay.quant_attach(4, group)
        lay.quant_sync()
        out = lay.decode_quant(q)
        lay.quant_detach()
        return out
    same_with_bad_rows(lay, lens, call)


@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("lens", [[129, 640], [300, 5], [1000, 1000]])
@pytest.mark.parametrize("r", [[80, 64], [128, 112]])
def test_blocks_and_trees(B, dtype, lens, r):
    lay = layer(B, dtype, 2, 2, 128, r, 1024, max(lens))
    q, qt, k, v = (randn((2, T, 2 * g, 128), 61 + T, dtype) for T, g in ((1, 2), (9, 2), (9, 1), (9, 1)))
    mask = mask_tensor(trees(2, 9, 3)[0])

    def sparse():
        lay.sparse_attach(32)
        lay.sparse_sync()
        return lay.decode_sparse(q, 5, group=2)
    same_with_bad_rows(lay, lens, sparse)
    lay.tree_attach(9, 2)
    same_with_bad_rows(lay, lens, lambda: lay.decode_tree(qt, k, v, mask, group=2))
    same_with_bad_rows(lay, lens, lambda: lay.decode_tree(qt[:, :, :2], k, v, mask))


@pytest.mark.parametrize("next_call", ["prefill", "decode_gqa", "decode_step", "decode_tree"])
def test_a_rejected_draft_leaves_no_trace(B, next_call):
    """Drafted tokens with infinities and NaN in their rows, rejected: what comes next is what comes after finite ones."""
    T, H, d = 40, 2, 128

    def run(bad):
        lay = layer(B, BF16, 2, H, d, [80, 64], 512, 150, max_prefill_tokens=128)
        lay.set_option(B.EA_OPT_GQA_IMPL, 1)
        lay.tree_attach(T)
        q, k, v = (randn((2, T, H, d), 71 + i, BF16) for i in range(3))
        k, v = k.clone(), v.clone()
        if bad is not None:
            k[:, 3:], v[:, 3:] = bad, bad
        masks = [[(2 << t) - 1 for t in range(T)]] * 2                # a chain
        lay.decode_tree(q, k, v, mask_tensor(masks))
        lay.tree_commit([[0, 1, 2], [0, 1]], T)
        x = [randn((2, 5, H, d), 81 + i, BF16) for i in range(3)]
        if next_call == "prefill":
            return lay.prefill(*x)
        if next_call == "decode_gqa":
            return lay.decode_gqa(randn((2, 1, 4 * H, d), 91, BF16), 4)
        if next_call == "decode_step":
            return lay.decode_step(*[t[:, :1] for t in x])
        return lay.decode_tree(*x, mask_tensor(trees(2, 5, 1)[0]))
    want = run(None)
    assert torch.isfinite(want).all()
    for bad in BAD:
        assert torch.equal(run(bad), want)
