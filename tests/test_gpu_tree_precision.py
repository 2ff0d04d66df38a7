"""16-bit layers: Q' and P enter the products as two 16-bit parts.  Rows and queries are made so that one part alone, its
rounding error all on one side, would be far outside the bound; that is checked on the expected value itself."""
import math

import numpy as np
import pytest
import torch

from mq_helpers import BF16, Case, check, mask_tensor, np64, randn, sparse_expected, tree_expected, trees

pytestmark = pytest.mark.gpu

LOG2E = 1.4426950408889634
PATHS = [(1, 4, 0), (1, 12, 0), (1, 20, 1), (1, 20, 0), (1, 50, 0), (4, 32, 0)]      # group, T, EA_OPT_TREE_IMPL


@pytest.fixture(scope="module")
def B():
    from paper_2408_05646_b200 import build
    build.build_library()
    from paper_2408_05646_b200 import binding
    return binding


def bf16(x):
    return torch.as_tensor(np.asarray(x, np.float32)).to(BF16).double().numpy()


class Layer(Case):
    def __init__(self, B, group, d, U_k, U_v, K, V, n_max):
        self.dtype, self.batch, self.H, self.group, self.d = BF16, 1, 1, group, d
        self.rk, self.rv = [U_k.shape[1]], [U_v.shape[1]]
        self.lens, self.slopes, self.table = [len(K)], None, None
        self.U_k, self.U_v = [U_k.astype(np.float32)], [U_v.astype(np.float32)]
        self.lay = B.EigenAttnLayer(1, 1, d, n_max, BF16, self.U_k, self.U_v)
        for which, rows in (("k", K), ("v", V)):
            self.lay.cache_rows(0, which)[0, :len(K)] = torch.as_tensor(rows).to(BF16)
        self.lay.set_len(len(K))


def test_queries_keep_sixteen_bits(B):
    """Scores of some 60 from 32 channels each, whose query entries round down on even rows and up on odd ones: rounded to
    16 bits they would shift the two kinds of rows against each other by half a unit of score."""
    d, r, n, X = 128, 64, 1500, 16.0
    kind = np.arange(r) // 32
    worst = np.where(kind == 0, 1 + 2.0 ** -8 - 2.0 ** -12, 1 + 2.0 ** -7 + 2.0 ** -8 + 2.0 ** -12)    # next to a halfway point
    a = worst * math.sqrt(d) / (LOG2E * X)
    U = np.zeros((d, r))
    U[2 * np.arange(r), np.arange(r)], U[2 * np.arange(r) + 1, np.arange(r)] = a, np.sqrt(1 - a * a)
    K, V = np.zeros((n, r)), np.zeros((n, r))
    for j in range(n):
        K[j, kind == j % 2] = 2.625
        V[j] = bf16(np.where(j % 2, -1.0, 1.0) * (1 + np.arange(r) / 64.0))
    x = torch.zeros(d)
    x[0::2] = X
    for group, T, impl in PATHS:
        c = Layer(B, group, d, U, np.eye(d)[:, :r], K, V, 2048)
        c.lay.set_option(B.EA_OPT_TREE_IMPL, impl)
        c.lay.tree_attach(T, group)
        q = x.to(BF16).cuda().expand(1, T, group, d).contiguous()
        k, v = torch.zeros((1, T, 1, d), dtype=BF16, device="cuda"), torch.zeros((1, T, 1, d), dtype=BF16, device="cuda")
        masks = [[0] * T]
        out = c.lay.decode_tree(q, k, v, mask_tensor(masks), group=group)
        want, slack = tree_expected(c, q, masks, T)
        check(out, want, slack, BF16, f"tree {group, T, impl}")
    c = Layer(B, 1, d, U, np.eye(d)[:, :r], K, V, 2048)
    c.lay.sparse_attach(32)
    q = x.to(BF16).cuda().view(1, 1, 1, d)
    out = c.lay.decode_sparse(q, 64)
    check(out, *sparse_expected(c, q, 32, 64, 1, 1)[:2], BF16, "sparse")
    # one part alone: outside the bound
    qp = np64(q)[0, 0, 0] @ np.float64(c.U_k[0])
    s = K @ (bf16(qp * LOG2E / math.sqrt(d)) / LOG2E)
    w = np.exp(s - s.max())
    w /= w.sum()
    assert (np.abs(w @ V - want[0, 0, 0, :r]) > 2.0 ** -7 * np.abs(want[0, 0, 0, :r]) + 10 * slack[0, 0, 0, :r]).all()


def test_weights_keep_sixteen_bits(B):
    """Every sixteenth row has the highest score, all others one whose weight against it lies just above a halfway point
    between two 16-bit numbers: rounded to one, all of them would be too large by the same 2^-8.  An output's own rounding
    hides that, the mean over many outputs does not.  With z = <out - want, want> / <want, want> over N outputs: each rounds
    by at most 2^-8 of its value, to either side alike, so that their part of z has a standard deviation of at most 2^-8
    sqrt(3 / N) / sqrt(3) (values are normally distributed: the fourth moment is three times the squared second); six of
    those, and twice e_w for the arithmetic (mq_helpers)."""
    d, n = 128, 2000
    eye = np.eye(d)
    g = np.random.default_rng(3)
    top = np.full(d, 0.5)
    x = np.full(d, 4 * math.sqrt(d) / (0.5 * d))          # the highest score: 4
    x = bf16(x)
    target = 0.5 * (1 + 2.0 ** -8 + 2.0 ** -12)
    low, best = None, 1.0
    for _ in range(4000):                                 # 16-bit keys whose score hits the target closely from above
        k = top - 0.1734 * g.random(d)
        k = bf16(k)
        p = math.exp((k - top) @ x / math.sqrt(d))
        over = p / (0.5 * (1 + 2.0 ** -8)) - 1
        if 2.0 ** -14 < over < best:
            low, best = k, over
    assert low is not None and best < 2.0 ** -10
    kinds = np.arange(n) % 16 == 0
    K = np.where(kinds[:, None], top, low)
    for group, T, impl in PATHS:
        V = bf16(g.standard_normal((n, d)))
        c = Layer(B, group, d, eye, eye, K, V, 2304)
        c.lay.set_option(B.EA_OPT_TREE_IMPL, impl)
        c.lay.tree_attach(T, group)
        q = torch.as_tensor(x).to(BF16).cuda().expand(1, T, group, d).contiguous()
        zero = torch.zeros((1, T, 1, d), dtype=BF16, device="cuda")
        out = np64(c.lay.decode_tree(q, zero, zero, mask_tensor([[0] * T]), group=group))[0, 0, 0]
        s = K @ x / math.sqrt(d)
        w = np.exp(s - s.max())
        want = w @ V / w.sum()
        e_s = (2.0 ** -16 + (2 * d + 4) * 2.0 ** -23) * s.max()
        e_w = 2.2 * e_s + 2.0 ** -15 + (n + 64) * 2.0 ** -24
        outs, wants = [out], [want]
        for i in range(15):                               # other values, the same weights: 16 x 128 outputs
            V = bf16(g.standard_normal((n, d)))
            c.lay.cache_rows(0, "v")[0, :n] = torch.as_tensor(V).to(BF16)
            outs.append(np64(c.lay.decode_tree(q, zero, zero, mask_tensor([[0] * T]), group=group))[0, 0, 0])
            wants.append(w @ V / w.sum())
        got, want = np.concatenate(outs), np.concatenate(wants)
        bound = 6 * 2.0 ** -8 / math.sqrt(len(want)) + 2 * e_w
        z = (got - want) @ want / (want @ want)
        assert abs(z) <= bound, (group, T, impl, z, bound)
        # one part alone: the numerator's weights too large, their sum as it is
        wrong = np.where(kinds, 1.0, bf16(w[1])) @ V / w.sum()
        want = w @ V / w.sum()
        assert (wrong - want) @ want / (want @ want) > 1.3 * bound
