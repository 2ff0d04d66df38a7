"""The fp64 definitions of the training calls and of the learned bias against what they are defined by."""
from fractions import Fraction

import numpy as np
import pytest

from oracle import training as oracle


@pytest.mark.parametrize("n_buckets,far", [(2, 2), (3, 7), (5, 3), (32, 128), (64, 1024), (21, 64)])
def test_buckets_by_their_inequality(n_buckets, far):
    half, rest = n_buckets // 2, n_buckets - n_buckets // 2
    got = [oracle.bucket_of(d, n_buckets, far) for d in range(2 * far + 3)]
    assert got[:half] == list(range(half)) and got == sorted(got)
    for d in range(half, len(got)):
        k = got[d] - half
        assert 0 <= k < rest
        assert Fraction(d, half) ** rest >= Fraction(far, half) ** k
        assert k == rest - 1 or Fraction(d, half) ** rest < Fraction(far, half) ** (k + 1)


@pytest.mark.parametrize("bias", [None, "alibi", "table"])
@pytest.mark.parametrize("T", [1, 2, 9])
def test_gradients_against_differences(T, bias):
    """Central differences of sum(o * d_out) at step h = 2^-10: their error is h^2 / 6 of a third derivative and 2^-53 / h of
    the value, both below 1e-5 for numbers of this size."""
    rng = np.random.default_rng(T)
    q, k, v, g = (rng.standard_normal((T, r)) for r in (5, 5, 3, 3))
    b = {None: np.zeros(T), "alibi": -0.25 * np.arange(T), "table": rng.standard_normal(T)}[bias]
    scale, h = 0.4, 2.0 ** -10
    dq, dk, dv, db = oracle.attention_gradients(q, k, v, g, scale, b)

    def loss():
        return np.sum(oracle.attention(q, k, v, scale, b)[0] * g)

    for x, dx in ((q, dq), (k, dk), (v, dv), (b, db)):
        assert x.shape == dx.shape
        for at in np.ndindex(x.shape):
            keep = x[at]
            x[at] = keep + h
            up = loss()
            x[at] = keep - h
            down = loss()
            x[at] = keep
            assert abs((up - down) / (2 * h) - dx[at]) < 1e-5, (at, dx[at])


def test_a_table_by_distance():
    table = np.arange(8.0).reshape(2, 4)
    by = oracle.bias_by_distance(table, 6, 10)
    for d in range(10):
        assert (by[:, d] == table[:, oracle.bucket_of(d, 4, 6)]).all()


def test_packed_calls_are_the_heads_one_by_one():
    """Shared heads add up, rows behind a sequence's end and padding columns are zero."""
    rng = np.random.default_rng(0)
    B, T, r_k, r_v, group, lens = 2, 6, [3, 8], [5, 2], 2, [4, 0]
    kq, wq = oracle.packed_columns(r_k, group)
    vq, wo = oracle.packed_columns(r_v, group)
    k1, wk = oracle.packed_columns(r_k)
    v1, wv = oracle.packed_columns(r_v)
    q, k, v, g = (rng.standard_normal((B, T, w)) for w in (wq, wk, wv, wo))
    got = oracle.train(q, k, v, g, r_k, r_v, 16, group, lens)
    want = {name: np.zeros_like(x) for name, x in (("out", g), ("dq", q), ("dk", k), ("dv", v))}
    n = lens[0]
    for h in range(2):
        for i in range(group):
            a, c = kq[h * group + i], vq[h * group + i]
            args = q[0, :n, a].T, k[0, :n, k1[h]].T, v[0, :n, v1[h]].T
            want["out"][0, :n, c] = oracle.attention(*args, 0.25)[0].T
            dq, dk, dv, _ = oracle.attention_gradients(*args, g[0, :n, c].T, 0.25)
            want["dq"][0, :n, a] = dq.T
            want["dk"][0, :n, k1[h]] += dk.T
            want["dv"][0, :n, v1[h]] += dv.T
    for name, x in want.items():
        np.testing.assert_allclose(got[name], x, rtol=1e-12, atol=1e-12, err_msg=name)
