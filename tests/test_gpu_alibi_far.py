"""A position bias behind more cached rows than single precision counts (2^24): trees and block lists."""
import math

import numpy as np
import pytest
import torch

from mq_helpers import BF16, FP32, check, mask_tensor, np64, randn, trees
from oracle import tree_sparse as ts

pytestmark = pytest.mark.gpu

N, NEAR, D, R, SLOPE = 2 ** 24 + 1001, 512, 16, 8, 0.5


@pytest.fixture(scope="module")
def B():
    from paper_2408_05646_b200 import build
    build.build_library()
    from paper_2408_05646_b200 import binding
    return binding


def layer(B, dtype):
    """16.8 million rows, zeros but for the newest 512.  A bias of 0.5 a row leaves the others e^-250 of the newest one's
    weight (keys move a score by less than 6 either way), so the newest ones alone, counted from their own first, give the
    expected values."""
    U = np.eye(D, dtype=np.float32)[:, :R]
    lay = B.EigenAttnLayer(1, 1, D, N + 87, dtype, [U], [U])
    for i, which in enumerate("kv"):
        lay.cache_rows(0, which)[0, N - NEAR:N] = randn((NEAR, R), 3 + i, dtype)
    lay.set_len(N)
    lay.set_alibi([SLOPE])
    K, V = (np64(lay.cache_rows(0, w)[0, N - NEAR:N]) for w in "kv")
    return lay, U.astype(np.float64), K, V


def slack(q, K, w, V, U):
    """What the arithmetic may add (the terms of mq_helpers, with the bias of the rows that weigh anything: 512 at most)."""
    A = (np.abs(K) @ (np.abs(q) @ np.abs(U))).max() / math.sqrt(D)
    e_s = (2.0 ** -16 + (D + R + 4) * 2.0 ** -23) * A + 2.0 ** -22 * SLOPE * NEAR
    e_w = 2.2 * e_s + 2.0 ** -15 + (len(w) + 64) * 2.0 ** -24
    o = 2 * e_w * (w @ np.abs(V)) + 2.0 ** -22 * np.abs(w @ V)
    return np.abs(U) @ o + ((R + 2) * 2.0 ** -24 + 2.0 ** -16) * (np.abs(U) @ np.abs(w @ V))


@pytest.mark.parametrize("dtype,T", [(BF16, 5), (BF16, 20), (FP32, 5)])       # one run of query rows, several, the CUDA cores
def test_tree_behind_more_rows_than_single_precision_counts(B, dtype, T):
    lay, U, K, V = layer(B, dtype)
    q, k, v = (randn((1, T, 1, D), 11 + i, dtype) for i in range(3))
    masks, _ = trees(1, T, 5)
    lay.tree_attach(T)
    out = lay.decode_tree(q, k, v, mask_tensor(masks))
    lay.poll_status()
    Kt, Vt = (np64(lay.cache_rows(0, w)[0, N:N + T]) for w in "kv")
    qn = np64(q)[0, :, 0]
    want = ts.tree_head(qn @ U, K, V, Kt, Vt, masks[0], U, False, SLOPE)
    rows, ws = ts.tree_weights(qn @ U, K, Kt, masks[0], D, SLOPE)
    K, V = np.concatenate([K, Kt]), np.concatenate([V, Vt])
    for t in range(T):
        check(out[0, t, 0], want[t], slack(qn[t], K[rows[t]], ws[t], V[rows[t]], U), dtype, f"token {t}")


@pytest.mark.parametrize("dtype", [BF16, FP32])
def test_blocks_behind_more_rows_than_single_precision_counts(B, dtype):
    lay, U, K, V = layer(B, dtype)
    lay.sparse_attach(64)
    lay.sparse_sync()
    q = randn((1, 1, 1, D), 17, dtype)
    out, index = lay.decode_sparse(q, 6, return_index=True)
    last = (N - 1) // 64
    assert index[0, 0].tolist() == [0] + list(range(last - 4, last + 1))       # a block further back is 32 lower
    first = 64 * (last - 4) - (N - NEAR)
    qn = np64(q)[0, 0, 0]
    s = K[first:] @ (qn @ U) / math.sqrt(D) - SLOPE * np.arange(NEAR - first)[::-1]
    w = np.exp(s - s.max())
    w /= w.sum()
    check(out[0, 0, 0], U @ (w @ V[first:]), slack(qn, K[first:], w, V[first:], U), dtype, "sparse")
