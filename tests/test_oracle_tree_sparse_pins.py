"""Pins of the fp64 definitions of tree attention and of decode over selected blocks (CPU only): special cases that other
definitions or a library routine cover, and properties that a wrong mask, axis or tie rule breaks."""
import math

import numpy as np
import pytest
import torch

from oracle import eigen_attention as orc
from oracle import tree_sparse as ts


def setup(n=9, T=5, d=16, r=6, seed=0):
    g = np.random.default_rng(seed)
    U_K, U_V = (np.linalg.qr(g.standard_normal((d, r)))[0] for _ in "kv")
    return g, U_K, U_V, g.standard_normal((T, d)), g.standard_normal((n + T, d)), g.standard_normal((n + T, d))


@pytest.mark.parametrize("n", [0, 1, 9])
@pytest.mark.parametrize("slope", [0.0, 0.3])
def test_a_chain_is_a_causal_prompt(n, slope):
    _, U_K, U_V, q, k, v = setup(n)
    T = q.shape[0]
    want = orc.prefill_head(q, k, v, U_K, U_V, len0=n, alibi_slope=slope)
    Kp, Vp = k @ U_K, v @ U_V
    got = ts.tree_head(q @ U_K, Kp[:n], Vp[:n], Kp[n:], Vp[n:], [(2 << t) - 1 for t in range(T)], U_V, slope=slope)
    assert np.abs(got - want).max() < 1e-12


def test_every_path_of_a_tree_is_a_sequence_of_its_own():
    n, slope = 7, 0.25
    _, U_K, U_V, q, k, v = setup(n, T=6, seed=1)
    parent = [-1, 0, 0, 2, -1, 3]
    paths = []
    for t in range(6):
        p = [t]
        while parent[p[0]] >= 0:
            p.insert(0, parent[p[0]])
        paths.append(p)
    masks = [sum(1 << s for s in p) for p in paths]
    Kp, Vp = k @ U_K, v @ U_V
    got = ts.tree_head(q @ U_K, Kp[:n], Vp[:n], Kp[n:], Vp[n:], masks, U_V, slope=slope)
    for t, p in enumerate(paths):
        rows = list(range(n)) + [n + s for s in p]
        want = orc.decode_head(q[t], k[rows], v[rows], U_K, U_V, alibi_slope=slope)
        assert np.abs(got[t] - want).max() < 1e-12


def test_tree_masks_against_library_attention():
    n, T, d = 5, 4, 16
    g, U_K, U_V, q, k, v = setup(n, T, d, r=d, seed=2)
    masks = [int(x) for x in g.integers(0, 1 << T, T)]
    allowed = torch.tensor([[True] * n + [bool((m >> s) & 1) for s in range(T)] for m in masks])
    want = torch.nn.functional.scaled_dot_product_attention(*[torch.from_numpy(x)[None, None] for x in (q, k, v)],
                                                            attn_mask=allowed[None, None])[0, 0].numpy()
    Kp, Vp = k @ U_K, v @ U_V                      # full rank: nothing is lost
    got = ts.tree_head(q @ U_K, Kp[:n], Vp[:n], Kp[n:], Vp[n:], masks, U_V)
    assert np.abs(got - want).max() < 1e-12


def test_a_token_that_sees_nothing_gets_zeros_and_high_bits_name_nothing():
    _, U_K, U_V, q, k, v = setup(0, T=3, seed=3)
    Kp, Vp = k @ U_K, v @ U_V
    got = ts.tree_head(q @ U_K, Kp[:0], Vp[:0], Kp, Vp, [0, 0b010, 0b101 | (1 << 40)], U_V)
    assert not got[0].any() and got[1].any()
    want = ts.tree_head(q @ U_K, Kp[:0], Vp[:0], Kp, Vp, [0, 0b010, 0b101], U_V)
    assert np.array_equal(got, want) and ts.tree_depth(0b101 | (1 << 40), 2, 3) == 1


def test_bounds_are_bounds_and_tight_for_one_row():
    g = np.random.default_rng(4)
    K, q = g.standard_normal((23, 7)), g.standard_normal(7)
    lo, hi = ts.block_bounds(K, 4)
    assert lo.shape == (5, 7)
    for j in range(5):
        s = K[4 * j:4 * j + 4] @ q / math.sqrt(16)
        top = ts.block_score(q, lo[j], hi[j], 16)
        assert top >= s.max() - 1e-12
        assert abs(top - sum(max(q[c] * lo[j, c], q[c] * hi[j, c]) for c in range(7)) / 4) < 1e-12
    one_lo, one_hi = ts.block_bounds(K, 1)
    assert abs(ts.block_score(q, one_lo[3], one_hi[3], 16) - K[3] @ q / 4) < 1e-12


def test_choice_forced_blocks_ties_and_groups():
    K = np.zeros((40, 2))
    K[8:12] = K[20:24] = [[3.0, 0.0]] * 4              # blocks 2 and 5 alike
    K[28:32] = [[0.0, 5.0]] * 4                        # block 7: only the second head wants it
    q = np.array([[1.0, 0.0]])
    assert ts.choose_blocks(q, K, 4, 3, 1, 1, 16) == [0, 2, 9]           # equal scores: the lower block
    assert ts.choose_blocks(q, K, 4, 4, 1, 1, 16) == [0, 2, 5, 9]
    assert ts.choose_blocks(q, K, 4, 5, 1, 1, 16) == [0, 1, 2, 5, 9]     # then zeros, lowest first
    assert ts.choose_blocks(np.array([[1.0, 0.0], [0.0, 1.0]]), K, 4, 4, 1, 1, 16) == [0, 2, 7, 9]
    assert ts.choose_blocks(q, K[:39], 4, 3, 0, 2, 16) == [2, 8, 9]      # the incomplete block counts as one
    assert ts.choose_blocks(q, K, 4, 10, 1, 1, 16) == list(range(10))
    assert ts.choose_blocks(q, K, 4, 3, 1, 1, 16, slope=1.0) == [0, 8, 9]   # a steep bias wants the newest


def test_all_blocks_is_ordinary_decode():
    _, U_K, U_V, q, k, v = setup(30, T=1, seed=5)
    Kp, Vp = k @ U_K, v @ U_V
    got = ts.blocks_head(q[0] @ U_K, Kp, Vp, range(8), 4, U_V, slope=0.2)
    assert np.abs(got - orc.decode_head(q[0], k, v, U_K, U_V, alibi_slope=0.2)).max() < 1e-12
    part = ts.blocks_head(q[0] @ U_K, Kp, Vp, [0, 3], 4, U_V)
    rows = [0, 1, 2, 3, 12, 13, 14, 15]
    assert np.abs(part - orc.decode_head(q[0], k[rows], v[rows], U_K, U_V)).max() < 1e-12
