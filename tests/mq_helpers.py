"""Shared by the tests of tree attention and of decode over selected blocks: layers with random rows, the 64-bit expected
values with a bound on what the kernels' arithmetic may add, and the drafted trees.

The bound (`expected`): the kernels round the stored rows (the expected value starts from the rows as the cache holds them,
so that costs nothing here) and the output, by at most half a step (2^-8 of the value in bf16, 2^-24 in fp32).  In between
everything is single precision or a pair of 16-bit numbers with 16 significant bits between them:
  * Q' is off by 2^-16 of its entries' size (a pair of 16-bit numbers holds a 32-bit one to 2^-18: once the basis, once Q'
    itself) and a sum of d_head products by d_head 2^-24 of the sum of their magnitudes,
    a score's sum of r products by r 2^-24, its bias by 2^-22: together a score is off by at most
        e_s = (2^-16 + (d_head + r + 4) 2^-23) A + 2^-22 |bias|,   A = sum_c (sum_d |q_d U_dc|) |k'_c| / sqrt(d_head);
  * a weight is off by e^{2 e_s} - 1 (numerator and the maximum that is taken out), 2^-16 for its 16-bit pair, 2^-21 for
    the exponential, and the sum over n rows by n 2^-24: e_w = 2.2 max e_s + 2^-15 + (n + 64) 2^-24, once for the
    numerator and once for the sum of the weights;
  * the lift adds (r + 2) 2^-24 of the sum of its products' magnitudes; with both factors as such pairs, and the product of
    their remainders left out, 3 * 2^-18 more, which is taken as 2^-16."""
import math

import numpy as np
import torch

from oracle import eigen_attention as orc
from oracle import tree_sparse as ts
from paper_2408_05646_b200 import synth

BF16, FP32 = torch.bfloat16, torch.float32
HALF_STEP = {BF16: 2.0 ** -8, FP32: 2.0 ** -24}


def np64(x):
    return x.detach().double().cpu().numpy()


def bases(H, d, rk, rv, seed):
    U_k = [synth.orthonormal_basis(d, r, seed * 101 + h).astype(np.float32) for h, r in enumerate(rk)]
    U_v = [synth.orthonormal_basis(d, r, seed * 103 + 50 + h).astype(np.float32) for h, r in enumerate(rv)]
    return U_k, U_v


def randn(shape, seed, dtype, scale=1.0, device="cuda:0"):
    g = torch.Generator(device="cpu").manual_seed(seed)
    return (torch.randn(shape, generator=g) * scale).to(dtype).to(device)


def trees(B, T, seed, kind="tree"):
    """masks: python ints [B][T]; parents [B][T]."""
    g = np.random.default_rng(seed)
    masks, parents = [], []
    for b in range(B):
        row, par = [], []
        for t in range(T):
            p = t - 1 if kind == "chain" else int(g.integers(-1, t)) if t else -1
            par.append(p)
            row.append((1 << t) | (row[p] if p >= 0 else 0))
        if kind == "any":                       # not a tree: any subset, the empty one among them, bits past T
            row = [int(g.integers(0, 1 << min(T, 62))) if t % 3 else 0 for t in range(T)]
            row = [x | (1 << 63) if T < 64 and t % 2 else x for t, x in enumerate(row)]
        masks.append(row)
        parents.append(par)
    return masks, parents


def mask_tensor(masks, device="cuda:0"):
    return torch.tensor([[x - (1 << 64) if x >> 63 else x for x in row] for row in masks], dtype=torch.int64, device=device)


class Case:
    """A layer on the GPU whose caches hold random rows, with what the oracle needs."""

    def __init__(self, B, dtype, batch, H, group, d, rk, rv, lens, n_max, seed, page_rows=0, slopes=None, peak=1.0):
        self.dtype, self.batch, self.H, self.group, self.d = dtype, batch, H, group, d
        self.rk, self.rv, self.lens, self.slopes = rk, rv, list(lens), slopes
        self.U_k, self.U_v = bases(H, d, rk, rv, seed)
        self.lay = lay = B.EigenAttnLayer(batch, H, d, n_max, dtype, self.U_k, self.U_v)
        self.page_rows, self.table = page_rows, None
        if page_rows:
            perm = np.random.default_rng(seed).permutation(batch * n_max // page_rows)
            per = len(perm) // batch
            self.table = [[int(x) for x in perm[b * per:(b + 1) * per]] for b in range(batch)]
            lay.set_page_table(self.table, page_rows)
        if slopes is not None:
            lay.set_alibi(slopes)
        n = max(self.lens)
        self.peak = peak
        if n:
            self.k, self.v = randn((batch, n, H, d), seed + 1, dtype), randn((batch, n, H, d), seed + 2, dtype)
            lay.append_kv(self.k, self.v)
        if len(set(self.lens)) > 1:
            lay.set_lens(self.lens)
        self.seed = seed

    def rows(self, b, h, count, which):
        """The first `count` rows of a unit as the cache holds them (64-bit copies)."""
        slab = self.lay.cache_rows(h, which)
        r = (self.rk if which == "k" else self.rv)[h]
        if self.table is None:
            return np64(slab[b, :count])[:, :r]
        return orc.paged_gather(np64(slab.reshape(-1, slab.shape[-1])), self.table[b], self.page_rows, count)[:, :r]

    def score_error(self, q, Kp, h, slope, span):
        """Largest |error| of a score: q [d] the query, Kp the rows it meets, span the largest distance under a bias."""
        if not len(Kp):
            return 0.0
        reach = np.abs(q) @ np.abs(np.float64(self.U_k[h]))
        A = (np.abs(Kp) @ reach).max() / math.sqrt(self.d)
        return (2.0 ** -16 + (self.d + self.rk[h] + 4) * 2.0 ** -23) * A + 2.0 ** -22 * slope * span

    def bound(self, w, V, e_s, h, lowrank=False):
        """Bound on what the arithmetic adds to an output with weights w over rows V."""
        if not len(w):
            return np.zeros(self.rv[h] if lowrank else self.d)
        e_w = 2.2 * e_s + 2.0 ** -15 + (len(w) + 64) * 2.0 ** -24
        o = 2 * e_w * (w @ np.abs(V)) + 2.0 ** -22 * np.abs(w @ V)
        if lowrank:
            return o
        U = np.abs(np.float64(self.U_v[h]))
        pairs = 2.0 ** -16 if self.dtype == BF16 else 0.0
        return U @ o + ((self.rv[h] + 2) * 2.0 ** -24 + pairs) * (U @ np.abs(w @ V))


def check(got, want, slack, dtype, what):
    got = np64(got) if torch.is_tensor(got) else got
    assert got.shape == want.shape, (what, got.shape, want.shape)
    assert np.isfinite(got).all(), f"{what}: non-finite output"
    over = np.abs(got - want) - (HALF_STEP[dtype] * np.abs(want) + slack)
    at = np.unravel_index(np.argmax(over), over.shape)
    assert over[at] <= 0, f"{what}: {got[at]} for {want[at]} at {at}, {over[at]:.3e} over the bound (slack {slack[at]:.3e})"


def tree_expected(c, q, masks, T, lowrank=False, rank_q=None, units=None):
    """(expected, slack) [batch][T][H * group][d] (lowrank: a list per head of [batch][T][group][r]) from the rows the cache
    holds after the call.  rank_q: the queries as rank-r rows, a function (b, h, i) -> [T, r].  units: only these (b, h); the
    rest stays zero."""
    want = np.zeros((c.batch, T, c.H * c.group, c.d))
    slack = np.zeros_like(want)
    low = [[np.zeros((c.batch, T, c.group, r)) for r in c.rv] for _ in range(2)]
    qn = None if q is None else np64(q)
    for b in range(c.batch):
        n = c.lens[b]
        for h in range(c.H):
            if units is not None and (b, h) not in units:
                continue
            K, V = c.rows(b, h, n + T, "k"), c.rows(b, h, n + T, "v")
            slope = c.slopes[h] if c.slopes is not None else 0.0
            for i in range(c.group):
                x = None if qn is None else qn[b, :, h * c.group + i]
                qp = x @ np.float64(c.U_k[h]) if rank_q is None else rank_q(b, h, i)
                out = ts.tree_head(qp, K[:n], V[:n], K[n:], V[n:], masks[b], c.U_v[h].astype(np.float64), lowrank, slope)
                rows_of, ws = ts.tree_weights(qp, K[:n], K[n:], masks[b], c.d, slope)
                for t in range(T):
                    full = x[t] if x is not None else qp[t] @ np.float64(c.U_k[h]).T
                    e_s = c.score_error(full, K[rows_of[t]], h, slope, n + T)
                    e = c.bound(ws[t], V[rows_of[t]], e_s, h, lowrank)
                    if lowrank:
                        low[0][h][b, t, i], low[1][h][b, t, i] = out[t], e
                    else:
                        want[b, t, h * c.group + i], slack[b, t, h * c.group + i] = out[t], e
    return low if lowrank else (want, slack)


def sparse_expected(c, q, block, n_blocks, sink, recent):
    """(expected, slack, index) of decode over the chosen blocks."""
    want = np.zeros((c.batch, 1, c.H * c.group, c.d))
    slack = np.zeros_like(want)
    index = -np.ones((c.batch, c.H, n_blocks), dtype=np.int64)
    qn = np64(q)
    for b in range(c.batch):
        n = c.lens[b]
        for h in range(c.H):
            K, V = c.rows(b, h, n, "k"), c.rows(b, h, n, "v")
            slope = c.slopes[h] if c.slopes is not None else 0.0
            x = qn[b, 0, h * c.group:(h + 1) * c.group]
            qp = x @ np.float64(c.U_k[h])
            blocks = ts.choose_blocks(qp, K, block, n_blocks, sink, recent, c.d, slope)
            index[b, h, :len(blocks)] = blocks
            chosen = set(blocks)
            rows = [j for j in range(n) if j // block in chosen]
            for i in range(c.group):
                s = K[rows] @ qp[i] / math.sqrt(c.d) - slope * ((n - 1) - np.asarray(rows, np.float64))
                w = orc.softmax_rows(s[None])[0]
                want[b, 0, h * c.group + i] = ts.blocks_head(qp[i], K, V, blocks, block, c.U_v[h].astype(np.float64), slope=slope)
                slack[b, 0, h * c.group + i] = c.bound(w, V[rows], c.score_error(x[i], K[rows], h, slope, n), h)
    return want, slack, index
