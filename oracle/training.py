"""fp64 CPU definitions of attention over rank-space rows with its gradients, and of the learned bias of relative positions.

Plain formulas, one sequence and head at a time; nothing is shared with the library."""
import math
from fractions import Fraction

import numpy as np


def bucket_of(distance, n_buckets, max_distance):
    """Bucket of one distance >= 0, from the definition: half = n_buckets // 2 buckets of one distance each, then the largest
    k with (d / half)^rest >= (max_distance / half)^k."""
    half = n_buckets // 2
    rest = n_buckets - half
    if distance < half:
        return distance
    k = 0
    while k + 1 < rest and Fraction(distance, half) ** rest >= Fraction(max_distance, half) ** (k + 1):
        k += 1
    return half + k


def bias_by_distance(table, max_distance, count):
    """[H][count]: bias of the distances 0 .. count - 1 for a table [H][n_buckets]."""
    table = np.asarray(table, dtype=np.float64)
    return table[:, [bucket_of(d, table.shape[1], max_distance) for d in range(count)]]


def attention(q, k, v, scale, bias=None):
    """Causal attention of one head: q [T][rk], k [T][rk], v [T][rv], bias [T] by distance.  Returns (o, P)."""
    T = q.shape[0]
    o, P = np.zeros((T, v.shape[1])), np.zeros((T, T))
    for i in range(T):
        s = k[:i + 1] @ q[i] * scale
        if bias is not None:
            s = s + bias[i::-1][:i + 1]
        w = np.exp(s - s.max())
        P[i, :i + 1] = w / w.sum()
        o[i] = P[i, :i + 1] @ v[:i + 1]
    return o, P


def attention_gradients(q, k, v, d_out, scale, bias=None):
    """(dq, dk, dv, by_distance): the gradients of sum(o * d_out); by_distance [T] of the bias of every distance."""
    o, P = attention(q, k, v, scale, bias)
    T = q.shape[0]
    dS = P * (d_out @ v.T - np.sum(d_out * o, axis=1)[:, None])
    by_distance = np.array([np.trace(dS, -d) for d in range(T)])
    return dS @ k * scale, dS.T @ q * scale, P.T @ d_out, by_distance


def term_sizes(q, k, v, d_out, scale, bias=None):
    """(out, dq, dk, dv, by_distance) with every product taken in absolute value: what a relative error of P, of dS's two
    parts or of a product is multiplied by."""
    o, P = attention(q, k, v, scale, bias)
    A = P * (np.abs(d_out) @ np.abs(v).T + np.sum(np.abs(d_out * o), axis=1)[:, None])
    return P @ np.abs(v), A @ np.abs(k) * scale, A.T @ np.abs(q) * scale, P.T @ np.abs(d_out), np.array([np.trace(A, -d) for d in range(len(q))])


def packed_columns(r, group=1):
    """(columns of every query head in packed rows, width): ranks r per K/V head, each padded to a multiple of 8."""
    cols, base = [], 0
    for x in r:
        for _ in range(group):
            cols.append(np.arange(base, base + x))
            base += -(-x // 8) * 8
    return cols, base


def train(q, k, v, d_out, r_k, r_v, d_head, group=1, lens=None, bias=None):
    """The whole of both calls on packed rows (numpy, any float dtype): {"out", "dq", "dk", "dv", "by_distance" [H][T]} and
    the same keys with "_size" behind them (term_sizes)."""
    B, T, _ = q.shape
    q, k, v, d_out = (np.asarray(x, dtype=np.float64) for x in (q, k, v, d_out))
    kq, _ = packed_columns(r_k, group)
    vq, _ = packed_columns(r_v, group)
    k1, _ = packed_columns(r_k)
    v1, _ = packed_columns(r_v)
    got = {"out": np.zeros_like(d_out), "dq": np.zeros_like(q), "dk": np.zeros_like(k), "dv": np.zeros_like(v),
           "by_distance": np.zeros((len(r_k), T))}
    got.update({key + "_size": np.zeros_like(x) for key, x in list(got.items())})
    scale = 1.0 / math.sqrt(d_head)
    for b in range(B):
        n = T if lens is None else max(0, min(T, int(lens[b])))
        if n == 0:
            continue
        for h in range(len(r_k)):
            K, V = k[b, :n][:, k1[h]], v[b, :n][:, v1[h]]
            for i in range(group):
                cq, cv = kq[h * group + i], vq[h * group + i]
                Q, dO = q[b, :n][:, cq], d_out[b, :n][:, cv]
                w = None if bias is None else bias[h]
                got["out"][b, :n, cv] = attention(Q, K, V, scale, w)[0].T
                dq, dk, dv, by = attention_gradients(Q, K, V, dO, scale, w)
                got["dq"][b, :n, cq] = dq.T
                got["dk"][b, :n, k1[h]] += dk.T
                got["dv"][b, :n, v1[h]] += dv.T
                got["by_distance"][h, :n] += by
                out, dq, dk, dv, by = term_sizes(Q, K, V, dO, scale, w)
                got["out_size"][b, :n, cv], got["dq_size"][b, :n, cq] = out.T, dq.T
                got["dk_size"][b, :n, k1[h]] += dk.T
                got["dv_size"][b, :n, v1[h]] += dv.T
                got["by_distance_size"][h, :n] += by
    return got
