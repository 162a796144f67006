"""Generation over a forest of cached segments, in float64 with numpy: e4m3
rounding with a power-of-two scale per vector, attention of the last rows of
segments over their chains, and the recurrent steps with their magnitudes
(the same sums over absolute values, which bound the rounding of a float32
evaluation)."""
from __future__ import annotations

import math

import numpy as np


def e4m3_scale(top):
    """Smallest integer e >= -126 with top <= 448 * 2^e."""
    if top == 0:
        return -126
    m, x = math.frexp(float(top))             # top = m 2^x, m in [0.5, 1)
    return max(-126, x - 9 if m <= 448 / 512 else x - 8)


def e4m3_round(y):
    """To nearest even among 1.mmm x 2^e, e >= -6, and steps of 2^-9 below."""
    y = np.asarray(y, np.float64)
    _, x = np.frexp(np.where(y == 0, 1.0, np.abs(y)))
    step = np.exp2(np.maximum(x - 1, -6) - 3.0)
    return np.rint(y / step) * step


def e4m3_vectors(x):
    """(values that the stored vectors stand for, scale exponents) of x [..., d].
    The values are bf16: 2^128, which the largest finite ones would round to, is
    past its range, and 240 x 2^120 is the largest that a code stands for."""
    x = np.asarray(x, np.float64)
    fin = np.isfinite(x)
    top = np.max(np.abs(np.where(fin, x, 0.0)), axis=-1)
    e = np.vectorize(e4m3_scale, otypes=[np.int64])(top)
    s = np.exp2(e.astype(np.float64))[..., None]
    most = 240 * 2.0 ** 120
    return np.where(fin, np.clip(e4m3_round(np.where(fin, x, 0.0) / s) * s, -most, most), np.nan), e


def chain(parent, s):
    out = [s]
    while parent[out[-1]] >= 0:
        out.append(int(parent[out[-1]]))
    return out[::-1]


def forest_decode(parent, n_new, K, V, q, scale):
    """K[s], V[s] [rows_s, Hkv, d] of every segment; q [n_rows, Hq, d], the last
    n_new[s] rows of every segment by ascending s.  Returns o, lse, and per
    output the weighted sum of |V| and per (row, head) the largest
    scale * sum |q||k| over visible keys."""
    n_rows, Hq, d = q.shape
    o, mag = np.zeros((n_rows, Hq, d)), np.zeros((n_rows, Hq, d))
    lse, reach = np.full((n_rows, Hq), -np.inf), np.zeros((n_rows, Hq))
    r = 0
    for s in range(len(parent)):
        if n_new[s] == 0:
            continue
        segs = chain(parent, s)
        k, v = (np.concatenate([x[c] for c in segs]) for x in (K, V))
        group = Hq // k.shape[1]
        for i in range(n_new[s]):
            see = k.shape[0] - len(K[s]) + max(0, len(K[s]) - n_new[s] + i + 1)
            for h in range(Hq):
                if see == 0:
                    continue
                kk, vv = k[:see, h // group], v[:see, h // group]
                z = scale * (kk @ q[r, h])
                if np.all(z == -np.inf):
                    continue
                top = np.max(z)
                w = np.exp(z - top)
                t = np.sum(w)
                lse[r, h] = top + np.log(t)
                o[r, h] = (w / t) @ vv
                mag[r, h] = (w / t) @ np.abs(vv)
                reach[r, h] = np.max(abs(scale) * (np.abs(kk) @ np.abs(q[r, h])))
            r += 1
    return o, lse, mag, reach


def step_tokens(q, k, v, g, beta, S, scale):
    """Tokens one after the other: q, k, v [T, H, d], g [T, H] (beta None) or
    [T, H, d] (KDA), S [H, d, d].  Returns (o, S, |o|, |S|): the last two from
    the same sums over absolute values."""
    o, mo = np.zeros_like(q, dtype=np.float64), np.zeros_like(q, dtype=np.float64)
    S, M = S.astype(np.float64), np.abs(S.astype(np.float64))
    for t in range(q.shape[0]):
        a = np.exp(g[t].astype(np.float64))
        a = a[:, None, None] if beta is None else a[:, :, None]
        S, M = a * S, a * M
        new, mnew = v[t].astype(np.float64), np.abs(v[t])
        if beta is not None:
            b = beta[t][:, None].astype(np.float64)
            new = b * (new - np.einsum("hi,hij->hj", k[t], S))
            mnew = np.abs(b) * (mnew + np.einsum("hi,hij->hj", np.abs(k[t]), M))
        S = S + k[t][:, :, None] * new[:, None, :]
        M = M + np.abs(k[t])[:, :, None] * mnew[:, None, :]
        o[t] = scale * np.einsum("hi,hij->hj", q[t], S)
        mo[t] = abs(scale) * np.einsum("hi,hij->hj", np.abs(q[t]), M)
    return o, S, mo, M
