"""fp64 CPU oracle of positions and windows: the norm and rotation of query and key heads,
and attention that sees a window of the last tokens and a few first ones.

TEST INFRASTRUCTURE, as the rest of this package: plain loops over rows and heads, sets of
positions instead of ranges, no code shared with the GPU path.
"""
from __future__ import annotations

import math

import numpy as np

from .stack import _fed_rows, _gate_up, bf16, rmsnorm, silu

__all__ = ["frequencies", "rotate", "seen", "row_position", "window_keys", "window_cascade",
           "window_prefill", "full_layer"]


def frequencies(rot: int, theta: float) -> np.ndarray:
    """theta^(-2 i / rot) in radians a position, i < rot / 2."""
    return np.array([theta ** (-2.0 * i / rot) for i in range(rot // 2)])


def rotate(x, pos, rot: int, style: str, freq, gain=None, eps: float = 1e-6,
           norm: bool = True) -> np.ndarray:
    """x [tokens, heads, d] at positions pos [tokens]: each head normalised (norm) and its
    first `rot` elements rotated by p f_i, the pairs half a rotation apart ("halves") or
    neighbours ("pairs")."""
    x = np.asarray(x, np.float64).copy()
    n, H, d = x.shape
    if norm:
        for t in range(n):
            for h in range(H):
                x[t, h] /= math.sqrt(float(np.mean(x[t, h] ** 2)) + eps)
        if gain is not None:
            x *= np.asarray(gain, np.float64)
    out = x.copy()
    for i in range(rot // 2):
        a, b = (i, i + rot // 2) if style == "halves" else (2 * i, 2 * i + 1)
        angle = np.asarray(pos, np.float64) * freq[i]
        c, s = np.cos(angle)[:, None], np.sin(angle)[:, None]
        out[:, :, a] = x[:, :, a] * c - x[:, :, b] * s
        out[:, :, b] = x[:, :, a] * s + x[:, :, b] * c
    return out


def seen(p: int, window: int, sinks: int):
    """The positions that position p sees, in order."""
    return [j for j in range(p + 1) if j > p - window or j < sinks]


def row_position(lay, n: int) -> int:
    """The position of row n: its request's last prefix token, or t past it."""
    r = int(lay["row_req"][n])
    P = int(lay["prefix_offset"][r + 1]) - int(lay["prefix_offset"][r])
    return P - 1 + (int(lay["row_pos"][n]) if int(lay["row_cand"][n]) >= 0 else 0)


def window_keys(lay, n: int, window: int, sinks: int):
    """(prefix key rows, fed-token rows) that row n sees."""
    r = int(lay["row_req"][n])
    p0 = int(lay["prefix_offset"][r])
    P = int(lay["prefix_offset"][r + 1]) - p0
    t = row_position(lay, n) - (P - 1)
    pre, fed = [], []
    for j in seen(P - 1 + t, window, sinks):
        if j < P:
            pre.append(p0 + j)
        else:  # own token y_{j - P + 1}; the row's own is y_t, fed token n - r - 1
            fed.append(n - r - 1 - (t - (j - P + 1)))
    return pre, fed


def _attend(qh, K, V, scale):
    s = (K @ qh) * scale
    w = np.exp(s - s.max())
    return (w / w.sum()) @ V


def window_cascade(lay, q, k_pre, v_pre, k_cand, v_cand, Hq, Hkv, window, sinks, rows):
    """The step's attention under the window: [rows, Hq, d]."""
    g, d = Hq // Hkv, q.shape[2]
    out = np.zeros((len(rows), Hq, d))
    for i, n in enumerate(rows):
        pre, fed = window_keys(lay, n, window, sinks)
        for h in range(Hq):
            K = np.concatenate([k_pre[pre, h // g], k_cand[fed, h // g].reshape(len(fed), d)])
            V = np.concatenate([v_pre[pre, h // g], v_cand[fed, h // g].reshape(len(fed), d)])
            out[i, h] = _attend(np.asarray(q[n, h], np.float64), K.astype(np.float64),
                                V.astype(np.float64), 1.0 / math.sqrt(d))
    return out


def window_prefill(prefix_len, q, k, v, Hq, Hkv, window, sinks, rows):
    """The prefill under the window: [rows, Hq, d]."""
    off = np.concatenate([[0], np.cumsum(prefix_len)])
    g, d = Hq // Hkv, q.shape[2]
    out = np.zeros((len(rows), Hq, d))
    for i, n in enumerate(rows):
        p0 = int(off[np.searchsorted(off, n, side="right") - 1])
        at = [p0 + j for j in seen(n - p0, window, sinks)]
        for h in range(Hq):
            out[i, h] = _attend(np.asarray(q[n, h], np.float64),
                                np.asarray(k[at, h // g], np.float64),
                                np.asarray(v[at, h // g], np.float64), 1.0 / math.sqrt(d))
    return out


def full_layer(lay, x, P, dims, window=None, sinks=0, rope=None):
    """A decoder stack's full layer with positions, at the stack oracle's storage points and one
    more, the rotated queries and keys: rope is None or a dict of rot, style, freq, eps and norm
    (gains gq and gk in P), window None or the tokens a token sees."""
    N = x.shape[0]
    fed = _fed_rows(lay)
    Hq, Hkv, d = dims["Hq"], dims["Hkv"], dims["d"]
    z = bf16(bf16(rmsnorm(x, P["g1"])) @ P["w_mix"].T)
    q = z[:, :Hq * d].reshape(N, Hq, d)
    k = z[:, Hq * d:(Hq + Hkv) * d].reshape(N, Hkv, d)
    v = z[:, (Hq + Hkv) * d:].reshape(N, Hkv, d)
    if rope is not None:
        pos = [row_position(lay, n) for n in range(N)]
        q, k = (bf16(rotate(t, pos, rope["rot"], rope["style"], rope["freq"], P.get(g),
                            rope["eps"], rope["norm"])) for t, g in ((q, "gq"), (k, "gk")))
    wide = 1 << 40 if window is None else window
    o = bf16(window_cascade(lay, q, P["k_pre"], P["v_pre"], k[fed], v[fed], Hq, Hkv, wide, sinks,
                            list(range(N))))
    x1 = bf16(x + o.reshape(N, Hq * d) @ P["w_o"].T)
    wg, wu = _gate_up(P["w_gu"], dims["Dff"])
    h2 = bf16(rmsnorm(x1, P["g2"]))
    return bf16(x1 + bf16(silu(h2 @ wg.T) * (h2 @ wu.T)) @ P["w_d"].T)
