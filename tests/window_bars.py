"""Attention under a window in 64 bits with the error that one output element may have, and
the same for the norm and rotation. Plain numpy on whole score matrices (the oracle of
oracle/window.py goes key by key; a host test holds the two against each other).

Attention, with w a row's normalised weights, s its scores in powers of e, A = sum w |v|:

* a score is a sum of d products: (2 d + 8) 2^-24 sum |q k| / sqrt(d), doubled where the
  hardware may cut instead of round; the scale and its rounding are among the 8;
* the exponential's argument, in powers of 2, and its result: 2^-23 (|s| + max |s| + 40) of
  the weight, which also covers the rescaling and the combine's factors;
* these move a weight by delta of itself: sum w delta |v| in the numerator, |o| sum w delta
  in the sum;
* bf16 rounds a weight to bf16 for the product, half a step, 2^-8 of it, and the weights'
  sum takes the rounded ones: 2^-8 (A + |o|);
* the sums in float32: a product of 16 keys and an addition are each off by 2^-22 of A (the
  hardware may cut), a float32 kernel's additions, one a key, by 2^-24;
* the output's rounding: 2^-8 of itself (bf16) or 2^-24, and half of its type's least step.

Norm and rotation, float32 inside: the sum of squares is off by at most 13 roundings (eight a
lane, five between lanes), the norm by half of that and by those of the mean, the root and
the quotient; with the products by it and by the gain an element is off by 11 2^-24 of
itself. A cosine or sine is off by 3 2^-24 (the angle's rest, at most pi / 4, rounded; the
function to two units). A pair's two products and their sum round twice more: 16 2^-24
(|a| + |b|), and then the output's rounding.
"""
import numpy as np

HALF = {True: 2.0 ** -8, False: 2.0 ** -24}      # bf16?
LEAST = {True: 2.0 ** -134, False: 2.0 ** -150}


def attention(q, k, v, sees, bf16):
    """q [rows, Hq, d], k and v [keys, Hkv, d], sees [rows, keys]: outputs and bars."""
    q, k, v = (np.asarray(x, np.float64) for x in (q, k, v))
    rows, Hq, d = q.shape
    Hkv = k.shape[1]
    g = Hq // Hkv
    out, bar = np.zeros(q.shape), np.zeros(q.shape)
    for h in range(Hq):
        K, V, Q = k[:, h // g], v[:, h // g], q[:, h]
        fine = np.where(np.isfinite(K), K, 0.0), np.where(np.isfinite(V), V, 0.0)
        s = np.where(sees, Q @ fine[0].T / d ** 0.5, -np.inf)
        w = np.exp(s - s.max(1, keepdims=True))
        w /= w.sum(1, keepdims=True)
        o, A = w @ fine[1], w @ np.abs(fine[1])
        mag = np.abs(Q) @ np.abs(fine[0]).T / d ** 0.5
        s0 = np.where(sees, s, 0.0)
        delta = (2 * d + 8) * 2.0 ** -24 * mag
        delta = delta + 2.0 ** -23 * (np.abs(s0) + np.abs(s0).max(1, keepdims=True) + 40)
        err = (w * delta) @ np.abs(fine[1]) + (w * delta).sum(1, keepdims=True) * np.abs(o)
        n = sees.sum(1, keepdims=True)
        if bf16:
            err = err + HALF[True] * (A + np.abs(o)) + (n / 16 + 40) * 2.0 ** -22 * A
        else:
            err = err + (n + 40) * 2.0 ** -24 * A
        err = err * 1.02  # the terms that two of these make together
        err = err + HALF[bf16] * (np.abs(o) + err) + LEAST[bf16]
        out[:, h], bar[:, h] = o, err
    return out, bar


def in_window(pos, key_pos, window, sinks):
    p, j = np.asarray(pos)[:, None], np.asarray(key_pos)[None, :]
    return (j <= p) & ((j > p - window) | (j < sinks))


def prefill(prefix_len, q, k, v, window, sinks, bf16=True, rows_of=None):
    """All positions, or those of rows_of[r] of request r: {request: (rows, out, bar)}."""
    res, p0 = {}, 0
    for r, P in enumerate(int(x) for x in prefix_len):
        at = np.arange(P) if rows_of is None else np.asarray(rows_of[r])
        if len(at):
            sees = in_window(at, np.arange(P), window, sinks)
            need = np.flatnonzero(sees.any(0))
            o, bar = attention(q[p0 + at], k[p0 + need], v[p0 + need], sees[:, need], bf16)
            res[r] = p0 + at, o, bar
        p0 += P
    return res


def cascade(lay, q, k, v, kc, vc, window, sinks, bf16, requests=None):
    """The step's rows of the given requests: {request: (rows, out, bar)}."""
    res = {}
    for r in range(int(lay["R"])) if requests is None else requests:
        p0, p1 = (int(lay["prefix_offset"][r + i]) for i in (0, 1))
        n0, n1 = (int(lay["row_offset"][r + i]) for i in (0, 1))
        rows, P = np.arange(n0, n1), p1 - p0
        cand = lay["row_cand"][rows].astype(np.int64)
        pos = P - 1 + np.where(cand >= 0, lay["row_pos"][rows], 0)
        fed = np.arange(n0 - r, n1 - r - 1)  # fed tokens of the request, rows 1 ..
        sees = np.concatenate([
            in_window(pos, np.arange(P), window, sinks),
            in_window(pos, pos[1:], window, sinks) & (cand[:, None] == cand[None, 1:])], 1)
        K = np.concatenate([k[p0:p1], kc[fed]])
        V = np.concatenate([v[p0:p1], vc[fed]])
        need = np.flatnonzero(sees.any(0))
        o, bar = attention(q[rows], K[need], V[need], sees[:, need], bf16)
        res[r] = rows, o, bar
    return res


def rotation(x, pos, rot, style, freq, gain, eps, norm, bf16):
    """Outputs and bars of the norm and rotation of x [tokens, heads, d]."""
    x = np.asarray(x, np.float64)
    if norm:
        x = x / np.sqrt((x * x).mean(-1, keepdims=True) + eps)
        if gain is not None:
            x = x * gain
    h = rot // 2
    ia, ib = ((np.arange(h), np.arange(h) + h) if style == "halves" else
              (2 * np.arange(h), 2 * np.arange(h) + 1))
    t = np.asarray(pos, np.float64)[:, None, None] * np.asarray(freq)
    c, s = np.cos(t), np.sin(t)
    out, mag = x.copy(), np.abs(x)
    out[..., ia] = x[..., ia] * c - x[..., ib] * s
    out[..., ib] = x[..., ia] * s + x[..., ib] * c
    mag[..., ia] = mag[..., ib] = np.abs(x[..., ia]) + np.abs(x[..., ib])
    err = 16 * 2.0 ** -24 * mag
    return out, err + HALF[bf16] * (np.abs(out) + err) + LEAST[bf16]


def worst(got, want, bar):
    """The largest error in bars; a non-finite element is infinitely off."""
    d = np.abs(np.asarray(got, np.float64) - want)
    return float(np.where(np.isfinite(d), d / bar, np.inf).max()) if d.size else 0.0
