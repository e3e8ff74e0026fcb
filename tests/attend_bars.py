"""The cascade attention over an 8-bit prefix cache in 64 bits, and the error that one
output element may have, of what the row itself weighs: sum w |v|, not the largest value
of its request. Plain numpy, for the GPU tests and for the host tests of the bar.

With w the row's normalised weights, s its scores in powers of e, A = sum w |v|:

* a score is a sum of n products (n = d; bf16 takes every query as two numbers, so 2 d,
  whose magnitudes add up to at most 17/16 of the query's). Each is off by 2^-24 and so is
  each addition, doubled where a product's hardware may cut instead of round: (2 n + 8) 2^-24
  sum |q k| / sqrt(d). Of bf16 queries, elements below 2^-9 of the row's largest lose up to
  2^-10 of a unit of which that largest takes at least 224;
* the exponential's argument, in powers of 2, and the result: 2^-23 (|s| + max |s| + 40) of
  the weight, which also covers the combine's factors;
* these move a weight by delta of itself, and so the output by sum w delta |v| in the
  numerator and |o| sum w delta in the sum;
* bf16 rounds a weight to f16 for the product: half a step, 2^-11 of it, or, below 2^-21 of
  the row's largest weight, 2^-32 of that largest;
* bf16 rounds a value to f16 in a unit that the largest value of the request's prefix, or a
  candidate's of up to 2^8 times that, takes at least 224 of: 2^-25 of the unit (2^-25
  2^-117 at least);
* the sums in float32: a product of 16 keys and an addition are each off by 2^-22 of A (the
  hardware may cut), a float32 kernel's additions, one a key, by 2^-24;
* the output's rounding: 2^-8 of itself (bf16), and half of the smallest step of its type.
"""
import numpy as np


def row_keys(lay, n):
    """The prefix [p0, p1) and the candidate tokens [f0, f1) that row n sees."""
    r, c = int(lay["row_req"][n]), int(lay["row_cand"][n])
    p0, p1 = (int(lay["prefix_offset"][r + j]) for j in (0, 1))
    if c < 0:
        return r, p0, p1, 0, 0
    return r, p0, p1, int(lay["cand_row_offset"][c]) - r - 1, n - r


def cascade(lay, q, k, v, kc, vc, Hq, Hkv, rows, bf16):
    """Outputs [rows, Hq, d] in float64 and the error each may have."""
    d, g = q.shape[2], Hq // Hkv
    out, bar = (np.zeros((len(rows), Hq, d)) for _ in range(2))
    tops = {}
    for i, n in enumerate(rows):
        r, p0, p1, f0, f1 = row_keys(lay, n)
        for kh in range(Hkv):
            if (r, kh) not in tops:
                tops[r, kh] = np.abs(v[p0:p1, kh]).max()
            K = np.concatenate([k[p0:p1, kh], kc[f0:f1, kh]])
            V = np.concatenate([v[p0:p1, kh], vc[f0:f1, kh]])
            cand = int(lay["row_offset"][r]) - r, int(lay["row_offset"][r + 1]) - r - 1
            ctop = np.abs(vc[cand[0]:cand[1], kh]).max(initial=0.0)
            unit = max(tops[r, kh], min(ctop, 512.0 * tops[r, kh]), 224 * 2.0 ** -117) / 224
            Q = q[n, kh * g:(kh + 1) * g]
            s = Q @ K.T / d ** 0.5
            w = np.exp(s - s.max(1, keepdims=True))
            w /= w.sum(1, keepdims=True)
            o, A = w @ V, w @ np.abs(V)
            mag = np.abs(Q) @ np.abs(K).T / d ** 0.5
            terms = 2 * d if bf16 else d
            delta = (2 * terms + 8) * 2.0 ** -24 * mag * (17 / 16 if bf16 else 1)
            delta += 2.0 ** -23 * (np.abs(s) + np.abs(s).max(1, keepdims=True) + 40)
            if bf16:
                top = np.abs(Q).max(1, keepdims=True)
                small = np.abs(Q) < 2.0 ** -9 * top
                delta += 2.0 ** -10 / 224 * top * (small @ np.abs(K).T) / d ** 0.5
            err = (w * delta) @ np.abs(V) + (w * delta).sum(1, keepdims=True) * np.abs(o)
            if bf16:
                floor = np.minimum(w, 2.0 ** -32 * w.max(1, keepdims=True))
                err += np.maximum(2.0 ** -11 * w, floor) @ np.abs(V)
                err += 2.0 ** -25 * unit
                err += (len(K) / 16 + 40) * 2.0 ** -22 * A
            else:
                err += (len(K) + 40) * 2.0 ** -24 * A
            err *= 1.02  # the terms that two of these make together
            half, least = (2.0 ** -8, 2.0 ** -134) if bf16 else (2.0 ** -24, 2.0 ** -150)
            err += half * (np.abs(o) + err) + least
            out[i, kh * g:(kh + 1) * g], bar[i, kh * g:(kh + 1) * g] = o, err
    return out, bar


def worst(got, want, bar):
    """The largest error in units of what is allowed (NaN counts as one)."""
    with np.errstate(invalid="ignore"):
        x = np.abs(got - want) / bar
    return np.inf if np.isnan(x).any() else float(x.max())


# ---------------------------------------------------------------------------
# inputs, for the GPU tests and for those of the bar
# ---------------------------------------------------------------------------
BLOCK = 64


def columns_of_blocks(rng, prefix_len, heads, d):
    """Values that make every block count: column e holds positive values in the blocks b
    with b % d == e % blocks only, of a scale of their own, and zeros elsewhere. A block
    that is lost, doubled or halved changes a column's output by its part of few."""
    v = np.zeros((sum(prefix_len), heads, d), np.float32)
    p0 = 0
    for P in prefix_len:
        blocks = -(-P // BLOCK)
        for b in range(blocks):
            cols = [e for e in range(d) if e % min(blocks, d) == b % d]
            t = slice(p0 + b * BLOCK, p0 + min(P, (b + 1) * BLOCK))
            x = rng.uniform(1.0, 2.0, (t.stop - t.start, heads, len(cols)))
            v[t, :, cols] = x * 2.0 ** (b % 5 - 2)
        p0 += P
    return v


def gaps(rng, prefix_len, heads, d, gap, target):
    """Keys and values of one prefix whose block `target` takes all the weight of queries
    of ones while another block's values are 2^gap larger: (k, v) for q = 1."""
    total = sum(prefix_len)
    k = (rng.standard_normal((total, heads, d)) * 0.1).astype(np.float32)
    v = rng.uniform(1.0, 2.0, (total, heads, d)).astype(np.float32)
    p0 = 0
    for P in prefix_len:
        t = slice(p0 + target * BLOCK, p0 + min(P, (target + 1) * BLOCK))
        k[p0:p0 + P] -= np.float32(80.0 / d ** 0.5)   # scores about -80 ...
        k[t] += np.float32(80.0 / d ** 0.5)           # ... but about 0 there
        v[p0:p0 + BLOCK] *= np.float32(2.0 ** gap)
        p0 += P
    return k, v


def outweighed(rng, total, heads, d, q_mean, below):
    """Keys and values of one prefix whose first key's score is `below` powers of e above
    the others', for queries of positive elements of that mean; its value is zero, so
    the outputs are what the many small weights make together."""
    k = (rng.standard_normal((total, heads, d)) * 0.05).astype(np.float32)
    k[0] = below / (q_mean * d ** 0.5)
    v = rng.uniform(1.0, 2.0, (total, heads, d)).astype(np.float32)
    v[0] = 0.0
    return k, v
