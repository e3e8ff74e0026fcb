"""fp64 CPU oracle of the 8-bit prefix K/V cache (e4m3 codes, a power-of-two scale
per block of 64 tokens and key/value head).

TEST INFRASTRUCTURE, like the rest of ``oracle``: only the tests use it; it shares
no code with the CUDA path and imports nothing from it.

What this module fixes (the paper keeps the prefix's keys and values and reuses them
for every candidate, Sec. 4.1, and names no format for them):

* A block is 64 consecutive tokens of one request, counted from its first; the last
  one may be shorter. Per key/value head it has one exponent X: the least integer in
  [-117, 119] with amax <= 448 2^X, amax being the largest magnitude of its finite
  elements; -117 where there is none or it is zero.
* An element's code is the E4M3 encoding (``oracle.e4m3.e4m3_encode``: nearest, ties
  to even, saturating at 448) of x 2^-X; infinities and NaN get a NaN code. Its
  value is 2^X decode(code).
* Tokens appended to a block that holds some keep the larger of its exponent and
  their own; where it grows, the codes held are encoded again at the new exponent.
* The attention over a cache is the attention over its values.
"""
from __future__ import annotations

import numpy as np

from .e4m3 import e4m3_decode, e4m3_encode

__all__ = ["BLOCK", "X_MIN", "X_MAX", "exponent", "encode", "value", "Cache"]

BLOCK = 64
X_MIN, X_MAX = -117, 119


def exponent(x) -> np.ndarray:
    """X per head of the elements x [tokens, heads, d] of one block."""
    a = np.abs(np.asarray(x, np.float64))
    top = np.where(np.isfinite(a), a, 0.0).max(axis=(0, 2), initial=0.0)
    X = np.full(top.shape, X_MIN, np.int64)
    for e in range(X_MIN, X_MAX):
        X += top > 448.0 * 2.0 ** e
    return X


def encode(x, X) -> np.ndarray:
    """Codes of x [tokens, heads, d] at the heads' exponents X [heads]."""
    x = np.asarray(x, np.float64)
    y = x * 2.0 ** (-X.astype(np.float64))[None, :, None]
    finite = np.isfinite(x)
    # the codes are those of the exact quotient: e4m3_encode takes float32, which
    # holds it unless it is below 2^-126, and then its code is a zero either way
    c = e4m3_encode(np.where(finite, np.clip(y, -448.0, 448.0), 0.0).astype(np.float32))
    return np.where(finite, c, 0x7F).astype(np.uint8)


def value(codes, X) -> np.ndarray:
    return e4m3_decode(codes) * 2.0 ** X.astype(np.float64)[None, :, None]


class Cache:
    """The codes [tokens, heads, d] of a batch's prefixes and, per request, the
    exponents [blocks, heads]; ``written`` marks the blocks that have one."""

    def __init__(self, prefix_len, heads: int, d: int):
        self.P = [int(p) for p in prefix_len]
        self.p0 = np.concatenate([[0], np.cumsum(self.P)]).astype(int)
        self.codes = np.zeros((self.p0[-1], heads, d), np.uint8)
        self.X = [np.zeros((-(-p // BLOCK), heads), np.int64) for p in self.P]
        self.written = [np.zeros(-(-p // BLOCK), bool) for p in self.P]

    def append(self, r: int, start: int, x) -> None:
        """Tokens x [n, heads, d] at positions start .. of request r."""
        end = start + len(x)
        assert 0 <= start and end <= self.P[r]
        for b in range(start // BLOCK, -(-end // BLOCK)):
            i, j = max(start, b * BLOCK), min(end, (b + 1) * BLOCK)
            if i >= j:
                continue
            new = x[i - start:j - start]
            X = exponent(new)
            at = self.p0[r]
            if i > b * BLOCK:
                held = self.X[r][b]
                X = np.maximum(X, held)
                old = slice(at + b * BLOCK, at + i)
                again = encode(value(self.codes[old], held), X)
                grown = X > held
                self.codes[old][:, grown] = again[:, grown]
            self.codes[at + i:at + j] = encode(new, X)
            self.X[r][b], self.written[r][b] = X, True

    def write(self, x) -> "Cache":
        """The whole prefix from x [tokens, heads, d]."""
        for r, p in enumerate(self.P):
            self.append(r, 0, x[self.p0[r]:self.p0[r] + p])
        return self

    def values(self) -> np.ndarray:
        out = np.zeros(self.codes.shape)
        for r, p in enumerate(self.P):
            X = np.repeat(self.X[r], BLOCK, axis=0)[:p]
            s = slice(self.p0[r], self.p0[r] + p)
            out[s] = e4m3_decode(self.codes[s]) * 2.0 ** X.astype(np.float64)[:, :, None]
        return out

    def buffer(self, background: int = 0) -> np.ndarray:
        """The cache as one byte buffer: codes padded to 256 bytes, then the bytes
        X + 127 [tokens // 64 + requests, heads], block b of request r at place
        p0 // 64 + r + b, padded too; ``background`` where nothing is written."""
        S, heads, d = self.codes.shape

        def up(n):
            return (n + 255) // 256 * 256

        nb = S // BLOCK + len(self.P)
        out = np.full(up(S * heads * d) + up(nb * heads), background, np.uint8)
        out[:S * heads * d] = self.codes.reshape(-1)
        e = out[up(S * heads * d):][:nb * heads].reshape(nb, heads)
        for r in range(len(self.P)):
            for b in range(len(self.X[r])):
                if self.written[r][b]:
                    e[self.p0[r] // BLOCK + r + b] = self.X[r][b] + 127
        return out
