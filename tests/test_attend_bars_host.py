"""The bars of attend_bars.py on the CPU: an emulation of what the kernels round passes
them, and each of the mistakes that they are there for does not - a block of the cache
lost, its values' or keys' exponent off by one, one key's value or many small weights
dropped - throughout prefixes of up to 40,000 tokens."""
import numpy as np
import pytest

import attend_bars as B
import oracle as O
from oracle import kv_e4m3 as K

HQ, HKV = 4, 2


def _bf16(x):
    import torch
    return torch.from_numpy(np.ascontiguousarray(x, np.float32)).bfloat16().double().numpy()


def _problem(P, d, k, v, q, seed=0):
    rng = np.random.default_rng(seed)
    lay = O.build_layout([P], [1], [3], [0] * 3, 2)
    kc, vc = (_bf16(rng.standard_normal((2, HKV, d))) for _ in range(2))
    cache = [K.Cache([P], HKV, d).write(_bf16(x)) for x in (k, v)]
    return lay, _bf16(q), cache[0].values(), cache[1].values(), kc, vc


def _ordinary(P, d, seed=1):
    rng = np.random.default_rng(seed)
    k = rng.standard_normal((P, HKV, d)) * np.exp(0.3 * rng.standard_normal((P, HKV, 1)))
    return k, B.columns_of_blocks(rng, [P], HKV, d), rng.standard_normal((3, HQ, d))


def _emulate(lay, q, k, v, kc, vc, rows):
    """Outputs with the kernels' roundings: queries in two e4m3 numbers, weights and values
    in f16, bf16 outputs."""
    d, g = q.shape[2], HQ // HKV
    out = np.zeros((len(rows), HQ, d))
    for i, n in enumerate(rows):
        _, p0, p1, f0, f1 = B.row_keys(lay, n)
        for h in range(HQ):
            kh = h // g
            X = K.exponent(q[n, h][None, None]).astype(np.float64)[0]
            y = q[n, h] * 2.0 ** -X
            hi = K.value(K.encode(y[None, None], np.array([0])), np.array([0]))[0, 0]
            lo = K.value(K.encode((y - hi)[None, None], np.array([0])), np.array([0]))[0, 0]
            s = np.concatenate([k[p0:p1, kh] @ ((hi + lo) * 2.0 ** X), kc[f0:f1, kh] @ q[n, h]])
            s /= d ** 0.5
            w = np.exp(s - s.max())
            V = np.concatenate([v[p0:p1, kh], vc[f0:f1, kh]])
            unit = 2.0 ** K.exponent(V[:, None])[0]
            P = (128 * w).astype(np.float16).astype(np.float64) / 128
            out[i, h] = P @ ((V / unit).astype(np.float16).astype(np.float64) * unit) / w.sum()
    return _bf16(out)


@pytest.mark.parametrize("d", [64, 256])
def test_what_the_kernels_round_passes(d):
    rows = [0, 1, 2]
    p = _problem(900, d, *_ordinary(900, d))
    want, bar = B.cascade(*p, HQ, HKV, rows, True)
    assert 0.1 < B.worst(_emulate(*p, rows), want, bar) <= 1.0
    rng = np.random.default_rng(2)
    q = np.abs(rng.standard_normal((3, HQ, d))) * 0.2
    for below in (9, 16):
        p = _problem(900, d, *B.outweighed(rng, 900, HKV, d, q.mean(), below), q)
        want, bar = B.cascade(*p, HQ, HKV, rows, True)
        assert B.worst(_emulate(*p, rows), want, bar) <= 1.0
    for gap in (13, 25, 40):
        p = _problem(400, d, *B.gaps(rng, [400], HKV, d, gap, 2), np.ones((3, HQ, d)))
        p = p[:4] + (p[4] * 0 - _bf16(80 / d ** 0.5), p[5])
        want, bar = B.cascade(*p, HQ, HKV, rows, True)
        assert B.worst(_emulate(*p, rows), want, bar) <= 1.0


@pytest.mark.parametrize("bf16", [True, False])
@pytest.mark.parametrize("P,d,blocks", [(5000, 256, range(0, 79, 6)), (6100, 128, range(0, 96, 19)),
                                        (40000, 128, (0, 1, 311, 623, 624))])
def test_a_mistake_in_any_block_is_seen(P, d, blocks, bf16):
    k, v, q = _ordinary(P, d)
    lay, q, k, v, kc, vc = _problem(P, d, k, v, q)
    rows = [0]
    want, bar = B.cascade(lay, q, k, v, kc, vc, HQ, HKV, rows, bf16)
    assert B.worst(want, want, bar) == 0.0 and B.worst(np.zeros_like(want), want, bar) > 1.0

    def seen(k2, v2):
        got = B.cascade(lay, q, k2, v2, kc, vc, HQ, HKV, rows, bf16)[0]
        return B.worst(got, want, bar) > 1.0
    for b in blocks:
        t = slice(64 * b, min(P, 64 * b + 64))
        for x, f in ((v, 0.0), (v, 2.0), (v, 0.5), (k, 2.0), (k, 0.5)):
            held = x[t, 1].copy()
            x[t, 1] *= f
            assert seen(k, v), (b, x is v, f)
            x[t, 1] = held
    # the last key of all left out of the product, its weight in the sum
    held = v[P - 1].copy()
    v[P - 1] = 0.0
    assert seen(k, v)
    v[P - 1] = held


@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("below", [9, 16])
def test_dropped_small_weights_are_seen(d, below):
    rng = np.random.default_rng(3)
    q = np.abs(rng.standard_normal((3, HQ, d))) * 0.2
    p = _problem(4000, d, *B.outweighed(rng, 4000, HKV, d, q.mean(), below), q)
    want, bar = B.cascade(*p, HQ, HKV, [0], True)
    # every second key's weight, or one in sixteen, lost
    for step in (2, 16):
        v = p[3].copy()
        v[1::step] = 0.0
        got = B.cascade(p[0], p[1], p[2], v, *p[4:], HQ, HKV, [0], True)[0]
        assert B.worst(got, want, bar) > 1.0
