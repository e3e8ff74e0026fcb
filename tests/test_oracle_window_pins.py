"""Pins of the window and rotation oracle, by hand and by what must hold, and of the bars
that the GPU tests use (tests/window_bars.py) against it. CPU only."""
import math

import numpy as np
import pytest

import jet_synth
import oracle as O
import window_bars as B
from oracle import window as W


def test_seen_by_hand():
    assert W.seen(0, 1, 0) == [0]
    assert W.seen(5, 1, 0) == [5]
    assert W.seen(5, 3, 0) == [3, 4, 5]
    assert W.seen(5, 3, 2) == [0, 1, 3, 4, 5]
    assert W.seen(5, 3, 4) == [0, 1, 2, 3, 4, 5]   # the first ones reach into the window
    assert W.seen(2, 10, 1) == [0, 1, 2]
    assert W.seen(5, 3, 100) == [0, 1, 2, 3, 4, 5]


def test_rotation_by_hand():
    x = np.array([[[3.0, 4.0, 0.0, 0.0]]])
    f = np.array([math.pi / 2, 0.0])
    out = W.rotate(x, [1], 4, "pairs", f, norm=False)
    np.testing.assert_allclose(out[0, 0], [-4.0, 3.0, 0.0, 0.0], atol=1e-15)
    out = W.rotate(x, [1], 4, "halves", f, norm=False)   # (3, 0) a quarter turn, (4, 0) none
    np.testing.assert_allclose(out[0, 0], [0.0, 4.0, 3.0, 0.0], atol=1e-15)
    out = W.rotate(x, [7], 0, "halves", [], gain=np.full(4, 2.0), eps=0.0)
    np.testing.assert_allclose(out[0, 0], np.array([3.0, 4.0, 0, 0]) / 2.5 * 2.0, atol=1e-15)


@pytest.mark.parametrize("style", ["halves", "pairs"])
def test_rotated_scores_depend_on_the_distance(style):
    rng = np.random.default_rng(3)
    q, k = rng.normal(size=(2, 1, 1, 16))
    f = W.frequencies(16, 1e4)
    dots = []
    for a, b in ((5, 2), (105, 102), (3, 0)):
        x, y = (W.rotate(t, [p], 16, style, f) for t, p in ((q, a), (k, b)))
        dots.append(float((x * y).sum()))
    np.testing.assert_allclose(dots, dots[0], rtol=1e-12)
    # and a rotation keeps the length
    np.testing.assert_allclose(np.linalg.norm(W.rotate(q, [9], 16, style, f, norm=False)),
                               np.linalg.norm(q), rtol=1e-13)


def _problem(**over):
    import dataclasses
    w = dataclasses.replace(jet_synth.WORKLOADS["tiny"], Hq=4, Hkv=2, d=64, **over)
    P, C = [1, 5, 40], [1, 2, 3]
    m = [3, 1, 4, 2, 5, 1]
    p = jet_synth.custom_problem(w, P, C, m, [0] * sum(m), seed=5)
    return p, O.build_layout(P, C, m, [0] * sum(m), w.V)


@pytest.mark.parametrize("sinks", [0, 3, 100])
def test_wide_window_is_the_plain_attention(sinks):
    p, lay = _problem()
    args = [p.f32(n) for n in ("q", "k_pre", "v_pre", "k_cand", "v_cand")]
    rows = list(range(lay["N"]))
    ref = O.cascade_attention(lay, *args, 4, 2)
    np.testing.assert_allclose(W.window_cascade(lay, *args, 4, 2, 1000, sinks, rows), ref,
                               atol=1e-13)
    # as are enough first tokens
    np.testing.assert_allclose(W.window_cascade(lay, *args, 4, 2, 1, 1000, rows), ref, atol=1e-13)
    qkv = [p.f32(n) for n in ("q_pre", "k_pre", "v_pre")]
    rows = list(range(46))
    np.testing.assert_allclose(W.window_prefill(p.prefix_len, *qkv, 4, 2, 1000, sinks, rows),
                               O.prefill_attention(p.prefix_len, *qkv, 4, 2), atol=1e-13)


def test_window_of_one_gives_the_own_value():
    p, lay = _problem()
    args = [p.f32(n) for n in ("q", "k_pre", "v_pre", "k_cand", "v_cand")]
    out = W.window_cascade(lay, *args, 4, 2, 1, 0, list(range(lay["N"])))
    for n in range(lay["N"]):
        r = int(lay["row_req"][n])
        v = (args[2][int(lay["prefix_offset"][r + 1]) - 1] if lay["row_cand"][n] < 0
             else args[4][n - r - 1])
        np.testing.assert_allclose(out[n], np.repeat(v, 2, 0), atol=1e-13)


@pytest.mark.parametrize("window,sinks", [(1, 0), (2, 1), (4, 7), (16, 3), (33, 0), (9, 41)])
def test_bars_compute_what_the_oracle_does(window, sinks):
    p, lay = _problem()
    args = [p.f32(n) for n in ("q", "k_pre", "v_pre", "k_cand", "v_cand")]
    for rows, o, bar in B.cascade(lay, *args, window, sinks, False).values():
        want = W.window_cascade(lay, *args, 4, 2, window, sinks, list(rows))
        np.testing.assert_allclose(o, want, atol=1e-12)
        assert (bar > 0).all() and bar.max() < 1e-3
    qkv = [p.f32(n) for n in ("q_pre", "k_pre", "v_pre")]
    for rows, o, _ in B.prefill(p.prefix_len, *qkv, window, sinks).values():
        np.testing.assert_allclose(
            o, W.window_prefill(p.prefix_len, *qkv, 4, 2, window, sinks, list(rows)), atol=1e-12)


@pytest.mark.parametrize("style", ["halves", "pairs"])
def test_rotation_bars_compute_what_the_oracle_does(style):
    rng = np.random.default_rng(0)
    x, gain, pos = rng.normal(size=(5, 3, 64)), rng.normal(size=64), [0, 1, 77, 1 << 20, -3]
    for rot in (0, 8, 40, 64):
        f = W.frequencies(rot, 1e5)
        o, _ = B.rotation(x, pos, rot, style, f, gain, 1e-6, True, False)
        np.testing.assert_allclose(o, W.rotate(x, pos, rot, style, f, gain), atol=1e-9)
