"""Attention under a window where outputs come out NaN or infinite and are computed again from what
their rows see alone: in the step's chunks, beside keys that a row does not see, and under windows
long enough for the second computation to take longer than any wait may."""
import numpy as np
import pytest

import window_bars as B
from test_gpu_timeout import JET_OK
from test_gpu_window import Prefill, Step, _np, _some

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def cuda(jet):
    import torch
    if not torch.cuda.is_available():
        pytest.fail("CUDA device required for -m gpu tests")
    yield jet
    jet.jet_set_wait_budget_ns(0)


@pytest.mark.parametrize("d,heads", [(64, (8, 8)), (128, (16, 2)), (256, (16, 2))])
def test_outputs_of_chunks_are_stored_once(cuda, d, heads):
    """Every row of a long window in chunks is computed again, as a key beside the first tokens is
    NaN: each output is the second computation's, call after call."""
    import torch
    P, window, sinks = 20000, 6000, 20
    s = Step(cuda, [P], [3], [5, 3, 9], *heads, d, True, seed=21)
    s.v[25] = s.k[25] = float("nan")   # seen by no row, loaded with the first ones
    ws = s.ws(window, sinks)
    s.run(window, sinks, ws=ws)
    s.check(window, sinks)
    first = s.o.clone()
    for _ in range(10):
        s.o.fill_(7.0)
        s.run(window, sinks, ws=ws)
        assert torch.equal(s.o, first)


def test_odd_rows_of_a_lying_candidate_are_written(cuda):
    """A candidate whose first row the layout puts past the row in question: no own tokens are
    read, and what the chunks gave is stored."""
    import torch
    s = Step(cuda, [20000], [2], [5, 3], 16, 2, 128, True, seed=29)
    s.v[25] = float("nan")
    s.run(6000, 20)
    first = s.o.clone()
    words = s.dev.words.clone()
    words[(s.dev.struct.cand_row_offset - s.dev.words.data_ptr()) // 4 + 1] = 1 << 30
    s.o.fill_(7.0)
    cuda.jet_prefix_attend_window(cuda.DeviceLayout(s.hl.sizes, words), s.dims, 6000, 20, s.q, s.k,
                                  s.v, s.kc, s.vc, s.o, s.ws(6000, 20))
    torch.cuda.synchronize()
    cuda.jet_device_status()
    of = torch.from_numpy(s.lay["row_cand"] == 1).cuda()
    assert (s.o[~of] == first[~of]).all() and not (s.o[of] == 7.0).any()


def _within(cuda, budget_ns, call):
    old = cuda.jet_set_wait_budget_ns(budget_ns)
    try:
        call()
        return cuda.jet_device_status()
    finally:
        cuda.jet_set_wait_budget_ns(old)


def _check_with_nan(got, rows, want, bar, sees, col, heads):
    """NaN in column `col` of `heads` where a row sees the key that has it; all else at the bars."""
    nan = np.zeros(want.shape, bool)
    nan[np.ix_(sees, heads, [col])] = True
    assert np.isnan(got[rows][nan]).all()
    assert B.worst(np.where(nan, 0.0, got[rows]), np.where(nan, 0.0, want), bar) <= 1.0


@pytest.mark.parametrize("d,heads", [(64, (8, 2)), (128, (8, 2)), (256, (8, 1))])
def test_prefill_of_a_long_window_whose_every_row_sees_a_nan(cuda, d, heads):
    # a first token with one NaN, under a budget far below what 32 vectors take key by key
    P, window, sinks = [6000, 40], 5000, 1
    p = Prefill(cuda, P, *heads, d, seed=22)
    ws = p.ws(window, sinks)
    p.run(window, sinks, ws=ws)
    p.v[0, 0, 3] = float("nan")
    p.o.fill_(7.0)
    assert _within(cuda, 5_000_000, lambda: cuda.jet_prefill_attend_window(
        p.dev, p.dims, window, sinks, p.q, p.k, p.v, p.o, ws)) == JET_OK
    got = _np(p.o)
    some = _some(P, np.random.default_rng(1), 60)
    for r, (rows, want, bar) in B.prefill(P, *(_np(x) for x in (p.q, p.k, p.v)), window, sinks,
                                          rows_of=some).items():
        sees = np.full(len(rows), r == 0)
        _check_with_nan(got, rows, want, bar, sees, 3, np.arange(heads[0] // heads[1]))
    assert np.isnan(got[:6000, :heads[0] // heads[1], 3]).all()
    assert np.isfinite(np.delete(got, 3, axis=-1)).all()


@pytest.mark.parametrize("d", [64, 128, 256])
def test_step_of_long_windows_whose_every_row_sees_a_nan(cuda, d):
    R, P, window, sinks, Hq, Hkv = 160, 5200, 5000, 2, 32, 2
    s = Step(cuda, [P] * R, [1] * R, [2] * R, Hq, Hkv, d, True, seed=23)
    ws = s.ws(window, sinks)
    s.run(window, sinks, ws=ws)
    s.v.view(R, P, Hkv, d)[:, 1, 1, 5] = float("nan")
    s.o.fill_(7.0)
    assert _within(cuda, 5_000_000, lambda: cuda.jet_prefix_attend_window(
        s.dev, s.dims, window, sinks, s.q, s.k, s.v, s.kc, s.vc, s.o, ws)) == JET_OK
    got = _np(s.o)
    at = [0, 1, 77, R - 1]
    lay, few = s.lay, [int(x) for x in s.lay["prefix_offset"]]
    k, v = (np.zeros((R * P, Hkv, d)) for _ in range(2))
    for r in at:
        for x, y in ((k, s.k), (v, s.v)):
            x[few[r]:few[r + 1]] = _np(y[few[r]:few[r + 1]])
    for r, (rows, want, bar) in B.cascade(lay, _np(s.q), k, v, _np(s.kc), _np(s.vc), window, sinks,
                                          True, at).items():
        _check_with_nan(got, rows, want, bar, np.ones(len(rows), bool), 5, np.arange(16, 32))
    assert np.isnan(got[:, 16:, 5]).all() and np.isfinite(np.delete(got, 5, axis=-1)).all()


def test_few_odd_outputs_among_many_items(cuda):
    """More items a CTA than one, some with rows that see a NaN, some with rows beside it."""
    rng = np.random.default_rng(24)
    window, sinks = 30, 2
    P = [int(x) for x in rng.integers(1, 300, size=400)]
    p = Prefill(cuda, P, 8, 2, 64, seed=24)
    s = Step(cuda, P, [2] * 400, [1 + int(x) for x in rng.integers(0, 5, size=800)], 8, 2, 64, True,
             seed=24)
    off = np.concatenate([[0], np.cumsum(P)])
    hit = {int(r): int(rng.integers(0, P[r])) for r in rng.choice(400, size=40, replace=False)}
    for r, j in hit.items():
        p.v[off[r] + j, 0, 3] = s.v[off[r] + j, 0, 3] = float("nan")
    p.run(window, sinks)
    got = _np(p.o)
    for r, (rows, want, bar) in B.prefill(P, *(_np(x) for x in (p.q, p.k, p.v)), window,
                                          sinks).items():
        sees = (B.in_window(rows - off[r], [hit[r]], window, sinks)[:, 0] if r in hit else
                np.zeros(len(rows), bool))
        _check_with_nan(got, rows, want, bar, sees, 3, np.arange(4))
    s.run(window, sinks)
    got, lay = _np(s.o), s.lay
    for r, (rows, want, bar) in B.cascade(lay, *(_np(x) for x in (s.q, s.k, s.v, s.kc, s.vc)),
                                          window, sinks, True).items():
        pos = P[r] - 1 + np.where(lay["row_cand"][rows] >= 0, lay["row_pos"][rows], 0)
        sees = (B.in_window(pos, [hit[r]], window, sinks)[:, 0] if r in hit else
                np.zeros(len(rows), bool))
        _check_with_nan(got, rows, want, bar, sees, 3, np.arange(4))


@pytest.mark.parametrize("d,heads", [(64, (8, 2)), (128, (8, 8)), (256, (16, 2))])
def test_float32_values_near_the_largest_float(cuda, d, heads):
    """Means whose sums pass the largest float: in a prefix, across chunks, among own tokens, with
    signs that would cancel as infinities. The second computation keeps a mean, a key's step of
    which rounds up to six times where the sums' rounds once: 5 n 2^-24 A beside the bars."""
    P = [300, 41, 9000]
    s = Step(cuda, P, [2, 1, 1], [3, 5, 30, 70], *heads, d, False, seed=25)
    for x in (s.v, s.vc):
        x.copy_(x.clamp(-3, 3) * 1e38)
    s.v[300:341] = 5e37                       # ten of them leave float32
    clean = s.v.clone()
    for window, sinks in ((60, 3), (8000, 0), (1000, 40)):
        s.v.copy_(clean)
        s.run(window, sinks)
        got = _np(s.o)
        assert np.isfinite(got).all()
        for r, (rows, want, bar) in B.cascade(s.lay, *(_np(x) for x in (
                s.q, s.k, s.v, s.kc, s.vc)), window, sinks, False).items():
            n = min(P[r] + 70, window + 70 + sinks)
            bar = bar + 5 * n * 2.0 ** -24 * 3e38
            assert B.worst(got[rows], want, bar) <= 1.0, (r, window, sinks)
            if r == 1:
                row = rows[0]                 # the shared row sees equal values only
                assert np.abs(got[row] / 5e37 - 1).max() <= (6 * n + 40) * 2.0 ** -24
        # a NaN that a row does not see stays away, and one that it sees comes out
        s.v[100] = float("nan")
        s.run(window, sinks)
        got = _np(s.o)
        sees = window >= 200
        assert np.isnan(got[0]).all() if sees else np.isfinite(got[0]).all()


def test_float32_outputs_of_ordinary_rows_are_their_sums(cuda):
    """Rows beside one whose sums overflow keep their bits."""
    s = Step(cuda, [100, 100], [1, 1], [2, 2], 4, 2, 64, False, seed=26)
    s.run(50, 2)
    first = _np(s.o)
    s.v[100:] = 3e38
    s.run(50, 2)
    assert (_np(s.o)[:2] == first[:2]).all() and np.isfinite(_np(s.o)).all()


@pytest.mark.parametrize("bf16", [True, False])
@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_a_seen_key_of_weight_zero_shows_its_values(cuda, bad, bf16):
    """A score of minus infinity weighs 0, and 0 times a NaN or an infinity is NaN: in a row that
    sees the key, in that column, whether the row is computed once or twice."""
    P, window, sinks = 90, 40, 2
    s = Step(cuda, [P], [1], [6], 4, 2, 64, bf16, seed=27)
    s.q.abs_().add_(0.125)
    s.k[70, 1] = s.kc[2, 1] = float("-inf")
    s.v[70, 1, 7] = s.vc[2, 1, 9] = bad
    s.run(window, sinks)
    got = _np(s.o)
    assert np.isnan(got[:, 2:, 7]).all()                       # every row sees key 70
    assert np.isnan(got[3:, 2:, 9]).all() and np.isfinite(got[:3, 2:, 9]).all()
    assert np.isfinite(np.delete(got, [7, 9], axis=-1)).all()
    if not bf16:
        return
    p = Prefill(cuda, [P], 4, 2, 64, seed=27)
    p.q.abs_().add_(0.125)
    p.k[70, 1], p.v[70, 1, 7] = float("-inf"), bad
    p.run(window, sinks)
    got = _np(p.o)
    assert np.isnan(got[70:, 2:, 7]).all()
    got[70:, 2:, 7] = 0.0
    assert np.isfinite(got).all()


@pytest.mark.parametrize("d,heads", [(64, (16, 2)), (128, (8, 8)), (256, (16, 2))])
@pytest.mark.parametrize("window,sinks", [(1000, 4), (2048, 0)])
def test_prefill_wide_windows_end_where_they_should(cuda, d, heads, window, sinks):
    """A key that is NaN, seen by the last row of whose window it is part and by none after, in
    windows of many tiles, whose middle ones are not masked: a key too few or too many there is
    less than the bars of the weights."""
    P = [3500]
    p = Prefill(cuda, P, *heads, d, seed=28)
    rng = np.random.default_rng(28)
    for j in (sinks, 127, 128, 611, 640, 1000, 1333):
        k = p.k[j].clone()
        p.k[j] = float("nan")
        p.run(window, sinks)
        got = np.isnan(_np(p.o))
        sees = B.in_window(np.arange(P[0]), [j], window, sinks)[:, 0]
        assert got[sees].all() and not got[~sees].any(), j
        rows = np.unique(np.clip([0, j - 1, j + window, j + window + 1, *rng.integers(0, 3500, 6)],
                                 0, P[0] - 1))
        rows = rows[~sees[rows]]
        p.check(window, sinks, rows_of=[rows])
        p.k[j] = k
