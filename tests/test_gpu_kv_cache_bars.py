"""The cascade attention over the 8-bit prefix cache against bars of what each row itself
weighs (attend_bars.py): blocks of very different values, every block of long prefixes,
many small weights beside a large one, a scoring step whose LM head takes the attention's
output. And layout words that name rows, keys or tokens outside the batch."""
import numpy as np
import pytest

import attend_bars as B
import oracle as O
from gpu_common import TOL_LOGPROB
from test_gpu_kv_cache import ATTEND, JET_ERR_DEVICE, Case, _np, _torch

pytestmark = pytest.mark.gpu


def _check(c, rows=None):
    got = c.result()
    rows = list(range(len(got))) if rows is None else rows
    want, bar = B.cascade(c.ref, _np(c.q), c.kd, c.vd, _np(c.kc), _np(c.vc), c.Hq, c.Hkv, rows,
                          c.dtype == "bf16")
    assert B.worst(got[rows], want, bar) <= 1.0


GAPS = [([384], 2, "f32", 60)] + [([384], 2, "bf16", g) for g in (13, 24, 25, 31, 34, 40, 60)] + [
    (P, heads, "bf16", g) for P, heads in (([700, 300], 2), ([3000] * 3, 8)) for g in (25, 34)]


@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("P,heads,dtype,gap", GAPS)
def test_blocks_of_very_different_values(jet, P, heads, dtype, gap, d):
    # one block's values are 2^gap larger than those of the block that takes the weight,
    # in one chunk and in several, with few vectors held several times over (eight heads)
    c = Case(jet, P, [1] * len(P), [3] * len(P), dtype, 2 * heads, heads, d, seed=gap)
    rng = np.random.default_rng(gap)
    c.k, c.v = B.gaps(rng, P, heads, d, gap, target=2)
    c.q.fill_(1.0)
    c.kc.fill_(-80.0 / d ** 0.5)
    c.quantise()
    _check(c, None if len(P) < 3 else [0, 4, 8])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("P,heads,rows,d", [
    ([5000], 2, [4], 256), ([6100, 20], 8, [1, 2], 128), ([40000, 3], 2, [3, 1], 128),
    ([4100, 2500, 65], 8, [4, 9, 2], 64), ([900 + 37 * i for i in range(8)], 4, [3] * 8, 256),
    ([3000, 3500], 2, [40, 33], 64),
])
def test_every_block_counts(jet, dtype, P, heads, rows, d):
    # few blocks make a column's output, so that any one that is lost, or whose keys' or
    # values' exponent is off by one, shows (shown of this bar in test_attend_bars_host.py)
    c = Case(jet, P, [1] * len(P), rows, dtype, 4 * heads, heads, d, seed=100)
    c.v = B.columns_of_blocks(np.random.default_rng(101), P, heads, d)
    c.quantise()
    n = c.ref["N"]
    _check(c, list(range(n)) if n * c.Hq * sum(P) < 4e5 else sorted({0, 1, n // 2, n - 1}))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("case", range(len(ATTEND)))
def test_ordinary_batches(jet, dtype, case):
    P, n_cand, cand_len, dims = ATTEND[case]
    c = Case(jet, P, n_cand, cand_len, dtype, seed=case, **dims)
    n = c.ref["N"]
    _check(c, sorted(set(range(0, n, max(1, n // 6))) | {n - 1}))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("below", [9, 16])
def test_small_weights_count(jet, dtype, d, below):
    # the first key's score is far above the others' and its value zero: the outputs are
    # what the many small weights make
    c = Case(jet, [4000], [1], [3], dtype, 8, 2, d, seed=102)
    c.q = _torch(np.abs(_np(c.q)) * 0.2, dtype)
    c.k, c.v = B.outweighed(np.random.default_rng(103), 4000, 2, d, _np(c.q).mean(), below)
    c.quantise()
    _check(c)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_scores_of_a_chained_step(jet, dtype):
    # the LM head on the attention's output: scores and decisions are the oracle's of the
    # step's own outputs, which are the attention's over the cache's values
    import torch
    from paper_2609_33874_gb300.step import ScoringStep, quantize_prefix
    P, n_cand, d, Hq, V = [300, 70, 1000], [3, 2, 4], 64, 8, 1500
    cand_len = [4, 1, 2, 3, 3, 1, 2, 6, 2]
    rng = np.random.default_rng(104)
    ids = rng.integers(0, V, sum(cand_len)).tolist()
    c = Case(jet, P, n_cand, cand_len, dtype, Hq, 2, d, seed=105)
    host = jet.jet_layout_build(P, n_cand, cand_len, ids, V)
    dims = jet.make_dims(jet.DTYPE_BF16 if dtype == "bf16" else jet.DTYPE_F32, Hq=Hq, Hkv=2, d=d,
                         D=Hq * d)
    lay = O.build_layout(P, n_cand, cand_len, ids, V)
    w_lm = _torch(rng.standard_normal((V, Hq * d)) * 0.2, dtype)
    step = ScoringStep(host, dims, jet.DECIDE_ARGMAX, chain=True, kv="e4m3")
    scores = []
    for v in (c.v, c.v[::-1].copy()):
        c.v = v
        c.quantise()
        k8, v8 = quantize_prefix(step.layout, dims, _torch(c.k, dtype), _torch(v, dtype))
        step.run(dict(q=c.q, k_pre=k8, v_pre=v8, k_cand=c.kc, v_cand=c.vc), w_lm)
        torch.cuda.synchronize()
        assert jet.jet_device_status() == 0
        want, bar = B.cascade(lay, _np(c.q), c.kd, c.vd, _np(c.kc), _np(c.vc), Hq, 2,
                              range(lay["N"]), dtype == "bf16")
        assert B.worst(_np(step.o), want, bar) <= 1.0
        ell = O.token_logprobs(lay, _np(step.o).reshape(lay["N"], -1), _np(w_lm))
        s = O.candidate_scores(lay, ell)
        got = step.cand_score.cpu().numpy()
        assert np.abs(got - s).max() <= TOL_LOGPROB
        scores.append(got)
    assert np.abs(scores[0] - scores[1]).max() > 10 * TOL_LOGPROB


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 256])
@pytest.mark.parametrize("rows,right", [([0, 0, 10, 15], 2), ([0, 5, 15, 15], 0)])
def test_rows_that_name_tokens_outside_the_batch(jet, dtype, d, rows, right):
    # row offsets inside the batch whose fed tokens would start before the first one or
    # end past the last one: reported, none of them read, the true request as it was.
    # The values are far above the prefix's, so that every way of reading them is taken.
    import torch
    c = Case(jet, [70, 200, 90], [1] * 3, [5] * 3, dtype, 8, 2, d, seed=5)
    c.vc *= 1e6
    want = c.result()
    words = c.host.words.copy()
    off = (c.host.struct.row_offset - c.host.words.ctypes.data) // 4
    assert words[off:off + 4].tolist() == [0, 5, 10, 15]
    words[off:off + 4] = rows
    c.lay.words.copy_(torch.from_numpy(words))
    c.o.fill_(99.0)
    c.run()
    torch.cuda.synchronize()
    assert jet.jet_device_status() == JET_ERR_DEVICE
    assert bool((c.ws[c.need:] == 0x5A).all())
    mine = [n for n in range(c.ref["N"]) if c.ref["row_req"][n] == right]
    np.testing.assert_array_equal(_np(c.o)[mine], want[mine])


@pytest.mark.parametrize("d", [64, 256])
def test_words_whose_difference_wraps(jet, d):
    # float32: neighbouring words 2^31 - 1 and -2^31 differ by 1 in 32 bits; the requests
    # beside them are left out and reported, the third is as it was
    import torch
    c = Case(jet, [70, 200, 90], [1] * 3, [5] * 3, "f32", 8, 2, d, seed=6)
    want = c.result()
    clean = c.host.words.copy()
    for name, true in (("row_offset", [0, 5, 10, 15]), ("prefix_offset", [0, 70, 270, 360])):
        off = (getattr(c.host.struct, name) - c.host.words.ctypes.data) // 4
        words = clean.copy()
        assert words[off:off + 4].tolist() == true
        words[off:off + 2] = [2 ** 31 - 1, -2 ** 31]
        c.lay.words.copy_(torch.from_numpy(words))
        c.o.fill_(99.0)
        c.run()
        torch.cuda.synchronize()
        assert jet.jet_device_status() == JET_ERR_DEVICE
        assert bool((c.ws[c.need:] == 0x5A).all())
        np.testing.assert_array_equal(_np(c.o)[10:], want[10:])
