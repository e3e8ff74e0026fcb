"""The cascade attention over the 8-bit prefix cache against bars of what each row itself
weighs (attend_bars.py): blocks of very different values, every block of long prefixes,
many small weights beside a large one."""
import numpy as np
import pytest

import attend_bars as B
from test_gpu_kv_cache import JET_ERR_DEVICE, Case, _np

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
