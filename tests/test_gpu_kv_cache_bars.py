"""The cascade attention over the 8-bit prefix cache against bars of what each row itself
weighs (attend_bars.py): blocks of very different values, every block of long prefixes,
many small weights beside a large one."""
import numpy as np
import pytest

import attend_bars as B
from test_gpu_kv_cache import ATTEND, Case, _np, _torch

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
