"""GPU parity of the norm and rotation of queries and keys against 64 bits, element by
element at derived bars (tests/window_bars.py): types, head sizes and layouts, both pair
styles, partial rotations, far and negative positions, a batch's prefixes and a step's rows,
in place, captured, on another stream, with a layout that lies."""
import numpy as np
import pytest

import oracle as O
import window_bars as B
from oracle import window as W

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def cuda(jet):
    import torch
    if not torch.cuda.is_available():
        pytest.fail("CUDA device required for -m gpu tests")
    return jet


def _tensor(rng, shape, bf16, scale=1.0):
    import torch
    x = torch.from_numpy((rng.normal(size=shape) * scale).astype(np.float32))
    return (x.bfloat16() if bf16 else x).cuda()


def _np(x):
    return x.double().cpu().numpy()


class Case:
    def __init__(self, jet, nq, nk, Hq, Hkv, d, bf16, seed=0, spread=True):
        rng = np.random.default_rng(seed)
        self.dims = jet.make_dims(jet.DTYPE_BF16 if bf16 else jet.DTYPE_F32, Hq=Hq, Hkv=Hkv, d=d)
        self.bf16, self.d = bf16, d
        self.q, self.k = _tensor(rng, (nq, Hq, d), bf16), _tensor(rng, (nk, Hkv, d), bf16)
        if spread:  # tokens of very different size
            for x in (self.q, self.k):
                x.mul_(_tensor(rng, (x.shape[0], 1, 1), bf16, 2.0).exp_())
        self.gq, self.gk = (_tensor(rng, (d,), bf16) for _ in range(2))
        self.qo, self.ko = self.q.new_full(self.q.shape, 7.0), self.k.new_full(self.k.shape, 7.0)

    def check(self, rope_args, pos_q, pos_k, q=None, k=None):
        a = dict(dict(style="halves", theta=1e4, freq=None, norm=True, eps=1e-6, gain=True),
                 **rope_args)
        f = W.frequencies(a["rot"], a["theta"]) if a["freq"] is None else a["freq"]
        for x, g, pos, got in ((self.q if q is None else q, self.gq, pos_q, self.qo),
                               (self.k if k is None else k, self.gk, pos_k, self.ko)):
            want, bar = B.rotation(_np(x), pos, a["rot"], a["style"], f,
                                   _np(g) if a["gain"] else None, a["eps"], a["norm"], self.bf16)
            assert B.worst(_np(got), want, bar) <= 1.0


def _sync(cuda):
    import torch
    torch.cuda.synchronize()
    assert cuda.jet_device_status() == 0


def _rope(jet, rot, style="halves", theta=1e4, freq=None, norm=True, eps=1e-6, gain=True):
    return jet.make_rope(rot, style=style, theta=theta, freq=freq, norm=norm, eps=eps)


HEADS = [(8, 2), (7, 1), (24, 4), (3, 3), (1, 1)]


@pytest.mark.parametrize("bf16", [True, False])
@pytest.mark.parametrize("style", ["halves", "pairs"])
@pytest.mark.parametrize("d,rot", [(64, 64), (64, 8), (64, 56), (128, 128), (128, 96), (128, 0),
                                   (256, 256), (256, 64), (256, 232)])
def test_given_positions(cuda, d, rot, style, bf16):
    import torch
    for i, (Hq, Hkv) in enumerate(HEADS):
        n = (1, 5, 3, 17, 33)[i]
        c = Case(cuda, n, n, Hq, Hkv, d, bf16, seed=i)
        rng = np.random.default_rng(i + 9)
        pos = rng.integers(-5, 1 << 24, size=n)
        pos[0] = 0
        a = dict(rot=rot, style=style, theta=1e6)
        cuda.jet_norm_rotate(c.dims, _rope(cuda, **a), torch.tensor(pos, dtype=torch.int32).cuda(),
                             c.q, c.k, c.gq, c.gk, c.qo, c.ko)
        _sync(cuda)
        c.check(a, pos, pos)


@pytest.mark.parametrize("bf16", [True, False])
@pytest.mark.parametrize("a", [dict(rot=64, norm=False), dict(rot=64, gain=False),
                               dict(rot=64, eps=0.5), dict(rot=16, freq=[6.0, -1.0, 0.0, 1e-9,
                                                                         40.0, 0.5, 3.1, -0.2])])
def test_forms_of_the_norm_and_frequencies(cuda, a, bf16):
    import torch
    c = Case(cuda, 40, 40, 8, 2, 64, bf16)
    pos = np.arange(40) * 50 - 100
    gains = (c.gq, c.gk) if a.get("gain", True) else (None, None)
    cuda.jet_norm_rotate(c.dims, _rope(cuda, **a), torch.tensor(pos, dtype=torch.int32).cuda(),
                         c.q, c.k, *gains, c.qo, c.ko)
    _sync(cuda)
    c.check(a, pos, pos)


@pytest.mark.parametrize("bf16", [True, False])
@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("eps", [0.0, 2.0 ** -136, 2.0 ** -116, 2.0 ** -20])
def test_heads_whose_squares_leave_float32(cuda, eps, d, bf16):
    import torch
    n, Hq, Hkv = 40, 6, 2
    c = Case(cuda, n, n, Hq, Hkv, d, bf16, spread=False)
    sizes = [-113, -66, 0, 60, 66, 125] + ([-126] if eps == 0.0 else [])
    for i, x in enumerate((c.q, c.k)):  # a size for each head, and heads of zeros
        e = torch.tensor(np.random.default_rng(i).choice(sizes, size=(n, x.shape[1], 1))).cuda()
        x.copy_(torch.ldexp(x.double(), e).to(x.dtype))
        x[3, 0] = 0.0
        x[7] = 0.0
    pos = np.arange(n) * 11
    a = dict(rot=64, eps=eps)
    cuda.jet_norm_rotate(c.dims, _rope(cuda, **a), torch.tensor(pos, dtype=torch.int32).cuda(),
                         c.q, c.k, c.gq, c.gk, c.qo, c.ko)
    _sync(cuda)
    for x, y, g in ((c.q, c.qo, c.gq), (c.k, c.ko, c.gk)):
        assert (y[3, 0] == 0.0).all() and (y[7] == 0.0).all()  # zeros stay, without eps too
        some = (x != 0).any(-1).cpu().numpy()
        one = x.clone()
        one[~torch.tensor(some)] = 1.0
        want, bar = B.rotation(_np(one), pos, 64, "halves", W.frequencies(64, 1e4), _np(g), eps,
                               True, bf16)
        assert B.worst(_np(y)[some], want[some], bar[some]) <= 1.0


@pytest.mark.parametrize("bf16", [True, False])
def test_infinite_and_nan_elements_stay_in_their_heads(cuda, bf16):
    import torch
    n = 5
    c = Case(cuda, n, n, 4, 2, 64, bf16, spread=False)
    c.q[1, 2, 3] = float("inf")
    c.q[2, 0, 9] = float("nan")
    pos = np.arange(n) * 11
    cuda.jet_norm_rotate(c.dims, _rope(cuda, 64), torch.tensor(pos, dtype=torch.int32).cuda(),
                         c.q, c.k, c.gq, c.gk, c.qo, c.ko)
    _sync(cuda)
    got = _np(c.qo)
    pair = [3, 35]  # x / infinity: zeros, and NaN where x is infinite and in its pair
    assert np.isnan(got[1, 2, pair]).all() and (np.delete(got[1, 2], pair) == 0.0).all()
    assert np.isnan(got[2, 0]).all()
    keep = np.ones((n, 4), bool)
    keep[1, 2] = keep[2, 0] = False
    want, bar = B.rotation(np.where(keep[..., None], _np(c.q), 1.0), pos, 64, "halves",
                           W.frequencies(64, 1e4), _np(c.gq), 1e-6, True, bf16)
    assert B.worst(got[keep], want[keep], bar[keep]) <= 1.0


def test_the_farthest_positions(cuda):
    # position 2^31 - 1 (and its negative) at frequencies with few binary digits, so that the
    # angle in 64 bits is exact: f = 2 pi m / 2^20 is not, but f = m / 2^21 times p < 2^31 is
    import torch
    c = Case(cuda, 6, 6, 4, 4, 64, False)
    freq = np.array([m / 2.0 ** 21 for m in (1, 3, 1 << 21, (1 << 21) - 1, 12345, 2, 700001, 0)])
    pos = np.array([2 ** 31 - 1, -2 ** 31, 2 ** 31 - 2, -(2 ** 31) + 1, 2 ** 30 + 1, 1])
    a = dict(rot=16, freq=freq)
    cuda.jet_norm_rotate(c.dims, _rope(cuda, **a), torch.tensor(pos, dtype=torch.int32).cuda(),
                         c.q, c.k, c.gq, c.gk, c.qo, c.ko)
    _sync(cuda)
    # f / (2 pi) keeps 53 digits: 2^31 f 2^-53 radians of an angle, within the 3 2^-24 of the bar
    c.check(a, pos, pos)


def _layout(cuda, P, m, n_cand):
    hl = cuda.jet_layout_build(P, n_cand, m, [0] * sum(m), 4)
    lay = O.build_layout(P, n_cand, m, [0] * sum(m), 4)
    return hl, lay, hl.to_device("cuda")


@pytest.mark.parametrize("bf16", [True, False])
@pytest.mark.parametrize("P", [[1], [3, 1, 200, 65], list(range(1, 71)), [2] * 1100])
def test_prefixes(cuda, P, bf16):
    R, S = len(P), sum(P)
    _, _, dev = _layout(cuda, P, [1] * R, [1] * R)
    pos = np.concatenate([np.arange(x) for x in P])
    for d, Hq, Hkv, a in ((64, 8, 2, dict(rot=64)), (256, 3, 1, dict(rot=64, style="pairs"))):
        c = Case(cuda, S, S, Hq, Hkv, d, bf16)
        cuda.jet_norm_rotate_prefix(dev, c.dims, _rope(cuda, **a), c.q, c.k, c.gq, c.gk, c.qo, c.ko)
        _sync(cuda)
        c.check(a, pos, pos)


def test_many_tokens_in_one_pass(cuda):
    # enough tokens that a block takes several, a ragged last block among them
    P = [4001, 1, 999, 7]
    _, _, dev = _layout(cuda, P, [1] * 4, [1] * 4)
    pos = np.concatenate([np.arange(x) for x in P])
    for d, H in ((64, 8), (128, 5), (256, 2)):
        c = Case(cuda, sum(P), sum(P), H, 1, d, True)
        cuda.jet_norm_rotate_prefix(dev, c.dims, _rope(cuda, rot=d), c.q, c.k, c.gq, c.gk, c.qo,
                                    c.ko)
        _sync(cuda)
        c.check(dict(rot=d), pos, pos)


@pytest.mark.parametrize("bf16", [True, False])
def test_rows_of_a_step(cuda, bf16):
    P, n_cand, m = [5, 1, 90], [2, 1, 3], [3, 1, 1, 4, 2, 9]
    _, lay, dev = _layout(cuda, P, m, n_cand)
    pos = np.array([W.row_position(lay, n) for n in range(lay["N"])])
    fed = lay["row_cand"] >= 0
    for d, rot in ((64, 64), (128, 64), (256, 256)):
        c = Case(cuda, int(lay["N"]), int(fed.sum()), 8, 2, d, bf16)
        cuda.jet_norm_rotate_rows(dev, c.dims, _rope(cuda, rot=rot), c.q, c.k, c.gq, c.gk, c.qo,
                                  c.ko)
        _sync(cuda)
        c.check(dict(rot=rot), pos, pos[fed])


def test_rows_without_fed_tokens(cuda):
    P, m = [5, 9], [1, 1]
    _, lay, dev = _layout(cuda, P, m, [1, 1])
    c = Case(cuda, 2, 0, 8, 2, 64, True)
    cuda.jet_norm_rotate_rows(dev, c.dims, _rope(cuda, rot=64), c.q, c.k, c.gq, c.gk, c.qo, c.ko)
    _sync(cuda)
    c.check(dict(rot=64), [4, 8], [])


def test_only_one_of_the_two_and_in_place(cuda):
    import torch
    c = Case(cuda, 50, 50, 8, 2, 128, True)
    pos = torch.arange(50, dtype=torch.int32).cuda()
    rope = _rope(cuda, rot=128)
    cuda.jet_norm_rotate(c.dims, rope, pos, c.q, c.k, c.gq, c.gk, c.qo, c.ko)
    both = c.qo.clone(), c.ko.clone()
    for x, y in ((c.q, both[0]), (c.k, both[1])):
        only = x.clone()
        qk = (only, None) if x is c.q else (None, only)
        gains = (c.gq, None) if x is c.q else (None, c.gk)
        cuda.jet_norm_rotate(c.dims, rope, pos, *qk, *gains, *qk)
        torch.cuda.synchronize()
        assert torch.equal(only, y)
    _sync(cuda)


def test_nan_and_infinity_stay_in_their_head(cuda):
    import torch
    c = Case(cuda, 9, 9, 8, 2, 64, True, spread=False)
    pos = torch.arange(9, dtype=torch.int32).cuda()
    rope = _rope(cuda, rot=64)
    cuda.jet_norm_rotate(c.dims, rope, pos, c.q, c.k, c.gq, c.gk, c.qo, c.ko)
    want = c.qo.clone(), c.ko.clone()
    c.q[3, 5, 7], c.k[2, 1, 0] = float("nan"), float("inf")
    cuda.jet_norm_rotate(c.dims, rope, pos, c.q, c.k, c.gq, c.gk, c.qo, c.ko)
    _sync(cuda)
    assert not torch.isfinite(c.qo[3, 5]).any() and not torch.isfinite(c.ko[2, 1]).all()
    want[0][3, 5], want[1][2, 1] = c.qo[3, 5], c.ko[2, 1]
    for got, x in zip((c.qo, c.ko), want):
        fine = torch.isfinite(x)
        assert torch.equal(got[fine], x[fine]) and int((~fine).sum()) <= 64


def test_captured_and_on_another_stream(cuda):
    import torch
    P = [30, 500]
    _, _, dev = _layout(cuda, P, [1, 1], [1, 1])
    c = Case(cuda, 530, 530, 8, 2, 64, True)
    rope, pos = _rope(cuda, rot=64), np.concatenate([np.arange(x) for x in P])
    s, g = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        cuda.jet_norm_rotate_prefix(dev, c.dims, rope, c.q, c.k, c.gq, c.gk, c.qo, c.ko)
    torch.cuda.synchronize()
    c.check(dict(rot=64), pos, pos)
    with torch.cuda.graph(g):
        cuda.jet_norm_rotate_prefix(dev, c.dims, rope, c.q, c.k, c.gq, c.gk, c.qo, c.ko)
    c.q.copy_(c.q.flip(0))     # the graph reads the tensors, not a copy, and its own rope
    rope.rot = 0
    g.replay()
    _sync(cuda)
    c.check(dict(rot=64), pos, pos)


def test_layouts_that_lie_are_reported(cuda):
    import torch
    P = [30, 40, 50]
    hl, lay, dev = _layout(cuda, P, [2, 2, 2], [1, 1, 1])
    c = Case(cuda, 120, 120, 8, 2, 64, True)
    rope = _rope(cuda, rot=64)
    off = (dev.struct.prefix_offset - dev.words.data_ptr()) // 4
    for bad in (-3, 1 << 30, 200):
        words = dev.words.clone()
        words[off + 1] = bad
        lied = cuda.DeviceLayout(hl.sizes, words)
        for call in (cuda.jet_norm_rotate_prefix, cuda.jet_norm_rotate_rows):
            call(lied, c.dims, rope, c.q, c.k, c.gq, c.gk, c.qo, c.ko)
            torch.cuda.synchronize()
            assert cuda.jet_device_status() == cuda_status(cuda, "JET_ERR_DEVICE")
    for name, bad in (("row_req", 3), ("row_req", -1), ("row_pos", -1), ("row_pos", 1 << 30)):
        words = dev.words.clone()
        words[(getattr(dev.struct, name) - dev.words.data_ptr()) // 4 + 1] = bad
        cuda.jet_norm_rotate_rows(cuda.DeviceLayout(hl.sizes, words), c.dims, rope, c.q, c.k, c.gq,
                                  c.gk, c.qo, c.ko)
        torch.cuda.synchronize()
        assert cuda.jet_device_status() == cuda_status(cuda, "JET_ERR_DEVICE")


def cuda_status(jet, name):
    return {v: k for k, v in jet.STATUS_NAMES.items()}[name]


def test_more_than_2_to_31_elements(cuda):
    import torch
    n, H, d = (1 << 31) // (32 * 256) + 3, 32, 256
    dims = cuda.make_dims(cuda.DTYPE_BF16, Hq=H, Hkv=1, d=d)
    q = torch.randn(n, H, d, device="cuda", dtype=torch.bfloat16)
    pos = torch.arange(n, dtype=torch.int32, device="cuda")
    tail = q[-2:].clone()
    cuda.jet_norm_rotate(dims, _rope(cuda, rot=256), pos, q, None, None, None, q, None)
    _sync(cuda)
    want, bar = B.rotation(_np(tail), [n - 2, n - 1], 256, "halves", W.frequencies(256, 1e4), None,
                           1e-6, True, True)
    assert B.worst(_np(q[-2:]), want, bar) <= 1.0
