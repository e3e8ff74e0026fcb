"""GPU parity of the attention under a window with first tokens, the step's and the
prefill's, against 64 bits at bars derived from what each row weighs
(tests/window_bars.py): windows and first tokens around the key tiles, candidates that leave
the window or are first tokens themselves, head sizes and layouts, what must not reach a row,
chained with the rotation, captured, on other streams, with layouts that lie."""
import ctypes

import numpy as np
import pytest

import oracle as O
import window_bars as B

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def cuda(jet):
    import torch
    if not torch.cuda.is_available():
        pytest.fail("CUDA device required for -m gpu tests")
    return jet


def _np(x):
    return x.double().cpu().numpy()


class Step:
    """A batch of the step with seeded tensors; n_cand candidates a request of lengths m."""

    def __init__(self, jet, P, n_cand, m, Hq, Hkv, d, bf16, seed=0, spread=1.0):
        import torch
        self.jet, self.bf16 = jet, bf16
        self.hl = jet.jet_layout_build(P, n_cand, m, [0] * int(sum(m)), 4)
        self.lay = O.build_layout(P, n_cand, m, [0] * int(sum(m)), 4)
        self.dev = self.hl.to_device("cuda")
        self.dims = jet.make_dims(jet.DTYPE_BF16 if bf16 else jet.DTYPE_F32, Hq=Hq, Hkv=Hkv, d=d)
        g = torch.Generator(device="cuda").manual_seed(seed)
        dt = torch.bfloat16 if bf16 else torch.float32

        def draw(*shape):
            return torch.randn(*shape, generator=g, device="cuda").to(dt)

        N, F, S = int(self.lay["N"]), int(self.lay["N"]) - len(P), int(sum(P))
        self.q = draw(N, Hq, d) * spread
        self.k, self.v = draw(S, Hkv, d), draw(S, Hkv, d)
        self.kc, self.vc = draw(F, Hkv, d), draw(F, Hkv, d)
        self.o = self.q.new_full(self.q.shape, 7.0)

    def ws(self, window, sinks):
        import torch
        nb = self.jet.jet_attend_window_workspace_bytes(self.hl.sizes, self.dims, window, sinks)
        assert nb > 0
        return torch.empty((nb + 15) // 16 * 4, device="cuda")

    def run(self, window, sinks, ws=None, stream=None, layout=None, status=0):
        import torch
        self.jet.jet_prefix_attend_window(
            self.dev if layout is None else layout, self.dims, window, sinks, self.q, self.k,
            self.v, self.kc, self.vc, self.o, self.ws(window, sinks) if ws is None else ws,
            stream=stream)
        torch.cuda.synchronize()
        assert self.jet.jet_device_status() == status

    def check(self, window, sinks, requests=None, o=None):
        got = _np(self.o if o is None else o)
        for r, (rows, want, bar) in B.cascade(
                self.lay, *(_np(x) for x in (self.q, self.k, self.v, self.kc, self.vc)), window,
                sinks, self.bf16, requests).items():
            assert B.worst(got[rows], want, bar) <= 1.0, (r, window, sinks)


class Prefill:
    def __init__(self, jet, P, Hq, Hkv, d, seed=0):
        import torch
        self.jet, self.P = jet, P
        R = len(P)
        self.hl = jet.jet_layout_build(P, [1] * R, [1] * R, [0] * R, 4)
        self.dev = self.hl.to_device("cuda")
        self.dims = jet.make_dims(jet.DTYPE_BF16, Hq=Hq, Hkv=Hkv, d=d)
        g = torch.Generator(device="cuda").manual_seed(seed)
        S = int(sum(P))
        self.q, self.k, self.v = (torch.randn(S, h, d, generator=g, device="cuda").bfloat16()
                                  for h in (Hq, Hkv, Hkv))
        self.o = self.q.new_full(self.q.shape, 7.0)

    def ws(self, window, sinks):
        import torch
        nb = self.jet.jet_prefill_window_workspace_bytes(self.hl.sizes, self.dims, window, sinks)
        assert nb > 0
        return torch.empty((nb + 15) // 16 * 4, device="cuda")

    def run(self, window, sinks, ws=None, stream=None, layout=None, status=0):
        import torch
        self.jet.jet_prefill_attend_window(
            self.dev if layout is None else layout, self.dims, window, sinks, self.q, self.k,
            self.v, self.o, self.ws(window, sinks) if ws is None else ws, stream=stream)
        torch.cuda.synchronize()
        assert self.jet.jet_device_status() == status

    def check(self, window, sinks, rows_of=None, o=None):
        got = _np(self.o if o is None else o)
        for r, (rows, want, bar) in B.prefill(
                self.P, *(_np(x) for x in (self.q, self.k, self.v)), window, sinks,
                rows_of=rows_of).items():
            assert B.worst(got[rows], want, bar) <= 1.0, (r, window, sinks)


# --------------------------------------------------------------------------
# the step
# --------------------------------------------------------------------------
WINDOWS = [(1, 0), (1, 1), (2, 3), (7, 0), (63, 1), (64, 4), (65, 64), (100, 16), (128, 17),
           (129, 63), (200, 65), (500, 130), (100000, 0), (1, 100000), (2 ** 31 - 1, 2 ** 31 - 1)]
PREFIXES = [1, 2, 15, 64, 65, 127, 200, 330]


def _mixed(jet, Hq, Hkv, d, bf16, seed=0):
    R = len(PREFIXES)
    n_cand = [1 + i % 3 for i in range(R)]
    m = [1 + (5 * i + 3 * seed) % 9 for i in range(sum(n_cand))]
    return Step(jet, PREFIXES, n_cand, m, Hq, Hkv, d, bf16, seed)


@pytest.mark.parametrize("bf16", [True, False])
@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("heads", [(8, 2), (7, 1), (3, 3)])
def test_step(cuda, heads, d, bf16):
    s = _mixed(cuda, *heads, d, bf16)
    for window, sinks in WINDOWS:
        s.o.fill_(7.0)
        s.run(window, sinks)
        s.check(window, sinks)


@pytest.mark.parametrize("bf16", [True, False])
def test_step_large_scores(cuda, bf16):
    R = len(PREFIXES)
    s = Step(cuda, PREFIXES, [2] * R, [4, 2] * R, 8, 2, 128, bf16, seed=3, spread=12.0)
    for window, sinks in ((1, 2), (70, 5), (300, 0)):
        s.run(window, sinks)
        s.check(window, sinks)


@pytest.mark.parametrize("bf16", [True, False])
def test_step_one_row_a_request(cuda, bf16):
    # the next token of each of many traces: no candidate tokens are fed
    P = [1 + 37 * i % 900 for i in range(70)]
    s = Step(cuda, P, [1] * 70, [1] * 70, 32, 8, 128, bf16, seed=1)
    for window, sinks in ((1, 0), (100, 4), (640, 1), (3000, 0)):
        s.run(window, sinks)
        s.check(window, sinks)


@pytest.mark.parametrize("bf16", [True, False])
def test_step_long_candidates_leave_the_window(cuda, bf16):
    # candidates longer than the window and than a key tile, over short and long prefixes,
    # which may be shorter than the first tokens
    s = Step(cuda, [3, 150, 700], [2, 1, 3], [150, 90, 200, 140, 2, 70], 4, 2, 64, bf16, seed=2)
    for window, sinks in ((1, 0), (5, 10), (64, 0), (65, 100), (130, 1), (1000, 5)):
        s.run(window, sinks)
        s.check(window, sinks)


@pytest.mark.parametrize("bf16", [True, False])
def test_step_many_rows_of_one_request(cuda, bf16):
    # more query vectors than a block holds
    s = Step(cuda, [400, 20], [40, 1], [3] * 20 + [12] * 20 + [5], 16, 2, 64, bf16, seed=4)
    for window, sinks in ((33, 2), (300, 4)):
        s.run(window, sinks)
        s.check(window, sinks)


@pytest.mark.parametrize("d,heads", [(128, (8, 2)), (256, (16, 2)), (64, (8, 8))])
def test_step_one_long_context_in_chunks(cuda, d, heads):
    s = Step(cuda, [20000], [3], [6, 1, 12], *heads, d, True, seed=5)
    for window, sinks in ((6000, 20), (8192, 0), (19990, 4), (129, 1)):
        s.run(window, sinks)
        s.check(window, sinks)


def test_step_many_long_contexts(cuda):
    P = [int(x) for x in np.random.default_rng(0).integers(1000, 6000, size=90)]
    s = Step(cuda, P, [2] * 90, [3, 5] * 90, 16, 2, 256, True, seed=6)
    for window, sinks in ((2000, 16), (300, 200)):
        s.run(window, sinks)
        s.check(window, sinks, requests=[0, 1, 17, 44, 88, 89])


@pytest.mark.parametrize("bf16", [True, False])
def test_wide_windows_give_the_plain_attention(cuda, bf16):
    import torch
    s = _mixed(cuda, 8, 2, 64, bf16)
    s.run(100000, 0)
    ws = torch.empty(cuda.jet_workspace_bytes(s.hl.sizes, s.dims) // 4 + 4, device="cuda")
    plain = torch.empty_like(s.o)
    cuda.jet_prefix_attend(s.dev, s.dims, s.q, s.k, s.v, s.kc, s.vc, plain, ws)
    torch.cuda.synchronize()
    s.check(100000, 0, o=plain)
    assert float((s.o.double() - plain.double()).abs().max()) <= (0.04 if bf16 else 1e-5)


@pytest.mark.parametrize("bf16", [True, False])
@pytest.mark.parametrize("P", [[64], [10, 64, 63, 17]])
def test_step_first_tokens_that_reach_the_window(cuda, P, bf16):
    # the first tokens' last box of 16 passes the window's first key, or the prefix's end
    s = Step(cuda, P, [2] * len(P), [3, 1] * len(P), 8, 2, 64, bf16, seed=10)
    for window, sinks in ((1, 2), (1, 50), (1, 61), (2, 49), (15, 33), (8, 1), (1, 1)):
        s.o.fill_(7.0)
        s.run(window, sinks)
        s.check(window, sinks)


# --------------------------------------------------------------------------
# the prefill
# --------------------------------------------------------------------------
@pytest.mark.parametrize("d,heads", [(64, (8, 2)), (128, (8, 8)), (256, (16, 2))])
def test_prefill_large_scores(cuda, d, heads):
    # scores of up to hundreds, and keys that grow along the prefix, so that the maximum does
    import torch
    p = Prefill(cuda, [700, 33, 260], *heads, d, seed=5)
    p.q *= 8.0
    p.k *= torch.linspace(0.25, 6.0, p.k.shape[0], device="cuda")[:, None, None].bfloat16()
    for window, sinks in ((40, 3), (300, 0), (1000, 0)):
        p.run(window, sinks)
        p.check(window, sinks)


@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("heads", [(8, 2), (7, 1), (3, 3), (24, 4)])
def test_prefill(cuda, heads, d):
    p = Prefill(cuda, [1, 2, 63, 64, 65, 130, 300], *heads, d)
    for window, sinks in WINDOWS:
        p.o.fill_(7.0)
        p.run(window, sinks)
        p.check(window, sinks)


def _some(P, rng, per=8):
    return [np.unique(np.concatenate([np.arange(min(3, x)), np.arange(max(0, x - 3), x),
                                      rng.integers(0, x, size=per)])) for x in P]


@pytest.mark.parametrize("d,heads", [(64, (16, 2)), (128, (32, 8)), (256, (16, 2)), (256, (1, 1)),
                                     (128, (100, 1)), (64, (128, 1))])
def test_prefill_long(cuda, d, heads):
    P = [5000, 17, 1300]
    p = Prefill(cuda, P, *heads, d, seed=1)
    rng = np.random.default_rng(d)
    for window, sinks in ((1, 0), (17, 40), (128, 1), (1000, 4), (1024, 128), (4096, 16)):
        p.run(window, sinks)
        p.check(window, sinks, rows_of=_some(P, rng))


def test_prefill_many_short(cuda):
    P = [1 + 7 * i % 90 for i in range(200)]
    p = Prefill(cuda, P, 24, 4, 256, seed=2)
    for window, sinks in ((5, 2), (32, 0), (64, 1)):
        p.run(window, sinks)
        p.check(window, sinks)


# --------------------------------------------------------------------------
# what a row does not see
# --------------------------------------------------------------------------
BAD = [float("nan"), float("inf"), float("-inf"), -3.3895e38]


@pytest.mark.parametrize("bf16", [True, False])
@pytest.mark.parametrize("d", [64, 256])
def test_step_unseen_keys_reach_no_row(cuda, d, bf16):
    window, sinks = 40, 3
    s = Step(cuda, [300, 41, 200, 64], [2, 1, 2, 1], [4, 9, 1, 60, 2, 3], 8, 2, d, bf16, seed=7)
    clean = {n: getattr(s, n).clone() for n in ("k", "v", "kc", "vc")}
    p0 = np.concatenate([[0], np.cumsum([300, 41, 200, 64])])
    for bad in BAD:
        for n, x in clean.items():
            getattr(s, n).copy_(x)
        # past every window and not a first token
        for r, P in enumerate((300, 41, 200, 64)):
            for t in (s.k, s.v):
                t[p0[r] + sinks:p0[r] + P - window] = bad
        # candidate tokens that another candidate's rows share a tile with; the rows that see
        # them are told apart below
        s.vc[0], s.kc[5], s.vc[-1] = bad, bad, bad
        s.run(window, sinks)
        got = _np(s.o)
        lay = s.lay
        hit = set()
        for n in range(int(lay["N"])):
            f = n - int(lay["row_req"][n]) - 1
            first = int(lay["cand_row_offset"][lay["row_cand"][n]]) - int(lay["row_req"][n]) - 1 \
                if lay["row_cand"][n] >= 0 else None
            last = len(s.vc) - 1
            if first is not None and any(max(first, f - window + 1) <= b <= f
                                         for b in (0, 5, last)):
                hit.add(n)
        rest = [n for n in range(int(lay["N"])) if n not in hit]
        assert len(rest) > 5 and hit
        for r, (rows, want, bar) in B.cascade(
                lay, *(_np(x) for x in (s.q, s.k, s.v, s.kc, s.vc)), window, sinks,
                bf16).items():
            keep = np.array([n in rest for n in rows])
            assert B.worst(got[rows[keep]], want[keep], bar[keep]) <= 1.0, (r, bad)
        # and those that see them show it
        if bad != BAD[3]:
            assert not np.isfinite(got[sorted(hit)]).all()


@pytest.mark.parametrize("d,heads", [(64, (8, 2)), (128, (8, 8)), (256, (16, 2))])
def test_prefill_unseen_keys_reach_no_row(cuda, d, heads):
    P, window, sinks = [400, 60, 150], 37, 2
    p = Prefill(cuda, P, *heads, d, seed=3)
    k, v = p.k.clone(), p.v.clone()
    for bad in BAD:
        p.k.copy_(k)
        p.v.copy_(v)
        at = [100, 231, 400 + 55, 460 + 2]   # in no other request's, nor a later, window
        for i, j in enumerate(at):
            (p.v if i != 1 else p.k)[j] = bad
        p.run(window, sinks)
        got = _np(p.o)
        for r, (rows, want, bar) in B.prefill(P, *(_np(x) for x in (p.q, p.k, p.v)), window,
                                              sinks).items():
            p0 = sum(P[:r])
            pos = rows - p0
            seen = np.zeros(len(rows), bool)
            for j in at:
                if p0 <= j < p0 + P[r]:
                    seen |= B.in_window(pos, [j - p0], window, sinks)[:, 0]
            assert B.worst(got[rows[~seen]], want[~seen], bar[~seen]) <= 1.0, (r, bad)
            if bad != BAD[3] and seen.any():
                assert not np.isfinite(got[rows[seen]]).all()


@pytest.mark.parametrize("d,heads", [(64, (8, 2)), (128, (8, 8)), (256, (16, 2))])
def test_values_near_the_largest_float(cuda, d, heads):
    # finite outputs whose unnormalised sums are not
    p = Prefill(cuda, [300, 41], *heads, d, seed=6)
    s = Step(cuda, [300, 41], [2, 1], [3, 5, 30], *heads, d, True, seed=6)
    for x in (p.v, s.v, s.vc):
        x.copy_(x.float().clamp(-3, 3) * 1e38)
    for window, sinks in ((60, 3), (1000, 0)):
        for x in (p, s):
            x.run(window, sinks)
            x.check(window, sinks)


@pytest.mark.parametrize("bf16", [True, False])
def test_scores_of_minus_infinity(cuda, bf16):
    """Keys of minus infinity under positive queries weigh nothing; a vector that sees no other
    is 0 / 0."""
    window, sinks = 3, 1
    s = Step(cuda, [100, 90], [2, 1], [1, 6, 8], 4, 2, 64, bf16, seed=11)
    p = Prefill(cuda, [100, 90], 4, 2, 64, seed=11)
    p0 = [0, 100]
    for x in (s, p):
        x.q.abs_().add_(0.125)
        x.k[p0[0] + 98, 0] = x.k[p0[1] + 20, 0] = float("-inf")      # one of several
        x.k[p0[1] + 40:p0[1] + 43] = float("-inf")                   # all but the first token
        x.run(window, sinks)
    f = 1 + np.flatnonzero(s.lay["row_req"] == 1)[0]                # request 1's first fed token
    s.kc[f - 1:f + 3] = float("-inf")
    s.run(window, sinks)

    def check(o, q, k, v, sees, rows):
        for h in range(2):  # a key/value head at a time: their unseen keys differ
            inf = ~np.isfinite(k[:, h, 0])
            want, bar = B.attention(q[:, 2 * h:2 * h + 2], k[:, h:h + 1], v[:, h:h + 1],
                                    sees & ~inf, bf16)
            assert B.worst(o[rows, 2 * h:2 * h + 2], want, bar) <= 1.0

    if bf16:
        at = np.arange(190)
        pos, req = np.concatenate([np.arange(100), np.arange(90)]), np.repeat([0, 1], [100, 90])
        sees = B.in_window(pos, pos, window, sinks) & (req[:, None] == req[None, :])
        check(_np(p.o), *(_np(x) for x in (p.q, p.k, p.v)), sees, at)
    lay = s.lay
    req, cand = lay["row_req"], lay["row_cand"].astype(np.int64)
    pos = np.array([100, 90])[req] - 1 + np.where(cand >= 0, lay["row_pos"], 0)
    key_req = np.repeat([0, 1], [100, 90])
    key_pos = np.concatenate([np.arange(100), np.arange(90)])
    fed = np.flatnonzero(cand >= 0)
    sees = np.concatenate([
        B.in_window(pos, key_pos, window, sinks) & (req[:, None] == key_req[None, :]),
        B.in_window(pos, pos[fed], window, sinks) & (cand[:, None] == cand[None, fed])], 1)
    check(_np(s.o), _np(s.q), np.concatenate([_np(s.k), _np(s.kc)]),
          np.concatenate([_np(s.v), _np(s.vc)]), sees, np.arange(len(req)))
    # and without the first token
    s.run(window, 0)
    got = _np(s.o)
    sees0 = np.concatenate([
        B.in_window(pos, key_pos, window, 0) & (req[:, None] == key_req[None, :]),
        B.in_window(pos, pos[fed], window, 0) & (cand[:, None] == cand[None, fed])], 1)
    none = ~(sees0 & np.isfinite(np.concatenate([_np(s.k), _np(s.kc)])[:, 1, 0])).any(1)
    assert none.any() and np.isnan(got[none, 2:]).all() and np.isfinite(got[~none, 2:]).all()
    if bf16:
        p.run(window, 0)
        got = _np(p.o)
        assert np.isnan(got[142]).all() and np.isfinite(np.delete(got, 142, axis=0)).all()


@pytest.mark.parametrize("bf16", [True, False])
@pytest.mark.parametrize("d,heads", [(128, (8, 2)), (256, (16, 2))])
def test_unseen_keys_reach_no_row_through_chunks(cuda, d, heads, bf16):
    # a long window in chunks: the oldest key of the shared row, seen by no other, and one
    # between the first tokens and the end of their box
    P, window, sinks = 20000, 6000, 20
    s = Step(cuda, [P], [2], [5, 3], *heads, d, bf16, seed=12)
    for bad in BAD:
        for at in (P - window, 25):
            k, v = s.k[at].clone(), s.v[at].clone()
            s.v[at] = bad
            s.k[at] = bad
            s.run(window, sinks)
            got = _np(s.o)
            for r, (rows, want, bar) in B.cascade(
                    s.lay, *(_np(x) for x in (s.q, s.k, s.v, s.kc, s.vc)), window, sinks,
                    bf16).items():
                rest = rows[1:] if at != 25 else rows
                assert B.worst(got[rest], want[rest], bar[rest]) <= 1.0, (bad, at)
                if at != 25 and bad != BAD[3]:
                    assert not np.isfinite(got[0]).any()
            s.k[at], s.v[at] = k, v


def test_offsets_past_32_bits(cuda):
    """A batch whose tensors have more than 2^31 elements: the rotation, the prefill and the
    step at its far end."""
    import torch
    P, H, d, window, sinks = [68000, 300], 128, 256, 200, 4
    p = Prefill(cuda, P, H, H, d, seed=7)
    assert p.q.numel() > 2 ** 31
    rope = cuda.make_rope(64, theta=1e6, norm=False)
    S, W0 = sum(P), 200 + 8

    def ends(x, r):  # the first tokens and the last ones of a request
        lo, hi = (0, P[0]) if r == 0 else (P[0], S)
        return _np(torch.cat([x[lo:lo + sinks], x[hi - W0:hi]]))

    from oracle import window as W
    raw = [ends(p.k, r) for r in range(2)]
    where = [np.concatenate([np.arange(sinks), np.arange(x - W0, x)]) for x in P]
    cuda.jet_norm_rotate_prefix(p.dev, p.dims, rope, p.q, p.k, None, None, p.q, p.k)
    p.run(window, sinks)
    s = Step(cuda, P, [1, 1], [3, 2], H, H, d, True, seed=7)
    s.k, s.v = p.k, p.v
    s.run(window, sinks)
    for r in range(2):
        want, bar = B.rotation(raw[r], where[r], 64, "halves", W.frequencies(64, 1e6), None, 1e-6,
                               False, True)
        k, v = ends(p.k, r), ends(p.v, r)
        assert B.worst(k, want, bar) <= 1.0
        at = np.arange(P[r] - 3, P[r])
        hi = P[0] if r == 0 else S
        heads = [0, 1, 77, 127]
        want, bar = B.attention(_np(p.q[hi - 3:hi])[:, heads], k[:, heads], v[:, heads],
                                B.in_window(at, where[r], window, sinks), True)
        assert B.worst(_np(p.o[hi - 3:hi])[:, heads], want, bar) <= 1.0
        n0, n1 = (int(s.lay["row_offset"][r + i]) for i in (0, 1))
        pos = P[r] - 1 + np.arange(n1 - n0)
        own = slice(n0 - r, n1 - r - 1)
        want, bar = B.attention(
            _np(s.q[n0:n1])[:, heads],
            np.concatenate([k, _np(s.kc[own])])[:, heads],
            np.concatenate([v, _np(s.vc[own])])[:, heads],
            B.in_window(pos, np.concatenate([where[r], pos[1:]]), window, sinks), True)
        assert B.worst(_np(s.o[n0:n1])[:, heads], want, bar) <= 1.0


def test_infinite_and_nan_values_come_out_where_they_are_seen(cuda):
    # a visible infinite value gives an infinity in its column, a NaN score a NaN row
    s = Step(cuda, [100], [1], [1], 4, 2, 64, True, seed=8)
    s.v[95, 0, 3] = float("inf")
    s.run(20, 0)
    assert np.isposinf(_np(s.o)[0, :2, 3]).all()
    assert np.isfinite(np.delete(_np(s.o)[0], 3, axis=-1)).all()
    s.v[95, 0, 3] = 0.0
    s.k[99, 1, 0] = float("nan")
    s.run(20, 0)
    assert np.isnan(_np(s.o)[0, 2:]).all() and np.isfinite(_np(s.o)[0, :2]).all()


# --------------------------------------------------------------------------
# use
# --------------------------------------------------------------------------
def test_rotate_prefill_and_step_in_one_run(cuda):
    """A model's layer: queries and keys normalised and rotated, the prefill, then the step
    over the cache it leaves; against 64 bits, whose inputs are the rotated tensors."""
    import torch
    P, n_cand, m = [70, 300], [2, 1], [4, 2, 6]
    s = Step(cuda, P, n_cand, m, 8, 2, 128, True, seed=9)
    p = Prefill(cuda, P, 8, 2, 128, seed=9)
    p.k, p.v = s.k, s.v
    rope = cuda.make_rope(128, theta=1e5)
    gain = torch.ones(128, dtype=torch.bfloat16, device="cuda")
    window, sinks = 48, 4
    cuda.jet_norm_rotate_prefix(s.dev, s.dims, rope, p.q, s.k, gain, gain, p.q, s.k)
    p.run(window, sinks)
    cuda.jet_norm_rotate_rows(s.dev, s.dims, rope, s.q, s.kc, gain, gain, s.q, s.kc)
    s.run(window, sinks)
    p.check(window, sinks)
    s.check(window, sinks)
    # the shared row is the prefill's last position when its query is
    last = np.cumsum(P) - 1
    n0 = [int(x) for x in s.lay["row_offset"][:2]]
    s.q[n0] = p.q[last]
    s.run(window, sinks)
    assert float((s.o[n0].double() - p.o[last].double()).abs().max()) <= 0.04


@pytest.mark.parametrize("bf16", [True, False])
def test_captured_and_replayed(cuda, bf16):
    import torch
    s = _mixed(cuda, 8, 2, 64, bf16)
    ws = s.ws(70, 4)
    s.run(70, 4, ws=ws)
    g, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    with torch.cuda.graph(g):
        cuda.jet_prefix_attend_window(s.dev, s.dims, 70, 4, s.q, s.k, s.v, s.kc, s.vc, s.o, ws)
    for seed in range(2):
        s.q.normal_(generator=torch.Generator(device="cuda").manual_seed(seed))
        ws.fill_(float("nan"))
        s.o.fill_(7.0)
        g.replay()
        torch.cuda.synchronize()
        s.check(70, 4)
    s.o.fill_(7.0)
    side.wait_stream(torch.cuda.current_stream())
    s.run(70, 4, ws=ws, stream=side)
    s.check(70, 4)


@pytest.mark.parametrize("bf16", [True, False])
def test_two_graphs_share_a_workspace(cuda, bf16):
    # long contexts in chunks, whose partials lie there, under two windows
    import torch
    s = Step(cuda, [9000, 40], [2, 1], [3, 4, 2], 8, 2, 128, bf16, seed=13)
    forms = [(4000, 3), (8000, 0)]
    ws = max((s.ws(*f) for f in forms), key=lambda x: x.numel())
    graphs = []
    for window, sinks in forms:
        s.run(window, sinks, ws=ws)
        g, o = torch.cuda.CUDAGraph(), torch.empty_like(s.o)
        with torch.cuda.graph(g):
            cuda.jet_prefix_attend_window(s.dev, s.dims, window, sinks, s.q, s.k, s.v, s.kc, s.vc,
                                          o, ws)
        graphs.append((g, o))
    for order in ((0, 1), (1, 0), (1, 1)):
        ws.fill_(float("nan"))
        for i in order:
            graphs[i][1].fill_(7.0)
        for i in order:
            graphs[i][0].replay()
        torch.cuda.synchronize()
        for i in order:
            s.check(*forms[i], o=graphs[i][1])


def test_two_calls_at_once(cuda):
    # each with its own workspace, on its own stream
    import torch
    s = Step(cuda, [6000] * 6, [2] * 6, [3, 4] * 6, 16, 2, 256, True, seed=14)
    p = Prefill(cuda, [3000, 500], 16, 2, 256, seed=14)
    ws, wp = s.ws(2000, 4), p.ws(300, 4)
    side = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(4):
        cuda.jet_prefix_attend_window(s.dev, s.dims, 2000, 4, s.q, s.k, s.v, s.kc, s.vc, s.o, ws,
                                      stream=side[0])
        cuda.jet_prefill_attend_window(p.dev, p.dims, 300, 4, p.q, p.k, p.v, p.o, wp,
                                       stream=side[1])
    torch.cuda.synchronize()
    assert cuda.jet_device_status() == 0
    s.check(2000, 4)
    p.check(300, 4, rows_of=_some(p.P, np.random.default_rng(0), 40))


def test_prefill_captured_and_on_another_stream(cuda):
    import torch
    p = Prefill(cuda, [300, 20, 77], 8, 2, 64)
    ws = p.ws(50, 2)
    p.run(50, 2, ws=ws)
    g, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    with torch.cuda.graph(g):
        cuda.jet_prefill_attend_window(p.dev, p.dims, 50, 2, p.q, p.k, p.v, p.o, ws)
    for seed in range(2):
        p.q.normal_(generator=torch.Generator(device="cuda").manual_seed(seed))
        ws.fill_(float("nan"))
        p.o.fill_(7.0)
        g.replay()
        torch.cuda.synchronize()
        p.check(50, 2)
    p.o.fill_(7.0)
    side.wait_stream(torch.cuda.current_stream())
    p.run(50, 2, ws=ws, stream=side)
    p.check(50, 2)


def test_same_inputs_same_bits(cuda):
    s, p = _mixed(cuda, 8, 2, 128, True), Prefill(cuda, [500, 333], 8, 2, 128)
    for x in (s, p):
        x.run(90, 5)
        first = x.o.clone()
        for _ in range(3):
            x.o.fill_(7.0)
            x.run(90, 5)
            assert (x.o == first).all()


def test_writes_its_outputs_only(cuda):
    """The rows past the last one, and the words past the workspace, stay as they were."""
    import torch
    s, p = _mixed(cuda, 7, 1, 64, True), Prefill(cuda, [130, 21], 7, 1, 64)
    for x, size in ((s, cuda.jet_attend_window_workspace_bytes),
                    (p, cuda.jet_prefill_window_workspace_bytes)):
        for window, sinks in ((30, 2), (100000, 0)):
            nb = (size(x.hl.sizes, x.dims, window, sinks) + 15) // 16 * 16
            big = x.o.new_full((x.o.shape[0] + 64, *x.o.shape[1:]), 7.0)
            ws = torch.full((nb + 4096,), 171, dtype=torch.uint8, device="cuda")
            keep, x.o = x.o, big
            x.run(window, sinks, ws=ws)
            assert (big[keep.shape[0]:] == 7.0).all() and (ws[nb:] == 171).all()
            x.o = keep
            x.check(window, sinks, o=big[:keep.shape[0]])


def test_layouts_that_lie_are_reported(cuda):
    import torch
    err = {v: k for k, v in cuda.STATUS_NAMES.items()}["JET_ERR_DEVICE"]
    for bf16 in (True, False):
        s = Step(cuda, [100, 50, 70], [1, 2, 1], [3, 2, 4, 1], 8, 2, 64, bf16, seed=10)
        names = [("prefix_offset", 1, v) for v in (-4, 1 << 30, 200, 2 ** 31 - 1)]
        names += [("row_req", 2, 3), ("row_req", 2, -1)]
        for name, i, bad in names:
            words = s.dev.words.clone()
            words[(getattr(s.dev.struct, name) - s.dev.words.data_ptr()) // 4 + i] = bad
            cuda.jet_prefix_attend_window(cuda.DeviceLayout(s.hl.sizes, words), s.dims, 20, 2, s.q,
                                          s.k, s.v, s.kc, s.vc, s.o, s.ws(20, 2))
            torch.cuda.synchronize()
            status = cuda.jet_device_status()
            # words that the call does not read may lie unnoticed; nothing else may come of it
            assert status == err or (name == "row_req" and status == 0), (name, bad)
    p = Prefill(cuda, [100, 50, 70], 8, 2, 64)
    for bad in (-4, 1 << 30, 230, 2 ** 31 - 1):
        words = p.dev.words.clone()
        words[(p.dev.struct.prefix_offset - p.dev.words.data_ptr()) // 4 + 1] = bad
        p.run(20, 2, layout=cuda.DeviceLayout(p.hl.sizes, words), status=err)


def test_cache_of_more_than_2_to_31_elements(cuda):
    """The last requests of a batch whose keys pass 2^31 elements, and one context that does."""
    import torch
    Hkv, d = 8, 256
    n = (1 << 31) // (Hkv * d)
    for P in ([n - 500, 700, 900], [n + 300]):
        S = sum(P)
        R = len(P)
        hl = cuda.jet_layout_build(P, [1] * R, [3] * R, [0] * (3 * R), 4)
        lay = O.build_layout(P, [1] * R, [3] * R, [0] * (3 * R), 4)
        dims = cuda.make_dims(cuda.DTYPE_BF16, Hq=8, Hkv=Hkv, d=d)
        g = torch.Generator(device="cuda").manual_seed(1)
        k, v = (torch.empty(S, Hkv, d, device="cuda", dtype=torch.bfloat16).normal_(generator=g)
                for _ in range(2))
        N = 3 * R
        q, kc, vc = (torch.randn(x, h, d, device="cuda", generator=g).bfloat16()
                     for x, h in ((N, 8), (2 * R, Hkv), (2 * R, Hkv)))
        o = torch.empty_like(q)
        window, sinks = 600, 4
        nb = cuda.jet_attend_window_workspace_bytes(hl.sizes, dims, window, sinks)
        cuda.jet_prefix_attend_window(hl.to_device("cuda"), dims, window, sinks, q, k, v, kc, vc, o,
                                      torch.empty(nb // 4 + 4, device="cuda"))
        torch.cuda.synchronize()
        assert cuda.jet_device_status() == 0
        r = R - 1
        p0, p1 = sum(P[:r]), sum(P)
        rows = np.arange(3 * r, 3 * r + 3)
        at = np.concatenate([np.arange(sinks), np.arange(P[r] - 600, P[r])])
        pos = P[r] - 1 + np.arange(3)
        sees = np.concatenate([B.in_window(pos, at, window, sinks),
                               B.in_window(pos, pos[1:], window, sinks)], 1)
        K = np.concatenate([_np(k[p0 + torch.from_numpy(at)]), _np(kc[2 * r:])])
        V = np.concatenate([_np(v[p0 + torch.from_numpy(at)]), _np(vc[2 * r:])])
        want, bar = B.attention(_np(q[rows]), K, V, sees, True)
        assert B.worst(_np(o[rows]), want, bar) <= 1.0
        assert p1 == S
        del k, v


def test_binding_keeps_the_callers_workspace_size(cuda):
    s = _mixed(cuda, 8, 2, 64, True)
    nb = cuda.jet_attend_window_workspace_bytes(s.hl.sizes, s.dims, 30, 2)
    ws = s.ws(30, 2)
    with pytest.raises(cuda.JetError):
        cuda.jet_prefix_attend_window(s.dev, s.dims, 30, 2, s.q, s.k, s.v, s.kc, s.vc, s.o, ws,
                                      ws_bytes=nb - 1)
    assert ctypes.sizeof(cuda.jet_rope) == 16 + 128 * 8
