"""The 8-bit prefix cache against its oracle: codes and exponents bit by bit (whole
prefixes, pieces, single tokens, zeros, the smallest and largest numbers, infinities
and NaN), nothing else written, the cache read back exactly, and the cascade
attention over it in both types, with what a mask hides kept out."""
import numpy as np
import pytest

import oracle as O
from oracle import kv_e4m3 as K

pytestmark = pytest.mark.gpu

JET_ERR_DEVICE = 10
GUARD = 4096


def _torch(x, dtype):
    import torch
    t = torch.from_numpy(np.ascontiguousarray(x, np.float32)).cuda()
    return t.to(torch.bfloat16) if dtype == "bf16" else t


def _np(t):
    return t.double().cpu().numpy()


def _batch(jet, prefix_len, n_cand=None, cand_len=None, **dims):
    n_cand = [1] * len(prefix_len) if n_cand is None else n_cand
    cand_len = [1] * int(np.sum(n_cand)) if cand_len is None else cand_len
    host = jet.jet_layout_build(prefix_len, n_cand, cand_len, [0] * int(np.sum(cand_len)), 2)
    dtype = jet.DTYPE_BF16 if dims.pop("dtype") == "bf16" else jet.DTYPE_F32
    return host, host.to_device(), jet.make_dims(dtype, **dims)


def _tokens(rng, n, heads, d, spread=1.0):
    """Elements of scales that differ from token to token and head to head."""
    s = np.exp(spread * rng.standard_normal((n, heads, 1)))
    return (rng.standard_normal((n, heads, d)) * s).astype(np.float32)


def _buffers(jet, host, dims, background):
    """Two cache buffers with guards after them, filled with a background byte."""
    import torch
    nb = jet.jet_kv_e4m3_bytes(host.sizes, dims)
    return nb, [torch.full((nb + GUARD,), background, dtype=torch.uint8, device="cuda")
                for _ in range(2)]


def _check_buffer(got, cache, nb, background):
    got = got.cpu().numpy()
    assert np.all(got[nb:] == background)
    np.testing.assert_array_equal(got[:nb], cache.buffer(background))


SHAPES = [
    ([1], 1, 64), ([64], 2, 256), ([65, 1, 63], 4, 128), ([1, 2, 127, 128, 129, 300], 8, 64),
    ([700, 31], 3, 256), (list(range(1, 90)), 2, 128), ([5] * 700, 1, 64),
]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("shape", range(len(SHAPES)))
def test_whole_prefix(jet, dtype, shape):
    import torch
    P, heads, d = SHAPES[shape]
    rng = np.random.default_rng(shape)
    host, lay, dims = _batch(jet, P, dtype=dtype, Hkv=heads, d=d)
    x = [_torch(_tokens(rng, sum(P), heads, d), dtype) for _ in range(2)]
    nb, buf = _buffers(jet, host, dims, 0xA5)
    jet.jet_quantize_kv_e4m3(lay, dims, *x, *buf)
    back = [torch.full_like(t, 7.0) for t in x]
    jet.jet_dequantize_kv_e4m3(lay, dims, *buf, *back)
    torch.cuda.synchronize()
    assert jet.jet_device_status() == 0
    for i in range(2):
        cache = K.Cache(P, heads, d).write(_np(x[i]))
        _check_buffer(buf[i], cache, nb, 0xA5)
        np.testing.assert_array_equal(_np(back[i]), cache.values())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_extreme_elements(jet, dtype):
    # blocks of zeros, of the least and the largest numbers, of halfway cases, of
    # infinities and NaN among numbers, and of nothing else
    import torch
    P, heads, d = [64 * 8 + 3], 2, 64
    rng = np.random.default_rng(3)
    host, lay, dims = _batch(jet, P, dtype=dtype, Hkv=heads, d=d)
    x = _tokens(rng, P[0], heads, d)
    with np.errstate(over="ignore", invalid="ignore"):
        x[0:64] = 0.0
        x[64:128] *= np.float32(2.0 ** -120)
        x[128:192] = np.float32(3.38e38) * np.sign(x[128:192])
        x[192:256] = (np.arange(64 * 2 * 64) % 512).reshape(64, 2, 64) / 16.0
        x[256:320, 0, ::7] = np.inf
        x[256:320, 1, ::5] = np.nan
        x[320:384] = np.nan
        x[384:448] = -np.inf
        x[448:512, 0] = -0.0
        x[512:] *= np.float32(2.0 ** 100)
    y = _torch(x, dtype)
    nb, buf = _buffers(jet, host, dims, 0)
    jet.jet_quantize_kv_e4m3(lay, dims, y, y, *buf)
    back = [torch.empty_like(y) for _ in range(2)]
    jet.jet_dequantize_kv_e4m3(lay, dims, *buf, *back)
    torch.cuda.synchronize()
    cache = K.Cache(P, heads, d).write(_np(y))
    for i in range(2):
        got = buf[i].cpu().numpy()
        want = cache.buffer(0)
        nan = (want[:P[0] * heads * d] & 0x7F) == 0x7F   # a NaN code has either sign
        got[:P[0] * heads * d][nan] &= 0x7F
        np.testing.assert_array_equal(got[:nb], want)
        np.testing.assert_array_equal(_np(back[i]), cache.values())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128, 256])
def test_append(jet, dtype, d):
    # single tokens, pieces that begin and end anywhere, requests without new tokens,
    # growing magnitudes so that exponents of begun blocks grow, by a little and by much
    import torch
    P, heads = [200, 1, 130, 64, 77], 3
    rng = np.random.default_rng(d)
    host, lay, dims = _batch(jet, P, dtype=dtype, Hkv=heads, d=d)
    nb, buf = _buffers(jet, host, dims, 0x5A)
    caches = [K.Cache(P, heads, d) for _ in range(2)]
    at, step = np.zeros(len(P), int), 0
    while (at < P).any():
        most = [1, 70, 3, 200, 1, 1, 40][step % 7]
        new = np.minimum(np.array(P) - at, rng.integers(0, most + 1, len(P)))
        n = int(new.sum())
        scale = 2.0 ** (step % 5 * (40 if step % 4 == 3 else 1))
        x = [_torch(_tokens(rng, n, heads, d) * scale, dtype) for _ in range(2)]
        off = np.concatenate([[0], np.cumsum(new)])
        words = [torch.tensor(w, dtype=torch.int32, device="cuda") for w in (at, off)]
        jet.jet_append_kv_e4m3(lay, dims, *words, *x, *buf)
        for r in range(len(P)):
            for i in range(2):
                caches[i].append(r, int(at[r]), _np(x[i])[off[r]:off[r + 1]])
        at, step = at + new, step + 1
        torch.cuda.synchronize()
        assert jet.jet_device_status() == 0
        for i in range(2):
            codes = buf[i].cpu().numpy()[:sum(P) * heads * d].reshape(-1, heads, d)
            held = np.concatenate([np.arange(p) < a for p, a in zip(P, at)])
            np.testing.assert_array_equal(codes[held], caches[i].codes[held])
            assert np.all(codes[~held] == 0x5A)  # the tokens to come: as they were
    for i in range(2):
        _check_buffer(buf[i], caches[i], nb, 0x5A)


def test_append_leaves_out_words_that_do_not_fit(jet):
    # requests whose new tokens end past their prefix, start before it or lie outside
    # the rows given are left out and reported; the others are written
    import torch
    P, heads, d = [100, 50, 70, 64], 2, 64
    host, lay, dims = _batch(jet, P, dtype="bf16", Hkv=heads, d=d)
    x = _torch(np.ones((9, heads, d)), "bf16")
    cases = [([98, 0, 0, 0], [0, 3, 6, 9, 9], [1, 2]), ([0, -1, 0, 0], [0, 3, 6, 9, 9], [0, 2]),
             ([0, 0, 0, 0], [0, 3, 6, 30, 40], [0, 1]), ([0, 0, 0, 0], [0, 3, 2, 5, 9], [0, 2, 3]),
             ([2 ** 31 - 1, 0, 0, 0], [0, 3, 6, 9, 9], [1, 2]),
             ([0, 0, 0, 0], [-5, 3, 6, 9, 9], [1, 2])]
    for start, off, done in cases:
        nb, buf = _buffers(jet, host, dims, 0)
        words = [torch.tensor(w, dtype=torch.int32, device="cuda") for w in (start, off)]
        jet.jet_append_kv_e4m3(lay, dims, *words, x, x, *buf)
        torch.cuda.synchronize()
        assert jet.jet_device_status() == JET_ERR_DEVICE
        cache = K.Cache(P, heads, d)
        for r in done:
            cache.append(r, start[r], _np(x)[off[r]:off[r + 1]])
        for b in buf:
            _check_buffer(b, cache, nb, 0)


# ---------------------------------------------------------------------------
# the attention
# ---------------------------------------------------------------------------
class Case:
    """A batch with its caches written, ready for jet_prefix_attend_e4m3."""

    def __init__(self, jet, P, n_cand, cand_len, dtype, Hq, Hkv, d, seed, k_scale=1.0):
        import torch
        self.jet, self.P, self.Hq, self.Hkv, self.d = jet, P, Hq, Hkv, d
        self.dtype = dtype
        self.host, self.lay, self.dims = _batch(jet, P, n_cand, cand_len, dtype=dtype, Hq=Hq,
                                                Hkv=Hkv, d=d)
        self.ref = O.build_layout(P, n_cand, cand_len, [0] * int(np.sum(cand_len)), 2)
        n = self.host.sizes
        rng = np.random.default_rng(seed)
        self.k = _tokens(rng, n.total_prefix, Hkv, d, 0.3) * k_scale
        self.v = _tokens(rng, n.total_prefix, Hkv, d, 0.3)
        self.q = _torch(rng.standard_normal((n.N, Hq, d)), dtype)
        self.kc = _torch(_tokens(rng, n.N - n.R, Hkv, d, 0.3), dtype)
        self.vc = _torch(_tokens(rng, n.N - n.R, Hkv, d, 0.3), dtype)
        self.o = torch.full((n.N, Hq, d), 99.0, dtype=self.q.dtype, device="cuda")
        self.need = jet.jet_attend_workspace_bytes_e4m3(n, self.dims)
        self.ws = torch.full((self.need + GUARD,), 0x5A, dtype=torch.uint8, device="cuda")
        self.quantise()

    def quantise(self):
        self.k8, self.v8 = _buffers(self.jet, self.host, self.dims, 0xFF)[1]
        k, v = _torch(self.k, self.dtype), _torch(self.v, self.dtype)
        self.jet.jet_quantize_kv_e4m3(self.lay, self.dims, k, v, self.k8, self.v8)
        self.kd = K.Cache(self.P, self.Hkv, self.d).write(_np(k)).values()
        self.vd = K.Cache(self.P, self.Hkv, self.d).write(_np(v)).values()

    def run(self, stream=None):
        self.jet.jet_prefix_attend_e4m3(self.lay, self.dims, self.q, self.k8, self.v8, self.kc,
                                        self.vc, self.o, self.ws, ws_bytes=self.need,
                                        stream=stream)

    def result(self):
        import torch
        self.run()
        torch.cuda.synchronize()
        assert self.jet.jet_device_status() == 0
        assert bool((self.ws[self.need:] == 0x5A).all())
        return _np(self.o)

    def check(self, got, rows=None):
        rows = list(range(len(got))) if rows is None else rows
        want = O.cascade_attention(self.ref, _np(self.q), self.kd, self.vd, _np(self.kc),
                                   _np(self.vc), self.Hq, self.Hkv, rows=rows)
        err = np.abs(got[rows] - want)
        assert np.all(err <= self.bar(rows)[..., None]), (err.max(), self.bar(rows).min())

    def bar(self, rows):
        """The error allowed to a row's head. Scores are sums of d products of
        which float32 makes an error of at most (d + 4) 2^-24 of the sum of
        magnitudes; the exponential of a base-2 score adds 2^-22 relative; together
        delta per weight, in the numerator and in the sum, with 2^-24 for each of
        the sums' terms. bf16 outputs round by 2^-8 of themselves; bf16 also rounds
        each weight by 2^-8 for the product with the values, which moves an average
        by at most twice that, and holds the queries as two e4m3 numbers, which
        leaves 2^-18 of the row's largest element (2^-10 of a scale of which it
        takes at least 224)."""
        q, g = np.abs(_np(self.q)), self.Hq // self.Hkv
        out = np.zeros((len(rows), self.Hq))
        for i, n in enumerate(rows):
            r = int(self.ref["row_req"][n])
            p0, p1 = (int(self.ref["prefix_offset"][r + j]) for j in (0, 1))
            f0, f1 = (int(self.ref["row_offset"][r + j]) - r - j for j in (0, 1))
            for h in range(self.Hq):
                kk = np.abs(np.concatenate([self.kd[p0:p1, h // g], _np(self.kc)[f0:f1, h // g]]))
                vmax = max(np.abs(self.vd[p0:p1, h // g]).max(),
                           np.abs(_np(self.vc)[f0:f1, h // g]).max(initial=0.0))
                delta = (self.d + 4) * 2.0 ** -24 * (kk @ q[n, h]).max() / self.d ** 0.5
                delta += 2.0 ** -22 + (len(kk) + 16) * 2.0 ** -24
                b = 2 * delta * vmax
                if self.dtype == "bf16":
                    coarse = 2.0 ** -17.8 * q[n, h].max() * kk.sum(1).max() / self.d ** 0.5
                    b += (2 * coarse + 3 * 2.0 ** -8) * vmax
                out[i, h] = b + 2.0 ** -24 * vmax
        return out


ATTEND = [
    # prefixes around the 64-token block, one row a request
    ([1, 63, 64, 65, 128, 129], [1] * 6, [1] * 6, dict(Hq=8, Hkv=2, d=64)),
    # candidates of many lengths, some rows past one block of 128 vectors
    ([200, 700, 30], [3, 2, 4], [5, 1, 9, 12, 2, 1, 1, 40, 3], dict(Hq=8, Hkv=2, d=128)),
    ([300, 77], [10, 10], [3] * 20, dict(Hq=16, Hkv=2, d=256)),
    # odd groups of heads, one kv head, as many as query heads
    ([500, 33], [2, 3], [4, 2, 1, 6, 3], dict(Hq=7, Hkv=1, d=256)),
    ([129, 450], [2, 2], [1, 2, 3, 4], dict(Hq=15, Hkv=3, d=128)),
    ([90, 2], [2, 2], [2, 2, 8, 1], dict(Hq=6, Hkv=6, d=64)),
    ([260, 5], [1, 2], [2, 1, 3], dict(Hq=128, Hkv=1, d=64)),
    # one long prefix (many chunks), and more items than SMs of uneven length
    ([5000], [2], [6, 3], dict(Hq=16, Hkv=2, d=256)),
    ([6100, 20], [1, 1], [1, 2], dict(Hq=8, Hkv=8, d=128)),
    ([20 + 37 * i % 800 for i in range(60)], [2] * 60, [1 + i % 5 for i in range(120)],
     dict(Hq=24, Hkv=4, d=64)),
    ([1500 + 311 * i for i in range(12)], [2] * 12, [3] * 24, dict(Hq=32, Hkv=8, d=128)),
    # a candidate of many tokens: several tiles of own keys, rows that see few of them
    ([100], [2], [180, 50], dict(Hq=4, Hkv=2, d=256)),
]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("case", range(len(ATTEND)))
def test_attention(jet, dtype, case):
    P, n_cand, cand_len, dims = ATTEND[case]
    c = Case(jet, P, n_cand, cand_len, dtype, seed=case, **dims)
    got = c.result()
    rng = np.random.default_rng(case)
    rows = list(range(len(got))) if len(got) * dims["Hq"] <= 400 else \
        sorted(set(rng.integers(0, len(got), 24).tolist()) | {0, len(got) - 1})
    c.check(got, rows)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128, 256])
def test_growing_maximum_and_scales(jet, dtype, d):
    # the scores' spread grows along the prefix, so running maxima keep growing, and
    # so do the blocks' exponents, of keys upwards and of values downwards
    c = Case(jet, [900, 333], [2, 2], [4, 3, 2, 5], dtype, 8, 2, d, seed=20)
    pos = np.concatenate([np.arange(900), np.arange(333)])[:, None, None]
    c.k = (c.k * (1.0 + pos / 8.0) * 0.2).astype(np.float32)
    c.v = (c.v * 2.0 ** -(pos // 40.0)).astype(np.float32)
    c.quantise()
    c.check(c.result())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128, 256])
def test_one_key_outweighs_a_long_prefix(jet, dtype, d):
    # the first key's score is some nine powers of e above the others': their weights
    # are small against its, and together they count all the same
    c = Case(jet, [4000], [1], [2], dtype, 4, 1, d, seed=21)
    c.q[:] = _torch(np.abs(_np(c.q)) * 0.2, dtype)
    c.k *= 0.05
    c.k[0] = 1.0
    c.k[0] *= 9.0 / (_np(c.q).mean() * d ** 0.5)
    c.quantise()
    c.check(c.result())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128, 256])
def test_hidden_places_stay_hidden(jet, dtype, d):
    # NaN and infinities in the other request's prefix (the rest of a tile), in the
    # places of blocks that no request has and in the padding reach nobody
    P = [70, 100, 65]
    c = Case(jet, P, [2] * 3, [3] * 6, dtype, 8, 2, d, seed=22)
    clean = c.result()
    c.k[70:170], c.v[70:170] = np.nan, np.inf
    c.quantise()
    got = c.result()
    rows = [n for n in range(len(got)) if c.ref["row_req"][n] != 1]
    np.testing.assert_array_equal(got[rows], clean[rows])
    bad = [n for n in range(len(got)) if c.ref["row_req"][n] == 1]
    assert np.isnan(got[bad]).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("P", [100, 3000])
def test_non_finite_elements_reach_their_outputs(jet, dtype, P):
    # a NaN key makes the outputs of its kv head NaN; a non-finite value its column
    c = Case(jet, [P], [2], [3, 2], dtype, 8, 2, 128, seed=23)
    c.k[P // 3, 1, 5] = np.nan
    c.quantise()
    got = c.result()
    assert np.isfinite(got[:, :4]).all() and np.isnan(got[:, 4:]).all()
    c = Case(jet, [P], [2], [3, 2], dtype, 8, 2, 128, seed=23)
    c.v[P // 3, 1, 5] = np.inf
    c.quantise()
    got = c.result()
    assert np.isnan(got[:, 4:, 5]).all()
    got[:, 4:, 5] = 0
    assert np.isfinite(got).all()
    # a query of a NaN: its own head's output alone
    c = Case(jet, [P], [2], [3, 2], dtype, 8, 2, 128, seed=23)
    c.q[1, 6, 3] = float("nan")
    got = c.result()
    assert np.isnan(got[1, 6]).all()
    got[1, 6] = 0
    assert np.isfinite(got).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_query_scales(jet, dtype):
    # rows of very small and very large queries, and rows of zeros
    c = Case(jet, [300], [2], [6, 6], dtype, 8, 2, 128, seed=24, k_scale=0.01)
    q = _np(c.q)
    q[1], q[2], q[3] = q[1] * 2.0 ** -100, q[2] * 2.0 ** 8, 0.0
    q[4, :, ::2] = 0.0
    c.q = _torch(q, dtype)
    c.check(c.result())


def test_streams_and_graphs(jet):
    # on another stream, captured and replayed on new inputs; two captures that share
    # the workspace, replayed one after the other; results are the eager ones
    import torch
    cases = [Case(jet, [300, 1200], [2, 2], [4, 3, 2, 5], "bf16", 8, 2, d, seed=30 + d)
             for d in (128, 256)]
    need = max(c.need for c in cases)
    ws = torch.empty(need, dtype=torch.uint8, device="cuda")
    want = [c.result() for c in cases]
    s = torch.cuda.Stream()
    graphs = []
    for c in cases:
        c.ws = ws
        c.o.zero_()
        torch.cuda.synchronize()
        with torch.cuda.stream(s):
            c.run()                    # the current stream
        s.synchronize()
        np.testing.assert_array_equal(_np(c.o), want[cases.index(c)])
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=s):
            k, v = _torch_pair(c)
            jet.jet_quantize_kv_e4m3(c.lay, c.dims, k, v, c.k8, c.v8)
            c.run()
        graphs.append((g, k, v))
    for c, (g, k, v) in zip(cases, graphs):
        for t, x in ((k, c.k), (v, c.v)):
            t.copy_(_torch(x, "bf16"))
        c.o.zero_()
        for b in (c.k8, c.v8):
            b.zero_()
    for _ in range(2):
        for g, _, _ in graphs:
            g.replay()
    torch.cuda.synchronize()
    assert jet.jet_device_status() == 0
    for c, w in zip(cases, want):
        np.testing.assert_array_equal(_np(c.o), w)


def _torch_pair(c):
    import torch
    n = c.host.sizes.total_prefix
    return [torch.empty(n, c.Hkv, c.d, dtype=torch.bfloat16, device="cuda") for _ in range(2)]


def test_attention_of_words_past_the_plan(jet):
    # words that hold a longer prefix than the sizes the workspace was planned for: that
    # request is left out and reported, the others get their answers
    import torch
    for dtype, planned, worded, dims in (
            ("bf16", [128, 100], [150, 78], dict(Hq=8, Hkv=2, d=64)),
            ("bf16", [500, 460, 300], [660, 300, 300], dict(Hq=16, Hkv=2, d=128)),
            ("f32", [128, 100], [150, 78], dict(Hq=8, Hkv=2, d=64))):
        R = len(planned)
        c = Case(jet, worded, [2] * R, [3] * (2 * R), dtype, seed=40, **dims)
        host, lay, _ = _batch(jet, planned, [2] * R, [3] * (2 * R), dtype=dtype, **dims)
        words = jet.jet_layout_build(worded, [2] * R, [3] * (2 * R), [0] * (6 * R), 2).words
        lay.words.copy_(torch.from_numpy(words.copy()))
        c.lay, c.need = lay, jet.jet_attend_workspace_bytes_e4m3(host.sizes, c.dims)
        c.ws = torch.full((c.need + (8 << 20),), 0x5A, dtype=torch.uint8, device="cuda")
        c.run()
        torch.cuda.synchronize()
        assert jet.jet_device_status() == JET_ERR_DEVICE
        assert bool((c.ws[c.need:] == 0x5A).all())
        rows = [n for n in range(c.ref["N"]) if c.ref["row_req"][n] != 0]
        c.check(_np(c.o), rows)


# ---------------------------------------------------------------------------
# together, as a scorer uses them
# ---------------------------------------------------------------------------
def test_step_over_an_8bit_cache(jet):
    """The prefix written in two pieces, the step over the caches, against the step
    over the caches read back; then the same batch from pinned host buffers."""
    import torch

    import jet_synth
    from gpu_common import TOL_LOGPROB, build_step, dims_for
    from paper_2609_33874_gb300.step import (HostBatch, HostResults, ScoringStep,
                                             quantize_prefix)
    p = jet_synth.make_problem("dense27b_mc", R=5)
    full, x, w_lm = build_step(jet, p)
    w = p.work
    host = full.host_layout
    step = ScoringStep(host, dims_for(jet, w), jet.MODES[w.mode], kv="e4m3")
    k8, v8 = quantize_prefix(step.layout, step.dims, x["k_pre"], x["v_pre"])
    # the same caches in two pieces, the first ending at a block's end: no code differs
    nb = jet.jet_kv_e4m3_bytes(host.sizes, step.dims)
    pieces = [torch.zeros(nb, dtype=torch.uint8, device="cuda") for _ in range(2)]
    P = np.asarray(p.prefix_len)
    p0 = np.concatenate([[0], np.cumsum(P)])
    cut = P // 128 * 64
    for a, b in ((np.zeros_like(P), cut), (cut, P)):
        rows = torch.from_numpy(np.concatenate(
            [np.arange(s + i, s + j) for s, i, j in zip(p0, a, b)])).cuda()
        off = torch.from_numpy(np.concatenate([[0], np.cumsum(b - a)]).astype(np.int32)).cuda()
        jet.jet_append_kv_e4m3(step.layout, step.dims, torch.from_numpy(a.astype(np.int32)).cuda(),
                               off, x["k_pre"][rows], x["v_pre"][rows], *pieces)
    n = int(p0[-1]) * w.Hkv * w.d
    assert torch.equal(pieces[0][:n], k8[:n]) and torch.equal(pieces[1][:n], v8[:n])
    x8 = dict(x, k_pre=pieces[0], v_pre=pieces[1])
    step.run(x8, w_lm)
    back = {k: torch.empty_like(x[k]) for k in ("k_pre", "v_pre")}
    jet.jet_dequantize_kv_e4m3(step.layout, step.dims, *pieces, back["k_pre"], back["v_pre"])
    full.run(dict(x, **back), w_lm)
    torch.cuda.synchronize()
    assert jet.jet_device_status() == 0
    # both round weights and outputs to bf16: 3 x 2^-8 of the largest value each
    vmax = float(torch.maximum(back["v_pre"].abs().max(), x["v_cand"].abs().max()))
    assert float((step.o.float() - full.o.float()).abs().max()) <= 6 * 2.0 ** -8 * vmax
    # the LM head takes its own hidden states here
    assert float((step.cand_score - full.cand_score).abs().max()) <= TOL_LOGPROB
    want = step.o.clone()
    batch = HostBatch(step, {k: x8[k].cpu() for k in step.input_names()},
                      torch.from_numpy(host.words))
    assert batch.nbytes < sum(x[k].nbytes for k in step.input_names())
    out = [HostResults(step) for _ in range(3)]
    step.o.zero_()
    step.run_pipelined([batch] * 3, w_lm, out)
    torch.cuda.synchronize()
    assert torch.equal(step.o, want)
    np.testing.assert_array_equal(out[2]["cand_score"].numpy(), step.cand_score.cpu().numpy())


def test_step_rejects_unknown_caches(jet):
    from paper_2609_33874_gb300.step import ScoringStep
    host, _, dims = _batch(jet, [5], dtype="bf16", Hq=2, Hkv=1, d=64)
    with pytest.raises(ValueError):
        ScoringStep(host, dims, jet.DECIDE_ARGMAX, kv="int8")
