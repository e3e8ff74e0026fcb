"""The 8-bit prefix cache's attention where its plan and its roles change: few query
vectors over much cache, held several times over; candidates' values and keys that are
not finite and reach only the rows that see them; values of very small, very large and
very different scales; caches past 2^31 codes; calls side by side; waits that run out."""
import numpy as np
import pytest

import oracle as O
from oracle import kv_e4m3 as K
from test_gpu_kv_cache import Case, _batch, _buffers, _check_buffer, _np, _tokens, _torch

pytestmark = pytest.mark.gpu

JET_OK, JET_ERR_TIMEOUT = 0, 9


def _some_rows(c, seed, n=24):
    rng = np.random.default_rng(seed)
    total = c.ref["N"]
    return sorted(set(rng.integers(0, total, n).tolist()) | {0, total - 1})


# query heads a kv head, and the rows of the requests with the most: 32 and 64 vectors
# bound the plans with four and two copies, 128 query heads fill a block
FEW = [
    (4, 8), (1, 32), (1, 33), (32, 1), (33, 1), (7, 4), (3, 11), (16, 4), (9, 7), (2, 32),
    (64, 1), (65, 1), (13, 5), (5, 6),
]


@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("g,rows", FEW)
def test_few_vectors_over_much_cache(jet, d, g, rows):
    # long prefixes in chunks, short ones in one, requests of one row beside the largest
    Hkv = 8
    P = [3100, 1, 64, 500, 1900, 129, 700, 63, 1100]
    n = [1] * len(P)
    lens = [rows if i % 3 == 0 else 1 + i % rows for i in range(len(P))]
    assert sum(P) * Hkv > 3 * 128 * 152
    c = Case(jet, P, n, lens, "bf16", g * Hkv, Hkv, d, seed=g * 100 + rows)
    most = 4 if rows * g <= 32 else 2 if rows * g <= 64 else 1
    per = c.ref["N"] * c.Hq * (4 * d + 8)      # a partial of every row and head
    assert c.need >= (most if d < 256 else 0) * per
    c.check(c.result(), _some_rows(c, rows, 8))


@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("rows,copies", [([30, 1, 2, 2, 1, 2, 4, 1, 2], 4),
                                         ([60, 5, 10, 8, 9, 10, 12, 3, 9], 2),
                                         ([61, 5, 10, 8, 9, 10, 12, 3, 9], 1),
                                         ([65, 1, 2, 1, 1, 1, 2, 1, 1], 1)])
def test_one_request_of_many_rows(jet, d, rows, copies):
    # a block holds the usual request's vectors several times over, and the one with many
    # rows takes several blocks; past that plan's bounds one block holds 128 vectors
    P = [1700, 1, 64, 500, 1900, 129, 700, 2063, 1100]
    c = Case(jet, P, [1] * 9, rows, "bf16", 32, 8, d, seed=9)
    per = c.ref["N"] * c.Hq * (4 * d + 8)
    assert c.need % ((copies if d < 256 else 1) * per) == 0
    last = int(c.ref["row_offset"][1]) - 1
    c.check(c.result(), sorted(set(_some_rows(c, 2, 10)) | {last, last // 2}))


@pytest.mark.parametrize("d", [64, 128])
def test_few_vectors_of_unsplit_prefixes(jet, d):
    # more items than SMs, each request one chunk: the copies' partials are joined alone
    P = [40 + 67 * i % 300 for i in range(60)]
    lens = [1 + i % 4 for i in range(60)]
    c = Case(jet, P, [1] * 60, lens, "bf16", 32, 8, d, seed=7)
    c.check(c.result(), _some_rows(c, 1))


@pytest.mark.parametrize("d", [64, 128, 256])
def test_one_very_long_prefix(jet, d):
    # more partials of a row than a warp of the combine has lanes
    c = Case(jet, [40000, 3], [1, 1], [3, 1], "bf16", 8, 2, d, seed=8)
    per = c.ref["N"] * c.Hq * (4 * d + 8)
    assert c.need > 64 * per
    c.check(c.result())


def _seen(c, n):
    """The candidates' tokens that row n sees, as rows of k_cand and v_cand."""
    r = int(c.ref["row_req"][n])
    cand = int(c.ref["row_cand"][n])
    if cand < 0:
        return []
    first = int(c.ref["cand_row_offset"][cand]) - r - 1
    return list(range(first, n - r))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d,few", [(64, 0), (128, 0), (256, 0), (64, 1), (128, 1)])
def test_candidates_that_are_not_finite(jet, dtype, d, few):
    # an infinite value reaches its column in the rows that see it, a NaN key whole rows
    # of its kv head, and no other row, of the same request or of another, differs by
    # more than two calls may
    Hkv, Hq = (8, 8) if few else (2, 8)
    P = [4000, 3000, 900] if few else [90, 700, 64]
    args = (P, [3] * 3, [4, 1, 3, 2, 2, 5, 9, 2, 40 if not few else 3], dtype, Hq, Hkv, d)
    clean = Case(jet, *args, seed=50)
    rows = list(range(clean.ref["N"]))
    want = clean.result()
    slack = 2 * clean.bar(rows)
    for what in ("value", "key"):
        c = Case(jet, *args, seed=50)
        tok = 3                                  # of request 0's third candidate
        seers = [n for n in rows if tok in _seen(c, n)]
        assert seers and len(seers) < len(rows)
        if what == "value":
            c.vc[tok, 1, 3], c.vc[tok, 1, 5] = float("inf"), float("nan")
            c.vc[tok, 1, 7] = float("-inf")
        else:
            c.kc[tok, 1, 2] = float("nan")
        got = c.result()
        heads = list(range(Hq // Hkv, 2 * Hq // Hkv))
        for n in seers:
            for h in heads:
                if what == "key":
                    assert np.isnan(got[n, h]).all()
                else:
                    assert got[n, h, 3] == np.inf and np.isnan(got[n, h, 5])
                    assert got[n, h, 7] == -np.inf
                    got[n, h, [3, 5, 7]] = want[n, h, [3, 5, 7]]
                if what == "key":
                    got[n, h] = want[n, h]
        assert np.all(np.abs(got - want) <= slack[..., None])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("low,high", [(-110, -110), (110, 110), (-60, 60), (-125, 0), (0, 30)])
def test_values_of_all_scales(jet, dtype, d, low, high):
    # the prefix's values around 2^low, the candidates' around 2^high, blocks of the prefix
    # of zeros: the outputs follow the larger, whichever a row sees
    c = Case(jet, [200, 70], [2, 1], [3, 2, 6], dtype, 8, 2, d, seed=60)
    c.v = np.clip(c.v, -4, 4) * np.float32(2.0 ** low)
    c.v[64:128] = 0.0
    c.quantise()
    c.vc = _torch(np.clip(_np(c.vc), -4, 4) * 2.0 ** high, dtype)
    _check_by_what_rows_see(c, c.result())


def _check_by_what_rows_see(c, got, rows=None):
    """As Case.check, the bar taken of what a row sees: the batch's other candidates,
    however large, add nothing to its error."""
    rows = list(range(len(got))) if rows is None else rows
    want = O.cascade_attention(c.ref, _np(c.q), c.kd, c.vd, _np(c.kc), _np(c.vc), c.Hq, c.Hkv,
                               rows=rows)
    kc, vc = c.kc.clone(), c.vc.clone()
    for i, n in enumerate(rows):
        hidden = sorted(set(range(len(vc))) - set(_seen(c, n)))
        c.kc, c.vc = kc.clone(), vc.clone()
        c.kc[hidden], c.vc[hidden] = 0.0, 0.0
        assert np.all(np.abs(got[n] - want[i]) <= c.bar([n])[0][:, None]), n
    c.kc, c.vc = kc, vc


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("size", [600.0, 3e5, 1e30, 3e37])
def test_large_values_stay_with_their_rows(jet, dtype, d, size):
    # one candidate's values (and those of one token in the middle of a long one) are far
    # larger than all others
    c = Case(jet, [150, 64], [3, 2], [4, 6, 2, 3, 150], dtype, 8, 2, d, seed=62)
    for tok in (3, 4, 5, 6, 7, 60):
        c.vc[tok] = c.vc[tok].sign() * size
    _check_by_what_rows_see(c, c.result())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128, 256])
def test_large_values_in_every_item(jet, dtype, d):
    # more items than SMs, and in two requests of three one candidate's values far above
    # the others': a CTA's later items take the slower way as its first ones do
    R = 90
    P = [20 + 53 * i % 400 for i in range(R)]
    c = Case(jet, P, [2] * R, [3] * (2 * R), dtype, 8, 4, d, seed=63)
    for r in range(R):
        if r % 3 < 2:
            c.vc[4 * r:4 * r + 2] *= 1e5 if r % 3 else 3e20   # the first candidate's tokens
    got = c.result()
    rng = np.random.default_rng(1)
    _check_by_what_rows_see(c, got, sorted(rng.choice(len(got), 40, replace=False).tolist()))


def test_zero_values_and_queries(jet):
    for d in (64, 128, 256):
        c = Case(jet, [130], [1], [3], "bf16", 8, 2, d, seed=61)
        c.v[:] = 0.0
        c.quantise()
        c.vc.zero_()
        c.q.zero_()
        assert not c.result().any()


@pytest.mark.parametrize("heads,d", [(8, 256)])
def test_caches_past_32_bits(jet, heads, d):
    # 2^31 codes end before the last request: written, read back and attended to there
    import torch
    P = [8192] * 131 + [77, 300]
    if torch.cuda.mem_get_info()[0] < 60 << 30:
        pytest.skip("no memory for it")
    assert sum(P[:-2]) * heads * d > 2 ** 31
    rng = np.random.default_rng(70)
    host, lay, dims = _batch(jet, P, dtype="bf16", Hq=16, Hkv=heads, d=d)
    n = host.sizes
    nb = jet.jet_kv_e4m3_bytes(n, dims)
    k, v = (torch.zeros(n.total_prefix, heads, d, dtype=torch.bfloat16, device="cuda")
            for _ in range(2))
    c = Case(jet, P[-2:], [1, 1], [1, 1], "bf16", 16, heads, d, seed=71)
    tail = sum(P[-2:])
    k[-tail:], v[-tail:] = _torch(c.k, "bf16"), _torch(c.v, "bf16")
    k8, v8 = (torch.empty(nb, dtype=torch.uint8, device="cuda") for _ in range(2))
    jet.jet_quantize_kv_e4m3(lay, dims, k, v, k8, v8)
    k.fill_(1.0)
    v.fill_(1.0)
    jet.jet_dequantize_kv_e4m3(lay, dims, k8, v8, k, v)
    np.testing.assert_array_equal(_np(k[-tail:]), c.kd)
    np.testing.assert_array_equal(_np(v[-tail:]), c.vd)
    assert not bool(k[:-tail].any()) and not bool(v[:-tail].any())
    # the last request's last 40 tokens again, as appended ones
    start = torch.tensor(P[:-1] + [260], dtype=torch.int32, device="cuda")
    off = torch.tensor([0] * len(P) + [40], dtype=torch.int32, device="cuda")
    new = _torch(_tokens(rng, 40, heads, d, 0.2), "bf16")
    before = k8.clone()
    jet.jet_append_kv_e4m3(lay, dims, start, off, new, new, k8, v8)
    first = (n.total_prefix - 40 - 4) * heads * d       # the last block has 44 tokens
    assert torch.equal(k8[:first], before[:first])
    del before, k, v
    for i, b in enumerate((k8, v8)):
        cache = K.Cache(P[-2:], heads, d).write((_np(_torch((c.k, c.v)[i], "bf16"))))
        cache.append(1, 260, _np(new))
        got = b[(n.total_prefix - tail) * heads * d:n.total_prefix * heads * d].cpu().numpy()
        np.testing.assert_array_equal(got.reshape(-1, heads, d), cache.codes)
        if i:
            c.vd = cache.values()
        else:
            c.kd = cache.values()
    q = torch.zeros(n.N, 16, d, dtype=torch.bfloat16, device="cuda")
    q[-2:] = c.q
    o = torch.full_like(q, 9.0)
    none = torch.zeros(0, heads, d, dtype=torch.bfloat16, device="cuda")
    ws = torch.empty(jet.jet_attend_workspace_bytes_e4m3(n, dims), dtype=torch.uint8, device="cuda")
    jet.jet_prefix_attend_e4m3(lay, dims, q, k8, v8, none, none, o, ws)
    torch.cuda.synchronize()
    assert jet.jet_device_status() == JET_OK
    assert not bool(o[:-2].any())
    c.check(_np(o[-2:]))


def test_calls_side_by_side(jet):
    # two batches on two streams at once, each with its caches and workspace, again and
    # again: the results are those of calls one after another
    import torch
    cases = [Case(jet, P, [1] * len(P), [2] * len(P), "bf16", 32, 8, d, seed=80 + d)
             for P, d in (([3000, 2000, 2500, 40], 128), ([900] * 9, 64), ([5000, 30], 256))]
    want = [c.result() for c in cases]
    streams = [torch.cuda.Stream() for _ in cases]
    for c in cases:
        c.o.zero_()
    torch.cuda.synchronize()
    for _ in range(20):
        for c, s in zip(cases, streams):
            c.run(stream=s.cuda_stream)
    torch.cuda.synchronize()
    assert jet.jet_device_status() == JET_OK
    for c, w in zip(cases, want):
        np.testing.assert_array_equal(_np(c.o), w)


@pytest.mark.parametrize("d,P,Hkv", [(64, [900, 100], 2), (128, [3000, 5000], 8),
                                     (256, [4000, 9000], 2), (256, [300], 4)])
def test_a_wait_that_runs_out_is_reported(jet, d, P, Hkv):
    # the first query block never lands: the call returns and reports it, and the next
    # one on the same context gives the answer
    import torch
    c = Case(jet, P, [2] * len(P), [3, 2] * len(P), "bf16", 4 * Hkv, Hkv, d, seed=90)
    want = c.result()
    budget = jet.jet_set_wait_budget_ns(1_000_000)
    jet.jet_set_test_stall(True)
    try:
        for _ in range(2):
            c.run()
            torch.cuda.synchronize()
            assert jet.jet_device_status() == JET_ERR_TIMEOUT
    finally:
        jet.jet_set_test_stall(False)
        jet.jet_set_wait_budget_ns(budget)
    np.testing.assert_array_equal(c.result(), want)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_many_heads_a_block(jet, dtype):
    # one block's pairs of (keys or values, head) do not divide by what a CTA takes, and
    # there are enough of them for it to take several
    P, heads, d = [64 * 9 + 5] * 40, 7, 64
    rng = np.random.default_rng(95)
    import torch
    host, lay, dims = _batch(jet, P, dtype=dtype, Hkv=heads, d=d)
    x = [_torch(_tokens(rng, sum(P), heads, d), dtype) for _ in range(2)]
    x[0][100, 2, 3] = float("inf")               # a second maximum in the middle of a CTA's
    nb, buf = _buffers(jet, host, dims, 0x11)
    jet.jet_quantize_kv_e4m3(lay, dims, *x, *buf)
    back = [torch.empty_like(t) for t in x]
    jet.jet_dequantize_kv_e4m3(lay, dims, *buf, *back)
    torch.cuda.synchronize()
    for i in range(2):
        cache = K.Cache(P, heads, d).write(_np(x[i]))
        _check_buffer(buf[i], cache, nb, 0x11)
        np.testing.assert_array_equal(_np(back[i]), cache.values())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 256])
def test_append_to_many_requests(jet, dtype, d):
    # enough requests for a CTA to take two of a block's pairs; every start and length
    # within two blocks, exponents that grow in some heads only
    import torch
    R, heads = 300, 5
    rng = np.random.default_rng(96)
    P = rng.integers(1, 140, R).tolist()
    host, lay, dims = _batch(jet, P, dtype=dtype, Hkv=heads, d=d)
    nb, buf = _buffers(jet, host, dims, 0x77)
    caches = [K.Cache(P, heads, d) for _ in range(2)]
    at = np.zeros(R, int)
    for step in range(3):
        new = np.minimum(np.array(P) - at, rng.integers(0, 80, R) if step < 2 else 140)
        off = np.concatenate([[0], np.cumsum(new)])
        scale = np.float32(4.0) ** rng.integers(-3, 4, (1, heads, 1))
        x = [_torch(_tokens(rng, int(off[-1]), heads, d) * scale, dtype) for _ in range(2)]
        words = [torch.tensor(w, dtype=torch.int32, device="cuda") for w in (at, off)]
        jet.jet_append_kv_e4m3(lay, dims, *words, *x, *buf)
        for i in range(2):
            rows = _np(x[i])
            for r in range(R):
                if new[r]:
                    caches[i].append(r, int(at[r]), rows[off[r]:off[r + 1]])
        at = at + new
    torch.cuda.synchronize()
    assert jet.jet_device_status() == JET_OK
    for i in range(2):
        _check_buffer(buf[i], caches[i], nb, 0x77)
