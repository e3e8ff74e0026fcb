"""Performance cases of the 8-bit prefix cache: writing it, appending to it,
reading it back, and the scoring step's attention over it.

The prefix keys and values of a batch are packed [tokens, kv heads, d], request
after request. Their 8-bit form holds an e4m3 code per element and one
power-of-two exponent X per (block of 64 tokens of a request, kv head), for keys
and values apart:

    X     the least integer in [-117, 119] with max |x| <= 448 * 2^X
    code  e4m3(x * 2^-X), to nearest even;  value = code * 2^X

in one buffer: the codes [tokens, kv heads, d], padded to a multiple of 256
bytes, then the bytes X + 127 [tokens // 64 + requests, kv heads], block b of
request r at place first_token[r] // 64 + r + b, padded likewise. Appending to a
block that holds tokens keeps the larger of its exponent and the new tokens',
and rounds its codes again where the exponent grows.

A case holds the batch structure as plain values: ``requests`` contexts of
``prefix_lo`` to ``prefix_hi`` tokens with ``cands`` candidates of 1 to
``len_hi`` tokens, drawn from ``shape_seed`` (so that the work of a case does not
depend on the seed of its inputs). Keys are N(0, 1) with a scale per channel
and a milder one per token, queries N(0, 1) over the channel's scale (scores of
unit variance), values N(0, 1) with a scale per token.
"""
import math

import numpy as np
import torch

own = False

BLOCK = 64            # tokens that share an exponent
LOW, HIGH = -117, 119  # range of the exponents


def _case(name, op, requests, prefix_lo, prefix_hi, cands, len_hi, dtype, Hq, Hkv, d, **more):
    return dict(name=name, op=op, requests=requests, prefix_lo=prefix_lo, prefix_hi=prefix_hi,
                cands=cands, len_hi=len_hi, shape_seed=7, dtype=dtype, Hq=Hq, Hkv=Hkv, d=d, **more)


def listed():
    wide = dict(Hq=24, Hkv=4, d=256)   # heads of the multiple-choice and yes/no batches
    slim = dict(Hq=16, Hkv=2, d=256)   # heads of the hybrid and the long-context batches
    many = dict(Hq=32, Hkv=8, d=128)
    return [
        # the caches of a batch of multiple-choice questions, after their prefill
        _case("write_choice", "write", 16, 200, 1200, 4, 12, "bf16", **wide),
        # the caches of a large batch over long contexts
        _case("write_long", "write", 256, 2048, 8192, 4, 12, "bf16", **slim),
        # a reasoning trace generated token by token: one token of each of 64 requests
        _case("append_token", "append", 64, 400, 2048, 1, 1, "bf16", new_lo=1, new_hi=1, **wide),
        # contexts that arrive in pieces: a few hundred tokens each, blocks begun before
        _case("append_piece", "append", 16, 2048, 8192, 1, 1, "bf16", new_lo=100, new_hi=700,
              **many),
        # a small float32 cache read back
        _case("read_small_f32", "read", 4, 64, 300, 4, 4, "f32", Hq=8, Hkv=2, d=64),
        # caches read back for a model part that takes bf16
        _case("read_long", "read", 32, 2048, 8192, 4, 12, "bf16", **slim),
        # one small float32 request: an interactive call, all launches and latency
        _case("attend_tiny_f32", "attend", 1, 128, 128, 4, 4, "f32", Hq=8, Hkv=2, d=64),
        # one long context with its answers: attention at batch 1
        _case("attend_single", "attend", 1, 6000, 6000, 4, 12, "bf16", **slim),
        # a batch of multiple-choice questions: short, ragged prefixes
        _case("attend_choice", "attend", 16, 200, 1200, 4, 12, "bf16", **wide),
        # one query row for each of 64 contexts: the next token of a trace, heads of 128
        _case("attend_token", "attend", 64, 1000, 6000, 1, 1, "bf16", **many),
        # ratings: ten short candidates for each of 32 contexts
        _case("attend_rating", "attend", 32, 512, 512, 10, 3, "bf16", **slim),
        # a large batch over long contexts
        _case("attend_long", "attend", 256, 2048, 8192, 4, 12, "bf16", **slim),
    ]


# --------------------------------------------------------------------------
# drawn cases: the ranges the listed ones stand for
# --------------------------------------------------------------------------
def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(("write", "append", "read", "attend", "attend", "attend"))
    Hq, Hkv = rng.choice(((8, 2), (16, 2), (24, 4), (32, 8), (8, 8), (7, 1)))
    d = rng.choice((64, 128, 256, 256))
    f32 = rng.random() < 0.25
    tokens = 1000000 * 512 // (Hkv * d)          # no larger cache than the long batch's
    if f32:
        tokens = 4096 if op == "attend" else tokens // 2
    hi = _log(rng, 1 if op != "attend" else 16, min(8192, tokens))
    lo = hi if rng.random() < 0.25 else max(1, int(hi * rng.uniform(0.2, 0.9)))
    r = _log(rng, 1, max(1, min(256, tokens // hi)))
    cands, len_hi = rng.choice(((1, 1), (2, 2), (4, 12), (rng.randint(3, 10), 3)))
    c = dict(op=op, requests=r, prefix_lo=lo, prefix_hi=hi, cands=cands, len_hi=len_hi,
             shape_seed=rng.randrange(1, 1 << 20), dtype="f32" if f32 else "bf16", Hq=Hq, Hkv=Hkv,
             d=d)
    if op == "append":
        new = 1 if rng.random() < 0.4 else _log(rng, 1, max(1, hi // 2))
        c.update(new_lo=min(new, max(1, new // 3)), new_hi=new)
    return c


# --------------------------------------------------------------------------
# batch structure
# --------------------------------------------------------------------------
def _shape(case):
    """Prefix lengths, candidate counts and lengths, and the tokens to append."""
    g = np.random.default_rng(case["shape_seed"])
    R, C = case["requests"], case["cands"]
    P = g.integers(case["prefix_lo"], case["prefix_hi"] + 1, size=R)
    # mostly short answers, the longest len_hi tokens (geometric, truncated)
    k = np.arange(1, case["len_hi"] + 1)
    w = 0.7 ** (k - 1) if case["len_hi"] > 3 else np.ones(len(k))
    m = g.choice(k, size=R * C, p=w / w.sum())
    new = np.minimum(P, g.integers(case.get("new_lo", 0), case.get("new_hi", 0) + 1, size=R))
    return P.astype(np.int32), np.full(R, C, np.int32), m.astype(np.int32), new.astype(np.int32)


def _counts(case):
    P, n_cand, m, new = _shape(case)
    R = len(P)
    rows = 1 + (m - 1).reshape(R, -1).sum(1)
    F = int((m - 1).sum())
    return dict(P=P, n_cand=n_cand, m=m, new=new, rows=rows, R=R, F=F, N=R + F, S=int(P.sum()),
                blocks=int(P.sum()) // BLOCK + R, used=int(((P + BLOCK - 1) // BLOCK).sum()))


def _starts(lens):
    return np.concatenate([[0], np.cumsum(lens)[:-1]]).astype(np.int64)


def _padded(lens):
    """[requests, longest]: the packed place of token i of request r, and whether it has one."""
    i = np.arange(max(1, int(np.max(lens))))[None, :]
    has = i < np.asarray(lens)[:, None]
    return np.where(has, _starts(lens)[:, None] + i, 0), has


def _ranges(lens):
    """The request of every packed token, and its place in the request."""
    r = np.repeat(np.arange(len(lens)), lens)
    return r, np.arange(len(r)) - _starts(lens)[r]


def _up(n):
    return (n + 255) // 256 * 256


def _gpu(x):
    return torch.from_numpy(np.ascontiguousarray(x)).cuda()


# --------------------------------------------------------------------------
# the plain form: elementary operations in 32 bits
# --------------------------------------------------------------------------
def _exponents(top):
    """The least X with top <= 448 * 2^X (448 = 0.875 * 2^9)."""
    m, e = torch.frexp(top)
    x = torch.where(m <= 0.875, e - 9, e - 8)
    return torch.where(top > 0, x, LOW).clamp(LOW, HIGH).to(torch.int32)


def _block_exponents(x, block, blocks):
    top = torch.zeros(blocks, x.shape[1], device=x.device)
    top.scatter_reduce_(0, block[:, None].expand(-1, x.shape[1]), x.float().abs().amax(-1), "amax")
    return _exponents(top)


def _power(x):
    """2^x in float32, exactly, for whole x in [-126, 127]."""
    return ((x + 127) << 23).view(torch.float32)


def _codes(x, X):
    """e4m3 codes of x [n, heads, d] for the exponents X [n, heads]."""
    y = (x.float() * _power(-X)[..., None]).clamp(-448.0, 448.0)
    return y.to(torch.float8_e4m3fn).view(torch.uint8)


def _values(codes, X):
    return codes.view(torch.float8_e4m3fn).float() * _power(X)[..., None]


def _parts(buf, c, n):
    """The codes and exponent bytes of a cache buffer."""
    size = n["S"] * c["Hkv"] * c["d"]
    codes = buf[:size].view(n["S"], c["Hkv"], c["d"])
    exps = buf[_up(size):_up(size) + n["blocks"] * c["Hkv"]].view(n["blocks"], c["Hkv"])
    return codes, exps


def _empty_cache(c, n):
    return torch.zeros(_up(n["S"] * c["Hkv"] * c["d"]) + _up(n["blocks"] * c["Hkv"]),
                       dtype=torch.uint8, device="cuda")


def _plain_write(x, buf, block, c, n):
    codes, exps = _parts(buf, c, n)
    X = _block_exponents(x, block, n["blocks"])
    used = torch.zeros(n["blocks"], 1, dtype=torch.bool, device=x.device)
    used[block] = True
    codes.copy_(_codes(x, X[block]))
    exps.copy_(torch.where(used, X + 127, exps.int()).to(torch.uint8))


def _plain_append(x, buf, s):
    c, n = s["case"], s["n"]
    codes, exps = _parts(buf, c, n)
    X = _block_exponents(x, s["new_block"], n["blocks"])
    held = exps.int() - 127
    touched = torch.zeros(n["blocks"], 1, dtype=torch.bool, device=x.device)
    touched[s["new_block"]] = True
    begun = torch.zeros_like(touched)
    begun[s["old_block"]] = True                  # blocks that hold tokens already
    X = torch.where(begun, torch.maximum(X, held), X)
    old, ob = s["old_place"], s["old_block"]      # those tokens, rounded again
    codes[old] = _codes(_values(codes[old], held[ob]), X[ob])
    codes[s["new_place"]] = _codes(x, X[s["new_block"]])
    exps.copy_(torch.where(touched, X + 127, exps.int()).to(torch.uint8))


def _plain_read(buf, s):
    codes, exps = _parts(buf, s["case"], s["n"])
    return _values(codes, (exps.int() - 127)[s["block"]])


def _plain_attend(s):
    c, n, x = s["case"], s["n"], s["x"]
    g, H, d = c["Hq"] // c["Hkv"], c["Hkv"], c["d"]
    R, rows = s["row_place"].shape
    keys, fed = s["key_place"].shape[1], s["fed_place"].shape[1]

    def heads(t, place, width):   # [R, Hkv, width, d]
        return t[place].permute(0, 2, 1, 3) if t.shape[0] else t.new_zeros(R, H, width, d)

    q = x["q"].float()[s["row_place"]].view(R, rows, H, g, d).permute(0, 2, 1, 3, 4)
    q = q.reshape(R, H, rows * g, d)
    k = torch.cat([heads(_plain_read(x["k8"], s), s["key_place"], keys),
                   heads(x["k_cand"].float(), s["fed_place"], fed)], 2)
    p = torch.matmul(q, k.transpose(2, 3)) * d ** -0.5
    del k
    sees = s["sees"][:, None, :, None, :].expand(R, 1, rows, g, keys + fed)
    p = p.masked_fill_(~sees.reshape(R, 1, rows * g, keys + fed), -math.inf)
    p = p.sub_(p.amax(-1, keepdim=True)).exp_()
    p = p.div_(p.sum(-1, keepdim=True))
    v = torch.cat([heads(_plain_read(x["v8"], s), s["key_place"], keys),
                   heads(x["v_cand"].float(), s["fed_place"], fed)], 2)
    o = torch.matmul(p, v).view(R, H, rows, g, d).permute(0, 2, 1, 3, 4)
    o = o.reshape(R, rows, H * g, d)[s["row_has"]]
    s["o"].copy_(o)
    return s["o"]


# --------------------------------------------------------------------------
# inputs
# --------------------------------------------------------------------------
class _Draw:
    """Tensors drawn one after the other from one seeded generator on the GPU."""

    def __init__(self, seed, c):
        self.g = torch.Generator(device="cuda").manual_seed(int(seed) + 1)
        self.dt = torch.bfloat16 if c["dtype"] == "bf16" else torch.float32
        self.channel = self.normal(c["Hkv"], c["d"]).float().mul_(0.5).exp_()
        self.c = c

    def normal(self, *shape):
        x = torch.empty(shape, device="cuda", dtype=self.dt)
        return x.normal_(0.0, 1.0, generator=self.g)

    def tokens(self, n):
        return self.normal(n, 1, 1).mul_(0.3).exp_()

    def keys(self, n):
        return self.normal(n, self.c["Hkv"], self.c["d"]).mul_(self.channel.to(self.dt)).mul_(
            self.tokens(n))

    def values(self, n):
        return self.normal(n, self.c["Hkv"], self.c["d"]).mul_(self.tokens(n))

    def queries(self, n):
        g = self.c["Hq"] // self.c["Hkv"]
        return self.normal(n, self.c["Hq"], self.c["d"]).div_(
            self.channel.to(self.dt).repeat_interleave(g, 0))


def _inputs(case, seed):
    c, n = case, _counts(case)
    t, op = _Draw(seed, c), c["op"]
    req, at = _ranges(n["P"])
    s = dict(case=c, n=n, block=_gpu(_starts(n["P"])[req] // BLOCK + req + at // BLOCK))
    x = s["x"] = {}
    if op == "write":
        x.update(k=t.keys(n["S"]), v=t.values(n["S"]), k8=_empty_cache(c, n), v8=_empty_cache(c, n))
        return s
    k, v = t.keys(n["S"]), t.values(n["S"])
    for name, y in (("k8", k), ("v8", v)):
        x[name] = _empty_cache(c, n)
        if op != "append":
            _plain_write(y, x[name], s["block"], c, n)
    if op == "append":
        # the cache holds a request's tokens but its last `new` ones
        start = n["P"] - n["new"]
        held = at < start[req]
        begun = (at // BLOCK == (start // BLOCK)[req]) & held & (n["new"] > 0)[req]
        s.update(old_place=_gpu(np.flatnonzero(begun)), new_place=_gpu(np.flatnonzero(~held)))
        s.update(old_block=s["block"][s["old_place"]], new_block=s["block"][s["new_place"]],
                 start=_gpu(start.astype(np.int32)),
                 new_offset=_gpu(np.concatenate([[0], np.cumsum(n["new"])]).astype(np.int32)))
        h = _gpu(held)
        for name, y in (("k8", k), ("v8", v)):
            _plain_write(torch.where(h[:, None, None], y, torch.zeros_like(y)), x[name], s["block"],
                         c, n)
        # new tokens a little larger, so that some blocks' exponents grow
        x.update(k=k[s["new_place"]] * 1.5, v=v[s["new_place"]] * 1.5)
    elif op == "attend":
        x.update(q=t.queries(n["N"]), k_cand=t.keys(n["F"]), v_cand=t.values(n["F"]))
    return s


def _plan(s):
    """Where rows, keys and candidate tokens stand when padded, and what a row sees."""
    c, n = s["case"], s["n"]
    row, row_has = _padded(n["rows"])
    key, key_has = _padded(n["P"])
    fed, fed_has = _padded(n["rows"] - 1)
    # candidate of every fed token; row i of a request is its fed token i - 1
    cand = np.repeat(np.arange(len(n["m"])), n["m"] - 1)
    fed_cand = np.where(fed_has, cand[fed] if len(cand) else -1, -2)
    row_cand = np.concatenate([np.full((n["R"], 1), -3), fed_cand], 1)[:, :row.shape[1]]
    i, j = np.arange(row.shape[1])[None, :, None], np.arange(fed.shape[1])[None, None, :]
    own_keys = (row_cand[:, :, None] == fed_cand[:, None, :]) & (j <= i - 1) & (
        fed_has[:, None, :])
    sees = np.concatenate([np.broadcast_to(key_has[:, None, :], (*row.shape, key.shape[1])),
                           own_keys], 2)
    s.update(row_place=_gpu(row), row_has=_gpu(row_has), key_place=_gpu(key), fed_place=_gpu(fed),
             sees=_gpu(sees))


def prepare(case, seed):
    s = _inputs(case, seed)
    c, n = s["case"], s["n"]
    dt = torch.bfloat16 if c["dtype"] == "bf16" else torch.float32
    if c["op"] == "attend":
        _plan(s)
        s["o"] = torch.empty(n["N"], c["Hq"], c["d"], device="cuda", dtype=dt)
    if c["op"] == "read":
        s["k"], s["v"] = (torch.empty(n["S"], c["Hkv"], c["d"], device="cuda", dtype=dt)
                          for _ in range(2))
    if own:
        # the layout on the device and the workspace, as a scorer keeps them per batch shape
        from paper_2609_33874_gb300 import jet

        host = jet.jet_layout_build(n["P"], n["n_cand"], n["m"], np.zeros(int(n["m"].sum())), 1)
        s["layout"] = host.to_device()
        s["dims"] = jet.make_dims(jet.DTYPE_BF16 if c["dtype"] == "bf16" else jet.DTYPE_F32,
                                  Hq=c["Hq"], Hkv=c["Hkv"], d=c["d"])
        if c["op"] == "attend":
            ws = jet.jet_attend_workspace_bytes_e4m3(host.sizes, s["dims"])
            s["ws"] = torch.empty((ws + 15) // 16 * 4, device="cuda")
    return s


def _held(s):
    """The caches as numbers: e4m3 codes, and the exponent bytes."""
    out = {}
    for name in ("k8", "v8"):
        codes, exps = _parts(s["x"][name], s["case"], s["n"])
        out[name] = codes.view(torch.float8_e4m3fn)
        out[name + "_exponents"] = exps
    return out


def run(state):
    s = state
    c, x, op = s["case"], s["x"], s["case"]["op"]
    if own:
        from paper_2609_33874_gb300 import jet

        if op == "write":
            jet.jet_quantize_kv_e4m3(s["layout"], s["dims"], x["k"], x["v"], x["k8"], x["v8"])
            return _held(s)
        if op == "append":
            jet.jet_append_kv_e4m3(s["layout"], s["dims"], s["start"], s["new_offset"], x["k"],
                                   x["v"], x["k8"], x["v8"])
            return _held(s)
        if op == "read":
            jet.jet_dequantize_kv_e4m3(s["layout"], s["dims"], x["k8"], x["v8"], s["k"], s["v"])
            return dict(k=s["k"], v=s["v"])
        jet.jet_prefix_attend_e4m3(s["layout"], s["dims"], x["q"], x["k8"], x["v8"], x["k_cand"],
                                   x["v_cand"], s["o"], s["ws"])
        return dict(o=s["o"])
    if op == "write":
        _plain_write(x["k"], x["k8"], s["block"], c, s["n"])
        _plain_write(x["v"], x["v8"], s["block"], c, s["n"])
        return _held(s)
    if op == "append":
        _plain_append(x["k"], x["k8"], s)
        _plain_append(x["v"], x["v8"], s)
        return _held(s)
    if op == "read":
        s["k"].copy_(_plain_read(x["k8"], s))
        s["v"].copy_(_plain_read(x["v8"], s))
        return dict(k=s["k"], v=s["v"])
    return dict(o=_plain_attend(s))


# --------------------------------------------------------------------------
# the definition in 64 bits, request by request
# --------------------------------------------------------------------------
# the magnitudes of the codes 0 .. 126 (4 exponent bits of bias 7, 3 mantissa bits)
_GRID = np.array([(i % 8) * 2.0 ** -9 if i < 8 else (1 + (i % 8) / 8.0) * 2.0 ** (i // 8 - 7)
                  for i in range(127)])


def _exact_exponent(top):
    """The least whole X in the range with top <= 448 * 2^X."""
    X = np.full(top.shape, LOW)
    for e in range(LOW, HIGH):
        X += top > 448.0 * 2.0 ** e
    return X


def _exact_codes(y):
    """The grid's nearest code of y (the even one of two as near), with its sign, as values."""
    a = np.minimum(np.abs(y), 448.0)
    hi = np.clip(np.searchsorted(_GRID, a), 0, 126)
    lo = np.maximum(hi - 1, 0)
    up, down = _GRID[hi] - a, a - _GRID[lo]
    pick = np.where((up < down) | ((up == down) & (hi % 2 == 0)), hi, lo)
    return np.copysign(_GRID[pick], y)


def _byte_values(b):
    return np.where(b & 128, -1.0, 1.0) * _GRID[np.minimum(b & 127, 126)]


def _host(t):
    return t.double().cpu().numpy() if t.is_floating_point() else t.cpu().numpy()


def _exact_cache(s, name):
    """Codes (as values) and exponents of a written or appended cache."""
    c, n = s["case"], s["n"]
    codes, exps = (_host(t) for t in _parts(s["x"][name], c, n))
    val, X = _byte_values(codes), exps.astype(np.int64) - 127
    x = _host(s["x"][name[0]])
    p0, new0 = _starts(n["P"]), _starts(n["new"])
    for r in range(n["R"]):
        P = int(n["P"][r])
        a = P - int(n["new"][r]) if c["op"] == "append" else 0
        src = new0[r] if c["op"] == "append" else p0[r]
        for b in range(a // BLOCK, -(-P // BLOCK)):
            i, j = max(a, b * BLOCK), min(P, (b + 1) * BLOCK)
            if i >= j:
                continue
            y, at = x[src + i - a:src + j - a], p0[r] // BLOCK + r + b
            e = _exact_exponent(np.abs(y).max((0, 2)))
            if i > b * BLOCK:
                e = np.maximum(e, X[at])
                o = slice(p0[r] + b * BLOCK, p0[r] + i)
                val[o] = _exact_codes(val[o] * 2.0 ** (X[at] - e)[None, :, None])
            val[p0[r] + i:p0[r] + j] = _exact_codes(y * 2.0 ** -e.astype(float)[None, :, None])
            X[at] = e
    return val, X + 127


def exact(case, seed):
    c, n = case, _counts(case)
    op = c["op"]
    searched = (n["S"] if op == "write" else int(n["new"].sum())) * c["Hkv"] * c["d"]
    if op in ("write", "append") and (searched > 2e7 or n["S"] * c["Hkv"] * c["d"] > 1.2e8):
        return None  # more elements than a search of the grid gets through
    s = _inputs(case, seed)
    if op in ("write", "append"):
        out = {}
        for name in ("k8", "v8"):
            val, e = _exact_cache(s, name)
            out[name] = torch.from_numpy(val)
            out[name + "_exponents"] = torch.from_numpy(e.astype(np.uint8))
        return out
    table = torch.from_numpy(np.concatenate([_GRID, [np.nan], -_GRID, [np.nan]])).cuda()

    def value(buf, r):
        codes, exps = _parts(buf, c, n)
        p0, P = int(_starts(n["P"])[r]), int(n["P"][r])
        at = p0 // BLOCK + r + torch.arange(P, device="cuda") // BLOCK
        two = ((exps[at].long() - 127 + 1023) << 52).view(torch.float64)   # 2^X
        return table[codes[p0:p0 + P].long()] * two[..., None]

    if op == "read":
        return dict(k=torch.cat([value(s["x"]["k8"], r) for r in range(n["R"])]),
                    v=torch.cat([value(s["x"]["v8"], r) for r in range(n["R"])]))
    g = c["Hq"] // c["Hkv"]
    out, row, f = [], 0, 0
    q, kc, vc = (s["x"][t].double() for t in ("q", "k_cand", "v_cand"))
    for r in range(n["R"]):
        k, v = value(s["x"]["k8"], r), value(s["x"]["v8"], r)
        P = k.shape[0]
        nr = int(n["rows"][r])
        k, v = torch.cat([k, kc[f:f + nr - 1]]), torch.cat([v, vc[f:f + nr - 1]])
        see = torch.zeros(nr, P + nr - 1, dtype=torch.bool)
        see[:, :P] = True
        i = 1
        for m in n["m"][r * c["cands"]:(r + 1) * c["cands"]]:
            for t in range(int(m) - 1):
                see[i + t, P + i - 1:P + i + t] = True
            i += int(m) - 1
        qr = q[row:row + nr].view(nr, c["Hkv"], g, c["d"]).permute(1, 2, 0, 3)
        z = torch.matmul(qr, k.permute(1, 2, 0)[:, None]) / math.sqrt(c["d"])
        z = torch.where(see.cuda(), z, -math.inf)
        w = torch.softmax(z, -1)
        o = torch.matmul(w, v.permute(1, 0, 2)[:, None])   # [Hkv, g, rows, d]
        out.append(o.permute(2, 0, 1, 3).reshape(nr, c["Hq"], c["d"]))
        row, f = row + nr, f + nr - 1
    return dict(o=torch.cat(out))


# --------------------------------------------------------------------------
# what a pass cannot do without
# --------------------------------------------------------------------------
def work(case):
    c, n = case, _counts(case)
    eb = 2 if c["dtype"] == "bf16" else 4
    wide = c["Hkv"] * c["d"]
    exps = 2 * n["used"] * c["Hkv"]
    if c["op"] in ("write", "read"):
        return dict(bytes=2 * n["S"] * wide * (eb + 1) + exps, flops=2 * n["S"] * wide)
    if c["op"] == "append":
        a = int(n["new"].sum())
        start = n["P"] - n["new"]
        touched = int(((n["P"] + BLOCK - 1) // BLOCK - start // BLOCK)[n["new"] > 0].sum())
        return dict(bytes=2 * a * wide * (eb + 1) + 2 * touched * c["Hkv"], flops=2 * a * wide)
    m = n["m"].astype(np.int64)
    pairs = int((n["rows"] * n["P"].astype(np.int64)).sum() + (m * (m - 1) // 2).sum())
    return dict(bytes=2 * n["S"] * wide + exps + 2 * n["F"] * wide * eb +
                2 * n["N"] * c["Hq"] * c["d"] * eb, flops=4 * pairs * c["Hq"] * c["d"])
