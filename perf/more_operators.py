"""Performance cases of positions and windows: the norm and rotation of queries and
keys, and attention that sees a window of the last tokens and a few first ones, in the
prefill and in the scoring step.

Norm and rotation of x [tokens, heads, d] at position p, gain g [d], frequencies f_i:

    y = x / sqrt(mean(x^2) + eps) * g             over each head
    (a, b) -> (a cos t - b sin t, a sin t + b cos t),   t = p f_i,  i < rot / 2
    of (a, b) = (y[i], y[i + rot / 2]) ("halves") or (y[2 i], y[2 i + 1]) ("pairs");
    elements from rot on stay.

Window: a token at position p sees the tokens at j <= p with j > p - window or
j < sinks. The prefix of a request stands at 0 .. P - 1, its shared row at P - 1, the row
fed with candidate token y_t (t = 1, 2, ...) at P - 1 + t, and it sees its own candidate's
tokens only.

A case holds the batch structure as plain values: ``requests`` contexts of ``prefix_lo``
to ``prefix_hi`` tokens with ``cands`` candidates of 1 to ``len_hi`` tokens, drawn from
``shape_seed`` (so that the work of a case does not depend on the seed of its inputs).
"""
import math

import numpy as np
import torch

own = False

EPS = 1e-6
BLOCK = 128   # positions of the plain prefill that share their gathered keys


def _case(name, op, requests, prefix_lo, prefix_hi, dtype, Hq, Hkv, d, cands=1, len_hi=1, **more):
    return dict(name=name, op=op, requests=requests, prefix_lo=prefix_lo, prefix_hi=prefix_hi,
                cands=cands, len_hi=len_hi, shape_seed=11, dtype=dtype, Hq=Hq, Hkv=Hkv, d=d, **more)


def listed():
    wide = dict(Hq=24, Hkv=4, d=256)   # heads of the multiple-choice and yes/no batches
    slim = dict(Hq=16, Hkv=2, d=256)   # heads of the hybrid and the long-context batches
    many = dict(Hq=32, Hkv=8, d=128)
    return [
        # a reasoning trace generated token by token: one token of each of 64 requests, far out
        _case("rotate_token", "rotate_token", 64, 1, 1 << 20, "bf16", rot=256, style="halves",
              theta=1e6, norm=True, **wide),
        # the rows of a batch of ratings, a quarter of each head rotated
        _case("rotate_rows", "rotate_rows", 32, 512, 512, "bf16", cands=10, len_hi=3, rot=64,
              style="halves", theta=1e7, norm=True, **slim),
        # a small float32 batch, neighbours rotated, without norms
        _case("rotate_small_f32", "rotate_prefix", 4, 64, 300, "f32", 8, 2, 64, rot=64,
              style="pairs", theta=1e4, norm=False),
        # the prefill's queries and keys of long contexts
        _case("rotate_long", "rotate_prefix", 16, 2048, 8192, "bf16", rot=256, style="halves",
              theta=1e6, norm=True, **wide),
        # multiple-choice questions: short, ragged prefixes
        _case("prefill_choice", "prefill", 16, 200, 1200, "bf16", window=256, sinks=4, **wide),
        # many short contexts under a narrow window, small heads
        _case("prefill_narrow", "prefill", 64, 100, 2000, "bf16", 16, 2, 64, window=128, sinks=1),
        # one long document under a wide window
        _case("prefill_single", "prefill", 1, 16000, 16000, "bf16", window=4096, sinks=16, **many),
        # long contexts under an ordinary window
        _case("prefill_long", "prefill", 16, 2048, 8192, "bf16", window=1024, sinks=4, **slim),
        # one small float32 request: an interactive call, all launches and latency
        _case("attend_tiny_f32", "attend", 1, 128, 128, "f32", 8, 2, 64, cands=4, len_hi=4,
              window=32, sinks=2),
        # a batch of multiple-choice questions under a narrow window
        _case("attend_choice", "attend", 16, 200, 1200, "bf16", cands=4, len_hi=12, window=128,
              sinks=4, **wide),
        # one query row for each of 64 contexts: the next token of a trace
        _case("attend_token", "attend", 64, 1000, 6000, "bf16", window=1024, sinks=4, **many),
        # a large batch over long contexts under a wide window
        _case("attend_long", "attend", 256, 2048, 8192, "bf16", cands=4, len_hi=12, window=2048,
              sinks=16, **slim),
    ]


# --------------------------------------------------------------------------
# drawn cases: the ranges the listed ones stand for
# --------------------------------------------------------------------------
def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(("rotate_token", "rotate_rows", "rotate_prefix", "prefill", "prefill",
                     "attend", "attend"))
    Hq, Hkv = rng.choice(((8, 2), (16, 2), (32, 8), (8, 8), (7, 1), (24, 4)))
    d = rng.choice((64, 128, 256)) if Hq != 24 else 256
    f32 = op != "prefill" and rng.random() < 0.25
    window = _log(rng, 1, 8192)
    hi = _log(rng, 1, 8192)
    # tokens of the batch: no more work than the largest listed case of the operator
    if op == "prefill":
        tokens = int(2.5e11 / (Hq * d * (min(window, hi) + 2 * BLOCK)))
    elif op == "attend":
        tokens = 1000000 * 512 // (Hkv * d) if not f32 else 32768
    else:
        tokens = 70000 * 28 * 256 // ((Hq + Hkv) * d) // (2 if f32 else 1)
    hi = min(hi, tokens)
    lo = hi if rng.random() < 0.25 else max(1, int(hi * rng.uniform(0.2, 0.9)))
    r = _log(rng, 1, max(1, min(256, tokens // hi)))
    cands, len_hi = rng.choice(((1, 1), (2, 2), (4, 12), (rng.randint(3, 10), 3)))
    if op in ("rotate_prefix", "prefill"):
        cands, len_hi = 1, 1
    c = dict(op=op, requests=r, prefix_lo=lo, prefix_hi=hi, cands=cands, len_hi=len_hi,
             shape_seed=rng.randrange(1, 1 << 20), dtype="f32" if f32 else "bf16", Hq=Hq, Hkv=Hkv,
             d=d)
    if op.startswith("rotate"):
        if op == "rotate_token":
            c.update(requests=_log(rng, 1, 1024), prefix_lo=1, prefix_hi=_log(rng, 2, 1 << 24))
        c.update(rot=16 * rng.randint(1, d // 16) if rng.random() < 0.5 else d,
                 style=rng.choice(("halves", "pairs")), theta=float(rng.choice((1e4, 5e5, 1e7))),
                 norm=rng.random() < 0.8)
    else:
        c.update(window=window, sinks=rng.choice((0, 1, 4, 16, rng.randint(2, 128))))
    return c


# --------------------------------------------------------------------------
# batch structure
# --------------------------------------------------------------------------
def _shape(case):
    """Prefix lengths and candidate lengths."""
    g = np.random.default_rng(case["shape_seed"])
    R = case["requests"]
    P = g.integers(case["prefix_lo"], case["prefix_hi"] + 1, size=R)
    # mostly short answers, the longest len_hi tokens (geometric, truncated)
    k = np.arange(1, case["len_hi"] + 1)
    w = 0.7 ** (k - 1) if case["len_hi"] > 3 else np.ones(len(k))
    m = g.choice(k, size=R * case["cands"], p=w / w.sum())
    return P.astype(np.int64), m.astype(np.int64)


def _starts(lens):
    return np.concatenate([[0], np.cumsum(lens)[:-1]]).astype(np.int64)


def _ranges(lens):
    """The owner of every packed thing, and its place with its owner."""
    r = np.repeat(np.arange(len(lens)), lens)
    return r, np.arange(len(r)) - _starts(lens)[r]


def _counts(case):
    P, m = _shape(case)
    R = len(P)
    rows = 1 + (m - 1).reshape(R, -1).sum(1)
    return dict(P=P, m=m, R=R, rows=rows, F=int((m - 1).sum()), N=int(rows.sum()), S=int(P.sum()))


def _rows(n):
    """Request, candidate (-1: the shared row), t and position of every row."""
    req, place = _ranges(n["rows"])
    cand, t = _ranges(n["m"] - 1)
    row_cand, row_t = np.full(n["N"], -1), np.zeros(n["N"], np.int64)
    row_cand[place > 0], row_t[place > 0] = cand, t + 1
    return req, row_cand, row_t, n["P"][req] - 1 + row_t


def _tokens(case, n):
    """Positions of the queries and of the keys that an operator of rotation takes."""
    if case["op"] == "rotate_token":
        return n["P"] - 1, n["P"] - 1
    if case["op"] == "rotate_prefix":
        at = _ranges(n["P"])[1]
        return at, at
    _, _, t, pos = _rows(n)
    return pos, pos[t > 0]


def _gpu(x):
    return torch.from_numpy(np.ascontiguousarray(x)).cuda()


def _dtype(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


# --------------------------------------------------------------------------
# inputs
# --------------------------------------------------------------------------
def _inputs(case, seed):
    c, n = case, _counts(case)
    g = torch.Generator(device="cuda").manual_seed(int(seed) + 1)
    dt, Hq, Hkv, d = _dtype(c), c["Hq"], c["Hkv"], c["d"]

    def normal(*shape):
        return torch.empty(shape, device="cuda", dtype=dt).normal_(0.0, 1.0, generator=g)

    s = dict(case=c, n=n)
    if c["op"].startswith("rotate"):
        # projections of a residual stream: a scale per token, gains around one
        pq, pk = _tokens(c, n)
        s.update(q=normal(len(pq), Hq, d).mul_(normal(len(pq), 1, 1).mul_(0.5).exp_()),
                 k=normal(len(pk), Hkv, d).mul_(normal(len(pk), 1, 1).mul_(0.5).exp_()),
                 gq=normal(d).mul_(0.2).add_(1.0), gk=normal(d).mul_(0.2).add_(1.0))
        return s
    # normalised and rotated queries and keys: scores of about unit variance, a scale per head;
    # values with a scale per token
    rows = n["S"] if c["op"] == "prefill" else n["N"]
    s.update(q=normal(rows, Hq, d).mul_(normal(1, Hq, 1).mul_(0.3).exp_()),
             k=normal(n["S"], Hkv, d),
             v=normal(n["S"], Hkv, d).mul_(normal(n["S"], 1, 1).mul_(0.3).exp_()))
    if c["op"] == "attend":
        s.update(kc=normal(n["F"], Hkv, d), vc=normal(n["F"], Hkv, d))
    return s


def _plan_prefill(s):
    """Blocks of BLOCK positions of a request, the keys that any of a block's positions sees
    - the first `sinks`, then a run that ends with the block - and who sees which."""
    c, n = s["case"], s["n"]
    W, sinks = c["window"], c["sinks"]
    blocks = -(-n["P"] // BLOCK)
    req, b = _ranges(blocks)
    P, p0 = n["P"][req][:, None], _starts(n["P"])[req][:, None]
    pos = b[:, None] * BLOCK + np.arange(BLOCK)[None, :]
    has = pos < P
    span = min(W - 1, int(n["P"].max())) + BLOCK
    run = (b[:, None] + 1) * BLOCK - span + np.arange(span)[None, :]
    first = np.broadcast_to(np.arange(sinks)[None, :], (len(b), sinks))
    key = np.concatenate([first, run], 1)
    # a first token stands in the run, too, where the run reaches it
    held = (key >= 0) & (key < P)
    held[:, :sinks] &= first < run[:, :1]
    s.update(row=_gpu(np.where(has, p0 + pos, p0)), has=_gpu(has),
             key=_gpu(np.where(held, p0 + key, p0)), pos=_gpu(pos.astype(np.int32)),
             key_pos=_gpu(np.where(held, key, 1 << 30).astype(np.int32)))


def _plan_attend(s):
    """Every request's rows and keys - first ones, the last `window` of the prefix, fed
    candidate tokens - padded, and who sees which."""
    c, n = s["case"], s["n"]
    W, sinks, R = c["window"], c["sinks"], n["R"]
    P, p0 = n["P"][:, None], _starts(n["P"])[:, None]
    i = np.arange(int(n["rows"].max()))[None, :]
    has = i < n["rows"][:, None]
    row = np.where(has, _starts(n["rows"])[:, None] + i, 0)
    _, cand, _, pos = _rows(n)
    longest = int(n["P"].max())
    span = min(W, longest)
    run = P - span + np.arange(span)[None, :]
    first = np.broadcast_to(np.arange(min(sinks, longest))[None, :], (R, min(sinks, longest)))
    key = np.concatenate([first, run], 1)
    held = (key >= 0) & (key < P)
    held[:, :first.shape[1]] &= first < P - span
    f = i[:, 1:]
    f_has = has[:, 1:]
    fed = np.where(f_has, _starts(n["rows"])[:, None] + f - np.arange(R)[:, None] - 1, 0)
    # a request's fed token f is row f + 1 of the request
    f_row = np.where(f_has, row[:, 1:], 0)
    key_pos = np.concatenate([np.where(held, key, 1 << 30),
                              np.where(f_has, pos[f_row], 1 << 30)], 1)
    key_cand = np.concatenate([np.full(key.shape, -1), np.where(f_has, cand[f_row], -2)], 1)
    s.update(row=_gpu(row), has=_gpu(has), key=_gpu(np.where(held, p0 + key, p0)), fed=_gpu(fed),
             pos=_gpu(pos[row].astype(np.int32)), key_pos=_gpu(key_pos.astype(np.int32)),
             cand=_gpu(cand[row].astype(np.int32)), key_cand=_gpu(key_cand.astype(np.int32)))


def prepare(case, seed):
    s = _inputs(case, seed)
    c, n = s["case"], s["n"]
    if c["op"].startswith("rotate"):
        pq, pk = _tokens(c, n)
        s.update(pos_q=_gpu(pq.astype(np.int32)), pos_k=_gpu(pk.astype(np.int32)),
                 qo=torch.empty_like(s["q"]), ko=torch.empty_like(s["k"]))
    else:
        (_plan_prefill if c["op"] == "prefill" else _plan_attend)(s)
        s["o"] = torch.empty_like(s["q"])
    if own:
        # the layout on the device, the frequencies and the workspace, as a scorer keeps them per
        # model and batch shape
        from paper_2609_33874_gb300 import jet

        s["dims"] = jet.make_dims(jet.DTYPE_BF16 if c["dtype"] == "bf16" else jet.DTYPE_F32,
                                  Hq=c["Hq"], Hkv=c["Hkv"], d=c["d"])
        if c["op"].startswith("rotate"):
            s["rope"] = jet.make_rope(c["rot"], style=c["style"], theta=c["theta"],
                                      norm=c["norm"], eps=EPS)
        if c["op"] != "rotate_token":
            host = jet.jet_layout_build(n["P"], np.full(n["R"], c["cands"]), n["m"],
                                        np.zeros(int(n["m"].sum())), 1)
            s["layout"] = host.to_device()
            size = {"prefill": jet.jet_prefill_window_workspace_bytes,
                    "attend": jet.jet_attend_window_workspace_bytes}.get(c["op"])
            if size:
                nb = size(host.sizes, s["dims"], c["window"], c["sinks"])
                s["ws"] = torch.empty((nb + 15) // 16 * 4, device="cuda")
    return s


# --------------------------------------------------------------------------
# the plain form: elementary operations in 32 bits, angles in 64
# --------------------------------------------------------------------------
def _plain_rotate(x, gain, pos, c):
    x = x.float()
    if c["norm"]:
        x = x / torch.sqrt((x * x).mean(-1, keepdim=True) + EPS) * gain.float()
    rot, h = c["rot"], c["rot"] // 2
    f = c["theta"] ** (-torch.arange(h, device=x.device, dtype=torch.float64) * 2 / rot)
    t = pos.double()[:, None, None] * f
    co, si = torch.cos(t).float(), torch.sin(t).float()
    if c["style"] == "halves":
        a, b = x[..., :h], x[..., h:rot]
        y = torch.cat([a * co - b * si, a * si + b * co], -1)
    else:
        a, b = x[..., 0:rot:2], x[..., 1:rot:2]
        y = torch.stack([a * co - b * si, a * si + b * co], -1).flatten(-2)
    return torch.cat([y, x[..., rot:]], -1)


def _plain_attention(q, k, v, sees, c):
    """q [B, rows, Hq, d], k and v [B, keys, Hkv, d], sees [B, rows, keys]."""
    B, rows, keys = sees.shape
    H, g, d = c["Hkv"], c["Hq"] // c["Hkv"], c["d"]
    q = q.float().view(B, rows, H, g, d).permute(0, 2, 1, 3, 4).reshape(B, H, rows * g, d)
    p = torch.matmul(q, k.float().permute(0, 2, 3, 1)).mul_(d ** -0.5)
    p = p.view(B, H, rows, g, keys).masked_fill_(~sees[:, None, :, None, :], -math.inf)
    p = p.sub_(p.amax(-1, keepdim=True)).exp_()
    p = p.div_(p.sum(-1, keepdim=True)).view(B, H, rows * g, keys)
    o = torch.matmul(p, v.float().permute(0, 2, 1, 3)).view(B, H, rows, g, d)
    return o.permute(0, 2, 1, 3, 4).reshape(B, rows, H * g, d)


def _in_window(pos, key_pos, c):
    """Whether positions [B, rows] see positions [B, keys] (those of no key are far ahead)."""
    p, j = pos[:, :, None], key_pos[:, None, :]
    return (j <= p) & ((j > p - c["window"]) | (j < c["sinks"]))


def _plain_window(s):
    c = s["case"]
    sees = _in_window(s["pos"], s["key_pos"], c)
    k, v = s["k"][s["key"]], s["v"][s["key"]]
    if c["op"] == "attend":
        sees &= (s["key_cand"][:, None, :] == -1) | (
            s["key_cand"][:, None, :] == s["cand"][:, :, None])
        if s["n"]["F"]:
            k, v = torch.cat([k, s["kc"][s["fed"]]], 1), torch.cat([v, s["vc"][s["fed"]]], 1)
    else:
        # padding rows of a block see one key, so that their softmax is one
        sees[:, :, -1] |= ~s["has"]
    o = _plain_attention(s["q"][s["row"]], k, v, sees, c)
    s["o"].copy_(o[s["has"]])
    return s["o"]


def run(state):
    s = state
    c = s["case"]
    if own:
        from paper_2609_33874_gb300 import jet

        if c["op"] == "rotate_token":
            jet.jet_norm_rotate(s["dims"], s["rope"], s["pos_q"], s["q"], s["k"], s["gq"], s["gk"],
                                s["qo"], s["ko"])
            return dict(q=s["qo"], k=s["ko"])
        if c["op"] == "rotate_prefix":
            jet.jet_norm_rotate_prefix(s["layout"], s["dims"], s["rope"], s["q"], s["k"], s["gq"],
                                       s["gk"], s["qo"], s["ko"])
            return dict(q=s["qo"], k=s["ko"])
        if c["op"] == "rotate_rows":
            jet.jet_norm_rotate_rows(s["layout"], s["dims"], s["rope"], s["q"], s["k"], s["gq"],
                                     s["gk"], s["qo"], s["ko"])
            return dict(q=s["qo"], k=s["ko"])
        if c["op"] == "prefill":
            jet.jet_prefill_attend_window(s["layout"], s["dims"], c["window"], c["sinks"], s["q"],
                                          s["k"], s["v"], s["o"], s["ws"])
        else:
            jet.jet_prefix_attend_window(s["layout"], s["dims"], c["window"], c["sinks"], s["q"],
                                         s["k"], s["v"], s["kc"], s["vc"], s["o"], s["ws"])
        return dict(o=s["o"])
    if c["op"].startswith("rotate"):
        s["qo"].copy_(_plain_rotate(s["q"], s["gq"], s["pos_q"], c))
        s["ko"].copy_(_plain_rotate(s["k"], s["gk"], s["pos_k"], c))
        return dict(q=s["qo"], k=s["ko"])
    return dict(o=_plain_window(s))


# --------------------------------------------------------------------------
# the definition in 64 bits, request by request
# --------------------------------------------------------------------------
def _exact_rotate(x, gain, pos, c):
    """Each pair as a complex number, times e^(i p f)."""
    x = x.double()
    if c["norm"]:
        x = x * gain.double() / (x.square().sum(-1, keepdim=True) / c["d"] + EPS).sqrt()
    rot, h = c["rot"], c["rot"] // 2
    i = torch.arange(h, dtype=torch.float64, device=x.device)
    t = _gpu(pos).double()[:, None, None] * torch.exp(-2 * i / rot * math.log(c["theta"]))
    turn = torch.polar(torch.ones_like(t), t)
    y = x.clone()
    ia = torch.arange(h, device=x.device) * (1 if c["style"] == "halves" else 2)
    ib = ia + (h if c["style"] == "halves" else 1)
    z = torch.complex(x[..., ia], x[..., ib]) * turn
    y[..., ia], y[..., ib] = z.real, z.imag
    return y


def _exact_attention(q, k, v, sees, c):
    """q [rows, Hq, d], k and v [keys, Hkv, d], sees [rows, keys]."""
    g, d = c["Hq"] // c["Hkv"], c["d"]
    q = q.view(q.shape[0], c["Hkv"], g, d).permute(1, 2, 0, 3)
    z = torch.matmul(q, k.permute(1, 2, 0)[:, None]) / math.sqrt(d)
    z = torch.where(sees, z, -math.inf)
    o = torch.matmul(torch.softmax(z, -1), v.permute(1, 0, 2)[:, None])   # [Hkv, g, rows, d]
    return o.permute(2, 0, 1, 3).reshape(-1, c["Hq"], d)


def exact(case, seed):
    s = _inputs(case, seed)
    c, n = s["case"], s["n"]
    if c["op"].startswith("rotate"):
        pq, pk = _tokens(c, n)
        return dict(q=_exact_rotate(s["q"], s["gq"], pq, c), k=_exact_rotate(s["k"], s["gk"], pk, c))
    W, sinks = c["window"], c["sinks"]
    out, row, f, p0 = [], 0, 0, 0
    for r in range(n["R"]):
        P = int(n["P"][r])
        k, v = s["k"][p0:p0 + P].double(), s["v"][p0:p0 + P].double()
        j = torch.arange(P, device="cuda")
        if c["op"] == "prefill":
            step = max(1, (1 << 28) // (c["Hq"] * P))
            for a in range(0, P, step):
                b = min(P, a + step)
                p = torch.arange(a, b, device="cuda")[:, None]
                sees = (j[:b] <= p) & ((p - j[:b] < W) | (j[:b] < sinks))
                out.append(_exact_attention(s["q"][p0 + a:p0 + b].double(), k[:b], v[:b], sees, c))
            p0 += P
            continue
        # the prefix from the first key of any window on, and the first keys
        a = max(0, P - W)
        keep = (j < sinks) | (j >= a)
        nr = int(n["rows"][r])
        m = n["m"][r * c["cands"]:(r + 1) * c["cands"]]
        at = torch.cat([j[keep], torch.zeros(nr - 1, dtype=j.dtype, device="cuda")]).cpu()
        held = int(keep.sum())
        sees = torch.zeros(nr, held + nr - 1, dtype=torch.bool)
        pos = torch.full((nr,), P - 1)
        sees[:, :held] = True
        i = 1
        for length in m:
            for t in range(1, int(length)):
                pos[i] = P - 1 + t
                at[held + i - 1] = P - 1 + t
                sees[i, held + i - t:held + i] = True
                i += 1
        sees &= (pos[:, None] - at[None, :] < W) | (at[None, :] < sinks)
        k = torch.cat([k[keep], s["kc"][f:f + nr - 1].double()])
        v = torch.cat([v[keep], s["vc"][f:f + nr - 1].double()])
        out.append(_exact_attention(s["q"][row:row + nr].double(), k, v, sees.cuda(), c))
        row, f, p0 = row + nr, f + nr - 1, p0 + P
    return dict(o=torch.cat(out))


# --------------------------------------------------------------------------
# what a pass cannot do without
# --------------------------------------------------------------------------
def _seen(p, c):
    """The tokens that a token at position p sees."""
    near = np.minimum(p + 1, c["window"])
    return near + np.minimum(c["sinks"], p + 1 - near)


def work(case):
    c, n = case, _counts(case)
    eb = 2 if c["dtype"] == "bf16" else 4
    Hq, Hkv, d = c["Hq"], c["Hkv"], c["d"]
    if c["op"].startswith("rotate"):
        pq, pk = _tokens(c, n)
        elements = (len(pq) * Hq + len(pk) * Hkv) * d
        return dict(bytes=2 * elements * eb + (2 * d * eb if c["norm"] else 0),
                    flops=elements * (4 if c["norm"] else 0) + elements * 3 * c["rot"] // d)
    if c["op"] == "prefill":
        pairs = int(_seen(_ranges(n["P"])[1], c).sum())
        return dict(bytes=2 * n["S"] * (Hq + Hkv) * d * eb, flops=4 * pairs * Hq * d)
    # a row's own candidate tokens: those of the last `window`, and any that are first ones
    pairs = int(_seen(_rows(n)[3], c).sum())
    keys = int(_seen(n["P"] - 1, c).sum())
    return dict(bytes=2 * (keys + n["F"]) * Hkv * d * eb + 2 * n["N"] * Hq * d * eb,
                flops=4 * pairs * Hq * d)
