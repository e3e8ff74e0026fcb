"""Positions and windows where the framework itself uses them: the scoring step and the decoder
stack, against the oracle; and the waits of the windowed kernels run out."""
import dataclasses

import numpy as np
import pytest

import jet_synth
import oracle as O
import window_bars as B
from gpu_common import oracle_layout
from oracle import stack as S
from oracle import window as W
from test_gpu_stack import (SMALL, TOL_STACK_MEAN_PER_LAYER, TOL_STACK_ROW_PER_LAYER, _layers,
                            _oracle_params)
from test_gpu_timeout import JET_ERR_TIMEOUT, JET_OK, _stalled
from test_gpu_window import Prefill, Step

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def cuda(jet):
    import torch
    if not torch.cuda.is_available():
        pytest.fail("CUDA device required for -m gpu tests")
    yield jet
    jet.jet_set_test_stall(False)
    jet.jet_set_wait_budget_ns(0)


def _np(x):
    return x.double().cpu().numpy()


def _scoring(cuda, bf16=True, **kw):
    from paper_2609_33874_gb300.step import ScoringStep
    w = dataclasses.replace(jet_synth.WORKLOADS["tiny"], dtype="bf16" if bf16 else "f32", Hq=8,
                            Hkv=2, d=64, D=256, V=500)
    m = [4, 1, 3, 2, 6]
    p = jet_synth.custom_problem(w, [90, 33], [3, 2], m, [5 * i % 500 for i in range(sum(m))],
                                 seed=31)
    hl = cuda.jet_layout_build(p.prefix_len, p.n_cand, p.cand_len, p.target_ids, w.V)
    dims = cuda.make_dims(cuda.DTYPE_BF16 if bf16 else cuda.DTYPE_F32, Hq=8, Hkv=2, d=64, D=256)
    step = ScoringStep(hl, dims, cuda.DECIDE_ARGMAX, device="cuda", **kw)
    x = {n: jet_synth.torch_tensor(p, n, device="cuda") for n in step.input_names()}
    return p, step, x, jet_synth.torch_tensor(p, "w_lm", device="cuda")


@pytest.mark.parametrize("bf16", [True, False])
def test_scoring_step_with_rope_and_window(cuda, bf16):
    import torch
    from paper_2609_33874_gb300.step import rotate_prefix
    rope = cuda.make_rope(32, style="pairs", theta=1e4)
    dt = torch.bfloat16 if bf16 else torch.float32
    gq, gk = (torch.rand(64, device="cuda").add(0.5).to(dt) for _ in range(2))
    p, step, x, w_lm = _scoring(cuda, bf16, window=20, sinks=3, rope=rope, gq=gq, gk=gk)
    raw = {n: x[n].clone() for n in x}
    x["k_pre"] = rotate_prefix(step.layout, step.dims, rope, x["k_pre"], gk)
    step.run(x, w_lm)
    torch.cuda.synchronize()
    assert cuda.jet_device_status() == 0
    lay = oracle_layout(p)
    f = W.frequencies(32, 1e4)
    pos = [W.row_position(lay, n) for n in range(lay["N"])]
    fed = lay["row_cand"] >= 0
    at = np.concatenate([np.arange(P) for P in p.prefix_len])
    # each rotation at its own bar, then the attention of what it gave
    for got, src, where, g in ((step._q, raw["q"], pos, gq),
                               (step._k_cand, raw["k_cand"], np.asarray(pos)[fed], gk),
                               (x["k_pre"], raw["k_pre"], at, gk)):
        want, bar = B.rotation(_np(src), where, 32, "pairs", f, _np(g), 1e-6, True, bf16)
        assert B.worst(_np(got), want, bar) <= 1.0
    for rows, want, bar in B.cascade(lay, *(_np(t) for t in (
            step._q, x["k_pre"], x["v_pre"], step._k_cand, x["v_cand"])), 20, 3, bf16).values():
        assert B.worst(_np(step.o)[rows], want, bar) <= 1.0
    for n in raw:   # the inputs stay as they were
        if n != "k_pre":
            assert torch.equal(x[n], raw[n])


def test_scoring_step_from_the_host_and_pipelined(cuda):
    import torch
    rope = cuda.make_rope(64)
    p, step, x, w_lm = _scoring(cuda, window=16, sinks=2, rope=rope)
    step.run(x, w_lm)
    torch.cuda.synchronize()
    want = step.cand_score.clone()
    from paper_2609_33874_gb300.step import HostBatch, HostResults
    host = {n: x[n].cpu().pin_memory() for n in step.input_names()}
    words = step.layout.words.cpu().pin_memory()
    out = {k: getattr(step, k).cpu().pin_memory()
           for k in ("tok_logprob", "cand_score", "q_cand", "choice", "value")}
    step.cand_score.zero_()
    step.run_from_host(host, words, w_lm, out)
    torch.cuda.synchronize()
    assert torch.equal(out["cand_score"], want.cpu())
    batches = [HostBatch(step, host, words) for _ in range(3)]
    outs = [HostResults(step) for _ in range(3)]
    step.overlap_min_bytes = 0
    step.run_pipelined(batches, w_lm, outs)
    torch.cuda.synchronize()
    for o in outs:
        assert torch.equal(o["cand_score"], want.cpu())
    assert cuda.jet_device_status() == 0


def test_scoring_step_refusals(cuda):
    for kw in (dict(window=8, kv="e4m3"), dict(sinks=2), dict(window=0), dict(window=4, sinks=-1),
               dict(gq=1)):
        with pytest.raises(ValueError):
            _scoring(cuda, **kw)


@pytest.mark.parametrize("window,sinks,rope", [(None, 0, True), (24, 3, True), (1, 0, False),
                                               (500, 9, True)])
def test_stack_with_rope_and_windows(cuda, window, sinks, rope):
    import torch
    from paper_2609_33874_gb300.step import DecoderStack
    spec = jet_synth.StackSpec(("full", "linear", "full"), 256)
    cl = [1, 3, 4, 2, 5]
    p = jet_synth.custom_problem(SMALL, [70, 33], [3, 2], cl,
                                 np.arange(sum(cl)) * 7 % SMALL.V, seed=43)
    w = p.work
    hl = cuda.jet_layout_build(p.prefix_len, p.n_cand, p.cand_len, p.target_ids, w.V)
    dims = cuda.make_dims(cuda.DTYPE_BF16, Hq=w.Hq, Hkv=w.Hkv, d=w.d, D=w.D, Hl=w.Hl, dk=w.dk,
                          dv=w.dv)
    layers = _layers(p, spec)
    gains = [torch.rand(w.d, device="cuda").add(0.5).bfloat16() for _ in range(4)]
    for i, l in enumerate((0, 2)):
        if rope:
            layers[l].update(gq=gains[2 * i], gk=gains[2 * i + 1])
        if window is not None and l == 2:   # the first full layer sees all
            layers[l].update(window=window, sinks=sinks)
    r = dict(rot=64, style="halves", freq=W.frequencies(64, 1e5), eps=1e-6, norm=True)
    st = DecoderStack(hl, dims, layers, spec.Dff, rope=cuda.make_rope(64, theta=1e5) if rope else None)
    x0 = jet_synth.array_to_torch(jet_synth.stack_x0(p), "cuda")
    outs = []
    for _ in range(2):
        outs.append(st.forward(x0).clone())
        torch.cuda.synchronize()
        assert cuda.jet_device_status() == 0
    assert torch.equal(*outs)
    lay = oracle_layout(p)
    od = dict(Hq=w.Hq, Hkv=w.Hkv, d=w.d, Hl=w.Hl, dk=w.dk, dv=w.dv, Dff=spec.Dff)
    x = jet_synth.bf16_to_f32(jet_synth.stack_x0(p)).astype(np.float64)
    for l, kind in enumerate(spec.kinds):
        P = _oracle_params(p, spec, l)
        if kind == "full":
            if rope:
                P.update(gq=_np(layers[l]["gq"]), gk=_np(layers[l]["gk"]))
            x = W.full_layer(lay, x, P, od, layers[l].get("window"), sinks, r if rope else None)
        else:
            x = S.layer_forward(lay, x, kind, P, od)
    # the bars of the stack without positions, per layer; the rotated queries and keys are
    # rounded once more (half a unit of 2^-8 each) before scores whose sum of squares is of the
    # order of one, which moves an output by less than the weights' rounding that the bars hold
    rms = np.sqrt(np.mean(x * x, axis=1, keepdims=True))
    rel = np.abs(_np(outs[0]) - x) / rms
    assert rel.max() <= 3 * TOL_STACK_ROW_PER_LAYER and rel.mean() <= 3 * TOL_STACK_MEAN_PER_LAYER


def test_stack_without_either_is_the_plain_stack(cuda):
    import torch
    from paper_2609_33874_gb300.step import DecoderStack
    spec = jet_synth.StackSpec(("full", "linear"), 256)
    p = jet_synth.custom_problem(SMALL, [70, 33], [2, 1], [3, 1, 4], [0] * 8, seed=44)
    w = p.work
    hl = cuda.jet_layout_build(p.prefix_len, p.n_cand, p.cand_len, p.target_ids, w.V)
    dims = cuda.make_dims(cuda.DTYPE_BF16, Hq=w.Hq, Hkv=w.Hkv, d=w.d, D=w.D, Hl=w.Hl, dk=w.dk,
                          dv=w.dv)
    st = DecoderStack(hl, dims, _layers(p, spec), spec.Dff)
    x0 = jet_synth.array_to_torch(jet_synth.stack_x0(p), "cuda")
    plain = st.forward(x0).clone()
    y = torch.empty_like(plain)
    attn = cuda.make_stack_attn([{}, {}])
    ws = torch.empty_like(st.ws)
    cuda.jet_stack_forward_window(st.layout, dims, st.stack, None, attn, x0, y, ws)
    torch.cuda.synchronize()
    assert torch.equal(plain, y) and cuda.jet_device_status() == 0


def test_stack_refusals(cuda):
    # nothing is launched: the addresses are never read
    import ctypes
    spec = jet_synth.StackSpec(("full",), 256)
    p = jet_synth.custom_problem(SMALL, [70], [1], [3], [0] * 3, seed=45)
    w = p.work
    hl = cuda.jet_layout_build(p.prefix_len, p.n_cand, p.cand_len, p.target_ids, w.V)
    dims = cuda.make_dims(cuda.DTYPE_BF16, Hq=w.Hq, Hkv=w.Hkv, d=w.d, D=w.D)
    lay = hl.to_device("cuda")
    stack, keep = cuda.make_stack([dict(L, kind=cuda.LAYER_FULL) for L in _layers(p, spec)], 256)
    rope = cuda.make_rope(64)
    A = 1 << 20
    for attn, r, status in (([dict(window=-1)], rope, "JET_ERR_ARG"),
                            ([dict(window=4, sinks=-1)], rope, "JET_ERR_ARG"),
                            ([dict(gq=A + 4)], rope, "JET_ERR_ALIGN"),
                            ([{}], cuda.make_rope(128), "JET_ERR_SHAPE")):
        with pytest.raises(cuda.JetError, match=status):
            cuda.jet_stack_forward_window(lay, dims, stack, r, cuda.make_stack_attn(attn), A, A, A,
                                          ws_bytes=1 << 40)
    n = cuda.jet_stack_window_workspace_bytes(hl.sizes, dims, 256, 1, cuda.make_stack_attn(
        [dict(window=20, sinks=2)]))
    assert n >= cuda.jet_stack_workspace_bytes(hl.sizes, dims, 256) > 0
    with pytest.raises(cuda.JetError, match="JET_ERR_WORKSPACE"):
        cuda.jet_stack_forward_window(lay, dims, stack, rope, cuda.make_stack_attn(
            [dict(window=20, sinks=2)]), A, A, A, ws_bytes=n - 1)
    assert cuda.jet_stack_window_workspace_bytes(hl.sizes, dims, 256, 1, cuda.make_stack_attn(
        [dict(window=-2)])) == 0
    with pytest.raises(ValueError):
        cuda.make_stack_attn([dict(window=1 << 31)])
    with pytest.raises(ValueError):
        big, _ = cuda.make_stack([{"kind": 0}] * 3, 256)
        cuda.jet_stack_forward_window(lay, dims, big, None, cuda.make_stack_attn([{}]), A, A, A,
                                      ws_bytes=0)
    assert keep is not None and ctypes.sizeof(cuda.jet_stack_attn) == 24


# --------------------------------------------------------------------------
# waits that run out
# --------------------------------------------------------------------------
@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("P", [[900, 90], [16] * 64])
def test_windowed_prefill_wait_runs_out(cuda, d, P):
    import torch
    p = Prefill(cuda, P, 32, 8, d, seed=7)
    ws = p.ws(300, 5)
    p.run(300, 5, ws=ws)
    first = p.o.clone()
    for _ in range(2):
        assert _stalled(cuda, lambda: cuda.jet_prefill_attend_window(
            p.dev, p.dims, 300, 5, p.q, p.k, p.v, p.o, ws)) == JET_ERR_TIMEOUT
    assert cuda.jet_device_status() == JET_OK
    p.o.fill_(7.0)
    p.run(300, 5, ws=ws)
    assert torch.equal(p.o, first)


@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("P", [[3000, 90], [40] * 200])
def test_windowed_step_wait_runs_out(cuda, d, P):
    import torch
    s = Step(cuda, P, [2] * len(P), [3, 2] * len(P), 8, 2, d, True, seed=7)
    ws = s.ws(2000, 5)
    s.run(2000, 5, ws=ws)
    first = s.o.clone()
    for _ in range(2):
        assert _stalled(cuda, lambda: cuda.jet_prefix_attend_window(
            s.dev, s.dims, 2000, 5, s.q, s.k, s.v, s.kc, s.vc, s.o, ws)) == JET_ERR_TIMEOUT
    assert cuda.jet_device_status() == JET_OK
    s.o.fill_(7.0)
    s.run(2000, 5, ws=ws)
    assert torch.equal(s.o, first)
