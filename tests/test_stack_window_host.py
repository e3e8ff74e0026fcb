"""Refusals of the decoder stack with positions and windows: what a layer would ignore. No call
here reaches a kernel."""
import pytest
import torch

# an address that passes the checks of alignment
A = 1 << 20
NAMES = ("g1", "g2", "w_mix", "w_o", "w_gu", "w_d", "s_prefix", "k_pre", "v_pre")


def _batch(jet):
    hl = jet.jet_layout_build([40, 7], [1, 1], [1, 3], [0] * 4, 4)
    dims = jet.make_dims(jet.DTYPE_BF16, Hq=8, Hkv=2, d=64, D=64, Hl=2, dk=128, dv=64)
    return hl, dims


BAD = [dict(sinks=2), dict(window=0, sinks=1), dict(gq=A), dict(gk=A), dict(window=9, gk=A)]


@pytest.mark.parametrize("bad", BAD)
@pytest.mark.parametrize("l", [0, 1])
def test_stack_call(jet, bad, l):
    hl, dims = _batch(jet)
    stack, keep = jet.make_stack([dict(kind=kind, **{n: A for n in NAMES})
                                  for kind in (jet.LAYER_LINEAR, jet.LAYER_FULL)], 128)
    attn = jet.make_stack_attn([bad if i == l else dict(window=9, sinks=1) for i in range(2)])
    with pytest.raises(jet.JetError, match="JET_ERR_ARG"):
        jet.jet_stack_forward_window(hl, dims, stack, None, attn, A, A, A, ws_bytes=1 << 40,
                                     stream=0)
    size = jet.jet_stack_window_workspace_bytes(hl.sizes, dims, 128, 2, attn)
    assert (size == 0) == ("sinks" in bad)
    assert keep is not None


@pytest.mark.parametrize("bad", BAD)
@pytest.mark.parametrize("l", [0, 1])
def test_decoder_stack(jet, bad, l):
    from paper_2609_33874_gb300.step import DecoderStack
    hl, dims = _batch(jet)
    x = torch.zeros(64)
    layers = [dict(kind=kind, **{n: x for n in NAMES}) for kind in ("linear", "full")]
    layers[l].update({k: x if k in ("gq", "gk") else v for k, v in bad.items()})
    with pytest.raises(ValueError, match="window|norm"):
        DecoderStack(hl, dims, layers, 128, device="cpu")
    # the same under a window and with a rope
    layers[l].update(window=5)
    DecoderStack(hl, dims, layers, 128, device="cpu", rope=jet.make_rope(64))
