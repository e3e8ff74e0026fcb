"""Host tests of positions and windows: the frequencies as fractions of a turn, what a
window sees (the kernels' arithmetic, compiled for the host, against the oracle's sets) and
the refusals. No call here reaches a kernel."""
import ctypes
import math
import os
import subprocess

import numpy as np
import pytest

from oracle import window as W

SRC = r"""
#include <cstdio>
#include "window.h"
int main() {
  int window, sinks, P, t;
  while (std::scanf("%d %d %d %d", &window, &sinks, &P, &t) == 4) {
    const jet::Seen s = jet::seen_at(jet::Window{window, sinks}, (long long)P - 1 + t);
    const jet::RowSeen r = jet::row_seen(jet::Window{window, sinks}, P, t);
    std::printf("%lld %lld %d %d %d %d", (long long)s.first, (long long)s.lo, r.pre_first,
                r.pre_lo, r.own_first, r.own_lo);
    const jet::Slots b = jet::step_slots(jet::Window{window, sinks}, P);
    std::printf(" %d %d %d\n", b.n, b.pad, b.off);
  }
}
"""


@pytest.fixture(scope="module")
def window_words(repo_root, tmp_path_factory):
    d = tmp_path_factory.mktemp("window")
    (d / "w.cpp").write_text(SRC)
    csrc = os.path.join(repo_root, "paper_2609_33874_gb300", "csrc")
    subprocess.run(["g++", "-std=c++17", "-Wall", "-Werror", "-I", csrc, str(d / "w.cpp"), "-o",
                    str(d / "w")], check=True)

    def run(cases):
        text = "\n".join(" ".join(map(str, c)) for c in cases)
        out = subprocess.run([str(d / "w")], input=text, capture_output=True, text=True, check=True)
        return [tuple(map(int, line.split())) for line in out.stdout.splitlines()]

    return run


def test_rows_see_what_the_oracle_says(window_words):
    rng = np.random.default_rng(4)
    cases = [(w, s, P, t) for w in (1, 2, 5, 40) for s in (0, 1, 3, 9, 60) for P in (1, 2, 8, 30)
             for t in (0, 1, 2, 11)]
    cases += [tuple(int(x) for x in rng.integers((1, 0, 1, 0), (50, 50, 60, 20)))
              for _ in range(500)]
    for (w, s, P, t), got in zip(cases, window_words(cases)):
        p = P - 1 + t
        first, lo, pre_first, pre_lo, own_first, own_lo = got[:6]
        assert first <= lo
        assert sorted({*range(first), *range(lo, p + 1)}) == W.seen(p, w, s)
        assert 0 <= pre_first <= pre_lo <= P and own_lo >= 1
        pre = {*range(pre_first), *range(pre_lo, P)}
        own = [*range(1, min(own_first, t) + 1)] + [*range(own_lo, t + 1)]
        assert len(own) == len(set(own))     # no token twice
        assert sorted(pre | {P - 1 + x for x in own}) == W.seen(p, w, s)


def test_slots_are_a_request_s_own_keys(window_words):
    """No slot is a key past the prefix, there are no more of them than the plans reckon with,
    and every key that the shared row sees has one."""
    cases = [(w, s, P, 0) for w in (1, 2, 17, 64) for s in (0, 1, 15, 16, 17, 49, 50, 62, 63, 200)
             for P in (1, 2, 10, 17, 63, 64, 65, 66, 80, 130, 300)]
    for (w, s, P, _), got in zip(cases, window_words(cases)):
        n, pad, off = got[6:]
        assert 1 <= n <= min(P, w + (s + 15) // 16 * 16) and pad % 16 == 0 and off >= 0
        keys = [i if i < pad else i + off for i in range(n)]
        assert len(set(keys)) == n and max(keys) == P - 1
        assert set(W.seen(P - 1, w, s)) <= set(keys)


def test_rows_at_the_largest_words(window_words):
    top = 2 ** 31 - 1
    for got in window_words([(top, 0, top, 5), (1, top, top, 5), (top, top, top, top)]):
        assert all(x >= 0 for x in got)
    # a window of one token at the far end, and every token a first one
    assert window_words([(1, 0, top, 0)])[0][:2] == (0, top - 1)
    assert window_words([(1, top, top, 0)])[0][:2] == (top - 1, top - 1)


def test_frequencies_are_fractions_of_a_turn(jet):
    r = jet.make_rope(64, theta=1e6, norm=False)
    f = W.frequencies(64, 1e6)
    for i in range(32):
        want = f[i] / (2 * math.pi) * 2.0 ** 64
        assert abs(float(r.turn[i]) - want) <= 2.0 ** -50 * want + 1
    assert all(r.turn[i] == 0 for i in range(32, 128))
    # whole turns count for nothing, and a backward one is its complement
    two = jet.make_rope(16, freq=[2 * math.pi, -math.pi / 2] + [0.25] * 6)
    assert two.turn[0] == 0 and two.turn[1] == 3 << 62
    assert (two.rot, two.style, two.norm) == (16, jet.ROPE_HALVES, 1)


@pytest.mark.parametrize("over,status", [
    (dict(rot=4), "JET_ERR_SHAPE"), (dict(rot=-8), "JET_ERR_SHAPE"),
    (dict(rot=264), "JET_ERR_SHAPE"), (dict(eps=-1e-6), "JET_ERR_ARG"),
    (dict(eps=math.inf), "JET_ERR_ARG"), (dict(eps=math.nan), "JET_ERR_ARG"),
    (dict(theta=0.0), "JET_ERR_ARG"), (dict(theta=math.inf), "JET_ERR_ARG"),
    (dict(theta=-1.0), "JET_ERR_ARG"), (dict(freq=[math.nan] * 4), "JET_ERR_ARG"),
    (dict(freq=[math.inf] * 4), "JET_ERR_ARG")])
def test_rope_refusals(jet, over, status):
    with pytest.raises(jet.JetError, match=status):
        jet.make_rope(**dict(dict(rot=8), **over))


def test_rope_refusals_of_the_binding(jet):
    with pytest.raises(ValueError):
        jet.make_rope(64, style="thirds")
    with pytest.raises(ValueError):
        jet.make_rope(64, freq=[1.0] * 31)
    out = jet.jet_rope()
    lib = jet.library()
    assert lib.jet_rope_init(8, 2, 1e4, None, 1, 1e-6, ctypes.byref(out)) == 1
    assert lib.jet_rope_init(8, 0, 1e4, None, 2, 1e-6, ctypes.byref(out)) == 1
    assert lib.jet_rope_init(8, 0, 1e4, None, 1, 1e-6, None) == 1


# addresses that pass the checks of alignment; no call below reaches a kernel
A, ODD = 1 << 20, (1 << 20) + 4


def _batch(jet, cand=(1, 3)):
    hl = jet.jet_layout_build([40, 7], [1, 1], list(cand), [0] * sum(cand), 4)
    return hl, jet.make_dims(jet.DTYPE_BF16, Hq=8, Hkv=2, d=64)


def _status(jet, call, *args, **kw):
    with pytest.raises(jet.JetError) as e:
        call(*args, **kw)
    return jet.STATUS_NAMES[e.value.status]


def test_rotation_refusals(jet):
    hl, dims = _batch(jet)
    rope = jet.make_rope(64)

    def given(rope=rope, dims=dims, n=3, pos=A, q=A, k=A, gq=A, gk=A, qo=A, ko=A):
        jet._check(jet.library().jet_norm_rotate(
            ctypes.byref(dims), ctypes.byref(rope), n, pos, q, k, gq, gk, qo, ko, None), "x")

    def of(form, **over):
        a = dict(dict(q=A, k=A, gq=A, gk=A, qo=A, ko=A), **over)
        form(hl, dims, rope, a["q"], a["k"], a["gq"], a["gk"], a["qo"], a["ko"], stream=0)

    bad = jet.jet_rope.from_buffer_copy(rope)
    bad.rot = 12
    assert _status(jet, given, rope=bad) == "JET_ERR_SHAPE"
    assert _status(jet, given, rope=jet.make_rope(128)) == "JET_ERR_SHAPE"   # heads of 64
    bad = jet.jet_rope.from_buffer_copy(rope)
    bad.style = 7
    assert _status(jet, given, rope=bad) == "JET_ERR_ARG"
    assert _status(jet, given, n=-1) == "JET_ERR_ARG"
    assert _status(jet, given, pos=None) == "JET_ERR_ARG"
    assert _status(jet, given, pos=A + 2) == "JET_ERR_ALIGN"
    wrong = jet.make_dims(jet.DTYPE_BF16, Hq=8, Hkv=3, d=64)
    assert _status(jet, given, dims=wrong) == "JET_ERR_SHAPE"
    wrong = jet.make_dims(jet.DTYPE_BF16, Hq=8, Hkv=2, d=96)
    assert _status(jet, given, dims=wrong) == "JET_ERR_UNSUPPORTED"
    wrong = jet.make_dims(7, Hq=8, Hkv=2, d=64)
    assert _status(jet, given, dims=wrong) == "JET_ERR_UNSUPPORTED"
    for form in (given, lambda **kw: of(jet.jet_norm_rotate_prefix, **kw),
                 lambda **kw: of(jet.jet_norm_rotate_rows, **kw)):
        for name in ("q", "k", "qo", "ko"):
            assert _status(jet, form, **{name: ODD}) == "JET_ERR_ALIGN"
            assert _status(jet, form, **{name: None}) == "JET_ERR_ARG"   # one without the other
        for name in ("gq", "gk"):
            assert _status(jet, form, **{name: ODD}) == "JET_ERR_ALIGN"
        assert _status(jet, form, q=None, k=None, qo=None, ko=None) == "JET_ERR_ARG"
    # no tokens: nothing to do
    given(n=0, pos=None)
    jet.jet_norm_rotate_rows(_batch(jet, (1, 1))[0], dims, rope, None, A, None, None, None, A,
                             stream=0)


def test_rotation_refusals_of_the_binding(jet):
    import torch
    _, dims = _batch(jet)
    rope = jet.make_rope(64)
    q, k = torch.zeros(3, 8, 64), torch.zeros(3, 2, 64)
    for pos in (torch.zeros(3), torch.zeros(3, dtype=torch.int64), torch.zeros(4, dtype=torch.int32),
                torch.zeros(3, 1, dtype=torch.int32)):
        with pytest.raises(ValueError):
            jet.jet_norm_rotate(dims, rope, pos, q, k, None, None, q, k, stream=0)


def test_window_refusals(jet):
    hl, dims = _batch(jet)
    size = jet.jet_attend_window_workspace_bytes(hl.sizes, dims, 16, 2)
    psize = jet.jet_prefill_window_workspace_bytes(hl.sizes, dims, 16, 2)
    assert size > 0 and psize > 0

    def step(dims=dims, window=16, sinks=2, q=A, k=A, v=A, kc=A, vc=A, o=A, ws=A, nb=1 << 30,
             hl=hl):
        jet.jet_prefix_attend_window(hl, dims, window, sinks, q, k, v, kc, vc, o, ws, ws_bytes=nb,
                                     stream=0)

    def prefill(dims=dims, window=16, sinks=2, q=A, k=A, v=A, o=A, ws=A, nb=1 << 30, hl=hl):
        jet.jet_prefill_attend_window(hl, dims, window, sinks, q, k, v, o, ws, ws_bytes=nb,
                                      stream=0)

    for call, need in ((step, size), (prefill, psize)):
        assert _status(jet, call, window=0) == "JET_ERR_ARG"
        assert _status(jet, call, window=-5) == "JET_ERR_ARG"
        assert _status(jet, call, sinks=-1) == "JET_ERR_ARG"
        assert _status(jet, call, ws=None) == "JET_ERR_WORKSPACE"
        assert _status(jet, call, nb=need - 1) == "JET_ERR_WORKSPACE"
        assert _status(jet, call, ws=ODD) == "JET_ERR_ALIGN"
        for name in ("q", "k", "v", "o") + (("kc", "vc") if call is step else ()):
            assert _status(jet, call, **{name: ODD}) == "JET_ERR_ALIGN"
            assert _status(jet, call, **{name: None}) == "JET_ERR_ARG"
        heads = jet.make_dims(jet.DTYPE_BF16, Hq=130, Hkv=1, d=64)
        assert _status(jet, call, dims=heads) == "JET_ERR_UNSUPPORTED"
        wrong = jet.make_dims(jet.DTYPE_BF16, Hq=8, Hkv=2, d=32)
        assert _status(jet, call, dims=wrong) == "JET_ERR_UNSUPPORTED"
        with pytest.raises(ValueError):
            call(window=1 << 32)
        with pytest.raises(ValueError):
            call(sinks=1 << 31)
    f32 = jet.make_dims(jet.DTYPE_F32, Hq=8, Hkv=2, d=64)
    assert _status(jet, prefill, dims=f32) == "JET_ERR_UNSUPPORTED"
    for f in (jet.jet_attend_window_workspace_bytes, jet.jet_prefill_window_workspace_bytes):
        assert f(hl.sizes, dims, 0, 0) == 0 and f(hl.sizes, dims, 4, -1) == 0
        assert f(hl.sizes, jet.make_dims(jet.DTYPE_BF16, Hq=8, Hkv=3, d=64), 4, 0) == 0
        assert f(hl.sizes, dims, 2 ** 31 - 1, 2 ** 31 - 1) > 0


def test_stack_refusals_hold_for_every_layer(jet):
    hl, _ = _batch(jet)
    dims = jet.make_dims(jet.DTYPE_BF16, Hq=8, Hkv=2, d=64, D=64, Hl=2, dk=128, dv=64)
    names = ("g1", "g2", "w_mix", "w_o", "w_gu", "w_d", "s_prefix", "k_pre", "v_pre")
    layers = [dict(kind=kind, **{n: A for n in names})
              for kind in (jet.LAYER_LINEAR, jet.LAYER_FULL)]
    stack, keep = jet.make_stack(layers, 128)
    good = [dict(window=9, sinks=1)] * 2
    n = jet.jet_stack_window_workspace_bytes(hl.sizes, dims, 128, 2, jet.make_stack_attn(good))
    assert n > 0

    def call(attn, nb=1 << 40):
        jet.jet_stack_forward_window(hl, dims, stack, None, jet.make_stack_attn(attn), A, A, A,
                                     ws_bytes=nb, stream=0)

    assert _status(jet, call, good, nb=n - 1) == "JET_ERR_WORKSPACE"
    for l in range(2):  # a linear layer's entry too
        for bad in (dict(window=-1), dict(window=9, sinks=-1)):
            attn = [bad if i == l else good[i] for i in range(2)]
            assert _status(jet, call, attn) == "JET_ERR_ARG"
            assert jet.jet_stack_window_workspace_bytes(hl.sizes, dims, 128, 2,
                                                        jet.make_stack_attn(attn)) == 0
    assert keep is not None


TILES = r"""
#include <cstdio>
#include "window.h"
// the keys that a vector sees, by slots and the words of a tile's mask
int main() {
  int window, sinks, P, t, first, end, prefill, tile;
  while (std::scanf("%d %d %d %d %d %d %d %d", &window, &sinks, &P, &t, &first, &end, &prefill,
                    &tile) == 8) {
    const jet::Window w{window, sinks};
    const jet::Slots s = prefill ? jet::block_slots(w, first, end) : jet::step_slots(w, P);
    long long vfirst, vlo, vend;
    if (prefill) {
      const jet::Seen x = jet::seen_at(w, t);
      vfirst = x.first, vlo = x.lo - s.off, vend = (long long)t + 1 - s.off;
    } else {
      const jet::RowSeen x = jet::row_seen(w, P, t);
      vfirst = x.pre_first, vlo = x.pre_lo - s.off, vend = P - s.off;
    }
    std::printf("%d %d %d :", s.n, s.pad, s.off);
    for (int k0 = 0; k0 < s.n; k0 += tile)
      for (int c0 = k0; c0 < k0 + tile; c0 += 32) {
        const unsigned see = jet::bit_range(-c0, int(vfirst) - c0) |
                             jet::bit_range(int(vlo) - c0, int(vend < s.n ? vend : s.n) - c0);
        for (int x = 0; x < 32; ++x)
          if (see >> x & 1u) std::printf(" %d", c0 + x < s.pad ? c0 + x : c0 + x + s.off);
      }
    std::printf("\n");
  }
}
"""


def test_slots_and_masks_give_what_the_oracle_says(repo_root, tmp_path):
    (tmp_path / "t.cpp").write_text(TILES)
    csrc = os.path.join(repo_root, "paper_2609_33874_gb300", "csrc")
    subprocess.run(["g++", "-std=c++17", "-Wall", "-Werror", "-I", csrc, str(tmp_path / "t.cpp"),
                    "-o", str(tmp_path / "t")], check=True)
    rng = np.random.default_rng(8)
    cases = []
    for w in (1, 2, 16, 50, 64, 200):
        for s in (0, 1, 15, 16, 17, 40, 64, 70, 130):
            for P in (1, 20, 64, 130, 300):
                for t in (0, 1, 5, 70):
                    cases.append((w, s, P, t, 0, 0, 0, 64))
                # a block of the prefill and a position in it
                first = int(rng.integers(0, P))
                end = min(P, first + int(rng.integers(1, 64)))
                cases.append((w, s, P, int(rng.integers(first, end)), first, end, 1, 128))
    text = "\n".join(" ".join(map(str, c)) for c in cases)
    out = subprocess.run([str(tmp_path / "t")], input=text, capture_output=True, text=True,
                         check=True).stdout.splitlines()
    assert len(out) == len(cases)
    for (w, s, P, t, first, end, prefill, _), line in zip(cases, out):
        head, keys = line.split(":")
        n, pad, off = map(int, head.split())
        keys = [int(k) for k in keys.split()]
        want = (W.seen(t, w, s) if prefill else
                [j for j in W.seen(P - 1 + t, w, s) if j < P])
        assert keys == want, (w, s, P, t, first, end, prefill)
        top = end if prefill else P
        assert n <= top + 15 and pad % 16 == 0
        assert n <= (end - first if prefill else 0) + w + -(-s // 16) * 16
        assert all(0 <= j < top for j in keys)
