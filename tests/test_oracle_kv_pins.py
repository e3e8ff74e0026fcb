"""Pins of the 8-bit prefix cache's oracle (oracle/kv_e4m3.py) by hand-made values,
and of the cache's arithmetic in csrc/kv_cache.h (places of blocks, exponents) by a
host program."""
import os
import subprocess

import numpy as np
import pytest

from oracle import kv_e4m3 as K


def test_exponents_by_hand():
    one = lambda v: K.exponent(np.array(v, np.float64).reshape(1, 1, -1))[0]  # noqa: E731
    assert one([448.0]) == 0 and one([-448.0, 3.0]) == 0
    assert one([448.0000001]) == 1 and one([224.0]) == -1 and one([224.5]) == 0
    assert one([1.75]) == -8 and one([1.0]) == -8 and one([1.7500001]) == -7
    assert one([0.0]) == -117 and one([1e-45]) == -117 and one([3.4e38]) == 119
    assert one([np.nan, 2.0, -np.inf]) == -7 and one([np.inf]) == -117


def test_codes_by_hand():
    X = np.array([0])
    x = np.array([448.0, -448.0, 1.0, 1.0625, 1.1875, 2.0 ** -9, 2.0 ** -10, -0.0, np.inf,
                  np.nan]).reshape(1, 1, -1)
    c = K.encode(x, X).reshape(-1)
    # 1.0625 and 1.1875 lie halfway: to the even mantissa; 2^-10 is half the least code
    assert c.tolist() == [0x7E, 0xFE, 0x38, 0x38, 0x3A, 0x01, 0x00, 0x80, 0x7F, 0x7F]
    v = K.value(c.reshape(1, 1, -1), np.array([3])).reshape(-1)
    assert v[0] == 448.0 * 8 and v[5] == 2.0 ** -6 and np.isnan(v[8])


def test_error_of_a_value():
    # half a step of e4m3 relative to the element, or half the least code
    rng = np.random.default_rng(0)
    x = (rng.standard_normal((64, 3, 64)) * np.exp(rng.standard_normal((64, 3, 64)))).astype(
        np.float32)
    X = K.exponent(x)
    err = np.abs(K.value(K.encode(x, X), X) - x)
    assert np.all(err <= np.maximum(np.abs(x) * 2.0 ** -4, 2.0 ** (X[None, :, None] - 10.0)))


def test_values_are_numbers_of_bf16():
    codes = np.arange(256, dtype=np.uint8).reshape(1, 1, -1)
    for X in (K.X_MIN, 0, K.X_MAX):
        v = K.value(codes, np.array([X]))
        v = v[np.isfinite(v)].astype(np.float32)
        bits = v.view(np.uint32)
        assert not (bits & 0xFFFF).any()
        assert np.all((v == 0) | (np.abs(v) >= 2.0 ** -126)) and np.isfinite(v).all()


def test_append_matches_whole_where_no_exponent_grows():
    rng = np.random.default_rng(1)
    x = rng.uniform(1.0, 1.7, (200, 2, 64))  # one binade: every block has the same exponent
    whole = K.Cache([130, 70], 2, 64).write(x)
    parts = K.Cache([130, 70], 2, 64)
    for r, p0, P in ((0, 0, 130), (1, 130, 70)):
        at = 0
        while at < P:
            n = min(P - at, int(rng.integers(1, 50)))
            parts.append(r, at, x[p0 + at:p0 + at + n])
            at += n
    np.testing.assert_array_equal(parts.buffer(), whole.buffer())


def test_append_rounds_again_where_it_grows():
    c = K.Cache([3], 1, 64)
    c.append(0, 0, np.full((1, 1, 64), 1.1))     # X = -8: code of 281.6 = 288
    c.append(0, 1, np.full((1, 1, 64), 1000.0))  # X = 2
    assert c.X[0][0, 0] == 2
    v = c.values().reshape(3, 64)
    # 288 2^-8 = 1.125 = 0.28125 2^2: a code
    assert np.all(v[0] == 1.125) and np.all(v[1] == 1024.0) and np.all(v[2] == 0)


HARNESS = r"""
#include <cmath>
#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <vector>
#include "kv_cache.h"
using namespace jet;
#define CHECK(x) do { if (!(x)) { std::printf("line %d: %s\n", __LINE__, #x); return 1; } } while (0)

static int rnd(int lo, int hi) { return lo + std::rand() % (hi - lo + 1); }

int main() {
  // no two blocks share a place, and every place lies within the buffer
  for (int it = 0; it < 2000; ++it) {
    std::srand(it);
    jet_sizes n{};
    jet_dims d{};
    d.Hkv = rnd(1, 5);
    d.d = 64;
    n.R = rnd(1, 40);
    const int most = it % 3 == 0 ? 3 : it % 3 == 1 ? 130 : 1000;
    std::vector<int> P(n.R);
    for (int& p : P) n.total_prefix += p = rnd(1, most);
    const KvSize z = kv_size(n, d);
    CHECK(z.exp_off >= size_t(n.total_prefix) * d.Hkv * d.d && z.exp_off % 256 == 0);
    CHECK(z.bytes >= z.exp_off + size_t(z.blocks) * d.Hkv && z.bytes % 256 == 0);
    std::vector<int> used(size_t(z.blocks), 0);
    for (int r = 0, p0 = 0; r < n.R; p0 += P[r++])
      for (int b = 0; b * kKvBlock < P[r]; ++b) {
        const int at = kv_place(p0, r, b);
        CHECK(at >= 0 && at < z.blocks && !used[at]);
        used[at] = 1;
      }
    // the places of appended tokens hold every block they touch
    int rows = 0;
    std::vector<int> off(1, 0), first(n.R), count(n.R);
    for (int r = 0; r < n.R; ++r) {
      first[r] = rnd(0, P[r]);
      count[r] = rnd(0, P[r] - first[r]);
      off.push_back(rows += count[r]);
    }
    for (int r = 0; r < n.R; ++r) {
      const int base = off[r] / kKvBlock + 2 * r, end = off[r + 1] / kKvBlock + 2 * (r + 1);
      CHECK(end <= kv_append_places(n, rows));
      if (count[r] == 0) continue;
      const int blocks = (first[r] + count[r] - 1) / kKvBlock - first[r] / kKvBlock + 1;
      CHECK(base + blocks <= end);
    }
  }
  // the exponent is the least of the range with amax <= 448 2^X
  for (int it = 0; it < 200000; ++it) {
    unsigned bits = (unsigned(std::rand()) << 16 ^ unsigned(std::rand())) & 0x7fffffffu;
    if (it < 300) bits = unsigned(it < 255 ? it : 254) << 23 | (it & 1 ? 0x600000u : 0x600001u);
    if (bits >= 0x7f800000u) continue;
    float f;
    std::memcpy(&f, &bits, 4);
    const int x = kv_exponent(bits);
    CHECK(x >= kKvLow && x <= kKvHigh);
    CHECK(x == kKvHigh || double(f) <= std::ldexp(448.0, x));
    CHECK(x == kKvLow || double(f) > std::ldexp(448.0, x - 1));
  }
  std::puts("ok");
  return 0;
}
"""


def test_places_and_exponents_on_the_host(repo_root, tmp_path):
    src = tmp_path / "kv.cpp"
    src.write_text(HARNESS)
    exe = tmp_path / "kv"
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-Werror", "-I",
                    os.path.join(repo_root, "include"), "-I",
                    os.path.join(repo_root, "paper_2609_33874_gb300", "csrc"), str(src), "-o",
                    str(exe)], check=True)
    out = subprocess.run([str(exe)], stdout=subprocess.PIPE, text=True)
    assert out.returncode == 0 and out.stdout.strip() == "ok", out.stdout


# ---------------------------------------------------------------------------
# the entry points' refusals: nothing is launched
# ---------------------------------------------------------------------------
FAKE = 1 << 40          # 16-byte aligned address that is never dereferenced
MIS = FAKE + 4


def _setup(jet):
    lay = jet.jet_layout_build([4, 130], [2, 2], [1, 3, 2, 1], list(range(7)), 16)
    return lay, jet.make_dims(jet.DTYPE_BF16, Hq=8, Hkv=2, d=64)


def _status(fn, *args, **kw):
    try:
        fn(*args, stream=0, **kw)
    except Exception as e:  # JetError
        return e.status
    return 0


def test_sizes(jet):
    lay, dims = _setup(jet)
    # 134 tokens x 2 heads x 64 codes, then 134 // 64 + 2 places x 2 heads, 256 each
    assert jet.jet_kv_e4m3_bytes(lay.sizes, dims) == 17152 + 256
    for kw in (dict(Hkv=2, d=96), dict(Hkv=0, d=64)):
        assert jet.jet_kv_e4m3_bytes(lay.sizes, jet.make_dims(jet.DTYPE_BF16, **kw)) == 0
    assert jet.jet_kv_e4m3_bytes(lay.sizes, jet.make_dims(3, Hkv=2, d=64)) == 0
    assert jet.jet_attend_workspace_bytes_e4m3(lay.sizes, dims) > 0
    assert jet.jet_attend_workspace_bytes_e4m3(lay.sizes, jet.make_dims(0, Hq=3, Hkv=2, d=64)) == 0


@pytest.mark.parametrize("call", ["jet_quantize_kv_e4m3", "jet_dequantize_kv_e4m3"])
def test_cache_refusals(jet, call):
    lay, dims = _setup(jet)
    fn = getattr(jet, call)
    for i in range(4):
        for what, status in ((None, 1), (MIS, 4)):
            args = [FAKE] * 4
            args[i] = what
            assert _status(fn, lay, dims, *args) == status
    for bad, status in ((dict(Hkv=2, d=96), 7), (dict(Hkv=0, d=64), 2)):
        assert _status(fn, lay, jet.make_dims(jet.DTYPE_F32, **bad), *[FAKE] * 4) == status
    assert _status(fn, lay, jet.make_dims(9, Hkv=2, d=64), *[FAKE] * 4) == 7
    # more CTAs than a grid holds
    big = jet.jet_layout_build([1 << 20], [1], [1], [0], 16)
    many = jet.make_dims(jet.DTYPE_BF16, Hkv=1 << 17, d=64)
    assert _status(fn, big, many, *[FAKE] * 4) == 6
    empty = jet.jet_layout_build([], [], [], [], 16)
    assert _status(fn, empty, dims, *[None] * 4) == 0


def test_append_refusals(jet):
    lay, dims = _setup(jet)
    lib = jet.library()
    import ctypes
    L, D = ctypes.byref(lay.struct), ctypes.byref(dims)

    def call(start=FAKE, off=FAKE, n=3, k=FAKE, v=FAKE, k8=FAKE, v8=FAKE):
        return lib.jet_append_kv_e4m3(L, D, start, off, n, k, v, k8, v8, None)

    assert call(n=-1) == 1 and call(n=135) == 2       # more new tokens than the prefixes hold
    assert call(n=0, k=None, v=None) == 0             # nothing to write
    assert call(start=None) == 1 and call(off=None) == 1
    assert call(start=FAKE + 2) == 4 and call(off=FAKE + 1) == 4
    for name in ("k", "v", "k8", "v8"):
        assert call(**{name: None}) == 1 and call(**{name: MIS}) == 4


def test_attend_refusals(jet):
    lay, dims = _setup(jet)
    ws = jet.jet_attend_workspace_bytes_e4m3(lay.sizes, dims)

    def call(d=dims, ws_bytes=ws, **at):
        args = [at.get(n, FAKE) for n in ("q", "k8", "v8", "k_cand", "v_cand", "o", "ws")]
        return _status(jet.jet_prefix_attend_e4m3, lay, d, *args, ws_bytes=ws_bytes)

    for name in ("q", "k8", "v8", "k_cand", "v_cand", "o"):
        assert call(**{name: None}) == 1 and call(**{name: MIS}) == 4
    assert call(ws_bytes=16) == 5 and call(ws=None) == 5 and call(ws=MIS) == 4
    assert call(d=jet.make_dims(jet.DTYPE_BF16, Hq=6, Hkv=4, d=64)) == 2
    assert call(d=jet.make_dims(jet.DTYPE_BF16, Hq=8, Hkv=2, d=96)) == 7
    assert call(d=jet.make_dims(7, Hq=8, Hkv=2, d=64)) == 7
    # more query heads a kv head than the tensor-core kernel's block holds
    assert call(d=jet.make_dims(jet.DTYPE_BF16, Hq=129, Hkv=1, d=64), ws_bytes=1 << 40) == 7
    empty = jet.jet_layout_build([], [], [], [], 16)
    assert _status(jet.jet_prefix_attend_e4m3, empty, dims, *[None] * 7, ws_bytes=0) == 0


def test_buffers_of_another_size_are_refused(jet):
    import torch
    lay, dims = _setup(jet)
    x = torch.zeros(134, 2, 64, dtype=torch.bfloat16)
    nb = jet.jet_kv_e4m3_bytes(lay.sizes, dims)
    good, short = torch.zeros(nb, dtype=torch.uint8), torch.zeros(nb - 1, dtype=torch.uint8)
    wide = torch.zeros(nb, dtype=torch.int16)
    for bad in (short, wide):
        for a, b in ((good, bad), (bad, good)):
            with pytest.raises(ValueError):
                jet.jet_quantize_kv_e4m3(lay, dims, x, x, a, b, stream=0)
            with pytest.raises(ValueError):
                jet.jet_append_kv_e4m3(lay, dims, FAKE, FAKE, x, x, a, b, stream=0)
            with pytest.raises(ValueError):
                jet.jet_dequantize_kv_e4m3(lay, dims, a, b, x, x, stream=0)
            with pytest.raises(ValueError):
                jet.jet_prefix_attend_e4m3(lay, dims, x, a, b, x, x, x, x, stream=0)
    with pytest.raises(ValueError):
        jet.jet_append_kv_e4m3(lay, dims, FAKE, FAKE, x, x[:5], good, good, stream=0)
