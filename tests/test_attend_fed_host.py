"""Which parts of a batch the words of a layout may name (csrc/attend_items.h, plain
arithmetic), on the host: over random plans and row offsets that pass the cut of a
request, true or not, fed_inside admits exactly the ranges of the batch's N - R fed
tokens, and every range of a true layout; span_inside exactly the parts of a total."""
import os
import subprocess

HARNESS = r"""
#include <cstdio>
#include <cstdlib>
#include "attend_items.h"
using namespace jet;
#define CHECK(x) do { if (!(x)) { std::printf("line %d: %s\n", __LINE__, #x); return 1; } } while (0)

static int rnd(int lo, int hi) { return lo + std::rand() % (hi - lo + 1); }

int main() {
  int before = 0, past = 0;  // ranges that start before the first token, end past the last
  for (int it = 0; it < 3000; ++it) {
    std::srand(it);
    ItemPlan a{};
    a.R = rnd(1, 6);
    a.Hkv = 1;
    a.g = rnd(1, 64);
    a.rb = 128 / a.g;
    a.has_cand = 1;
    a.total_prefix = 1000;
    a.chunk = 128;
    a.splits = 8;
    int nr[6], n0 = 0;
    for (int r = 0; r < a.R; ++r) a.N += nr[r] = rnd(1, 30);
    a.qgroups = (a.N + a.rb - 1) / a.rb;
    const int F = a.N - a.R;
    for (int r = 0; r < a.R; ++r) {
      // the request as it is: all of its blocks' tokens, from any of them on
      const RequestCut cut = request_cut(a, n0, nr[r], 0, 100);
      for (int qb = 0; qb < cut.nq; ++qb) {
        const ItemGeo e = item_geo_at(a, r, 0, qb, 0, n0, nr[r], 0, 100, cut);
        const int fed = e.row0 + e.nv / a.g - 1;
        CHECK(e.ok);
        for (int lo = 0; lo <= fed; ++lo) CHECK(fed_inside(a, e.f_begin + lo, fed - lo));
      }
      n0 += nr[r];
      // other words
      const int x = rnd(0, a.N - 1), n = rnd(1, a.N - x);
      const RequestCut other = request_cut(a, x, n, 0, 100);
      CHECK(other.nq > 0);
      for (int qb = 0; qb < other.nq; ++qb) {
        const ItemGeo e = item_geo_at(a, r, 0, qb, 0, x, n, 0, 100, other);
        const int fed = e.row0 + e.nv / a.g - 1;
        for (int lo = 0; lo <= fed; ++lo) {
          const int f = e.f_begin + lo, k = fed - lo;
          CHECK(fed_inside(a, f, k) == (f >= 0 && f + k <= F));
          before += k > 0 && f < 0;
          past += k > 0 && f + k > F;
        }
      }
    }
  }
  CHECK(before > 100 && past > 100);  // such words do pass the cut
  ItemPlan a{};
  a.R = 3;
  a.N = 13;
  const int big = 2147483647;
  CHECK(fed_inside(a, 0, 10) && fed_inside(a, 10, 0) && !fed_inside(a, 11, 0));
  CHECK(!fed_inside(a, big, big) && !fed_inside(a, 5, big) && !fed_inside(a, big, 1));
  CHECK(!fed_inside(a, -1, 2) && !fed_inside(a, -big - 1, big) && !fed_inside(a, 0, -1));
  const int word[] = {-big - 1, -big, -7, -1, 0, 1, 6, 9, 10, 11, big - 1, big};
  const int total[] = {0, 1, 9, 10, big};
  for (int b : word)
    for (int e : word)
      for (int t : total)
        CHECK(span_inside(b, e, t) ==
              ((long long)b >= 0 && (long long)e - b >= 0 && (long long)e <= t));
  CHECK(!span_inside(big, -big - 1, 10));  // whose difference wraps to 1
  a.R = 20;  // fewer rows than requests: no token at all
  CHECK(!fed_inside(a, 0, 0) && !fed_inside(a, 0, 1));
  return 0;
}
"""


def test_fed_tokens_stay_inside_the_batch(tmp_path, repo_root):
    src, exe = tmp_path / "fed.cpp", tmp_path / "fed"
    src.write_text(HARNESS)
    inc = os.path.join(repo_root, "paper_2609_33874_gb300", "csrc")
    subprocess.run([os.environ.get("CXX", "g++"), "-std=c++17", "-O1", "-Wall", "-Werror", "-I", inc,
                    str(src), "-o", str(exe)], check=True)
    run = subprocess.run([str(exe)], capture_output=True, text=True)
    assert run.returncode == 0, run.stdout
