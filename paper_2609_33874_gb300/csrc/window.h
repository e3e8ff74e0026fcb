// Which keys a token sees under a window (jet_prefix_attend_window,
// jet_prefill_attend_window): of the tokens up to its own position p, the last `window` and
// the first `sinks`. Plain arithmetic, for the kernels and for host tests.
#pragma once

#include <stdint.h>

#ifndef JET_HD
#ifdef __CUDACC__
#define JET_HD __host__ __device__ __forceinline__
#else
#define JET_HD inline
#endif
#endif

namespace jet {

struct Window {
  int window, sinks;
};

// The tokens [0, first) and [lo, p] that position p sees, first <= lo.
struct Seen {
  int64_t first, lo;
};
JET_HD Seen seen_at(const Window& w, int64_t p) {
  Seen s;
  s.lo = p - w.window + 1;
  if (s.lo < 0) s.lo = 0;
  s.first = w.sinks < s.lo ? w.sinks : s.lo;
  return s;
}

// The same in 32 bits, of a position of a prefix (below 2^31).
struct Seen32 {
  int first, lo;
};
JET_HD Seen32 seen_at32(const Window& w, int p) {
  Seen32 s;
  s.lo = p - (w.window - 1);  // p >= 0 and window >= 1: above -2^31
  if (s.lo < 0) s.lo = 0;
  s.first = w.sinks < s.lo ? w.sinks : s.lo;
  return s;
}

// The same of a row of the step at t (0: the shared row) over a prefix of P tokens: prefix
// keys [0, pre_first) and [pre_lo, P), own candidate tokens [1, own_first] and [own_lo, t].
struct RowSeen {
  int pre_first, pre_lo, own_first, own_lo;
};
JET_HD RowSeen row_seen(const Window& w, int P, int t) {
  const Seen s = seen_at(w, int64_t(P) - 1 + t);
  RowSeen r;
  r.pre_lo = int(s.lo < P ? s.lo : P);
  r.pre_first = int(s.first < r.pre_lo ? s.first : r.pre_lo);
  const int64_t lo = s.lo - P + 1, first = s.first - P;
  r.own_lo = int(lo > 1 ? lo : 1);
  r.own_first = int(first > 0 ? first : 0);
  return r;
}

// Keys as the tiles of a tensor-core kernel take them: the first `sinks` keys and [lo, end)
// laid end to end. Slot i < pad holds key i (those from `sinks` on are masked), a later one
// key i + off. pad is a multiple of kSlotBox, the keys of one copy into a tile that holds both;
// 0 where lo lies before the end of the first keys' last box: then all of [0, end) are slots. So
// no slot is a key at or past end, and there are no more of them than keys.
constexpr int kSlotBox = 16;
struct Slots {
  int n, pad, off;
};
JET_HD Slots window_slots(const Window& w, int64_t lo, int64_t end) {
  Slots s;
  const int64_t pad = (int64_t(w.sinks) + kSlotBox - 1) / kSlotBox * kSlotBox;
  if (pad >= lo) {
    s.pad = s.off = 0;
    s.n = int(end);
  } else {
    s.pad = int(pad);
    s.off = int(lo - s.pad);
    s.n = int(s.pad + end - lo);
  }
  return s;
}

// The slots of a step's request (its shared row's window reaches back the farthest) and of a
// block of positions [first, end) of the prefill.
JET_HD Slots step_slots(const Window& w, int P) {
  return window_slots(w, seen_at(w, int64_t(P) - 1).lo, P);
}
JET_HD Slots block_slots(const Window& w, int first, int end) {
  return window_slots(w, seen_at(w, first).lo, end);
}

// Bits [lo, hi) of a word, of what lies in it.
JET_HD uint32_t bit_range(int lo, int hi) {
  if (lo < 0) lo = 0;
  if (hi > 32) hi = 32;
  if (hi <= lo) return 0u;
  return (hi == 32 ? ~0u : (1u << hi) - 1u) & (~0u << lo);
}

}  // namespace jet
