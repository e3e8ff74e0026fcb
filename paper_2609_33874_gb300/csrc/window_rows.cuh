// Attention of one query vector under a window by one warp, key by key in float32: what the
// kernels fall back on for a vector whose output came out NaN or infinite. The float32 step's sums
// of weighted values may pass the largest float where their mean does not. The tensor-core kernels'
// products take whole tiles, and a weight of zero times an infinite or NaN value that the vector
// does not see is NaN; here nothing but what it sees is read. A key takes a warp some 0.15 us, so
// in them this comes after a CTA's last item, when no role waits for another: they note the items
// with such an output, and all of the CTA's warps look those over.
#pragma once

#include "jet_device.cuh"
#include "window.h"

namespace jet {
namespace {

template <int PER>
__device__ __forceinline__ void load_row(const float* p, float (&v)[PER]) {
#pragma unroll
  for (int i = 0; i < PER; i += 2) {
    const float2 x = *reinterpret_cast<const float2*>(p + i);
    v[i] = x.x;
    v[i + 1] = x.y;
  }
}
template <int PER>
__device__ __forceinline__ void load_row(const __nv_bfloat16* p, float (&v)[PER]) {
#pragma unroll
  for (int i = 0; i < PER; i += 2) {
    const float2 x = __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162*>(p + i));
    v[i] = x.x;
    v[i + 1] = x.y;
  }
}

// A query vector's running softmax over keys in pieces: elements lane PER .. + PER - 1. acc is
// the mean so far, not its product with l, so it is no larger than the values.
template <int DH>
struct RowState {
  static constexpr int PER = DH / 32;
  float q[PER], acc[PER], m, l;
  bool over;  // every element is NaN, whatever comes

  // keys [begin, end) of k and v, rows `step` elements apart
  template <typename T>
  __device__ __forceinline__ void add(const T* k, const T* v, size_t step, int begin, int end,
                                      int lane) {
    constexpr int kAtOnce = 4;
    for (int j0 = begin; j0 < end && !over; j0 += kAtOnce) {
      float kv[kAtOnce][PER], vv[kAtOnce][PER], s[kAtOnce];
#pragma unroll
      for (int t = 0; t < kAtOnce; ++t) {
        const size_t at = size_t(min(j0 + t, end - 1)) * step + lane * PER;
        load_row<PER>(k + at, kv[t]);
        load_row<PER>(v + at, vv[t]);
      }
#pragma unroll
      for (int t = 0; t < kAtOnce; ++t) {
        s[t] = 0.f;
#pragma unroll
        for (int i = 0; i < PER; ++i) s[t] = fmaf(q[i], kv[t][i], s[t]);
        s[t] = warp_sum(s[t]);
      }
#pragma unroll
      for (int t = 0; t < kAtOnce; ++t) {
        if (j0 + t >= end) break;
        if (s[t] == -INFINITY) {  // weight 0, and 0 times an infinity or a NaN is NaN
#pragma unroll
          for (int i = 0; i < PER; ++i) acc[i] = fmaf(vv[t][i], 0.f, acc[i]);
          continue;
        }
        const float mn = fmaxf(m, s[t]);
        const float a = l * exp2f(m - mn), b = exp2f(s[t] - mn);
        l = a + b;
        m = mn;
        const float inv = 1.f / l;
#pragma unroll
        for (int i = 0; i < PER; ++i) acc[i] = acc[i] * (a * inv) + vv[t][i] * (b * inv);
      }
      bool nan = true;
#pragma unroll
      for (int i = 0; i < PER; ++i) nan &= isnan(acc[i]);
      over = __all_sync(0xffffffffu, nan);
    }
  }
};

template <int DH, typename T>
__device__ __forceinline__ void begin_row(RowState<DH>& s, const T* q, int lane) {
  const float scale = 1.4426950408889634f * rsqrtf(float(DH));  // base-2 scores
  load_row<RowState<DH>::PER>(q + lane * RowState<DH>::PER, s.q);
#pragma unroll
  for (int i = 0; i < RowState<DH>::PER; ++i) {
    s.q[i] *= scale;
    s.acc[i] = 0.f;
  }
  s.m = -INFINITY;
  s.l = 0.f;
  s.over = false;
}

template <int DH, typename T>
__device__ __forceinline__ void end_row(const RowState<DH>& s, T* o, int lane) {
  // scores all minus infinity: 0 / 0
  const float nan = s.l == 0.f ? __int_as_float(0x7fffffff) : 0.f;
#pragma unroll
  for (int i = 0; i < RowState<DH>::PER; ++i)
    o[lane * RowState<DH>::PER + i] = T(s.acc[i] + nan);
}

// one row of the step: its prefix keys from kp on, its own fed tokens from kc on (the first
// of them y_1), t of them
template <int DH, typename T>
__device__ __forceinline__ void row_attend(const Window& w, const T* q, const T* kp, const T* vp,
                                           const T* kc, const T* vc, size_t step, int P, int t,
                                           T* o, int lane) {
  const RowSeen see = row_seen(w, P, t);
  RowState<DH> s;
  begin_row(s, q, lane);
  s.add(kp, vp, step, 0, see.pre_first, lane);
  s.add(kp, vp, step, see.pre_lo, P, lane);
  if (t > 0) {
    s.add(kc, vc, step, 0, min(see.own_first, t), lane);
    s.add(kc, vc, step, see.own_lo - 1, t, lane);
  }
  end_row(s, o, lane);
}

// one position of the prefill
template <int DH>
__device__ __forceinline__ void position_attend(const Window& w, const __nv_bfloat16* q,
                                                const __nv_bfloat16* kp, const __nv_bfloat16* vp,
                                                size_t step, int p, __nv_bfloat16* o, int lane) {
  const Seen see = seen_at(w, p);
  RowState<DH> s;
  begin_row(s, q, lane);
  s.add(kp, vp, step, 0, int(see.first), lane);
  s.add(kp, vp, step, int(see.lo), p + 1, lane);
  end_row(s, o, lane);
}

// Which of a CTA's items have an output to compute again: a bit an item, those of kOddItems apart
// together.
constexpr int kOddItems = 1024;
struct OddItems {
  uint32_t bits[kOddItems / 32];
  __device__ __forceinline__ void note(int u) {
    atomicOr(bits + (u % kOddItems) / 32, 1u << (u % 32));
  }
  __device__ __forceinline__ bool has(int u) const {
    return bits[(u % kOddItems) / 32] >> (u % 32) & 1u;
  }
  __device__ __forceinline__ bool any(int lane) const {
    return __any_sync(0xffffffffu, bits[lane] != 0);
  }
};
static_assert(kOddItems == 32 * 32, "a word a lane");

// Whether a vector's stored output, whole, has a NaN or an infinity.
template <int DH>
__device__ __forceinline__ bool stored_odd(const __nv_bfloat16* o, int lane) {
  bool odd = false;
#pragma unroll
  for (int i = 0; i < DH / 32; i += 2) {
    const uint32_t x = *reinterpret_cast<const uint32_t*>(o + lane * (DH / 32) + i);
    odd |= (x & 0x7f80u) == 0x7f80u || (x & 0x7f800000u) == 0x7f800000u;
  }
  return __any_sync(0xffffffffu, odd);
}

}  // namespace
}  // namespace jet
