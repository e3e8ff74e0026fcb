// Attention under a window with first tokens that stay visible: one warp a query vector,
// key by key, in float32, for both types and every shape.
#include <algorithm>

#include "attend_items.h"
#include "jet_device.cuh"
#include "jet_internal.h"
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

// A query vector's running softmax over keys in pieces: elements lane PER .. + PER - 1
template <int DH>
struct RowState {
  static constexpr int PER = DH / 32;
  float q[PER], acc[PER], m, l;

  // keys [begin, end) of k and v, rows `step` elements apart
  template <typename T>
  __device__ __forceinline__ void add(const T* k, const T* v, size_t step, int begin, int end,
                                      int lane) {
    constexpr int kAtOnce = 4;
    for (int j0 = begin; j0 < end; j0 += kAtOnce) {
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
        const float mn = fmaxf(m, s[t]);
        const float a = mn == -INFINITY ? 1.f : exp2f(m - mn);
        const float b = mn == -INFINITY ? 0.f : exp2f(s[t] - mn);
#pragma unroll
        for (int i = 0; i < PER; ++i) acc[i] = acc[i] * a + b * vv[t][i];
        l = l * a + b;
        m = mn;
      }
    }
  }
};

struct RowArgs {
  Window w;
  const int32_t* prefix_offset;
  const int32_t* row_offset;
  const int32_t* row_req;
  const int32_t* row_cand;
  const int32_t* row_pos;
  int R, N, total, Hq, Hkv;
  int* status;
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
}

template <int DH, typename T>
__device__ __forceinline__ void end_row(const RowState<DH>& s, T* o, int lane) {
  const float inv = 1.f / s.l;
#pragma unroll
  for (int i = 0; i < RowState<DH>::PER; ++i)
    o[lane * RowState<DH>::PER + i] = from_f32<T>(s.acc[i] * inv);
}

// the step: one warp per (row, query head)
template <int DH, typename T>
__global__ void __launch_bounds__(128)
attend_window_rows_kernel(const RowArgs a, const T* q, const T* k_pre, const T* v_pre,
                          const T* k_cand, const T* v_cand, T* o) {
  pdl_begin();
  const int lane = threadIdx.x & 31;
  const long long idx = (long long)blockIdx.x * (blockDim.x >> 5) + (threadIdx.x >> 5);
  if (idx >= (long long)a.N * a.Hq) return;
  const int n = int(idx / a.Hq), h = int(idx % a.Hq), kh = h / (a.Hq / a.Hkv);
  const int r = a.row_req[n], c = a.row_cand[n], t = c < 0 ? 0 : a.row_pos[n];
  bool ok = r >= 0 && r < a.R && t >= 0 && t <= n;
  int p0 = 0, p1 = 0;
  if (ok) {
    p0 = a.prefix_offset[r];
    p1 = a.prefix_offset[r + 1];
    ok = span_inside(p0, p1, a.total) && p1 > p0;
  }
  // the row's fed tokens y_1 .. y_t are [f0 + 1, f0 + t]
  const int f0 = n - r - 1 - t;
  if (ok && t > 0) ok = f0 >= -1 && n - r - 1 < a.N - a.R;
  if (!ok) {
    if (lane == 0) flag(a.status, JET_ERR_DEVICE);
    return;
  }
  const RowSeen see = row_seen(a.w, p1 - p0, t);
  RowState<DH> s;
  begin_row(s, q + size_t(idx) * DH, lane);
  const size_t step = size_t(a.Hkv) * DH;
  const T* kp = k_pre + size_t(p0) * step + size_t(kh) * DH;
  const T* vp = v_pre + size_t(p0) * step + size_t(kh) * DH;
  s.add(kp, vp, step, 0, see.pre_first, lane);
  s.add(kp, vp, step, see.pre_lo, p1 - p0, lane);
  if (t > 0) {
    const T* kc = k_cand + size_t(kh) * DH;
    const T* vc = v_cand + size_t(kh) * DH;
    s.add(kc, vc, step, f0 + 1, f0 + 1 + min(see.own_first, t), lane);
    s.add(kc, vc, step, f0 + see.own_lo, f0 + t + 1, lane);
  }
  end_row<DH, T>(s, o + size_t(idx) * DH, lane);
}

// the prefill: one warp per (position, query head); a request's positions are its rows
template <int DH>
__global__ void __launch_bounds__(128)
prefill_window_rows_kernel(const RowArgs a, const __nv_bfloat16* q, const __nv_bfloat16* k,
                           const __nv_bfloat16* v, __nv_bfloat16* o) {
  pdl_begin();
  const int lane = threadIdx.x & 31;
  const int r = int(blockIdx.y);
  const int p0 = a.prefix_offset[r], p1 = a.prefix_offset[r + 1];
  if (!span_inside(p0, p1, a.total)) {
    if (threadIdx.x == 0) flag(a.status, JET_ERR_DEVICE);
    return;
  }
  const long long idx = (long long)blockIdx.x * (blockDim.x >> 5) + (threadIdx.x >> 5);
  if (idx >= (long long)(p1 - p0) * a.Hq) return;
  const int p = int(idx / a.Hq), h = int(idx % a.Hq), kh = h / (a.Hq / a.Hkv);
  const Seen see = seen_at(a.w, p);
  const size_t step = size_t(a.Hkv) * DH, at = (size_t(p0 + p) * a.Hq + h) * DH;
  RowState<DH> s;
  begin_row(s, q + at, lane);
  const __nv_bfloat16* kp = k + size_t(p0) * step + size_t(kh) * DH;
  const __nv_bfloat16* vp = v + size_t(p0) * step + size_t(kh) * DH;
  s.add(kp, vp, step, 0, int(see.first), lane);
  s.add(kp, vp, step, int(see.lo), p + 1, lane);
  end_row<DH, __nv_bfloat16>(s, o + at, lane);
}

template <int DH, typename T>
cudaError_t launch_rows(const RowArgs& a, const void* q, const void* k_pre, const void* v_pre,
                        const void* k_cand, const void* v_cand, void* o, cudaStream_t st) {
  const long long warps = (long long)a.N * a.Hq;
  return launch_pdl(attend_window_rows_kernel<DH, T>, dim3(unsigned((warps + 3) / 4)), dim3(128), 0,
                    st, a, static_cast<const T*>(q), static_cast<const T*>(k_pre),
                    static_cast<const T*>(v_pre), static_cast<const T*>(k_cand),
                    static_cast<const T*>(v_cand), static_cast<T*>(o));
}

RowArgs row_args(const jet_layout& lay, const jet_dims& d, int window, int sinks, int* status) {
  RowArgs a{};
  a.w = Window{window, sinks};
  a.prefix_offset = lay.prefix_offset;
  a.row_offset = lay.row_offset;
  a.row_req = lay.row_req;
  a.row_cand = lay.row_cand;
  a.row_pos = lay.row_pos;
  a.R = lay.n.R;
  a.N = lay.n.N;
  a.total = lay.n.total_prefix;
  a.Hq = d.Hq;
  a.Hkv = d.Hkv;
  a.status = status;
  return a;
}

}  // namespace

size_t attend_window_bytes(const jet_sizes&, const jet_dims&, int, int) { return 16; }

size_t prefill_window_bytes(const jet_sizes&, const jet_dims&, int, int) { return 16; }

cudaError_t launch_attend_window(const jet_layout& lay, const jet_dims& d, int window, int sinks,
                                 const void* q, const void* k_pre, const void* v_pre,
                                 const void* k_cand, const void* v_cand, void* o, void*,
                                 int* status, cudaStream_t st) {
  const RowArgs a = row_args(lay, d, window, sinks, status);
#define JET_WIN(DH)                                                                             \
  if (d.d == DH)                                                                                \
    return d.dtype == JET_DTYPE_BF16                                                            \
               ? launch_rows<DH, __nv_bfloat16>(a, q, k_pre, v_pre, k_cand, v_cand, o, st)      \
               : launch_rows<DH, float>(a, q, k_pre, v_pre, k_cand, v_cand, o, st)
  JET_WIN(64);
  JET_WIN(128);
  JET_WIN(256);
#undef JET_WIN
  return cudaErrorInvalidValue;
}

cudaError_t launch_prefill_window(const jet_layout& lay, const jet_dims& d, int window, int sinks,
                                  const void* q, const void* k, const void* v, void* o, void*,
                                  int* status, cudaStream_t st) {
  const RowArgs a = row_args(lay, d, window, sinks, status);
  const long long warps = (long long)lay.n.max_prefix * d.Hq;
  const dim3 grid{unsigned((warps + 3) / 4), unsigned(lay.n.R)};
  const auto* qb = static_cast<const __nv_bfloat16*>(q);
  const auto* kb = static_cast<const __nv_bfloat16*>(k);
  const auto* vb = static_cast<const __nv_bfloat16*>(v);
  auto* ob = static_cast<__nv_bfloat16*>(o);
  if (d.d == 64)
    return launch_pdl(prefill_window_rows_kernel<64>, grid, dim3(128), 0, st, a, qb, kb, vb, ob);
  if (d.d == 128)
    return launch_pdl(prefill_window_rows_kernel<128>, grid, dim3(128), 0, st, a, qb, kb, vb, ob);
  if (d.d == 256)
    return launch_pdl(prefill_window_rows_kernel<256>, grid, dim3(128), 0, st, a, qb, kb, vb, ob);
  return cudaErrorInvalidValue;
}

}  // namespace jet
