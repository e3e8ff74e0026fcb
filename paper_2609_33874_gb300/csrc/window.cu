// Attention of the step under a window with first tokens that stay visible, float32: one
// warp a query vector, key by key.
#include <algorithm>

#include "attend_items.h"
#include "jet_device.cuh"
#include "jet_internal.h"
#include "window_rows.cuh"

namespace jet {
namespace {

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
  const size_t step = size_t(a.Hkv) * DH, pre = size_t(p0) * step + size_t(kh) * DH;
  const size_t own = t > 0 ? size_t(f0 + 1) * step + size_t(kh) * DH : 0;
  row_attend<DH, T>(a.w, q + size_t(idx) * DH, k_pre + pre, v_pre + pre, k_cand + own, v_cand + own,
                    step, p1 - p0, t, o + size_t(idx) * DH, lane);
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

size_t attend_window_bytes(const jet_sizes& n, const jet_dims& d, int window, int sinks) {
  if (d.dtype != JET_DTYPE_BF16) return 16;
  return std::max<size_t>(16, attend_window_plan(n, d, window, sinks).bytes);
}

cudaError_t launch_attend_window(const jet_layout& lay, const jet_dims& d, int window, int sinks,
                                 const void* q, const void* k_pre, const void* v_pre,
                                 const void* k_cand, const void* v_cand, void* o, void* ws,
                                 int* status, cudaStream_t st) {
  if (d.dtype == JET_DTYPE_BF16)
    return launch_attend_window_tc(lay, d, window, sinks, q, k_pre, v_pre, k_cand, v_cand, o, ws,
                                   status, st);
  const RowArgs a = row_args(lay, d, window, sinks, status);
  if (d.d == 64) return launch_rows<64, float>(a, q, k_pre, v_pre, k_cand, v_cand, o, st);
  if (d.d == 128) return launch_rows<128, float>(a, q, k_pre, v_pre, k_cand, v_cand, o, st);
  if (d.d == 256) return launch_rows<256, float>(a, q, k_pre, v_pre, k_cand, v_cand, o, st);
  return cudaErrorInvalidValue;
}

}  // namespace jet
