// What the tensor-core attention kernels share (attend_tc.cu over bf16 keys and values,
// attend_kv8.cu over an 8-bit prefix cache): the launch arguments, the work items and
// their schedule, TMA maps and copies, and the combine of a split request's chunks.
#pragma once

#include <cuda.h>
#include <cudaTypedefs.h>

#include <mutex>

#include "attend_items.h"
#include "jet_device.cuh"
#include "jet_internal.h"
#include "sm100_ptx.cuh"

namespace jet {
namespace {

using namespace sm100;

constexpr int kBV = 128;        // query vectors per CTA (MMA M, TMEM lanes)
constexpr int kBN = kItemTile;  // keys per tile
constexpr uint64_t kDrainNs = 200000000ull;
constexpr float kRescaleLog2 = 8.f;  // rescale O only when the max grows by > 2^8

struct AttArgs : ItemPlan {
  const int32_t* prefix_offset;
  const int32_t* row_offset;
  const int32_t* req_order;
  const int32_t* row_cand;
  const int32_t* cand_row_offset;
  const __nv_bfloat16* q;
  __nv_bfloat16* o;  // final output, written directly by single-chunk requests
  float* o_part;
  float2* ml_part;
  int* status;
  int4* items;       // work list (attend_items_kernel)
  int* item_count;
  int* item_next;    // next item to take (dynamic schedule)
  int C, Hq;
  int sorted;        // 1: take items from the longest-first work list; 0: a static deal of
                     // the items in the order of nth_item
  long long n_all;   // upper bound of the items: (request, kv head, block, chunk) slots
  int prefill;       // 1: causal self-attention over the prefixes (rows = prefix positions)
  float scale_log2;  // log2(e) / sqrt(d)
  uint64_t wait_ns;  // budget of one bounded wait (jet_set_wait_budget_ns)
  int hold_first;    // test hook (jet_set_test_stall): withhold the first query block
};

// SW128 K-major position of 16-byte chunk c of row i inside one 64-wide slice
__device__ __forceinline__ uint32_t sw128(int i, int c) {
  return uint32_t(i) * 128u + (uint32_t(c ^ (i & 7)) << 4);
}

__device__ __forceinline__ void fence_proxy_async_smem() {
  asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
}

__device__ __forceinline__ uint32_t pack_bf16(float a, float b) {
  const __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
  return *reinterpret_cast<const uint32_t*>(&h);
}

// 3-D TMA load: box {64 d, 1 head, 64 keys} at (x = d, y = head, z = key)
__device__ __forceinline__ void tma_load_3d(void* dst, const CUtensorMap* map, uint64_t* bar,
                                            int32_t x, int32_t y, int32_t z, uint64_t policy) {
  asm volatile(
      "cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes.L2::cache_hint"
      " [%0], [%1, {%2, %3, %4}], [%5], %6;" ::"r"(smem_u32(dst)),
      "l"(reinterpret_cast<uint64_t>(map)), "r"(x), "r"(y), "r"(z), "r"(smem_u32(bar)),
      "l"(policy)
      : "memory");
}

// 3-D TMA prefetch of the same box into L2 only
__device__ __forceinline__ void tma_prefetch_3d(const CUtensorMap* map, int32_t x, int32_t y,
                                                int32_t z) {
  asm volatile("cp.async.bulk.prefetch.tensor.3d.L2.global.tile [%0, {%1, %2, %3}];" ::"l"(
                   reinterpret_cast<uint64_t>(map)),
               "r"(x), "r"(y), "r"(z)
               : "memory");
}

// Of an item of the work list; *fits: its request is one to work on
__device__ __forceinline__ ItemGeo item_geo(const AttArgs& a, int4 it, bool* fits) {
  *fits = false;
  if (!a.prefill) {
    if (it.x < 0 || it.x >= a.R) return ItemGeo{};
    const int n0 = a.row_offset[it.x], nr = a.row_offset[it.x + 1] - n0;
    const int p0 = a.prefix_offset[it.x], P = a.prefix_offset[it.x + 1] - p0;
    const RequestCut cut = request_cut(a, n0, nr, p0, P);
    *fits = cut.nq > 0;
    return item_geo_at(a, it.x, it.y, it.z, it.w, n0, nr, p0, P, cut);
  }
  // prefill: the rows are the request's prefix positions and a block of
  // them sees the keys up to its last position (per-row causal mask in the
  // softmax); one chunk per item, the output written directly
  ItemGeo e{};
  e.r = it.x;
  e.kh = it.y;
  const int qb = it.z;
  e.split = it.w;
  if (e.r < 0 || e.r >= a.R || e.kh < 0 || e.kh >= a.Hkv) return e;
  e.p0 = a.prefix_offset[e.r];
  e.P = a.prefix_offset[e.r + 1] - e.p0;
  *fits = e.p0 >= 0 && e.P >= 1 && e.P <= a.total_prefix && e.p0 <= a.total_prefix - e.P &&
          e.P <= (long long)a.qgroups * a.rb;
  if (!*fits || e.split != 0) return e;
  e.n0 = e.p0;
  e.nr = e.P;
  e.row0 = qb * a.rb;
  if (e.row0 >= e.nr) return e;
  e.vbase = e.row0 * a.g;
  e.nv = min(a.rb, e.nr - e.row0) * a.g;
  e.splits_r = 1;
  e.k_end = min(e.P, e.row0 + a.rb);
  e.npt = (e.k_end + kBN - 1) / kBN;
  e.ntiles = e.npt;
  e.ok = true;
  return e;
}

// The offsets of the requests a lane stands for: its request in the order, its
// rows [n0, n0 + nr), its prefix [p0, p0 + P) and how it is cut.
struct LaneReq {
  int r, n0, nr, p0, P;
  RequestCut cut;
};

// The requests [base, base + 32) of the order, one a lane.
__device__ __forceinline__ LaneReq lane_req(const AttArgs& a, int base, int lane) {
  LaneReq q{-1, 0, 0, 0, 0, {}};
  const int ri = base + lane;
  if (a.R <= 32) {
    // all offsets beside the order, then one lane from another: one memory
    // latency instead of two before the kernel's first loads
    int p0 = 0, p1 = 0, n0 = 0, n1 = 0;
    if (lane < a.R) {
      q.r = a.req_order[lane];
      p0 = a.prefix_offset[lane];
      p1 = a.prefix_offset[lane + 1];
      n0 = a.row_offset[lane];
      n1 = a.row_offset[lane + 1];
    }
    const bool in = q.r >= 0 && q.r < a.R;
    const int src = in ? q.r : 0;
    q.p0 = __shfl_sync(0xffffffffu, p0, src);
    q.P = __shfl_sync(0xffffffffu, p1 - p0, src);
    q.n0 = __shfl_sync(0xffffffffu, n0, src);
    q.nr = __shfl_sync(0xffffffffu, n1 - n0, src);
    if (!in) q = LaneReq{-1, 0, 0, 0, 0, {}};
  } else if (ri < a.R) {
    const int r = a.req_order[ri];
    if (r >= 0 && r < a.R) {
      q.r = r;
      q.p0 = a.prefix_offset[r];
      q.P = a.prefix_offset[r + 1] - q.p0;
      q.n0 = a.row_offset[r];
      q.nr = a.row_offset[r + 1] - q.n0;
    }
  }
  return q;
}

// The k-th work item of the unsorted order - requests by decreasing prefix
// length (req_order); within a request kv head, query block and chunk, the
// chunk fastest - counting only items that have keys and vectors, and only
// requests that fit the plan (at most n_all items in all, then). One warp
// scans the requests' item counts 32 at a time; false past the last item.
// The geometry comes with it. A CTA asks for growing k, so the scan goes on from
// the window of the last item, `w` (from the first one at every item, 512 requests
// of 1,024 keys took 235 us instead of 197, 300 of 512 90 instead of 75).
struct ItemWindow {
  LaneReq q;   // its requests, when held
  bool held;
  int base, before;  // its first request in the order; the items before it
};
__device__ __forceinline__ bool nth_item(const AttArgs& a, int k, int lane, ItemWindow& w,
                                         int4* out, ItemGeo* geo) {
  LaneReq& q = w.q;
  for (; w.base < a.R; w.base += 32) {
    if (!w.held) {
      q = lane_req(a, w.base, lane);
      if (q.r >= 0) q.cut = request_cut(a, q.n0, q.nr, q.p0, q.P);
      // a request that the layout or the plan does not hold is left out
      if (q.cut.nq == 0 && w.base + lane < a.R) flag(a.status, JET_ERR_DEVICE);
      w.held = true;
    }
    const int before = w.before;
    const int cnt = a.Hkv * q.cut.nq * q.cut.sp;
    int inc = cnt;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int y = __shfl_up_sync(0xffffffffu, inc, o);
      if (lane >= o) inc += y;
    }
    const int total = __shfl_sync(0xffffffffu, inc, 31);
    if (k < before + total) {
      const unsigned hit = __ballot_sync(0xffffffffu, k < before + inc);
      const int src = __ffs(hit) - 1;
      const int kk = k - before - __shfl_sync(0xffffffffu, inc - cnt, src);
      const int r = __shfl_sync(0xffffffffu, q.r, src);
      const RequestCut cut{__shfl_sync(0xffffffffu, q.cut.nq, src),
                           __shfl_sync(0xffffffffu, q.cut.sp, src),
                           __shfl_sync(0xffffffffu, q.cut.per, src)};
      const int nq = cut.nq, sp = cut.sp;
      const int split = kk % sp, rest = kk / sp;
      *out = make_int4(r, rest / nq, rest % nq, split);
      *geo = item_geo_at(a, r, rest / nq, rest % nq, split, __shfl_sync(0xffffffffu, q.n0, src),
                         __shfl_sync(0xffffffffu, q.nr, src), __shfl_sync(0xffffffffu, q.p0, src),
                         __shfl_sync(0xffffffffu, q.P, src), cut);
      return true;
    }
    w.before += total;
    w.held = false;
  }
  return false;
}

// One work item as the scheduler warp publishes it: the item and the geometry
// every role needs (16-byte aligned entries: the ring is read with vector loads).
struct __align__(16) RingItem {
  int4 it;
  ItemGeo e;
};
static_assert(sizeof(RingItem) % 16 == 0, "ring entries keep 16-byte alignment");

PFN_cuTensorMapEncodeTiled_v12000 encode_fn() {
  static PFN_cuTensorMapEncodeTiled_v12000 fn = nullptr;
  static std::once_flag once;
  std::call_once(once, [] {
    void* p = nullptr;
    cudaDriverEntryPointQueryResult q;
    if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &p, 12000, cudaEnableDefault,
                                         &q) == cudaSuccess &&
        q == cudaDriverEntryPointSuccess)
      fn = reinterpret_cast<PFN_cuTensorMapEncodeTiled_v12000>(p);
  });
  return fn;
}

// packed [keys, Hkv, DH] bf16 K or V: box of 64 d x 1 head x 64 keys
// packed [rows, heads, DH] bf16: box of 64 d x box_heads heads x box_rows rows
bool encode_3d(CUtensorMap* map, const void* base, int rows, int heads, int DH, int box_heads,
               int box_rows) {
  auto fn = encode_fn();
  if (!fn) return false;
  const cuuint64_t dims[3] = {cuuint64_t(DH), cuuint64_t(heads), cuuint64_t(rows)};
  const cuuint64_t strides[2] = {cuuint64_t(DH) * 2, cuuint64_t(heads) * DH * 2};
  const cuuint32_t box[3] = {64, cuuint32_t(box_heads), cuuint32_t(box_rows)};
  const cuuint32_t estr[3] = {1, 1, 1};
  return fn(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<void*>(base), dims, strides, box,
            estr, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
            CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// One warp per (row, query head) of a request whose prefix spans several
// chunks: combine the chunks' base-2 partials (the last chunk also holds the
// candidate's own keys) and normalise. Single-chunk requests were written by
// the attention kernel itself; it also left every chunk's (m, l) in place, empty
// for the chunks a request does not have, so that nothing here waits for the
// layout. `ahead`: the partials are read beside their (m, l), wanted or not.
template <int DH>
__global__ void __launch_bounds__(128)
attend_combine_kernel(const int32_t* __restrict__ row_req, int N, int R, int Hq, int splits,
                      bool ahead, const float* __restrict__ o_part,
                      const float2* __restrict__ ml_part, __nv_bfloat16* __restrict__ o,
                      int* status) {
  pdl_begin();
  const int lane = threadIdx.x & 31;
  const long long idx = (long long)blockIdx.x * (blockDim.x >> 5) + (threadIdx.x >> 5);
  if (idx >= (long long)N * Hq) return;
  const int n = int(idx / Hq), h = int(idx % Hq);
  const int r = row_req[n];
  // written by the attention kernel itself (l = -1 in the first chunk's place)
  const bool direct = ml_part[size_t(n) * Hq + h].y < 0.f;
  if (!ahead && direct) return;
  constexpr int PER = DH / 32;
  float acc[PER];
  float m, l;
  combine_chunks<DH>(ahead, splits, N, Hq, n, h, lane, ml_part, o_part, m, l, acc);
  if (r < 0 || r >= R) {
    if (lane == 0) flag(status, JET_ERR_DEVICE);
    return;
  }
  if (direct) return;
  const float inv = l > 0.f ? 1.f / l : 0.f;
#pragma unroll
  for (int i = 0; i < PER; ++i)
    o[(size_t(n) * Hq + h) * DH + lane + 32 * i] = __float2bfloat16_rn(acc[i] * inv);
}

}  // namespace
}  // namespace jet
