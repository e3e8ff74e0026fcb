// The prefill under a window: causal self-attention in which a position sees its last
// `window` positions and the first `sinks`, on pairs of SMs with the 5th-generation tensor
// cores; bf16, head dimensions 64, 128 and 256.
//
// An item is (request, kv head, block of 2 rb positions), rb = 128 / g whole positions of
// g = Hq / Hkv heads per SM; its keys, the first ones and the run that ends with the block,
// are slots laid end to end (window.h), 128 a tile. Two SMs share a tile (tcgen05
// cta_group::2, M = 256): each holds its own 128 query vectors and half of every tile, 64
// keys of K and half of the columns of V. Roles of each CTA:
//   warp 0        TMA producer: query blocks, K and V halves in rings
//   warp 1        TMEM allocation; in the even CTA the MMA issuer:
//                   S_j  = Q K_j^T  (256 vectors x 128 keys)
//                   O   += P_j V_j  (256 vectors x d)
//                 P_j (bf16) takes the place of half of S_j. The issuing thread's MMAs run
//                 in order, so a new S overwrites a P after its PV.
//   warp 2        schedule: which items this pair runs, up to kRing ahead
//   warps 3..10   softmax: a query vector is a TMEM lane, and two warps share each lane, 32 of
//                 every 64 of the tile's columns each: they tell each other their maximum
//   warps 11..14  output: O / l to memory
// and after the last item all of them: outputs that came out NaN or infinite (window_rows.cuh).
// Items are short under a narrow window (two tiles for 16/2 heads under 128; 33 for 32/8 under
// 4,096), so what counts is that they overlap: at d
// 64 and 128 there are two query blocks in shared memory and two O in TMEM, and an item's
// products begin while the last one's output is read. All barriers an MMA waits for live in
// the even CTA; the commits reach both.
#include <algorithm>
#include <type_traits>

#include "attend_tc.cuh"
#include "window_rows.cuh"

namespace jet {
namespace {

constexpr int kKeys = 128;          // keys per tile of the pair
constexpr int kHalfKeys = kKeys / 2;
constexpr int kSoftWarps = 8, kOutWarps = 4;
constexpr int kFirstSoft = 3, kFirstOut = kFirstSoft + kSoftWarps;
constexpr int kWinThreads = 32 * (kFirstOut + kOutWarps);

// Item as the schedule warp publishes it (ntiles 0: no more items).
struct __align__(16) WinItem {
  int p0;      // the request's first position in the packed prefixes
  int kh;      // key/value head
  int row0;    // this CTA's first position within the request
  int nv;      // this CTA's query vectors (may be 0 in the odd CTA)
  int slots, pad, off;  // Slots of the block
  int ntiles;
};
static_assert(sizeof(WinItem) == 32, "");

template <int DH>
struct WinGeo {
  static constexpr int kStages = DH == 64 ? 6 : DH == 128 ? 4 : 2;  // of K and of V
  static constexpr int kQBufs = DH == 256 ? 1 : 2;
  // TMEM holds 512 columns: a third S tile lets QK^T run on while a tile's softmax lasts
  // (d 128, 16,000 positions under 4,096: 727 us with two S and two O, 715 with three S)
  static constexpr int kSBufs = DH == 256 ? 2 : 3;
  static constexpr int kOBufs = DH == 64 ? 2 : 1;
  // Items the roles may be apart. Their query blocks are on the way into L2, so more of them than
  // it takes to hide that displace others before their use (d 256: two of 64 KB a CTA; with
  // eight a third of the queries were read twice, 16 requests under 256 85.5 us instead of 77.3)
  static constexpr int kRing = DH == 64 ? 4 : 2;
  static constexpr int kSlices = DH / 64;                  // 64-wide d slices of Q and K
  static constexpr int kVCols = DH / 2;                    // this CTA's columns of V
  static constexpr int kVWide = kVCols < 64 ? kVCols : 64;  // of a swizzled row of V
  static constexpr int kVSlices = kVCols / kVWide;
  static constexpr uint32_t kQBytes = kBV * DH * 2;
  static constexpr uint32_t kKBytes = kHalfKeys * DH * 2;
  static constexpr uint32_t kVBytes = kKeys * kVCols * 2;
  static constexpr uint32_t kOffK = kQBufs * kQBytes;
  static constexpr uint32_t kOffV = kOffK + kStages * kKBytes;
  static constexpr uint32_t kOffStage = kOffV + kStages * kVBytes;  // 4 KB per output warp
  static constexpr uint32_t kOffL = kOffStage + kOutWarps * 4096;  // l of two items, halves
  static constexpr uint32_t kOffMax = kOffL + 2 * 2 * kBV * 4;     // maxima, two tiles, halves
  static constexpr uint32_t kOffBar = kOffMax + 2 * 2 * kBV * 4;
  static constexpr uint32_t kOffOdd = kOffBar + 1024 - sizeof(OddItems);
  static constexpr uint32_t kBytes = kOffBar + 1024;
  // TMEM: the S tiles, then O
  static constexpr uint32_t kOCol = kSBufs * kKeys;
  static constexpr uint32_t kTmemCols = 512;
  static_assert(kOCol + kOBufs * DH <= kTmemCols, "");
};
static_assert(WinGeo<256>::kBytes + 1024 <= 232448, "shared memory of one CTA");
static_assert(WinGeo<128>::kBytes + 1024 <= 232448, "shared memory of one CTA");

struct WinPreArgs {
  const int32_t* prefix_offset;
  const int32_t* req_order;
  const __nv_bfloat16 *q, *k, *v;
  __nv_bfloat16* o;
  int* status;
  Window win;
  int R, total, Hq, Hkv, g, rb;
  float scale_log2;  // log2(e) / sqrt(d)
  uint64_t wait_ns;  // budget of one bounded wait (jet_set_wait_budget_ns)
  int hold_first;    // test hook (jet_set_test_stall): withhold the first query block
};

// 3-D tiled load into this CTA's shared memory, counted on the even CTA's
// barrier (a mapa address)
__device__ __forceinline__ void tma_load_3d_pair(void* dst, const CUtensorMap* map, uint32_t bar,
                                                 int32_t x, int32_t y, int32_t z,
                                                 uint64_t policy) {
  asm volatile(
      "cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes.cta_group::2"
      ".L2::cache_hint [%0], [%1, {%2, %3, %4}], [%5], %6;" ::"r"(smem_u32(dst)),
      "l"(reinterpret_cast<uint64_t>(map)), "r"(x), "r"(y), "r"(z), "r"(bar), "l"(policy)
      : "memory");
}

// KEYS slots from slot0 on into a tile (SLICES slices of WIDE columns from x0): one box a
// slice, or kSlotBox keys at a time where first keys and window meet
template <int KEYS, int SLICES, int WIDE>
__device__ __forceinline__ void load_slots(uint8_t* dst, const CUtensorMap* map,
                                           const CUtensorMap* map16, uint32_t bar,
                                           const WinItem& e, int slot0, int x0, uint64_t pol) {
  if (slot0 < e.pad && slot0 + KEYS > e.pad) {
#pragma unroll 1
    for (int b = 0; b < KEYS / kSlotBox; ++b) {
      const int slot = slot0 + b * kSlotBox;
      const int key = e.p0 + (slot < e.pad ? slot : slot + e.off);
#pragma unroll
      for (int i = 0; i < SLICES; ++i)
        tma_load_3d_pair(dst + (i * KEYS + b * kSlotBox) * (WIDE * 2), map16, bar, x0 + i * WIDE,
                         e.kh, key, pol);
    }
  } else {
    const int key = e.p0 + slot0 + (slot0 < e.pad ? 0 : e.off);
#pragma unroll
    for (int i = 0; i < SLICES; ++i)
      tma_load_3d_pair(dst + i * KEYS * (WIDE * 2), map, bar, x0 + i * WIDE, e.kh, key, pol);
  }
}

// descriptor of an MN-major operand tile of rows of 32 elements written by TMA with 64-byte
// swizzling: 8-row groups along K 512 bytes apart
__device__ __forceinline__ uint64_t desc_mn_sw64(uint32_t addr) {
  uint64_t d = 0;
  d |= uint64_t((addr >> 4) & 0x3FFFu);
  d |= uint64_t(1) << 16;                // one slice only
  d |= uint64_t(512 >> 4) << 32;
  d |= uint64_t(1) << 46;
  d |= uint64_t(4) << 61;                // layout: 64-byte swizzle
  return d;
}

__device__ __forceinline__ void tmem_st_16cols_u32(uint32_t taddr, const uint32_t (&v)[16]) {
  float f[16];
#pragma unroll
  for (int i = 0; i < 16; ++i) f[i] = __uint_as_float(v[i]);
  tmem_st_16cols(taddr, f);
}

__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c) {
  float2 d;
  asm("{\n\t.reg .b64 a, b, c, d;\n\t"
      "mov.b64 a, {%2, %3};\n\tmov.b64 b, {%4, %5};\n\tmov.b64 c, {%6, %7};\n\t"
      "fma.rn.f32x2 d, a, b, c;\n\tmov.b64 {%0, %1}, d;\n\t}"
      : "=f"(d.x), "=f"(d.y)
      : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y), "f"(c.x), "f"(c.y));
  return d;
}

__device__ __forceinline__ float2 add2(float2 a, float2 b) {
  float2 d;
  asm("{\n\t.reg .b64 a, b, d;\n\t"
      "mov.b64 a, {%2, %3};\n\tmov.b64 b, {%4, %5};\n\t"
      "add.rn.f32x2 d, a, b;\n\tmov.b64 {%0, %1}, d;\n\t}"
      : "=f"(d.x), "=f"(d.y)
      : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
  return d;
}

__device__ __forceinline__ float max3(float a, float b, float c) {
  float d;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
  return d;
}

// bits [lo, hi) of a word, of what lies in it
__device__ __forceinline__ uint32_t bit_span(int lo, int hi) {
  uint32_t m;
  const int at = max(lo, 0);
  asm("bmsk.clamp.b32 %0, %1, %2;" : "=r"(m) : "r"(at), "r"(max(hi - at, 0)));
  return m;
}

// a place in a ring of N barriers, and the parity of its phase
template <int N>
struct Ring {
  uint32_t at = 0, phase = 0;
  __device__ __forceinline__ void next() {
    if (++at == N) {
      at = 0;
      phase ^= 1u;
    }
  }
};

// arrive at a named barrier without waiting for it
__device__ __forceinline__ void named_bar_arrive(uint32_t id, uint32_t threads) {
  asm volatile("bar.arrive %0, %1;" ::"r"(id), "r"(threads) : "memory");
}

// wait for this thread's TMEM loads, v's values among them (named, so that no use of them is
// moved before the wait)
__device__ __forceinline__ void tmem_wait_ld_of(float (&v)[32]) {
  asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
#pragma unroll
  for (int i = 0; i < 32; ++i) asm volatile("" : "+f"(v[i]));
}
__device__ __forceinline__ void tmem_wait_ld_of(float (&v)[32], float (&w)[32]) {
  tmem_wait_ld_of(v);
#pragma unroll
  for (int i = 0; i < 32; ++i) asm volatile("" : "+f"(w[i]));
}

// what position p of an item's request sees, as slots: [0, first) and [lo, end)
struct RowBounds {
  int first, lo, end;
};
__device__ __forceinline__ RowBounds row_bounds(const Window& w, const WinItem& e, int p) {
  const Seen32 s = seen_at32(w, p);
  return RowBounds{s.first, s.lo - e.off, min(e.slots, p + 1 - e.off)};
}

// A pair's items, one after the other. Requests by decreasing length, a request's blocks from
// the last to the first, kv heads fastest, so that the pairs at work share one request's K and V
// in L2; the pairs deal them out back and forth (0 .. n-1, n-1 .. 0, ...), without a work list or
// a counter. Both CTAs derive the same items.
struct WinSchedule {
  long long before = 0;  // items of the requests before this window of 32
  int base = 0, total = -1, cnt = 0, inc = 0, r = 0, P = 0, first = 0;  // total -1: not counted
};

// The deal's item number `round`, of growing numbers. One warp; ntiles 0: no more items.
__device__ __forceinline__ WinItem next_item(const WinPreArgs& a, WinSchedule& s, int round,
                                             int pair, int npairs, int rank, int lane) {
  const int g = a.g, rb = a.rb;
  const long long k = (long long)round * npairs + ((round & 1) ? npairs - 1 - pair : pair);
  WinItem it{};
  for (;;) {
    if (s.total < 0) {  // the window's block counts
      const int ri = s.base + lane;
      s.cnt = s.r = s.P = s.first = 0;
      if (ri < a.R) {
        s.r = a.req_order[ri];
        if (s.r >= 0 && s.r < a.R) {
          s.first = a.prefix_offset[s.r];
          const int end = a.prefix_offset[s.r + 1];
          if (span_inside(s.first, end, a.total) && end > s.first) {
            s.P = end - s.first;
          } else {
            flag(a.status, JET_ERR_DEVICE);
          }
        } else {
          flag(a.status, JET_ERR_DEVICE);
        }
        s.cnt = a.Hkv * ((s.P + 2 * rb - 1) / (2 * rb));
      }
      s.inc = s.cnt;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const int y = __shfl_up_sync(0xffffffffu, s.inc, o);
        if (lane >= o) s.inc += y;
      }
      s.total = __shfl_sync(0xffffffffu, s.inc, 31);
    }
    if (k < s.before + s.total) {
      const unsigned hit = __ballot_sync(0xffffffffu, k < s.before + s.inc);
      const int src = __ffs(hit) - 1;
      const int kk = int(k - s.before) - __shfl_sync(0xffffffffu, s.inc - s.cnt, src);
      const int PP = __shfl_sync(0xffffffffu, s.P, src);
      const int nq = __shfl_sync(0xffffffffu, s.cnt, src) / a.Hkv;
      const int qb = nq - 1 - kk / a.Hkv;
      const Slots sl = block_slots(a.win, 2 * qb * rb, min(PP, (qb + 1) * 2 * rb));
      it.p0 = __shfl_sync(0xffffffffu, s.first, src);
      it.kh = kk % a.Hkv;
      it.row0 = (2 * qb + rank) * rb;
      it.nv = min(rb, max(0, PP - it.row0)) * g;
      it.slots = sl.n;
      it.pad = sl.pad;
      it.off = sl.off;
      it.ntiles = (sl.n + kKeys - 1) / kKeys;
      break;
    }
    s.before += s.total;
    s.base += 32;
    if (s.base >= a.R) break;  // no more items
    s.total = -1;
  }
  return it;
}

// a position's query vector, key by key
template <int DH>
__device__ __noinline__ void again(const WinPreArgs& a, const WinItem& e, int gi, int lane) {
  const int p = e.row0 + gi / a.g;
  const size_t at = (size_t(e.p0 + p) * a.Hq + e.kh * a.g + gi % a.g) * DH;
  const size_t step = size_t(a.Hkv) * DH, pre = size_t(e.p0) * step + size_t(e.kh) * DH;
  position_attend<DH>(a.win, a.q + at, a.k + pre, a.v + pre, step, p, a.o + at, lane);
}

// The outputs of this CTA's noted items that came out NaN or infinite, a warp each.
template <int DH>
__device__ __noinline__ void odd_outputs(const WinPreArgs& a, const OddItems& odd, int rank,
                                         int warp, int lane) {
  WinSchedule order{};
  for (int u = 0;; ++u) {
    const WinItem e =
        next_item(a, order, u, int(blockIdx.x >> 1), int(gridDim.x >> 1), rank, lane);
    if (e.ntiles == 0) break;
    if (!odd.has(u)) continue;
    const __nv_bfloat16* out = a.o + (size_t(e.p0 + e.row0) * a.Hq + size_t(e.kh) * a.g) * DH;
    for (int gi = warp; gi < e.nv; gi += kWinThreads / 32)
      if (stored_odd<DH>(out + size_t(gi / a.g * a.Hq + gi % a.g) * DH, lane))
        again<DH>(a, e, gi, lane);
  }
}

// (a call: inlined, the output warps' code cost d 64 and 128 0.4 %)
__device__ __noinline__ void note_odd(OddItems* odd, int u) { odd->note(u); }

template <int DH, bool SKIP>
__global__ void __launch_bounds__(kWinThreads, 1)
prefill_window_kernel(const __grid_constant__ CUtensorMap tmQ,
                      const __grid_constant__ CUtensorMap tmK,
                      const __grid_constant__ CUtensorMap tmV,
                      const __grid_constant__ CUtensorMap tmK16,
                      const __grid_constant__ CUtensorMap tmV16,
                      const __grid_constant__ WinPreArgs a) {
  using G = WinGeo<DH>;
  constexpr int kStages = G::kStages, kQBufs = G::kQBufs, kSBufs = G::kSBufs, kOBufs = G::kOBufs;
  constexpr int kRing = G::kRing;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) &
                                             ~uintptr_t(1023));
  float* lsum = reinterpret_cast<float*>(smem + G::kOffL);       // [2 items][2 halves][kBV]
  float* maxima = reinterpret_cast<float*>(smem + G::kOffMax);   // [2 tiles][2 halves][kBV]
  WinItem* ring = reinterpret_cast<WinItem*>(smem + G::kOffBar);
  uint64_t* k_full = reinterpret_cast<uint64_t*>(ring + kRing);  // even CTA
  uint64_t* k_empty = k_full + kStages;
  uint64_t* v_full = k_empty + kStages;                          // even CTA
  uint64_t* v_empty = v_full + kStages;
  uint64_t* s_full = v_empty + kStages;                          // [kSBufs]
  uint64_t* p_full = s_full + kSBufs;                            // [kSBufs], even CTA
  uint64_t* item_full = p_full + kSBufs;                         // [kRing]
  uint64_t* item_empty = item_full + kRing;                      // [kRing]
  uint64_t* q_full = item_empty + kRing;                         // [kQBufs], even CTA
  uint64_t* q_free = q_full + kQBufs;   // [kQBufs]: the item's last QK^T is done
  uint64_t* o_full = q_free + kQBufs;   // [kOBufs]: the item's last PV is done
  uint64_t* o_free = o_full + kOBufs;   // [kOBufs]: O has been read out (even CTA)
  uint64_t* l_full = o_free + kOBufs;   // [2]: the item's sums are in lsum
  uint64_t* l_free = l_full + 2;        // [2]: and have been read
  uint64_t* drain = l_free + 2;
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(drain + 1);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
  // (by its offset at each use: an address held all along cost d 128 and 64 up to 3 %)
  auto odd_items = [&] { return reinterpret_cast<OddItems*>(smem + G::kOffOdd); };

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t rank = cluster_rank();
  const int pair = int(blockIdx.x >> 1), npairs = int(gridDim.x >> 1);
  const int g = a.g, rb = a.rb;
  if (threadIdx.x == 0) {
    for (int s = 0; s < kStages; ++s) {
      mbar_init(k_full + s, 1);
      mbar_init(k_empty + s, 1);
      mbar_init(v_full + s, 1);
      mbar_init(v_empty + s, 1);
    }
    for (int b = 0; b < kSBufs; ++b) {
      mbar_init(s_full + b, 1);
      mbar_init(p_full + b, 2 * kSoftWarps);  // both CTAs' softmax warps
    }
    for (int b = 0; b < 2; ++b) {
      mbar_init(l_full + b, kSoftWarps);
      mbar_init(l_free + b, kOutWarps);
    }
    // producer, softmax and output warps, and the even CTA's MMA thread
    for (int b = 0; b < kRing; ++b) {
      mbar_init(item_full + b, 1);
      mbar_init(item_empty + b, 1 + kSoftWarps + kOutWarps + (rank == 0 ? 1 : 0));
    }
    for (int b = 0; b < kQBufs; ++b) {
      mbar_init(q_full + b, 1);
      mbar_init(q_free + b, 1);
    }
    for (int b = 0; b < kOBufs; ++b) {
      mbar_init(o_full + b, 1);
      mbar_init(o_free + b, 2 * kOutWarps);  // both CTAs' output warps
    }
    mbar_init(drain, 1);
    *abort_flag = 0;
    fence_barrier_init();
  }
  if (warp == 1) odd_items()->bits[lane] = 0;
  if (warp == 0 && lane == 0) {
    tma_prefetch_desc(&tmQ);
    tma_prefetch_desc(&tmK);
    tma_prefetch_desc(&tmV);
    tma_prefetch_desc(&tmK16);
    tma_prefetch_desc(&tmV16);
  }
  // the query blocks arrive by TMA (rows [0, rb g)); zero the rows past them
  // once so that no stale shared memory enters the MMA
  for (int b = 0; b < kQBufs; ++b)
    for (int e = int(threadIdx.x); e < (kBV - rb * g) * (DH / 8); e += kWinThreads) {
      const int i = rb * g + e / (DH / 8), c = e % (DH / 8);
      *reinterpret_cast<uint4*>(smem + b * G::kQBytes + (c >> 3) * (kBV * 128) +
                                sw128(i, c & 7)) = make_uint4(0, 0, 0, 0);
    }
  fence_proxy_async_shared();
  // global memory and TMEM only after the previous kernel of the stream is done
  pdl_begin();
  if (warp == 1) {
    tmem_alloc_pair(tmem_slot, G::kTmemCols);
    tmem_relinquish_pair();
  }
  tc_fence_before();
  __syncthreads();
  cluster_sync();  // the even CTA's barriers and both query tails are ready
  tc_fence_after();
  const uint32_t tmem = *tmem_slot;

  if (warp == 2) {
    // ---------------------------------------------------------------- schedule
    WinSchedule order{};
    for (int u = 0;; ++u) {
      const WinItem it = next_item(a, order, u, pair, npairs, int(rank), lane);
      const int slot = u % kRing;
      bool okw = true;
      if (lane == 0)
        okw = mbar_wait(item_empty + slot, ((u / kRing) & 1) ^ 1u, a.wait_ns, abort_flag);
      if (!__shfl_sync(0xffffffffu, okw ? 1 : 0, 0)) {
        if (lane == 0) {
          *abort_flag = 1;
          flag(a.status, JET_ERR_TIMEOUT);
        }
        break;
      }
      if (lane == 0) {
        ring[slot] = it;
        mbar_arrive(item_full + slot);
        if (it.nv > 0) {  // start the query block on its way into L2
#pragma unroll
          for (int sl = 0; sl < G::kSlices; ++sl)
            tma_prefetch_3d(&tmQ, sl * 64, it.kh * g, it.p0 + it.row0);
        }
      }
      if (it.ntiles == 0) break;
    }
  } else if (warp == 0) {
    // ---------------------------------------------------------------- producer
    if (elect_one()) {
      // queries are read once, but are asked for before they are read: as what leaves L2 first they
      // may leave it again (256 requests of 10 - 300 under 64, d 256: 201 us, 186 as the rest)
      const uint64_t pol = policy_evict_normal();
      const uint32_t bar_q = mapa_shared(q_full, 0), bar_k = mapa_shared(k_full, 0),
                     bar_v = mapa_shared(v_full, 0);
      uint32_t k_issued = 0, k_par = 0, v_issued = 0, v_par = 0, q_issued = 0, q_par = 0;
      int T = 0;  // tiles so far
      bool ok = true;
      for (int u = 0; ok; ++u) {
        const int slot = u % kRing;
        if (!mbar_wait(item_full + slot, (u / kRing) & 1, a.wait_ns, abort_flag)) {
          ok = false;
          break;
        }
        const WinItem e = ring[slot];
        mbar_arrive(item_empty + slot);
        if (e.ntiles == 0) break;
        int jq = 0, jk = 0, jv = 0;  // issued: the query block, K and V tiles
        IdleClock clk;
        while (jq == 0 || jv < e.ntiles) {
          bool progressed = false;
          // the query block, once the last QK^T of the item that had its buffer is done
          const int qs = u % kQBufs;
          if (jq == 0 && (u < kQBufs || mbar_test(q_free + qs, ((u / kQBufs) - 1) & 1))) {
            if (u == 0 && a.hold_first) {
              // test hook: the first query block never lands
            } else {
              if (rank == 0)
                mbar_arrive_expect_tx(q_full + qs, 2u * G::kSlices * 64 * 2 * g * rb);
#pragma unroll
              for (int sl = 0; sl < G::kSlices; ++sl)
                tma_load_3d_pair(smem + qs * G::kQBytes + sl * (kBV * 128), &tmQ, bar_q + 8 * qs,
                                 sl * 64, e.kh * g, e.p0 + e.row0, pol);
              q_issued |= 1u << qs;
              q_par = (q_par & ~(1u << qs)) | (((u / kQBufs) & 1) << qs);
            }
            jq = 1;
            progressed = true;
          }
          if (jk < e.ntiles) {
            const int s = (T + jk) % kStages;
            const uint32_t ph = ((T + jk) / kStages) & 1;
            if (mbar_test(k_empty + s, ph ^ 1u)) {
              if (rank == 0) mbar_arrive_expect_tx(k_full + s, 2 * G::kKBytes);
              load_slots<kHalfKeys, G::kSlices, 64>(smem + G::kOffK + s * G::kKBytes, &tmK, &tmK16,
                                                    bar_k + 8 * s, e,
                                                    jk * kKeys + int(rank) * kHalfKeys, 0, pol);
              k_issued |= 1u << s;
              k_par = (k_par & ~(1u << s)) | (ph << s);
              ++jk;
              progressed = true;
            }
          }
          if (jv < jk) {
            const int s = (T + jv) % kStages;
            const uint32_t ph = ((T + jv) / kStages) & 1;
            if (mbar_test(v_empty + s, ph ^ 1u)) {
              if (rank == 0) mbar_arrive_expect_tx(v_full + s, 2 * G::kVBytes);
              load_slots<kKeys, G::kVSlices, G::kVWide>(smem + G::kOffV + s * G::kVBytes, &tmV,
                                                        &tmV16, bar_v + 8 * s, e, jv * kKeys,
                                                        int(rank) * G::kVCols, pol);
              v_issued |= 1u << s;
              v_par = (v_par & ~(1u << s)) | (ph << s);
              ++jv;
              progressed = true;
            }
          }
          if (clk.expired(progressed, abort_flag, a.wait_ns)) {
            ok = false;
            break;
          }
        }
        T += e.ntiles;
      }
      if (!ok) {
        *abort_flag = 1;
        flag(a.status, JET_ERR_TIMEOUT);
        // let the copies in flight land: the even CTA's barriers count both
        // CTAs' bytes; the odd CTA waits out a fixed bounded time
        if (rank == 0) {
          for (int t = 0; t < kQBufs; ++t)
            if (q_issued & (1u << t)) mbar_wait(q_full + t, (q_par >> t) & 1u, kDrainNs, nullptr);
          for (int t = 0; t < kStages; ++t) {
            if (k_issued & (1u << t)) mbar_wait(k_full + t, (k_par >> t) & 1u, kDrainNs, nullptr);
            if (v_issued & (1u << t)) mbar_wait(v_full + t, (v_par >> t) & 1u, kDrainNs, nullptr);
          }
        } else if (q_issued | k_issued | v_issued) {
          const uint64_t t0 = global_timer_ns();
          while (global_timer_ns() - t0 < kDrainNs / 16) {
          }
        }
      }
    }
  } else if (warp == 1) {
    // ---------------------------------------------------------------- MMA issuer
    if (rank == 0 && elect_one()) {
      const uint32_t id_s = idesc_bf16_f32(2 * kBV, kKeys);
      const uint32_t id_o = idesc_bf16_f32(2 * kBV, DH) | (1u << 16);  // B (V) is MN-major
      // QK^T runs at most kSBufs tiles ahead of PV, across items. Short tiles leave this
      // thread few hundred cycles each, beside softmax warps that issue all the time: places in
      // the rings are counted, not divided for .
      Ring<kStages> k, v;               // tiles of K and of V
      Ring<kSBufs> sq, sp;              // S tiles of QK^T, of PV
      Ring<kRing> iq, ip;               // items of each
      Ring<kQBufs> qq;                  // query blocks
      Ring<kOBufs> op;                  // outputs
      int ahead = 0, jq = 0, jp = 0;    // tiles between the two, tiles of their items so far
      int nq = 0, np = 0, kend = 0;     // tiles of their items; slots of PV's
      int begun = 0;                    // items that PV has begun, up to kOBufs
      bool more = true, ok = true;
      const uint64_t dq0 = desc_k_sw128(smem_u32(smem));
      const uint64_t dk0 = desc_k_sw128(smem_u32(smem + G::kOffK));
      const uint32_t vs0 = smem_u32(smem + G::kOffV);
      const uint64_t dv0 = DH == 64 ? desc_mn_sw64(vs0) : desc_mn_sw128(vs0, kKeys * 128);
      IdleClock clk;
      while (ok && (more || ahead > 0)) {
        bool progressed = false;
        if (ahead > 0 && mbar_test(p_full + sp.at, sp.phase)) {
          if (np == 0) {
            np = ring[ip.at].ntiles;
            kend = ring[ip.at].slots;
          }
          // the item's first PV overwrites its O: the item that had it must be out
          if (mbar_test(v_full + v.at, v.phase) &&
              (jp > 0 || begun < kOBufs || mbar_test(o_free + op.at, op.phase ^ 1u))) {
            tc_fence_after();
            const uint32_t pt = tmem + sp.at * kKeys;  // P_j over the first columns of S_j
            const uint32_t ot = tmem + G::kOCol + op.at * DH;
            const uint64_t dv = dv0 + (v.at * G::kVBytes >> 4);
            // the keys past the block's last are not read (16 per instruction)
            const int steps = min(kKeys, kend - jp * kKeys + 15) >> 4;
#pragma unroll 1
            for (int x = 0; x < steps; ++x)
              mma_f16_ta_pair(ot, pt + uint32_t(8 * x), dv + (x * 16 * G::kVWide * 2 >> 4), id_o,
                              (jp | x) != 0);
            mma_commit_pair(v_empty + v.at, 0x3);
            --ahead;
            v.next();
            sp.next();
            if (++jp == np) {
              mma_commit_pair(o_full + op.at, 0x3);
              mbar_arrive(item_empty + ip.at);
              op.next();
              ip.next();
              if (begun < kOBufs) ++begun;
              jp = np = 0;
            }
            progressed = true;
          }
        }
        if (more && ahead < kSBufs) {
          if (nq == 0 && mbar_test(item_full + iq.at, iq.phase)) {
            nq = ring[iq.at].ntiles;
            if (nq == 0) more = false;
          }
          if (nq > 0 && (jq > 0 || mbar_test(q_full + qq.at, qq.phase)) &&
              mbar_test(k_full + k.at, k.phase)) {
            tc_fence_after();
            const uint64_t dq = dq0 + (qq.at * G::kQBytes >> 4);
            const uint64_t dk = dk0 + (k.at * G::kKBytes >> 4);
#pragma unroll
            for (int st = 0; st < DH / 16; ++st) {
              const int sl = st >> 2, x = st & 3;
              mma_f16_pair(tmem + sq.at * kKeys, dq + (sl * (kBV * 128) >> 4) + 2 * x,
                           dk + (sl * (kHalfKeys * 128) >> 4) + 2 * x, id_s, st != 0);
            }
            mma_commit_pair(s_full + sq.at, 0x3);
            mma_commit_pair(k_empty + k.at, 0x3);
            ++ahead;
            k.next();
            sq.next();
            if (++jq == nq) {
              mma_commit_pair(q_free + qq.at, 0x3);  // the query blocks may be replaced
              qq.next();
              iq.next();
              jq = nq = 0;
            }
            progressed = true;
          }
        }
        if (clk.expired(progressed, abort_flag, a.wait_ns)) ok = false;
      }
      if (!ok) {
        *abort_flag = 1;
        flag(a.status, JET_ERR_TIMEOUT);
        mma_commit_pair(drain, 0x1);
        mbar_wait(drain, 0, kDrainNs, nullptr);
      }
    }
  } else if (warp < kFirstOut) {
    // ---------------------------------------------------------------- softmax
    const int q4 = warp & 3, half = (warp - kFirstSoft) >> 2;
    const int i = q4 * 32 + lane;  // query vector within the block = TMEM lane
    const uint32_t lane_off = uint32_t(q4 * 32) << 16;
    const uint32_t p_full_even = mapa_shared(p_full, 0);
    // positions of this vector, and of the warp's first and last, in the block
    const int at = i / g, at0 = q4 * 32 / g, at1 = (q4 * 32 + 31) / g;
    bool ok = true;
    Ring<kSBufs> sr;    // S tiles
    Ring<kStages> vr;   // the V tile of the tile before, of which O was last added to
    vr.at = kStages - 1;
    vr.phase = 1;
    int T = 0;
    for (int u = 0; ok; ++u) {
      const int slot = u % kRing, ob = u % kOBufs, ls = u & 1;
      if (!warp_mbar_wait(item_full + slot, (u / kRing) & 1, a.wait_ns, abort_flag)) {
        ok = false;
        break;
      }
      const WinItem e = ring[slot];
      __syncwarp();
      if (lane == 0) mbar_arrive(item_empty + slot);
      if (e.ntiles == 0) break;
      // this vector sees the slots [0, see.first) and [see.lo, see.end); all of the warp's see
      // [lo_max, end_min), and none sees any of [first_max, ...) before its own window
      const RowBounds see = row_bounds(a.win, e, e.row0 + at);
      const int end_min = min(e.slots, e.row0 + at0 + 1 - e.off);
      const RowBounds last = row_bounds(a.win, e, e.row0 + at1);
      const int lo_max = last.lo, first_max = last.first;
      float m_used = -INFINITY, l = 0.f;
      for (int j = 0; j < e.ntiles; ++j, sr.next(), vr.next()) {
        const uint32_t b = sr.at;
        const int mb = (T + j) & 1;
        if (!warp_mbar_wait(s_full + b, sr.phase, a.wait_ns, abort_flag)) {
          ok = false;
          break;
        }
        tc_fence_after();
        const uint32_t scol = tmem + lane_off + b * kKeys;
        // this warp's columns: 32 from 32 half on and 32 from 64 + 32 half on. SKIP: the second
        // ones of a tile whose slots end before them are neither read nor weighed
        const int t0 = j * kKeys, s0 = t0 + 32 * half;  // the tile's first and the warp's, as slots
        const bool two = !SKIP || t0 + kHalfKeys < e.slots;
        float v[2][32];
        tmem_ld_32cols(scol + 32 * half, v[0]);
        if (two) tmem_ld_32cols(scol + kHalfKeys + 32 * half, v[1]);
        tmem_wait_ld_of(v[0], v[1]);
        tc_fence_before();
        // What this vector sees, and of it what all of the warp's do, and what any does. (The
        // empty statements keep the branches: without them the compiler makes the selects of
        // most tiles' 64 columns unconditional, d 64 under 1,708 546 -> 598 us.)
        auto mask = [&](float(&x)[32], int sc) {
          asm volatile("" ::: "memory");
          uint32_t word = bit_span(see.lo - sc, see.end - sc);
          if (sc < first_max) word |= bit_span(0, see.first - sc);
          const uint32_t all = __reduce_and_sync(0xffffffffu, word);
          const uint32_t any = __reduce_or_sync(0xffffffffu, word);
#pragma unroll
          for (int c = 0; c < 32; c += 16) {
            const uint32_t of = 0xffffu << c;
            if ((all & of) == of) continue;
            asm volatile("" ::: "memory");
            if ((any & of) == 0u) {
              asm volatile("" ::: "memory");
#pragma unroll
              for (int y = c; y < c + 16; ++y) x[y] = -INFINITY;
            } else {
              asm volatile("" ::: "memory");
#pragma unroll
              for (int y = c; y < c + 16; ++y)
                if (!(word >> y & 1u)) x[y] = -INFINITY;
            }
          }
        };
        if (t0 < lo_max || t0 + kKeys > end_min) {
          mask(v[0], s0);
          if (two) mask(v[1], s0 + kHalfKeys);
        }
        float top[8];
        if (two) {
          if (SKIP) asm volatile("" ::: "memory");
#pragma unroll
          for (int x = 0; x < 8; ++x) top[x] = fmaxf(v[0][x], v[1][x]);
#pragma unroll
          for (int x = 8; x < 32; ++x) top[x & 7] = max3(top[x & 7], v[0][x], v[1][x]);
        } else {
          asm volatile("" ::: "memory");
#pragma unroll
          for (int x = 0; x < 8; ++x)
            top[x] = max3(v[0][x], v[0][x + 8], fmaxf(v[0][x + 16], v[0][x + 24]));
        }
        const float own = a.scale_log2 * max3(max3(top[0], top[1], top[2]),
                                              max3(top[3], top[4], top[5]), fmaxf(top[6], top[7]));
        // the other half's maximum; that it is there also says that the other warp has read
        // its scores, over which this one's weights may go
        maxima[(mb * 2 + half) * kBV + i] = own;
        named_bar_sync(1 + q4, 64);
        // the other warp may not come again; one outcome for the whole warp, as the flag may be
        // raised between its lanes' looks
        if (__any_sync(0xffffffffu, *abort_flag)) {
          ok = false;
          break;
        }
        tc_fence_after();
        const float mt = fmaxf(own, maxima[(mb * 2 + (half ^ 1)) * kBV + i]);
        const bool grow = mt > m_used + kRescaleLog2;
        if (__any_sync(0xffffffffu, grow)) {
          const float m_new = grow ? mt : m_used;
          if (j >= 1) {
            // O holds this item's PV so far: wait for the last one (its V stage
            // drained), rescale this warp's half of the columns in TMEM
            if (!warp_mbar_wait(v_empty + vr.at, vr.phase, a.wait_ns, abort_flag)) {
              ok = false;
              break;
            }
            tc_fence_after();
            const float f = grow ? ex2(m_used - m_new) : 1.f;
            const uint32_t ocol = tmem + lane_off + G::kOCol + ob * DH + half * (DH / 2);
#pragma unroll 1
            for (int c = 0; c < DH / 2; c += 16) {
              float ov[16];
              tmem_ld_16cols(ocol + c, ov);
              tmem_wait_ld();
#pragma unroll
              for (int x = 0; x < 16; ++x) ov[x] *= f;
              tmem_st_16cols(ocol + c, ov);
            }
            l *= f;
          }
          m_used = m_new;
        }
        // P = 2^(s scale - m_used) as bf16 pairs over the tile's S columns (a vector that has
        // seen no key yet: zeros). The sum takes the weights before their rounding, half a step
        // of bf16 either way: its own error averages out as the product's does, and the rounded
        // ones would cost two instructions more a pair (d 64, window 128: 187 -> 175 us)
        const float mneg = m_used == -INFINITY ? 0.f : -m_used;
        const float2 sc2 = make_float2(a.scale_log2, a.scale_log2), mn2 = make_float2(mneg, mneg);
        // the columns v[FIRST] to v[END - 1]
        auto weigh = [&](auto first, auto end) {
          uint32_t pw[2][16];
#pragma unroll
          for (int c = first; c < end; ++c) {
            float2 ps[4];
#pragma unroll
            for (int x = 0; x < 16; ++x) {
              const float2 y = fma2(make_float2(v[c][2 * x], v[c][2 * x + 1]), sc2, mn2);
              const float2 p = make_float2(ex2(y.x), ex2(y.y));
              pw[c][x] = pack_bf16(p.x, p.y);
              ps[x & 3] = x < 4 ? p : add2(ps[x & 3], p);
            }
            ps[0] = add2(add2(ps[0], ps[1]), add2(ps[2], ps[3]));
            l += ps[0].x + ps[0].y;
          }
#pragma unroll
          for (int c = first; c < end; ++c)
            tmem_st_16cols_u32(scol + (kHalfKeys * c + 32 * half) / 2, pw[c]);
        };
        constexpr std::integral_constant<int, 0> k0;
        constexpr std::integral_constant<int, 1> k1;
        constexpr std::integral_constant<int, 2> k2;
        if constexpr (SKIP) {
          weigh(k0, k1);
          if (two) {
            asm volatile("" ::: "memory");
            weigh(k1, k2);
          }
        } else {
          weigh(k0, k2);
        }
        tmem_wait_st();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive_remote(p_full_even + 8u * b);
      }
      if (!ok) break;
      // the output warps have read what the item before last left there
      if (!warp_mbar_wait(l_free + ls, ((u >> 1) & 1) ^ 1u, a.wait_ns, abort_flag)) {
        ok = false;
        break;
      }
      lsum[(ls * 2 + half) * kBV + i] = l;
      __syncwarp();
      if (lane == 0) mbar_arrive(l_full + ls);
      T += e.ntiles;
    }
    if (!ok) {
      *abort_flag = 1;
      flag(a.status, JET_ERR_TIMEOUT);
      // release the warp that shares this one's lanes, should it wait for the maximum: it looks
      // at the flag next
      __threadfence_block();
      __syncwarp();
      named_bar_arrive(1 + q4, 64);
    }
  } else {
    // ---------------------------------------------------------------- output
    const int q4 = warp & 3;
    const int i = q4 * 32 + lane;
    const uint32_t lane_off = uint32_t(q4 * 32) << 16;
    const uint32_t o_free_even = mapa_shared(o_free, 0);
    // the output is transposed through this warp's 4 KB of the stage so that
    // every global store covers whole 128-byte pieces of one vector
    uint4* stage = reinterpret_cast<uint4*>(smem + G::kOffStage + (warp - kFirstOut) * 4096);
    // the vectors this lane stores (4 s + lane / 8 of the warp's, 16 bytes each): their places
    // from the block's first on, in elements (128 / g positions of Hq heads fit an int)
    int place[8];
#pragma unroll
    for (int s = 0; s < 8; ++s) {
      const int gi = q4 * 32 + 4 * s + (lane >> 3);
      place[s] = (gi / g * a.Hq + gi % g) * DH;
    }
    bool ok = true;
    for (int u = 0; ok; ++u) {
      const int slot = u % kRing, ob = u % kOBufs, ls = u & 1;
      if (!warp_mbar_wait(item_full + slot, (u / kRing) & 1, a.wait_ns, abort_flag)) {
        ok = false;
        break;
      }
      const WinItem e = ring[slot];
      __syncwarp();
      if (lane == 0) mbar_arrive(item_empty + slot);
      if (e.ntiles == 0) break;
      __nv_bfloat16* out = a.o + (size_t(e.p0 + e.row0) * a.Hq + size_t(e.kh) * g) * DH;
      if (!warp_mbar_wait(l_full + ls, (u >> 1) & 1, a.wait_ns, abort_flag) ||
          !warp_mbar_wait(o_full + ob, (u / kOBufs) & 1, a.wait_ns, abort_flag)) {
        ok = false;
        break;
      }
      tc_fence_after();
      const float l = lsum[ls * 2 * kBV + i] + lsum[(ls * 2 + 1) * kBV + i];
      // scores all minus infinity, or a NaN among them: NaN until it is computed again
      const float inv = l > 0.f ? 1.f / l : __int_as_float(0x7fffffff);
      __syncwarp();
      if (lane == 0) mbar_arrive(l_free + ls);
      // up to 128 columns of O into registers as bf16 at a time; the next item's PV waits
      // only for the last of these reads and not for its stores
      constexpr int kCols = DH < 128 ? DH : 128;
      __nv_bfloat162 most = __floats2bfloat162_rn(0.f, 0.f);  // the largest output, or NaN
#pragma unroll 1
      for (int h0 = 0; h0 < DH; h0 += kCols) {
        uint32_t pk[kCols / 2];
#pragma unroll
        for (int c = 0; c < kCols; c += 32) {
          float ov[32];
          tmem_ld_32cols(tmem + lane_off + G::kOCol + ob * DH + h0 + c, ov);
          tmem_wait_ld();
#pragma unroll
          for (int x = 0; x < 16; ++x)
            pk[c / 2 + x] = pack_bf16(ov[2 * x] * inv, ov[2 * x + 1] * inv);
        }
        if (h0 + kCols == DH) {
          tc_fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive_remote(o_free_even + 8u * ob);
        }
#pragma unroll
        for (int x = 0; x < kCols / 2; ++x)
          most = __hmax2_nan(most, __habs2(*reinterpret_cast<const __nv_bfloat162*>(&pk[x])));
#pragma unroll
        for (int c = 0; c < kCols; c += 64) {
#pragma unroll
          for (int x = 0; x < 8; ++x)
            stage[lane * 8 + (x ^ (lane & 7))] =
                make_uint4(pk[c / 2 + 4 * x], pk[c / 2 + 4 * x + 1], pk[c / 2 + 4 * x + 2],
                           pk[c / 2 + 4 * x + 3]);
          __syncwarp();
#pragma unroll
          for (int s = 0; s < 8; ++s) {
            const int iv = 4 * s + (lane >> 3), c8 = lane & 7;
            const uint4 val = stage[iv * 8 + (c8 ^ (iv & 7))];
            if (q4 * 32 + iv < e.nv)
              *reinterpret_cast<uint4*>(out + place[s] + h0 + c + c8 * 8) = val;
          }
          __syncwarp();
        }
      }
      // vectors with a NaN or an infinity (a weight above 1 may have taken a large value past the
      // largest float) are computed again from what they see alone, after the last item
      const bool odd = !(l > 0.f) || __hisnan(most.x) || __hisnan(most.y) || __hisinf(most.x) ||
                       __hisinf(most.y);
      if (__any_sync(0xffffffffu, i < e.nv && odd) && lane == 0) note_odd(odd_items(), u);
    }
    if (!ok) {
      *abort_flag = 1;
      flag(a.status, JET_ERR_TIMEOUT);
    }
  }

  tc_fence_before();
  __syncthreads();
  // neither CTA leaves (or frees its TMEM) while the partner's MMAs, copies or
  // arrivals may still use its shared memory or TMEM
  cluster_sync();
  if (warp == 1) {
    tc_fence_after();
    tmem_dealloc_pair(tmem, G::kTmemCols);
  }
  if (odd_items()->any(lane) && !*abort_flag)
    odd_outputs<DH>(a, *odd_items(), int(rank), warp, lane);
}

// packed [keys, Hkv, DH] bf16: box of 32 d x 1 head x box_rows keys, 64-byte swizzle
bool encode_v64(CUtensorMap* map, const void* base, int rows, int heads, int box_rows) {
  auto fn = encode_fn();
  if (!fn) return false;
  const cuuint64_t dims[3] = {64, cuuint64_t(heads), cuuint64_t(rows)};
  const cuuint64_t strides[2] = {128, cuuint64_t(heads) * 128};
  const cuuint32_t box[3] = {32, 1, cuuint32_t(box_rows)};
  const cuuint32_t estr[3] = {1, 1, 1};
  return fn(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<void*>(base), dims, strides, box,
            estr, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_64B,
            CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <int DH, bool SKIP>
cudaError_t launch_pairs(const jet_layout& lay, const jet_dims& d, const Window& win,
                         const void* q, const void* k, const void* v, void* o, int* status,
                         cudaStream_t st) {
  const jet_sizes& n = lay.n;
  const int g = d.Hq / d.Hkv;
  if (g > kBV) return cudaErrorInvalidValue;
  CUtensorMap tmQ, tmK, tmV, tmK16, tmV16;
  if (!encode_3d(&tmQ, q, n.total_prefix, d.Hq, DH, g, kBV / g) ||
      !encode_3d(&tmK, k, n.total_prefix, d.Hkv, DH, 1, kHalfKeys) ||
      !encode_3d(&tmK16, k, n.total_prefix, d.Hkv, DH, 1, kSlotBox))
    return cudaErrorInvalidValue;
  const bool maps = DH == 64 ? encode_v64(&tmV, v, n.total_prefix, d.Hkv, kKeys) &&
                                   encode_v64(&tmV16, v, n.total_prefix, d.Hkv, kSlotBox)
                             : encode_3d(&tmV, v, n.total_prefix, d.Hkv, DH, 1, kKeys) &&
                                   encode_3d(&tmV16, v, n.total_prefix, d.Hkv, DH, 1, kSlotBox);
  if (!maps) return cudaErrorInvalidValue;
  WinPreArgs a{};
  a.wait_ns = wait_budget_ns();
  a.hold_first = test_stall();
  a.prefix_offset = lay.prefix_offset;
  a.req_order = lay.req_order;
  a.q = static_cast<const __nv_bfloat16*>(q);
  a.k = static_cast<const __nv_bfloat16*>(k);
  a.v = static_cast<const __nv_bfloat16*>(v);
  a.o = static_cast<__nv_bfloat16*>(o);
  a.status = status;
  a.win = win;
  a.R = n.R;
  a.total = n.total_prefix;
  a.Hq = d.Hq;
  a.Hkv = d.Hkv;
  a.g = g;
  a.rb = kBV / g;
  a.scale_log2 = 1.4426950408889634f / sqrtf(float(DH));
  const size_t smem = WinGeo<DH>::kBytes + 1024;
  auto kern = prefill_window_kernel<DH, SKIP>;
  cudaError_t e =
      cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, int(smem));
  if (e != cudaSuccess) return e;
  const long long items = (long long)n.R * d.Hkv * ((n.max_prefix - 1) / (2 * a.rb) + 1);
  // the static schedule deals the items to the pairs that are resident at once
  const int held = resident_pairs(reinterpret_cast<const void*>(kern), kWinThreads, smem);
  const int pairs = int(std::max<long long>(1, std::min<long long>(held, items)));
  return launch_pdl_pairs(kern, dim3(unsigned(2 * pairs)), dim3(kWinThreads), smem, st, tmQ, tmK,
                          tmV, tmK16, tmV16, a);
}

// Whether the softmax looks for tiles that end in their first half. The branches cost it 8 % of a
// tile, so it pays where most items are short and end so: the slots of a block in the longest
// prefix end in the first half of their third tile or before (24,000 positions, d 64, 16/2 heads,
// 2, 3, 4 and 6 tiles: 52.6, 68.5, 85.1 and 118 us with them, 55.2, 69.8, 84.7 and 114 without; d 128,
// 32/8 heads: 117, 154, 183 and 247, and 124, 157, 182 and 238). At d 256 the tensor pipe takes
// longer than the softmax and they never cost more than they give (2 to 8 tiles 1 to 3 %).
bool skips(const jet_sizes& n, const jet_dims& d, const Window& win) {
  const int block = 2 * (kBV / (d.Hq / d.Hkv));
  const int slots = block_slots(win, std::max(0, n.max_prefix - block), n.max_prefix).n;
  return slots <= 3 * kKeys && (slots - 1) % kKeys < kHalfKeys;
}

}  // namespace

cudaError_t launch_prefill_window(const jet_layout& lay, const jet_dims& d, int window, int sinks,
                                  const void* q, const void* k, const void* v, void* o,
                                  int* status, cudaStream_t st) {
  const Window win{window, sinks};
  if (d.Hq / d.Hkv > kBV) return cudaErrorInvalidValue;
  const bool skip = skips(lay.n, d, win);
  if (d.d == 64)
    return skip ? launch_pairs<64, true>(lay, d, win, q, k, v, o, status, st)
                : launch_pairs<64, false>(lay, d, win, q, k, v, o, status, st);
  if (d.d == 128)
    return skip ? launch_pairs<128, true>(lay, d, win, q, k, v, o, status, st)
                : launch_pairs<128, false>(lay, d, win, q, k, v, o, status, st);
  if (d.d == 256) return launch_pairs<256, true>(lay, d, win, q, k, v, o, status, st);
  return cudaErrorInvalidValue;
}

}  // namespace jet
