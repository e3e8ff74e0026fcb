// Cascade attention over an 8-bit prefix cache on the 5th-generation tensor cores
// (Sec. 4.1; bf16 queries, candidates' keys and values, and outputs; f32 accumulation).
//
// As in attend_tc.cu a CTA owns one (request r, key/value head kh, prefix chunk, block of
// up to 128 query vectors), streams the chunk's 64-key tiles once for all of them and
// leaves a partial that the combine merges, or the output where the request is one
// chunk. A cache tile is half the bytes of a bf16 one, so at the HBM rate an SM has half
// the time for it (d 256: 32 KB, 0.73 us): what follows keeps each unit below that.
//
//   scores   S = Q K^T on the codes as they are (kind::f8f6f4). A query is held as two
//            e4m3 numbers, q = 2^x (hi + lo), x per row: hi has the first four of a bf16
//            number's eight digits, lo the other four, so the split is exact for
//            elements within 2^-10 of the row's largest and leaves 2^-10 of 2^x, at
//            most 2^-18 of that largest element, below. (Keys widened to bf16 instead
//            would pass shared memory twice more: 1,536 cycles a tile of d 256, 1,393
//            at the HBM rate.) S = acc 2^(x + X), X the tile's exponent: the 64 tokens of
//            a block are a tile.
//   outputs  O += P V with P in bf16 and V widened from the codes to bf16, exactly, by
//            four warps on the way (P in e4m3 would lose the many small weights next
//            to a large one).
//
//   warp 0       TMA producer: rings of K tiles, of V tiles, and the query block
//   warp 1       TMEM allocator, MMA issuer
//   warp 2       scheduler: work items one ahead
//   warps 4..11  softmax, two groups of four on alternating tiles: thread = query
//                vector = TMEM lane. The running maximum of a row passes from group to
//                group through shared memory, ahead of the exponentials. P_j overwrites
//                S_j in TMEM.
//   warps 12..15 per item the queries' split into TMEM, per tile V to bf16. Values of
//                keys past the chunk (other requests') become zeros there.
// The candidates' own tokens come first in a request's last chunk, as 32-key tiles of
// bf16 keys and values (the same bytes as a cache tile) against the bf16 queries; their
// values pass the widening warps too, which take non-finite ones out, as a weight of
// zero would spread them to the rows that do not see them; the output adds them back
// for the rows that do.
#include <algorithm>
#include <cmath>
#include <type_traits>

#include "attend_tc.cuh"
#include "kv_cache.h"

namespace jet {
namespace {

constexpr int kBC = 32;  // candidate tokens per tile
constexpr int kThreads = 512;
constexpr int kProdWarp = 0, kMmaWarp = 1, kSchedWarp = 2, kSoftWarp = 4, kWideWarp = 12;

template <int DH>
struct Geo {
  static constexpr uint32_t kTile = kBN * DH;             // bytes of a K or V tile
  static constexpr int kK = DH == 256 ? 3 : 6;            // K tiles in flight
  static constexpr int kV = kK;                           // V tiles in flight
  static constexpr int kW = DH == 256 ? 1 : 2;            // widened V tiles
  static constexpr int kS = DH == 256 ? 2 : 4;            // S buffers
  static constexpr uint32_t kOffK = kBV * DH * 2;         // after the bf16 query block
  static constexpr uint32_t kOffV = kOffK + kK * kTile;
  static constexpr uint32_t kOffW = kOffV + kV * kTile;
  static constexpr uint32_t kOffStage = kOffW + kW * 2 * kTile;  // 2 KB per softmax warp
  static constexpr uint32_t kOffSmall = kOffStage + 8 * 2048;
  static constexpr uint32_t kBytes = kOffSmall + 8192;
  // TMEM: O, the S buffers (P in place of S), the queries' hi and lo codes
  static constexpr uint32_t kTmemCols = 512;
  static constexpr uint32_t kSCol = DH;
  static constexpr uint32_t kQCol = kSCol + kS * kBN;
  static_assert(kQCol + DH / 2 <= kTmemCols, "TMEM columns");
  static_assert(kBytes + 1024 <= 232448, "shared memory");
};

struct Kv8Args : AttArgs {
  const uint8_t* k_exp;  // exponent bytes of the caches
  const uint8_t* v_exp;
  const __nv_bfloat16* v_cand;
};

// One work item as the scheduler publishes it: its geometry, with nct tiles of
// candidate tokens [f_begin, f_begin + fed) before npt tiles of the prefix.
struct __align__(16) KvItem {
  ItemGeo e;
  int fed;
  int live;  // 0: no more items
};

struct Small {
  KvItem ring[2];
  uint64_t k_full[6], k_empty[6], v_full[6], v_empty[6];
  uint64_t w_full[2], w_empty[2];        // widened V tiles
  uint64_t s_full[4], p_full[4], pv_done[4];
  uint64_t m_full[2][4];                 // a tile's running maxima, per softmax warp
  uint64_t l_full[4];                    // both groups' sums of an item
  uint64_t item_full[2], item_empty[2];
  uint64_t q_full, q_free;               // the bf16 query block
  uint64_t qt_full, qt_free;             // the queries' codes in TMEM
  uint64_t qx_read;                      // their exponents are in the softmax's registers
  uint64_t o_free;                       // an item's O is out of TMEM
  uint64_t drain;
  uint32_t tmem;
  volatile int abort;
  volatile int bad[2][4];                // non-finite candidate values, per widening warp
  float m[2][kBV];                       // running maxima after an even / odd tile
  float2 ml[2][2][kBV];                  // [item parity][group] (m, l)
  int qx[2][kBV];                        // [item parity] the queries' exponents
};
static_assert(sizeof(Small) <= 8192, "the small part of shared memory");

// D[tmem] (+)= A[tmem] B[smem]^T, e4m3 inputs, f32 accumulation; four A elements per
// 32-bit TMEM column
__device__ __forceinline__ void mma_e4m3_ta(uint32_t d_tmem, uint32_t a_tmem, uint64_t b_desc,
                                            uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], [%1], %2, %3, p;\n\t}" ::"r"(d_tmem),
      "r"(a_tmem), "l"(b_desc), "r"(idesc), "r"(accumulate)
      : "memory");
}

// e4m3 A and B (format 0, both K-major), f32 accumulator
constexpr uint32_t idesc_e4m3_f32(int M, int N) {
  return (1u << 4) | (uint32_t(N >> 3) << 17) | (uint32_t(M >> 4) << 24);
}

// K-major operand rows of 64 bytes under 64-byte swizzling: 8-row atoms of 512 bytes
__device__ __forceinline__ uint64_t desc_k_sw64(uint32_t addr) {
  uint64_t d = 0;
  d |= uint64_t((addr >> 4) & 0x3FFFu);
  d |= uint64_t(1) << 16;
  d |= uint64_t(512 >> 4) << 32;
  d |= uint64_t(1) << 46;
  d |= uint64_t(4) << 61;
  return d;
}

// 16 consecutive 32-bit columns of this warp's 32 TMEM lanes
__device__ __forceinline__ void tmem_st_16cols_u32(uint32_t taddr, const uint32_t (&v)[16]) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], "
      "{%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};" ::"r"(taddr),
      "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7]),
      "r"(v[8]), "r"(v[9]), "r"(v[10]), "r"(v[11]), "r"(v[12]), "r"(v[13]), "r"(v[14]),
      "r"(v[15])
      : "memory");
}

__device__ __forceinline__ uint32_t mul_bf16x2(uint32_t a, uint32_t b) {
  uint32_t d;
  asm("mul.rn.bf16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
  return d;
}

// 2^x as a bf16 number, twice; x in [-126, 127]
__device__ __forceinline__ uint32_t pow2_bf16x2(int x) {
  const uint32_t h = uint32_t(x + 127) << 7;
  return h | h << 16;
}

// Two e4m3 codes in the high bytes of the halves of w as bf16 numbers times 2^-120: the
// four exponent and three fraction bits under bf16's exponent (subnormal codes are
// subnormal there)
__device__ __forceinline__ uint32_t widen2(uint32_t w) {
  return ((w >> 4) & 0x07f007f0u) | (w & 0x80008000u);
}

// 0x80 in each byte of w that is a NaN code
__device__ __forceinline__ uint32_t nan_codes(uint32_t w) {
  return ((w & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u;
}

__device__ __forceinline__ bool any_nonfinite_bf16x2(uint32_t w) {
  return (w & 0x7f80u) == 0x7f80u || (w & 0x7f800000u) == 0x7f800000u;
}

__device__ __forceinline__ uint32_t drop_nonfinite_bf16x2(uint32_t w) {
  if ((w & 0x7f80u) == 0x7f80u) w &= 0xffff0000u;
  if ((w & 0x7f800000u) == 0x7f800000u) w &= 0x0000ffffu;
  return w;
}

template <int DH>
__global__ void __launch_bounds__(kThreads, 1)
attend_kv8_kernel(const __grid_constant__ CUtensorMap tmQ, const __grid_constant__ CUtensorMap tmK,
                  const __grid_constant__ CUtensorMap tmV, const __grid_constant__ CUtensorMap tmKc,
                  const __grid_constant__ CUtensorMap tmVc, const Kv8Args a) {
  using G = Geo<DH>;
  constexpr int NK = G::kK, NV = G::kV, NW = G::kW, NS = G::kS;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) &
                                             ~uintptr_t(1023));
  Small& sh = *reinterpret_cast<Small*>(smem + G::kOffSmall);
  volatile int* abort_flag = &sh.abort;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int g = a.g, rb = a.rb;
  if (threadIdx.x == 0) {
    for (int s = 0; s < NK; ++s) {
      mbar_init(sh.k_full + s, 1);
      mbar_init(sh.k_empty + s, 1);
    }
    for (int s = 0; s < NV; ++s) {
      mbar_init(sh.v_full + s, 1);
      mbar_init(sh.v_empty + s, 4);
    }
    for (int s = 0; s < NW; ++s) {
      mbar_init(sh.w_full + s, 4);
      mbar_init(sh.w_empty + s, 1);
    }
    for (int b = 0; b < NS; ++b) {
      mbar_init(sh.s_full + b, 1);
      mbar_init(sh.p_full + b, 4);
      mbar_init(sh.pv_done + b, 1);
    }
    for (int q = 0; q < 4; ++q) {
      mbar_init(&sh.m_full[0][q], 1);
      mbar_init(&sh.m_full[1][q], 1);
      mbar_init(sh.l_full + q, 2);
    }
    for (int b = 0; b < 2; ++b) {
      mbar_init(sh.item_full + b, 1);
      mbar_init(sh.item_empty + b, 14);  // producer, MMA thread, 8 softmax and 4 widening warps
    }
    mbar_init(&sh.q_full, 1);
    mbar_init(&sh.q_free, 5);            // the split's four warps, the last product with it
    mbar_init(&sh.qt_full, 4);
    mbar_init(&sh.qt_free, 1);
    mbar_init(&sh.qx_read, 8);
    mbar_init(&sh.o_free, 8);
    mbar_init(&sh.drain, 1);
    sh.abort = 0;
    fence_barrier_init();
  }
  if (warp == kProdWarp && lane == 0) {
    tma_prefetch_desc(&tmQ);
    tma_prefetch_desc(&tmK);
    tma_prefetch_desc(&tmV);
    if (a.has_cand) {
      tma_prefetch_desc(&tmKc);
      tma_prefetch_desc(&tmVc);
    }
  }
  // global memory and TMEM only after the previous kernel of the stream is done
  pdl_begin();
  if (warp == kMmaWarp) {
    tmem_alloc(&sh.tmem, G::kTmemCols);
    tmem_relinquish();
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = sh.tmem;
  // registers to the softmax warps, which hold a tile's scores: 72 + 168 + 168 + 104 are
  // the four warpgroups' launch share of 128 each
  if (warp < kSoftWarp) {
  asm volatile("setmaxnreg.dec.sync.aligned.u32 72;");
  if (warp == kSchedWarp) {
    // ---------------------------------------------------------------- scheduler
    const int count = a.sorted ? *a.item_count : 0;
    ItemWindow window{};
    for (int u = 0;; ++u) {
      const int slot = u & 1;
      if (!warp_mbar_wait(sh.item_empty + slot, ((u >> 1) & 1) ^ 1u, a.wait_ns, abort_flag)) {
        if (lane == 0) {
          sh.abort = 1;
          flag(a.status, JET_ERR_TIMEOUT);
        }
        break;
      }
      ItemGeo e{};
      bool live = false;
      if (a.sorted) {
        // the CTA's first item is number blockIdx.x, later ones come from the shared
        // counter, past the grid's first items
        if (lane == 0) {
          for (bool first = (u == 0);; first = false) {
            const int idx = first ? int(blockIdx.x) : int(gridDim.x) + atomicAdd(a.item_next, 1);
            if (idx >= count) break;
            bool fits;
            e = item_geo(a, a.items[idx], &fits);
            live = e.ok;
            if (live) break;
            flag(a.status, JET_ERR_DEVICE);  // the list holds an item the layout lacks
          }
        }
      } else {
        // dealt out back and forth, as the bf16 kernel does
        const int n = int(gridDim.x);
        const int k = u * n + ((u & 1) ? n - 1 - int(blockIdx.x) : int(blockIdx.x));
        int4 it;
        if (k < a.n_all && nth_item(a, k, lane, window, &it, &e)) {
          live = e.ok;
          if (!live && lane == 0) flag(a.status, JET_ERR_DEVICE);
        }
      }
      if (lane == 0) {
        int fed = 0;
        if (live) {
          if (e.nct > 0) {
            // the fed tokens that a row of this block sees: up to its last row's own,
            // from the first of its first row's candidate on
            fed = e.row0 + e.nv / g - 1;
            int lo = 0;
            if (fed > kBC && e.row0 > 0) {
              const int c = a.row_cand[e.n0 + e.row0];
              if (c >= 0 && c < a.C)
                lo = min(max(a.cand_row_offset[c] - e.n0 - 1, 0), fed);
            }
            e.f_begin += lo;
            fed -= lo;
          }
          e.nct = (fed + kBC - 1) / kBC;
          e.ntiles = e.npt + e.nct;
        }
        sh.ring[slot].e = e;
        sh.ring[slot].fed = fed;
        sh.ring[slot].live = live;
        mbar_arrive(sh.item_full + slot);
        if (live) {  // the query block on its way into L2
#pragma unroll
          for (int sl = 0; sl < DH / 64; ++sl)
            tma_prefetch_3d(&tmQ, sl * 64, e.kh * g, e.n0 + e.row0);
        }
      }
      if (!__shfl_sync(0xffffffffu, live ? 1 : 0, 0)) break;
    }
  } else if (warp == kProdWarp) {
    // ---------------------------------------------------------------- producer
    if (elect_one()) {
      const uint64_t pol = policy_evict_first();
      uint32_t k_issued = 0, k_par = 0, v_issued = 0, v_par = 0, q_issued = 0, q_par = 0;
      int T = 0;  // tiles of earlier items
      bool ok = true;
      for (int u = 0; ok; ++u) {
        const int slot = u & 1;
        if (!mbar_wait(sh.item_full + slot, (u >> 1) & 1, a.wait_ns, abort_flag)) {
          ok = false;
          break;
        }
        if (!sh.ring[slot].live) break;
        const ItemGeo e = sh.ring[slot].e;
        // K_j, V_j and the query block are issued as soon as their places drain
        int jk = 0, jv = 0;
        bool q_sent = false;
        IdleClock clk;
        while (jv < e.ntiles || !q_sent) {
          bool progressed = false;
          if (!q_sent && (u == 0 || mbar_test(&sh.q_free, (u - 1) & 1))) {
            if (!(u == 0 && a.hold_first)) {  // test hook: the first block never lands
              mbar_arrive_expect_tx(&sh.q_full, uint32_t(DH / 64) * 64 * 2 * g * rb);
#pragma unroll
              for (int sl = 0; sl < DH / 64; ++sl)
                tma_load_3d(smem + sl * (kBV * 128), &tmQ, &sh.q_full, sl * 64, e.kh * g,
                            e.n0 + e.row0, pol);
              q_issued = 1;
              q_par = u & 1;
            }
            q_sent = progressed = true;
          }
          if (jk < e.ntiles) {
            const int s = (T + jk) % NK;
            const uint32_t ph = ((T + jk) / NK) & 1;
            if (mbar_test(sh.k_empty + s, ph ^ 1u)) {
              uint8_t* ks = smem + G::kOffK + s * G::kTile;
              mbar_arrive_expect_tx(sh.k_full + s, G::kTile);
              if (jk < e.nct) {
#pragma unroll
                for (int sl = 0; sl < DH / 64; ++sl)
                  tma_load_3d(ks + sl * (kBC * 128), &tmKc, sh.k_full + s, sl * 64, e.kh,
                              e.f_begin + jk * kBC, pol);
              } else {
                const int key = e.p0 + e.k_begin + (jk - e.nct) * kBN;
#pragma unroll
                for (int sl = 0; sl < (DH + 127) / 128; ++sl)
                  tma_load_3d(ks + sl * (kBN * 128), &tmK, sh.k_full + s, sl * 128, e.kh, key, pol);
              }
              k_issued |= 1u << s;
              k_par = (k_par & ~(1u << s)) | (ph << s);
              ++jk;
              progressed = true;
            }
          }
          if (jv < jk) {
            const int s = (T + jv) % NV;
            const uint32_t ph = ((T + jv) / NV) & 1;
            if (mbar_test(sh.v_empty + s, ph ^ 1u)) {
              uint8_t* vs = smem + G::kOffV + s * G::kTile;
              mbar_arrive_expect_tx(sh.v_full + s, G::kTile);
              if (jv < e.nct) {
#pragma unroll
                for (int sl = 0; sl < DH / 64; ++sl)
                  tma_load_3d(vs + sl * (kBC * 128), &tmVc, sh.v_full + s, sl * 64, e.kh,
                              e.f_begin + jv * kBC, pol);
              } else {
                tma_load_3d(vs, &tmV, sh.v_full + s, 0, e.kh,
                            e.p0 + e.k_begin + (jv - e.nct) * kBN, pol);
              }
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
        if (!ok) break;
        mbar_arrive(sh.item_empty + slot);
        T += e.ntiles;
      }
      if (!ok) {
        sh.abort = 1;
        flag(a.status, JET_ERR_TIMEOUT);
        // let every copy already issued land before the CTA can exit
        if (q_issued) mbar_wait(&sh.q_full, q_par, kDrainNs, nullptr);
        for (int t = 0; t < NK; ++t)
          if (k_issued & (1u << t)) mbar_wait(sh.k_full + t, (k_par >> t) & 1u, kDrainNs, nullptr);
        for (int t = 0; t < NV; ++t)
          if (v_issued & (1u << t)) mbar_wait(sh.v_full + t, (v_par >> t) & 1u, kDrainNs, nullptr);
      }
    }
  } else if (warp == kMmaWarp) {
    // ---------------------------------------------------------------- MMA issuer
    if (elect_one()) {
      constexpr uint32_t id_s = idesc_e4m3_f32(kBV, kBN);
      constexpr uint32_t id_c = idesc_bf16_f32(kBV, kBC);
      constexpr uint32_t id_o = idesc_bf16_f32(kBV, DH) | (1u << 16);  // B (V) is MN-major
      const uint32_t qs = smem_u32(smem);
      bool ok = true;
      int T = 0;
      for (int u = 0; ok; ++u) {
        const int slot = u & 1;
        if (!mbar_wait(sh.item_full + slot, (u >> 1) & 1, a.wait_ns, abort_flag)) {
          ok = false;
          break;
        }
        if (!sh.ring[slot].live) break;
        const int nct = sh.ring[slot].e.nct, ntiles = sh.ring[slot].e.ntiles;
        if (nct == 0) mbar_arrive(&sh.q_free);  // only the split reads the bf16 block
        int js = 0, jo = 0;
        IdleClock clk;
        while (jo < ntiles) {
          bool progressed = false;
          if (js < ntiles) {
            const int Tj = T + js;
            const int s = Tj % NK, b = Tj % NS;
            if (mbar_test(sh.k_full + s, (Tj / NK) & 1) &&
                mbar_test(sh.pv_done + b, ((Tj / NS) & 1) ^ 1u) &&
                mbar_test(js < nct ? &sh.q_full : &sh.qt_full, u & 1)) {
              tc_fence_after();
              const uint32_t ks = smem_u32(smem + G::kOffK + s * G::kTile);
              const uint32_t d = tmem + G::kSCol + b * kBN;
              if (js < nct) {
#pragma unroll
                for (int st = 0; st < DH / 16; ++st) {
                  const int sl = st >> 2, k = st & 3;
                  mma_f16(d, desc_k_sw128(qs + sl * (kBV * 128) + 32 * k),
                          desc_k_sw128(ks + sl * (kBC * 128) + 32 * k), id_c, st != 0);
                }
                if (js == nct - 1) mma_commit(&sh.q_free);
              } else {
#pragma unroll
                for (int st = 0; st < DH / 16; ++st) {  // hi, then lo, over the same keys
                  const int kk = st % (DH / 32);
                  const uint64_t kd = DH == 64 ? desc_k_sw64(ks + 32 * kk)
                                               : desc_k_sw128(ks + (kk >> 2) * (kBN * 128) +
                                                              32 * (kk & 3));
                  mma_e4m3_ta(d, tmem + G::kQCol + uint32_t(8 * st), kd, id_s, st != 0);
                }
                if (js == ntiles - 1) mma_commit(&sh.qt_free);
              }
              mma_commit(sh.s_full + b);
              mma_commit(sh.k_empty + s);
              ++js;
              progressed = true;
            }
          }
          if (jo < js) {
            const int Tj = T + jo;
            const int w = Tj % NW, b = Tj % NS;
            // the item's first P V overwrites O: the previous item's O must be out
            if ((jo > 0 || u == 0 || mbar_test(&sh.o_free, (u - 1) & 1)) &&
                mbar_test(sh.p_full + b, (Tj / NS) & 1) &&
                mbar_test(sh.w_full + w, (Tj / NW) & 1)) {
              tc_fence_after();
              const uint32_t pt = tmem + G::kSCol + b * kBN;
              const uint32_t vs = smem_u32(smem + G::kOffW + w * 2 * G::kTile);
              if (jo < nct) {
#pragma unroll
                for (int k = 0; k < kBC / 16; ++k)
                  mma_f16_ta(tmem, pt + uint32_t(8 * k), desc_mn_sw128(vs + k * 2048, kBC * 128),
                             id_o, (jo | k) != 0);
              } else {
#pragma unroll
                for (int k = 0; k < kBN / 16; ++k)
                  mma_f16_ta(tmem, pt + uint32_t(8 * k), desc_mn_sw128(vs + k * 2048, kBN * 128),
                             id_o, (jo | k) != 0);
              }
              mma_commit(sh.pv_done + b);
              mma_commit(sh.w_empty + w);
              ++jo;
              progressed = true;
            }
          }
          if (clk.expired(progressed, abort_flag, a.wait_ns)) {
            ok = false;
            break;
          }
        }
        if (!ok) break;
        mbar_arrive(sh.item_empty + slot);
        T += ntiles;
      }
      if (!ok) {
        sh.abort = 1;
        flag(a.status, JET_ERR_TIMEOUT);
        mma_commit(&sh.drain);
        mbar_wait(&sh.drain, 0, kDrainNs, nullptr);
      }
    }
  }
  } else if (warp >= kWideWarp) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 104;");
    // ---------------------------------------------------------------- queries and V
    const int q4 = warp - kWideWarp, t = threadIdx.x - kWideWarp * 32;  // row, thread of 128
    const uint32_t lane_off = uint32_t(q4 * 32) << 16;
    bool ok = true;
    int T = 0;
    for (int u = 0; ok; ++u) {
      const int slot = u & 1;
      if (!warp_mbar_wait(sh.item_full + slot, (u >> 1) & 1, a.wait_ns, abort_flag)) {
        ok = false;
        break;
      }
      if (!sh.ring[slot].live) break;
      const ItemGeo e = sh.ring[slot].e;
      const int fed = sh.ring[slot].fed;
      const size_t ex = size_t(kv_place(e.p0, e.r, e.k_begin / kBN)) * a.Hkv + e.kh;
      int byte = a.v_exp[ex];
      if (lane == 0) sh.bad[slot][q4] = 0;  // item u - 2's output is out (below)
      if (!warp_mbar_wait(&sh.q_full, u & 1, a.wait_ns, abort_flag)) {
        ok = false;
        break;
      }
      // the row's largest magnitude (NaN and infinities lie above all): rows past the
      // block's vectors hold what an earlier block left and go unread
      {
        uint32_t top = 0;
#pragma unroll 4
        for (int c = 0; c < DH / 8; ++c) {
          const uint4 x = *reinterpret_cast<const uint4*>(smem + (c >> 3) * (kBV * 128) +
                                                          sw128(t, c & 7));
          top = __vmaxu2(top, __vmaxu2(__vmaxu2(x.x & 0x7fff7fffu, x.y & 0x7fff7fffu),
                                       __vmaxu2(x.z & 0x7fff7fffu, x.w & 0x7fff7fffu)));
        }
        top = max(top & 0xffffu, top >> 16);
        const bool finite = top < 0x7f80u;
        const int x = finite ? kv_exponent(top << 16) : 0;
        const float inv = pow2(-x);
        // the codes of the item before are read by its last product with the keys; a
        // softmax warp must not find qt_full two items on
        if (u >= 1 && (!warp_mbar_wait(&sh.qt_free, (u - 1) & 1, a.wait_ns, abort_flag) ||
                       !warp_mbar_wait(&sh.qx_read, (u - 1) & 1, a.wait_ns, abort_flag))) {
          ok = false;
          break;
        }
        sh.qx[slot][t] = x;
        tc_fence_after();
#pragma unroll 1
        for (int sl = 0; sl < DH / 64; ++sl) {
          uint32_t hi[16], lo[16];
#pragma unroll
          for (int c = 0; c < 8; ++c) {
            const uint4 xv = *reinterpret_cast<const uint4*>(smem + sl * (kBV * 128) + sw128(t, c));
            const uint32_t w[4] = {xv.x, xv.y, xv.z, xv.w};
#pragma unroll
            for (int i = 0; i < 2; ++i) {
              uint32_t hw = 0, lw = 0;
#pragma unroll
              for (int k = 0; k < 2; ++k) {
                const uint32_t p = w[2 * i + k];
                const float q0 = __uint_as_float(p << 16) * inv;
                const float q1 = __uint_as_float(p & 0xffff0000u) * inv;
                // the first four digits by their bits, the rest exactly
                const float h0 = __uint_as_float(__float_as_uint(q0) & 0xfff00000u);
                const float h1 = __uint_as_float(__float_as_uint(q1) & 0xfff00000u);
                const uint32_t ph = __nv_cvt_float2_to_fp8x2(make_float2(h0, h1), __NV_SATFINITE,
                                                             __NV_E4M3);
                const float2 back = e4m3x2_to_f32(ph);  // below 2^-6 the code is shorter
                const uint32_t pl = __nv_cvt_float2_to_fp8x2(
                    make_float2(q0 - back.x, q1 - back.y), __NV_SATFINITE, __NV_E4M3);
                hw |= ph << (16 * k);
                lw |= pl << (16 * k);
              }
              if (!finite) hw = 0x7f7f7f7fu;  // the whole row's output is NaN
              hi[2 * c + i] = hw;
              lo[2 * c + i] = lw;
            }
          }
          const uint32_t at = tmem + lane_off + G::kQCol + uint32_t(16 * sl);
          tmem_st_16cols_u32(at, hi);
          tmem_st_16cols_u32(at + DH / 4, lo);
        }
        tmem_wait_st();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) {
          mbar_arrive(&sh.qt_full);
          mbar_arrive(&sh.q_free);
        }
      }
      // V tiles: 16 codes to 16 bf16 numbers at a time
      for (int j = 0; j < e.ntiles; ++j) {
        const int Tj = T + j;
        const int s = Tj % NV, w = Tj % NW;
        // before item u can end: item u - 1's output is out, so that item u + 1 may take
        // its places (a wait past the end could miss the phase)
        if (j == e.ntiles - 1 && u >= 1 &&
            !warp_mbar_wait(&sh.o_free, (u - 1) & 1, a.wait_ns, abort_flag)) {
          ok = false;
          break;
        }
        if (!warp_mbar_wait(sh.v_full + s, (Tj / NV) & 1, a.wait_ns, abort_flag) ||
            !warp_mbar_wait(sh.w_empty + w, ((Tj / NW) & 1) ^ 1u, a.wait_ns, abort_flag)) {
          ok = false;
          break;
        }
        const uint8_t* vs = smem + G::kOffV + s * G::kTile;
        uint8_t* ws = smem + G::kOffW + w * 2 * G::kTile;
        if (j < e.nct) {
          // candidate values: bf16 already, in the places the product reads
          const int left = fed - j * kBC;
          bool found = false;
#pragma unroll 4
          for (int i = t; i < int(G::kTile) / 16; i += 128) {
            uint4 x = *reinterpret_cast<const uint4*>(vs + 16 * i);
            if (((i >> 3) & (kBC - 1)) >= left) x = make_uint4(0u, 0u, 0u, 0u);
            if (any_nonfinite_bf16x2(x.x) || any_nonfinite_bf16x2(x.y) ||
                any_nonfinite_bf16x2(x.z) || any_nonfinite_bf16x2(x.w)) {
              found = true;
              x = make_uint4(drop_nonfinite_bf16x2(x.x), drop_nonfinite_bf16x2(x.y),
                             drop_nonfinite_bf16x2(x.z), drop_nonfinite_bf16x2(x.w));
            }
            *reinterpret_cast<uint4*>(ws + 16 * i) = x;
          }
          if (__any_sync(0xffffffffu, found) && lane == 0) sh.bad[slot][q4] = 1;
        } else {
          const int pt = j - e.nct;
          const int X = min(max(byte - 127, kKvLow), kKvHigh);
          if (pt + 1 < e.npt) byte = a.v_exp[ex + size_t(pt + 1) * a.Hkv];
          const int left = e.k_end - (e.k_begin + pt * kBN);
          // 2^(120 + X) in one factor, or two where bf16 does not hold it
          const uint32_t f = pow2_bf16x2(min(120 + X, 127));
          const uint32_t f2 = pow2_bf16x2(max(X - 7, 0));
          constexpr int kC = DH / 16;  // 16-code pieces of a key
#pragma unroll
          for (int i = 0; i < kBN * kC / 128; ++i) {
            const int key = (t + i * 128) / kC, c = t % kC;
            const uint4 x = *reinterpret_cast<const uint4*>(vs + key * DH + c * 16);
            const uint32_t in[4] = {x.x, x.y, x.z, x.w};
            uint32_t y[8];
#pragma unroll
            for (int q = 0; q < 4; ++q) {
              y[2 * q] = mul_bf16x2(widen2(__byte_perm(in[q], 0u, 0x1404)), f);
              y[2 * q + 1] = mul_bf16x2(widen2(__byte_perm(in[q], 0u, 0x3424)), f);
            }
            if (X > 7) {
#pragma unroll
              for (int q = 0; q < 8; ++q) y[q] = mul_bf16x2(y[q], f2);
            }
            if (nan_codes(x.x) | nan_codes(x.y) | nan_codes(x.z) | nan_codes(x.w)) {
#pragma unroll
              for (int q = 0; q < 4; ++q) {
                const uint32_t n = nan_codes(in[q]);
                if (n & 0x80u) y[2 * q] = (y[2 * q] & 0xffff0000u) | 0x7fffu;
                if (n & 0x8000u) y[2 * q] = (y[2 * q] & 0xffffu) | 0x7fff0000u;
                if (n & 0x800000u) y[2 * q + 1] = (y[2 * q + 1] & 0xffff0000u) | 0x7fffu;
                if (n & 0x80000000u) y[2 * q + 1] = (y[2 * q + 1] & 0xffffu) | 0x7fff0000u;
              }
            }
            if (key >= left) {  // other requests' keys
#pragma unroll
              for (int q = 0; q < 8; ++q) y[q] = 0u;
            }
            // pieces 2 c and 2 c + 1 of the key's row; odd slices in the other order,
            // so that eight lanes' 16-byte stores fall in different banks
            uint8_t* row = ws + (c >> 2) * (kBN * 128);
            const int first = (c >> 2) & 1;
            const uint4 p0 = make_uint4(y[0], y[1], y[2], y[3]);
            const uint4 p1 = make_uint4(y[4], y[5], y[6], y[7]);
            *reinterpret_cast<uint4*>(row + sw128(key, (2 * c + first) & 7)) = first ? p1 : p0;
            *reinterpret_cast<uint4*>(row + sw128(key, (2 * c + 1 - first) & 7)) = first ? p0 : p1;
          }
        }
        fence_proxy_async_smem();
        __syncwarp();
        if (lane == 0) {
          mbar_arrive(sh.w_full + w);
          mbar_arrive(sh.v_empty + s);
        }
      }
      if (!ok) break;
      if (lane == 0) mbar_arrive(sh.item_empty + slot);
      T += e.ntiles;
    }
    if (!ok) {
      sh.abort = 1;
      flag(a.status, JET_ERR_TIMEOUT);
    }
  } else {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 168;");
    // ---------------------------------------------------------------- softmax
    const int q4 = warp & 3, grp = (warp - kSoftWarp) >> 2;
    const int i = q4 * 32 + lane;  // query vector within the block = TMEM lane
    const uint32_t lane_off = uint32_t(q4 * 32) << 16;
    uint4* stage = reinterpret_cast<uint4*>(smem + G::kOffStage + (warp - kSoftWarp) * 2048);
    bool ok = true;
    int T = 0;
    for (int u = 0; ok; ++u) {
      const int slot = u & 1;
      if (!warp_mbar_wait(sh.item_full + slot, (u >> 1) & 1, a.wait_ns, abort_flag)) {
        ok = false;
        break;
      }
      if (!sh.ring[slot].live) break;
      const ItemGeo e = sh.ring[slot].e;
      const bool valid = i < e.nv;
      const bool some = q4 * 32 < e.nv;  // a warp without vectors only keeps the barriers going
      int fa = 1, fb = 0;                // fed tokens this vector sees (none: shared row)
      if (valid && e.nct > 0) {
        const int n = e.n0 + (e.vbase + i) / g;
        const int c = a.row_cand[n];
        if (c >= 0 && c < a.C) {
          fa = a.cand_row_offset[c] - e.r - 1;  // y_{c,1}
          fb = n - e.r - 1;                     // the row's own fed token, inclusive
        }
      }
      const uint8_t* ex = a.k_exp + size_t(kv_place(e.p0, e.r, e.k_begin / kBN)) * a.Hkv + e.kh;
      const int j0 = (grp ^ T) & 1;  // this group's tiles: j0, j0 + 2, ..
      int byte = 0;
      if (j0 >= e.nct && j0 < e.ntiles) byte = ex[size_t(j0 - e.nct) * a.Hkv];
      int qx = 0;
      bool qx_read = false;
      auto read_qx = [&]() -> bool {
        if (!warp_mbar_wait(&sh.qt_full, u & 1, a.wait_ns, abort_flag)) return false;
        qx = sh.qx[slot][i];
        qx_read = true;
        __syncwarp();
        if (lane == 0) mbar_arrive(&sh.qx_read);
        return true;
      };
      float m_own = -INFINITY, l = 0.f;  // l: the sum over this group's tiles, relative to m_own

      // scores of W keys in columns klo .. khi, times mul in base 2, to weights
      auto tile = [&](auto width, int j, float mul, int klo, int khi) -> bool {
        constexpr int W = decltype(width)::value;
        const int Tj = T + j, b = Tj % NS;
        const uint32_t at = tmem + lane_off + G::kSCol + b * kBN;
        float sv[W];
        if (some) {
          float t0[W / 32][32];
#pragma unroll
          for (int k = 0; k < W / 32; ++k) tmem_ld_32cols(at + 32 * k, t0[k]);
          tmem_wait_ld();
#pragma unroll
          for (int c = 0; c < W; ++c) sv[c] = t0[c >> 5][c & 31];
          if (__any_sync(0xffffffffu, klo > 0 || khi < W)) {
#pragma unroll
            for (int c = 0; c < W; ++c)
              if (c < klo || c >= khi) sv[c] = -INFINITY;
          }
        }
        float mt = -INFINITY;
        if (some) {
          float mq[8];
#pragma unroll
          for (int q = 0; q < 8; ++q) mq[q] = sv[q];
#pragma unroll
          for (int c = 8; c < W; ++c) mq[c & 7] = fmaxf(mq[c & 7], sv[c]);
          mt = mul * fmaxf(fmaxf(fmaxf(mq[0], mq[1]), fmaxf(mq[2], mq[3])),
                           fmaxf(fmaxf(mq[4], mq[5]), fmaxf(mq[6], mq[7])));
        }
        // the row's maximum after the tile before, which the other group has
        if (Tj > 0 && !warp_mbar_wait(&sh.m_full[(Tj - 1) & 1][q4], ((Tj - 1) >> 1) & 1, a.wait_ns,
                                      abort_flag))
          return false;
        const float m_prev = j > 0 ? sh.m[(Tj - 1) & 1][i] : -INFINITY;
        const bool grow = j == 0 || (valid && mt > m_prev + kRescaleLog2);
        const float m_new = grow ? mt : m_prev;
        sh.m[Tj & 1][i] = m_new;
        __syncwarp();
        if (lane == 0) mbar_arrive(&sh.m_full[Tj & 1][q4]);
        if (some) {
          if (j > 0 && __any_sync(0xffffffffu, grow)) {
            // O holds this item's P V so far: wait for the last one, rescale in TMEM
            const int b1 = (Tj - 1) % NS;
            if (!warp_mbar_wait(sh.pv_done + b1, ((Tj - 1) / NS) & 1, a.wait_ns, abort_flag))
              return false;
            tc_fence_after();
            const float f = grow ? ex2(m_prev - m_new) : 1.f;
#pragma unroll 1
            for (int c0 = 0; c0 < DH; c0 += 32) {
              float ov[32];
              tmem_ld_32cols(tmem + lane_off + c0, ov);
              tmem_wait_ld();
#pragma unroll
              for (int c = 0; c < 32; ++c) ov[c] *= f;
              tmem_st_32cols(tmem + lane_off + c0, ov);
            }
          }
          if (m_new != m_own) {
            l = m_own == -INFINITY ? 0.f : l * ex2(m_own - m_new);
            m_own = m_new;
          }
          const float sub = m_new == -INFINITY ? 0.f : m_new;  // no key seen yet: weights of 0
          float ps[8];
#pragma unroll
          for (int q = 0; q < 8; ++q) ps[q] = 0.f;
          // the row sum uses the rounded values, which are what the tensor core multiplies
          auto weights = [&](int c) {
            const float x0 = ex2(fmaf(sv[c], mul, -sub)), x1 = ex2(fmaf(sv[c + 1], mul, -sub));
            const uint32_t w = pack_bf16(x0, x1);
            ps[(c >> 1) & 7] += __uint_as_float(w << 16) + __uint_as_float(w & 0xffff0000u);
            return w;
          };
#pragma unroll
          for (int k = 0; k < W / 32; ++k) {
            uint32_t pw[16];
#pragma unroll
            for (int c = 0; c < 16; ++c) pw[c] = weights(32 * k + 2 * c);
            tmem_st_16cols_u32(at + 16 * k, pw);
          }
          l += ((ps[0] + ps[1]) + (ps[2] + ps[3])) + ((ps[4] + ps[5]) + (ps[6] + ps[7]));
          tmem_wait_st();
        }
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(sh.p_full + b);
        return true;
      };

      for (int j = j0; j < e.ntiles; j += 2) {
        const int Tj = T + j, b = Tj % NS;
        if (j >= e.nct && !qx_read && !read_qx()) {
          ok = false;
          break;
        }
        if (!warp_mbar_wait(sh.s_full + b, (Tj / NS) & 1, a.wait_ns, abort_flag)) {
          ok = false;
          break;
        }
        tc_fence_after();
        const int held = byte;
        // the exponent of this group's next tile, a tile ahead of its use
        if (j + 2 >= e.nct && j + 2 < e.ntiles) byte = ex[size_t(j + 2 - e.nct) * a.Hkv];
        if (j < e.nct) {
          const int f0 = e.f_begin + j * kBC;
          ok = tile(std::integral_constant<int, kBC>(), j, a.scale_log2, max(0, fa - f0),
                    min(kBC, fb - f0 + 1));
        } else {
          const int X = min(max(held - 127, kKvLow), kKvHigh);
          const float mul = a.scale_log2 * pow2(min(max(qx + X, -126), 126));
          ok = tile(std::integral_constant<int, kBN>(), j, mul, 0,
                    min(kBN, e.k_end - (e.k_begin + (j - e.nct) * kBN)));
        }
        if (!ok) break;
      }
      if (!ok) break;
      if (!qx_read && !read_qx()) {
        ok = false;
        break;
      }
      // both groups' sums, relative to the maximum after the last tile
      sh.ml[slot][grp][i] = make_float2(m_own, l);
      __syncwarp();
      if (lane == 0) mbar_arrive(sh.l_full + q4);
      if (!warp_mbar_wait(sh.l_full + q4, u & 1, a.wait_ns, abort_flag)) {
        ok = false;
        break;
      }
      const int Tl = T + e.ntiles - 1;
      const float m_fin = sh.m[Tl & 1][i];
      const float2 x0 = sh.ml[slot][0][i], x1 = sh.ml[slot][1][i];
      l = (x0.x == -INFINITY && x0.y == 0.f ? 0.f : x0.y * ex2(x0.x - m_fin)) +
          (x1.x == -INFINITY && x1.y == 0.f ? 0.f : x1.y * ex2(x1.x - m_fin));
      if (valid && (m_fin == -INFINITY)) l = x0.y + x1.y;
      const bool direct = e.splits_r == 1;
      long long dst[4];  // of the vectors this lane stores (8 s + lane / 4, 16 bytes each)
#pragma unroll
      for (int s = 0; s < 4; ++s) {
        const int gi = q4 * 32 + 8 * s + (lane >> 2);
        dst[s] = -1;
        if (gi < e.nv) {
          const int gv = e.vbase + gi;
          const int n = e.n0 + gv / g, h = e.kh * g + gv % g;
          dst[s] = (long long)(size_t(direct ? n : e.split * (long long)a.N + n) * a.Hq + h) * DH;
        }
      }
      if (valid && a.splits > 1 && grp == 0) {
        // as the bf16 kernel leaves them for the combine
        const int gv = e.vbase + i;
        const size_t at = size_t(e.n0 + gv / g) * a.Hq + e.kh * g + gv % g;
        const size_t step = size_t(a.N) * a.Hq;
        a.ml_part[at + (direct ? 0 : e.split * step)] =
            direct ? make_float2(0.f, -1.f) : make_float2(m_fin, l);
        if (!direct && e.split == e.splits_r - 1)
          for (int sp = e.splits_r; sp < a.splits; ++sp)
            a.ml_part[at + sp * step] = make_float2(-INFINITY, 0.f);
      }
      const float inv = l > 0.f ? 1.f / l : 0.f;
      if (!warp_mbar_wait(sh.pv_done + Tl % NS, (Tl / NS) & 1, a.wait_ns, abort_flag)) {
        ok = false;
        break;
      }
      tc_fence_after();
      if (some) {
        const bool bad = e.nct > 0 && (sh.bad[slot][0] | sh.bad[slot][1] | sh.bad[slot][2] |
                                       sh.bad[slot][3]) != 0;
        // 64 bytes of each vector at a time through this warp's 2 KB stage: four 16-byte
        // pieces a row, rotated so that eight lanes meet different banks
        auto put = [&](const uint4(&x)[4], char* base, size_t esize, int col) {
#pragma unroll
          for (int q = 0; q < 4; ++q) stage[lane * 4 + (q ^ ((lane >> 1) & 3))] = x[q];
          __syncwarp();
#pragma unroll
          for (int s = 0; s < 4; ++s) {
            const int iv = 8 * s + (lane >> 2), c = lane & 3;
            const uint4 val = stage[iv * 4 + (c ^ ((iv >> 1) & 3))];
            if (dst[s] >= 0)
              *reinterpret_cast<uint4*>(base + (dst[s] + col) * esize + c * 16) = val;
          }
          __syncwarp();
        };
        // each group writes half of the columns
#pragma unroll 1
        for (int c0 = grp * (DH / 2); c0 < (grp + 1) * (DH / 2); c0 += 32) {
          float ov[32];
          tmem_ld_32cols(tmem + lane_off + c0, ov);
          tmem_wait_ld();
          if (bad) {  // the non-finite values of the tokens this row sees
            for (int f = max(fa, e.f_begin); f <= fb; ++f) {
              const __nv_bfloat16* v = a.v_cand + (size_t(f) * a.Hkv + e.kh) * DH + c0;
#pragma unroll
              for (int c = 0; c < 32; ++c) {
                const float x = __bfloat162float(v[c]);
                if (!isfinite(x)) ov[c] += x;
              }
            }
          }
          if (direct) {
            uint4 x[4];
#pragma unroll
            for (int q = 0; q < 4; ++q) {
              const float* y = ov + 8 * q;
              x[q] = make_uint4(pack_bf16(y[0] * inv, y[1] * inv), pack_bf16(y[2] * inv, y[3] * inv),
                                pack_bf16(y[4] * inv, y[5] * inv), pack_bf16(y[6] * inv, y[7] * inv));
            }
            put(x, reinterpret_cast<char*>(a.o), 2, c0);
          } else {
#pragma unroll
            for (int k = 0; k < 2; ++k) {
              uint4 x[4];
#pragma unroll
              for (int q = 0; q < 4; ++q) {
                const float* y = ov + 16 * k + 4 * q;
                x[q] = make_uint4(__float_as_uint(y[0]), __float_as_uint(y[1]),
                                  __float_as_uint(y[2]), __float_as_uint(y[3]));
              }
              put(x, reinterpret_cast<char*>(a.o_part), 4, c0 + 16 * k);
            }
          }
        }
      }
      // O may be overwritten by the next item's first P V; the ring slot is free
      tc_fence_before();
      __syncwarp();
      if (lane == 0) {
        mbar_arrive(&sh.o_free);
        mbar_arrive(sh.item_empty + slot);
      }
      T += e.ntiles;
    }
    if (!ok) {
      sh.abort = 1;
      flag(a.status, JET_ERR_TIMEOUT);
    }
  }

  tc_fence_before();
  __syncthreads();
  if (warp == kMmaWarp) {
    tc_fence_after();
    tmem_dealloc(tmem, G::kTmemCols);
  }
}

// codes [keys, heads, DH]: box of box_d codes x 1 head x kBN keys
bool encode_codes(CUtensorMap* map, const void* base, int rows, int heads, int DH, int box_d,
                  CUtensorMapSwizzle swizzle) {
  auto fn = encode_fn();
  if (!fn) return false;
  const cuuint64_t dims[3] = {cuuint64_t(DH), cuuint64_t(heads), cuuint64_t(rows)};
  const cuuint64_t strides[2] = {cuuint64_t(DH), cuuint64_t(heads) * DH};
  const cuuint32_t box[3] = {cuuint32_t(box_d), 1, cuuint32_t(kBN)};
  const cuuint32_t estr[3] = {1, 1, 1};
  return fn(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 3, const_cast<void*>(base), dims, strides, box,
            estr, CU_TENSOR_MAP_INTERLEAVE_NONE, swizzle, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
            CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <int DH>
cudaError_t launch_dh(const jet_layout& lay, const jet_dims& d, const AttnPlan& plan,
                      const void* q, const void* k8, const void* v8, const void* k_cand,
                      const void* v_cand, void* o, void* ws, int* status, cudaStream_t st) {
  const jet_sizes& n = lay.n;
  const int F = n.N - n.R;
  const int g = d.Hq / d.Hkv;
  if (g > kBV) return cudaErrorInvalidValue;
  CUtensorMap tmQ, tmK, tmV, tmKc, tmVc;
  if (!encode_3d(&tmQ, q, n.N, d.Hq, DH, g, kBV / g) ||
      !encode_codes(&tmK, k8, n.total_prefix, d.Hkv, DH, std::min(DH, 128),
                    DH == 64 ? CU_TENSOR_MAP_SWIZZLE_64B : CU_TENSOR_MAP_SWIZZLE_128B) ||
      !encode_codes(&tmV, v8, n.total_prefix, d.Hkv, DH, DH, CU_TENSOR_MAP_SWIZZLE_NONE))
    return cudaErrorInvalidValue;
  if (F > 0) {
    if (!encode_3d(&tmKc, k_cand, F, d.Hkv, DH, 1, kBC) ||
        !encode_3d(&tmVc, v_cand, F, d.Hkv, DH, 1, kBC))
      return cudaErrorInvalidValue;
  } else {
    tmKc = tmK;  // never read: no request has candidate tiles
    tmVc = tmV;
  }
  const size_t vecs = size_t(plan.splits) * n.N * d.Hq;
  const size_t exp_off = kv_size(n, d).exp_off;
  Kv8Args a{};
  a.wait_ns = wait_budget_ns();
  a.hold_first = test_stall();
  a.prefix_offset = lay.prefix_offset;
  a.row_offset = lay.row_offset;
  a.req_order = lay.req_order;
  a.row_cand = lay.row_cand;
  a.cand_row_offset = lay.cand_row_offset;
  a.o = static_cast<__nv_bfloat16*>(o);
  a.o_part = static_cast<float*>(ws);
  a.ml_part = reinterpret_cast<float2*>(a.o_part + vecs * DH);
  a.status = status;
  a.R = n.R;
  a.N = n.N;
  a.C = n.C;
  a.total_prefix = n.total_prefix;
  a.Hq = d.Hq;
  a.Hkv = d.Hkv;
  a.chunk = plan.chunk;
  a.g = g;
  a.rb = kBV / g;
  a.has_cand = F > 0;
  a.scale_log2 = 1.4426950408889634f / sqrtf(float(DH));
  a.k_exp = static_cast<const uint8_t*>(k8) + exp_off;
  a.v_exp = static_cast<const uint8_t*>(v8) + exp_off;
  a.v_cand = static_cast<const __nv_bfloat16*>(v_cand);
  // the work list follows the (m, l) partials in the workspace
  uintptr_t ctrl = reinterpret_cast<uintptr_t>(a.ml_part + vecs);
  ctrl = (ctrl + 15) & ~uintptr_t(15);
  a.item_next = reinterpret_cast<int*>(ctrl);
  a.item_count = a.item_next + 1;
  a.items = reinterpret_cast<int4*>(ctrl + 16);
  a.splits = plan.splits;
  a.qgroups = plan.qgroups;
  a.n_all = (long long)n.R * d.Hkv * plan.qgroups * plan.splits;
  a.sorted = plan.sorted;
  const int sms = sm_count();
  if (sms < 1) return cudaErrorInvalidValue;
  const int grid = int(std::max<long long>(1, std::min<long long>(sms, a.n_all)));
  cudaError_t e = cudaSuccess;
  if (a.sorted)
    e = launch_pdl(attend_items_kernel, dim3(1), dim3(1024), 0, st, static_cast<const AttArgs&>(a),
                   plan.qgroups, plan.splits);
  if (e != cudaSuccess) return e;
  const size_t smem = Geo<DH>::kBytes + 1024;
  e = cudaFuncSetAttribute(attend_kv8_kernel<DH>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                           int(smem));
  if (e != cudaSuccess) return e;
  e = launch_pdl(attend_kv8_kernel<DH>, dim3(grid), dim3(kThreads), smem, st, tmQ, tmK, tmV, tmKc,
                 tmVc, a);
  if (e != cudaSuccess || plan.splits <= 1) return e;
  const long long blocks = ((long long)n.N * d.Hq + 3) / 4;
  return launch_pdl(attend_combine_kernel<DH>, dim3(unsigned(blocks)), dim3(128), 0, st,
                    lay.row_req, n.N, n.R, d.Hq, plan.splits, blocks <= 8LL * sms, a.o_part,
                    a.ml_part, a.o, status);
}

}  // namespace

cudaError_t launch_attend_kv8_tc(const jet_layout& lay, const jet_dims& d, const AttnPlan& plan,
                                 const void* q, const void* k8, const void* v8,
                                 const void* k_cand, const void* v_cand, void* o, void* ws,
                                 int* status, cudaStream_t st) {
#define JET_KV8(DH) \
  return launch_dh<DH>(lay, d, plan, q, k8, v8, k_cand, v_cand, o, ws, status, st)
  if (d.d == 64) JET_KV8(64);
  if (d.d == 128) JET_KV8(128);
  if (d.d == 256) JET_KV8(256);
#undef JET_KV8
  return cudaErrorInvalidValue;
}

}  // namespace jet
