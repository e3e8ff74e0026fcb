// Cascade attention over an 8-bit prefix cache on the 5th-generation tensor cores
// (Sec. 4.1; bf16 queries, candidates' keys and values, and outputs; f32 accumulation).
//
// As in attend_tc.cu a CTA owns one (request r, key/value head kh, prefix chunk, block of
// up to 128 query vectors), streams the chunk's tiles of 64 or 128 keys once for all of them and
// leaves a partial that the combine merges, or the output where the request is one
// chunk. A cache tile is half the bytes of a bf16 one, so at the HBM rate an SM has half
// the time for it (d 256: 32 KB, 0.73 us): what follows keeps each unit below that.
//
//   scores   S = Q K^T on the codes as they are (kind::f8f6f4). A query is held as two
//            e4m3 numbers, q = 2^x (hi + lo), x per row: hi is the nearest code, lo that of
//            what is left, at most four binary digits of a bf16 number's eight, so the
//            split is exact for elements of 2^-2 of 2^x or more, 2^-9.8 of the row's
//            largest, and leaves 2^-10 of 2^x, at most 2^-17.8 of that largest, below. (Keys
//            widened to bf16 instead would pass shared memory twice more: 1,536 cycles
//            a tile of d 256, 1,393 at the HBM rate.) S = acc 2^(x + X), X the exponent
//            of the 64 tokens: a tile has one or two.
//   outputs  O += P V with P in f16, as weights 2^(s - m + 7) <= 2^15 (f16 keeps eleven
//            digits down to 2^-14, so weights 2^-21 of a maximum's, and rounds
//            at 2^-25 below; e4m3 would lose the many small weights next to a large
//            one), and V widened from the codes to f16 in units of 2^vx, the item's
//            largest exponent, by eight warps on the way: exact but for values below
//            2^-14 of that unit, which are rounded at 2^-25 of it. (A block whose scale
//            is out of f16's range in that unit, 2^-25 or less, takes it in two factors.)
//
//   warp 0       TMA producer: rings of K tiles, of V tiles, and the query block
//   warp 1       TMEM allocator, issues S_j = Q K_j^T
//   warp 2       scheduler: work items one ahead
//   warp 3       issues O += P_j V_j
//   warps 4..11  softmax: two threads a query vector (TMEM lane), each with half of a
//                tile's columns; they exchange their maxima through shared memory. P_j
//                overwrites S_j in TMEM.
//   warps 12..19 per item the queries' split into TMEM, per tile V to f16. Values of
//                keys past the chunk (other requests') become zeros there.
// The candidates' own tokens come first in a request's last chunk, in tiles of half the
// keys in bf16 (the same bytes as a cache tile) against the bf16 queries; their values
// pass the widening warps too. Values that are not finite, or so large that V's unit
// would take the prefix's digits with it, are left out there, as a weight of zero would
// not keep them from the rows that do not see them; the output adds such an item's
// candidate tokens one by one, each to the rows that do (16 multiple-choice requests whose
// last chunks hold zeros, so that all take this way: 112 us instead of 27).
//
// What bounds it: long prefixes, at 60 % of the copy rate, the units of an SM in turn (256
// requests of 2,048 - 8,192 tokens, d 256, two kv heads: 344 us; 128 of them at d 128, eight
// kv heads: 354 us). Of the some 1,600 cycles of a d 256 tile, whose bytes take 1,393, the
// tensor pipe is busy for 1,024 (two passes over the keys, one over the values), and the
// softmax and widening warps fill half of the issue slots, where a conversion or an
// exponential holds its unit for two to four cycles. At one query row a request the copies
// below leave the widening of V (64 requests of 1,000 - 6,000, d 128: 108 us, 66 %). Small
// calls take an item's way through all roles, some 30,000 cycles or 16 us: the schedule
// (3,800), the queries' arrival (5,900) and split (3,900), the tiles, the output (2,400).
// (Softmax warps that take whole tiles in turn, instead of half of each tile's columns,
// need no exchange of maxima but hold an S buffer twice as long: 406 us instead of 352.)
//
// With R copies a block of 128 / R vectors stands R times in the TMEM lanes, and copy c's
// softmax warps take columns c of R of their half's, with zeros for the others' in P: a
// partial each.
#include <algorithm>
#include <climits>
#include <cmath>

#include "attend_tc.cuh"
#include "kv_cache.h"

namespace jet {
namespace {

constexpr float kWeightLog2 = 7.f;  // weights are 2^7 at a row's maximum
constexpr int kThreads = 640;
constexpr int kProdWarp = 0, kMmaWarp = 1, kSchedWarp = 2, kPvWarp = 3, kSoftWarp = 4;
constexpr int kWideWarp = 12;
constexpr int kWideThreads = kThreads - 32 * kWideWarp;

template <int DH>
struct Geo {
  // A tile of 64 keys for d 256, where O, two S and the queries' codes leave TMEM room for
  // no more; else of 128, so that half as many steps of the pipeline carry the same
  // bytes (d 128, long prefixes: 415 us instead of 487 before other steps)
  static constexpr int kT = DH == 256 ? 64 : 128;
  static constexpr int kHalf = kT / 2;                    // columns of a softmax warp
  static constexpr int kC = kT / 2;                       // candidate tokens per tile
  static constexpr uint32_t kTile = kT * DH;              // bytes of a K or V tile
  static constexpr int kS = DH == 64 ? 3 : 2;             // S buffers
  static constexpr int kK = DH == 256 ? 2 : DH == 128 ? 3 : 4;  // K tiles in flight
  static constexpr int kV = DH == 256 ? 2 : DH == 128 ? 3 : 6;  // V tiles in flight
  static constexpr int kW = 2;                            // widened V tiles
  static constexpr uint32_t kOffK = kBV * DH * 2;         // after the bf16 query block
  static constexpr uint32_t kOffV = kOffK + kK * kTile;
  static constexpr uint32_t kOffW = kOffV + kV * kTile;
  static constexpr uint32_t kOffStage = kOffW + kW * 2 * kTile;  // 2 KB per softmax warp
  static constexpr uint32_t kOffSmall = kOffStage + 8 * 2048;
  static constexpr uint32_t kBytes = kOffSmall + 9216;
  // TMEM: O, the S buffers (P in place of S), the queries' hi and lo codes
  static constexpr uint32_t kTmemCols = 512;
  static constexpr uint32_t kSCol = DH;
  static constexpr uint32_t kQCol = kSCol + kS * kT;
  static_assert(kQCol + DH / 2 <= kTmemCols, "TMEM columns");
  static_assert(kBytes + 1024 <= 232448, "shared memory");
};

struct Kv8Args : AttArgs {
  const uint8_t* k_exp;  // exponent bytes of the caches
  const uint8_t* v_exp;
  const __nv_bfloat16* k_cand;
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
  uint64_t w_full[2];                    // widened V tiles
  uint64_t s_full[4], p_full[4], pv_done[4];
  uint64_t m_full[2][4];                 // both halves' maxima of an even / odd tile
  uint64_t l_full[4];                    // both groups' sums of an item
  uint64_t aux_full[2];                  // sees, vx of an item
  uint64_t a_full[4];                    // both halves' maxima of the queries
  uint64_t item_full[2], item_empty[2];
  uint64_t q_full, q_free;               // the bf16 query block
  uint64_t qt_full, qt_free;             // the queries' codes in TMEM
  uint64_t qx_read;                      // their exponents are in the softmax's registers
  uint64_t o_free;                       // an item's O is out of TMEM
  uint64_t drain[2];
  uint32_t tmem;
  volatile int abort;
  float m[2][2][kBV];                    // [tile parity][half] maxima
  float l[2][2][kBV];                    // [item parity][half] sums
  int qx[2][kBV];                        // [item parity] the queries' exponents
  int vx[2];                             // [item parity] the chunk's largest exponent of V
  uint32_t vtop[2];                      // [item parity] the candidates' largest value's bits
  uint32_t qmax[2][kBV];                 // [half] largest magnitudes of the queries
  int2 sees[2][kBV];                     // [item parity] the fed tokens a vector sees, from
                                         // f_begin on: first, end
};
static_assert(sizeof(Small) <= 9216, "the small part of shared memory");

// The bounded waits of this kernel, in few instructions: two dozen of them stand between
// the roles' working code, which the instruction caches barely hold. (try_wait itself
// sleeps for a while, so the clock is read seldom enough.)
__device__ __forceinline__ bool poll(uint64_t* bar, uint32_t parity, uint64_t budget_ns,
                                     volatile int* abort) {
  const uint64_t t0 = global_timer_ns();
#pragma unroll 1
  while (!mbar_try_wait(bar, parity))
    if (*abort || global_timer_ns() - t0 > budget_ns) return false;
  return true;
}
__device__ __forceinline__ bool wait1(uint64_t* bar, uint32_t parity, uint64_t budget_ns,
                                      volatile int* abort) {
  return mbar_try_wait(bar, parity) || poll(bar, parity, budget_ns, abort);
}
// by every lane of a warp, with one outcome for the whole warp
__device__ __forceinline__ bool wait32(uint64_t* bar, uint32_t parity, uint64_t budget_ns,
                                       volatile int* abort) {
  if (__all_sync(0xffffffffu, mbar_try_wait(bar, parity))) return true;
  return __all_sync(0xffffffffu, poll(bar, parity, budget_ns, abort));
}

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

// and 8 columns
__device__ __forceinline__ void tmem_st_8cols_u32(uint32_t taddr, const uint32_t (&v)[8]) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"r"(taddr),
      "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7])
      : "memory");
}

template <int N>
__device__ __forceinline__ void tmem_st_cols(uint32_t taddr, const uint32_t (&v)[N]) {
  static_assert(N == 16 || N == 8);
  if constexpr (N == 16) tmem_st_16cols_u32(taddr, v);
  if constexpr (N == 8) tmem_st_8cols_u32(taddr, v);
}

template <int N>
__device__ __forceinline__ void tmem_ld_cols(uint32_t taddr, float (&v)[N]) {
  static_assert(N == 64 || N == 32 || N == 16);
  if constexpr (N == 64) {
    tmem_ld_32cols(taddr, *reinterpret_cast<float(*)[32]>(v));
    tmem_ld_32cols(taddr + 32, *reinterpret_cast<float(*)[32]>(v + 32));
  }
  if constexpr (N == 32) tmem_ld_32cols(taddr, v);
  if constexpr (N == 16) tmem_ld_16cols(taddr, v);
}

// the codes of a word's two halves as f16 numbers, and two f16 numbers' nearest codes
__device__ __forceinline__ void e4m3x4_to_f16x4(uint32_t codes, uint32_t& lo, uint32_t& hi) {
  asm("{\n\t.reg .b16 a, b;\n\tmov.b32 {a, b}, %2;\n\t"
      "cvt.rn.f16x2.e4m3x2 %0, a;\n\tcvt.rn.f16x2.e4m3x2 %1, b;\n\t}"
      : "=r"(lo), "=r"(hi)
      : "r"(codes));
}
__device__ __forceinline__ uint32_t f16x4_to_e4m3x4(uint32_t lo, uint32_t hi) {
  uint32_t d;
  asm("{\n\t.reg .b16 a, b;\n\t"
      "cvt.rn.satfinite.e4m3x2.f16x2 a, %1;\n\tcvt.rn.satfinite.e4m3x2.f16x2 b, %2;\n\t"
      "mov.b32 %0, {a, b};\n\t}"
      : "=r"(d)
      : "r"(lo), "r"(hi));
  return d;
}

__device__ __forceinline__ uint32_t sub_f16x2(uint32_t a, uint32_t b) {
  uint32_t d;
  asm("sub.rn.f16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
  return d;
}

__device__ __forceinline__ uint32_t mul_f16x2(uint32_t a, uint32_t b) {
  uint32_t d;
  asm("mul.rn.f16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
  return d;
}

// 2^k twice, k in [-24, 15]
__device__ __forceinline__ uint32_t pow2_f16x2(int k) {
  const uint32_t h = k > -15 ? uint32_t(k + 15) << 10 : 1u << (k + 24);
  return h | h << 16;
}

__device__ __forceinline__ uint32_t pack_f16(float a, float b) {
  uint32_t d;
  asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(d) : "f"(b), "f"(a));
  return d;
}

// f16 A and B (format 0), f32 accumulator; B is MN-major
constexpr uint32_t idesc_f16_f32_mn(int M, int N) {
  return (1u << 4) | (1u << 16) | (uint32_t(N >> 3) << 17) | (uint32_t(M >> 4) << 24);
}

// where a V tile's TMA copy leaves the 16 codes c of a key: slices of 128 codes under
// 128-byte swizzling, d 64 rows of 64 bytes under 64-byte swizzling
template <int DH, int KT>
__device__ __forceinline__ uint32_t raw_piece(int key, int c) {
  if constexpr (DH == 64) return uint32_t(key) * 64u + (uint32_t(c ^ ((key >> 1) & 3)) << 4);
  return uint32_t(c >> 3) * (KT * 128) + sw128(key, c & 7);
}

// An exponent byte, asked for a tile ahead of its use: the compiler is not to touch the
// register in between, as that would wait for the load (1,000 cycles a tile of d 128)
__device__ __forceinline__ uint32_t load_ahead(const uint8_t* p) {
  uint32_t v;
  asm volatile("ld.global.nc.u8 %0, [%1];" : "=r"(v) : "l"(p));
  return v;
}
__device__ __forceinline__ int exponent_of(uint32_t byte) {
  asm volatile("" : "+r"(byte));
  return min(max(int(byte) - 127, kKvLow), kKvHigh);
}

// two float32 at a time
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

// The bits of the largest magnitude of the candidate values at tokens [f, f + n), by a
// warp (of several that step together): the largest that it meets
template <int DH>
__device__ __forceinline__ uint32_t cand_top(const Kv8Args& a, int kh, int f, int n, int first,
                                             int step) {
  const __nv_bfloat16* v = a.v_cand + (size_t(f) * a.Hkv + kh) * DH;
  uint32_t top = 0;  // two magnitudes
#pragma unroll 8
  for (int i = first; i < n * (DH / 8); i += step) {
    const uint4 x = *reinterpret_cast<const uint4*>(v + size_t(i / (DH / 8)) * a.Hkv * DH +
                                                    8 * (i % (DH / 8)));
    top = __vmaxu2(__vmaxu2(top, x.x & 0x7fff7fffu), x.y & 0x7fff7fffu);
    top = __vmaxu2(__vmaxu2(top, x.z & 0x7fff7fffu), x.w & 0x7fff7fffu);
  }
  return __reduce_max_sync(0xffffffffu, max(top & 0xffff0000u, top << 16));
}

// The unit of V and O of an item, from its chunk's largest exponent byte and its
// candidates' largest magnitude, and whether the candidates' values stay out of P V: every
// row of the block sees the chunk's keys, but not every candidate, so values that would
// cost the others digits (f16 has room for 2^8 of the prefix's largest), or are not
// finite, do.
__device__ __forceinline__ int2 value_unit(int vx, uint32_t top) {
  const int cx = top ? kv_exponent(top) + 127 : 0;
  const int apart = top >= 0x7f800000u || cx > vx + 8;
  return make_int2(min(max((apart ? vx : max(vx, cx)) - 127, kKvLow), kKvHigh), apart);
}

template <int DH, int R>
__global__ void __launch_bounds__(kThreads, 1)
attend_kv8_kernel(const __grid_constant__ CUtensorMap tmQ, const __grid_constant__ CUtensorMap tmK,
                  const __grid_constant__ CUtensorMap tmV, const __grid_constant__ CUtensorMap tmKc,
                  const __grid_constant__ CUtensorMap tmVc, const Kv8Args a) {
  using G = Geo<DH>;
  constexpr int NK = G::kK, NV = G::kV, NW = G::kW, NS = G::kS, KT = G::kT, KC = G::kC;
  constexpr int RV = kBV / R;  // vectors of an item; R copies of them fill the lanes
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
      mbar_init(sh.v_empty + s, 8);
    }
    for (int s = 0; s < NW; ++s) mbar_init(sh.w_full + s, 8);
    for (int b = 0; b < NS; ++b) {
      mbar_init(sh.s_full + b, 1);
      mbar_init(sh.p_full + b, 8);
      mbar_init(sh.pv_done + b, 1);
    }
    for (int q = 0; q < 4; ++q) {
      mbar_init(&sh.m_full[0][q], 2);
      mbar_init(&sh.m_full[1][q], 2);
      mbar_init(sh.l_full + q, 2);
      mbar_init(sh.a_full + q, 2);
    }
    for (int b = 0; b < 2; ++b) {
      mbar_init(sh.item_full + b, 1);
      mbar_init(sh.aux_full + b, 9);     // the scheduler, 8 widening warps
      mbar_init(sh.item_empty + b, 19);  // producer, two MMA threads, 8 softmax, 8 widening warps
    }
    mbar_init(&sh.q_full, 1);
    mbar_init(&sh.q_free, 9);  // the split's eight warps, the last product with it
    mbar_init(&sh.qt_full, 8);
    mbar_init(&sh.qt_free, 1);
    mbar_init(&sh.qx_read, 8);
    mbar_init(&sh.o_free, 8);
    mbar_init(sh.drain, 1);
    mbar_init(sh.drain + 1, 1);
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
  // registers to the softmax warps, which hold a tile's scores: 80 + 2 x 112 + 2 x 88 are
  // the five warpgroups' launch share of 96 each
  if (warp < kSoftWarp) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 80;");
    if (warp == kSchedWarp) {
      // ---------------------------------------------------------------- scheduler
      ItemWindow window{};
      for (int u = 0;; ++u) {
        const int slot = u & 1;
        if (!wait32(sh.item_empty + slot, ((u >> 1) & 1) ^ 1u, a.wait_ns, abort_flag)) {
          if (lane == 0) {
            sh.abort = 1;
            flag(a.status, JET_ERR_TIMEOUT);
          }
          break;
        }
        ItemGeo e{};
        bool live = false;
        // dealt out back and forth, as the bf16 kernel does
        const int n = int(gridDim.x);
        const int k = u * n + ((u & 1) ? n - 1 - int(blockIdx.x) : int(blockIdx.x));
        int4 it;
        if (k < a.n_all && nth_item(a, k, lane, window, &it, &e)) {
          live = e.ok;
          if (!live && lane == 0) flag(a.status, JET_ERR_DEVICE);
        }
        int fed = 0;
        if (lane == 0) {
          if (live) {
            if (e.nct > 0) {
              // the fed tokens that a row of this block sees: up to its last row's own,
              // from the first of its first row's candidate on
              fed = e.row0 + e.nv / g - 1;
              int lo = 0;
              if (fed > KC && e.row0 > 0) {
                const int c = a.row_cand[e.n0 + e.row0];
                if (c >= 0 && c < a.C)
                  lo = min(max(a.cand_row_offset[c] - e.n0 - 1, 0), fed);
              }
              e.f_begin += lo;
              fed -= lo;
              if (!fed_inside(a, e.f_begin, fed)) {
                flag(a.status, JET_ERR_DEVICE);
                fed = 0;  // the block's rows get the prefix alone
              }
            }
            e.nct = (fed + KC - 1) / KC;
            e.npt = (e.k_end - e.k_begin + KT - 1) / KT;
            e.ntiles = e.npt + e.nct;
          }
          sh.ring[slot].e = e;
          sh.ring[slot].fed = fed;
          sh.ring[slot].live = live;
          sh.vtop[slot] = 0;
          mbar_arrive(sh.item_full + slot);
          if (live) {  // the query block on its way into L2
  #pragma unroll
            for (int sl = 0; sl < DH / 64; ++sl)
              tma_prefetch_3d(&tmQ, sl * 64, e.kh * g, e.n0 + e.row0);
          }
        }
        if (!__shfl_sync(0xffffffffu, live ? 1 : 0, 0)) break;
        // What the other warps need a little later, and would wait for memory to know: the
        // fed tokens that each vector sees, and V's unit, the largest exponent of the
        // item's blocks and of its candidates' values
        {
          __syncwarp();
          const ItemGeo& it = sh.ring[slot].e;
          fed = __shfl_sync(0xffffffffu, fed, 0);
          const int f_begin = it.f_begin;
          const int blocks = (it.k_end - it.k_begin + kKvBlock - 1) / kKvBlock;
          if (fed > 0) {
            for (int row = lane; row < it.nv / g; row += 32) {
              const int n = it.n0 + it.row0 + row;
              const int c = a.row_cand[n];
              int from = 0, end = 0;  // none: shared row
              if (c >= 0 && c < a.C) {
                from = min(max(a.cand_row_offset[c] - it.r - 1 - f_begin, 0), fed);  // y_{c,1}
                end = min(n - it.r - f_begin, fed);  // past the row's own fed token
              }
              for (int i = 0; i < g; ++i) sh.sees[slot][row * g + i] = make_int2(from, end);
            }
          }
          const uint8_t* ex =
              a.v_exp + size_t(kv_place(it.p0, it.r, it.k_begin / kKvBlock)) * a.Hkv + it.kh;
          int vx = kKvLow + 127;
          for (int b = lane; b < blocks; b += 32) vx = max(vx, int(ex[size_t(b) * a.Hkv]));
          vx = __reduce_max_sync(0xffffffffu, vx);
          // (the first item's candidates are looked over by the widening warps, which have
          // nothing else to do yet)
          if (u > 0) {
            const uint32_t top = cand_top<DH>(a, it.kh, f_begin, fed, lane, 32);
            if (lane == 0) sh.vtop[slot] = top;
          }
          if (lane == 0) sh.vx[slot] = vx;
          __syncwarp();
          if (lane == 0) mbar_arrive(sh.aux_full + slot);
        }
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
          if (!wait1(sh.item_full + slot, (u >> 1) & 1, a.wait_ns, abort_flag)) {
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
                mbar_arrive_expect_tx(&sh.q_full, uint32_t(R * (DH / 64)) * 64 * 2 * g * rb);
  #pragma unroll
                for (int c = 0; c < R; ++c)
  #pragma unroll
                  for (int sl = 0; sl < DH / 64; ++sl)
                    tma_load_3d(smem + sl * (kBV * 128) + c * RV * 128, &tmQ, &sh.q_full, sl * 64,
                                e.kh * g, e.n0 + e.row0, pol);
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
                    tma_load_3d(ks + sl * (KC * 128), &tmKc, sh.k_full + s, sl * 64, e.kh,
                                e.f_begin + jk * KC, pol);
                } else {
                  const int key = e.p0 + e.k_begin + (jk - e.nct) * KT;
  #pragma unroll
                  for (int sl = 0; sl < (DH + 127) / 128; ++sl)
                    tma_load_3d(ks + sl * (KT * 128), &tmK, sh.k_full + s, sl * 128, e.kh, key,
                                pol);
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
                    tma_load_3d(vs + sl * (KC * 128), &tmVc, sh.v_full + s, sl * 64, e.kh,
                                e.f_begin + jv * KC, pol);
                } else {
                  const int key = e.p0 + e.k_begin + (jv - e.nct) * KT;
  #pragma unroll
                  for (int sl = 0; sl < (DH + 127) / 128; ++sl)
                    tma_load_3d(vs + sl * (KT * 128), &tmV, sh.v_full + s, sl * 128, e.kh, key,
                                pol);
                }
                v_issued |= 1u << s;
                v_par = (v_par & ~(1u << s)) | (ph << s);
                ++jv;
                progressed = true;
              }
            }
            if (!progressed) __nanosleep(100);
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
        }
        // let every copy issued land before the CTA can exit (where no wait ran out they are
        // used by now)
        if (q_issued) mbar_wait(&sh.q_full, q_par, kDrainNs, nullptr);
        for (int t = 0; t < NK; ++t)
          if (k_issued & (1u << t)) mbar_wait(sh.k_full + t, (k_par >> t) & 1u, kDrainNs, nullptr);
        for (int t = 0; t < NV; ++t)
          if (v_issued & (1u << t)) mbar_wait(sh.v_full + t, (v_par >> t) & 1u, kDrainNs, nullptr);
      }
    } else if (warp == kMmaWarp) {
      // ---------------------------------------------------------------- scores
      if (elect_one()) {
        constexpr uint32_t id_s = idesc_e4m3_f32(kBV, KT);
        constexpr uint32_t id_c = idesc_bf16_f32(kBV, KC);
        const uint64_t q0 = desc_k_sw128(smem_u32(smem));
        const uint64_t kc0 = desc_k_sw128(smem_u32(smem + G::kOffK));
        const uint64_t k0 = DH == 64 ? desc_k_sw64(smem_u32(smem + G::kOffK)) : kc0;
        auto wait = [&](uint64_t* bar, uint32_t parity) {
          return wait1(bar, parity, a.wait_ns, abort_flag);
        };
        bool ok = true;
        int T = 0;
        for (int u = 0; ok; ++u) {
          const int slot = u & 1;
          ok = wait(sh.item_full + slot, (u >> 1) & 1);
          if (!ok || !sh.ring[slot].live) break;
          const int nct = sh.ring[slot].e.nct, ntiles = sh.ring[slot].e.ntiles;
          if (nct == 0) mbar_arrive(&sh.q_free);  // only the split reads the bf16 block
          for (int j = 0; j < ntiles; ++j) {
            const int Tj = T + j, b = Tj % NS, kb = Tj % NK;
            ok = (j > 0 && j != nct) || wait(j < nct ? &sh.q_full : &sh.qt_full, u & 1);
            ok = ok && wait(sh.k_full + kb, (Tj / NK) & 1) &&
                 wait(sh.pv_done + b, ((Tj / NS) & 1) ^ 1u);
            if (!ok) break;
            tc_fence_after();
            const uint32_t d = tmem + G::kSCol + b * KT;
            // (a descriptor of another address: its low field counts 16 bytes)
            if (j < nct) {
              const uint64_t kd = kc0 + kb * (G::kTile >> 4);
  #pragma unroll
              for (int st = 0; st < DH / 16; ++st) {
                const int sl = st >> 2, k = st & 3;
                mma_f16(d, q0 + ((sl * (kBV * 128) + 32 * k) >> 4),
                        kd + ((sl * (KC * 128) + 32 * k) >> 4), id_c, st != 0);
              }
              if (j == nct - 1) mma_commit(&sh.q_free);
            } else {
              const uint64_t kd = k0 + kb * (G::kTile >> 4);
  #pragma unroll
              for (int st = 0; st < DH / 16; ++st) {  // hi, then lo, over the same keys
                const int kk = st % (DH / 32);
                mma_e4m3_ta(d, tmem + G::kQCol + uint32_t(8 * st),
                            kd + (((kk >> 2) * (KT * 128) + 32 * (kk & 3)) >> 4), id_s, st != 0);
              }
            }
            mma_commit(sh.s_full + b);
            mma_commit(sh.k_empty + kb);
            if (j == ntiles - 1) mma_commit(&sh.qt_free);
          }
          if (!ok) break;
          mbar_arrive(sh.item_empty + slot);
          T += ntiles;
        }
        if (!ok) {
          sh.abort = 1;
          flag(a.status, JET_ERR_TIMEOUT);
        }
        mma_commit(sh.drain);  // nor may its products outlive it
        mbar_wait(sh.drain, 0, kDrainNs, nullptr);
      }
    } else if (warp == kPvWarp) {
      // ---------------------------------------------------------------- outputs
      if (elect_one()) {
        constexpr uint32_t id_o = idesc_f16_f32_mn(kBV, DH);
        const uint64_t v0 = desc_mn_sw128(smem_u32(smem + G::kOffW), KT * 128);
        const uint64_t vc0 = desc_mn_sw128(smem_u32(smem + G::kOffW), KC * 128);
        auto wait = [&](uint64_t* bar, uint32_t parity) {
          return wait1(bar, parity, a.wait_ns, abort_flag);
        };
        bool ok = true;
        int T = 0;
        for (int u = 0; ok; ++u) {
          const int slot = u & 1;
          ok = wait(sh.item_full + slot, (u >> 1) & 1);
          if (!ok || !sh.ring[slot].live) break;
          const int nct = sh.ring[slot].e.nct, ntiles = sh.ring[slot].e.ntiles;
          for (int j = 0; j < ntiles; ++j) {
            const int Tj = T + j, b = Tj % NS, w = Tj % NW;
            // the item's first P V overwrites O: the previous item's O must be out
            ok = j > 0 || u == 0 || wait(&sh.o_free, (u - 1) & 1);
            ok = ok && wait(sh.w_full + w, (Tj / NW) & 1) && wait(sh.p_full + b, (Tj / NS) & 1);
            if (!ok) break;
            tc_fence_after();
            const uint32_t pt = tmem + G::kSCol + b * KT;
            const uint64_t vd = (j < nct ? vc0 : v0) + w * (2 * G::kTile >> 4);
  #pragma unroll
            for (int k = 0; k < KC / 16; ++k)
              mma_f16_ta(tmem, pt + uint32_t(8 * k), vd + (k * 2048 >> 4), id_o, (j | k) != 0);
            if (j >= nct) {
  #pragma unroll
              for (int k = KC / 16; k < KT / 16; ++k)
                mma_f16_ta(tmem, pt + uint32_t(8 * k), vd + (k * 2048 >> 4), id_o, 1);
            }
            mma_commit(sh.pv_done + b);
          }
          if (!ok) break;
          mbar_arrive(sh.item_empty + slot);
          T += ntiles;
        }
        if (!ok) {
          sh.abort = 1;
          flag(a.status, JET_ERR_TIMEOUT);
        }
        mma_commit(sh.drain + 1);  // nor may its products outlive it
        mbar_wait(sh.drain + 1, 0, kDrainNs, nullptr);
      }
    }
  } else if (warp >= kWideWarp) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 88;");
    // ---------------------------------------------------------------- queries and V
    const int wi = warp - kWideWarp, q4 = wi & 3, half = wi >> 2;
    const int t = threadIdx.x - kWideWarp * 32;
    const int row = q4 * 32 + lane;  // of the queries, in two halves of their elements
    const uint32_t lane_off = uint32_t(q4 * 32) << 16;
    // of a V tile: one key's pieces of 16 codes, every kPer-th one. Eight lanes are eight
    // keys, whose swizzled places differ in their banks, before and after.
    constexpr int kPer = kWideThreads / KT, kMine = DH / 16 / kPer;
    const int key = t & (KT - 1), c0 = t / KT;
    const int block = key / kKvBlock;  // of the tile's, the key's: the same for a warp
    bool ok = true;
    int T = 0, n_q = 0;  // tiles of earlier items; items whose queries this warp split
    for (int u = 0; ok; ++u) {
      const int slot = u & 1;
      if (!wait32(sh.item_full + slot, (u >> 1) & 1, a.wait_ns, abort_flag)) {
        ok = false;
        break;
      }
      if (!sh.ring[slot].live) break;
      const ItemGeo e = sh.ring[slot].e;
      const int fed = sh.ring[slot].fed, keys = e.k_end - e.k_begin;
      const uint8_t* ex = a.v_exp + size_t(kv_place(e.p0, e.r, e.k_begin / kKvBlock)) * a.Hkv + e.kh;
      const int blocks = (keys + kKvBlock - 1) / kKvBlock;
      uint32_t byte = block < blocks ? load_ahead(ex + size_t(block) * a.Hkv) : 0;
      if (u == 0 && fed > 0) {
        const uint32_t top = cand_top<DH>(a, e.kh, e.f_begin, fed, t, kWideThreads);
        if (lane == 0) atomicMax(&sh.vtop[slot], top);
      }
      if (lane == 0) mbar_arrive(sh.aux_full + slot);
      if (!wait32(&sh.q_full, u & 1, a.wait_ns, abort_flag)) {
        ok = false;
        break;
      }
      if (q4 * 32 % RV < e.nv) {
        // the row's largest magnitude (NaN and infinities lie above all), this half's and
        // the other's: rows past the block's vectors hold what an earlier block left and
        // go unread
        constexpr int kMyPieces = DH / 16;  // of eight elements
        uint32_t mx[4] = {0, 0, 0, 0};
#pragma unroll 4  // (code that runs once an item is fetched anew each time)
        for (int i = 0; i < kMyPieces; ++i) {
          const int c = kMyPieces * half + i;
          const uint4 q = *reinterpret_cast<const uint4*>(smem + (c >> 3) * (kBV * 128) +
                                                          sw128(row, c & 7));
          mx[0] = __vmaxu2(mx[0], q.x & 0x7fff7fffu);
          mx[1] = __vmaxu2(mx[1], q.y & 0x7fff7fffu);
          mx[2] = __vmaxu2(mx[2], q.z & 0x7fff7fffu);
          mx[3] = __vmaxu2(mx[3], q.w & 0x7fff7fffu);
        }
        mx[0] = __vmaxu2(__vmaxu2(mx[0], mx[1]), __vmaxu2(mx[2], mx[3]));
        sh.qmax[half][row] = max(mx[0] & 0xffffu, mx[0] >> 16);
        __syncwarp();
        if (lane == 0) mbar_arrive(sh.a_full + q4);
        if (!wait32(sh.a_full + q4, n_q & 1, a.wait_ns, abort_flag)) {
          ok = false;
          break;
        }
        ++n_q;
        const uint32_t top = max(sh.qmax[0][row], sh.qmax[1][row]);
        const bool finite = top < 0x7f80u;
        const int qx = finite ? kv_exponent(top << 16) : 0;
        const float inv = pow2(-qx);
        // the codes of the item before are read by its last product with the keys; a
        // softmax warp must not find qt_full two items on
        if (u >= 1 && (!wait32(&sh.qt_free, (u - 1) & 1, a.wait_ns, abort_flag) ||
                       !wait32(&sh.qx_read, (u - 1) & 1, a.wait_ns, abort_flag))) {
          ok = false;
          break;
        }
        if (half == 0) sh.qx[slot][row] = qx;
        tc_fence_after();
        // 32 elements at a time: eight columns of four codes
#pragma unroll 1
        for (int k32 = DH / 64 * half; k32 < DH / 64 * (half + 1); ++k32) {
          uint32_t hi[8], lo[8];
#pragma unroll
          for (int c = 0; c < 4; ++c) {
            const uint4 xv = *reinterpret_cast<const uint4*>(
                smem + (k32 >> 1) * (kBV * 128) + sw128(row, 4 * (k32 & 1) + c));
            const uint32_t w[4] = {xv.x, xv.y, xv.z, xv.w};
            uint32_t y[4];
#pragma unroll
            for (int k = 0; k < 4; ++k)  // (f16 holds a bf16 number's eight digits)
              y[k] = pack_f16(__uint_as_float(w[k] << 16) * inv,
                              __uint_as_float(w[k] & 0xffff0000u) * inv);
#pragma unroll
            for (int i = 0; i < 2; ++i) {
              uint32_t h0, h1;
              const uint32_t h = f16x4_to_e4m3x4(y[2 * i], y[2 * i + 1]);
              e4m3x4_to_f16x4(h, h0, h1);
              hi[2 * c + i] = finite ? h : 0x7f7f7f7fu;
              lo[2 * c + i] =
                  f16x4_to_e4m3x4(sub_f16x2(y[2 * i], h0), sub_f16x2(y[2 * i + 1], h1));
            }
          }
          const uint32_t at = tmem + lane_off + G::kQCol + uint32_t(8 * k32);
          tmem_st_8cols_u32(at, hi);
          tmem_st_8cols_u32(at + DH / 4, lo);
        }
        tmem_wait_st();
        tc_fence_before();
      } else if (u >= 1 && (!wait32(&sh.qt_free, (u - 1) & 1, a.wait_ns, abort_flag) ||
                            !wait32(&sh.qx_read, (u - 1) & 1, a.wait_ns, abort_flag))) {
        ok = false;
        break;
      }
      __syncwarp();
      if (lane == 0) {
        mbar_arrive(&sh.qt_full);
        mbar_arrive(&sh.q_free);
      }
      if (!wait32(sh.aux_full + slot, (u >> 1) & 1, a.wait_ns, abort_flag)) {
        ok = false;
        break;
      }
      const int2 unit = value_unit(sh.vx[slot], sh.vtop[slot]);
      const int vx = unit.x;
      // a V tile's codes there, and the place that its widened values take free
      auto ready = [&](int Tj) -> bool {
        return wait32(sh.v_full + Tj % NV, (Tj / NV) & 1, a.wait_ns, abort_flag) &&
               (Tj < NW || wait32(sh.pv_done + (Tj - NW) % NS, ((Tj - NW) / NS) & 1, a.wait_ns,
                                  abort_flag));
      };
      auto done = [&](int Tj) {
        fence_proxy_async_smem();
        __syncwarp();
        if (lane == 0) {
          mbar_arrive(sh.w_full + Tj % NW);
          mbar_arrive(sh.v_empty + Tj % NV);
        }
      };
      for (int j = 0; j < e.nct; ++j) {
        const int Tj = T + j;
        ok = ready(Tj);
        if (!ok) break;
        const uint8_t* vs = smem + G::kOffV + (Tj % NV) * G::kTile;
        uint8_t* ws = smem + G::kOffW + (Tj % NW) * 2 * G::kTile;
        // candidate values, in the places the product reads
        const int left = unit.y ? 0 : fed - j * KC;
        const float inv = pow2(-vx);
#pragma unroll 2
        for (int k = 0; k < kMine; ++k) {
          const int i = t + k * kWideThreads;
          const uint4 v = *reinterpret_cast<const uint4*>(vs + 16 * i);
          const uint32_t in[4] = {v.x, v.y, v.z, v.w};
          uint32_t y[4];
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            y[q] = pack_f16(__uint_as_float(in[q] << 16) * inv,
                            __uint_as_float(in[q] & 0xffff0000u) * inv);
            if (((i >> 3) & (KC - 1)) >= left) y[q] = 0u;
          }
          *reinterpret_cast<uint4*>(ws + 16 * i) = make_uint4(y[0], y[1], y[2], y[3]);
        }
        done(Tj);
      }
      if (!ok) break;
      int left = keys, next = block;  // the keys past `left` of a tile are another request's
      for (int Tj = T + e.nct; Tj < T + e.ntiles; ++Tj, left -= KT) {
        ok = ready(Tj);
        if (!ok) break;
        const uint8_t* vs = smem + G::kOffV + (Tj % NV) * G::kTile;
        uint8_t* ws = smem + G::kOffW + (Tj % NW) * 2 * G::kTile;
        uint4 x[kMine];
#pragma unroll
        for (int i = 0; i < kMine; ++i)
          x[i] = *reinterpret_cast<const uint4*>(vs + raw_piece<DH, KT>(key, c0 + kPer * i));
        // 2^(X - vx), what the block's codes are worth in the unit. Where f16 does not hold it
        // the codes, multiples of 2^-9, take 2^-15 here, exactly, and the rest below.
        const int exact_k2 = exponent_of(byte) - vx;
        const int k2 = exact_k2 < -24 ? -15 : exact_k2;
        next += KT / kKvBlock;
        if (next < blocks) byte = load_ahead(ex + size_t(next) * a.Hkv);
        if (__builtin_expect(left < KT && key >= left, 0)) {
#pragma unroll
          for (int i = 0; i < kMine; ++i) x[i] = make_uint4(0u, 0u, 0u, 0u);
        }
        const uint32_t f = pow2_f16x2(k2);
#pragma unroll
        for (int i = 0; i < kMine; ++i) {
          const uint32_t in[4] = {x[i].x, x[i].y, x[i].z, x[i].w};
          uint32_t y[8];
#pragma unroll
          for (int q = 0; q < 4; ++q) e4m3x4_to_f16x4(in[q], y[2 * q], y[2 * q + 1]);
          if (k2 != 0) {
#pragma unroll
            for (int q = 0; q < 8; ++q) y[q] = mul_f16x2(y[q], f);
          }
          const int c = c0 + kPer * i;  // pieces 2 c and 2 c + 1 of the f16 row
          uint8_t* to = ws + (c >> 2) * (KT * 128);
          *reinterpret_cast<uint4*>(to + sw128(key, (2 * c) & 7)) =
              make_uint4(y[0], y[1], y[2], y[3]);
          *reinterpret_cast<uint4*>(to + sw128(key, (2 * c + 1) & 7)) =
              make_uint4(y[4], y[5], y[6], y[7]);
        }
        if (__builtin_expect(exact_k2 < -24, 0)) {
          // (values rounded here only; from 2^-34 on to zeros, as 448 2^-34 < 2^-25)
          const uint32_t rest = pow2_f16x2(max(exact_k2, -39) + 15);
#pragma unroll 1
          for (int i = 0; i < 2 * kMine; ++i) {
            const int c = 2 * (c0 + kPer * (i >> 1)) + (i & 1);
            uint4* at = reinterpret_cast<uint4*>(ws + (c >> 3) * (KT * 128) + sw128(key, c & 7));
            const uint4 y = *at;
            *at = make_uint4(mul_f16x2(y.x, rest), mul_f16x2(y.y, rest), mul_f16x2(y.z, rest),
                             mul_f16x2(y.w, rest));
          }
        }
        done(Tj);
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
    asm volatile("setmaxnreg.inc.sync.aligned.u32 112;");
    // ---------------------------------------------------------------- softmax
    const int q4 = warp & 3, half = (warp - kSoftWarp) >> 2;
    // the query vector of this TMEM lane, and which of its copies
    const int i = q4 * 32 % RV + lane, copy = q4 * 32 / RV;
    const uint32_t lane_off = uint32_t(q4 * 32) << 16;
    uint4* stage = reinterpret_cast<uint4*>(smem + G::kOffStage + (warp - kSoftWarp) * 2048);
    bool ok = true;
    int T = 0, x = 0;  // tiles of earlier items; tiles that this warp has worked on
    for (int u = 0; ok; ++u) {
      const int slot = u & 1;
      if (!wait32(sh.item_full + slot, (u >> 1) & 1, a.wait_ns, abort_flag)) {
        ok = false;
        break;
      }
      if (!sh.ring[slot].live) break;
      const ItemGeo& e = sh.ring[slot].e;  // (read again where needed: registers are few)
      const int nct = e.nct, ntiles = e.ntiles, keys = e.k_end - e.k_begin, f_begin = e.f_begin;
      const bool valid = i < e.nv;
      // a warp without vectors only keeps the barriers going
      const bool some = q4 * 32 % RV < e.nv;
      if (nct > 0 && !wait32(sh.aux_full + slot, (u >> 1) & 1, a.wait_ns, abort_flag)) {
        ok = false;
        break;
      }
      const uint8_t* ex = a.k_exp + size_t(kv_place(e.p0, e.r, e.k_begin / kKvBlock)) * a.Hkv + e.kh;
      constexpr int kCols = G::kHalf / R;
      const int col0 = kCols * copy;  // of this half's
      // this half's blocks of the tiles: every tile's (d 256), or every second block
      constexpr int kBlocks = KT / kKvBlock;
      const int blocks = (keys + kKvBlock - 1) / kKvBlock;
      int next = kBlocks == 2 ? half : 0;
      ex += size_t(next) * a.Hkv;
      const size_t ex_step = size_t(kBlocks) * a.Hkv;
      uint32_t byte = next < blocks ? load_ahead(ex) : 0;
      int qx = 0;
      float m = -INFINITY, l = 0.f;  // the running maximum; the sum over this half's columns
      for (int j = 0; j < ntiles; ++j) {
        const int Tj = T + j, b = Tj % NS;
        if (j == nct) {
          if (!wait32(&sh.qt_full, u & 1, a.wait_ns, abort_flag)) {
            ok = false;
            break;
          }
          qx = sh.qx[slot][q4 * 32 + lane];
          __syncwarp();
          if (lane == 0) mbar_arrive(&sh.qx_read);
        }
        // the scores' factor in base 2, and this half's columns [klo, khi) of the tile
        // where not all of them count
        float mul = a.scale_log2;
        bool cut = false;
        int klo = 0, khi = kCols;
        if (j < nct) {
          const int2 sees = sh.sees[slot][i];
          klo = sees.x - j * KC - col0;
          khi = half == 0 && valid ? sees.y - j * KC - col0 : 0;
          cut = true;
        } else {
          mul *= pow2(min(max(qx + exponent_of(byte), -126), 126));
          next += kBlocks;
          ex += ex_step;
          if (next < blocks) byte = load_ahead(ex);
          if (j == ntiles - 1) {
            khi = keys - (j - nct) * KT - G::kHalf * half - col0;
            cut = khi < kCols;
          }
        }
        if (!wait32(sh.s_full + b, (Tj / NS) & 1, a.wait_ns, abort_flag)) {
          ok = false;
          break;
        }
        tc_fence_after();
        if (some) {
          float sv[kCols];
          tmem_ld_cols(tmem + lane_off + G::kSCol + b * KT + G::kHalf * half + col0, sv);
          tmem_wait_ld();
          if (__builtin_expect(cut, 0)) {
#pragma unroll
            for (int c = 0; c < kCols; ++c)
              if (c < klo || c >= khi) sv[c] = -INFINITY;
          }
          float mq[4];
#pragma unroll
          for (int q = 0; q < 4; ++q) mq[q] = fmaxf(sv[q], sv[4 + q]);
#pragma unroll
          for (int c = 8; c < kCols; c += 8)
#pragma unroll
            for (int q = 0; q < 4; ++q) mq[q] = max3(mq[q], sv[c + q], sv[c + 4 + q]);
          float mt = max3(mq[0], mq[1], fmaxf(mq[2], mq[3]));
          mt *= mul;
          // the other half's: then both know the row's maximum over the tile
          sh.m[x & 1][half][q4 * 32 + lane] = mt;
          __syncwarp();
          if (lane == 0) mbar_arrive(&sh.m_full[x & 1][q4]);
          if (!wait32(&sh.m_full[x & 1][q4], (x >> 1) & 1, a.wait_ns, abort_flag)) {
            ok = false;
            break;
          }
          mt = fmaxf(mt, sh.m[x & 1][half ^ 1][q4 * 32 + lane]);
          ++x;
          const bool grow = j == 0 || (valid && mt > m + kRescaleLog2);
          if (__builtin_expect(__any_sync(0xffffffffu, grow), 0)) {
            const float m_new = grow ? mt : m;
            if (j > 0) {
              // O holds this item's P V so far: wait for the last one, rescale this half of
              // its columns in TMEM
              if (!wait32(sh.pv_done + (Tj - 1) % NS, ((Tj - 1) / NS) & 1, a.wait_ns,
                                  abort_flag)) {
                ok = false;
                break;
              }
              tc_fence_after();
              const float f = !grow ? 1.f : m == -INFINITY ? 0.f : ex2(m - m_new);
#pragma unroll 1
              for (int c0 = half * (DH / 2); c0 < (half + 1) * (DH / 2); c0 += 16) {
                float ov[16];
                tmem_ld_16cols(tmem + lane_off + c0, ov);
                tmem_wait_ld();
#pragma unroll
                for (int c = 0; c < 16; ++c) ov[c] *= f;
                tmem_st_16cols(tmem + lane_off + c0, ov);
              }
              l *= f;
            }
            m = m_new;
          }
          // weights 2^(s - m + 7): f16 holds them from 2^-24 to the 2^15 that a maximum not
          // yet taken over may give; no key seen yet: weights of 0
          const float sub = m == -INFINITY ? 0.f : kWeightLog2 - m;
          const float2 mul2 = make_float2(mul, mul), sub2 = make_float2(sub, sub);
          float2 ps[4];
#pragma unroll
          for (int q = 0; q < 4; ++q) ps[q] = make_float2(0.f, 0.f);
          // P takes the place of scores that are in registers by now; where the vectors are
          // there R times, each copy has weights in its own columns and zeros in the others'
          constexpr int kWords = G::kHalf / 2;
          const uint32_t pt = tmem + lane_off + G::kSCol + b * KT + kWords * half;
          if constexpr (R > 1) {
            const uint32_t zeros[16] = {};
#pragma unroll
            for (int k = 0; k < kWords; k += 16) tmem_st_16cols_u32(pt + k, zeros);
            tmem_wait_st();
          }
          constexpr int kStep = kCols / 2 < 16 ? kCols / 2 : 16;
#pragma unroll
          for (int k = 0; k < kCols / 2; k += kStep) {
            uint32_t pw[kStep];
#pragma unroll
            for (int c = 0; c < kStep; ++c) {
              const int at = 2 * (k + c);
              const float2 y = fma2(make_float2(sv[at], sv[at + 1]), mul2, sub2);
              const float2 p = make_float2(ex2(y.x), ex2(y.y));
              ps[c & 3] = add2(ps[c & 3], p);
              pw[c] = pack_f16(p.x, p.y);
            }
            tmem_st_cols(pt + col0 / 2 + k, pw);
          }
          const float2 p = add2(add2(ps[0], ps[1]), add2(ps[2], ps[3]));
          l += p.x + p.y;
          tmem_wait_st();
        }
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(sh.p_full + b);
      }
      if (!ok) break;
      // both halves' sums
      sh.l[slot][half][q4 * 32 + lane] = l;
      __syncwarp();
      if (lane == 0) mbar_arrive(sh.l_full + q4);
      if (!wait32(sh.l_full + q4, u & 1, a.wait_ns, abort_flag)) {
        ok = false;
        break;
      }
      l += sh.l[slot][half ^ 1][q4 * 32 + lane];
      const int Tl = T + ntiles - 1;
      const bool direct = R == 1 && e.splits_r == 1;
      const int part = e.split * R + copy;  // the partial that is written
      char* dst[4];  // of the vectors this lane stores (8 s + lane / 4, 16 bytes each)
      {
        char* base = direct ? reinterpret_cast<char*>(a.o) : reinterpret_cast<char*>(a.o_part);
        const int esize = direct ? 2 : 4;
#pragma unroll
        for (int s = 0; s < 4; ++s) {
          const int gi = q4 * 32 % RV + 8 * s + (lane >> 2);
          dst[s] = nullptr;
          if (gi < e.nv) {
            const int gv = e.vbase + gi;
            const int n = e.n0 + gv / g, h = e.kh * g + gv % g;
            const size_t row = size_t(direct ? n : part * (long long)a.N + n) * a.Hq + h;
            dst[s] = base + (row * DH + half * (DH / 2)) * esize + (lane & 3) * 16;
          }
        }
      }
      if (valid && a.splits * R > 1 && half == 0) {
        // as the bf16 kernel leaves them for the combine, but with the partial divided by
        // its sum (l 1, the sum in m), as a sum of large values may pass float32
        const int gv = e.vbase + i;
        const size_t at = size_t(e.n0 + gv / g) * a.Hq + e.kh * g + gv % g;
        const size_t step = size_t(a.N) * a.Hq;
        a.ml_part[at + (direct ? 0 : part * step)] =
            direct ? make_float2(0.f, -1.f) : make_float2(m + log2f(l), l > 0.f ? 1.f : l);
        if (!direct && part == e.splits_r * R - 1)
          for (int sp = e.splits_r * R; sp < a.splits * R; ++sp)
            a.ml_part[at + sp * step] = make_float2(-INFINITY, 0.f);
      }
      if (!wait32(sh.aux_full + slot, (u >> 1) & 1, a.wait_ns, abort_flag)) {
        ok = false;
        break;
      }
      const float inv = l > 0.f ? 1.f / l : 0.f, unit = pow2(value_unit(sh.vx[slot], sh.vtop[slot]).x);
      // 1 / l and V's unit in one factor, unless the factor would not be a normal number
      const bool plain = __all_sync(0xffffffffu, fabsf(inv * unit) > 0x1p-100f) != 0;
      if (!wait32(sh.pv_done + Tl % NS, (Tl / NS) & 1, a.wait_ns, abort_flag)) {
        ok = false;
        break;
      }
      tc_fence_after();
      if (some) {
        float2 scale = make_float2(inv * (plain ? unit : 1.f), inv * (plain ? unit : 1.f));
        bool rest = !plain;  // V's unit still to come
        if (__builtin_expect(nct > 0 && value_unit(sh.vx[slot], sh.vtop[slot]).y, 0)) {
          // O normalised where it is, then the candidates' tokens one by one, each weight
          // from its key and the row's query
#pragma unroll 1
          for (int c0 = half * (DH / 2); c0 < (half + 1) * (DH / 2); c0 += 16) {
            float ov[16];
            tmem_ld_16cols(tmem + lane_off + c0, ov);
            tmem_wait_ld();
#pragma unroll
            for (int c = 0; c < 16; ++c) ov[c] = ov[c] * inv * unit;
            tmem_st_16cols(tmem + lane_off + c0, ov);
          }
          scale = make_float2(1.f, 1.f);
          rest = false;
          const int2 sees = valid ? sh.sees[slot][i] : make_int2(0, 0);
          const int first = __reduce_min_sync(0xffffffffu, sees.x < sees.y ? sees.x : INT_MAX);
          const int end = __reduce_max_sync(0xffffffffu, sees.y);
          const int gv = e.vbase + min(i, e.nv - 1);
          const uint4* q = reinterpret_cast<const uint4*>(
              a.q + (size_t(e.n0 + gv / g) * a.Hq + e.kh * g + gv % g) * DH);
          const float sub = m == -INFINITY ? 0.f : kWeightLog2 - m;
#pragma unroll 1
          for (int f = first; f < end; ++f) {
            const size_t at = (size_t(f_begin + f) * a.Hkv + e.kh) * DH;
            const uint4* kc = reinterpret_cast<const uint4*>(a.k_cand + at);
            float s = 0.f;
#pragma unroll 1
            for (int c = 0; c < DH / 8; ++c) {
              const uint4 x = q[c], y = kc[c];
              const uint32_t xw[4] = {x.x, x.y, x.z, x.w}, yw[4] = {y.x, y.y, y.z, y.w};
#pragma unroll
              for (int k = 0; k < 4; ++k) {
                s = fmaf(__uint_as_float(xw[k] << 16), __uint_as_float(yw[k] << 16), s);
                s = fmaf(__uint_as_float(xw[k] & 0xffff0000u),
                         __uint_as_float(yw[k] & 0xffff0000u), s);
              }
            }
            const bool mine = f >= sees.x && f < sees.y && f % KC / kCols == copy;
            const float w = ex2(fmaf(s, a.scale_log2, sub)) * inv;
#pragma unroll 1
            for (int c0 = half * (DH / 2); c0 < (half + 1) * (DH / 2); c0 += 16) {
              float ov[16];
              tmem_wait_st();
              tmem_ld_16cols(tmem + lane_off + c0, ov);
              tmem_wait_ld();
#pragma unroll
              for (int c = 0; c < 16; ++c) {
                const float x = __bfloat162float(a.v_cand[at + c0 + c]);
                if (mine) ov[c] += isfinite(x) ? w * x : x;
              }
              tmem_st_16cols(tmem + lane_off + c0, ov);
            }
          }
          tmem_wait_st();
        }
        // 64 bytes of each vector at a time through this warp's 2 KB stage: four 16-byte
        // pieces a row, rotated so that eight lanes meet different banks
        auto put = [&](const uint4(&x)[4]) {
#pragma unroll
          for (int q = 0; q < 4; ++q) stage[lane * 4 + (q ^ ((lane >> 1) & 3))] = x[q];
          __syncwarp();
          uint4 val[4];
#pragma unroll
          for (int s = 0; s < 4; ++s) {
            const int iv = 8 * s + (lane >> 2), c = lane & 3;
            val[s] = stage[iv * 4 + (c ^ ((iv >> 1) & 3))];
          }
#pragma unroll
          for (int s = 0; s < 4; ++s) {
            if (dst[s]) {
              *reinterpret_cast<uint4*>(dst[s]) = val[s];
              dst[s] += 64;
            }
          }
          __syncwarp();
        };
        // each of a row's two warps writes half of the columns
        const float2 zero = make_float2(0.f, 0.f);
#pragma unroll 1
        for (int c0 = half * (DH / 2); c0 < (half + 1) * (DH / 2); c0 += 32) {
          float ov[32];
          tmem_ld_32cols(tmem + lane_off + c0, ov);
          tmem_wait_ld();
#pragma unroll
          for (int c = 0; c < 32; c += 2) {
            const float2 y = fma2(make_float2(ov[c], ov[c + 1]), scale, zero);
            ov[c] = y.x;
            ov[c + 1] = y.y;
          }
          if (rest) {
#pragma unroll
            for (int c = 0; c < 32; ++c) ov[c] *= unit;
          }
          if (direct) {
            uint4 x[4];
#pragma unroll
            for (int q = 0; q < 4; ++q) {
              const float* y = ov + 8 * q;
              x[q] = make_uint4(pack_bf16(y[0], y[1]), pack_bf16(y[2], y[3]),
                                pack_bf16(y[4], y[5]), pack_bf16(y[6], y[7]));
            }
            put(x);
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
              put(x);
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
      T += ntiles;
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

// codes [keys, heads, DH]: box of 128 (or all 64) codes x 1 head x box_keys keys
bool encode_codes(CUtensorMap* map, const void* base, int rows, int heads, int DH, int box_keys) {
  auto fn = encode_fn();
  if (!fn) return false;
  const cuuint64_t dims[3] = {cuuint64_t(DH), cuuint64_t(heads), cuuint64_t(rows)};
  const cuuint64_t strides[2] = {cuuint64_t(DH), cuuint64_t(heads) * DH};
  const cuuint32_t box[3] = {cuuint32_t(std::min(DH, 128)), 1, cuuint32_t(box_keys)};
  const cuuint32_t estr[3] = {1, 1, 1};
  return fn(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 3, const_cast<void*>(base), dims, strides, box,
            estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
            DH == 64 ? CU_TENSOR_MAP_SWIZZLE_64B : CU_TENSOR_MAP_SWIZZLE_128B,
            CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <int DH, int R>
cudaError_t launch_dh(const jet_layout& lay, const jet_dims& d, const AttnPlan& plan,
                      const void* q, const void* k8, const void* v8, const void* k_cand,
                      const void* v_cand, void* o, void* ws, int* status, cudaStream_t st) {
  const jet_sizes& n = lay.n;
  const int F = n.N - n.R;
  const int g = d.Hq / d.Hkv;
  if (g > kBV / R) return cudaErrorInvalidValue;
  CUtensorMap tmQ, tmK, tmV, tmKc, tmVc;
  if (!encode_3d(&tmQ, q, n.N, d.Hq, DH, g, kBV / R / g) ||
      !encode_codes(&tmK, k8, n.total_prefix, d.Hkv, DH, Geo<DH>::kT) ||
      !encode_codes(&tmV, v8, n.total_prefix, d.Hkv, DH, Geo<DH>::kT))
    return cudaErrorInvalidValue;
  if (F > 0) {
    if (!encode_3d(&tmKc, k_cand, F, d.Hkv, DH, 1, Geo<DH>::kC) ||
        !encode_3d(&tmVc, v_cand, F, d.Hkv, DH, 1, Geo<DH>::kC))
      return cudaErrorInvalidValue;
  } else {
    tmKc = tmK;  // never read: no request has candidate tiles
    tmVc = tmV;
  }
  const size_t vecs = size_t(plan.splits) * R * n.N * d.Hq;
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
  a.rb = kBV / R / g;
  a.has_cand = F > 0;
  a.scale_log2 = 1.4426950408889634f / sqrtf(float(DH));
  a.k_exp = static_cast<const uint8_t*>(k8) + exp_off;
  a.v_exp = static_cast<const uint8_t*>(v8) + exp_off;
  a.q = static_cast<const __nv_bfloat16*>(q);
  a.k_cand = static_cast<const __nv_bfloat16*>(k_cand);
  a.v_cand = static_cast<const __nv_bfloat16*>(v_cand);
  a.splits = plan.splits;
  a.qgroups = plan.qgroups;
  a.n_all = (long long)n.R * d.Hkv * plan.qgroups * plan.splits;
  const int sms = sm_count();
  if (sms < 1) return cudaErrorInvalidValue;
  const int grid = int(std::max<long long>(1, std::min<long long>(sms, a.n_all)));
  const size_t smem = Geo<DH>::kBytes + 1024;
  cudaError_t e = cudaFuncSetAttribute(attend_kv8_kernel<DH, R>,
                                       cudaFuncAttributeMaxDynamicSharedMemorySize, int(smem));
  if (e != cudaSuccess) return e;
  e = launch_pdl(attend_kv8_kernel<DH, R>, dim3(grid), dim3(kThreads), smem, st, tmQ, tmK, tmV,
                 tmKc, tmVc, a);
  if (e != cudaSuccess || plan.splits * R <= 1) return e;
  const long long blocks = ((long long)n.N * d.Hq + 3) / 4;
  return launch_pdl(attend_combine_kernel<DH>, dim3(unsigned(blocks)), dim3(128), 0, st,
                    lay.row_req, n.N, n.R, d.Hq, plan.splits * R, blocks <= 8LL * sms, a.o_part,
                    a.ml_part, a.o, status);
}

}  // namespace

cudaError_t launch_attend_kv8_tc(const jet_layout& lay, const jet_dims& d, const AttnPlan& plan,
                                 const void* q, const void* k8, const void* v8,
                                 const void* k_cand, const void* v_cand, void* o, void* ws,
                                 int* status, cudaStream_t st) {
#define JET_KV8(DH, R)                                                                     \
  if (d.d == DH && plan.copies == R)                                                       \
  return launch_dh<DH, R>(lay, d, plan, q, k8, v8, k_cand, v_cand, o, ws, status, st)
  JET_KV8(64, 1);
  JET_KV8(64, 2);
  JET_KV8(64, 4);
  JET_KV8(128, 1);
  JET_KV8(128, 2);
  JET_KV8(128, 4);
  JET_KV8(256, 1);
#undef JET_KV8
  return cudaErrorInvalidValue;
}

}  // namespace jet
