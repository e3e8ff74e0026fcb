// The norm of every query and key head and its rotation by position, in one pass over the
// projected queries and keys.
//
// Every element is read and written once, so HBM bounds long inputs and latencies short
// ones; what stands between a long input and HBM is the number of instructions. A warp takes
// one token, or every parts-th piece of it, 256 elements at a time - one head of 256, two of
// 128, four of 64 - eight a lane. The two elements of a pair lie in one lane (two groups of
// four, half a rotation apart, or eight in a row), so the rotation needs no shuffle and the
// norm three to five, and a lane's four cosines and sines, of the same four pairs in every
// head, stay in registers for the whole token.
//
// An angle is a 64-bit fraction of a turn, position times frequency modulo 2^64; its
// nearest quarter turn is taken off exactly and the rest, at most an eighth of a turn, is
// rounded to float32 for sincospif, by less than 2^-25 radians at any position. (The frequency's
// own digits count |p f| 2^-52 beside that: 2^-21 at f = 1 and the farthest int32 positions.)
//
// Everything is float32 from the load to the one rounding of the store. 74,210 tokens of 24 + 4
// heads of 256 (1.06 GB each way in bf16) take 350 us, 91 % of the copy rate. A warp's loads are
// one step ahead of its arithmetic, too few bytes in flight for HBM, so a token's queries are asked
// for at its start (386 -> 361; d 128, 92,227 tokens of 32 + 8 heads 326 -> 287), and the outputs
// leave L2 first (361 -> 352, 280). 64 rows take 4 to 5 us, a launch and two latencies in a row.
#include <algorithm>

#include "jet_device.cuh"
#include "jet_internal.h"

namespace jet {
namespace {

constexpr int kThreads = 128;
constexpr int kWarps = kThreads / 32;
// bytes of a token's queries that are asked for ahead: 44 MB for all of the chip's warps
constexpr int kAhead = 8192;

enum { kGiven = 0, kPrefix = 1, kRows = 2 };  // where the positions come from

struct RotArgs {
  const int32_t* pos;            // kGiven
  const int32_t* prefix_offset;  // kPrefix, kRows
  const int32_t* row_req;        // kRows
  const int32_t* row_cand;
  const int32_t* row_pos;
  const void* q;
  const void* k;
  const void* gq;
  const void* gk;
  void* qo;
  void* ko;
  int* status;
  int n, R, total, Hq, Hkv, nfed;
  int parts;   // warps that share a token's heads
};

// cos and sin of the angle `turn` (2^-64 turns a position) at position p
__device__ __forceinline__ float2 turn_cos_sin(uint64_t turn, int p) {
  const uint64_t a = turn * uint64_t(int64_t(p));
  const uint64_t quarter = (a + (uint64_t(1) << 61)) >> 62;  // the nearest one
  const int64_t rest = int64_t(a - (quarter << 62));         // [-2^61, 2^61)
  float s, c;
  sincospif(__ll2float_rn(rest) * 1.0842021724855044e-19f, &s, &c);  // 2^-63 half turns
  const bool odd = quarter & 1, flip = quarter & 2;
  const float x = odd ? -s : c, y = odd ? c : s;
  return make_float2(flip ? -x : x, flip ? -y : y);
}

// the position of token n and, in *fed, the key that goes with it (-1: none); false where
// the layout does not hold it. One warp, every lane the same.
template <int FROM>
__device__ __forceinline__ bool token_at(const RotArgs& a, int n, int lane, int* pos, int* fed) {
  if constexpr (FROM == kGiven) {
    *pos = a.pos[n];
    *fed = n;
    return true;
  } else if constexpr (FROM == kRows) {
    const int r = a.row_req[n], c = a.row_cand[n], t = a.row_pos[n];
    *fed = -1;
    if (r < 0 || r >= a.R) return false;
    const int p0 = a.prefix_offset[r], p1 = a.prefix_offset[r + 1];
    if (p0 < 0 || p1 <= p0 || p1 > a.total || t < 0 || t > a.n) return false;
    *pos = p1 - p0 - 1 + t;
    if (c < 0) return true;
    *fed = n - r - 1;
    return *fed >= 0 && *fed < a.nfed;
  } else {
    // the request whose span holds token n: 32 places of the offsets at a time
    int lo = 0, hi = a.R;  // offset[lo] <= n < offset[hi]
    while (hi - lo > 1) {
      const int step = (hi - lo + 31) / 32;
      const int at = min(lo + lane * step, hi);
      const unsigned le = __ballot_sync(0xffffffffu, at < hi && a.prefix_offset[at] <= n);
      if (!(le & 1u)) break;
      lo = lo + (31 - __clz(le)) * step;
      hi = min(lo + step, hi);
    }
    const int p0 = a.prefix_offset[lo], p1 = a.prefix_offset[lo + 1];
    *pos = n - p0;
    *fed = n;
    return p0 >= 0 && p0 <= n && n < p1 && p1 <= a.total;
  }
}

// four elements as they are in memory, and their values
template <typename T>
struct Raw4 {
  uint2 x;
  __device__ __forceinline__ void load(const T* p) { x = *reinterpret_cast<const uint2*>(p); }
  __device__ __forceinline__ void values(float (&v)[4]) const {
    v[0] = __uint_as_float(x.x << 16);
    v[1] = __uint_as_float(x.x & 0xffff0000u);
    v[2] = __uint_as_float(x.y << 16);
    v[3] = __uint_as_float(x.y & 0xffff0000u);
  }
};
template <>
struct Raw4<float> {
  float4 x;
  __device__ __forceinline__ void load(const float* p) { x = *reinterpret_cast<const float4*>(p); }
  __device__ __forceinline__ void values(float (&v)[4]) const {
    v[0] = x.x;
    v[1] = x.y;
    v[2] = x.z;
    v[3] = x.w;
  }
};

template <typename T>
__device__ __forceinline__ void store4(T* p, const float (&v)[4]) {
  if constexpr (sizeof(T) == 4) {
    __stcs(reinterpret_cast<float4*>(p), make_float4(v[0], v[1], v[2], v[3]));
  } else {
    uint2 x;
    *reinterpret_cast<__nv_bfloat162*>(&x.x) = __floats2bfloat162_rn(v[0], v[1]);
    *reinterpret_cast<__nv_bfloat162*>(&x.y) = __floats2bfloat162_rn(v[2], v[3]);
    __stcs(reinterpret_cast<uint2*>(p), x);
  }
}

// v over the root of the mean of its head's squares, times g. The root's reciprocal is the
// hardware's and one step of Newton's: two units of the last place at most, as a root and a
// quotient would be, for six instructions. Heads whose squares leave float32, or nearly, are
// scaled by a power of two first.
template <int DH>
__device__ __forceinline__ void normalise(float (&v)[2][4], const float (&g)[2][4], float eps) {
  auto squares = [&]() {
    float ss = 0.f;
#pragma unroll
    for (int j = 0; j < 4; ++j) ss = fmaf(v[0][j], v[0][j], fmaf(v[1][j], v[1][j], ss));
#pragma unroll
    for (int o = DH / 16; o > 0; o >>= 1) ss += __shfl_xor_sync(0xffffffffu, ss, o);
    return ss;
  };
  float x = fmaf(squares(), 1.f / float(DH), eps);
  if (__any_sync(0xffffffffu, !(x > 1e-30f && x < 1e30f))) {
    float top = 0.f;
#pragma unroll
    for (int j = 0; j < 4; ++j) top = fmaxf(top, fmaxf(fabsf(v[0][j]), fabsf(v[1][j])));
#pragma unroll
    for (int o = DH / 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
    const float m = fmaxf(top, sqrtf(eps));
    const int e = m > 0.f && m < INFINITY ? ilogbf(m) : 0;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      v[0][j] = ldexpf(v[0][j], -e);
      v[1][j] = ldexpf(v[1][j], -e);
    }
    x = fmaf(squares(), 1.f / float(DH), ldexpf(ldexpf(eps, -e), -e));
    if (top == 0.f) x = 1.f;  // zeros stay
    if (x == INFINITY) {      // an infinite element: NaN, and zeros beside it
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        v[0][j] *= 0.f;
        v[1][j] *= 0.f;
      }
      x = 1.f;
    }
  }
  const float r = rsqrtf(x);
  const float inv = r * fmaf(-0.5f * x * r, r, 1.5f);
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    v[0][j] = v[0][j] * inv * g[0][j];
    v[1][j] = v[1][j] * inv * g[1][j];
  }
}

// 8 elements a lane in two groups of four, v[0] and v[1]. Halves: the groups are half a
// rotation apart in the lanes that rotate, and in a row past them. Pairs: in a row.
template <int DH, int STYLE, int FROM, typename T>
__global__ void __launch_bounds__(kThreads, 9)
norm_rotate_kernel(const RotArgs a, const __grid_constant__ jet_rope rope) {
  pdl_begin();
  constexpr int kLanes = DH / 8;        // lanes of a head
  constexpr int kHeads = 32 / kLanes;   // heads of a warp's step
  const int lane = threadIdx.x & 31;
  const long long w = (long long)blockIdx.x * kWarps + (threadIdx.x >> 5);
  const int n = int(w / a.parts), part = int(w % a.parts);
  if (n >= a.n) return;
  const int half = rope.rot / 2;
  const int hl = lane % kLanes, hs = lane / kLanes;
  int e0, e1;  // the groups' elements
  bool rotates;
  if constexpr (STYLE == JET_ROPE_HALVES) {
    rotates = hl < half / 4;
    const int j = hl - half / 4;
    e0 = rotates ? 4 * hl : rope.rot + 8 * j;
    e1 = rotates ? half + 4 * hl : e0 + 4;
  } else {
    rotates = 8 * hl < rope.rot;
    e0 = 8 * hl;
    e1 = e0 + 4;
  }
  // The first step's elements come beside the token's position, and each later step's beside
  // the step before it
  const int nq = a.q ? (a.Hq + kHeads - 1) / kHeads : 0;
  Raw4<T> r0, r1;
  auto fetch = [&](const T* x, int at) {
    r0.load(x + at + e0);
    r1.load(x + at + e1);
  };
  if (part < nq && part * kHeads + hs < a.Hq)
    fetch(static_cast<const T*>(a.q) + size_t(n) * a.Hq * DH, (part * kHeads + hs) * DH);
  // and of a token that is one warp's, what comes after them starts on its way into L2
  if (a.q && a.parts == 1) {
    const char* row = static_cast<const char*>(a.q) + size_t(n) * a.Hq * DH * sizeof(T);
    const int bytes = min(kAhead, a.Hq * DH * int(sizeof(T)));
    for (int at = lane * 128; at < bytes; at += 32 * 128)
      asm volatile("prefetch.global.L2 [%0];" ::"l"(row + at));
  }
  int pos = 0, fed = -1;
  const bool ok = token_at<FROM>(a, n, lane, &pos, &fed);
  if (!ok) {
    if (lane == 0) flag(a.status, JET_ERR_DEVICE);
    return;
  }
  // the cosines and sines of pairs 4 hl .. + 3: DH / 64 pairs a lane, then from lane to lane
  float2 cs[4];
  {
    constexpr int kOwn = DH / 64;
    float2 own[kOwn];
#pragma unroll
    for (int i = 0; i < kOwn; ++i) {
      const int pair = lane * kOwn + i;
      own[i] = turn_cos_sin(pair < half ? rope.turn[pair] : 0, pos);
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int src = (4 * hl + j) / kOwn;
      cs[j].x = __shfl_sync(0xffffffffu, own[j % kOwn].x, src);
      cs[j].y = __shfl_sync(0xffffffffu, own[j % kOwn].y, src);
    }
  }

  // the H heads of row `row`, kHeads a step, every parts-th step from `st` on; returns the
  // step past them that is the next array's
  auto run = [&](const void* xs, void* ys, const void* gs, int H, int steps, size_t row, int st,
                 bool held) {
    float g[2][4];
#pragma unroll
    for (int j = 0; j < 4; ++j) g[0][j] = g[1][j] = 1.f;
    if (rope.norm && gs) {
      Raw4<T> r;
      r.load(static_cast<const T*>(gs) + e0);
      r.values(g[0]);
      r.load(static_cast<const T*>(gs) + e1);
      r.values(g[1]);
    }
    const T* x = static_cast<const T*>(xs) + row * H * DH;
    T* y = static_cast<T*>(ys) + row * H * DH;
    int head = st * kHeads + hs, at = head * DH;   // a token's heads: an int holds them
    const int step = a.parts * kHeads;
    if (!held && st < steps && head < H) fetch(x, at);
    for (; st < steps; st += a.parts) {
      float v[2][4];
      r0.values(v[0]);
      r1.values(v[1]);
      const bool in = head < H;
      T* out = y + at;
      head += step;
      at += step * DH;
      if (head < H) fetch(x, at);
      if (rope.norm) normalise<DH>(v, g, rope.eps);
      if (rotates) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          float& x0 = STYLE == JET_ROPE_HALVES ? v[0][j] : v[j >> 1][(2 * j) & 3];
          float& x1 = STYLE == JET_ROPE_HALVES ? v[1][j] : v[j >> 1][(2 * j + 1) & 3];
          const float y0 = x0, y1 = x1;
          x0 = y0 * cs[j].x - y1 * cs[j].y;
          x1 = y0 * cs[j].y + y1 * cs[j].x;
        }
      }
      if (in) {
        store4(out + e0, v[0]);
        store4(out + e1, v[1]);
      }
    }
    return st - steps;
  };
  int st = part;
  if (a.q) st = run(a.q, a.qo, a.gq, a.Hq, nq, size_t(n), st, true);
  if (a.k && fed >= 0)
    run(a.k, a.ko, a.gk, a.Hkv, (a.Hkv + kHeads - 1) / kHeads, size_t(fed), st, false);
}

template <int FROM, typename T>
cudaError_t launch_from(RotArgs a, const jet_dims& d, const jet_rope& rope, cudaStream_t st) {
  const int heads = 256 / d.d;
  const int steps =
      (a.q ? (d.Hq + heads - 1) / heads : 0) + (a.k ? (d.Hkv + heads - 1) / heads : 0);
  // few tokens: several warps each, down to a step a warp
  const long long want = 8LL * kPlanSMs;
  a.parts = int(std::min<long long>(steps, std::max<long long>(1, want / a.n)));
  const long long blocks = ((long long)a.n * a.parts + kWarps - 1) / kWarps;
  if (blocks > INT32_MAX) return cudaErrorInvalidConfiguration;
  const dim3 grid{unsigned(blocks)};
#define JET_ROT(DH)                                                                             \
  if (d.d == DH)                                                                                \
    return rope.style == JET_ROPE_HALVES                                                        \
               ? launch_pdl(norm_rotate_kernel<DH, JET_ROPE_HALVES, FROM, T>, grid,             \
                            dim3(kThreads), 0, st, a, rope)                                     \
               : launch_pdl(norm_rotate_kernel<DH, JET_ROPE_PAIRS, FROM, T>, grid,              \
                            dim3(kThreads), 0, st, a, rope)
  JET_ROT(64);
  JET_ROT(128);
  JET_ROT(256);
#undef JET_ROT
  return cudaErrorInvalidValue;
}

template <int FROM>
cudaError_t launch_type(const RotArgs& a, const jet_dims& d, const jet_rope& rope,
                        cudaStream_t st) {
  return d.dtype == JET_DTYPE_BF16 ? launch_from<FROM, __nv_bfloat16>(a, d, rope, st)
                                   : launch_from<FROM, float>(a, d, rope, st);
}

}  // namespace

cudaError_t launch_norm_rotate(const jet_layout* lay, bool rows, const jet_dims& d,
                               const jet_rope& rope, int n, const int32_t* pos, const void* q,
                               const void* k, const void* gq, const void* gk, void* qo, void* ko,
                               int* status, cudaStream_t st) {
  RotArgs a{};
  a.pos = pos;
  a.q = q;
  a.k = k;
  a.gq = q ? gq : nullptr;
  a.gk = k ? gk : nullptr;
  a.qo = qo;
  a.ko = ko;
  a.status = status;
  a.n = n;
  a.Hq = d.Hq;
  a.Hkv = d.Hkv;
  if (!lay) return launch_type<kGiven>(a, d, rope, st);
  a.prefix_offset = lay->prefix_offset;
  a.row_req = lay->row_req;
  a.row_cand = lay->row_cand;
  a.row_pos = lay->row_pos;
  a.R = lay->n.R;
  a.total = lay->n.total_prefix;
  a.nfed = lay->n.N - lay->n.R;
  return rows ? launch_type<kRows>(a, d, rope, st) : launch_type<kPrefix>(a, d, rope, st);
}

}  // namespace jet
