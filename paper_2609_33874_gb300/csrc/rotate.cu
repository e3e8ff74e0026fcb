// The norm of every query and key head and its rotation by position, in one pass over the
// projected queries and keys.
//
// Every element is read and written once, so HBM bounds long inputs and latencies short
// ones. A warp takes 256 elements at a time - one head of 256, two of 128, four of 64 - of
// one token, eight a lane: the two elements of a pair lie in one lane (two groups of four,
// half a rotation apart, or eight in a row), so the rotation needs no shuffle and the norm
// four to five. The angles are common to a token's heads: a block takes kTokens tokens, or
// a part of one token's heads where there are few tokens, and computes each (token, pair)'s
// cosine and sine once into shared memory.
//
// An angle is a 64-bit fraction of a turn, position times frequency modulo 2^64; its
// nearest quarter turn is taken off exactly and the rest, at most an eighth of a turn, is
// rounded to float32 for sincospif: off by less than 2^-25 radians at any position.
#include <algorithm>

#include "jet_device.cuh"
#include "jet_internal.h"

namespace jet {
namespace {

constexpr int kThreads = 256;
constexpr int kWarps = kThreads / 32;
constexpr int kTokens = 4;  // tokens a block takes, at most

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
  int tokens;  // of a block
  int parts;   // blocks that share a token's heads
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

template <typename T>
__device__ __forceinline__ void load4(const T* p, float (&v)[4]) {
  if constexpr (sizeof(T) == 4) {
    const float4 x = *reinterpret_cast<const float4*>(p);
    v[0] = x.x;
    v[1] = x.y;
    v[2] = x.z;
    v[3] = x.w;
  } else {
    const uint2 x = *reinterpret_cast<const uint2*>(p);
    const float2 a = __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162*>(&x.x));
    const float2 b = __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162*>(&x.y));
    v[0] = a.x;
    v[1] = a.y;
    v[2] = b.x;
    v[3] = b.y;
  }
}

template <typename T>
__device__ __forceinline__ void store4(T* p, const float (&v)[4]) {
  if constexpr (sizeof(T) == 4) {
    *reinterpret_cast<float4*>(p) = make_float4(v[0], v[1], v[2], v[3]);
  } else {
    uint2 x;
    *reinterpret_cast<__nv_bfloat162*>(&x.x) = __floats2bfloat162_rn(v[0], v[1]);
    *reinterpret_cast<__nv_bfloat162*>(&x.y) = __floats2bfloat162_rn(v[2], v[3]);
    *reinterpret_cast<uint2*>(p) = x;
  }
}

// 8 elements a lane in two groups of four, v[0] and v[1]. Halves: the groups are half a
// rotation apart in the lanes that rotate, and in a row past them. Pairs: in a row.
template <int DH, int STYLE, int FROM, typename T>
__global__ void __launch_bounds__(kThreads)
norm_rotate_kernel(const RotArgs a, const __grid_constant__ jet_rope rope) {
  pdl_begin();
  constexpr int kLanes = DH / 8;        // lanes of a head
  constexpr int kHeads = 32 / kLanes;   // heads of a warp's step
  __shared__ float2 cs[kTokens][128];
  __shared__ int2 token[kTokens];       // position; key's place, -1 none, -2 no token
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int block = int(blockIdx.x) / a.parts, part = int(blockIdx.x) % a.parts;
  const int n0 = block * a.tokens, count = min(a.tokens, a.n - n0);
  if (warp < count) {
    int pos = 0, fed = -1;
    const bool ok = token_at<FROM>(a, n0 + warp, lane, &pos, &fed);
    if (lane == 0) {
      token[warp] = make_int2(pos, ok ? fed : -2);
      if (!ok) flag(a.status, JET_ERR_DEVICE);
    }
  }
  const int half = rope.rot / 2;
  const int pair = int(threadIdx.x) & 127;
  const uint64_t turn = pair < half ? rope.turn[pair] : 0;
  __syncthreads();
  if (pair < half)
    for (int t = int(threadIdx.x) >> 7; t < count; t += kThreads / 128)
      cs[t][pair] = turn_cos_sin(turn, token[t].x);
  __syncthreads();

  const int hl = lane % kLanes, hs = lane / kLanes;
  int e0, e1, p0;  // the groups' elements, the lane's first pair
  bool rotates;
  if constexpr (STYLE == JET_ROPE_HALVES) {
    rotates = hl < half / 4;
    const int j = hl - half / 4;
    e0 = rotates ? 4 * hl : rope.rot + 8 * j;
    e1 = rotates ? half + 4 * hl : e0 + 4;
    p0 = 4 * hl;
  } else {
    rotates = 8 * hl < rope.rot;
    e0 = 8 * hl;
    e1 = e0 + 4;
    p0 = 4 * hl;
  }
  float gq[2][4], gk[2][4];
#pragma unroll
  for (int i = 0; i < 4; ++i) gq[0][i] = gq[1][i] = gk[0][i] = gk[1][i] = 1.f;
  if (rope.norm) {
    if (a.gq) {
      load4(static_cast<const T*>(a.gq) + e0, gq[0]);
      load4(static_cast<const T*>(a.gq) + e1, gq[1]);
    }
    if (a.gk) {
      load4(static_cast<const T*>(a.gk) + e0, gk[0]);
      load4(static_cast<const T*>(a.gk) + e1, gk[1]);
    }
  }
  const int nq = a.q ? (a.Hq + kHeads - 1) / kHeads : 0;
  const int nk = a.k ? (a.Hkv + kHeads - 1) / kHeads : 0;
  const int steps = nq + nk;
  const int items = count * steps;
  for (int i = part * kWarps + warp; i < items; i += a.parts * kWarps) {
    const int t = i / steps, st = i % steps;
    const int2 tok = token[t];
    const bool is_q = st < nq;
    if (tok.y == -2 || (!is_q && tok.y < 0)) continue;
    const int head = (is_q ? st : st - nq) * kHeads + hs;
    const int H = is_q ? a.Hq : a.Hkv;
    const bool in = head < H;
    const size_t at = (size_t(is_q ? n0 + t : tok.y) * H + (in ? head : H - 1)) * DH;
    const T* x = static_cast<const T*>(is_q ? a.q : a.k) + at;
    float v[2][4];
    load4(x + e0, v[0]);
    load4(x + e1, v[1]);
    if (rope.norm) {
      float ss = 0.f;
#pragma unroll
      for (int j = 0; j < 4; ++j) ss = fmaf(v[0][j], v[0][j], fmaf(v[1][j], v[1][j], ss));
#pragma unroll
      for (int o = kLanes / 2; o > 0; o >>= 1) ss += __shfl_xor_sync(0xffffffffu, ss, o);
      const float inv = 1.f / sqrtf(ss / float(DH) + rope.eps);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        v[0][j] *= inv * (is_q ? gq[0][j] : gk[0][j]);
        v[1][j] *= inv * (is_q ? gq[1][j] : gk[1][j]);
      }
    }
    if (rotates) {
      float2 c[4];
      const float4* tc = reinterpret_cast<const float4*>(&cs[t][p0]);
      *reinterpret_cast<float4*>(&c[0]) = tc[0];
      *reinterpret_cast<float4*>(&c[2]) = tc[1];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        float& x0 = STYLE == JET_ROPE_HALVES ? v[0][j] : v[j >> 1][(2 * j) & 3];
        float& x1 = STYLE == JET_ROPE_HALVES ? v[1][j] : v[j >> 1][(2 * j + 1) & 3];
        const float y0 = x0, y1 = x1;
        x0 = y0 * c[j].x - y1 * c[j].y;
        x1 = y0 * c[j].y + y1 * c[j].x;
      }
    }
    if (in) {
      T* y = static_cast<T*>(is_q ? a.qo : a.ko) + at;
      store4(y + e0, v[0]);
      store4(y + e1, v[1]);
    }
  }
}

template <int FROM, typename T>
cudaError_t launch_from(RotArgs a, const jet_dims& d, const jet_rope& rope, cudaStream_t st) {
  const int heads = 256 / d.d;
  const int steps = (a.q ? (d.Hq + heads - 1) / heads : 0) + (a.k ? (d.Hkv + heads - 1) / heads : 0);
  // few tokens: one a block, its heads over several blocks, a step a warp
  const long long want = 8LL * kPlanSMs;
  a.tokens = a.n >= want * kTokens ? kTokens : 1;
  const int most = (steps + kWarps - 1) / kWarps;
  a.parts = 1;
  if (a.tokens == 1) a.parts = int(std::min<long long>(most, std::max<long long>(1, want / a.n)));
  const long long blocks = ((long long)a.n + a.tokens - 1) / a.tokens * a.parts;
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
