// The prefix K/V cache in 8 bits (Sec. 4.1: the prefix is evaluated once and its
// keys and values are read by every candidate): written, appended to and read back.
//
// 64 tokens of a request share, per key/value head, an exponent X, and an element x is
// held as the e4m3 code of x 2^-X. The scale is a power of two because e4m3 is a
// floating format: a finer scale would gain no digits, only range at the small end
// (the codes reach 2^-15 of the block's largest magnitude before they lose any),
// while products with 2^X are exact. So a code depends on nothing but its element
// and X, reading back rounds nothing in bf16 or float32, and the attention takes the
// scales out of its sums.
//
// All three are streams: each element is read and written once, and HBM bounds them
// (1.38e9 bf16 elements of d 256 written: 573 us, 7.2 TB/s; 172e6 read back: 77 us, 6.7 TB/s).
// One CTA works on one (block of 64 tokens, keys or values, head) at a time: its
// elements stay in registers between their maximum and their codes.
#include <algorithm>

#include "jet_device.cuh"
#include "jet_internal.h"
#include "kv_cache.h"

namespace jet {
namespace {

constexpr int kThreads = 256;

struct KvArgs {
  const int32_t* prefix_offset;
  const int32_t* start;       // append: a request's tokens that the cache holds
  const int32_t* new_offset;  // append: its new tokens, in rows of k and v
  const void* x[2];           // k, v: rows [tokens, Hkv, DH]
  void* out[2];               // read back: k, v
  uint8_t* codes[2];          // the caches' codes and exponent bytes
  uint8_t* exps[2];
  int R, Hkv, total_prefix;
  int rows;                   // rows of k and v
  int each;                   // written: (keys or values, head) pairs that a CTA takes
  int* status;
};

// What one CTA works on: tokens [t0, t1) of block b of request r, found in rows row0 ..
// of k and v.
struct KvSpan {
  int r, p0, b, t0, t1, row0;
};

// The request and block of the CTA's place `slot`: with `off` the requests' row offsets,
// request r has the places [off[r] / 64 + per r, off[r + 1] / 64 + per (r + 1)).
// Appended tokens may begin inside a block, so they touch up to one block more than as
// many tokens from a block's start: two places a request instead of one. The threads
// try the requests 256 at a time, which costs one memory latency; a search by halves
// would cost one a step. (The places grow with the requests too, so many short requests pay
// for it: with 100 tokens each in two kv heads of 128, one more token appended takes 7.2 us
// for 256 requests, 18.5 for 1,024, 114 for 4,096 and 1,330 for 16,384, and the write of
// all 8.9, 31, 122 and 812, of which the bytes are 6, 23, 92 and 370.)
// False for a place without tokens.
template <bool APPEND>
__device__ __forceinline__ bool find_span(const KvArgs& a, int slot, KvSpan* s) {
  constexpr int per = APPEND ? 2 : 1;
  const int32_t* off = APPEND ? a.new_offset : a.prefix_offset;
  __shared__ int claimed;
  __shared__ KvSpan span;
  if (threadIdx.x == 0) claimed = -1;
  __syncthreads();
  for (int r = threadIdx.x; r < a.R; r += kThreads) {
    const int o0 = off[r], o1 = off[r + 1];
    const int p0 = APPEND ? a.prefix_offset[r] : o0;
    const int P = (APPEND ? a.prefix_offset[r + 1] : o1) - p0;
    const int first = APPEND ? a.start[r] : 0;
    const int count = o1 - o0;
    // (compared so that no sum of words leaves 32 bits)
    if (o0 < 0 || o1 < o0 || o1 > a.rows || p0 < 0 || p0 > a.total_prefix || P < 0 ||
        P > a.total_prefix - p0 || first < 0 || first > P || count > P - first) {
      if (slot == 0) flag(a.status, JET_ERR_DEVICE);  // the request is left out
      continue;
    }
    const int base = o0 / kKvBlock + per * r;
    if (slot < base || slot >= o1 / kKvBlock + per * (r + 1)) continue;
    const int b = first / kKvBlock + (slot - base);
    const int t0 = max(first, b * kKvBlock), t1 = min(first + count, (b + 1) * kKvBlock);
    if (t0 < t1 && atomicCAS(&claimed, -1, r) == -1)
      span = KvSpan{r, p0, b, t0, t1, o0 + (t0 - first)};
  }
  __syncthreads();
  if (claimed < 0) return false;
  *s = span;
  return true;
}

// (an index would copy the arguments to the stack)
template <typename P>
__device__ __forceinline__ P pick(P const (&p)[2], int kv) {
  return kv ? p[1] : p[0];
}

__device__ __forceinline__ uint32_t encode2(float a, float b) {
  return __nv_cvt_float2_to_fp8x2(make_float2(a, b), __NV_SATFINITE, __NV_E4M3);
}

// one element of a 16-byte piece as float32
template <typename T>
__device__ __forceinline__ float element(const uint4& v, int i);
template <>
__device__ __forceinline__ float element<float>(const uint4& v, int i) {
  return __uint_as_float(i == 0 ? v.x : i == 1 ? v.y : i == 2 ? v.z : v.w);
}
template <>
__device__ __forceinline__ float element<__nv_bfloat16>(const uint4& v, int i) {
  const uint32_t w = (i >> 1) == 0 ? v.x : (i >> 1) == 1 ? v.y : (i >> 1) == 2 ? v.z : v.w;
  return __uint_as_float((i & 1) ? (w & 0xffff0000u) : (w << 16));
}

// the larger magnitude of `top` and a piece's finite elements, as float32 bits
template <typename T>
__device__ __forceinline__ uint32_t top_finite(uint32_t top, const uint4& v) {
#pragma unroll
  for (int i = 0; i < int(16 / sizeof(T)); ++i) {
    const uint32_t u = __float_as_uint(element<T>(v, i)) & 0x7fffffffu;
    top = max(top, u >= 0x7f800000u ? 0u : u);
  }
  return top;
}

// the largest magnitude of a thread's pieces, as float32 bits; the bits of bf16's
// magnitudes are compared two at once
template <typename T, int N>
__device__ __forceinline__ uint32_t top_bits(const uint4 (&v)[N]) {
  constexpr bool bf16 = sizeof(T) == 2;
  uint32_t top = 0;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const uint32_t w[4] = {v[i].x, v[i].y, v[i].z, v[i].w};
#pragma unroll
    for (int q = 0; q < 4; ++q)
      top = bf16 ? __vmaxu2(top, w[q] & 0x7fff7fffu) : max(top, w[q] & 0x7fffffffu);
  }
  return bf16 ? max(top & 0xffff0000u, top << 16) : top;
}

// the CTA's largest v; calls take the two halves of `part` in turn, so that a barrier
// stands between a read of one and its next write
__device__ __forceinline__ uint32_t block_max(uint32_t v, int* turn) {
  __shared__ uint32_t part[2][kThreads / 32];
  uint32_t* mine = part[*turn];
  *turn ^= 1;
  v = __reduce_max_sync(0xffffffffu, v);
  if ((threadIdx.x & 31) == 0) mine[threadIdx.x >> 5] = v;
  __syncthreads();
  return __reduce_max_sync(0xffffffffu, mine[threadIdx.x % (kThreads / 32)]);
}

// A CTA takes `each` of a block's 2 Hkv (keys or values, head) pairs, one after another.
// The launch bounds are the CTAs an SM that hide the loads; left to itself the compiler
// takes more registers where that costs (0.69e9 bf16 elements of d 64 345 us instead of
// 304; float32: 0.52e9 of d 256 677 instead of 485, of d 128 563 instead of 492, of d 64
// 376 instead of 363; 256 pieces of 100 - 700 tokens appended, float32 d 256 257 instead of
// 156, d 128 214 instead of 155). Appends of d 64 spill within it and lose a little: 94.8
// instead of 92.4, bf16 77 instead of 74.
template <typename T, int DH, bool APPEND>
__global__ void __launch_bounds__(kThreads, DH == 256 ? (sizeof(T) == 2 ? 4 : 3) : DH == 128 ? 5 : 8)
kv_quantize_kernel(const KvArgs a) {
  pdl_begin();
  constexpr int kPer = 16 / int(sizeof(T));          // elements of a 16-byte piece
  constexpr int kRow = DH / kPer;                    // pieces of a token
  constexpr int kMine = kKvBlock * kRow / kThreads;  // of a thread
  constexpr int kStep = kThreads / kRow;             // tokens between a thread's pieces
  const int groups = (2 * a.Hkv + a.each - 1) / a.each;
  const int first = int(blockIdx.x % groups) * a.each;
  KvSpan s;
  if (!find_span<APPEND>(a, blockIdx.x / groups, &s)) return;
  const int nt = s.t1 - s.t0, tid = threadIdx.x;
  const int j0 = tid / kRow, c0 = tid % kRow * kPer;
  const size_t step = size_t(a.Hkv) * DH;
  int turn = 0;
#pragma unroll 1
  for (int u = first; u < min(first + a.each, 2 * a.Hkv); ++u) {
    const int kv = u >= a.Hkv, h = u - kv * a.Hkv;
    uint8_t* exp = pick(a.exps, kv) + size_t(kv_place(s.p0, s.r, s.b)) * a.Hkv + h;
    // a block begun before: the exponent of the tokens it holds
    const bool begun = APPEND && s.t0 > s.b * kKvBlock;
    const int held = begun ? min(max(int(*exp) - 127, kKvLow), kKvHigh) : kKvLow;
    const T* x = static_cast<const T*>(pick(a.x, kv)) + (size_t(s.row0 + j0) * a.Hkv + h) * DH + c0;
    uint4 v[kMine];
#pragma unroll
    for (int i = 0; i < kMine; ++i) {
      v[i] = make_uint4(0u, 0u, 0u, 0u);
      if (j0 + i * kStep < nt) v[i] = *reinterpret_cast<const uint4*>(x + i * kStep * step);
    }
    uint32_t top = block_max(top_bits<T>(v), &turn);
    const bool finite = top < 0x7f800000u;
    if (!finite) {
      top = 0;
#pragma unroll
      for (int i = 0; i < kMine; ++i) top = top_finite<T>(top, v[i]);
      top = block_max(top, &turn);
    }
    const int X = max(kv_exponent(top), held);
    const float inv = pow2(-X);
    uint8_t* codes = pick(a.codes, kv) + (size_t(s.p0 + s.t0 + j0) * a.Hkv + h) * DH + c0;
#pragma unroll
    for (int i = 0; i < kMine; ++i) {
      if (j0 + i * kStep >= nt) continue;
      uint32_t w[kPer / 4];
#pragma unroll
      for (int q = 0; q < kPer / 4; ++q) {
        const float f0 = element<T>(v[i], 4 * q), f1 = element<T>(v[i], 4 * q + 1);
        const float f2 = element<T>(v[i], 4 * q + 2), f3 = element<T>(v[i], 4 * q + 3);
        w[q] = encode2(f0 * inv, f1 * inv) | encode2(f2 * inv, f3 * inv) << 16;
        if (!finite) {  // the format has no infinity: it is held as NaN too
          if (isinf(f0)) w[q] |= 0x7fu;
          if (isinf(f1)) w[q] |= 0x7f00u;
          if (isinf(f2)) w[q] |= 0x7f0000u;
          if (isinf(f3)) w[q] |= 0x7f000000u;
        }
      }
      uint8_t* to = codes + i * kStep * step;
      if constexpr (kPer == 8)
        *reinterpret_cast<uint2*>(to) = make_uint2(w[0], w[1]);
      else
        *reinterpret_cast<uint32_t*>(to) = w[0];
    }
    if (begun && X > held) {
      // the tokens before, rounded again (codes that stay normal keep their values)
      const float f = pow2(max(held - X, -126));
      uint8_t* old = pick(a.codes, kv) + (size_t(s.p0 + s.b * kKvBlock) * a.Hkv + h) * DH;
      for (int e = tid; e < (s.t0 - s.b * kKvBlock) * (DH / 8); e += kThreads) {
        uint2* at = reinterpret_cast<uint2*>(old + (e / (DH / 8)) * step + 8 * (e % (DH / 8)));
        uint2 w = *at;
#pragma unroll
        for (int q = 0; q < 2; ++q) {
          uint32_t& y = q ? w.y : w.x;
          const float2 lo = e4m3x2_to_f32(y), hi = e4m3x2_to_f32(y >> 16);
          y = encode2(lo.x * f, lo.y * f) | encode2(hi.x * f, hi.y * f) << 16;
        }
        *at = w;
      }
    }
    if (tid == 0) *exp = uint8_t(X + 127);  // block_max: every thread has read what it held
  }
}

template <typename T, int DH>
__global__ void __launch_bounds__(kThreads) kv_dequantize_kernel(const KvArgs a) {
  pdl_begin();
  constexpr int kPer = 16 / int(sizeof(T));
  constexpr int kRow = DH / kPer;
  constexpr int kMine = kKvBlock * kRow / kThreads;
  constexpr int kStep = kThreads / kRow;
  const int h = blockIdx.x % a.Hkv, rest = blockIdx.x / a.Hkv, kv = rest & 1;
  KvSpan s;
  if (!find_span<false>(a, rest >> 1, &s)) return;
  const int nt = s.t1 - s.t0, tid = threadIdx.x;
  const int j0 = tid / kRow, c0 = tid % kRow * kPer;
  const size_t step = size_t(a.Hkv) * DH;
  const uint8_t held = pick(a.exps, kv)[size_t(kv_place(s.p0, s.r, s.b)) * a.Hkv + h];
  const float f = kv_scale(held);
  const size_t at = (size_t(s.p0 + s.t0 + j0) * a.Hkv + h) * DH + c0;
  const uint8_t* codes = pick(a.codes, kv) + at;
  T* out = static_cast<T*>(pick(a.out, kv)) + at;
  uint32_t w[kMine][kPer / 4];
#pragma unroll
  for (int i = 0; i < kMine; ++i) {
    if (j0 + i * kStep >= nt) continue;
    const uint8_t* from = codes + i * kStep * step;
    if constexpr (kPer == 8) {
      const uint2 y = *reinterpret_cast<const uint2*>(from);
      w[i][0] = y.x;
      w[i][1] = y.y;
    } else {
      w[i][0] = *reinterpret_cast<const uint32_t*>(from);
    }
  }
#pragma unroll
  for (int i = 0; i < kMine; ++i) {
    if (j0 + i * kStep >= nt) continue;
    uint32_t y[4];
#pragma unroll
    for (int q = 0; q < kPer / 4; ++q) {
      const float2 lo = e4m3x2_to_f32(w[i][q]), hi = e4m3x2_to_f32(w[i][q] >> 16);
      if constexpr (kPer == 8) {
        const __nv_bfloat162 p = __floats2bfloat162_rn(lo.x * f, lo.y * f);
        const __nv_bfloat162 r = __floats2bfloat162_rn(hi.x * f, hi.y * f);
        y[2 * q] = *reinterpret_cast<const uint32_t*>(&p);
        y[2 * q + 1] = *reinterpret_cast<const uint32_t*>(&r);
      } else {
        y[0] = __float_as_uint(lo.x * f);
        y[1] = __float_as_uint(lo.y * f);
        y[2] = __float_as_uint(hi.x * f);
        y[3] = __float_as_uint(hi.y * f);
      }
    }
    *reinterpret_cast<uint4*>(out + i * kStep * step) = make_uint4(y[0], y[1], y[2], y[3]);
  }
}

KvArgs kv_args(const jet_layout& lay, const jet_dims& d, const void* k8, const void* v8,
               int* status) {
  KvArgs a{};
  const KvSize z = kv_size(lay.n, d);
  const void* buf[2] = {k8, v8};
  for (int i = 0; i < 2; ++i) {
    a.codes[i] = static_cast<uint8_t*>(const_cast<void*>(buf[i]));
    a.exps[i] = a.codes[i] + z.exp_off;
  }
  a.prefix_offset = lay.prefix_offset;
  a.R = lay.n.R;
  a.Hkv = d.Hkv;
  a.total_prefix = lay.n.total_prefix;
  a.rows = lay.n.total_prefix;
  a.status = status;
  return a;
}

// How many pairs a CTA takes: four of bf16 heads of up to 128 elements, whose CTAs would
// else be gone before their launch is paid (one, two, four pairs: 1.38e9 elements of d 128
// 646, 596, 579 us, 0.69e9 of d 64 369, 323, 304), two of others (bf16 d 256 573, 570,
// 574; 0.52e9 of float32 d 256 479, 478, 485) and of an append, whose blocks are mostly
// partial (16 pieces of 100 to 700 tokens 8.7, 8.2, 10.2); but no more than leaves 512
// CTAs, three or four an SM.
template <typename T, bool APPEND>
int pairs_each(int DH, long long pairs) {
  const long long most = sizeof(T) == 2 && DH <= 128 && !APPEND ? 4 : 2;
  return int(std::min(most, std::max(1LL, pairs / 512)));
}

template <typename T, bool APPEND>
cudaError_t launch_quantize(KvArgs a, int DH, long long places, cudaStream_t st) {
  a.each = pairs_each<T, APPEND>(DH, places * 2 * a.Hkv);
  const dim3 grid(unsigned(places * ((2 * a.Hkv + a.each - 1) / a.each)));
  if (DH == 64) return launch_pdl(kv_quantize_kernel<T, 64, APPEND>, grid, dim3(kThreads), 0, st, a);
  if (DH == 128)
    return launch_pdl(kv_quantize_kernel<T, 128, APPEND>, grid, dim3(kThreads), 0, st, a);
  return launch_pdl(kv_quantize_kernel<T, 256, APPEND>, grid, dim3(kThreads), 0, st, a);
}

template <typename T>
cudaError_t launch_dequantize(const KvArgs& a, int DH, long long places, cudaStream_t st) {
  const dim3 grid(unsigned(places * 2 * a.Hkv));
  if (DH == 64) return launch_pdl(kv_dequantize_kernel<T, 64>, grid, dim3(kThreads), 0, st, a);
  if (DH == 128) return launch_pdl(kv_dequantize_kernel<T, 128>, grid, dim3(kThreads), 0, st, a);
  return launch_pdl(kv_dequantize_kernel<T, 256>, grid, dim3(kThreads), 0, st, a);
}

}  // namespace

cudaError_t launch_kv_quantize(const jet_layout& lay, const jet_dims& d, const void* k,
                               const void* v, void* k8, void* v8, int* status, cudaStream_t st) {
  KvArgs a = kv_args(lay, d, k8, v8, status);
  a.x[0] = k;
  a.x[1] = v;
  const long long places = kv_size(lay.n, d).blocks;
  return d.dtype == JET_DTYPE_BF16 ? launch_quantize<__nv_bfloat16, false>(a, d.d, places, st)
                                   : launch_quantize<float, false>(a, d.d, places, st);
}

cudaError_t launch_kv_append(const jet_layout& lay, const jet_dims& d, const int32_t* start,
                             const int32_t* new_offset, int n_new, const void* k, const void* v,
                             void* k8, void* v8, int* status, cudaStream_t st) {
  KvArgs a = kv_args(lay, d, k8, v8, status);
  a.x[0] = k;
  a.x[1] = v;
  a.start = start;
  a.new_offset = new_offset;
  a.rows = n_new;
  const long long places = kv_append_places(lay.n, n_new);
  return d.dtype == JET_DTYPE_BF16 ? launch_quantize<__nv_bfloat16, true>(a, d.d, places, st)
                                   : launch_quantize<float, true>(a, d.d, places, st);
}

cudaError_t launch_kv_dequantize(const jet_layout& lay, const jet_dims& d, const void* k8,
                                 const void* v8, void* k, void* v, int* status, cudaStream_t st) {
  KvArgs a = kv_args(lay, d, k8, v8, status);
  a.out[0] = k;
  a.out[1] = v;
  const long long places = kv_size(lay.n, d).blocks;
  return d.dtype == JET_DTYPE_BF16 ? launch_dequantize<__nv_bfloat16>(a, d.d, places, st)
                                   : launch_dequantize<float>(a, d.d, places, st);
}

}  // namespace jet
