// The 8-bit prefix cache: where its blocks stand, and the rule of a block's exponent.
// Plain arithmetic, for the kernels and for host checks.
#pragma once

#include <stddef.h>
#include <stdint.h>

#include "jet.h"

#ifdef __CUDACC__
#include <cuda_fp16.h>
#include <cuda_fp8.h>
#define JET_KV_HD __host__ __device__ __forceinline__
#else
#define JET_KV_HD inline
#endif

namespace jet {

constexpr int kKvBlock = JET_KV_BLOCK;  // tokens that share an exponent
// With X in this range every code times 2^X is zero or a normal number of bf16 and
// float32 (the least 2^-9 2^-117 = 2^-126), so reading a cache back rounds nothing.
constexpr int kKvLow = -117, kKvHigh = 119;

// Block b of request r, whose prefix starts at p0, stands at place
// p0 / 64 + r + b: a request's ceil(P / 64) blocks fit before the next one's, as
// floor((p0 + P) / 64) + 1 >= floor(p0 / 64) + ceil(P / 64), and no place depends on
// more than the request's own offset. Places past a request's last block stay unused.
JET_KV_HD int kv_place(int p0, int r, int b) { return p0 / kKvBlock + r + b; }

struct KvSize {
  long long blocks;  // places of blocks
  size_t exp_off;    // the exponent bytes' offset in the buffer
  size_t bytes;      // of one buffer (keys, or values)
};

inline KvSize kv_size(const jet_sizes& n, const jet_dims& d) {
  auto up = [](size_t x) { return (x + 255) & ~size_t(255); };
  KvSize s{};
  s.blocks = n.R > 0 ? (long long)n.total_prefix / kKvBlock + n.R : 0;
  s.exp_off = up(size_t(n.R > 0 ? n.total_prefix : 0) * d.Hkv * d.d);
  s.bytes = s.exp_off + up(size_t(s.blocks) * d.Hkv);
  return s;
}

// Places of n_new appended tokens' blocks: two a request beyond n_new / 64, as they may
// begin and end inside a block
inline long long kv_append_places(const jet_sizes& n, int n_new) {
  return n_new / kKvBlock + 2LL * n.R;
}

// The exponent of a block whose largest finite magnitude has these float32 bits: the
// least X of the range with it <= 448 2^X, 448 = 1.75 2^8
JET_KV_HD int kv_exponent(uint32_t bits) {
  const int x = int(bits >> 23) - 127 - ((bits & 0x7fffffu) <= 0x600000u ? 8 : 7);
  return x < kKvLow ? kKvLow : (x > kKvHigh ? kKvHigh : x);
}

#ifdef __CUDACC__
__device__ __forceinline__ float pow2(int x) {  // 2^x, x in [-126, 127]
  return __uint_as_float(uint32_t(x + 127) << 23);
}

// the scale 2^X of an exponent byte (a byte that no write leaves is taken as the
// nearest that one does)
__device__ __forceinline__ float kv_scale(uint8_t byte) {
  return pow2(min(max(int(byte) - 127, kKvLow), kKvHigh));
}

// the values of the two low bytes' codes, exactly
__device__ __forceinline__ float2 e4m3x2_to_f32(uint32_t codes) {
  const __half2_raw h =
      __nv_cvt_fp8x2_to_halfraw2(static_cast<__nv_fp8x2_storage_t>(codes & 0xffffu), __NV_E4M3);
  return __half22float2(__half2(h));
}
#endif

}  // namespace jet
