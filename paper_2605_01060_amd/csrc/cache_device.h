// Device-side helpers of the kernels that go through a cache's pages.
#pragma once

#include "cache.h"
#include "device_common.h"

namespace surge {

// Bytes of a page's part of one key head, and where the parts of a token lie
// in it: codes of keys and values, then scales.
template <int DH>
struct PageLayout {
  static constexpr int CODES = DH / 2, SCALES = DH / 32;
  static __device__ __forceinline__ int64_t head_bytes(int shift) {
    return (int64_t)(2 * (CODES + SCALES)) << shift;
  }
  static __device__ __forceinline__ uint32_t codes(int shift, int slot, int value) {
    return ((uint32_t)value << shift) * CODES + (uint32_t)slot * CODES;
  }
  static __device__ __forceinline__ uint32_t scales(int shift, int slot, int value) {
    return (2u << shift) * CODES + ((uint32_t)value << shift) * SCALES + (uint32_t)slot * SCALES;
  }
};

// A scale's float: 2^(byte - 127); 255, which marks 32 values of which one was
// not finite, makes every value that is decoded with it a NaN.
__device__ __forceinline__ float scale_of(uint32_t byte) { return __uint_as_float(byte << 23); }
constexpr uint32_t NAN_SCALE = 255;

// Eight codes as bf16, exactly: a code has two significant bits, a scale is a
// power of two.
__device__ __forceinline__ bf16x8 decode8(uint32_t codes, float scale) {
  const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 0);
  const bf16x2 b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 1);
  const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 2);
  const bf16x2 d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 3);
  bf16x8 v;
  v[0] = a[0], v[1] = a[1], v[2] = b[0], v[3] = b[1];
  v[4] = c[0], v[5] = c[1], v[6] = d[0], v[7] = d[1];
  return v;
}

__device__ __forceinline__ int length_of(const CacheView& c, int seq) {
  return min(max(c.lengths[seq], 0), c.max_length);
}

}  // namespace surge
