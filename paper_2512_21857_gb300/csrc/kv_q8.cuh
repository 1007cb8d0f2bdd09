// The 8-bit cache: what its entry points share (internal, not part of the ABI).
//
// A row (one kv head of one token) is D e4m3 values and a byte s: value = e4m3 *
// 2^(s - 127), s = 255 for a row that is not finite.  A power of two scales
// without a rounding of its own, either way, so that a row has one rounding, to
// 4 significant bits, and its values are exact in bf16.
#pragma once

#include <cuda_fp8.h>

#include "adt_common.cuh"
#include "slices.h"

namespace adt {

constexpr int64_t kMaxCacheStride = int64_t{1} << 40;

// Strides of the 8-bit caches (in elements, which are bytes) and their scales:
// layer, tree, kv head.
struct Q8Strides {
  int64_t cache[3], scale[3];
};

// Host checks of a pair of 8-bit caches with `rows` rows a slice.  Where `written`
// no two slices may share memory.  *cache_span and *scale_span: bytes from the
// first to the last.
inline adt_status check_q8_cache(const void* kc, const void* vc, const void* ks, const void* vs, const Q8Strides& s,
                                 int32_t layers, int32_t B, int32_t Hkv, int32_t D, int64_t rows, bool written,
                                 int64_t* cache_span, int64_t* scale_span) {
  const int64_t counts[3] = {layers, B, Hkv};
  *cache_span = rows * D;
  *scale_span = rows;
  for (int i = 0; i < 3; ++i) {
    if (counts[i] == 1) continue;
    ADT_REQUIRE(s.cache[i] >= rows * D && s.cache[i] % 16 == 0 && s.cache[i] <= kMaxCacheStride);
    ADT_REQUIRE(s.scale[i] >= rows && s.scale[i] <= kMaxCacheStride);
    *cache_span += (counts[i] - 1) * s.cache[i];
    *scale_span += (counts[i] - 1) * s.scale[i];
  }
  ADT_REQUIRE(aligned16(kc) && aligned16(vc));
  ADT_REQUIRE(!spans_overlap(kc, *cache_span, ks, *scale_span) && !spans_overlap(kc, *cache_span, vs, *scale_span) &&
              !spans_overlap(vc, *cache_span, ks, *scale_span) && !spans_overlap(vc, *cache_span, vs, *scale_span));
  if (!written || rows == 0) return ADT_OK;
  // (K and V may lie in one allocation, slices of both in turn.)
  auto diff = [](const void* a, const void* b) {
    return static_cast<int64_t>(reinterpret_cast<uintptr_t>(b) - reinterpret_cast<uintptr_t>(a));
  };
  const int64_t cd = diff(kc, vc), sd = diff(ks, vs);
  ADT_REQUIRE(cd != 0 && !slices_meet(counts, s.cache, rows * D, 0) && !slices_meet(counts, s.cache, rows * D, cd));
  ADT_REQUIRE(sd != 0 && !slices_meet(counts, s.scale, rows, 0) && !slices_meet(counts, s.scale, rows, sd));
  return ADT_OK;
}

// 2^(s - 127); NaN for s = 255.
__device__ __forceinline__ float q8_scale(uint32_t s) {
  return __uint_as_float(s == 0u ? 0x00400000u : s == 255u ? 0x7fc00000u : s << 23);
}

// Two e4m3 values (low byte first) in fp32.
__device__ __forceinline__ float2 e4m3x2_to_f32(uint32_t two) {
  const __half2_raw h = __nv_cvt_fp8x2_to_halfraw2(static_cast<__nv_fp8x2_storage_t>(two), __NV_E4M3);
  return __half22float2(*reinterpret_cast<const __half2*>(&h));
}

// Two fp32 values within +-448 as e4m3, nearest, halves to even.
__device__ __forceinline__ uint32_t f32x2_to_e4m3(float lo, float hi) {
  return __nv_cvt_float2_to_fp8x2(make_float2(lo, hi), __NV_SATFINITE, __NV_E4M3);
}

// The scale of a row whose largest magnitude is `most` (finite): the least e >=
// -120 with most <= 448 * 2^e = 1.75 * 2^(e + 8), as s = e + 127.
__device__ __forceinline__ uint32_t q8_row_scale(float most) {
  const uint32_t bits = __float_as_uint(most);
  const int e = static_cast<int>(bits >> 23) - 127 - 8 + ((bits & 0x7fffffu) > 0x600000u ? 1 : 0);
  return static_cast<uint32_t>(max(e, -120) + 127);
}

}  // namespace adt
