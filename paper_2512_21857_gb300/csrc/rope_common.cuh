// What the kernels that rotate heads share: angles, 16-byte vectors, host checks
// (internal, not part of the ABI).
#pragma once

#include "adt_common.cuh"
#include "slices.h"

namespace adt {

constexpr int kMaxRows = 1 << 30;               // token numbers, and those of a CTA past the last, take 32 bits
constexpr int64_t kMaxSpan = int64_t{1} << 40;  // elements of all rows with what lies between: their bytes take 64 bits
constexpr int kMaxRotary = 1024;  // cosines and sines of a token: 4 KB of shared memory
constexpr double kTwoPi = 6.283185307179586476925286766559;

__device__ __forceinline__ float to_f32(float x) { return x; }
__device__ __forceinline__ float to_f32(__nv_bfloat16 x) { return __bfloat162float(x); }

// Cosines and sines of `tokens` tokens from n0 on, m included (of p: rot, pos, inv_freq, magnitude).
// row: entries of a token, those from rot / 2 on turn nothing.
template <class Params>
__device__ __forceinline__ void token_angles(const Params& p, int n0, int tokens, float2* cs, int row) {
  for (int i = threadIdx.x; i < row * tokens; i += blockDim.x) {
    const int t = tokens == 1 ? 0 : i / row, pair = i - t * row;
    if (pair >= p.rot / 2) {
      cs[i] = make_float2(1.f, 0.f);
      continue;
    }
    double turns = static_cast<double>(p.pos[n0 + t]) * (1.0 / kTwoPi) * p.inv_freq[pair];
    turns -= rint(turns);
    float s, c;
    sincospif(2.f * static_cast<float>(turns), &s, &c);
    cs[i] = make_float2(c * p.magnitude, s * p.magnitude);
  }
  __syncthreads();
}
template <class Params>
__device__ __forceinline__ void token_angles(const Params& p, int n0, int tokens, float2* cs) {
  token_angles(p, n0, tokens, cs, p.rot / 2);
}

// Eight consecutive elements of a row.
template <typename T>
struct Eight {
  uint4 v[sizeof(T) / 2];
  __device__ __forceinline__ void load(const T* src) {
#pragma unroll
    for (int i = 0; i < static_cast<int>(sizeof(T) / 2); ++i) v[i] = reinterpret_cast<const uint4*>(src)[i];
  }
  __device__ __forceinline__ void get(float (&x)[8]) const {
    if constexpr (sizeof(T) == 2) {
      const uint32_t w[4] = {v[0].x, v[0].y, v[0].z, v[0].w};
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        x[2 * i] = __uint_as_float(w[i] << 16);
        x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
      }
    } else {
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        x[4 * i] = __uint_as_float(v[i].x);
        x[4 * i + 1] = __uint_as_float(v[i].y);
        x[4 * i + 2] = __uint_as_float(v[i].z);
        x[4 * i + 3] = __uint_as_float(v[i].w);
      }
    }
  }
};

__device__ __forceinline__ void put(__nv_bfloat16* dst, const float (&x)[8]) {
  uint32_t w[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const __nv_bfloat162 b = __floats2bfloat162_rn(x[2 * i], x[2 * i + 1]);
    w[i] = *reinterpret_cast<const uint32_t*>(&b);
  }
  *reinterpret_cast<uint4*>(dst) = make_uint4(w[0], w[1], w[2], w[3]);
}

}  // namespace adt
