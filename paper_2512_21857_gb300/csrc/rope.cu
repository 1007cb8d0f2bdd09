// adt_rope_freqs, adt_rope_qkv: rotary positions.
//
// Pair p of a head at position t turns by t * inv_freq[p] radians:
//   (a, b) -> (a c - b s, b c + a s),  c = m cos(t f), s = m sin(t f).
// The angle is formed in 64 bits as a number of turns, t * f / (2 pi), and only
// its fraction goes on to fp32: at t = 10^6 the angle of a pair with f = 1 has
// 20 bits before the point, so that in fp32 the cosine would be off by 0.03.
//
// Bound by HBM where there are many tokens: 16384 of 32 / 32 heads x 128 124 us
// for 805 MB (119 at the measured copy rate); 4096 of 32 / 8 heads 19 to 20 us for
// 101 MB (14.9; the angles' 64-bit chain is a fifth of a CTA's time there), 26.2
// with one unit a thread; and by a launch (2 us) up to about 300.  Halves spill at
// the register limits that their CTAs an SM leave them: 48 bytes a thread for bf16
// rows (64 registers), 32 for fp32 (80).
//
// A CTA takes one token or a few (and, where there are few tokens, a share of
// their heads): one thread a pair makes the cosines and sines once, in shared
// memory, and every head of the token uses them.
#include <math.h>

#include "adt_common.cuh"
#include "rope_common.cuh"

namespace {

using adt::Eight;
using adt::kMaxRotary;
using adt::kMaxRows;
using adt::kMaxSpan;
using adt::kTwoPi;
using adt::put;
using adt::spans_overlap;
using adt::to_f32;
using adt::token_angles;

constexpr int kThreads = 256;

struct RopeParams {
  const void* in[3];        // rows of q, k, v
  int64_t ld[3];            // row strides in elements
  __nv_bfloat16* out[3];    // [N][heads][D]
  int heads[3];
  const int32_t* pos;
  const double* inv_freq;
  float magnitude;
  int D, rot, interleaved;
};

// Moves 16-byte vectors.  A unit is what a thread rotates at a time: eight
// pairs of a half layout (two vectors of its row), four pairs side by side
// (one), or eight copied elements.  A thread keeps its place within the heads,
// so that its cosines and sines are read once, and its first units are on
// their way while the angles are made.
template <typename T, bool kInterleaved>
__global__ void __launch_bounds__(kThreads, sizeof(T) == 2 ? 4 : 3)
    rope_vec_kernel(const RopeParams p, int N, int tokens, int lanes, int units) {
  extern __shared__ float2 cs[];
  constexpr int kBatch = 2;
  constexpr int kVecs = kInterleaved ? 1 : 2;
  adt::pdl_wait_then_release();
  const int n0 = blockIdx.x * tokens, here = min(tokens, N - n0);
  const int tok = threadIdx.x / lanes, lane = threadIdx.x - tok * lanes;
  const bool active = tok < here;
  const int64_t n = n0 + (active ? tok : 0);
  const int half = p.rot / 2;
  const int per_pass = lanes / units, hl = lane / units, u = lane - hl * units;
  const bool turned = kInterleaved ? u * 8 < p.rot : u * 16 < p.rot;
  // First element of the unit, and of its second vector.
  const int e0 = kInterleaved || turned ? u * 8 : p.rot + (u - p.rot / 16) * 8, e1 = e0 + half;
  const int heads = p.heads[0] + p.heads[1];
  const int h0 = static_cast<int>(blockIdx.y) * per_pass + hl, hstep = static_cast<int>(gridDim.y) * per_pass;
  const int v0 = static_cast<int>(blockIdx.y) * lanes + lane, vstep = static_cast<int>(gridDim.y) * lanes;
  const int vectors = active ? p.heads[2] * p.D / 8 : 0;
  const int most = active && hl < per_pass ? heads : 0;

  Eight<T> x[kBatch][kVecs], v[kBatch];
  auto at = [&](int h, const T** src, __nv_bfloat16** dst) {
    const bool q = h < p.heads[0];
    const int hh = q ? h : h - p.heads[0];
    *src = static_cast<const T*>(q ? p.in[0] : p.in[1]) + n * (q ? p.ld[0] : p.ld[1]) + hh * p.D;
    *dst = (q ? p.out[0] : p.out[1]) + (n * (q ? p.heads[0] : p.heads[1]) + hh) * p.D;
  };
  auto fetch = [&](int h, int vi) {
#pragma unroll
    for (int k = 0; k < kBatch; ++k) {
      const T* src;
      __nv_bfloat16* dst;
      if (h + k * hstep < most) {
        at(h + k * hstep, &src, &dst);
        x[k][0].load(src + e0);
        if (!kInterleaved && turned) x[k][kVecs - 1].load(src + e1);
      }
      if (vi + k * vstep < vectors)
        v[k].load(static_cast<const T*>(p.in[2]) + n * p.ld[2] + static_cast<int64_t>(vi + k * vstep) * 8);
    }
  };
  fetch(h0, v0);
  token_angles(p, n0, here, cs);
  constexpr int kPairs = kInterleaved ? 4 : 8;
  float c[kPairs], s[kPairs];
  if (turned && active) {
#pragma unroll
    for (int i = 0; i < kPairs; ++i) {
      const float2 z = cs[tok * half + u * kPairs + i];
      c[i] = z.x;
      s[i] = z.y;
    }
  }
  int h = h0, vi = v0;
  while (h < most || vi < vectors) {
#pragma unroll
    for (int k = 0; k < kBatch; ++k) {
      if (h + k * hstep < most) {
        const T* src;
        __nv_bfloat16* dst;
        at(h + k * hstep, &src, &dst);
        float a[8], b[8], y[8], z[8];
        x[k][0].get(a);
        if (!turned) {
          put(dst + e0, a);
        } else if constexpr (kInterleaved) {
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            y[2 * i] = a[2 * i] * c[i] - a[2 * i + 1] * s[i];
            y[2 * i + 1] = a[2 * i + 1] * c[i] + a[2 * i] * s[i];
          }
          put(dst + e0, y);
        } else {
          x[k][1].get(b);
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            y[i] = a[i] * c[i] - b[i] * s[i];
            z[i] = b[i] * c[i] + a[i] * s[i];
          }
          put(dst + e0, y);
          put(dst + e1, z);
        }
      }
      if (vi + k * vstep < vectors) {
        float a[8];
        v[k].get(a);
        put(p.out[2] + n * p.heads[2] * p.D + static_cast<int64_t>(vi + k * vstep) * 8, a);
      }
    }
    h += kBatch * hstep;
    vi += kBatch * vstep;
    fetch(h, vi);
  }
}

// Rotary sizes whose vectors would hold parts of both halves, or turned and
// copied elements: heads go through shared memory in fp32, loaded as vectors, and
// a thread takes two neighbouring elements with their partners, wherever they
// lie, at a time (4-byte stores of a warp are a row's 128 bytes).  Straight from
// global memory one element at a time 4096 tokens of 32 / 8 heads x 128 with 50
// turned took 56 us, so 34 (14.9 at the copy rate: every element passes through
// shared memory in fp32, and stores are 4 bytes a thread).
constexpr int kStaged = 4096;  // elements: 16 KB

template <typename T>
__global__ void __launch_bounds__(kThreads) rope_staged_kernel(const RopeParams p, int group) {
  extern __shared__ float2 shared[];
  constexpr int kBatch = 4;
  float2* cs = shared;
  float* rows = reinterpret_cast<float*>(shared + ((p.rot / 2 + 1) & ~1));
  adt::pdl_wait_then_release();
  const int64_t n = blockIdx.x;
  const int half = p.rot / 2, heads = p.heads[0] + p.heads[1], vpr = p.D / 8;
  const T* q = static_cast<const T*>(p.in[0]) + n * p.ld[0];
  const T* k = static_cast<const T*>(p.in[1]) + n * p.ld[1];
  auto head = [&](int h) { return h < p.heads[0] ? q + h * p.D : k + (h - p.heads[0]) * p.D; };
  // Place within a head: of the vectors loaded, and of the elements turned.
  const int lh = threadIdx.x / vpr, lv = threadIdx.x - lh * vpr, lstep = kThreads / vpr;
  const int twos = p.D / 2, th = threadIdx.x / twos, e = 2 * (threadIdx.x - th * twos), tstep = kThreads / twos;
  float c[2], s[2];  // y = x c + partner s
  int partner[2];
  for (int h0 = blockIdx.y * group; h0 < heads; h0 += gridDim.y * group) {
    const int here = min(group, heads - h0);
    for (int h = lh < lstep ? lh : here; h < here; h += kBatch * lstep) {
      Eight<T> v[kBatch];
#pragma unroll
      for (int k = 0; k < kBatch; ++k)
        if (h + k * lstep < here) v[k].load(head(h0 + h + k * lstep) + lv * 8);
#pragma unroll
      for (int k = 0; k < kBatch; ++k) {
        if (h + k * lstep >= here) break;
        float x[8];
        v[k].get(x);
        float4* to = reinterpret_cast<float4*>(rows + (h + k * lstep) * p.D + lv * 8);
        to[0] = make_float4(x[0], x[1], x[2], x[3]);
        to[1] = make_float4(x[4], x[5], x[6], x[7]);
      }
    }
    if (h0 == static_cast<int>(blockIdx.y) * group) {
      token_angles(p, blockIdx.x, 1, cs);  // (ends with a barrier)
#pragma unroll
      for (int w = 0; w < 2; ++w) {
        const int at = e + w, pair = p.interleaved ? at >> 1 : at < half ? at : at - half;
        const bool turned = at < p.rot, first = p.interleaved ? w == 0 : at < half;
        const float2 z = turned ? cs[pair] : make_float2(1.f, 0.f);
        c[w] = z.x;
        s[w] = first ? -z.y : z.y;
        partner[w] = !turned ? at : p.interleaved ? at ^ 1 : first ? at + half : at - half;
      }
    } else {
      __syncthreads();
    }
    for (int h = th < tstep ? th : here; h < here; h += tstep) {
      const float* row = rows + h * p.D;
      const float2 x = *reinterpret_cast<const float2*>(row + e);
      // (A copied element is its own partner: not multiplied, it may be infinite.)
      const float y0 = partner[0] == e ? x.x : x.x * c[0] + row[partner[0]] * s[0];
      const float y1 = partner[1] == e + 1 ? x.y : x.y * c[1] + row[partner[1]] * s[1];
      const int hh = h0 + h;
      __nv_bfloat16* dst = hh < p.heads[0] ? p.out[0] + (n * p.heads[0] + hh) * p.D
                                           : p.out[1] + (n * p.heads[1] + hh - p.heads[0]) * p.D;
      *reinterpret_cast<__nv_bfloat162*>(dst + e) = __floats2bfloat162_rn(y0, y1);
    }
    __syncthreads();  // before the rows are overwritten
  }
  const T* in = static_cast<const T*>(p.in[2]) + n * p.ld[2];
  __nv_bfloat16* out = p.out[2] + n * p.heads[2] * p.D;
  for (int i = blockIdx.y * kThreads + threadIdx.x; i < p.heads[2] * vpr; i += gridDim.y * kThreads) {
    Eight<T> v;
    float x[8];
    v.load(in + i * 8);
    v.get(x);
    put(out + i * 8, x);
  }
}

// One pair or one copied element at a time: any even rotary_dim, any head
// size, row stride and alignment.  4096 tokens of 32 / 8 heads x 128 in rows off a
// 16-byte boundary take 41 us (19 to 20 as vectors, 14.9 at the copy rate): loads
// and stores of 2 bytes a thread.
template <typename T>
__global__ void __launch_bounds__(kThreads) rope_scalar_kernel(const RopeParams p) {
  __shared__ float2 cs[kMaxRotary / 2];
  adt::pdl_wait_then_release();
  const int n = blockIdx.x;
  token_angles(p, n, 1, cs);
  const int half = p.rot / 2, units = p.D - half;
  for (int x = 0; x < 3; ++x) {
    const T* in = static_cast<const T*>(p.in[x]) + n * p.ld[x];
    __nv_bfloat16* out = p.out[x] + static_cast<int64_t>(n) * p.heads[x] * p.D;
    const int count = p.heads[x] * (x < 2 ? units : p.D);
    for (int i = blockIdx.y * kThreads + threadIdx.x; i < count; i += gridDim.y * kThreads) {
      if (x == 2) {
        out[i] = __float2bfloat16(to_f32(in[i]));
        continue;
      }
      const int h = i / units, u = i - h * units;
      const T* row = in + h * p.D;
      __nv_bfloat16* dst = out + h * p.D;
      if (u >= half) {
        dst[u + half] = __float2bfloat16(to_f32(row[u + half]));
        continue;
      }
      const int ia = p.interleaved ? 2 * u : u, ib = p.interleaved ? 2 * u + 1 : u + half;
      const float a = to_f32(row[ia]), b = to_f32(row[ib]), c = cs[u].x, s = cs[u].y;
      dst[ia] = __float2bfloat16(a * c - b * s);
      dst[ib] = __float2bfloat16(b * c + a * s);
    }
  }
}

}  // namespace

extern "C" {

adt_status adt_rope_freqs(const adt_rope_params* params, double* inv_freq, float* magnitude) {
  ADT_REQUIRE(params && inv_freq && magnitude);
  const adt_rope_params& r = *params;
  ADT_REQUIRE(r.rotary_dim >= 2 && r.rotary_dim % 2 == 0 && r.rotary_dim <= kMaxRotary);
  ADT_REQUIRE(isfinite(r.theta) && r.theta >= 1.0);
  ADT_REQUIRE(r.scaling >= ADT_ROPE_NONE && r.scaling <= ADT_ROPE_BY_PARTS);
  const bool scaled = r.scaling != ADT_ROPE_NONE;
  ADT_REQUIRE(!scaled || (isfinite(r.factor) && r.factor >= 1.0));
  ADT_REQUIRE(r.scaling != ADT_ROPE_NTK || r.rotary_dim > 2);
  ADT_REQUIRE(r.scaling != ADT_ROPE_BY_PARTS ||
              (r.orig_len >= 1 && r.turns_lo >= 0.0 && r.turns_hi > r.turns_lo && isfinite(r.turns_hi)));
  const int R = r.rotary_dim;
  const double theta = r.scaling == ADT_ROPE_NTK ? r.theta * pow(r.factor, static_cast<double>(R) / (R - 2)) : r.theta;
  for (int i = 0; i < R / 2; ++i) {
    double f = pow(theta, -2.0 * i / R);
    if (r.scaling == ADT_ROPE_LINEAR) f /= r.factor;
    if (r.scaling == ADT_ROPE_BY_PARTS) {
      const double turns = r.orig_len * f / kTwoPi;
      const double keep = fmin(1.0, fmax(0.0, (turns - r.turns_lo) / (r.turns_hi - r.turns_lo)));
      f *= keep + (1.0 - keep) / r.factor;
    }
    inv_freq[i] = f;
  }
  *magnitude = r.scaling == ADT_ROPE_BY_PARTS ? static_cast<float>(0.1 * log(r.factor) + 1.0) : 1.f;
  return ADT_OK;
}

adt_status adt_rope_qkv(const void* q, int64_t ld_q, const void* k, int64_t ld_k, const void* v, int64_t ld_v,
                        adt_dtype in_type, const int32_t* positions, const double* inv_freq, float magnitude,
                        adt_rope_layout layout, int32_t N, int32_t H, int32_t Hkv, int32_t D, int32_t rotary_dim,
                        adt_bf16* q_out, adt_bf16* k_out, adt_bf16* v_out, void* stream) {
  adt::TraceRange trace_("adt_rope_qkv");
  ADT_REQUIRE(in_type == ADT_TYPE_BF16 || in_type == ADT_TYPE_F32);
  ADT_REQUIRE(layout == ADT_ROPE_HALF || layout == ADT_ROPE_INTERLEAVED);
  ADT_REQUIRE(N >= 0 && N <= kMaxRows && D >= 1 && D <= 4096 && rotary_dim >= 0 && rotary_dim % 2 == 0 && rotary_dim <= D);
  if (rotary_dim > kMaxRotary) return ADT_ERR_UNSUPPORTED;
  ADT_REQUIRE(isfinite(magnitude));
  if (N == 0) return ADT_OK;
  ADT_REQUIRE((q != nullptr) == (q_out != nullptr) && (k != nullptr) == (k_out != nullptr) &&
              (v != nullptr) == (v_out != nullptr));
  ADT_REQUIRE(q || k || v);
  ADT_REQUIRE((!q || (H >= 1 && H <= 65535)) && ((!k && !v) || (Hkv >= 1 && Hkv <= 65535)));
  ADT_REQUIRE(positions && (inv_freq || rotary_dim == 0));
  RopeParams p{};
  const void* in[3] = {q, k, v};
  adt_bf16* out[3] = {q_out, k_out, v_out};
  const int64_t ld[3] = {ld_q, ld_k, ld_v};
  const int esize = in_type == ADT_TYPE_BF16 ? 2 : 4;
  int64_t in_bytes[3], out_bytes[3];
  for (int x = 0; x < 3; ++x) {
    p.heads[x] = !in[x] ? 0 : x == 0 ? H : Hkv;
    const int64_t width = static_cast<int64_t>(p.heads[x]) * D;
    ADT_REQUIRE(!in[x] || (ld[x] >= width && ld[x] <= kMaxSpan / N));
    ADT_REQUIRE(reinterpret_cast<uintptr_t>(in[x]) % esize == 0 && reinterpret_cast<uintptr_t>(out[x]) % 2 == 0);
    in_bytes[x] = in[x] ? ((N - 1) * ld[x] + width) * esize : 0;
    out_bytes[x] = in[x] ? N * width * 2 : 0;
    p.in[x] = in[x];
    p.ld[x] = ld[x];
    p.out[x] = reinterpret_cast<__nv_bfloat16*>(out[x]);
  }
  // An output may be its own input (every thread reads what it overwrites
  // first); nothing else may overlap.
  for (int x = 0; x < 3; ++x) {
    for (int y = 0; y < 3; ++y) {
      if (spans_overlap(out[x], out_bytes[x], in[y], in_bytes[y]))
        ADT_REQUIRE(x == y && out[x] == in[x] && esize == 2 && ld[x] == static_cast<int64_t>(p.heads[x]) * D);
      ADT_REQUIRE(x == y || !spans_overlap(out[x], out_bytes[x], out[y], out_bytes[y]));
    }
  }
  p.pos = positions;
  p.inv_freq = inv_freq;
  p.magnitude = magnitude;
  p.D = D;
  p.rot = rotary_dim;
  p.interleaved = layout == ADT_ROPE_INTERLEAVED;
  adt::DeviceInfo info;
  adt_status st = adt::device_info(&info);
  if (st != ADT_OK) return st;
  cudaLaunchConfig_t cfg = {};
  cfg.blockDim = dim3(kThreads, 1, 1);
  cfg.stream = adt::as_stream(stream);
  cudaLaunchAttribute attr[1] = {adt::pdl_attribute()};
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  // Vectors where everything lies on 16-byte boundaries and a vector never
  // holds both turned and copied elements, or parts of both halves.
  const int units = p.interleaved ? D / 8 : D / 8 - rotary_dim / 16;
  bool aligned = D % 8 == 0;
  for (int x = 0; x < 3; ++x)
    aligned = aligned && (!in[x] || (adt::aligned16(in[x]) && adt::aligned16(out[x]) && ld[x] * esize % 16 == 0));
  const bool vec = aligned && rotary_dim % (p.interleaved ? 8 : 16) == 0 && units <= kThreads;
  const int heads = p.heads[0] + p.heads[1];
  if (vec) {
    // Threads of a token: enough for one unit of its heads and one vector of its
    // values each, or where there are many tokens for two of each (what a thread
    // has in flight at a time); tokens fill the CTA.
    const int qk = heads * units, vs = p.heads[2] * (D / 8), want = qk > vs ? qk : vs;
    auto lanes_of = [&](int each) {
      int l = ((want + each - 1) / each + 31) / 32 * 32;
      l = l < units ? (units + 31) / 32 * 32 : l;
      return l < kThreads ? l : kThreads;
    };
    const bool many = static_cast<int64_t>(N) * lanes_of(2) >= int64_t{4} * kThreads * info.sm_count;
    const int lanes = lanes_of(many ? 2 : 1);
    const int tokens = kThreads / lanes;
    const int passes = (want + lanes - 1) / lanes;
    const int groups = (N + tokens - 1) / tokens;
    // Few tokens: their heads over several CTAs, up to two an SM.
    int split = 2 * info.sm_count / groups;
    split = split < 1 ? 1 : split > passes ? passes : split;
    cfg.gridDim = dim3(static_cast<unsigned>(groups), static_cast<unsigned>(split), 1);
    cfg.blockDim = dim3(static_cast<unsigned>(lanes * tokens), 1, 1);
    cfg.dynamicSmemBytes = static_cast<size_t>(tokens) * (rotary_dim / 2) * sizeof(float2);
    if (esize == 2)
      ADT_CUDA_TRY(p.interleaved
                       ? cudaLaunchKernelEx(&cfg, rope_vec_kernel<__nv_bfloat16, true>, p, N, tokens, lanes, units)
                       : cudaLaunchKernelEx(&cfg, rope_vec_kernel<__nv_bfloat16, false>, p, N, tokens, lanes, units));
    else
      ADT_CUDA_TRY(p.interleaved ? cudaLaunchKernelEx(&cfg, rope_vec_kernel<float, true>, p, N, tokens, lanes, units)
                                 : cudaLaunchKernelEx(&cfg, rope_vec_kernel<float, false>, p, N, tokens, lanes, units));
    return adt::launch_status();
  }
  if (aligned && D <= 2 * kThreads) {
    // Heads staged at a time: few enough that few tokens fill the SMs.
    int group = kStaged / D;
    while (group > 1 && static_cast<int64_t>(N) * ((heads + group - 1) / group) < info.sm_count) group = (group + 1) / 2;
    int split = 2 * info.sm_count / N;
    const int most = heads > 0 ? (heads + group - 1) / group : 1;
    split = split < 1 ? 1 : split > most ? most : split;
    cfg.gridDim = dim3(static_cast<unsigned>(N), static_cast<unsigned>(split), 1);
    cfg.dynamicSmemBytes = ((rotary_dim / 2 + 1) & ~1) * sizeof(float2) + static_cast<size_t>(group < heads ? group : heads) * D * 4;
    if (esize == 2)
      ADT_CUDA_TRY(cudaLaunchKernelEx(&cfg, rope_staged_kernel<__nv_bfloat16>, p, group));
    else
      ADT_CUDA_TRY(cudaLaunchKernelEx(&cfg, rope_staged_kernel<float>, p, group));
    return adt::launch_status();
  }
  const int64_t most = static_cast<int64_t>(heads > p.heads[2] ? heads : p.heads[2]) * D;
  int64_t split = 2 * info.sm_count / N;
  const int64_t passes = (most + kThreads - 1) / kThreads;
  split = split < 1 ? 1 : split > passes ? passes : split;
  cfg.gridDim = dim3(static_cast<unsigned>(N), static_cast<unsigned>(split), 1);
  if (esize == 2)
    ADT_CUDA_TRY(cudaLaunchKernelEx(&cfg, rope_scalar_kernel<__nv_bfloat16>, p));
  else
    ADT_CUDA_TRY(cudaLaunchKernelEx(&cfg, rope_scalar_kernel<float>, p));
  return adt::launch_status();
}

}  // extern "C"
