// adt_norm_rope_qkv: norms of the query and key heads, then their rotation, in
// one pass over a projection's rows.
//
// Head row x of D elements: RMS y = x / sqrt(mean x^2 + eps); LAYER the same of
// x - mean x; then y w + b, the rotation of adt_rope_qkv, and one rounding to
// bf16.  Everything before it is fp32; the variance is a sum over centred values
// (E x^2 - (E x)^2 loses what is left of them where a row's mean is large).
//
// A head is split over a group of lanes, 16 elements each, which are such that
// the partner of every rotated element lies in the same lane: two vectors of 8, in
// a half layout those of a pair's two sides.  So a norm costs two or four rounds of
// shuffles of one value and the rotation none.  (Where the sides of a half layout do
// not begin at a vector, partners meet in shared memory.)
//
// Bound by HBM, each element is read and written once: 16384 tokens of 32 / 32 heads
// x 128 in bf16 (805 MB) 126 us, 94 % of a copy's rate; between a unit's load and
// its store lie the sums' shuffles, which the next unit's load hides in part.  501
// tokens of 32 / 8 heads in fp32 with a LayerNorm 7.8 us, one token 4.0 us (its launch).
// 4096 tokens of 32 / 8 heads (14.8 at the copy rate): 22 us with pairs side by side,
// 24.5 as halves, 42 with 50 elements turned as halves, through shared memory.
#include <math.h>

#include "adt_common.cuh"
#include "rope_common.cuh"

namespace {

using adt::Eight;
using adt::kMaxRotary;
using adt::kMaxRows;
using adt::kMaxSpan;
using adt::put;
using adt::spans_overlap;
using adt::to_f32;
using adt::token_angles;

constexpr int kThreads = 256;
constexpr int kUnit = 16;     // elements of a head in a thread
constexpr int kMaxHead = 4096;
constexpr int kMaxTurns = 4, kTurnCtas = 8;
constexpr int kAngleBytes = 30 * 1024;  // of a CTA's tokens: with all else within the 48 KB that need no opting in

struct NormParams {
  const void* in[3];        // rows of q, k, v
  int64_t ld[3];            // row strides in elements
  __nv_bfloat16* out[3];    // [N][heads][D]
  int heads[3];
  const void* weight[2];    // of q and k; NULL: ones
  const void* bias[2];      // NULL: zeros
  int wld[2];               // elements from a head's weights to the next one's, 0: shared
  const int32_t* pos;
  const double* inv_freq;
  float magnitude, eps;
  int D, rot, interleaved, layer;
};

// Sum over the aligned group of `width` (a power of two) lanes.
__device__ __forceinline__ float group_sum(float v, int width) {
  for (int o = width >> 1; o > 0; o >>= 1) v += __shfl_xor_sync(adt::kFullMask, v, o);
  return v;
}

constexpr int kPadded = kUnit + 1;  // of a thread's elements in shared memory: 16 lanes' lie in 16 banks

// Vectors: 16 | D <= 512, 16-byte boundaries.  Where rot is not a multiple of a vector
// (in a half layout of two): kPairs, pairs side by side, of which a lane may turn some
// only; kMeet, a half layout, whose partners lie in different lanes.  A CTA takes a token or a few
// at a time, one after the other (and where there are few, a share of their heads);
// a thread keeps its place within the heads, so that it reads a token's cosines and
// sines once.  Once a thread's unit is widened, its next one is on its way.
enum Rotation { kVectors, kPairs, kMeet };

template <typename T, typename W, int kRot, bool kEarly>
__global__ void __launch_bounds__(kThreads, !kEarly ? (sizeof(T) == 2 ? 4 : 3)
                                            : sizeof(T) + sizeof(W) == 4 ? 4
                                            : sizeof(T) + sizeof(W) == 6 ? 3
                                                                         : 2)
    norm_rope_vec_kernel(const NormParams p, int N, int tokens, int lanes, int width, int turns) {
  extern __shared__ float2 cs[];
  adt::pdl_wait_then_release();
  const int n0 = blockIdx.x * tokens * turns, here = min(tokens * turns, N - n0);
  const int tok0 = threadIdx.x / lanes, lane = threadIdx.x - tok0 * lanes;
  const int half = p.rot / 2, units = p.D / kUnit;
  const int row = kRot == kPairs ? (half + 7) & ~7 : half;  // angles of a token
  const int per_pass = lanes / width, hl = lane / width, u = lane - hl * width;
  // Two vectors of 8, of each half of what a group of lanes covers, so that a warp's
  // loads and stores take whole lines: a half layout's turned elements, then the rest;
  // else the head.  (As one run of 16: 30 us for the 22 above, 9.5 for the 7.8.)
  const bool split_pair = kRot == kVectors && !p.interleaved && u * kUnit < p.rot;
  const int covered = kRot == kVectors && !p.interleaved ? (split_pair ? p.rot : p.D - p.rot) : p.D;
  const int e0 = covered == p.D || split_pair ? u * 8 : p.rot + (u - p.rot / kUnit) * 8, e1 = e0 + covered / 2;
  const int heads = p.heads[0] + p.heads[1], vectors = p.heads[2] * p.D / 8;
  const int first = static_cast<int>(blockIdx.y) * per_pass, hstep = static_cast<int>(gridDim.y) * per_pass;
  const int vfirst = static_cast<int>(blockIdx.y) * lanes, vstep = static_cast<int>(gridDim.y) * lanes;
  const float inv_d = 1.f / static_cast<float>(p.D);

  // What is on its way: the unit of head base + hl, vectors vb + lane and vstep after
  // it, of token tok.  (base and vb are the same for a warp: its lanes make the same
  // rounds, the sums are exchanged by all.  Lanes past a head's elements, or without
  // a head or a token, add zeros.)
  int tok = tok0, base = first, vb = vfirst;
  Eight<T> x[2], v[2];
  auto have_unit = [&]() { return tok < here && u < units && base + hl < heads; };
  auto fetch = [&]() {
    const int64_t n = n0 + tok;
    if (have_unit()) {
      const int h = base + hl;
      const bool q = h < p.heads[0];
      const T* src = static_cast<const T*>(q ? p.in[0] : p.in[1]) + n * (q ? p.ld[0] : p.ld[1]) + (q ? h : h - p.heads[0]) * p.D;
      x[0].load(src + e0);
      x[1].load(src + e1);
    }
#pragma unroll
    for (int k = 0; k < 2; ++k)
      if (tok < here && vb + lane + k * vstep < vectors)
        v[k].load(static_cast<const T*>(p.in[2]) + n * p.ld[2] + static_cast<int64_t>(vb + lane + k * vstep) * 8);
  };
  fetch();
  token_angles(p, n0, here, cs, row);
  for (int turn = 0; turn < turns;) {
    const bool have = have_unit();
    const int64_t n = n0 + tok;
    const int h = base + hl, which = h < p.heads[0] ? 0 : 1, hh = which ? h - p.heads[0] : h, at = tok * row;
    const bool any = base < heads;  // (uniform)
    float y[kUnit];
    {
      float a[8], b[8];
      x[0].get(a);
      x[1].get(b);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        y[i] = have ? a[i] : 0.f;
        y[8 + i] = have ? b[i] : 0.f;
      }
    }
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      if (tok < here && vb + lane + k * vstep < vectors) {
        float a[8];
        v[k].get(a);
        put(p.out[2] + n * p.heads[2] * p.D + static_cast<int64_t>(vb + lane + k * vstep) * 8, a);
      }
    }
    base += hstep;
    vb += 2 * vstep;
    if (base >= heads && vb >= vectors) {
      ++turn;
      tok += tokens;
      base = first;
      vb = vfirst;
    }
    if (turn < turns) fetch();
    if (!any) continue;
    const W* w = static_cast<const W*>(which ? p.weight[1] : p.weight[0]);
    const W* bi = static_cast<const W*>(which ? p.bias[1] : p.bias[0]);
    const int64_t woff = static_cast<int64_t>(hh) * (which ? p.wld[1] : p.wld[0]);
    // Weights: early, beside the rows' sums, where a call is a chain of a few loads (501
    // tokens 9.5 us, late 10.4, both with vectors side by side); else where they are used, from L1, and the registers
    // that they would lie in hold more CTAs (16384 tokens 127 us, early 145; 4096 of 32 / 8
    // heads 24, early 32).
    Eight<W> tw[2], tb[2];
    if (kEarly && have && w) {
      tw[0].load(w + woff + e0);
      tw[1].load(w + woff + e1);
    }
    if (kEarly && have && bi) {
      tb[0].load(bi + woff + e0);
      tb[1].load(bi + woff + e1);
    }
    if (p.layer) {
      float sum = 0.f;
#pragma unroll
      for (int i = 0; i < kUnit; ++i) sum += y[i];
      const float mean = group_sum(sum, width) * inv_d;
#pragma unroll
      for (int i = 0; i < kUnit; ++i) y[i] = have ? y[i] - mean : 0.f;
    }
    float sq = 0.f;
#pragma unroll
    for (int i = 0; i < kUnit; ++i) sq = fmaf(y[i], y[i], sq);
    const float r = rsqrtf(fmaf(group_sum(sq, width), inv_d, p.eps));
    if (kRot != kMeet && !have) continue;
#pragma unroll
    for (int i = 0; i < kUnit; ++i) y[i] *= r;
    if (w && have) {
      float a[8], b[8];
      if (!kEarly) {
        tw[0].load(w + woff + e0);
        tw[1].load(w + woff + e1);
      }
      tw[0].get(a);
      tw[1].get(b);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        y[i] *= a[i];
        y[8 + i] *= b[i];
      }
    }
    if (bi && have) {
      float a[8], b[8];
      if (!kEarly) {
        tb[0].load(bi + woff + e0);
        tb[1].load(bi + woff + e1);
      }
      tb[0].get(a);
      tb[1].get(b);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        y[i] += a[i];
        y[8 + i] += b[i];
      }
    }
    if (split_pair) {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float2 z = cs[at + e0 + i];
        const float a = y[i], b = y[8 + i];
        y[i] = a * z.x - b * z.y;
        y[8 + i] = b * z.x + a * z.y;
      }
    } else if (kRot != kMeet && p.interleaved) {
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        if ((k ? e1 : e0) >= p.rot) continue;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float2 z = cs[at + (k ? e1 : e0) / 2 + i];
          const float a = y[8 * k + 2 * i], b = y[8 * k + 2 * i + 1];
          y[8 * k + 2 * i] = a * z.x - b * z.y;
          y[8 * k + 2 * i + 1] = b * z.x + a * z.y;
        }
      }
    }
    if (kRot == kMeet) {  // (by all lanes of the warp)
      float* head = reinterpret_cast<float*>(cs + tokens * turns * row) + (threadIdx.x - u) * kPadded;
#pragma unroll
      for (int i = 0; i < kUnit; ++i) {
        const int e = (i < 8 ? e0 : e1 - 8) + i;
        if (u < units) head[e + e / kUnit] = y[i];
      }
      __syncwarp();
#pragma unroll
      for (int i = 0; i < kUnit; ++i) {
        const int e = (i < 8 ? e0 : e1 - 8) + i;
        if (!have || e >= p.rot) continue;
        const bool lead = e < half;
        const int other = lead ? e + half : e - half;
        const float2 z = cs[at + (lead ? e : other)];
        const float x = head[other + other / kUnit];
        y[i] = y[i] * z.x + x * (lead ? -z.y : z.y);
      }
      __syncwarp();  // before they are overwritten
      if (!have) continue;
    }
    __nv_bfloat16* dst = (which ? p.out[1] : p.out[0]) + (n * (which ? p.heads[1] : p.heads[0]) + hh) * p.D;
    float za[8], zb[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      za[i] = y[i];
      zb[i] = y[8 + i];
    }
    put(dst + e0, za);
    put(dst + e1, zb);
  }
}

// Any head size, row stride and alignment: a warp takes a head
// at a time, in shared memory as fp32, element by element.
template <typename T, typename W>
__global__ void __launch_bounds__(kThreads) norm_rope_any_kernel(const NormParams p) {
  extern __shared__ float2 shared[];
  float2* cs = shared;
  adt::pdl_wait_then_release();
  const int64_t n = blockIdx.x;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
  const int half = p.rot / 2, heads = p.heads[0] + p.heads[1];
  float* row = reinterpret_cast<float*>(shared + half) + warp * p.D;
  token_angles(p, blockIdx.x, 1, cs);
  for (int h = blockIdx.y * warps + warp; h < heads; h += gridDim.y * warps) {
    const int which = h < p.heads[0] ? 0 : 1, hh = which ? h - p.heads[0] : h;
    const T* src = static_cast<const T*>(p.in[which]) + n * p.ld[which] + static_cast<int64_t>(hh) * p.D;
    const W* w = static_cast<const W*>(p.weight[which]);
    const W* bi = static_cast<const W*>(p.bias[which]);
    const int64_t woff = static_cast<int64_t>(hh) * p.wld[which];
    float sum = 0.f;
    for (int e = lane; e < p.D; e += 32) {
      const float x = to_f32(src[e]);
      row[e] = x;
      sum += x;
    }
    const float mean = p.layer ? adt::warp_sum(sum) / static_cast<float>(p.D) : 0.f;
    float sq = 0.f;
    for (int e = lane; e < p.D; e += 32) {
      const float x = row[e] - mean;
      sq = fmaf(x, x, sq);
    }
    const float r = rsqrtf(adt::warp_sum(sq) / static_cast<float>(p.D) + p.eps);
    for (int e = lane; e < p.D; e += 32) {
      float y = (row[e] - mean) * r;
      if (w) y *= to_f32(w[woff + e]);
      if (bi) y += to_f32(bi[woff + e]);
      row[e] = y;
    }
    __syncwarp();
    __nv_bfloat16* dst = p.out[which] + (n * p.heads[which] + hh) * p.D;
    for (int e = lane; e < p.D; e += 32) {
      float y = row[e];
      if (e < p.rot) {
        const int pair = p.interleaved ? e >> 1 : e < half ? e : e - half;
        const bool lead = p.interleaved ? (e & 1) == 0 : e < half;
        const float2 z = cs[pair];
        const float other = row[p.interleaved ? e ^ 1 : lead ? e + half : e - half];
        y = y * z.x + other * (lead ? -z.y : z.y);
      }
      dst[e] = __float2bfloat16(y);
    }
    __syncwarp();  // before the row is overwritten
  }
  const T* in = static_cast<const T*>(p.in[2]) + n * p.ld[2];
  __nv_bfloat16* out = p.out[2] + n * p.heads[2] * p.D;
  for (int i = blockIdx.y * blockDim.x + threadIdx.x; i < p.heads[2] * p.D; i += gridDim.y * blockDim.x)
    out[i] = __float2bfloat16(to_f32(in[i]));
}

template <typename T, typename W>
adt_status launch(const NormParams& p, bool vec, int N, const adt::DeviceInfo& info, cudaLaunchConfig_t* cfg) {
  const int heads = p.heads[0] + p.heads[1];
  if (vec) {
    const int units = p.D / kUnit, width = adt::next_pow2(units), row = (p.rot / 2 + 7) & ~7;
    // Threads of a token: one unit of its heads and one pair of vectors of its values
    // each, or with many tokens two of each.
    const int qk = heads * width, vs = (p.heads[2] * units + 1) / 2, want = qk > vs ? qk : vs;
    auto lanes_of = [&](int each) {
      int l = ((want + each - 1) / each + 31) / 32 * 32;
      return l < kThreads ? l : kThreads;
    };
    const bool many = static_cast<int64_t>(N) * lanes_of(2) >= int64_t{4} * kThreads * info.sm_count;
    const int lanes = lanes_of(many ? 2 : 1);
    const int tokens = kThreads / lanes;
    const int passes = (want + lanes - 1) / lanes;
    // With many tokens up to four of them a CTA, so that the next one's rows are on their
    // way while one is normed (16384 tokens 150 us, with one a CTA and each unit loaded when
    // it is normed 175; both before weights were loaded late), but not all in a few CTAs
    // an SM (152 to 162).
    int turns = 1;
    while (turns < kMaxTurns && static_cast<int64_t>(N) >= int64_t{2} * turns * tokens * kTurnCtas * info.sm_count &&
           2 * turns * tokens * row * static_cast<int>(sizeof(float2)) <= kAngleBytes)
      turns *= 2;
    const int groups = (N + tokens * turns - 1) / (tokens * turns);
    // Few tokens: their heads over several CTAs, up to two an SM.
    int split = 2 * info.sm_count / groups;
    split = split < 1 ? 1 : split > passes ? passes : split;
    cfg->gridDim = dim3(static_cast<unsigned>(groups), static_cast<unsigned>(split), 1);
    cfg->blockDim = dim3(static_cast<unsigned>(lanes * tokens), 1, 1);
    const int rot = p.rot % (p.interleaved ? 8 : kUnit) == 0 ? kVectors : p.interleaved ? kPairs : kMeet;
    cfg->dynamicSmemBytes = static_cast<size_t>(tokens) * turns * row * sizeof(float2) + (rot == kMeet ? kThreads * kPadded * 4 : 0);
    const auto kernel = rot == kVectors ? (many ? norm_rope_vec_kernel<T, W, kVectors, false> : norm_rope_vec_kernel<T, W, kVectors, true>)
                        : rot == kPairs ? norm_rope_vec_kernel<T, W, kPairs, false>
                                        : norm_rope_vec_kernel<T, W, kMeet, false>;
    ADT_CUDA_TRY(cudaLaunchKernelEx(cfg, kernel, p, N, tokens, lanes, width, turns));
    return adt::launch_status();
  }
  // Rows of shared memory: within the 48 KB that need no opting in.
  int warps = (48 * 1024 - kMaxRotary * 4) / (p.D * 4);
  warps = warps > kThreads / 32 ? kThreads / 32 : warps;
  const int most = heads > 0 ? (heads + warps - 1) / warps : 1;
  int split = 2 * info.sm_count / N;
  split = split < 1 ? 1 : split > most ? most : split;
  cfg->gridDim = dim3(static_cast<unsigned>(N), static_cast<unsigned>(split), 1);
  cfg->blockDim = dim3(static_cast<unsigned>(warps * 32), 1, 1);
  cfg->dynamicSmemBytes = p.rot / 2 * sizeof(float2) + static_cast<size_t>(warps) * p.D * 4;
  ADT_CUDA_TRY(cudaLaunchKernelEx(cfg, norm_rope_any_kernel<T, W>, p));
  return adt::launch_status();
}

static_assert((48 * 1024 - kMaxRotary * 4) / (kMaxHead * 4) >= 1, "a warp's row fits");

}  // namespace

extern "C" {

adt_status adt_norm_rope_qkv(const void* q, int64_t ld_q, const void* k, int64_t ld_k, const void* v, int64_t ld_v,
                             adt_dtype in_type, adt_norm norm, float eps, const void* q_weight, const void* q_bias,
                             int32_t q_weight_stride, const void* k_weight, const void* k_bias, int32_t k_weight_stride,
                             adt_dtype weight_type, const int32_t* positions, const double* inv_freq, float magnitude,
                             adt_rope_layout layout, int32_t N, int32_t H, int32_t Hkv, int32_t D, int32_t rotary_dim,
                             adt_bf16* q_out, adt_bf16* k_out, adt_bf16* v_out, void* stream) {
  adt::TraceRange trace_("adt_norm_rope_qkv");
  ADT_REQUIRE(in_type == ADT_TYPE_BF16 || in_type == ADT_TYPE_F32);
  ADT_REQUIRE(weight_type == ADT_TYPE_BF16 || weight_type == ADT_TYPE_F32);
  ADT_REQUIRE(norm == ADT_NORM_RMS || norm == ADT_NORM_LAYER);
  ADT_REQUIRE(layout == ADT_ROPE_HALF || layout == ADT_ROPE_INTERLEAVED);
  ADT_REQUIRE(N >= 0 && N <= kMaxRows && D >= 1 && D <= kMaxHead && rotary_dim >= 0 && rotary_dim % 2 == 0 &&
              rotary_dim <= D);
  if (rotary_dim > kMaxRotary) return ADT_ERR_UNSUPPORTED;
  ADT_REQUIRE(isfinite(magnitude) && isfinite(eps) && eps >= 0.f);
  if (N == 0) return ADT_OK;
  ADT_REQUIRE((q != nullptr) == (q_out != nullptr) && (k != nullptr) == (k_out != nullptr) &&
              (v != nullptr) == (v_out != nullptr));
  ADT_REQUIRE(q || k || v);
  ADT_REQUIRE((!q || (H >= 1 && H <= 65535)) && ((!k && !v) || (Hkv >= 1 && Hkv <= 65535)));
  ADT_REQUIRE(positions && (inv_freq || rotary_dim == 0));
  NormParams p{};
  const void* in[3] = {q, k, v};
  adt_bf16* out[3] = {q_out, k_out, v_out};
  const int64_t ld[3] = {ld_q, ld_k, ld_v};
  const void* weight[2] = {q_weight, k_weight};
  const void* bias[2] = {q_bias, k_bias};
  const int32_t wld[2] = {q_weight_stride, k_weight_stride};
  const int esize = in_type == ADT_TYPE_BF16 ? 2 : 4, wsize = weight_type == ADT_TYPE_BF16 ? 2 : 4;
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
  bool aligned = D % 8 == 0;
  for (int x = 0; x < 2; ++x) {
    const void* params[2] = {weight[x], bias[x]};
    for (const void* w : params) {
      if (!w || !in[x]) continue;
      ADT_REQUIRE(wld[x] == 0 || wld[x] >= D);
      ADT_REQUIRE(reinterpret_cast<uintptr_t>(w) % wsize == 0);
      const int64_t bytes = (static_cast<int64_t>(p.heads[x] - 1) * wld[x] + D) * wsize;
      for (int y = 0; y < 3; ++y) ADT_REQUIRE(!spans_overlap(out[y], out_bytes[y], w, bytes));
      aligned = aligned && adt::aligned16(w) && static_cast<int64_t>(wld[x]) * wsize % 16 == 0;
    }
    p.weight[x] = weight[x];
    p.bias[x] = bias[x];
    p.wld[x] = wld[x];
  }
  // An output may be its own input (a head is read before it is overwritten);
  // nothing else may overlap.
  for (int x = 0; x < 3; ++x) {
    for (int y = 0; y < 3; ++y) {
      if (spans_overlap(out[x], out_bytes[x], in[y], in_bytes[y]))
        ADT_REQUIRE(x == y && out[x] == in[x] && esize == 2 && ld[x] == static_cast<int64_t>(p.heads[x]) * D);
      ADT_REQUIRE(x == y || !spans_overlap(out[x], out_bytes[x], out[y], out_bytes[y]));
    }
    aligned = aligned && (!in[x] || (adt::aligned16(in[x]) && adt::aligned16(out[x]) && ld[x] * esize % 16 == 0));
  }
  p.pos = positions;
  p.inv_freq = inv_freq;
  p.magnitude = magnitude;
  p.eps = eps;
  p.D = D;
  p.rot = rotary_dim;
  p.interleaved = layout == ADT_ROPE_INTERLEAVED;
  p.layer = norm == ADT_NORM_LAYER;
  adt::DeviceInfo info;
  adt_status st = adt::device_info(&info);
  if (st != ADT_OK) return st;
  cudaLaunchConfig_t cfg = {};
  cfg.stream = adt::as_stream(stream);
  cudaLaunchAttribute attr[1] = {adt::pdl_attribute()};
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  const bool vec = aligned && D % kUnit == 0 && D <= 32 * kUnit;
  if (esize == 2)
    return wsize == 2 ? launch<__nv_bfloat16, __nv_bfloat16>(p, vec, N, info, &cfg)
                      : launch<__nv_bfloat16, float>(p, vec, N, info, &cfg);
  return wsize == 2 ? launch<float, __nv_bfloat16>(p, vec, N, info, &cfg) : launch<float, float>(p, vec, N, info, &cfg);
}

}  // extern "C"
