// adt_kv_compact_q8, adt_kv_read_q8: the 8-bit cache written and read back.
//
// Both move each byte once and compute next to nothing: bound by HBM where there
// are many rows, by a launch where there are few.  Written: 36 layers, 20 heads x
// 64, paths of 3979 tokens in two trees (1.11 GB) 173 us, 94 % of a copy's rate;
// one token of one layer 3.1 us.
#include <math.h>

#include "adt_common.cuh"
#include "kv_q8.cuh"

namespace {

constexpr int kThreads = 256;

struct CompactQ8Params {
  uint8_t* cache[2];  // K, V
  uint8_t* scale[2];
  const int32_t* kv_len;
  int32_t* kv_len_out;
  const __nv_bfloat16* tree[2];
  const int32_t* offs;
  const int32_t* path;
  const int32_t* alen;
  int max_path, Hkv, max_kv;
  adt::Q8Strides s;
  int64_t tls;
  int entries, heads_per_cta, head_groups;
  unsigned* err;
};

// A CTA takes `entries` (a power of two up to 32) consecutive path entries of a
// tree's layer and some of its kv heads; a row is D / 16 lanes', 8 elements of each
// half: a warp's loads of 16 bytes cover whole lines.
// Neighbouring groups of lanes take neighbouring entries, whose rows and scales
// are neighbours in the cache.
template <int D>
__global__ void __launch_bounds__(kThreads) kv_compact_q8_kernel(const CompactQ8Params p) {
  constexpr int kLanes = D / 16, kRows = kThreads / kLanes;
  adt::pdl_wait_then_release();
  const int tid = threadIdx.x, b = blockIdx.y, l = blockIdx.z;
  const int group = blockIdx.x % p.head_groups, i0 = blockIdx.x / p.head_groups * p.entries;
  const int a = p.alen[b], L = p.kv_len[b], node0 = p.offs[b], n = p.offs[b + 1] - node0;
  const int32_t* path = p.path + static_cast<int64_t>(b) * p.max_path;
  const bool fits = a >= 0 && a < p.max_path && L >= 0 && static_cast<int64_t>(L) + a + 1 <= p.max_kv;
  // The whole path is checked by every CTA of the tree: a malformed one skips it.
  int bad = 0;
  for (int j = tid; fits && j <= a; j += kThreads) {
    const int node = path[j];
    bad |= node < 0 || node >= n || node0 < 0 || (j == 0 && node != 0);
  }
  bad = __syncthreads_or(bad);
  const bool ok = fits && !bad;
  if (tid == 0 && blockIdx.x == 0 && l == 0) {
    if (!ok) adt::raise_error(p.err, fits ? ADT_DEVERR_BAD_PATH : ADT_DEVERR_KV_RANGE);
    if (p.kv_len_out) p.kv_len_out[b] = ok ? L + a + 1 : L;
  }
  if (!ok || i0 > a) return;
  const int row = tid / kLanes, lane = tid % kLanes;
  const int i = i0 + row % p.entries, gstep = kRows / p.entries;
  const int g1 = min(p.Hkv, (group + 1) * p.heads_per_cta);
  const bool there = i <= a;
  const int64_t node = node0 + (there ? path[i] : 0);
  // (All lanes of a warp make the same rounds: amax is exchanged by all.)
  for (int gb = group * p.heads_per_cta; gb < g1; gb += gstep) {
    const int g = gb + row / p.entries;
    const bool have = there && g < g1;
    uint4 x[2][2];
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const uint4* src = reinterpret_cast<const uint4*>(p.tree[t] + l * p.tls + (node * p.Hkv + (have ? g : 0)) * D) + lane;
      x[t][0] = have ? src[0] : make_uint4(0u, 0u, 0u, 0u);
      x[t][1] = have ? src[kLanes] : make_uint4(0u, 0u, 0u, 0u);
    }
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const uint32_t w[8] = {x[t][0].x, x[t][0].y, x[t][0].z, x[t][0].w, x[t][1].x, x[t][1].y, x[t][1].z, x[t][1].w};
      // Magnitudes of bf16 bit patterns compare as integers; not finite is above all.
      uint32_t most = 0u;
#pragma unroll
      for (int k = 0; k < 8; ++k) most = max(most, max(w[k] << 16 & 0x7fff0000u, w[k] & 0x7fff0000u));
#pragma unroll
      for (int o = kLanes / 2; o > 0; o >>= 1) most = max(most, __shfl_xor_sync(adt::kFullMask, most, o));
      const bool finite = most < 0x7f800000u;
      const uint32_t s = finite ? adt::q8_row_scale(__uint_as_float(most)) : 255u;
      const float inv = finite ? __uint_as_float((254u - s) << 23) : 0.f;  // 2^(127 - s), s from 7 to 247
      uint32_t out[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        out[k] = 0u;
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const uint32_t z = w[2 * k + e];
          out[k] |= adt::f32x2_to_e4m3(__uint_as_float(z << 16) * inv, __uint_as_float(z & 0xffff0000u) * inv) << (16 * e);
        }
        if (!finite) out[k] = 0u;
      }
      if (have) {
        const int64_t pos = L + i;
        uint8_t* dst = p.cache[t] + l * p.s.cache[0] + b * p.s.cache[1] + g * p.s.cache[2] + pos * D;
        reinterpret_cast<uint2*>(dst)[lane] = make_uint2(out[0], out[1]);
        reinterpret_cast<uint2*>(dst)[lane + kLanes] = make_uint2(out[2], out[3]);
        if (lane == 0) p.scale[t][l * p.s.scale[0] + b * p.s.scale[1] + g * p.s.scale[2] + pos] = static_cast<uint8_t>(s);
      }
    }
  }
}

struct ReadQ8Params {
  const uint8_t* cache[2];
  const uint8_t* scale[2];
  const int32_t* kv_len;
  __nv_bfloat16* out[2];
  int B, Hkv, max_kv, blocks;
  adt::Q8Strides s;
  int64_t os[3];
  unsigned* err;
};

constexpr int kReadPasses = 2;  // rows of a thread, of K and of V

// A row is D / 16 lanes', each with 8 elements of its first half and 8 of its second,
// so that a warp's stores of 16 bytes cover whole lines (16 elements in a run would
// make each store of a warp every other 16 bytes: 144 against 123 us for 8 layers of
// 8 heads x 128 over 16398 rows, 808 MB at 96 % of a copy's rate).

template <int D>
__global__ void __launch_bounds__(kThreads) kv_read_q8_kernel(const ReadQ8Params p) {
  constexpr int kLanes = D / 16, kRows = kThreads / kLanes;
  adt::pdl_wait_then_release();
  const int slice = blockIdx.x / p.blocks, block = blockIdx.x - slice * p.blocks;
  const int g = slice % p.Hkv, b = slice / p.Hkv % p.B, l = slice / p.Hkv / p.B;
  const int L = p.kv_len[b];
  if (L < 0 || L > p.max_kv) {
    if (threadIdx.x == 0 && block == 0 && g == 0 && l == 0) adt::raise_error(p.err, ADT_DEVERR_KV_RANGE);
    return;
  }
  const int row = threadIdx.x / kLanes, lane = threadIdx.x % kLanes;
  const int64_t c0 = l * p.s.cache[0] + b * p.s.cache[1] + g * p.s.cache[2];
  const int64_t s0 = l * p.s.scale[0] + b * p.s.scale[1] + g * p.s.scale[2];
  const int64_t o0 = l * p.os[0] + b * p.os[1] + g * p.os[2];
  const int64_t first = static_cast<int64_t>(block) * (kRows * kReadPasses) + row;
  uint2 x[2][kReadPasses][2];
  uint32_t s[2][kReadPasses];
#pragma unroll
  for (int k = 0; k < kReadPasses; ++k) {
    const int64_t r = first + k * kRows;
    if (r >= L) continue;
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const uint2* src = reinterpret_cast<const uint2*>(p.cache[t] + c0 + r * D) + lane;
      x[t][k][0] = src[0];
      x[t][k][1] = src[kLanes];
      s[t][k] = p.scale[t][s0 + r];
    }
  }
#pragma unroll
  for (int k = 0; k < kReadPasses; ++k) {
    const int64_t r = first + k * kRows;
    if (r >= L) continue;
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const float scale = adt::q8_scale(s[t][k]);
      const uint32_t w[4] = {x[t][k][0].x, x[t][k][0].y, x[t][k][1].x, x[t][k][1].y};
      uint32_t o[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float2 f = adt::e4m3x2_to_f32(w[e >> 1] >> (16 * (e & 1)) & 0xffffu);
        const __nv_bfloat162 y = __floats2bfloat162_rn(f.x * scale, f.y * scale);
        o[e] = *reinterpret_cast<const uint32_t*>(&y);
      }
      uint4* dst = reinterpret_cast<uint4*>(p.out[t] + o0 + r * D) + lane;
      dst[0] = make_uint4(o[0], o[1], o[2], o[3]);
      dst[kLanes] = make_uint4(o[4], o[5], o[6], o[7]);
    }
  }
}

}  // namespace

extern "C" {

adt_status adt_kv_compact_q8(uint8_t* k_cache, uint8_t* v_cache, uint8_t* k_scale, uint8_t* v_scale,
                             const int32_t* kv_len, int32_t* kv_len_out, const adt_bf16* k_tree, const adt_bf16* v_tree,
                             const int32_t* node_offsets, const int32_t* path, int32_t max_path,
                             const int32_t* accept_len, int32_t B, int32_t Hkv, int32_t D, int32_t num_layers,
                             int32_t max_kv, int64_t cache_layer_stride, int64_t cache_stride_b, int64_t cache_stride_h,
                             int64_t scale_layer_stride, int64_t scale_stride_b, int64_t scale_stride_h,
                             int64_t tree_layer_stride, void* stream) {
  adt::TraceRange trace_("adt_kv_compact_q8");
  ADT_REQUIRE(k_cache && v_cache && k_scale && v_scale && kv_len && k_tree && v_tree && node_offsets && path && accept_len);
  ADT_REQUIRE(B >= 1 && B <= 65535 && Hkv >= 1 && Hkv <= 65535 && num_layers >= 1 && num_layers <= 65535);
  ADT_REQUIRE(max_path >= 1 && max_path <= (1 << 20) && max_kv >= 1 && max_kv < (1 << 30));
  if (D != 64 && D != 128) return ADT_ERR_UNSUPPORTED;
  const adt::Q8Strides s = {{cache_layer_stride, cache_stride_b, cache_stride_h},
                            {scale_layer_stride, scale_stride_b, scale_stride_h}};
  int64_t cache_span, scale_span;
  adt_status st = adt::check_q8_cache(k_cache, v_cache, k_scale, v_scale, s, num_layers, B, Hkv, D, max_kv, true,
                                      &cache_span, &scale_span);
  if (st != ADT_OK) return st;
  // (Every layer's CTAs read what one of the first layer's would write over.)
  const struct { const void* p; int64_t bytes; } others[] = {
      {kv_len, B * 4ll}, {accept_len, B * 4ll}, {node_offsets, (B + 1) * 4ll}, {path, B * 4ll * max_path},
      {k_cache, cache_span}, {v_cache, cache_span}, {k_scale, scale_span}, {v_scale, scale_span}};
  for (const auto& x : others) ADT_REQUIRE(!kv_len_out || !adt::spans_overlap(x.p, x.bytes, kv_len_out, B * 4ll));
  ADT_REQUIRE(num_layers == 1 || (tree_layer_stride >= 0 && tree_layer_stride % 8 == 0 &&
                                  tree_layer_stride <= adt::kMaxCacheStride));
  ADT_REQUIRE(adt::aligned16(k_tree) && adt::aligned16(v_tree));
  adt::DeviceInfo info;
  st = adt::device_info(&info);
  if (st != ADT_OK) return st;
  CompactQ8Params p{};
  p.cache[0] = k_cache, p.cache[1] = v_cache;
  p.scale[0] = k_scale, p.scale[1] = v_scale;
  p.kv_len = kv_len;
  p.kv_len_out = kv_len_out;
  p.tree[0] = reinterpret_cast<const __nv_bfloat16*>(k_tree);
  p.tree[1] = reinterpret_cast<const __nv_bfloat16*>(v_tree);
  p.offs = node_offsets;
  p.path = path;
  p.alen = accept_len;
  p.max_path = max_path;
  p.Hkv = Hkv;
  p.max_kv = max_kv;
  p.s = s;
  p.tls = num_layers > 1 ? tree_layer_stride : 0;
  p.err = info.error_word;
  // Entries of a CTA, and its kv heads: all of them, or few enough that the call
  // has two CTAs an SM.
  const int rows = kThreads / (D / 16);
  p.entries = max_path >= 32 ? 32 : adt::next_pow2(max_path);
  const int64_t chunks = (max_path + p.entries - 1) / p.entries;
  const int per_round = rows / p.entries, rounds = (Hkv + per_round - 1) / per_round;
  int64_t groups = (2 * info.sm_count + chunks * B * num_layers - 1) / (chunks * B * num_layers);
  groups = groups > rounds ? rounds : groups;
  p.heads_per_cta = static_cast<int>((rounds + groups - 1) / groups) * per_round;
  p.head_groups = (Hkv + p.heads_per_cta - 1) / p.heads_per_cta;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(static_cast<unsigned>(chunks * p.head_groups), static_cast<unsigned>(B),
                     static_cast<unsigned>(num_layers));
  cfg.blockDim = dim3(kThreads, 1, 1);
  cfg.stream = adt::as_stream(stream);
  cudaLaunchAttribute attr[1] = {adt::pdl_attribute()};
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  ADT_CUDA_TRY(D == 128 ? cudaLaunchKernelEx(&cfg, kv_compact_q8_kernel<128>, p)
                        : cudaLaunchKernelEx(&cfg, kv_compact_q8_kernel<64>, p));
  return adt::launch_status();
}

adt_status adt_kv_read_q8(const uint8_t* k_cache, const uint8_t* v_cache, const uint8_t* k_scale, const uint8_t* v_scale,
                          const int32_t* kv_len, adt_bf16* k_out, adt_bf16* v_out, int32_t B, int32_t Hkv, int32_t D,
                          int32_t num_layers, int32_t max_kv, int64_t cache_layer_stride, int64_t cache_stride_b,
                          int64_t cache_stride_h, int64_t scale_layer_stride, int64_t scale_stride_b,
                          int64_t scale_stride_h, int64_t out_layer_stride, int64_t out_stride_b, int64_t out_stride_h,
                          void* stream) {
  adt::TraceRange trace_("adt_kv_read_q8");
  ADT_REQUIRE(k_cache && v_cache && k_scale && v_scale && kv_len && k_out && v_out);
  ADT_REQUIRE(B >= 1 && B <= 65535 && Hkv >= 1 && Hkv <= 65535 && num_layers >= 1 && num_layers <= 65535);
  ADT_REQUIRE(max_kv >= 1 && max_kv < (1 << 30));
  if (D != 64 && D != 128) return ADT_ERR_UNSUPPORTED;
  const adt::Q8Strides s = {{cache_layer_stride, cache_stride_b, cache_stride_h},
                            {scale_layer_stride, scale_stride_b, scale_stride_h}};
  int64_t cache_span, scale_span;
  adt_status st = adt::check_q8_cache(k_cache, v_cache, k_scale, v_scale, s, num_layers, B, Hkv, D, max_kv, false,
                                      &cache_span, &scale_span);
  if (st != ADT_OK) return st;
  const int64_t counts[3] = {num_layers, B, Hkv};
  const int64_t os[3] = {out_layer_stride, out_stride_b, out_stride_h};
  const int64_t slice = static_cast<int64_t>(max_kv) * D;
  int64_t out_span = slice;
  for (int i = 0; i < 3; ++i) {
    if (counts[i] == 1) continue;
    ADT_REQUIRE(os[i] >= slice && os[i] % 8 == 0 && os[i] <= adt::kMaxCacheStride);
    out_span += (counts[i] - 1) * os[i];
  }
  ADT_REQUIRE(adt::aligned16(k_out) && adt::aligned16(v_out));
  const void* in[4] = {k_cache, v_cache, k_scale, v_scale};
  for (int i = 0; i < 4; ++i)
    ADT_REQUIRE(!adt::spans_overlap(in[i], i < 2 ? cache_span : scale_span, k_out, out_span * 2) &&
                !adt::spans_overlap(in[i], i < 2 ? cache_span : scale_span, v_out, out_span * 2));
  ADT_REQUIRE(!adt::spans_overlap(kv_len, B * 4ll, k_out, out_span * 2) && !adt::spans_overlap(kv_len, B * 4ll, v_out, out_span * 2));
  const int64_t v_off = static_cast<int64_t>(reinterpret_cast<uintptr_t>(v_out) - reinterpret_cast<uintptr_t>(k_out)) / 2;
  ADT_REQUIRE(v_off != 0 && !adt::slices_meet(counts, os, slice, 0) && !adt::slices_meet(counts, os, slice, v_off));
  ReadQ8Params p{};
  const int rows = kThreads / (D / 16) * kReadPasses;
  p.blocks = (max_kv + rows - 1) / rows;
  const int64_t slices = counts[0] * counts[1] * counts[2];
  if (slices > (int64_t{1} << 31) - 1 || slices * p.blocks > (int64_t{1} << 31) - 1) return ADT_ERR_UNSUPPORTED;
  adt::DeviceInfo info;
  st = adt::device_info(&info);
  if (st != ADT_OK) return st;
  p.cache[0] = k_cache, p.cache[1] = v_cache;
  p.scale[0] = k_scale, p.scale[1] = v_scale;
  p.kv_len = kv_len;
  p.out[0] = reinterpret_cast<__nv_bfloat16*>(k_out);
  p.out[1] = reinterpret_cast<__nv_bfloat16*>(v_out);
  p.B = B;
  p.Hkv = Hkv;
  p.max_kv = max_kv;
  p.s = s;
  for (int i = 0; i < 3; ++i) p.os[i] = counts[i] > 1 ? os[i] : 0;
  p.err = info.error_word;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(static_cast<unsigned>(slices * p.blocks), 1, 1);
  cfg.blockDim = dim3(kThreads, 1, 1);
  cfg.stream = adt::as_stream(stream);
  cudaLaunchAttribute attr[1] = {adt::pdl_attribute()};
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  ADT_CUDA_TRY(D == 128 ? cudaLaunchKernelEx(&cfg, kv_read_q8_kernel<128>, p)
                        : cudaLaunchKernelEx(&cfg, kv_read_q8_kernel<64>, p));
  return adt::launch_status();
}

}  // extern "C"
