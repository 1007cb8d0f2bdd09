// adt_tree_attn_q8: tree-masked attention, and that of single tokens, whose
// prefix is the 8-bit cache.
//
// A CTA makes one query row of one head: 128 keys at a time, a thread a key for
// the scores, then a thread a column for the values.
#include <math.h>

#include "adt_common.cuh"
#include "kv_q8.cuh"

namespace {

constexpr int kThreads = 128;
constexpr int kMaxTreeNodes = 256;
constexpr int64_t kMaxRows = 1 << 24;  // query rows of a call
constexpr float kLog2e = 1.44269504088896340736f;
constexpr float kLn2 = 0.69314718055994530942f;

struct AttnQ8Params {
  const __nv_bfloat16* q;
  const uint8_t* cache[2];
  const uint8_t* scale[2];
  const int32_t* kv_len;
  const __nv_bfloat16* tree[2];
  const int32_t* parents;
  const int32_t* offs;
  int B, H, Hkv, group, max_nodes, max_kv;
  int64_t sb, sh, ssb, ssh;
  float scale_log2;
  __nv_bfloat16* out;
  float* lse;
  unsigned* err;
};

template <int D>
__global__ void __launch_bounds__(kThreads) tree_attn_q8_kernel(const AttnQ8Params p) {
  __shared__ float qs[D], ps[kThreads], red[4];
  __shared__ int line[kMaxTreeNodes + 1], s_count;
  adt::pdl_wait_then_release();
  const int h = blockIdx.x, t = blockIdx.y, b = blockIdx.z, tid = threadIdx.x, g = h / p.group;
  const int L = p.kv_len[b], node0 = p.offs[b], n = p.offs[b + 1] - node0;
  const bool bad_tree = n < 1 || n > p.max_nodes || node0 < 0, bad_kv = L < 0 || L > p.max_kv;
  if (bad_tree || bad_kv) {
    if (tid == 0 && h == 0 && t == 0) adt::raise_error(p.err, bad_tree ? ADT_DEVERR_BAD_TREE : ADT_DEVERR_KV_RANGE);
    return;
  }
  if (t >= n) return;
  if (tid == 0) {
    int c = 0, j = t;
    while (true) {
      line[c++] = j;
      const int up = p.parents[node0 + j];
      if (j == 0 ? up >= 0 : (up < 0 || up >= j)) {
        c = -1;
        break;
      }
      if (j == 0) break;
      j = up;
    }
    s_count = c;
  }
  const int64_t row = static_cast<int64_t>(node0 + t) * p.H + h;
  for (int d = tid; d < D; d += kThreads) qs[d] = __bfloat162float(p.q[row * D + d]);
  __syncthreads();
  const int own = s_count;
  if (own < 0) {
    if (tid == 0 && h == 0) adt::raise_error(p.err, ADT_DEVERR_BAD_TREE);
    return;
  }
  const int64_t c0 = b * p.sb + g * p.sh, s0 = b * p.ssb + g * p.ssh;
  const int64_t keys = static_cast<int64_t>(L) + own;
  float m = -INFINITY, l = 0.f, acc = 0.f;
  for (int64_t j0 = 0; j0 < keys; j0 += kThreads) {
    const int64_t j = j0 + tid;
    float x = -INFINITY;
    if (j < keys) {
      x = 0.f;
      if (j < L) {
        const uint8_t* k = p.cache[0] + c0 + j * D;
        for (int d = 0; d < D; d += 2) {
          const float2 f = adt::e4m3x2_to_f32(*reinterpret_cast<const uint16_t*>(k + d));
          x = fmaf(f.x, qs[d], fmaf(f.y, qs[d + 1], x));
        }
        x *= adt::q8_scale(p.scale[0][s0 + j]);
      } else {
        const __nv_bfloat16* k = p.tree[0] + (static_cast<int64_t>(node0 + line[j - L]) * p.Hkv + g) * D;
        for (int d = 0; d < D; ++d) x = fmaf(__bfloat162float(k[d]), qs[d], x);
      }
      x *= p.scale_log2;
    }
    const float w = adt::warp_max(x);
    if ((tid & 31) == 0) red[tid >> 5] = w;
    __syncthreads();
    const float top = fmaxf(m, fmaxf(fmaxf(red[0], red[1]), fmaxf(red[2], red[3])));
    const float base = top == -INFINITY ? 0.f : top, shrink = exp2f(m - base);
    ps[tid] = j < keys ? exp2f(x - base) : 0.f;
    __syncthreads();
    m = top;
    const int here = static_cast<int>(keys - j0 < kThreads ? keys - j0 : kThreads);
    acc *= shrink;
    l *= shrink;
    for (int i = 0; i < here; ++i) {
      l += ps[i];
      if (tid < D) {
        const int64_t jj = j0 + i;
        const float v = jj < L ? adt::e4m3x2_to_f32(p.cache[1][c0 + jj * D + tid]).x * adt::q8_scale(p.scale[1][s0 + jj])
                               : __bfloat162float(p.tree[1][(static_cast<int64_t>(node0 + line[jj - L]) * p.Hkv + g) * D + tid]);
        acc = fmaf(ps[i], v, acc);
      }
    }
    __syncthreads();
  }
  if (tid < D) p.out[row * D + tid] = __float2bfloat16(acc / l);
  if (tid == 0 && p.lse) p.lse[row] = (m + log2f(l)) * kLn2;
}

}  // namespace

extern "C" {

size_t adt_tree_attn_q8_workspace_size(int32_t B, int32_t H, int32_t Hkv, int32_t D, int32_t max_nodes, int32_t max_kv) {
  if (B < 1 || H < 1 || Hkv < 1 || H % Hkv != 0 || (D != 64 && D != 128) || max_kv < 0 || max_nodes < 1 ||
      max_nodes > kMaxTreeNodes || static_cast<int64_t>(B) * max_nodes * H > kMaxRows)
    return 0;
  return 16;
}

adt_status adt_tree_attn_q8(const adt_bf16* q, const uint8_t* k_cache, const uint8_t* v_cache, const uint8_t* k_scale,
                            const uint8_t* v_scale, const int32_t* kv_len, int64_t cache_stride_b,
                            int64_t cache_stride_h, int64_t scale_stride_b, int64_t scale_stride_h,
                            const adt_bf16* k_tree, const adt_bf16* v_tree, const int32_t* parents,
                            const int32_t* node_offsets, int32_t B, int32_t H, int32_t Hkv, int32_t D,
                            int32_t max_nodes, int32_t max_kv, float softmax_scale, adt_bf16* out, float* lse,
                            void* workspace, size_t workspace_bytes, void* stream) {
  adt::TraceRange trace_("adt_tree_attn_q8");
  ADT_REQUIRE(q && k_cache && v_cache && k_scale && v_scale && kv_len && k_tree && v_tree && parents && node_offsets && out);
  ADT_REQUIRE(B >= 1 && B <= 65535 && H >= 1 && H <= 65535 && Hkv >= 1 && H % Hkv == 0);
  ADT_REQUIRE(max_nodes >= 1 && max_kv >= 0 && max_kv < (1 << 30));
  ADT_REQUIRE(static_cast<int64_t>(B) * max_nodes * H <= kMaxRows);
  if (max_nodes > kMaxTreeNodes) return ADT_ERR_UNSUPPORTED;
  ADT_REQUIRE(softmax_scale > 0.f && softmax_scale < 1e30f);
  if (D != 64 && D != 128) return ADT_ERR_UNSUPPORTED;
  const adt::Q8Strides s = {{0, cache_stride_b, cache_stride_h}, {0, scale_stride_b, scale_stride_h}};
  int64_t cache_span, scale_span;
  adt_status st = adt::check_q8_cache(k_cache, v_cache, k_scale, v_scale, s, 1, B, Hkv, D, max_kv, false, &cache_span,
                                      &scale_span);
  if (st != ADT_OK) return st;
  ADT_REQUIRE(adt::aligned16(q) && adt::aligned16(k_tree) && adt::aligned16(v_tree) && adt::aligned16(out));
  if (!workspace || workspace_bytes < 16 || !adt::aligned16(workspace)) return ADT_ERR_WORKSPACE;
  adt::DeviceInfo info;
  st = adt::device_info(&info);
  if (st != ADT_OK) return st;
  AttnQ8Params p{};
  p.q = reinterpret_cast<const __nv_bfloat16*>(q);
  p.cache[0] = k_cache, p.cache[1] = v_cache;
  p.scale[0] = k_scale, p.scale[1] = v_scale;
  p.kv_len = kv_len;
  p.tree[0] = reinterpret_cast<const __nv_bfloat16*>(k_tree);
  p.tree[1] = reinterpret_cast<const __nv_bfloat16*>(v_tree);
  p.parents = parents;
  p.offs = node_offsets;
  p.B = B;
  p.H = H;
  p.Hkv = Hkv;
  p.group = H / Hkv;
  p.max_nodes = max_nodes;
  p.max_kv = max_kv;
  p.sb = B > 1 ? cache_stride_b : 0, p.sh = Hkv > 1 ? cache_stride_h : 0;
  p.ssb = B > 1 ? scale_stride_b : 0, p.ssh = Hkv > 1 ? scale_stride_h : 0;
  p.scale_log2 = softmax_scale * kLog2e;
  p.out = reinterpret_cast<__nv_bfloat16*>(out);
  p.lse = lse;
  p.err = info.error_word;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(static_cast<unsigned>(H), static_cast<unsigned>(max_nodes), static_cast<unsigned>(B));
  cfg.blockDim = dim3(kThreads, 1, 1);
  cfg.stream = adt::as_stream(stream);
  cudaLaunchAttribute attr[1] = {adt::pdl_attribute()};
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  ADT_CUDA_TRY(D == 128 ? cudaLaunchKernelEx(&cfg, tree_attn_q8_kernel<128>, p)
                        : cudaLaunchKernelEx(&cfg, tree_attn_q8_kernel<64>, p));
  return adt::launch_status();
}

}  // extern "C"
