// adt_kv_score: the attention weight that every cached row got from the tokens
// just committed, added to a running score (what adt_kv_evict goes by).
//
// Row j of the cache gets exp(scale q_i . k_j - lse_i) from path node i and
// head h, where lse is what adt_tree_attn returned for that query: the softmax
// is known to be normalised by it, so one pass over K does, with no running
// maximum and no V.
#include "adt_common.cuh"

namespace {

constexpr int kThreads = 128;  // keys of a CTA, a thread each
constexpr int kRows = 16;      // query rows staged at a time
constexpr float kLog2e = 1.44269504088896340736f;

struct ScoreParams {
  const __nv_bfloat16* q;
  const float* lse;
  const __nv_bfloat16* k;
  const int32_t* kv_len;
  const int32_t* offs;
  const int32_t* path;
  const int32_t* alen;
  const float* score_in;
  float* score_out;
  int B, H, Hkv, group, max_path, max_kv;
  int64_t qls, lls;            // layer strides of q and lse
  int64_t cls, csb, csh;       // cache strides
  int64_t sls, ssb, ssh;       // score strides
  float scale_log2, decay;
  unsigned* err;
};

template <int D>
__global__ void __launch_bounds__(kThreads) kv_score_kernel(const ScoreParams p) {
  __shared__ float s_q[kRows][D];
  __shared__ float s_lse[kRows];
  adt::pdl_wait_then_release();
  const int slice = blockIdx.x, tid = threadIdx.x;
  const int g = slice % p.Hkv, b = slice / p.Hkv % p.B, l = slice / p.Hkv / p.B;
  const int L = p.kv_len[b], a = p.alen[b];
  if (a < 0 || a >= p.max_path || L < 0 || static_cast<int64_t>(L) + a + 1 > p.max_kv) {
    if (blockIdx.y == 0 && g == 0 && l == 0 && tid == 0) adt::raise_error(p.err, ADT_DEVERR_KV_RANGE);
    return;
  }
  const int j0 = blockIdx.y * kThreads, j = j0 + tid;
  if (j0 > L + a) return;
  const bool there = j <= L + a;
  float key[D];
  const __nv_bfloat16* row = p.k + l * p.cls + b * p.csb + g * p.csh + static_cast<int64_t>(there ? j : 0) * D;
#pragma unroll
  for (int d = 0; d < D; ++d) key[d] = __bfloat162float(row[d]);
  const int node0 = p.offs[b], n = p.offs[b + 1] - node0;
  const int rows = (a + 1) * p.group;
  float acc = 0.f;
  for (int r0 = 0; r0 < rows; r0 += kRows) {
    __syncthreads();
    for (int e = tid; e < kRows * D; e += kThreads) {
      const int r = r0 + e / D, d = e % D;
      float x = 0.f;
      if (r < rows) {
        const int i = r / p.group, h = g * p.group + r % p.group;
        const int node = p.path[static_cast<int64_t>(b) * p.max_path + i];
        const bool ok = node >= 0 && node < n;
        const int64_t at = static_cast<int64_t>(node0 + (ok ? node : 0)) * p.H + h;
        if (ok) x = __bfloat162float(p.q[l * p.qls + at * D + d]);
        if (d == 0) {
          const float lse = ok ? p.lse[l * p.lls + at] : -INFINITY;
          s_lse[e / D] = lse == -INFINITY ? INFINITY : lse * kLog2e;
          if (!ok && j0 == 0 && g == 0 && l == 0) adt::raise_error(p.err, ADT_DEVERR_BAD_PATH);
        }
      }
      s_q[e / D][d] = x;
    }
    __syncthreads();
    for (int r = 0; r < kRows && r0 + r < rows; ++r) {
      if (j > L + (r0 + r) / p.group || s_lse[r] == INFINITY) continue;
      float s = 0.f;
#pragma unroll
      for (int d = 0; d < D; ++d) s += s_q[r][d] * key[d];
      acc += exp2f(s * p.scale_log2 - s_lse[r]);
    }
  }
  if (there) {
    const int64_t o = l * p.sls + b * p.ssb + g * p.ssh + j;
    p.score_out[o] = (j < L && p.decay != 0.f ? p.decay * p.score_in[o] : 0.f) + acc;
  }
}

}  // namespace

extern "C" {

adt_status adt_kv_score(const adt_bf16* q, const float* lse, const adt_bf16* k_cache, const int32_t* kv_len,
                        const int32_t* node_offsets, const int32_t* path, int32_t max_path, const int32_t* accept_len,
                        int32_t B, int32_t H, int32_t Hkv, int32_t D, int32_t num_layers, int32_t max_kv,
                        int64_t q_layer_stride, int64_t lse_layer_stride, int64_t cache_layer_stride,
                        int64_t cache_stride_b, int64_t cache_stride_h, float softmax_scale, float decay,
                        const float* score_in, float* score_out, int64_t score_layer_stride, int64_t score_stride_b,
                        int64_t score_stride_h, void* stream) {
  adt::TraceRange trace_("adt_kv_score");
  ADT_REQUIRE(q && lse && k_cache && kv_len && node_offsets && path && accept_len && score_in && score_out);
  ADT_REQUIRE(B >= 1 && B <= 65535 && Hkv >= 1 && H >= Hkv && H % Hkv == 0 && H <= 65535);
  ADT_REQUIRE(num_layers >= 1 && num_layers <= 65535);
  ADT_REQUIRE(max_path >= 1 && max_path <= (1 << 20) && max_kv >= 1 && max_kv < (1 << 30));
  ADT_REQUIRE(softmax_scale > 0.f && softmax_scale < 1e30f && decay >= 0.f && decay <= 1.f);
  if (D != 64 && D != 128) return ADT_ERR_UNSUPPORTED;
  ADT_REQUIRE(cache_layer_stride >= 0 && cache_stride_b >= 0 && cache_stride_h >= 0 && q_layer_stride >= 0 &&
              lse_layer_stride >= 0 && score_layer_stride >= 0 && score_stride_b >= 0 && score_stride_h >= 0);
  ADT_REQUIRE(cache_layer_stride % 8 == 0 && cache_stride_b % 8 == 0 && cache_stride_h % 8 == 0 &&
              q_layer_stride % 8 == 0);
  const int64_t rows = static_cast<int64_t>(max_kv) * D;
  ADT_REQUIRE((Hkv == 1 || (cache_stride_h >= rows && score_stride_h >= max_kv)) &&
              (B == 1 || (cache_stride_b >= rows && score_stride_b >= max_kv)) &&
              (num_layers == 1 || (cache_layer_stride >= rows && score_layer_stride >= max_kv)));
  ADT_REQUIRE(adt::aligned16(q) && adt::aligned16(k_cache));
  const int64_t slices = static_cast<int64_t>(num_layers) * B * Hkv;
  if (score_in != score_out) {
    const uint64_t span = (static_cast<uint64_t>(num_layers - 1) * score_layer_stride + (B - 1) * score_stride_b +
                           (Hkv - 1) * score_stride_h + max_kv) * sizeof(float);
    const uintptr_t x = reinterpret_cast<uintptr_t>(score_in), y = reinterpret_cast<uintptr_t>(score_out);
    ADT_REQUIRE(x >= y + span || y >= x + span);
  }
  if (slices > (1 << 22)) return ADT_ERR_UNSUPPORTED;
  adt::DeviceInfo info;
  adt_status st = adt::device_info(&info);
  if (st != ADT_OK) return st;
  ScoreParams p{};
  p.q = reinterpret_cast<const __nv_bfloat16*>(q);
  p.lse = lse;
  p.k = reinterpret_cast<const __nv_bfloat16*>(k_cache);
  p.kv_len = kv_len;
  p.offs = node_offsets;
  p.path = path;
  p.alen = accept_len;
  p.score_in = score_in;
  p.score_out = score_out;
  p.B = B;
  p.H = H;
  p.Hkv = Hkv;
  p.group = H / Hkv;
  p.max_path = max_path;
  p.max_kv = max_kv;
  p.qls = q_layer_stride;
  p.lls = lse_layer_stride;
  p.cls = cache_layer_stride;
  p.csb = cache_stride_b;
  p.csh = cache_stride_h;
  p.sls = score_layer_stride;
  p.ssb = score_stride_b;
  p.ssh = score_stride_h;
  p.scale_log2 = softmax_scale * kLog2e;
  p.decay = decay;
  p.err = info.error_word;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(static_cast<unsigned>(slices), static_cast<unsigned>((max_kv + kThreads - 1) / kThreads), 1);
  cfg.blockDim = dim3(kThreads, 1, 1);
  cfg.stream = adt::as_stream(stream);
  cudaLaunchAttribute attr[1] = {adt::pdl_attribute()};
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  if (D == 128)
    ADT_CUDA_TRY(cudaLaunchKernelEx(&cfg, kv_score_kernel<128>, p));
  else
    ADT_CUDA_TRY(cudaLaunchKernelEx(&cfg, kv_score_kernel<64>, p));
  return adt::launch_status();
}

}  // extern "C"
