// adt_kv_evict: the cache cut down to `budget` rows a tree, layer and kv head:
// the first n_sink rows, the last n_recent, and between them those with the
// highest scores (ties to the lowest index), in the order they had.
//
// A CTA selects the rows of one (layer, tree, kv head) slice by a radix search
// for the lowest score that stays, marks them in a bit mask in shared memory,
// and moves them.  A kept row never moves up, so chunks of rows taken in
// ascending order can be moved in place: a chunk's destinations lie below the
// sources of every later chunk, and only its own loads have to be done before
// its stores.
#include <math.h>

#include "adt_common.cuh"

namespace {

constexpr int kThreads = 256;
constexpr int kMaxRows = 1 << 20;  // max_kv: the bit mask takes 128 KB
constexpr int kWindow = 4096;      // rows whose kept ones are listed at a time
constexpr int kVecs = 8;           // 16-byte vectors that a thread moves at a time

struct EvictParams {
  const uint4* src[2];   // K, V
  uint4* dst[2];
  const float* score;
  float* score_out;      // or NULL
  const int32_t* kv_len;
  int32_t* kv_len_out;   // or NULL
  int32_t* keep_idx;     // [layers][B][Hkv][budget], or NULL
  int B, Hkv, D, max_kv, budget, n_sink, n_recent, in_place;
  int64_t sls, ssb, ssh;     // source cache strides (elements)
  int64_t dls, dsb, dsh;     // destination cache strides
  int64_t cls, csb, csh;     // score strides
  int64_t ols, osb, osh;     // score_out strides
  unsigned* err;
};

// Order of a score: larger scores get larger keys, NaN the largest.
__device__ __forceinline__ uint32_t score_key(float s) { return isnan(s) ? 0xffffffffu : adt::float_order_key(s); }

struct Scratch {
  uint32_t hist[2048];
  uint16_t list[kWindow];   // kept rows of a window, relative to its first
  float score[kWindow];     // their scores
  uint32_t warp[kThreads / 32];
  uint32_t prefix, need, count;
};

// Exclusive prefix sum of one value a thread; *total gets the sum.
__device__ __forceinline__ uint32_t block_scan(uint32_t v, uint32_t* warp_sums, uint32_t* total) {
  const int lane = threadIdx.x & 31, w = threadIdx.x >> 5;
  uint32_t x = v;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const uint32_t y = __shfl_up_sync(adt::kFullMask, x, o);
    if (lane >= o) x += y;
  }
  if (lane == 31) warp_sums[w] = x;
  __syncthreads();
  uint32_t base = 0, all = 0;
#pragma unroll
  for (int i = 0; i < kThreads / 32; ++i) {
    const uint32_t s = warp_sums[i];
    if (i < w) base += s;
    all += s;
  }
  __syncthreads();
  *total = all;
  return base + x - v;
}

// Marks in `mask` the rows of [0, L) that stay; `want` of the rows [lo, hi) do.
__device__ void select_rows(const float* score, int L, int lo, int hi, int want, uint32_t* mask, Scratch* sc) {
  const int tid = threadIdx.x, words = (L + 31) / 32;
  // Threshold: keys whose high bits (of the digits found) exceed `prefix` stay,
  // of those that equal it the first `need`.
  uint32_t prefix = 0, digits = 0, need = want, count = 0;
  if (want > 0) {
    const int shift[3] = {21, 10, 0}, bits[3] = {11, 11, 10};
    for (int d = 0; d < 3; ++d) {
      for (int i = tid; i < 2048; i += kThreads) sc->hist[i] = 0;
      __syncthreads();
      for (int j = lo + tid; j < hi; j += kThreads) {
        const uint32_t k = score_key(score[j]);
        if ((k & digits) == prefix) atomicAdd(&sc->hist[(k >> shift[d]) & ((1u << bits[d]) - 1)], 1u);
      }
      __syncthreads();
      // Thread t holds eight bins, the highest first; the bin where the count
      // from above reaches `need` is the digit.
      uint32_t c[8], sum = 0, total;
#pragma unroll
      for (int i = 0; i < 8; ++i) sum += c[i] = sc->hist[2047 - (tid * 8 + i)];
      uint32_t above = block_scan(sum, sc->warp, &total);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        if (above < need && need <= above + c[i]) {
          sc->prefix = prefix | (static_cast<uint32_t>(2047 - (tid * 8 + i)) << shift[d]);
          sc->need = need - above;
          sc->count = c[i];
        }
        above += c[i];
      }
      __syncthreads();
      prefix = sc->prefix;
      need = sc->need;
      count = sc->count;
      digits |= ((1u << bits[d]) - 1) << shift[d];
      __syncthreads();
      if (count == need) break;
    }
  }
  uint32_t ties = 0;  // rows before this turn whose key equals the threshold
  const bool all_ties = want == 0 || count == need;
  for (int j0 = 0; j0 < words * 32; j0 += kThreads) {
    const int j = j0 + tid;
    bool stay = j < L && (j < lo || j >= hi), tie = false;
    if (want > 0 && j >= lo && j < hi) {
      const uint32_t k = score_key(score[j]) & digits;
      stay = k > prefix;
      tie = k == prefix;
    }
    if (all_ties) {
      stay |= tie && want > 0;
    } else {
      uint32_t total;
      const uint32_t before = block_scan(tie ? 1u : 0u, sc->warp, &total);
      stay |= tie && ties + before < need;
      ties += total;
    }
    const uint32_t bits = __ballot_sync(adt::kFullMask, stay);
    if ((tid & 31) == 0 && j < words * 32) mask[j >> 5] = bits;
  }
  __syncthreads();
}

__global__ void __launch_bounds__(kThreads) kv_evict_kernel(const EvictParams p) {
  extern __shared__ uint32_t mask[];
  __shared__ Scratch sc;
  adt::pdl_wait_then_release();
  const int slice = blockIdx.x, tid = threadIdx.x;
  const int g = slice % p.Hkv, b = slice / p.Hkv % p.B, l = slice / p.Hkv / p.B;
  const int L = p.kv_len[b];
  const bool ok = L >= 0 && L <= p.max_kv;
  const int n = ok ? min(L, p.budget) : 0;
  if (g == 0 && l == 0 && tid == 0) {
    if (!ok) adt::raise_error(p.err, ADT_DEVERR_KV_RANGE);
    if (p.kv_len_out) p.kv_len_out[b] = ok ? n : L;
  }
  if (!ok) return;
  const float* score = p.score + l * p.cls + b * p.csb + g * p.csh;
  float* score_out = p.score_out ? p.score_out + l * p.ols + b * p.osb + g * p.osh : nullptr;
  int32_t* idx = p.keep_idx ? p.keep_idx + static_cast<int64_t>(slice) * p.budget : nullptr;
  const int lo = L > n ? p.n_sink : L, hi = L > n ? L - p.n_recent : L;
  select_rows(score, L, lo, hi, n - lo - (L - hi), mask, &sc);
  const int vpr = p.D / 8;
  const int64_t src0 = (l * p.sls + b * p.ssb + g * p.ssh) / 8, dst0 = (l * p.dls + b * p.dsb + g * p.dsh) / 8;
  int done = 0;  // rows moved before this window
  for (int w0 = 0; w0 < L; w0 += kWindow) {
    const int words = (min(L - w0, kWindow) + 31) / 32;
    uint32_t m = tid < words ? mask[w0 / 32 + tid] : 0u, listed;
    uint32_t at = block_scan(__popc(m), sc.warp, &listed);
    const int rows = static_cast<int>(listed);
    for (; m; m &= m - 1) sc.list[at++] = static_cast<uint16_t>(tid * 32 + __ffs(m) - 1);
    __syncthreads();
    if (score_out)
      for (int r = tid; r < rows; r += kThreads) sc.score[r] = score[w0 + sc.list[r]];
    __syncthreads();
    for (int r = tid; r < rows; r += kThreads) {
      if (score_out) score_out[done + r] = sc.score[r];
      if (idx) idx[done + r] = w0 + sc.list[r];
    }
    const int total = rows * vpr;
    for (int x = 0; x < 2; ++x) {
      const uint4* src = p.src[x] + src0;
      uint4* dst = p.dst[x] + dst0;
      for (int i0 = 0; i0 < total; i0 += kThreads * kVecs) {
        uint4 v[kVecs];
#pragma unroll
        for (int e = 0; e < kVecs; ++e) {
          const int i = i0 + e * kThreads + tid, r = i / vpr;
          if (i < total) v[e] = src[static_cast<int64_t>(w0 + sc.list[r]) * vpr + i % vpr];
        }
        if (p.in_place) __syncthreads();
#pragma unroll
        for (int e = 0; e < kVecs; ++e) {
          const int i = i0 + e * kThreads + tid, r = i / vpr;
          if (i < total && !(p.in_place && w0 + sc.list[r] == done + r))
            dst[static_cast<int64_t>(done + r) * vpr + i % vpr] = v[e];
        }
      }
    }
    __syncthreads();
    done += rows;
  }
  if (idx)
    for (int r = n + tid; r < p.budget; r += kThreads) idx[r] = -1;
}

// Whether the byte ranges that two caches of the same shape span overlap.
bool caches_overlap(const void* a, int64_t na, const void* b, int64_t nb) {
  const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
  return x < y + nb && y < x + na;
}

}  // namespace

extern "C" {

adt_status adt_kv_evict(const adt_bf16* k_src, const adt_bf16* v_src, int64_t src_layer_stride, int64_t src_stride_b,
                        int64_t src_stride_h, const float* score, int64_t score_layer_stride, int64_t score_stride_b,
                        int64_t score_stride_h, const int32_t* kv_len, int32_t* kv_len_out, adt_bf16* k_dst,
                        adt_bf16* v_dst, int64_t dst_layer_stride, int64_t dst_stride_b, int64_t dst_stride_h,
                        float* score_out, int64_t score_out_layer_stride, int64_t score_out_stride_b,
                        int64_t score_out_stride_h, int32_t* keep_idx, int32_t B, int32_t Hkv, int32_t D,
                        int32_t num_layers, int32_t max_kv, int32_t budget, int32_t n_sink, int32_t n_recent,
                        void* stream) {
  adt::TraceRange trace_("adt_kv_evict");
  ADT_REQUIRE(k_src && v_src && score && kv_len && k_dst && v_dst);
  ADT_REQUIRE(B >= 1 && B <= 65535 && Hkv >= 1 && Hkv <= 65535 && num_layers >= 1 && num_layers <= 65535);
  ADT_REQUIRE(max_kv >= 1 && budget >= 1 && n_sink >= 0 && n_recent >= 0 &&
              static_cast<int64_t>(n_sink) + n_recent <= budget);
  ADT_REQUIRE(kv_len_out != kv_len);
  if (D != 64 && D != 128) return ADT_ERR_UNSUPPORTED;
  if (max_kv > kMaxRows) return ADT_ERR_UNSUPPORTED;
  const int64_t keep = max_kv < budget ? max_kv : budget;  // rows that a destination slice holds
  const int64_t counts[3] = {num_layers, B, Hkv};
  const int64_t ss[3] = {src_layer_stride, src_stride_b, src_stride_h};
  const int64_t ds[3] = {dst_layer_stride, dst_stride_b, dst_stride_h};
  const int64_t cs[3] = {score_layer_stride, score_stride_b, score_stride_h};
  const int64_t os[3] = {score_out_layer_stride, score_out_stride_b, score_out_stride_h};
  int64_t src_span = static_cast<int64_t>(max_kv) * D, dst_span = keep * D, c_span = max_kv, o_span = keep;
  for (int i = 0; i < 3; ++i) {
    ADT_REQUIRE(ss[i] >= 0 && ds[i] >= 0 && cs[i] >= 0 && ss[i] % 8 == 0 && ds[i] % 8 == 0 &&
                (!score_out || os[i] >= 0));
    ADT_REQUIRE(counts[i] == 1 || (ss[i] >= static_cast<int64_t>(max_kv) * D && ds[i] >= keep * D && cs[i] >= max_kv &&
                                   (!score_out || os[i] >= keep)));
    src_span += (counts[i] - 1) * ss[i];
    dst_span += (counts[i] - 1) * ds[i];
    c_span += (counts[i] - 1) * cs[i];
    o_span += (counts[i] - 1) * os[i];
  }
  ADT_REQUIRE(adt::aligned16(k_src) && adt::aligned16(v_src) && adt::aligned16(k_dst) && adt::aligned16(v_dst));
  // In place (both caches where they are), or into caches apart from the source.
  auto same = [&](const int64_t* a, const int64_t* c) {
    return (counts[0] == 1 || a[0] == c[0]) && (counts[1] == 1 || a[1] == c[1]) && (counts[2] == 1 || a[2] == c[2]);
  };
  const bool in_place = k_src == k_dst && v_src == v_dst && same(ss, ds);
  if (!in_place)
    ADT_REQUIRE(!caches_overlap(k_src, src_span * 2, k_dst, dst_span * 2) &&
                !caches_overlap(v_src, src_span * 2, v_dst, dst_span * 2) &&
                !caches_overlap(k_src, src_span * 2, v_dst, dst_span * 2) &&
                !caches_overlap(v_src, src_span * 2, k_dst, dst_span * 2));
  if (score_out && !(score_out == score && same(cs, os)))
    ADT_REQUIRE(!caches_overlap(score, c_span * 4, score_out, o_span * 4));
  const int64_t slices = counts[0] * counts[1] * counts[2];
  if (slices > (1 << 28)) return ADT_ERR_UNSUPPORTED;
  adt::DeviceInfo info;
  adt_status st = adt::device_info(&info);
  if (st != ADT_OK) return st;
  EvictParams p{};
  p.src[0] = reinterpret_cast<const uint4*>(k_src);
  p.src[1] = reinterpret_cast<const uint4*>(v_src);
  p.dst[0] = reinterpret_cast<uint4*>(k_dst);
  p.dst[1] = reinterpret_cast<uint4*>(v_dst);
  p.score = score;
  p.score_out = score_out;
  p.kv_len = kv_len;
  p.kv_len_out = kv_len_out;
  p.keep_idx = keep_idx;
  p.B = B;
  p.Hkv = Hkv;
  p.D = D;
  p.max_kv = max_kv;
  p.budget = budget;
  p.n_sink = n_sink;
  p.n_recent = n_recent;
  p.in_place = in_place;
  p.sls = ss[0], p.ssb = ss[1], p.ssh = ss[2];
  p.dls = ds[0], p.dsb = ds[1], p.dsh = ds[2];
  p.cls = cs[0], p.csb = cs[1], p.csh = cs[2];
  p.ols = os[0], p.osb = os[1], p.osh = os[2];
  p.err = info.error_word;
  const size_t smem = static_cast<size_t>((max_kv + 31) / 32) * 4;
  if (smem > 8 * 1024) {  // with the static part, past what needs no opt-in
    static unsigned configured[2] = {0u, 0u};  // bit per device (< 64)
    const unsigned bit = 1u << (info.device & 31);
    unsigned& word = configured[(info.device >> 5) & 1];
    if (!(__atomic_load_n(&word, __ATOMIC_ACQUIRE) & bit)) {
      ADT_CUDA_TRY(cudaFuncSetAttribute(kv_evict_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kMaxRows / 8));
      __atomic_fetch_or(&word, bit, __ATOMIC_ACQ_REL);
    }
  }
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(static_cast<unsigned>(slices), 1, 1);
  cfg.blockDim = dim3(kThreads, 1, 1);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = adt::as_stream(stream);
  cudaLaunchAttribute attr[1] = {adt::pdl_attribute()};
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  ADT_CUDA_TRY(cudaLaunchKernelEx(&cfg, kv_evict_kernel, p));
  return adt::launch_status();
}

}  // extern "C"
