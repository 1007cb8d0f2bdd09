// adt_kv_evict: the cache cut down to `budget` rows a tree, layer and kv head:
// the first n_sink rows, the last n_recent, and between them those with the
// highest scores (ties to the lowest index), in the order they had.
//
// A CTA (or a few, each with K or V or some of their columns) takes one (layer,
// tree, kv head) slice.  It searches for the lowest score that stays: a
// histogram of the scores over their range (by order, 2048 bins), then over the
// range of the bin that the last kept score falls into, until that bin is kept
// whole or holds one value.  Then, window by window, it lists the rows that stay
// and moves them: every thread copies its vectors of a chunk of rows into slots
// of its own in shared memory, asynchronously and three chunks ahead, and from
// there to the rows' new place.  A kept row never moves up, so chunks of rows
// taken in ascending order can be moved in place: a chunk's destinations lie
// below the sources of every later chunk, whose loads may be under way, and its
// stores wait (at a barrier) for all loads of its own and the chunks before.
//
// Bound by HBM where slices are many: 32 layers of a 7B cache, 2304 of 2400 rows
// kept, 370 us for 2.4 GB read and written (97 % of the measured copy rate).
// With fewer, nothing hides the search: its chain of passes over a slice's
// scores takes 4 us at 1700 rows and 8 us at 5120 (a pass is bound by its
// instructions, so keys are kept, not scores; a tenth of it is instructions
// fetched cold).  256 slices of 1777 to 6001 rows, 2048 kept, 83 us of 61 (76 in a
// graph of such calls); 1440 of 1577 and 1693 rows of 128 bytes, 512 kept, 76 us
// of 58.  Four CTAs an SM hide loads best with three chunks ahead (six chunks and
// half the CTAs: 75 -> 87 us for the last); 512 threads a CTA cost it 5 us, 128
// 6 us and the first 38.  Bulk copies a run of rows at a time were as fast for long
// runs (371 us) but not for short ones (431 against 93 us then for the 256
// slices).  Bins over the scores' range spread the counts; those over the top bits
// of fp32 met 30 bins and cost 4 us at 5120 rows.
#include <math.h>

#include "adt_common.cuh"
#include "slices.h"
#include "sm100.cuh"

namespace {

constexpr int kVecs = 2;   // 16-byte vectors of a thread in a chunk
constexpr int kDepth = 4;  // chunks that its slots hold
constexpr int kAhead = 3;  // chunks that loads run ahead of stores
constexpr int64_t kMaxStride = int64_t{1} << 40;
constexpr int kBinBits = 11;
constexpr int kBins = 1 << kBinBits;

// Sizes of a CTA of T threads.
template <int T>
struct Cta {
  static constexpr int kWarps = T / 32;
  static constexpr int kWindow = T * 32;  // rows whose kept ones are listed at a time: a word of bits for every thread
  static constexpr int kSlotBytes = kDepth * kVecs * T * 16;
  static_assert(kWindow * 4 <= kSlotBytes, "a window's keys share the slots");
  static_assert(kBins * 4 <= kWindow * 2, "its bins share the list");
  struct Scratch {
    union {
      uint16_t list[kWindow];  // kept rows of a window, relative to its first
      uint32_t hist[kBins];    // the search's bins
    };
    uint32_t warp[2 * kWarps];
    uint32_t bin, need, count;
  };
  static constexpr int kSmem = kSlotBytes + static_cast<int>(sizeof(Scratch));
};

struct EvictParams {
  const uint8_t* src[2];  // K, V
  uint8_t* dst[2];
  const float* score;
  float* score_out;       // or NULL
  const int32_t* kv_len;
  int32_t* kv_len_out;    // or NULL
  int32_t* keep_idx;      // [layers][B][Hkv][budget], or NULL
  int B, Hkv, max_kv, budget, n_sink, n_recent, in_place;
  int parts;              // CTAs a slice: 1, or K and V apart (2) with 1, 2 or 4 shares of their columns
  int row_bytes;          // of a cache row
  int64_t sls, ssb, ssh;  // source cache strides (bytes)
  int64_t dls, dsb, dsh;  // destination cache strides (bytes)
  int64_t cls, csb, csh;  // score strides (elements)
  int64_t ols, osb, osh;  // score_out strides (elements)
  unsigned* err;
};

// Order of a score: larger scores get larger keys, from 2^23 - 2 for -inf up.
// Adding zero makes -0 equal +0 and every NaN the canonical one (sign clear, all
// bits set), the largest.
__device__ __forceinline__ uint32_t score_key(float s) {
  const uint32_t u = __float_as_uint(__fadd_rn(s, 0.f));
  return (u ^ (static_cast<uint32_t>(static_cast<int32_t>(u) >> 31) | 0x80000000u)) - 1u;
}
// Above every score's key: rows that stay whatever their score.  (Below every
// key: 0, rows that are not there.)
constexpr uint32_t kStays = 0xffffffffu;

// Exclusive prefix sum of one value a thread; *total gets the sum.
template <int T>
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
  for (int i = 0; i < Cta<T>::kWarps; ++i) {
    const uint32_t s = warp_sums[i];
    if (i < w) base += s;
    all += s;
  }
  __syncthreads();
  *total = all;
  return base + x - v;
}

// Rows with keys above `last` stay, and of those with keys in [first, last] the
// lowest `ties` rows (ties < 0: all).
struct Cut {
  uint32_t first, last;
  int ties;
};

// Keys of the rows w0 .. of a window, into shared memory; the rows from `hi` on
// and those before `lo` stay.
template <int T>
__device__ __forceinline__ void window_keys(const float* score, int w0, int L, int lo, int hi, uint32_t* keys,
                                            uint32_t* low, uint32_t* high) {
  const int rows = min(L - w0, Cta<T>::kWindow);
#pragma unroll 8
  for (int r = threadIdx.x; r < rows; r += T) {
    uint32_t k = score_key(score[w0 + r]);
    if (w0 + r >= lo && w0 + r < hi) {
      *low = min(*low, k);
      *high = max(*high, k);
    } else {
      k = kStays;
    }
    keys[r] = k;
  }
  const int end = (rows + 31) & ~31;
  if (rows + static_cast<int>(threadIdx.x) < end) keys[rows + threadIdx.x] = 0u;
}

// The cut that keeps `want` of the rows [lo, hi).  Of a slice that is one window
// the keys are left in shared memory.
template <int T>
__device__ __forceinline__ Cut find_cut(const float* score, uint32_t* keys, bool small, int L, int lo, int hi, int want,
                                        typename Cta<T>::Scratch* sc) {
  constexpr int kThreads = T, kWarps = Cta<T>::kWarps, kWindow = Cta<T>::kWindow;
  const int tid = threadIdx.x;
  uint32_t low = 0xffffffffu, high = 0u;
  for (int i = tid; i < kBins; i += kThreads) sc->hist[i] = 0;
  for (int w0 = 0; w0 < L; w0 += kWindow) window_keys<T>(score, w0, L, lo, hi, keys, &low, &high);
  low = __reduce_min_sync(adt::kFullMask, low);
  high = __reduce_max_sync(adt::kFullMask, high);
  if ((tid & 31) == 0) {
    sc->warp[tid >> 5] = low;
    sc->warp[kWarps + (tid >> 5)] = high;
  }
  __syncthreads();
  if (want == 0) return Cut{kStays - 1u, kStays - 1u, 0};  // (the lowest none of whatever ties)
#pragma unroll
  for (int i = 0; i < kWarps; ++i) {
    low = min(low, sc->warp[i]);
    high = max(high, sc->warp[kWarps + i]);
  }
  uint32_t base = low, span = high - low;  // keys that still compete: base .. base + span
  uint32_t need = want;
  bool whole;
  while (true) {
    const int bits = 32 - __clz(span), shift = bits > kBinBits ? bits - kBinBits : 0;
    if (small) {
#pragma unroll 4
      for (int j = tid; j < L; j += kThreads) {
        const uint32_t k = keys[j] - base;
        if (k <= span) atomicAdd(&sc->hist[k >> shift], 1u);
      }
    } else {
#pragma unroll 4
      for (int j = lo + tid; j < hi; j += kThreads) {
        const uint32_t k = score_key(score[j]) - base;
        if (k <= span) atomicAdd(&sc->hist[k >> shift], 1u);
      }
    }
    __syncthreads();
    // Each thread holds a few bins, the highest first; the one where the count
    // from above reaches `need` is the last that is kept, in whole or in part.
    constexpr int kOwn = kBins / kThreads;
    uint32_t c[kOwn], sum = 0, total;
#pragma unroll
    for (int i = 0; i < kOwn; ++i) sum += c[i] = sc->hist[kBins - 1 - (tid * kOwn + i)];
    uint32_t above = block_scan<T>(sum, sc->warp, &total);
#pragma unroll
    for (int i = 0; i < kOwn; ++i) {
      if (above < need && need <= above + c[i]) {
        sc->bin = kBins - 1 - (tid * kOwn + i);
        sc->need = need - above;
        sc->count = c[i];
      }
      above += c[i];
    }
    __syncthreads();
    need = sc->need;
    base += sc->bin << shift;
    span = min((1u << shift) - 1u, high - base);
    whole = sc->count == need;
    if (shift == 0 || whole) break;
    for (int i = tid; i < kBins; i += kThreads) sc->hist[i] = 0;
    __syncthreads();
  }
  return Cut{base, base + span, whole ? -1 : static_cast<int>(need)};
}

// The threads that move a tensor: all of the CTA, or half of it.
__device__ __forceinline__ void mover_sync(int id, int threads) {
  if (id == 1)
    asm volatile("bar.sync 1, %0;\n" ::"r"(threads) : "memory");
  else
    asm volatile("bar.sync 2, %0;\n" ::"r"(threads) : "memory");
}

// Moves rows first .. rows - 1 of the list: list[r] of src to row r of dst, by
// `threads` threads of which this is number t.  A row is 2^pitch bytes, of which
// 2^shift vectors are moved; slots: this thread's first.  (A window's rows are
// within 8 MB, so that offsets take 32 bits.)
template <int T>
__device__ __forceinline__ void move_rows(uint8_t* slots, const uint8_t* src, uint8_t* dst, const uint16_t* list, int first,
                                          int rows, int shift, int pitch, int t, int threads, int barrier, bool in_place) {
  const int step = threads >> shift;  // rows that one vector of every thread makes
  const int chunks = (rows - first + kVecs * step - 1) / (kVecs * step);
  const int r0 = first + (t >> shift), column = (t & ((1 << shift) - 1)) * 16;
  src += column;
  dst += column + (static_cast<uint32_t>(r0) << pitch);
  list += r0;
  int to_load = rows - r0, to_store = rows - r0;  // rows from this thread's next one on
  const uint32_t smem = sm100::smem_addr(slots), dstep = static_cast<uint32_t>(step) << pitch;
  auto load = [&](int slot) {
#pragma unroll
    for (int v = 0; v < kVecs; ++v)
      if (v * step < to_load)
        sm100::cp_async16(smem + (slot * kVecs + v) * (T * 16), src + (static_cast<uint32_t>(list[v * step]) << pitch), 16);
    list += kVecs * step;
    to_load -= kVecs * step;
    asm volatile("cp.async.commit_group;\n" ::: "memory");
  };
#pragma unroll
  for (int c = 0; c < kAhead; ++c) load(c);
  for (int c = 0; c < chunks; c += kDepth) {
#pragma unroll
    for (int u = 0; u < kDepth; ++u) {
      if (c + u < chunks) {
        load((u + kAhead) % kDepth);
        asm volatile("cp.async.wait_group %0;\n" ::"n"(kAhead) : "memory");
        if (in_place) mover_sync(barrier, threads);
#pragma unroll
        for (int v = 0; v < kVecs; ++v)
          if (v * step < to_store)
            *reinterpret_cast<uint4*>(dst + v * dstep) =
                *reinterpret_cast<const uint4*>(slots + (u * kVecs + v) * (T * 16));
        dst += kVecs * dstep;
        to_store -= kVecs * step;
      }
    }
  }
  asm volatile("cp.async.wait_group 0;\n" ::: "memory");
}

template <int T>
__global__ void __launch_bounds__(T) kv_evict_kernel(const EvictParams p) {
  constexpr int kThreads = T, kWarps = Cta<T>::kWarps, kWindow = Cta<T>::kWindow;
  extern __shared__ __align__(128) uint8_t smem[];  // the movers' slots, then the scratch
  typename Cta<T>::Scratch& sc = *reinterpret_cast<typename Cta<T>::Scratch*>(smem + Cta<T>::kSlotBytes);
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int rank = p.parts == 1 ? 0 : static_cast<int>(blockIdx.x) % p.parts, slice = blockIdx.x / p.parts;
  const int g = slice % p.Hkv, b = slice / p.Hkv % p.B, l = slice / p.Hkv / p.B;
  adt::pdl_wait_then_release();
  const int L = p.kv_len[b];
  const bool ok = L >= 0 && L <= p.max_kv;
  const int n = ok ? min(L, p.budget) : 0;
  if (g == 0 && l == 0 && rank == 0 && tid == 0) {
    if (!ok) adt::raise_error(p.err, ADT_DEVERR_KV_RANGE);
    if (p.kv_len_out) p.kv_len_out[b] = ok ? n : L;
  }
  if (!ok) return;  // (all CTAs of the slice)
  const float* score = p.score + l * p.cls + b * p.csb + g * p.csh;
  float* score_out = p.score_out && rank == 0 ? p.score_out + l * p.ols + b * p.osb + g * p.osh : nullptr;
  int32_t* idx = p.keep_idx && rank == 0 ? p.keep_idx + static_cast<int64_t>(slice) * p.budget : nullptr;
  const int lo = L > n ? p.n_sink : L, hi = L > n ? L - p.n_recent : L;
  uint32_t* keys = reinterpret_cast<uint32_t*>(smem);  // of a window's rows
  const bool small = L <= kWindow;
  Cut cut = find_cut<T>(score, keys, small, L, lo, hi, n - lo - (L - hi), &sc);
  // K by one half of the threads and V by the other, or one of them by all.
  const int movers = p.parts == 1 ? kThreads / 2 : kThreads;
  const int x = p.parts == 1 ? tid / movers : rank & 1;
  const int width = p.parts <= 2 ? p.row_bytes : 2 * p.row_bytes / p.parts, shift = __ffs(width / 16) - 1;
  const int64_t column = p.parts <= 2 ? 0 : (rank >> 1) * width;
  const uint8_t* src = (x ? p.src[1] : p.src[0]) + l * p.sls + b * p.ssb + g * p.ssh + column;
  uint8_t* dst = (x ? p.dst[1] : p.dst[0]) + l * p.dls + b * p.dsb + g * p.dsh + column;
  int done = 0;  // rows moved before this window
  for (int w0 = 0; w0 < L; w0 += kWindow) {
    if (!small) {  // (all movers have left the slots)
      uint32_t low = 0u, high = 0u;
      window_keys<T>(score, w0, L, lo, hi, keys, &low, &high);
      __syncthreads();
    }
    // Bits of the rows that stay and of those that tie, a word a lane: a warp
    // takes `own` words one after the other, so that the threads' words are in
    // the rows' order.
    const int words = (min(L - w0, kWindow) + 31) / 32, own = (words + kWarps - 1) / kWarps, first = warp * own;
    const int here = min(own, words - first);
    const bool by_row = cut.ties >= 0;
    const uint32_t* key = keys + first * 32 + lane;
    uint32_t stay = 0, tie = 0, total;
    if (!by_row) {
#pragma unroll 4
      for (int i = 0; i < here; ++i) {
        const uint32_t s = __ballot_sync(adt::kFullMask, key[i * 32] >= cut.first);
        stay = lane == i ? s : stay;
      }
    } else {
      for (int i = 0; i < here; ++i) {
        const uint32_t k = key[i * 32];
        const uint32_t s = __ballot_sync(adt::kFullMask, k > cut.last);
        const uint32_t t = __ballot_sync(adt::kFullMask, k >= cut.first && k <= cut.last);
        stay = lane == i ? s : stay;
        tie = lane == i ? t : tie;
      }
    }
    if (by_row) {
      const int before = static_cast<int>(block_scan<T>(__popc(tie), sc.warp, &total));
      int most = min(max(cut.ties - before, 0), __popc(tie));  // of this word's ties, the lowest rows
      for (; most > 0; --most) {
        stay |= tie & (0u - tie);
        tie &= tie - 1;
      }
      cut.ties -= min(cut.ties, static_cast<int>(total));
    }
    uint32_t at = block_scan<T>(__popc(stay), sc.warp, &total);
    const int rows = static_cast<int>(total);
    // Rows before the first that goes are in place.
    const uint32_t gone = lane < here && stay != 0xffffffffu ? (first + lane) * 32 + __ffs(~stay) - 1 : kWindow;
    const uint32_t lead_here = __reduce_min_sync(adt::kFullMask, gone);
    if (lane == 0) sc.warp[warp] = lead_here;
#pragma unroll 4
    for (int i = 0; i < here; ++i) {
      const uint32_t bits = __shfl_sync(adt::kFullMask, stay, i), to = __shfl_sync(adt::kFullMask, at, i);
      if (bits >> lane & 1u) sc.list[to + __popc(bits & ((1u << lane) - 1u))] = static_cast<uint16_t>((first + i) * 32 + lane);
    }
    if (p.parts > 1) {
      // Scores may move in place: not before every CTA of the slice has read them.
      sm100::cluster_arrive_release();
      sm100::cluster_wait_acquire();
    }
    __syncthreads();
    int lead = p.in_place && w0 == done ? rows : 0;
#pragma unroll
    for (int i = 0; i < kWarps; ++i) lead = min(lead, static_cast<int>(sc.warp[i]));
    if (idx)
      for (int r = tid; r < rows; r += kThreads) idx[done + r] = w0 + sc.list[r];
    if (score_out) {
      for (int r0 = 0; r0 < rows; r0 += 4 * kThreads) {  // (in place as the rows are, below)
        float v[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int r = r0 + e * kThreads + tid;
          if (r < rows) v[e] = score[w0 + sc.list[r]];
        }
        __syncthreads();
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int r = r0 + e * kThreads + tid;
          if (r < rows) score_out[done + r] = v[e];
        }
      }
    }
    __syncthreads();  // the slots take the place of the keys
    move_rows<T>(smem + tid * 16, src + static_cast<int64_t>(w0) * p.row_bytes, dst + static_cast<int64_t>(done) * p.row_bytes,
              sc.list, lead, rows, shift, __ffs(p.row_bytes) - 1, p.parts == 1 ? tid - x * movers : tid, movers, 1 + x,
              p.in_place != 0);
    __syncthreads();  // the list is read
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

template <int T>
adt_status launch(const EvictParams& p, cudaLaunchConfig_t* cfg, int dev) {
  static unsigned configured[2] = {0u, 0u};  // bit per device (< 64), per instantiation
  const unsigned bit = 1u << (dev & 31);
  unsigned& word = configured[(dev >> 5) & 1];
  if (!(__atomic_load_n(&word, __ATOMIC_ACQUIRE) & bit)) {
    ADT_CUDA_TRY(cudaFuncSetAttribute(kv_evict_kernel<T>, cudaFuncAttributeMaxDynamicSharedMemorySize, Cta<T>::kSmem));
    __atomic_fetch_or(&word, bit, __ATOMIC_ACQ_REL);
  }
  cfg->blockDim = dim3(T, 1, 1);
  cfg->dynamicSmemBytes = Cta<T>::kSmem;
  ADT_CUDA_TRY(cudaLaunchKernelEx(cfg, kv_evict_kernel<T>, p));
  return adt::launch_status();
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
  ADT_REQUIRE(max_kv >= 1 && max_kv < (1 << 30) && budget >= 1 && budget < (1 << 30) && n_sink >= 0 && n_recent >= 0 &&
              static_cast<int64_t>(n_sink) + n_recent <= budget);
  ADT_REQUIRE(!kv_len_out || !caches_overlap(kv_len, B * 4ll, kv_len_out, B * 4ll));
  if (D != 64 && D != 128) return ADT_ERR_UNSUPPORTED;
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
    ADT_REQUIRE(ss[i] <= kMaxStride && ds[i] <= kMaxStride && cs[i] <= kMaxStride && (!score_out || os[i] <= kMaxStride));
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
  // No two slices that are written share memory, none of K's with one of V's
  // either.  (Both may lie in one allocation, slices of both in turn.)
  const int64_t slice = (in_place ? max_kv : keep) * D;
  const int64_t v_off = static_cast<int64_t>(reinterpret_cast<uintptr_t>(v_dst) - reinterpret_cast<uintptr_t>(k_dst)) / 2;
  ADT_REQUIRE(v_off != 0 && !adt::slices_meet(counts, ds, slice, 0) && !adt::slices_meet(counts, ds, slice, v_off));
  if (score_out) {
    const bool scores_in_place = score_out == score && same(cs, os);
    ADT_REQUIRE(scores_in_place || !caches_overlap(score, c_span * 4, score_out, o_span * 4));
    ADT_REQUIRE(!adt::slices_meet(counts, os, scores_in_place ? max_kv : keep, 0));
  }
  const int64_t slices = counts[0] * counts[1] * counts[2];
  if (slices > (1 << 28)) return ADT_ERR_UNSUPPORTED;
  adt::DeviceInfo info;
  adt_status st = adt::device_info(&info);
  if (st != ADT_OK) return st;
  EvictParams p{};
  p.src[0] = reinterpret_cast<const uint8_t*>(k_src);
  p.src[1] = reinterpret_cast<const uint8_t*>(v_src);
  p.dst[0] = reinterpret_cast<uint8_t*>(k_dst);
  p.dst[1] = reinterpret_cast<uint8_t*>(v_dst);
  p.score = score;
  p.score_out = score_out;
  p.kv_len = kv_len;
  p.kv_len_out = kv_len_out;
  p.keep_idx = keep_idx;
  p.B = B;
  p.Hkv = Hkv;
  p.max_kv = max_kv;
  p.budget = budget;
  p.n_sink = n_sink;
  p.n_recent = n_recent;
  p.in_place = in_place;
  p.sls = 2 * ss[0], p.ssb = 2 * ss[1], p.ssh = 2 * ss[2];
  p.dls = 2 * ds[0], p.dsb = 2 * ds[1], p.dsh = 2 * ds[2];
  p.cls = cs[0], p.csb = cs[1], p.csh = cs[2];
  p.ols = os[0], p.osb = os[1], p.osh = os[2];
  p.err = info.error_word;
  p.row_bytes = D * 2;
  // Few slices: K and V, then shares of their columns (32 bytes of a row at
  // least) by CTAs of their own, until every SM has one.  Each selects the rows
  // anew, and rows in pieces cost the memory more, so not beyond.  us with this
  // rule, with one CTA a slice, and with a CTA more an SM: 8 heads, 576 rows of
  // 64 6.0, 7.6, 5.9; 8 heads, 2400 rows of 128 9.4, 19.0, 9.4; 128 slices 33.2,
  // 37.4, 36.5; 256 slices (in graphs) 77.2, 77.2, 87.2.
  p.parts = 1;
  while (p.parts < 8 && slices * p.parts < info.sm_count) p.parts *= 2;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(static_cast<unsigned>(slices * p.parts), 1, 1);
  cfg.stream = adt::as_stream(stream);
  cudaLaunchAttribute attr[2];
  attr[0] = adt::pdl_attribute();
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = static_cast<unsigned>(p.parts);
  attr[1].val.clusterDim.y = 1;
  attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = p.parts > 1 ? 2 : 1;
  // One CTA an SM at most and many rows to search: more threads.  us with 256 and
  // 512 threads, one layer, half the rows kept: 2 heads x 128, 2400 rows 9.0, 9.1,
  // 4800 13.5, 12.2, 16000 45.5, 27.9, 60000 177, 123; 16 heads, 2400 rows 11.1,
  // 12.9, 4800 17.5, 17.9, 8000 29.8, 27.9.
  return slices * p.parts <= info.sm_count && max_kv > 4096 ? launch<512>(p, &cfg, info.device)
                                                            : launch<256>(p, &cfg, info.device);
}

}  // extern "C"
