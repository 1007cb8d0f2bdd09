// adt_kv_score: the attention weight that every cached row got from the tokens
// just committed, added to a running score (what adt_kv_evict goes by).
//
// Row j of the cache gets exp(scale q_i . k_j - lse_i) from path node i and
// head h, where lse is what adt_tree_attn returned for that query: the softmax
// is known to be normalised by it, so one pass over K does, with no running
// maximum and no V.  S^T = K Q^T is made on the tensor cores with the keys as
// the 128 rows of a tile, so that a tensor-memory lane, and with it a thread,
// owns a key: its sum over the queries needs no exchange, a row that holds
// garbage spoils its own sum only, and the order of the sum is fixed.
//
// Persistent CTAs, one an SM, are dealt contiguous shares of all tiles of the
// call (128 keys x up to 128 queries each; tree by tree, within a tree layer by
// layer and kv head by kv head).  Warp roles (384 threads):
//   warps 0-3, 4-7  two groups that take the key tiles of a slice in turn, a
//                   thread a key: exponentials of its row of S^T, their sum;
//   warp 8          TMA loads of K (boxes of 32 keys x 64 columns, no more of
//                   the last tile than holds keys) into a ring of tiles;
//   warp 9          tcgen05.mma, a tile's product into one of four tiles of
//                   tensor memory;
//   warps 10, 11    the next queries (path rows of a kv head's heads) into one
//                   of two buffers.
// Queries past 128 take further passes over the share's keys of that slice,
// whose sums the same thread carries on in score_out.
#include <cuda.h>

#include "adt_common.cuh"
#include "sm100.cuh"

namespace {

constexpr int kKeys = 128;     // keys of a tile
constexpr int kQueries = 128;  // queries of a pass
constexpr int kBoxKeys = 32;
constexpr int kGroupWarps = 4;
constexpr int kKLoadWarp = 8, kMmaWarp = 9, kQLoadWarp = 10;
constexpr int kQThreads = 64;
constexpr int kThreads = 12 * 32;
constexpr uint32_t kTmemCols = 512;  // four tiles of S^T
constexpr uint32_t kWaitLimit = 1u << 20;
constexpr float kLog2e = 1.44269504088896340736f;

template <int D>
struct Cfg {
  static constexpr int kBlocks = D / 64;                 // 128-byte column blocks of a row
  static constexpr int kBlock = kKeys * 128;             // one of them, 128 rows
  static constexpr int kTile = kBlocks * kBlock;         // 128 rows of K or Q
  static constexpr int kStages = D == 128 ? 4 : 8;
  static constexpr int kDynSmem = (2 + kStages) * kTile + 1024;  // + alignment slack
};

struct ScoreParams {
  const __nv_bfloat16* q;
  const float* lse;
  const int32_t* kv_len;
  const int32_t* offs;
  const int32_t* path;
  const int32_t* alen;
  const float* score_in;
  float* score_out;
  int layers, B, H, Hkv, group, max_path, max_kv;
  int64_t qls, lls;            // layer strides of q and lse
  int64_t sls, ssb, ssh;       // score strides
  float scale, decay;
  unsigned* err;
  uint32_t wait_limit;
};

// A tree's part of the work: its slices (layer, kv head) have `tiles` key tiles
// each, every one of which takes `passes` passes of up to 128 queries.
struct Tree {
  int L, rows, tiles, passes;  // rows: queries of a kv head, (a + 1) * group
};

__device__ __forceinline__ Tree tree_of(const ScoreParams& p, int b) {
  const int L = p.kv_len[b], a = p.alen[b];
  Tree t{L, 0, 0, 0};
  if (a < 0 || a >= p.max_path || L < 0 || static_cast<int64_t>(L) + a + 1 > p.max_kv) return t;
  t.rows = (a + 1) * p.group;
  t.tiles = (L + a + kKeys) / kKeys;
  t.passes = (t.rows + kQueries - 1) / kQueries;
  return t;
}

// The part of a CTA's share that lies in one slice: tiles first .. first + count - 1.
struct Segment {
  int b, l, g, first, count;
  Tree t;
};

// Walks a CTA's share slice by slice.  `at` counts tiles of tree b over its
// slices.
struct Walk {
  int b;
  int64_t at, left;  // left: passes over tiles still to do
  Tree t;
  __device__ __forceinline__ bool next(const ScoreParams& p, Segment* s) {
    if (left <= 0) return false;
    const int64_t slices = static_cast<int64_t>(p.layers) * p.Hkv;
    while (t.tiles == 0 || at >= slices * t.tiles) {
      if (++b >= p.B) return false;
      t = tree_of(p, b);
      at = 0;
    }
    const int64_t slice = at / t.tiles;
    s->b = b;
    s->t = t;
    s->l = static_cast<int>(slice / p.Hkv);
    s->g = static_cast<int>(slice % p.Hkv);
    s->first = static_cast<int>(at - slice * t.tiles);
    const int64_t most = (left + t.passes - 1) / t.passes;
    s->count = static_cast<int>(min(static_cast<int64_t>(t.tiles - s->first), most));
    at += s->count;
    left -= static_cast<int64_t>(s->count) * t.passes;
    return true;
  }
};

struct Bars {
  uint64_t k_full[8], k_free[8];
  uint64_t q_full[2], q_free[2];
  uint64_t s_full[4], s_free[4];  // group g's tiles: 2 g, 2 g + 1
  uint64_t drain;
};

// A barrier of the two query warps, at which they leave together: whether any
// of their threads says so.
__device__ __forceinline__ bool q_warps_any(bool x) {
  uint32_t any;
  asm volatile(
      "{\n.reg .pred p, q;\nsetp.ne.u32 p, %1, 0;\nbarrier.cta.red.or.pred q, 1, 64, p;\nselp.u32 %0, 1, 0, q;\n}\n"
      : "=r"(any)
      : "r"(x ? 1u : 0u)
      : "memory");
  return any != 0;
}

template <int D>
__global__ void __launch_bounds__(kThreads, 1)
    kv_score_kernel(const __grid_constant__ CUtensorMap tm_k, const ScoreParams p) {
  using C = Cfg<D>;
  constexpr int NS = C::kStages;
  extern __shared__ __align__(1024) uint8_t smem_raw[];
  uint8_t* smem = smem_raw + ((1024u - (sm100::smem_addr(smem_raw) & 1023u)) & 1023u);
  __shared__ Bars bars;
  __shared__ __align__(16) float s_nlse[2][kQueries];  // -lse of the queries of a buffer
  __shared__ int64_t s_row[kQueries];                  // their rows of q (those being loaded), or -1
  __shared__ Walk s_walk;
  __shared__ uint32_t tmem_slot;
  __shared__ volatile int s_abort;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  uint8_t* sQ = smem;
  uint8_t* sK = smem + 2 * C::kTile;

  // Set-up that touches no memory an earlier kernel writes.
  if (tid == 0) {
    s_abort = 0;
    for (int i = 0; i < NS; ++i) {
      sm100::mbar_init(sm100::smem_addr(&bars.k_full[i]), 1);
      sm100::mbar_init(sm100::smem_addr(&bars.k_free[i]), 1);
    }
    for (int i = 0; i < 2; ++i) {
      sm100::mbar_init(sm100::smem_addr(&bars.q_full[i]), kQThreads / 32);
      sm100::mbar_init(sm100::smem_addr(&bars.q_free[i]), 1 + 2 * kGroupWarps);
    }
    for (int i = 0; i < 4; ++i) {
      sm100::mbar_init(sm100::smem_addr(&bars.s_full[i]), 1);
      sm100::mbar_init(sm100::smem_addr(&bars.s_free[i]), kGroupWarps);
    }
    sm100::mbar_init(sm100::smem_addr(&bars.drain), 1);
    sm100::fence_mbar_init();
  }
  if (warp == kMmaWarp) {
    sm100::tmem_alloc(sm100::smem_addr(&tmem_slot), kTmemCols);
    sm100::tmem_relinquish();
  }
  if (warp == kKLoadWarp && lane == 0) sm100::prefetch_tensormap(&tm_k);
  asm volatile("griddepcontrol.wait;\n" ::: "memory");
  if (warp == 0) {
    // This CTA's share: of all passes over tiles, from x on, in units that
    // neither a tree's number of passes nor its tiles need divide (a tile that
    // straddles two shares belongs to the first).
    const int64_t slices = static_cast<int64_t>(p.layers) * p.Hkv;
    int64_t total = 0, mine = 0;
    for (int b0 = 0; b0 < p.B; b0 += 32) {
      const Tree t = b0 + lane < p.B ? tree_of(p, b0 + lane) : Tree{0, 0, 0, 0};
      if (b0 + lane < p.B && t.tiles == 0 && blockIdx.x == 0) adt::raise_error(p.err, ADT_DEVERR_KV_RANGE);
      mine += slices * t.tiles * t.passes;
    }
    total = adt::warp_sum(mine);
    const int64_t x0 = total / gridDim.x * blockIdx.x + total % gridDim.x * blockIdx.x / gridDim.x;
    const int64_t next = blockIdx.x + 1ll;
    const int64_t x1 = total / gridDim.x * next + total % gridDim.x * next / gridDim.x;
    // The tree that holds x0, and its tile; x1 the same way.
    int64_t before = 0;
    Walk w{0, 0, 0, Tree{0, 0, 0, 0}};
    int64_t skip = 0;  // passes between x0 and the first tile that begins at or after it
    for (int b0 = 0; b0 < p.B; b0 += 32) {
      const Tree t = b0 + lane < p.B ? tree_of(p, b0 + lane) : Tree{0, 0, 0, 0};
      const int64_t cost = slices * t.tiles * t.passes;
      int64_t upto = cost;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const int64_t y = __shfl_up_sync(adt::kFullMask, upto, o);
        if (lane >= o) upto += y;
      }
      const unsigned hit = __ballot_sync(adt::kFullMask, before + upto > x0);
      if (hit) {
        const int src = __ffs(hit) - 1;
        const int64_t off = x0 - (before + __shfl_sync(adt::kFullMask, upto - cost, src));
        w.b = b0 + src;
        w.t.L = __shfl_sync(adt::kFullMask, t.L, src);
        w.t.rows = __shfl_sync(adt::kFullMask, t.rows, src);
        w.t.tiles = __shfl_sync(adt::kFullMask, t.tiles, src);
        w.t.passes = __shfl_sync(adt::kFullMask, t.passes, src);
        w.at = (off + w.t.passes - 1) / w.t.passes;
        skip = w.at * w.t.passes - off;
        break;
      }
      before += __shfl_sync(adt::kFullMask, upto, 31);
    }
    w.left = x1 - x0 - skip;
    if (lane == 0) s_walk = w;
  }
  sm100::tc_fence_before();
  __syncthreads();
  sm100::tc_fence_after();
  const uint32_t tmem = tmem_slot;
  Walk walk = s_walk;
  Segment sg;
  auto wait = [&](uint64_t* bar, uint32_t phase) { return sm100::wait_bar(bar, phase & 1u, &s_abort, p.err, p.wait_limit); };

  if (warp == kKLoadWarp) {
    // ------------------------------------------------------------ K tiles
    if (lane == 0) {
      uint32_t it = 0;
      bool ok = true;
      while (ok && walk.next(p, &sg)) {
        const int keys = sg.t.L + sg.t.rows / p.group;
        for (int pass = 0; ok && pass < sg.t.passes; ++pass) {
          for (int t = 0; t < sg.count; ++t, ++it) {
            const int st = it % NS;
            if (it >= NS && !wait(&bars.k_free[st], it / NS - 1)) {
              ok = false;
              break;
            }
            const int key0 = (sg.first + t) * kKeys;
            const int boxes = (min(keys - key0, kKeys) + kBoxKeys - 1) / kBoxKeys;
            const uint32_t bar = sm100::smem_addr(&bars.k_full[st]);
            sm100::mbar_arrive_expect_tx(bar, boxes * kBoxKeys * D * 2);
            const uint32_t dst = sm100::smem_addr(sK) + st * C::kTile;
            for (int x = 0; x < boxes; ++x)
#pragma unroll
              for (int blk = 0; blk < C::kBlocks; ++blk)
                sm100::tma_load_5d(dst + blk * C::kBlock + x * kBoxKeys * 128, &tm_k, blk * 64, key0 + x * kBoxKeys, sg.g,
                                   sg.b, sg.l, bar);
          }
        }
      }
      asm volatile("griddepcontrol.launch_dependents;\n" ::: "memory");
      // Every copy issued lands before the CTA goes on (also after an abort).
      for (uint32_t j = it > NS ? it - NS : 0; j < it; ++j)
        (void)sm100::mbar_wait_bounded(sm100::smem_addr(&bars.k_full[j % NS]), (j / NS) & 1u, kWaitLimit);
    }
    __syncwarp();
  } else if (warp == kMmaWarp) {
    // ------------------------------------------------------------ S^T = K Q^T
    if (lane == 0) {
      uint32_t it = 0, round = 0, seq[2] = {0, 0};
      bool ok = true;
      while (ok && walk.next(p, &sg)) {
        for (int pass = 0; ok && pass < sg.t.passes; ++pass, ++round) {
          const int cols = min(sg.t.rows - pass * kQueries, kQueries);
          const uint32_t idesc = sm100::idesc_bf16_f32(kKeys, (cols + 15) & ~15, 0, 0);
          const uint32_t q_addr = sm100::smem_addr(sQ) + (round & 1) * C::kTile;
          if (!wait(&bars.q_full[round & 1], round >> 1)) {
            ok = false;
            break;
          }
          for (int t = 0; t < sg.count; ++t, ++it) {
            const int grp = t & 1, st = it % NS;
            const uint32_t n = grp ? seq[1]++ : seq[0]++;
            const int buf = 2 * grp + (n & 1);
            if ((n >= 2 && !wait(&bars.s_free[buf], (n >> 1) - 1)) || !wait(&bars.k_full[st], it / NS)) {
              ok = false;
              break;
            }
            sm100::tc_fence_after();
            const uint32_t k_addr = sm100::smem_addr(sK) + st * C::kTile;
#pragma unroll
            for (int kk = 0; kk < D / 16; ++kk) {
              const uint32_t off = (kk >> 2) * C::kBlock + (kk & 3) * 32;
              sm100::mma_bf16_ss(tmem + buf * kQueries, sm100::smem_desc_sw128(k_addr + off, 16, 1024),
                                 sm100::smem_desc_sw128(q_addr + off, 16, 1024), idesc, kk > 0 ? 1u : 0u);
            }
            sm100::mma_commit(sm100::smem_addr(&bars.s_full[buf]));
            sm100::mma_commit(sm100::smem_addr(&bars.k_free[st]));
          }
          if (ok) sm100::mma_commit(sm100::smem_addr(&bars.q_free[round & 1]));
        }
      }
      sm100::mma_commit(sm100::smem_addr(&bars.drain));
      (void)sm100::mbar_wait_bounded(sm100::smem_addr(&bars.drain), 0, kWaitLimit);
    }
    __syncwarp();
  } else if (warp >= kQLoadWarp) {
    // ------------------------------------------------------------ queries
    const int qt = tid - kQLoadWarp * 32;
    constexpr int kCh = D / 8, kRowsPass = kQThreads / kCh;
    uint32_t round = 0;
    bool ok = true;
    while (ok && walk.next(p, &sg)) {
      const int node0 = p.offs[sg.b], nodes = p.offs[sg.b + 1] - node0;
      for (int pass = 0; pass < sg.t.passes; ++pass, ++round) {
        const int buf = round & 1;
        const bool got = round < 2 || wait(&bars.q_free[buf], (round >> 1) - 1);
        ok = !q_warps_any(!got);
        if (!ok) break;
        const int cols = min(sg.t.rows - pass * kQueries, kQueries);
        for (int c = qt; c < kQueries; c += kQThreads) {
          int64_t row = -1;
          float nl = -INFINITY;
          if (c < cols) {
            const int r = pass * kQueries + c, i = r / p.group, h = sg.g * p.group + (r - i * p.group);
            const int node = p.path[static_cast<int64_t>(sg.b) * p.max_path + i];
            if (node >= 0 && node < nodes) {
              row = static_cast<int64_t>(node0 + node) * p.H + h;
              nl = -p.lse[sg.l * p.lls + row];
              if (nl == INFINITY) nl = -INFINITY;  // a query that saw nothing adds nothing
            } else if (sg.first == 0 && sg.l == 0 && sg.g == 0) {
              adt::raise_error(p.err, ADT_DEVERR_BAD_PATH);
            }
          }
          s_row[c] = row;
          s_nlse[buf][c] = nl;
        }
        asm volatile("bar.sync 1, 64;\n" ::: "memory");
        const int padded = (cols + 15) & ~15, ch = qt % kCh;
        const uint32_t dst = sm100::smem_addr(sQ) + buf * C::kTile;
        const __nv_bfloat16* q = p.q + sg.l * p.qls + ch * 8;
#pragma unroll 4
        for (int c = qt / kCh; c < padded; c += kRowsPass) {
          const int64_t row = s_row[c];
          sm100::cp_async16(dst + sm100::sw128_off(c, ch, kQueries), q + (row < 0 ? 0 : row * D), row < 0 ? 0 : 16);
        }
        asm volatile("cp.async.wait_all;\n" ::: "memory");
        sm100::fence_proxy_async_smem();
        __syncwarp();
        if (lane == 0) sm100::mbar_arrive(sm100::smem_addr(&bars.q_full[buf]));
      }
    }
  } else {
    // ------------------------------------------------------------ exponentials and sums
    const int grp = warp / kGroupWarps, row = tid & (kKeys - 1);
    const uint32_t lane_addr = tmem + (static_cast<uint32_t>((warp & 3) * 32) << 16);
    uint32_t n = 0, round = 0;
    bool ok = true;
    while (ok && walk.next(p, &sg)) {
      const int keys = sg.t.L + sg.t.rows / p.group;
      const int64_t base = sg.l * p.sls + sg.b * p.ssb + sg.g * p.ssh;
      for (int pass = 0; ok && pass < sg.t.passes; ++pass, ++round) {
        const int cols = min(sg.t.rows - pass * kQueries, kQueries);
        const float* nlse = s_nlse[round & 1];
        // (The products of a round follow its queries: s_full orders the reads of s_nlse too, but a group
        // that has no tile in the round waits for them here, before it frees them.)
        if (!__all_sync(adt::kFullMask, wait(&bars.q_full[round & 1], round >> 1))) {
          ok = false;
          break;
        }
        for (int t = grp; t < sg.count; t += 2, ++n) {
          const int j = (sg.first + t) * kKeys + row;
          const int buf = 2 * grp + (n & 1);
          float acc = 0.f, old = 0.f;
          if (pass > 0) {
            if (j < keys) old = p.score_out[base + j];
          } else if (j < sg.t.L && p.decay != 0.f) {
            old = p.decay * p.score_in[base + j];
          }
          if (!__all_sync(adt::kFullMask, wait(&bars.s_full[buf], n >> 1))) {
            ok = false;
            break;
          }
          sm100::tc_fence_after();
          // The first query of this pass that sees row j; only the last rows,
          // the path's own, are not seen by all.
          const int from = j < sg.t.L ? 0 : max(0, (j - sg.t.L) * p.group - pass * kQueries);
          const bool masked = __any_sync(adt::kFullMask, from > 0);
          for (int c0 = 0; c0 < cols; c0 += 32) {
            uint32_t r[32];
            sm100::tmem_ld_32(lane_addr + buf * kQueries + c0, r);
            sm100::tmem_wait_ld_into(r);
            if (masked || c0 + 32 > cols) {
#pragma unroll
              for (int e = 0; e < 32; ++e) {
                const float w = sm100::ex2_approx(fmaf(__uint_as_float(r[e]), p.scale, nlse[c0 + e]) * kLog2e);
                acc += c0 + e >= from && c0 + e < cols ? w : 0.f;
              }
            } else {
#pragma unroll
              for (int e = 0; e < 32; ++e)
                acc += sm100::ex2_approx(fmaf(__uint_as_float(r[e]), p.scale, nlse[c0 + e]) * kLog2e);
            }
          }
          sm100::tc_fence_before();
          __syncwarp();
          if (lane == 0) sm100::mbar_arrive(sm100::smem_addr(&bars.s_free[buf]));
          if (j < keys) p.score_out[base + j] = old + acc;
        }
        __syncwarp();
        if (ok && lane == 0) sm100::mbar_arrive(sm100::smem_addr(&bars.q_free[round & 1]));
      }
    }
  }
  __syncthreads();
  if (warp == kMmaWarp) sm100::tmem_dealloc(tmem, kTmemCols);
}

// 5-D map of a cache (d, row, kv head, tree, layer) with the 128-byte swizzle
// and boxes of 64 columns x 32 rows; rows at or past max_kv read as zero.
adt_status make_map(CUtensorMap* map, const void* base, int D, int max_kv, int Hkv, int B, int layers, int64_t sh,
                    int64_t sb, int64_t sl) {
  const adt::EncodeTiledFn encode = adt::encode_tiled();
  if (!encode) return ADT_ERR_CUDA;
  const int64_t row = static_cast<int64_t>(D) * 2, span = row * max_kv;  // of a dimension of one: any stride
  const cuuint64_t dims[5] = {static_cast<cuuint64_t>(D), static_cast<cuuint64_t>(max_kv), static_cast<cuuint64_t>(Hkv),
                              static_cast<cuuint64_t>(B), static_cast<cuuint64_t>(layers)};
  const cuuint64_t strides[4] = {static_cast<cuuint64_t>(row), static_cast<cuuint64_t>(Hkv > 1 ? sh * 2 : span),
                                 static_cast<cuuint64_t>(B > 1 ? sb * 2 : span),
                                 static_cast<cuuint64_t>(layers > 1 ? sl * 2 : span)};
  const cuuint32_t box[5] = {64, kBoxKeys, 1, 1, 1}, estr[5] = {1, 1, 1, 1, 1};
  const CUresult r = encode(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 5, const_cast<void*>(base), dims, strides, box, estr,
                            CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                            CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
  return r == CUDA_SUCCESS ? ADT_OK : ADT_ERR_INVALID_ARG;
}

template <int D>
adt_status launch(const ScoreParams& p, const CUtensorMap& map, int grid, int dev, cudaStream_t stream) {
  static unsigned configured[2] = {0u, 0u};  // bit per device (< 64), per instantiation
  const unsigned bit = 1u << (dev & 31);
  unsigned& word = configured[(dev >> 5) & 1];
  if (!(__atomic_load_n(&word, __ATOMIC_ACQUIRE) & bit)) {
    ADT_CUDA_TRY(cudaFuncSetAttribute(kv_score_kernel<D>, cudaFuncAttributeMaxDynamicSharedMemorySize, Cfg<D>::kDynSmem));
    __atomic_fetch_or(&word, bit, __ATOMIC_ACQ_REL);
  }
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(static_cast<unsigned>(grid), 1, 1);
  cfg.blockDim = dim3(kThreads, 1, 1);
  cfg.dynamicSmemBytes = Cfg<D>::kDynSmem;
  cfg.stream = stream;
  cudaLaunchAttribute attr[1] = {adt::pdl_attribute()};
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  ADT_CUDA_TRY(cudaLaunchKernelEx(&cfg, kv_score_kernel<D>, map, p));
  return adt::launch_status();
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
  ADT_REQUIRE(static_cast<int64_t>(max_path) * (H / Hkv) < (1 << 30));
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
  p.kv_len = kv_len;
  p.offs = node_offsets;
  p.path = path;
  p.alen = accept_len;
  p.score_in = score_in;
  p.score_out = score_out;
  p.layers = num_layers;
  p.B = B;
  p.H = H;
  p.Hkv = Hkv;
  p.group = H / Hkv;
  p.max_path = max_path;
  p.max_kv = max_kv;
  p.qls = q_layer_stride;
  p.lls = lse_layer_stride;
  p.sls = score_layer_stride;
  p.ssb = score_stride_b;
  p.ssh = score_stride_h;
  p.scale = softmax_scale;
  p.decay = decay;
  p.err = info.error_word;
  p.wait_limit = adt::wait_limit(kWaitLimit);
  CUtensorMap map;
  st = make_map(&map, k_cache, D, max_kv, Hkv, B, num_layers, cache_stride_h, cache_stride_b, cache_layer_stride);
  if (st != ADT_OK) return st;
  const int64_t passes = (static_cast<int64_t>(max_path) * p.group + kQueries - 1) / kQueries;
  const int64_t most = slices * ((max_kv + kKeys - 1) / kKeys) * passes;
  const int grid = static_cast<int>(most < info.sm_count ? most : info.sm_count);
  return D == 128 ? launch<128>(p, map, grid, info.device, adt::as_stream(stream))
                  : launch<64>(p, map, grid, info.device, adt::as_stream(stream));
}

}  // extern "C"
