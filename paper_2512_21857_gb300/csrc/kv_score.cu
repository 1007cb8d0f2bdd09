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
// layer and kv head by kv head).  Warp roles (for few queries, and for many):
//   8 or 16 warps  two or four groups of four that take the key tiles of a slice
//                  in turn, a thread a key: exponentials of its row of S^T,
//                  their sum;
//   1 warp         TMA loads of K (of the last tile no more than boxes of 32
//                  keys that hold some) into a ring of tiles for each of
//   2 or 1 warps   tcgen05.mma, a tile's product into its group's tile of tensor
//                  memory;
//   4 or 2 warps   the next queries (path rows of a kv head's heads) into one of
//                  two buffers.
// Queries past 128 take further passes over the share's keys of that slice,
// whose sums the same thread carries on in score_out.
//
// Bound by HBM with few queries: 32 layers of 32 heads x 128, 2400 rows, a path of
// eight 102 us (96 at the measured copy rate); four trees of 3500 to 6001 rows, 8
// layers, 32 / 8 heads 54.4 us (48.5).  A call's fixed cost is 4 us (the lengths,
// the share, the first tile, the last) and a launch.  With many queries by waits:
// two prompts of 256 tokens, 36 layers, 20 heads x 64, 83 us (33 for the bytes, 30
// for 281 million exponentials at 32 a cycle and SM and 1.95 GHz).  The unit that
// makes those is busy 38 % of the time there, issue slots 55 %, the tensor cores
// 23 %; a warp is stalled longest for loads (tensor memory, the scores so far), of
// which it has one chunk on the way at a time.  What took how much: a score read
// when it was needed 5 us of the second; the product's thread polling one
// barrier after the other (1000 cycles a tile) 3 us of the first, 10 of the
// prompts; divisions in the walk from slice to slice 2 us; queries masked at
// all of a tile instead of where the path ends 20 us of the prompts.  A
// polynomial for a quarter of the exponentials made the prompts slower (104 ->
// 121 us then: it takes issue slots too), as did the next chunk's load ahead.
#include <cuda.h>

#include <utility>

#include "adt_common.cuh"
#include "slices.h"
#include "sm100.cuh"

namespace {

constexpr int kKeys = 128;     // keys of a tile
constexpr int kQueries = 128;  // queries of a pass
constexpr int kBoxKeys = 32;
constexpr int kGroupWarps = 4;
constexpr uint32_t kTmemCols = 512;
constexpr int kTiles = kTmemCols / kQueries;  // of S^T in tensor memory
constexpr uint32_t kWaitLimit = 1u << 24;  // polls: a round of queries can last as long as a CTA's whole share
constexpr int64_t kMaxStride = int64_t{1} << 40;
constexpr int64_t kMaxRows = int64_t{1} << 36;  // of all slices (8 TB of keys): what they cost takes 64 bits
constexpr float kLog2e = 1.44269504088896340736f;

// Warps of the roles.  Few queries a key: the products' and loads' threads are
// what a tile waits for.  Many: the exponentials are, and more groups take
// turns (20 warps leave a thread 96 registers).
template <bool kMany>
struct Roles {
  static constexpr int kGroups = kMany ? 4 : 2;
  static constexpr int kMmaWarps = kMany ? 1 : 2;
  static constexpr int kQWarps = kMany ? 2 : 4;
  static constexpr int kBufs = kTiles / kGroups;  // tiles of S^T of a group
  static constexpr int kKLoadWarp = kGroups * kGroupWarps, kMmaWarp = kKLoadWarp + 1, kQLoadWarp = kMmaWarp + kMmaWarps;
  static constexpr int kThreads = (kQLoadWarp + kQWarps) * 32;
  static_assert(kGroups % kMmaWarps == 0, "a group's tiles are one warp's");
};

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
  int L, keys, rows, tiles, passes;  // keys: with the path's own; rows: queries of a kv head, (a + 1) * group
};

__device__ __forceinline__ Tree tree_of(const ScoreParams& p, int b) {
  const int L = p.kv_len[b], a = p.alen[b];
  Tree t{L, 0, 0, 0, 0};
  if (a < 0 || a >= p.max_path || L < 0 || static_cast<int64_t>(L) + a + 1 > p.max_kv) return t;
  t.keys = L + a + 1;
  t.rows = (a + 1) * p.group;
  t.tiles = (t.keys + kKeys - 1) / kKeys;
  t.passes = (t.rows + kQueries - 1) / kQueries;
  return t;
}

// What a slice costs, in passes over a tile: those of its tiles, and for each
// round of queries kRound more, before its first tile.  (Without them the slices
// of a short tree beside long ones all fall to one CTA: 64 slices of one tile
// beside 448 of 24 to 47 141 us, 100 with.)
constexpr int kRound = 2;

__device__ __forceinline__ int64_t slice_cost(const Tree& t) {
  return t.tiles == 0 ? 0 : static_cast<int64_t>(t.tiles + kRound) * t.passes;
}

// A CTA's share, slice by slice: tiles first .. first + count - 1 of slice (l,
// g) of tree b.  Every role walks it for itself (no divisions on the way: they
// would stall the one thread that loads or multiplies for a tile's time).
struct Walk {
  int b, l, g, first, count;
  int64_t left;  // of the share, from the start of tile `first`
  Tree t;
  // The tiles that start within the share.
  __device__ __forceinline__ bool clip(const ScoreParams& p) {
    if (left <= 0) return false;
    count = t.tiles - first;
    const int before = first == 0 ? kRound : 0;  // rounds' cost between the starts of the first two tiles
    if (static_cast<int64_t>(count + before) * t.passes > left)
      count = max(1, min(count, static_cast<int>((left + t.passes - 1) / t.passes) - before));
    return true;
  }
  // The first segment, from a walk that starts at its first tile (which may be
  // one past the slice's last).
  __device__ __forceinline__ bool start(const ScoreParams& p) {
    if (left <= 0) return false;
    return first < t.tiles ? clip(p) : advance(p);
  }
  __device__ __forceinline__ bool advance(const ScoreParams& p) {
    first = 0;
    if (++g == p.Hkv) {
      g = 0;
      if (++l == p.layers) {
        l = 0;
        do {
          if (++b >= p.B) return false;
          t = tree_of(p, b);
        } while (t.tiles == 0);
      }
    }
    return clip(p);
  }
  __device__ __forceinline__ bool next(const ScoreParams& p) {
    if (first + count < t.tiles) return false;  // (the rest is others')
    left -= static_cast<int64_t>(count + (first == 0 ? kRound : 0)) * t.passes;
    return advance(p);
  }
};

// A wait for a phase of a barrier is only meaningful to a thread that knows the
// phase before complete (parities alternate).  So every K stage belongs to the
// ring of one product warp, every tile of tensor memory to one group and one
// product warp, and each waits for all phases of its own in turn.
constexpr int kMaxStages = 8;

struct Bars {
  uint64_t k_full[kMaxStages], k_free[kMaxStages];
  uint64_t q_full[2], q_free[2];
  uint64_t s_full[kTiles], s_free[kTiles];  // of group g the kBufs from kBufs g on
  uint64_t drain[2];
};

// e^(scale s - lse) of two queries.  (Scaled and shifted before the change of
// base: the difference is what has to be exact.)
__device__ __forceinline__ uint64_t weights(uint32_t s0, uint32_t s1, uint64_t scale2, uint64_t nlse2) {
  const uint64_t t = sm100::fma_f32x2(sm100::pack_u32x2(s0, s1), scale2, nlse2);
  float t0, t1;
  sm100::unpack_f32x2(sm100::fma_f32x2(t, sm100::pack_f32x2(kLog2e, kLog2e), 0ull), t0, t1);
  return sm100::pack_f32x2(sm100::ex2_approx(t0), sm100::ex2_approx(t1));
}

// Eight columns of a lane, there when it returns.
__device__ __forceinline__ void tmem_ld_8(uint32_t taddr, uint32_t (&r)[8]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];\ntcgen05.wait::ld.sync.aligned;\n"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7])
      : "r"(taddr)
      : "memory");
}

// A row's sum over the queries from `from` on, those that add nothing left out
// by name: e^-inf is 0 of a finite product only, and a key that is not finite
// has none, not even with their zeros.  Apart from the loop that makes the sums,
// where a test of every query costs the prompts 2 us (82.6 -> 84.5).
__device__ __noinline__ float masked_sum(uint32_t s_addr, const float* nlse, int from, int cols, float scale) {
  float sum = 0.f;
  for (int c = 0; c < cols; ++c) {
    uint32_t s;
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x1.b32 {%0}, [%1];\ntcgen05.wait::ld.sync.aligned;\n"
                 : "=r"(s)
                 : "r"(s_addr + c)
                 : "memory");
    const float z = nlse[c], w = sm100::ex2_approx(fmaf(__uint_as_float(s), scale, z) * kLog2e);
    if (c >= from && z != -INFINITY) sum += w;
  }
  return sum;
}

// A barrier of the query warps, at which they leave together: whether any of
// their threads says so.
template <int kQWarps>
__device__ __forceinline__ bool q_warps_any(bool x) {
  uint32_t any;
  asm volatile(
      "{\n.reg .pred p, q;\nsetp.ne.u32 p, %1, 0;\nbarrier.cta.red.or.pred q, 1, %2, p;\nselp.u32 %0, 1, 0, q;\n}\n"
      : "=r"(any)
      : "r"(x ? 1u : 0u), "n"(kQWarps * 32)
      : "memory");
  return any != 0;
}

// seq[i], and its increment, without indexed registers.
template <int N>
__device__ __forceinline__ uint32_t next_of(const uint32_t (&seq)[N], int i) {
  uint32_t v = seq[0];
#pragma unroll
  for (int k = 1; k < N; ++k) v = k == i ? seq[k] : v;
  return v;
}
template <int N>
__device__ __forceinline__ void next_done(uint32_t (&seq)[N], int i) {
#pragma unroll
  for (int k = 0; k < N; ++k) seq[k] += k == i ? 1u : 0u;
}

template <int D, bool kMany>
__global__ void __launch_bounds__(Roles<kMany>::kThreads, 1)
    kv_score_kernel(const __grid_constant__ CUtensorMap tm_tile, const __grid_constant__ CUtensorMap tm_rows,
                    const ScoreParams p) {
  using C = Cfg<D>;
  using R = Roles<kMany>;
  constexpr int kGroups = R::kGroups, kMmaWarps = R::kMmaWarps, kQWarps = R::kQWarps, kBufs = R::kBufs;
  constexpr int kKLoadWarp = R::kKLoadWarp, kMmaWarp = R::kMmaWarp, kQLoadWarp = R::kQLoadWarp;
  constexpr int NS = C::kStages, NR = NS / kMmaWarps;  // stages of a ring
  static_assert(NS <= kMaxStages && NS % kMmaWarps == 0, "barriers");
  extern __shared__ __align__(1024) uint8_t smem_raw[];
  uint8_t* smem = smem_raw + ((1024u - (sm100::smem_addr(smem_raw) & 1023u)) & 1023u);
  __shared__ Bars bars;
  __shared__ __align__(16) float s_nlse[2][kQueries];  // -lse of the queries of a buffer; -inf: adds nothing
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
      sm100::mbar_init(sm100::smem_addr(&bars.q_full[i]), kQWarps);
      sm100::mbar_init(sm100::smem_addr(&bars.q_free[i]), kMmaWarps + kGroups * kGroupWarps);
    }
    for (int i = 0; i < kTiles; ++i) {
      sm100::mbar_init(sm100::smem_addr(&bars.s_full[i]), 1);
      sm100::mbar_init(sm100::smem_addr(&bars.s_free[i]), kGroupWarps);
    }
    for (int i = 0; i < kMmaWarps; ++i) sm100::mbar_init(sm100::smem_addr(&bars.drain[i]), 1);
    sm100::fence_mbar_init();
  }
  if (warp == kMmaWarp) {
    sm100::tmem_alloc(sm100::smem_addr(&tmem_slot), kTmemCols);
    sm100::tmem_relinquish();
  }
  if (warp == kKLoadWarp && lane < 2) sm100::prefetch_tensormap(lane ? &tm_rows : &tm_tile);
  asm volatile("griddepcontrol.wait;\n" ::: "memory");
  if (warp == 0) {
    // This CTA's share of all the cost: from x0 to before x1 (a tile belongs to
    // the share that it starts in).
    const int64_t slices = static_cast<int64_t>(p.layers) * p.Hkv;
    int64_t total = 0, mine = 0;
    for (int b0 = 0; b0 < p.B; b0 += 32) {
      const Tree t = b0 + lane < p.B ? tree_of(p, b0 + lane) : Tree{0, 0, 0, 0, 0};
      if (b0 + lane < p.B && t.tiles == 0 && blockIdx.x == 0) adt::raise_error(p.err, ADT_DEVERR_KV_RANGE);
      mine += slices * slice_cost(t);
    }
    total = adt::warp_sum(mine);
    const int64_t x0 = total / gridDim.x * blockIdx.x + total % gridDim.x * blockIdx.x / gridDim.x;
    const int64_t next = blockIdx.x + 1ll;
    const int64_t x1 = total / gridDim.x * next + total % gridDim.x * next / gridDim.x;
    // The tree that holds x0, and the first of its tiles that begins there or later.
    int64_t before = 0;
    Walk w{0, 0, 0, 0, 0, x1 - x0, Tree{0, 0, 0, 0, 0}};
    for (int b0 = 0; b0 < p.B; b0 += 32) {
      const Tree t = b0 + lane < p.B ? tree_of(p, b0 + lane) : Tree{0, 0, 0, 0, 0};
      const int64_t cost = slices * slice_cost(t);
      int64_t upto = cost;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const int64_t y = __shfl_up_sync(adt::kFullMask, upto, o);
        if (lane >= o) upto += y;
      }
      const unsigned hit = __ballot_sync(adt::kFullMask, before + upto > x0);
      if (hit) {
        if (lane == __ffs(hit) - 1) {
          const int64_t off = x0 - (before + upto - cost), slice = off / slice_cost(t);
          const int64_t r = off - slice * slice_cost(t);
          w.b = b0 + lane;
          w.l = static_cast<int>(slice / p.Hkv);
          w.g = static_cast<int>(slice - static_cast<int64_t>(w.l) * p.Hkv);
          // Tile k > 0 starts kRound + k passes into its slice; one past the last is the slice's end.
          if (r > 0) {
            w.first = static_cast<int>(min(max(int64_t{1}, (r + t.passes - 1) / t.passes - kRound), int64_t{t.tiles}));
            w.left -= static_cast<int64_t>(w.first + kRound) * t.passes - r;
          }
          w.t = t;
          s_walk = w;
        }
        break;
      }
      before += __shfl_sync(adt::kFullMask, upto, 31);
      if (b0 + 32 >= p.B && lane == 0) s_walk = w;  // (x0 is the end: nothing to do)
    }
  }
  sm100::tc_fence_before();
  __syncthreads();
  sm100::tc_fence_after();
  const uint32_t tmem = tmem_slot;
  Walk sg = s_walk;
  auto wait = [&](uint64_t* bar, uint32_t phase) { return sm100::wait_bar(bar, phase & 1u, &s_abort, p.err, p.wait_limit); };

  if (warp == kKLoadWarp) {
    // ------------------------------------------------------------ K tiles
    if (lane == 0) {
      uint32_t seq[kMmaWarps] = {};
      bool ok = true;
      for (bool more = sg.start(p); ok && more; more = sg.next(p)) {
        const int keys = sg.t.keys;
        for (int pass = 0; ok && pass < sg.t.passes; ++pass) {
          for (int t = 0; t < sg.count; ++t) {
            const uint32_t n = next_of(seq, t % kMmaWarps);
            const int st = t % kMmaWarps * NR + n % NR;
            if (n >= NR && !wait(&bars.k_free[st], n / NR - 1)) {
              ok = false;
              break;
            }
            next_done(seq, t % kMmaWarps);
            const int key0 = (sg.first + t) * kKeys;
            const int boxes = (min(keys - key0, kKeys) + kBoxKeys - 1) / kBoxKeys;
            const uint32_t bar = sm100::smem_addr(&bars.k_full[st]), dst = sm100::smem_addr(sK) + st * C::kTile;
            sm100::mbar_arrive_expect_tx(bar, boxes * kBoxKeys * D * 2);
#pragma unroll
            for (int blk = 0; blk < C::kBlocks; ++blk) {
              if (boxes * kBoxKeys == kKeys) {
                sm100::tma_load_5d(dst + blk * C::kBlock, &tm_tile, blk * 64, key0, sg.g, sg.b, sg.l, bar);
              } else {
                for (int x = 0; x < boxes; ++x)
                  sm100::tma_load_5d(dst + blk * C::kBlock + x * kBoxKeys * 128, &tm_rows, blk * 64, key0 + x * kBoxKeys,
                                     sg.g, sg.b, sg.l, bar);
              }
            }
          }
        }
      }
      asm volatile("griddepcontrol.launch_dependents;\n" ::: "memory");
      // Every copy issued lands before the CTA goes on (also after an abort).
#pragma unroll
      for (int w = 0; w < kMmaWarps; ++w)
        for (uint32_t n = seq[w] > NR ? seq[w] - NR : 0; n < seq[w]; ++n)
          (void)sm100::mbar_wait_bounded(sm100::smem_addr(&bars.k_full[w * NR + n % NR]), n / NR & 1u, kWaitLimit);
    }
    __syncwarp();
  } else if (warp >= kMmaWarp && warp < kQLoadWarp) {
    // ------------------------------------------------------------ S^T = K Q^T
    if (lane == 0) {
      const int mine = warp - kMmaWarp;  // every kMmaWarps-th tile
      uint32_t round = 0, tiles = 0, seq[kGroups] = {};
      bool ok = true;
      for (bool more = sg.start(p); ok && more; more = sg.next(p)) {
        for (int pass = 0; ok && pass < sg.t.passes; ++pass, ++round) {
          const int cols = min(sg.t.rows - pass * kQueries, kQueries);
          const uint32_t idesc = sm100::idesc_bf16_f32(kKeys, (cols + 15) & ~15, 0, 0);
          const uint64_t q_desc = sm100::smem_desc_sw128(sm100::smem_addr(sQ) + (round & 1) * C::kTile, 16, 1024);
          if (!wait(&bars.q_full[round & 1], round >> 1)) {
            ok = false;
            break;
          }
          for (int t = mine; t < sg.count; t += kMmaWarps, ++tiles) {
            const int grp = t % kGroups, st = mine * NR + tiles % NR;
            const uint32_t n = next_of(seq, grp);
            next_done(seq, grp);
            const int buf = kBufs * grp + n % kBufs;
            // (Both polled before either is waited for: a poll takes 200 cycles.)
            const uint32_t k_full = sm100::smem_addr(&bars.k_full[st]), k_phase = tiles / NR & 1u;
            const uint32_t s_free = sm100::smem_addr(&bars.s_free[buf]), s_phase = (n / kBufs - 1) & 1u;
            const bool k_there = sm100::mbar_try_wait(k_full, k_phase);
            const bool s_there = n < kBufs || sm100::mbar_try_wait(s_free, s_phase);
            if ((!s_there && !wait(&bars.s_free[buf], s_phase)) || (!k_there && !wait(&bars.k_full[st], k_phase))) {
              ok = false;
              break;
            }
            sm100::tc_fence_after();
            const uint64_t k_desc = sm100::smem_desc_sw128(sm100::smem_addr(sK) + st * C::kTile, 16, 1024);
#pragma unroll
            for (int kk = 0; kk < D / 16; ++kk) {
              const uint32_t off = ((kk >> 2) * C::kBlock + (kk & 3) * 32) >> 4;
              sm100::mma_bf16_ss(tmem + buf * kQueries, k_desc + off, q_desc + off, idesc, kk > 0 ? 1u : 0u);
            }
            sm100::mma_commit(sm100::smem_addr(&bars.s_full[buf]));
            sm100::mma_commit(sm100::smem_addr(&bars.k_free[st]));
          }
          if (ok) sm100::mma_commit(sm100::smem_addr(&bars.q_free[round & 1]));
        }
      }
      sm100::mma_commit(sm100::smem_addr(&bars.drain[mine]));
      (void)sm100::mbar_wait_bounded(sm100::smem_addr(&bars.drain[mine]), 0, kWaitLimit);
    }
    __syncwarp();
  } else if (warp >= kQLoadWarp) {
    // ------------------------------------------------------------ queries
    const int qt = tid - kQLoadWarp * 32;
    constexpr int kCh = D / 8, kRowsPass = kQWarps * 32 / kCh;
    uint32_t round = 0;
    bool ok = true;
    for (bool more = sg.start(p); ok && more; more = sg.next(p)) {
      const int node0 = p.offs[sg.b], nodes = p.offs[sg.b + 1] - node0;
      for (int pass = 0; pass < sg.t.passes; ++pass, ++round) {
        const int buf = round & 1;
        const bool got = round < 2 || wait(&bars.q_free[buf], (round >> 1) - 1);
        ok = !q_warps_any<kQWarps>(!got);
        if (!ok) break;
        const int cols = min(sg.t.rows - pass * kQueries, kQueries);
        for (int c = qt; c < kQueries; c += kQWarps * 32) {
          int64_t row = -1;
          float nl = -INFINITY;
          if (c < cols) {
            const int r = pass * kQueries + c, i = r / p.group, h = sg.g * p.group + (r - i * p.group);
            const int node = p.path[static_cast<int64_t>(sg.b) * p.max_path + i];
            if (node >= 0 && node < nodes) {
              row = static_cast<int64_t>(node0 + node) * p.H + h;
              nl = -p.lse[sg.l * p.lls + row];
              if (nl == INFINITY) {  // a query that saw nothing adds nothing, whatever it holds
                nl = -INFINITY;
                row = -1;
              }
            } else if (sg.first == 0 && sg.l == 0 && sg.g == 0) {
              adt::raise_error(p.err, ADT_DEVERR_BAD_PATH);
            }
          }
          s_row[c] = row;
          s_nlse[buf][c] = nl;
        }
        (void)q_warps_any<kQWarps>(false);
        const int padded = (cols + 15) & ~15, ch = qt % kCh;
        const uint32_t dst = sm100::smem_addr(sQ) + buf * C::kTile;
        const __nv_bfloat16* q = p.q + sg.l * p.qls + ch * 8;
#pragma unroll 4
        for (int c = qt / kCh; c < padded; c += kRowsPass) {
          const int64_t row = s_row[c];
          sm100::cp_async16(dst + sm100::sw128_off(c, ch, kKeys), q + (row < 0 ? 0 : row * D), row < 0 ? 0 : 16);
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
    const uint64_t scale2 = sm100::pack_f32x2(p.scale, p.scale);
    uint32_t n = 0, round = 0;
    bool ok = true;
    for (bool more = sg.start(p); ok && more; more = sg.next(p)) {
      const int keys = sg.t.keys;
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
        // The score so far, on its way a tile ahead: its latency is as long as
        // a tile takes.
        auto so_far = [&](int t) {
          const int j = (sg.first + t) * kKeys + row;
          if (t >= sg.count) return 0.f;
          if (pass > 0) return j < keys ? p.score_out[base + j] : 0.f;
          return j < sg.t.L && p.decay != 0.f ? p.score_in[base + j] : 0.f;
        };
        float ahead = so_far(grp);
        for (int t = grp; t < sg.count; t += kGroups, ++n) {
          const int j = (sg.first + t) * kKeys + row;
          const int buf = kBufs * grp + n % kBufs;
          const float old = ahead;
          ahead = so_far(t + kGroups);
          if (!__all_sync(adt::kFullMask, wait(&bars.s_full[buf], n / kBufs))) {
            ok = false;
            break;
          }
          sm100::tc_fence_after();
          // The first query of this pass that sees row j; only the last rows,
          // the path's own, are not seen by all.  Of the warp's rows: queries
          // before some_from are seen by none, those from all_from on by all.
          const int from = j < sg.t.L ? 0 : max(0, (j - sg.t.L) * p.group - pass * kQueries);
          const int some_from = __reduce_min_sync(adt::kFullMask, from), all_from = __reduce_max_sync(adt::kFullMask, from);
          const uint32_t s_addr = lane_addr + buf * kQueries;
          uint64_t acc[2] = {0ull, 0ull};
          // Chunks of 32 queries that all rows see, two fp32 values an
          // instruction but for the exponentials; others by eights, masked.
          // (Both short: unrolled further, with the next chunk's load ahead, a
          // pass takes longer, bound by fetching its code.)
          int c0 = some_from & ~7;
          while (c0 < cols) {
            const ulonglong2* nl = reinterpret_cast<const ulonglong2*>(nlse + c0);
            if (c0 >= all_from && c0 + 32 <= cols) {
              uint32_t r[32];
              sm100::tmem_ld_32(s_addr + c0, r);
              sm100::tmem_wait_ld_into(r);
#pragma unroll
              for (int e = 0; e < 8; ++e) {
                const ulonglong2 z = nl[e];
                acc[0] = sm100::add_f32x2(acc[0], weights(r[4 * e], r[4 * e + 1], scale2, z.x));
                acc[1] = sm100::add_f32x2(acc[1], weights(r[4 * e + 2], r[4 * e + 3], scale2, z.y));
              }
              c0 += 32;
            } else {
              uint32_t r[8];
              tmem_ld_8(s_addr + c0, r);
#pragma unroll
              for (int e = 0; e < 2; ++e) {
                const ulonglong2 z = nl[e];
                float w[4];
                sm100::unpack_f32x2(weights(r[4 * e], r[4 * e + 1], scale2, z.x), w[0], w[1]);
                sm100::unpack_f32x2(weights(r[4 * e + 2], r[4 * e + 3], scale2, z.y), w[2], w[3]);
#pragma unroll
                for (int k = 0; k < 4; ++k) w[k] = c0 + 4 * e + k >= from && c0 + 4 * e + k < cols ? w[k] : 0.f;
                acc[0] = sm100::add_f32x2(acc[0], sm100::pack_f32x2(w[0], w[1]));
                acc[1] = sm100::add_f32x2(acc[1], sm100::pack_f32x2(w[2], w[3]));
              }
              c0 += 8;
            }
          }
          float a0, a1, a2, a3;
          sm100::unpack_f32x2(acc[0], a0, a1);
          sm100::unpack_f32x2(acc[1], a2, a3);
          float sum = (a0 + a1) + (a2 + a3);
          const bool nan = j < keys && sum != sum;
          if (__any_sync(adt::kFullMask, nan)) {
            const float x = masked_sum(s_addr, nlse, from, cols, p.scale);
            sum = nan ? x : sum;
          }
          sm100::tc_fence_before();
          __syncwarp();
          if (lane == 0) sm100::mbar_arrive(sm100::smem_addr(&bars.s_free[buf]));
          if (j < keys) p.score_out[base + j] = (pass > 0 ? old : p.decay * old) + sum;
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
// and boxes of 64 columns x box_rows rows; rows at or past max_kv read as zero.
adt_status make_map(CUtensorMap* map, int box_rows, const void* base, int D, int max_kv, int Hkv, int B, int layers, int64_t sh,
                    int64_t sb, int64_t sl) {
  const adt::EncodeTiledFn encode = adt::encode_tiled();
  if (!encode) return ADT_ERR_CUDA;
  const int64_t row = static_cast<int64_t>(D) * 2, span = row * max_kv;  // of a dimension of one: any stride
  const cuuint64_t dims[5] = {static_cast<cuuint64_t>(D), static_cast<cuuint64_t>(max_kv), static_cast<cuuint64_t>(Hkv),
                              static_cast<cuuint64_t>(B), static_cast<cuuint64_t>(layers)};
  const cuuint64_t strides[4] = {static_cast<cuuint64_t>(row), static_cast<cuuint64_t>(Hkv > 1 ? sh * 2 : span),
                                 static_cast<cuuint64_t>(B > 1 ? sb * 2 : span),
                                 static_cast<cuuint64_t>(layers > 1 ? sl * 2 : span)};
  const cuuint32_t box[5] = {64, static_cast<cuuint32_t>(box_rows), 1, 1, 1}, estr[5] = {1, 1, 1, 1, 1};
  const CUresult r = encode(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 5, const_cast<void*>(base), dims, strides, box, estr,
                            CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                            CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
  return r == CUDA_SUCCESS ? ADT_OK : ADT_ERR_INVALID_ARG;
}

template <int D, bool kMany>
adt_status launch(const ScoreParams& p, const CUtensorMap& tile, const CUtensorMap& rows, int grid, int dev, cudaStream_t stream) {
  static unsigned configured[2] = {0u, 0u};  // bit per device (< 64), per instantiation
  const unsigned bit = 1u << (dev & 31);
  unsigned& word = configured[(dev >> 5) & 1];
  if (!(__atomic_load_n(&word, __ATOMIC_ACQUIRE) & bit)) {
    ADT_CUDA_TRY(cudaFuncSetAttribute(kv_score_kernel<D, kMany>, cudaFuncAttributeMaxDynamicSharedMemorySize, Cfg<D>::kDynSmem));
    __atomic_fetch_or(&word, bit, __ATOMIC_ACQ_REL);
  }
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(static_cast<unsigned>(grid), 1, 1);
  cfg.blockDim = dim3(Roles<kMany>::kThreads, 1, 1);
  cfg.dynamicSmemBytes = Cfg<D>::kDynSmem;
  cfg.stream = stream;
  cudaLaunchAttribute attr[1] = {adt::pdl_attribute()};
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  ADT_CUDA_TRY(cudaLaunchKernelEx(&cfg, kv_score_kernel<D, kMany>, tile, rows, p));
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
  ADT_REQUIRE(score_layer_stride <= kMaxStride && score_stride_b <= kMaxStride && score_stride_h <= kMaxStride &&
              q_layer_stride <= kMaxStride && lse_layer_stride <= kMaxStride);
  ADT_REQUIRE(adt::aligned16(q) && adt::aligned16(k_cache));
  ADT_REQUIRE(static_cast<int64_t>(max_path) * (H / Hkv) < (1 << 30));
  const int64_t slices = static_cast<int64_t>(num_layers) * B * Hkv;
  if (score_in != score_out) {
    const uint64_t span = (static_cast<uint64_t>(num_layers - 1) * score_layer_stride + (B - 1) * score_stride_b +
                           (Hkv - 1) * score_stride_h + max_kv) * sizeof(float);
    const uintptr_t x = reinterpret_cast<uintptr_t>(score_in), y = reinterpret_cast<uintptr_t>(score_out);
    ADT_REQUIRE(x >= y + span || y >= x + span);
  }
  if (slices > (1 << 22) || slices * max_kv > kMaxRows) return ADT_ERR_UNSUPPORTED;
  // No two slices of the scores share memory: CTAs of their own add to them.
  const int64_t counts[3] = {num_layers, B, Hkv}, ss[3] = {score_layer_stride, score_stride_b, score_stride_h};
  ADT_REQUIRE(!adt::slices_meet(counts, ss, max_kv, 0));
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
  CUtensorMap tile, boxes;
  for (auto [map, box] : {std::pair{&tile, kKeys}, std::pair{&boxes, kBoxKeys}}) {
    st = make_map(map, box, k_cache, D, max_kv, Hkv, B, num_layers, cache_stride_h, cache_stride_b, cache_layer_stride);
    if (st != ADT_OK) return st;
  }
  const int64_t passes = (static_cast<int64_t>(max_path) * p.group + kQueries - 1) / kQueries;
  const int64_t most = slices * ((max_kv + kKeys - 1) / kKeys) * passes;
  const int grid = static_cast<int>(most < info.sm_count ? most : info.sm_count);
  // Roles by the most queries a key may meet (the path's length is known on the
  // device only).  us with those for few and for many, 16 layers of 16 heads, 1500
  // rows: D = 64, 32 queries 15.9, 17.0, 64 18.9, 18.6, 128 25.4, 23.1; D = 128, 32
  // queries 22.9, 23.9, 96 25.8, 27.3, 128 28.4, 28.5, 256 46.0, 45.0.
  const cudaStream_t cs = adt::as_stream(stream);
  if (static_cast<int64_t>(max_path) * p.group > D)
    return D == 128 ? launch<128, true>(p, tile, boxes, grid, info.device, cs)
                    : launch<64, true>(p, tile, boxes, grid, info.device, cs);
  return D == 128 ? launch<128, false>(p, tile, boxes, grid, info.device, cs)
                  : launch<64, false>(p, tile, boxes, grid, info.device, cs);
}

}  // extern "C"
