// adt_tree_attn_q8: tree-masked attention, and that of single tokens, whose
// prefix is the 8-bit cache.
//
// The rows of a (tree, kv head) are its nodes' query heads of that group, node
// by node, in blocks of 128 = the tensor core's M.  An item is such a block with
// its keys, in chunks of 128: the prefix, then the tree's own.  The chunks of all
// items, with kItemCost more for each item's start, are dealt to one persistent
// CTA an SM in equal contiguous shares, so ragged batches and few long sequences
// fill the device alike; an item that a share's end cuts is joined from partial
// rows (O, maximum, sum) in the workspace by the CTA that ends its part last.
//
// S = Q K^T is made of e4m3 products, K as it lies in the cache: a query row,
// scaled by a power of two to at most 448, is cut into an e4m3 row and another of
// what that leaves, and both products add up in one accumulator (as many
// instructions as one product of bf16 has).  What the two leave is below 2^-17 of the row's
// largest magnitude.  The tree's own keys are cut the same way (four products).
// The key's scale meets the score in fp32.  A weight takes on its value row's
// scale before it is rounded to bf16, and V is widened to bf16 in shared memory:
// e4m3 weights, even two of them, would lose keys of 2^-18 of the largest one's
// weight, of which a long cache can have enough to matter.
//
// Warp roles (16 warps):
//   0-3, 4-7  two softmax groups that take the chunks in turn, a thread a row;
//             the running maximum passes from group to group through shared
//             memory, P goes to tensor memory;
//   8         K tiles by TMA into a ring, and the scales of both, eight chunks deep;
//   9         V tiles (packed rows: plain bulk copies) into a ring;
//   10        S products;
//   11        PV products;
//   12-15     V from e4m3 to bf16 (the rows past the prefix zeroed), the queries
//             of the next item, a tree's keys, values and ancestor bits.
// Every wait is bounded; a timeout sets ADT_DEVERR_TIMEOUT.
#include <math.h>

#include <cuda.h>

#include "adt_common.cuh"
#include "kv_q8.cuh"
#include "sm100.cuh"

namespace {

using sm100::add_f32x2;
using sm100::ex2_approx;
using sm100::fma_f32x2;
using sm100::mul_f32x2;
using sm100::pack_f32x2;
using sm100::pack_u32x2;
using sm100::sw128_off;
using sm100::tmem_ld_32;
using sm100::tmem_st_16;
using sm100::tmem_st_32;
using sm100::tmem_wait_ld_into;
using sm100::unpack_f32x2;

constexpr int kRows = 128;              // query rows of an item
constexpr int kChunk = 128;             // keys of a chunk
constexpr int kMaxTreeNodes = 256;
constexpr int64_t kMaxRows = 1 << 24;   // query rows of a call
constexpr int kItemCost = 2;            // chunks that an item's start and end take the time of
constexpr int kMinShare = 6;            // coordinates (see Walk) of a CTA's share, where there are few
constexpr int kSoftmaxThreads = 256;
constexpr int kKWarp = 8, kVWarp = 9, kSWarp = 10, kPvWarp = 11, kConvWarp = 12;
constexpr int kConvThreads = 128;
constexpr int kThreads = 512;
constexpr int kMaxScaleSlots = 16;
constexpr int kMaxStages = 6;
constexpr int kMaxGrid = 1024;          // tickets of the workspace
constexpr uint32_t kTmemCols = 512;
constexpr uint32_t kOCol = 256, kPCol = 384;  // after two S tiles of 128 columns; two P tiles of 64
constexpr uint32_t kWaitLimit = 1u << 22;
constexpr uint32_t kDrainLimit = 1u << 20;  // of the waits for what is in flight
constexpr float kLog2e = 1.44269504088896340736f;
constexpr float kLn2 = 0.69314718055994530942f;
constexpr float kRescaleThreshold = 8.0f;  // log2 units

template <int D>
struct Cfg {
  static constexpr int kKStages = D == 128 ? 3 : 6;
  static constexpr int kVStages = D == 128 ? 2 : 4;
  static constexpr int kScaleSlots = D == 128 ? 8 : 16;
  static constexpr int kTile = kChunk * D;                // 128 rows of e4m3
  static constexpr int kBlock = kChunk * 128;             // one 64-column block of 128 rows of bf16
  static constexpr int kWide = D / 64 * kBlock;           // 128 rows of bf16
  static constexpr int kQOff = 0;                         // [2 items][high, low]
  static constexpr int kKOff = kQOff + 4 * kTile;
  static constexpr int kVOff = kKOff + kKStages * kTile;
  static constexpr int kWideOff = kVOff + kVStages * kTile;
  static constexpr int kScaleOff = kWideOff + 2 * kWide;  // [slots][K, V][128] fp32
  static constexpr int kDynSmem = kScaleOff + kScaleSlots * 2 * kChunk * 4 + 1024;  // + alignment slack
  static constexpr uint32_t kIdescS = sm100::idesc_e4m3_f32(kRows, kChunk);
  static constexpr uint32_t kIdescO = sm100::idesc_bf16_f32(kRows, D, 0, 1);
  static_assert(kKStages <= kMaxStages && kVStages <= kMaxStages && kScaleSlots <= kMaxScaleSlots && kOCol + D <= kPCol, "sizes");
};

struct AttnParams {
  const __nv_bfloat16* q;
  const uint8_t* v_cache;
  const uint8_t* scale[2];
  const int32_t* kv_len;
  const __nv_bfloat16* tree[2];
  const int32_t* parents;
  const int32_t* offs;
  int B, H, Hkv, group, max_nodes, max_kv, slot_rows;
  int64_t sb, sh, ssb, ssh;
  float scale_log2;
  __nv_bfloat16* out;
  float* lse;
  unsigned* tickets;   // [grid], of the items that start in a CTA's share and end in another's
  float2* part_ml;     // [2 grid][slot_rows]: of a CTA's first and of its last item
  float* part_o;       // [2 grid][slot_rows][D]
  unsigned* err;
  uint32_t wait_limit;
};

struct Tree {
  int node0, n, L, chunks, prefix, blocks;  // chunks of an item, those of the prefix, row blocks of a kv head
};

// Tree b; one that is malformed or out of range has no items.
__device__ __forceinline__ Tree tree_of(const AttnParams& p, int b, unsigned* bits) {
  Tree t;
  t.node0 = p.offs[b];
  t.n = p.offs[b + 1] - t.node0;
  t.L = p.kv_len[b];
  const bool bad_tree = t.n < 1 || t.n > p.max_nodes || t.node0 < 0, bad_kv = t.L < 0 || t.L > p.max_kv;
  *bits |= bad_tree ? ADT_DEVERR_BAD_TREE : bad_kv ? ADT_DEVERR_KV_RANGE : 0u;
  if (bad_tree || bad_kv) t.n = t.L = 0;
  t.prefix = (t.L + kChunk - 1) / kChunk;
  t.chunks = t.n ? t.prefix + (t.n + kChunk - 1) / kChunk : 0;
  t.blocks = (t.n * p.group + kRows - 1) / kRows;
  return t;
}

// Item by item (tree, kv head, block) a coordinate runs through kItemCost units
// and then a unit a chunk; a share is a range of coordinates and takes the chunks
// that lie in it.  Share c of G of a total of X starts at c X / G, rounded down.
struct Walk {
  int b, g, blk;
  Tree t;
  int64_t start, end;  // the item's first coordinate; the end of the share
  int k0, k1;          // the share's chunks of the item
  bool first;          // of the share's items
  __device__ __forceinline__ void clip(int64_t from) {
    const int64_t base = start + kItemCost;
    k0 = from > base ? static_cast<int>(from - base) : 0;
    k1 = static_cast<int>(min(static_cast<int64_t>(t.chunks), end - base));
  }
  __device__ __forceinline__ bool some() const { return k1 > k0; }
  __device__ __forceinline__ bool next(const AttnParams& p) {
    start += kItemCost + t.chunks;
    first = false;
    if (start + kItemCost >= end) return false;
    if (++blk == t.blocks) {
      blk = 0;
      if (++g == p.Hkv) {
        g = 0;
        unsigned bits = 0u;
        do {
          if (++b >= p.B) return false;
          t = tree_of(p, b, &bits);
        } while (t.chunks == 0);
      }
    }
    clip(start);
    return some();
  }
};

struct Bars {
  uint64_t k_full[kMaxStages], k_free[kMaxStages];
  uint64_t v_full[kMaxStages], v_free[kMaxStages];
  uint64_t scale_full[kMaxScaleSlots];
  uint64_t wide_full[2];     // a V tile in bf16
  uint64_t q_full[2], q_free[2];
  uint64_t s_full[2], s_free[2], p_full[2];
  uint64_t mu[2][4];         // the running maxima after a chunk are in shared memory, per group and warp
  uint64_t done[4];          // the PV product of chunk j is done (barrier j % 4)
  uint64_t o_free;           // an item's O is read
  uint64_t drain[2];
};

__device__ __forceinline__ void conv_sync() { asm volatile("bar.sync 1, 128;\n" ::: "memory"); }
__device__ __forceinline__ void softmax_sync() { asm volatile("bar.sync 2, 256;\n" ::: "memory"); }

// The same barriers (kBar, kCount threads), at which all leave together: whether any of their threads says so.
template <int kBar, int kCount>
__device__ __forceinline__ bool any_of(bool x) {
  uint32_t any;
  asm volatile(
      "{\n.reg .pred p, q;\nsetp.ne.u32 p, %1, 0;\nbarrier.cta.red.or.pred q, %2, %3, p;\nselp.u32 %0, 1, 0, q;\n}\n"
      : "=r"(any)
      : "r"(x ? 1u : 0u), "n"(kBar), "n"(kCount)
      : "memory");
  return any != 0;
}

__device__ __forceinline__ uint32_t pack_bf16x2(float lo, float hi) {
  const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&v);
}

// Offset of the 16 bytes ch of row r of an e4m3 tile as TMA writes it: rows of 128
// bytes with the 128-byte swizzle, rows of 64 with the 64-byte one.
template <int D>
__device__ __forceinline__ uint32_t tile_off(int r, int ch) {
  return D == 128 ? r * 128 + ((ch ^ (r & 7)) << 4) : r * 64 + ((ch ^ ((r >> 1) & 3)) << 4);
}
template <int D>
__device__ __forceinline__ uint64_t tile_desc(uint32_t addr) {
  return D == 128 ? sm100::smem_desc_sw128(addr, 16, 1024) : sm100::smem_desc_sw64(addr);
}

// 16 elements of a bf16 row, D / 16 neighbouring lanes to a row (all lanes of the
// warp take part): cut into two e4m3 rows at `high` and `low`.  Returns the scale, a
// power of two, that their sum goes with.  A row that is not finite becomes NaN.
template <int D>
__device__ __forceinline__ float cut_row(const uint4 (&x)[2], uint8_t* high, uint8_t* low, bool store) {
  const uint32_t w[8] = {x[0].x, x[0].y, x[0].z, x[0].w, x[1].x, x[1].y, x[1].z, x[1].w};
  uint32_t most = 0u;
#pragma unroll
  for (int k = 0; k < 8; ++k) most = max(most, max(w[k] << 16 & 0x7fff0000u, w[k] & 0x7fff0000u));
#pragma unroll
  for (int o = D / 32; o > 0; o >>= 1) most = max(most, __shfl_xor_sync(adt::kFullMask, most, o));
  const bool finite = most < 0x7f800000u;
  const uint32_t s = finite ? adt::q8_row_scale(__uint_as_float(most)) : 127u;
  const float inv = __uint_as_float((254u - s) << 23);
  uint32_t h[4], l[4];
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    h[k] = l[k] = 0u;
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      const uint32_t z = w[2 * k + e];
      const float a = __uint_as_float(z << 16) * inv, b = __uint_as_float(z & 0xffff0000u) * inv;
      const uint32_t two = adt::f32x2_to_e4m3(a, b);
      const float2 back = adt::e4m3x2_to_f32(two);
      h[k] |= two << (16 * e);
      l[k] |= adt::f32x2_to_e4m3(a - back.x, b - back.y) << (16 * e);
    }
    if (!finite) h[k] = l[k] = 0x7f7f7f7fu;
  }
  if (store) {
    *reinterpret_cast<uint4*>(high) = make_uint4(h[0], h[1], h[2], h[3]);
    *reinterpret_cast<uint4*>(low) = make_uint4(l[0], l[1], l[2], l[3]);
  }
  return __uint_as_float(s << 23);
}

template <int D>
__global__ void __launch_bounds__(kThreads, 1)
    tree_attn_q8_kernel(const __grid_constant__ CUtensorMap tm_k, const AttnParams p) {
  using C = Cfg<D>;
  constexpr int KS = C::kKStages, VS = C::kVStages, kScaleSlots = C::kScaleSlots;
  extern __shared__ __align__(1024) uint8_t smem_raw[];
  uint8_t* smem = smem_raw + ((1024u - (sm100::smem_addr(smem_raw) & 1023u)) & 1023u);
  __shared__ Bars bars;
  __shared__ uint4 s_anc[2][kRows];          // the keys of a tree chunk that a row sees
  __shared__ int16_t s_par[kMaxTreeNodes];
  __shared__ float s_mu[kRows], s_l[2][2][kRows], s_qscale[4][kRows];
  __shared__ int s_odd[8];                   // an item's tree has values that are not finite
  __shared__ Walk s_walk;
  __shared__ int64_t s_total;
  __shared__ int s_grid, s_last;
  __shared__ uint32_t tmem_slot;
  __shared__ volatile int s_abort;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  float* s_scale = reinterpret_cast<float*>(smem + C::kScaleOff);

  // Set-up that touches no memory an earlier kernel writes.
  if (tid == 0) {
    s_abort = 0;
    auto init = [](uint64_t* bar, int n, uint32_t count) {
      for (int i = 0; i < n; ++i) sm100::mbar_init(sm100::smem_addr(bar + i), count);
    };
    init(bars.k_full, KS, 1);
    init(bars.k_free, KS, 1);
    init(bars.v_full, VS, 1);
    init(bars.v_free, VS, 1);
    init(bars.scale_full, kScaleSlots, 1);
    init(bars.wide_full, 2, 4);
    init(bars.q_full, 2, 1);
    init(bars.q_free, 2, 1);
    init(bars.s_full, 2, 1);
    init(bars.s_free, 2, 4);
    init(bars.p_full, 2, 4);
    init(bars.mu[0], 8, 1);
    init(bars.done, 4, 1);
    init(&bars.o_free, 1, 8);
    init(bars.drain, 2, 1);
    sm100::fence_mbar_init();
  }
  if (tid < 8) s_odd[tid] = 0;
  if (warp == kPvWarp) {
    sm100::tmem_alloc(sm100::smem_addr(&tmem_slot), kTmemCols);
    sm100::tmem_relinquish();
  }
  if (warp == kKWarp && lane == 0) sm100::prefetch_tensormap(&tm_k);
  asm volatile("griddepcontrol.wait;\n" ::: "memory");
  if (warp == 0) {
    // This CTA's share.
    unsigned bits = 0u;
    auto cost = [&](const Tree& t) -> int64_t {
      return t.chunks ? static_cast<int64_t>(t.chunks + kItemCost) * t.blocks * p.Hkv : 0;
    };
    Tree t{};
    int64_t mine = 0;
    for (int b = lane; b < p.B; b += 32) {
      t = tree_of(p, b, &bits);
      mine += cost(t);
    }
    if (blockIdx.x == 0 && bits) adt::raise_error(p.err, bits);
    const int64_t total = adt::warp_sum(mine);
    int64_t shares = total / kMinShare;
    shares = shares < 1 ? 1 : shares > gridDim.x ? gridDim.x : shares;
    const int64_t c = blockIdx.x;
    const int64_t x0 = c < shares ? c * total / shares : total, x1 = c < shares ? (c + 1) * total / shares : total;
    Walk w{};
    w.first = true;
    int64_t before = 0;
    for (int b0 = 0; x0 < x1 && b0 < p.B; b0 += 32) {
      if (p.B > 32) t = b0 + lane < p.B ? tree_of(p, b0 + lane, &bits) : Tree{};
      const int64_t mine_here = b0 + lane < p.B ? cost(t) : 0;
      int64_t upto = mine_here;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const int64_t y = __shfl_up_sync(adt::kFullMask, upto, o);
        if (lane >= o) upto += y;
      }
      const unsigned hit = __ballot_sync(adt::kFullMask, before + upto > x0);
      if (hit) {
        if (lane == __ffs(hit) - 1) {
          const int64_t off = x0 - (before + upto - mine_here), each = t.chunks + kItemCost, item = off / each;
          w.b = b0 + lane;
          w.g = static_cast<int>(item / t.blocks);
          w.blk = static_cast<int>(item % t.blocks);
          w.t = t;
          w.start = x0 - off + item * each;
          w.end = x1;
          w.clip(x0);
          s_walk = w;
        }
        break;
      }
      before += __shfl_sync(adt::kFullMask, upto, 31);
    }
    if (lane == 0) {
      if (x0 >= x1) s_walk = w;  // (no chunks)
      s_total = total;
      s_grid = static_cast<int>(shares);
    }
  }
  sm100::tc_fence_before();
  __syncthreads();
  sm100::tc_fence_after();
  const uint32_t tmem = tmem_slot;
  Walk w = s_walk;
  if (!w.some()) {  // (all threads alike)
    __syncthreads();
    if (warp == kPvWarp) sm100::tmem_dealloc(tmem, kTmemCols);
    return;
  }
  uint8_t* sQ = smem + C::kQOff;
  uint8_t* sK = smem + C::kKOff;
  uint8_t* sV = smem + C::kVOff;
  uint8_t* sWide = smem + C::kWideOff;
  auto wait = [&](uint64_t* bar, uint32_t phase) { return sm100::wait_bar(bar, phase & 1u, &s_abort, p.err, p.wait_limit); };
  auto all_wait = [&](uint64_t* bar, uint32_t phase) { return __all_sync(adt::kFullMask, wait(bar, phase)); };
  auto arrive = [&](uint64_t* bar) { sm100::mbar_arrive(sm100::smem_addr(bar)); };
  // Chunk j (counted over the whole share) has slot j % stages of a ring, its
  // phase there j / stages.  A wait on a parity is only meaningful to a thread
  // that knows the phase before complete; each comment below says how.
  uint32_t j = 0;

  if (warp == kKWarp) {
    // ------------------------------------------------------------ K tiles, scales
    uint32_t issued = 0;  // one past the last tile requested
    bool ok = true;
    float pend[8] = {};
    int pend_slot = -1;
    auto flush = [&]() {
      if (pend_slot < 0) return;
      float4* dst = reinterpret_cast<float4*>(s_scale + pend_slot * 2 * kChunk);
      dst[lane] = make_float4(pend[0], pend[1], pend[2], pend[3]);
      dst[32 + lane] = make_float4(pend[4], pend[5], pend[6], pend[7]);
      __syncwarp();
      if (lane == 0) arrive(&bars.scale_full[pend_slot]);
      pend_slot = -1;
    };
    for (bool more = true; ok && more; more = w.next(p)) {
      const int64_t s0 = w.b * p.ssb + w.g * p.ssh;
      for (int k = w.k0; k < w.k1; ++k, ++j) {
        if (k >= w.t.prefix) {  // (the tree's: warps 12-15)
          flush();
          continue;
        }
        const int st = j % KS;
        // (S products end in order: where tree chunks are left out, a later wait
        // of this warp covers theirs.)
        if (lane == 0) ok = j < KS || wait(&bars.k_free[st], j / KS - 1);
        ok = __shfl_sync(adt::kFullMask, ok ? 1 : 0, 0) != 0;
        if (!ok) break;
        if (lane == 0) {
          const uint32_t bar = sm100::smem_addr(&bars.k_full[st]);
          sm100::mbar_arrive_expect_tx(bar, C::kTile);
          sm100::tma_load_4d(sm100::smem_addr(sK + st * C::kTile), &tm_k, 0, k * kChunk, w.g, w.b, bar);
        }
        issued = j + 1;
        // The scales, written when the next chunk's are asked for.  Their slot was
        // read last for a chunk kScaleSlots before, which was done with before S of
        // four chunks on could start, and S(j - KS) is done.
        static_assert(kScaleSlots >= KS + 4, "a slot that is read");
        flush();
        float now[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const int key = k * kChunk + lane * 4 + (i & 3);
          // (Rows past the prefix: a score times 1 is masked, a weight of 0 stays 0.)
          now[i] = key < w.t.L ? adt::q8_scale(p.scale[i >> 2][s0 + key]) : 1.f;
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) pend[i] = now[i];
        pend_slot = static_cast<int>(j % kScaleSlots);
      }
    }
    flush();
    asm volatile("griddepcontrol.launch_dependents;\n" ::: "memory");
    // Every copy issued lands before the CTA goes on (also after an abort).
    if (lane == 0)
      for (int st = 0; st < KS; ++st) {
        // the last use of the slot before `issued` (tree chunks among them, which have no copy)
        if (issued <= static_cast<uint32_t>(st)) continue;
        const uint32_t use = (issued - 1 - st) / KS;
        (void)sm100::mbar_wait_bounded(sm100::smem_addr(&bars.k_full[st]), use & 1u, kDrainLimit);
      }
    __syncwarp();
  } else if (warp == kVWarp) {
    // ------------------------------------------------------------ V tiles
    if (lane == 0) {
      uint32_t issued = 0;
      bool ok = true;
      for (bool more = true; ok && more; more = w.next(p)) {
        const uint8_t* v = p.v_cache + w.b * p.sb + w.g * p.sh;
        for (int k = w.k0; k < w.k1; ++k, ++j) {
          const int st = j % VS;
          const uint32_t bar = sm100::smem_addr(&bars.v_full[st]);
          if (j >= VS && !wait(&bars.v_free[st], j / VS - 1)) {
            ok = false;
            break;
          }
          if (k >= w.t.prefix) {
            // Warps 12-15 write the tree's keys to this chunk's slots of both rings.
            // (S(j - 2 KS) is done: V(j - VS) was widened after PV(j - VS - 2).)
            static_assert(VS + 2 <= 2 * KS, "a phase of k_free that is known complete");
            if (j >= KS && !wait(&bars.k_free[j % KS], j / KS - 1)) {
              ok = false;
              break;
            }
            sm100::mbar_arrive(bar);
          } else {
            const int rows = min(w.t.L - k * kChunk, kChunk);
            sm100::mbar_arrive_expect_tx(bar, rows * D);
            sm100::bulk_load(sm100::smem_addr(sV + st * C::kTile), v + static_cast<int64_t>(k) * kChunk * D, rows * D, bar);
          }
          issued = j + 1;
        }
      }
      for (int st = 0; st < VS; ++st) {
        if (issued <= static_cast<uint32_t>(st)) continue;
        const uint32_t use = (issued - 1 - st) / VS;
        (void)sm100::mbar_wait_bounded(sm100::smem_addr(&bars.v_full[st]), use & 1u, kDrainLimit);
      }
    }
    __syncwarp();
  } else if (warp == kSWarp) {
    // ------------------------------------------------------------ S = Q K^T
    if (lane == 0) {
      bool ok = true;
      uint32_t item = 0;
      for (bool more = true; ok && more; more = w.next(p), ++item) {
        const uint32_t q = sm100::smem_addr(sQ + (item & 1) * 2 * C::kTile);
        ok = wait(&bars.q_full[item & 1], item >> 1);
        for (int k = w.k0; ok && k < w.k1; ++k, ++j) {
          const int grp = j & 1;
          ok = wait(&bars.k_full[j % KS], j / KS) && (j < 2 || wait(&bars.s_free[grp], (j >> 1) - 1));
          if (!ok) break;
          sm100::tc_fence_after();
          const uint32_t kt = sm100::smem_addr(sK + (j % KS) * C::kTile);
          const uint32_t d = tmem + grp * kChunk;
#pragma unroll
          for (int part = 0; part < 2; ++part) {
#pragma unroll
            for (int kk = 0; kk < D / 32; ++kk)
              sm100::mma_f8_ss(d, tile_desc<D>(q + part * C::kTile + kk * 32), tile_desc<D>(kt + kk * 32), C::kIdescS,
                               part > 0 || kk > 0 ? 1u : 0u);
          }
          if (k >= w.t.prefix) {  // the low part of the tree's keys
            const uint32_t lt = sm100::smem_addr(sV + (j % VS) * C::kTile);
#pragma unroll
            for (int part = 0; part < 2; ++part) {
#pragma unroll
              for (int kk = 0; kk < D / 32; ++kk)
                sm100::mma_f8_ss(d, tile_desc<D>(q + part * C::kTile + kk * 32), tile_desc<D>(lt + kk * 32), C::kIdescS, 1u);
            }
            sm100::mma_commit(sm100::smem_addr(&bars.v_free[j % VS]));
          }
          sm100::mma_commit(sm100::smem_addr(&bars.s_full[grp]));
          sm100::mma_commit(sm100::smem_addr(&bars.k_free[j % KS]));
        }
        if (ok) sm100::mma_commit(sm100::smem_addr(&bars.q_free[item & 1]));
      }
      sm100::mma_commit(sm100::smem_addr(&bars.drain[0]));
      (void)sm100::mbar_wait_bounded(sm100::smem_addr(&bars.drain[0]), 0, kDrainLimit);
    }
    __syncwarp();
  } else if (warp == kPvWarp) {
    // ------------------------------------------------------------ O += P V
    if (lane == 0) {
      bool ok = true;
      uint32_t item = 0;
      for (bool more = true; ok && more; more = w.next(p), ++item) {
        for (int k = w.k0; ok && k < w.k1; ++k, ++j) {
          ok = wait(&bars.p_full[j & 1], j >> 1) && wait(&bars.wide_full[j & 1], j >> 1) &&
               (k > w.k0 || item == 0 || wait(&bars.o_free, item - 1));
          if (!ok) break;
          sm100::tc_fence_after();
          const uint32_t a = tmem + kPCol + (j & 1) * 64;
          const uint64_t vd = sm100::smem_desc_sw128(sm100::smem_addr(sWide + (j & 1) * C::kWide), C::kBlock, 1024);
          const int keys = k < w.t.prefix ? w.t.L - k * kChunk : w.t.n - (k - w.t.prefix) * kChunk;
          const int steps = min(kChunk / 16, (keys + 15) / 16);
          sm100::mma_bf16_ts(tmem + kOCol, a, vd, C::kIdescO, k > w.k0 ? 1u : 0u);
          if (steps == kChunk / 16) {
#pragma unroll
            for (int kk = 1; kk < kChunk / 16; ++kk)
              sm100::mma_bf16_ts(tmem + kOCol, a + kk * 8, vd + kk * 128, C::kIdescO, 1u);
          } else {
            for (int kk = 1; kk < steps; ++kk)
              sm100::mma_bf16_ts(tmem + kOCol, a + kk * 8, vd + kk * 128, C::kIdescO, 1u);
          }
          sm100::mma_commit(sm100::smem_addr(&bars.done[j & 3]));
        }
      }
      sm100::mma_commit(sm100::smem_addr(&bars.drain[1]));
      (void)sm100::mbar_wait_bounded(sm100::smem_addr(&bars.drain[1]), 0, kDrainLimit);
    }
    __syncwarp();
  } else if (warp >= kConvWarp) {
    // ------------------------------------------------------------ operands
    constexpr int kLanes = D / 16, kPass = kConvThreads / kLanes;  // lanes of a row, rows of a pass
    const int ct = tid - kConvWarp * 32, cl = ct % kLanes, cr = ct / kLanes;
    uint32_t item = 0;
    // Item `it`'s queries, rows without a node left out.
    auto queries = [&](const Walk& v, uint32_t it) -> bool {
      if (it >= 2 && any_of<1, kConvThreads>(!wait(&bars.q_free[it & 1], (it >> 1) - 1))) return false;
      const int rows = min(v.t.n * p.group - v.blk * kRows, kRows);
      uint8_t* high = sQ + (it & 1) * 2 * C::kTile;
#pragma unroll 2
      for (int r0 = 0; r0 < rows; r0 += kPass) {
        const int r = r0 + cr, row = v.blk * kRows + r;
        uint4 x[2] = {};
        if (r < rows) {
          const int t = row / p.group, hh = row - t * p.group;
          const uint4* src = reinterpret_cast<const uint4*>(
              p.q + (static_cast<int64_t>(v.t.node0 + t) * p.H + v.g * p.group + hh) * D) + cl * 2;
          x[0] = src[0];
          x[1] = src[1];
        }
        const uint32_t off = tile_off<D>(r, cl);
        const float s = cut_row<D>(x, high + off, high + C::kTile + off, r < rows);
        if (r < rows && cl == 0) s_qscale[it & 3][r] = s * p.scale_log2;
      }
      sm100::fence_proxy_async_smem();
      conv_sync();
      if (ct == 0) arrive(&bars.q_full[it & 1]);
      return true;
    };
    bool ok = queries(w, 0), more = true;
    while (ok && more) {
      Walk nw = w;
      bool has_next = false;
      for (int k = w.k0; k < w.k1; ++k, ++j) {
        const int st = j % VS;
        uint8_t* wide = sWide + (j & 1) * C::kWide;
        // PV(j - 2) read this tile.  (Known complete before: PV(j - 3), and so PV(j - 6).)
        if (any_of<1, kConvThreads>((j >= 2 && !wait(&bars.done[(j - 2) & 3], (j - 2) >> 2)) ||
                                    !wait(&bars.v_full[st], j / VS))) {
          ok = false;
          break;
        }
        if (k < w.t.prefix) {
          const int rows = w.t.L - k * kChunk;
          const uint8_t* src = sV + st * C::kTile;
#pragma unroll 4
          for (int i = 0; i < kChunk / kPass; ++i) {
            const int r = i * kPass + cr;
            uint4 v = make_uint4(0u, 0u, 0u, 0u);
            if (r < rows) v = *reinterpret_cast<const uint4*>(src + r * D + cl * 16);
            const uint32_t x[4] = {v.x, v.y, v.z, v.w};
            uint32_t y[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) {
              const float2 f = adt::e4m3x2_to_f32(x[e >> 1] >> (16 * (e & 1)) & 0xffffu);
              y[e] = pack_bf16x2(f.x, f.y);
            }
            // (The order of the two halves: eight lanes' stores fall on all banks.)
            const int swap = cl >> 2 & 1;
            const uint4 lo = make_uint4(y[0], y[1], y[2], y[3]), hi = make_uint4(y[4], y[5], y[6], y[7]);
            *reinterpret_cast<uint4*>(wide + sw128_off(r, 2 * cl + swap, kChunk)) = swap ? hi : lo;
            *reinterpret_cast<uint4*>(wide + sw128_off(r, 2 * cl + 1 - swap, kChunk)) = swap ? lo : hi;
          }
          sm100::fence_proxy_async_smem();
          __syncwarp();
          if (lane == 0) arrive(&bars.wide_full[j & 1]);
          conv_sync();  // all have read the e4m3 tile
          if (ct == 0) arrive(&bars.v_free[st]);
        } else {
          // The tree's chunk: its parents and ancestor bits; its keys, cut in two,
          // and their scales; its values, those that are not finite as zeros
          // (a weight of 0 times them would reach rows that do not see them).
          const int t0 = (k - w.t.prefix) * kChunk, n = w.t.n, node0 = w.t.node0;
          float* ks = s_scale + (j % kScaleSlots) * 2 * kChunk;
          for (int t = ct; t < n; t += kConvThreads) s_par[t] = static_cast<int16_t>(min(max(p.parents[node0 + t], -1), kMaxTreeNodes));
          int odd = 0;
#pragma unroll 2
          for (int i = 0; i < kChunk / kPass; ++i) {
            const int r = i * kPass + cr, t = t0 + r;
            uint4 x[2] = {}, v[2] = {};
            if (t < n) {
              const int64_t at = (static_cast<int64_t>(node0 + t) * p.Hkv + w.g) * D;
              const uint4* src = reinterpret_cast<const uint4*>(p.tree[0] + at) + cl * 2;
              x[0] = src[0];
              x[1] = src[1];
              src = reinterpret_cast<const uint4*>(p.tree[1] + at) + cl * 2;
              v[0] = src[0];
              v[1] = src[1];
            }
            const uint32_t off = tile_off<D>(r, cl);
            const float s = cut_row<D>(x, sK + (j % KS) * C::kTile + off, sV + st * C::kTile + off, true);
            if (cl == 0) {
              ks[r] = t < n ? s : 1.f;
              ks[kChunk + r] = 1.f;
            }
#pragma unroll
            for (int half = 0; half < 2; ++half) {
              uint32_t y[4] = {v[half].x, v[half].y, v[half].z, v[half].w};
#pragma unroll
              for (int e = 0; e < 4; ++e) {
                const bool a = (y[e] & 0x7f80u) == 0x7f80u, b = (y[e] & 0x7f800000u) == 0x7f800000u;
                odd |= a || b;
                if (a) y[e] &= 0xffff0000u;
                if (b) y[e] &= 0xffffu;
              }
              *reinterpret_cast<uint4*>(wide + sw128_off(r, 2 * cl + half, kChunk)) = make_uint4(y[0], y[1], y[2], y[3]);
            }
          }
          if (odd) s_odd[item & 7] = 1;
          conv_sync();
          for (int t = ct; t < n; t += kConvThreads) {
            const int up = s_par[t];
            if ((t == 0) != (up < 0) || up >= t) adt::raise_error(p.err, ADT_DEVERR_BAD_TREE);
          }
          {
            uint32_t m[4] = {0u, 0u, 0u, 0u};
            const int row = w.blk * kRows + ct;
            int t = row / p.group;
            if (t < n) {
              for (;;) {
                const int at = t - t0;
#pragma unroll
                for (int e = 0; e < 4; ++e) m[e] |= at >> 5 == e ? 1u << (at & 31) : 0u;
                const int up = s_par[t];
                if (up < 0 || up >= t) break;
                t = up;
              }
            }
            s_anc[j & 1][ct] = make_uint4(m[0], m[1], m[2], m[3]);
          }
          sm100::fence_proxy_async_smem();
          conv_sync();
          if (lane == 0) arrive(&bars.wide_full[j & 1]);
          if (ct == 0) {
            arrive(&bars.k_full[j % KS]);
            arrive(&bars.scale_full[j % kScaleSlots]);
          }
        }
        if (k == w.k0) {
          has_next = nw.next(p);
          if (has_next && !queries(nw, item + 1)) {
            ok = false;
            break;
          }
        }
      }
      w = nw;
      more = has_next;
      ++item;
      // (Read last seven items back; of the one four back O is read at least.)
      if (ct == 0) s_odd[(item + 1) & 7] = 0;
    }
  } else {
    // ------------------------------------------------------------ softmax
    const int grp = warp >> 2, w4 = warp & 3, row = w4 * 32 + lane;
    const uint32_t lanes = static_cast<uint32_t>(w4 * 32) << 16;
    const uint32_t s_col = tmem + lanes + grp * kChunk, o_col = tmem + lanes + kOCol, p_col = tmem + lanes + kPCol + grp * 64;
    uint32_t item = 0;
    bool ok = true;
    for (bool more = true; ok && more; more = w.next(p), ++item) {
      const int index = w.blk * kRows + row, node = index / p.group, hh = index - node * p.group;
      const bool valid = node < w.t.n, active = __any_sync(adt::kFullMask, valid);
      const uint32_t j0 = j, j1 = j + static_cast<uint32_t>(w.k1 - w.k0);
      float mu = -INFINITY, l = 0.f, scale = 0.f;
      if ((j0 & 1) != static_cast<uint32_t>(grp)) ++j;
      for (; j < j1; j += 2) {
        const int k = w.k0 + static_cast<int>(j - j0);
        if (!all_wait(&bars.s_full[grp], j >> 1) || !all_wait(&bars.scale_full[j % kScaleSlots], j / kScaleSlots)) {
          ok = false;
          break;
        }
        sm100::tc_fence_after();
        if (j <= j0 + 1) scale = s_qscale[item & 3][row];  // (S came of these queries)
        const bool tree_j = k >= w.t.prefix;
        const int kl = tree_j ? w.t.n - (k - w.t.prefix) * kChunk : w.t.L - k * kChunk;
        const int quarters = min(4, (kl + 31) / 32);
        if (active) {
          if (tree_j || kl < kChunk) {
            // -inf where the row does not see the key, in place.
            const uint32_t* bits = reinterpret_cast<const uint32_t*>(&s_anc[j & 1][row]);
#pragma unroll 1
            for (int s = 0; s < quarters; ++s) {
              const int left = kl - 32 * s;
              const uint32_t keep = tree_j ? bits[s] : left >= 32 ? ~0u : (1u << left) - 1u;
              uint32_t r[32];
              tmem_ld_32(s_col + 32 * s, r);
              tmem_wait_ld_into(r);
#pragma unroll
              for (int e = 0; e < 32; ++e) r[e] = (keep >> e) & 1u ? r[e] : 0xFF800000u;
              tmem_st_32(s_col + 32 * s, r);
            }
            sm100::tmem_wait_st();
          }
          const ulonglong2* ks = reinterpret_cast<const ulonglong2*>(s_scale + (j % kScaleSlots) * 2 * kChunk);
          const ulonglong2* vf = ks + kChunk / 4;
          uint32_t x[32], y[32];
          float mq[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
          auto largest = [&](const uint32_t (&r)[32], int s) {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
              const ulonglong2 f = ks[8 * s + e];
              float a, b;
              unpack_f32x2(mul_f32x2(pack_u32x2(r[4 * e], r[4 * e + 1]), f.x), a, b);
              mq[e & 1] = fmaxf(fmaxf(mq[e & 1], a), b);
              unpack_f32x2(mul_f32x2(pack_u32x2(r[4 * e + 2], r[4 * e + 3]), f.y), a, b);
              mq[2 + (e & 1)] = fmaxf(fmaxf(mq[2 + (e & 1)], a), b);
            }
          };
          // The quarters in turn, each loaded while the one before is used; at
          // the end the first one again, for the exponentials.
          tmem_ld_32(s_col, x);
          tmem_wait_ld_into(x);
          if (quarters == 4) {
#pragma unroll
            for (int s = 0; s < 4; s += 2) {
              tmem_ld_32(s_col + 32 * s + 32, y);
              largest(x, s);
              tmem_wait_ld_into(y);
              tmem_ld_32(s_col + (s == 0 ? 64 : 0), x);
              largest(y, s + 1);
              tmem_wait_ld_into(x);
            }
          } else {
            largest(x, 0);
#pragma unroll 1
            for (int s = 1; s < quarters; ++s) {
              tmem_ld_32(s_col + 32 * s, y);
              tmem_wait_ld_into(y);
              largest(y, s);
            }
          }
          const float mx = valid ? fmaxf(fmaxf(mq[0], mq[1]), fmaxf(mq[2], mq[3])) * scale : -INFINITY;  // scale > 0
          // The running maximum after the chunk before (the other group's).  (An
          // item's last chunk is done before the next one's: so are its maxima.)
          float prev = -INFINITY;
          if (j > j0) {
            if (!all_wait(&bars.mu[grp ^ 1][w4], (j - 1) >> 1)) {
              ok = false;
              break;
            }
            prev = s_mu[row];
          }
          // Raised only when a row grows by more than 2^8; then O (once the chunks
          // before are in it) is scaled.
          const float nm = mx > prev + kRescaleThreshold ? mx : prev;
          s_mu[row] = nm;
          __syncwarp();
          if (lane == 0) arrive(&bars.mu[grp][w4]);
          if (nm != mu) l *= ex2_approx(mu - nm);
          // P's tile was last read by PV(j - 2).
          if (j >= 2 && !all_wait(&bars.done[(j - 2) & 3], (j - 2) >> 2)) {
            ok = false;
            break;
          }
          if (j > j0 && __any_sync(adt::kFullMask, nm != prev)) {
            if (!all_wait(&bars.done[(j - 1) & 3], (j - 1) >> 2)) {
              ok = false;
              break;
            }
            sm100::tc_fence_after();
            const float alpha = nm == prev ? 1.f : ex2_approx(prev - nm);
#pragma unroll 1
            for (int c = 0; c < D; c += 32) {
              uint32_t r[32];
              tmem_ld_32(o_col + c, r);
              tmem_wait_ld_into(r);
#pragma unroll
              for (int e = 0; e < 32; ++e) r[e] = __float_as_uint(__uint_as_float(r[e]) * alpha);
              tmem_st_32(o_col + c, r);
            }
          }
          mu = nm;
          sm100::tc_fence_after();
          const float base = mu == -INFINITY ? 0.f : mu;
          const uint64_t scale2 = pack_f32x2(scale, scale), base2 = pack_f32x2(-base, -base);
          uint64_t l2[2] = {0ull, 0ull};
          // 32 scores -> 16 pairs of weights, in bf16 with their values' scales.
          auto quarter = [&](const uint32_t (&r)[32], int s) {
            uint32_t pk[16];
#pragma unroll
            for (int e = 0; e < 8; ++e) {
              const ulonglong2 f = ks[8 * s + e], g = vf[8 * s + e];
#pragma unroll
              for (int h = 0; h < 2; ++h) {
                const uint64_t z = mul_f32x2(pack_u32x2(r[4 * e + 2 * h], r[4 * e + 2 * h + 1]), h ? f.y : f.x);
                float a, b;
                unpack_f32x2(fma_f32x2(z, scale2, base2), a, b);
                const uint64_t wt = pack_f32x2(ex2_approx(a), ex2_approx(b));
                l2[h] = add_f32x2(l2[h], wt);
                unpack_f32x2(mul_f32x2(wt, h ? g.y : g.x), a, b);
                pk[2 * e + h] = pack_bf16x2(a, b);
              }
            }
            tmem_st_16(p_col + 16 * s, pk);
          };
          auto release_s = [&]() {  // S is in registers: its tile may be written again
            sm100::tc_fence_before();
            __syncwarp();
            if (lane == 0) arrive(&bars.s_free[grp]);
          };
          if (quarters == 4) {
#pragma unroll 1
            for (int s = 0; s < 4; s += 2) {
              tmem_ld_32(s_col + 32 * s + 32, y);
              quarter(x, s);
              tmem_wait_ld_into(y);
              if (s == 0)
                tmem_ld_32(s_col + 64, x);
              else
                release_s();
              quarter(y, s + 1);
              tmem_wait_ld_into(x);
            }
          } else {
#pragma unroll 1
            for (int s = 0; s < quarters; ++s) {
              if (s > 0) {
                tmem_ld_32(s_col + 32 * s, x);
                tmem_wait_ld_into(x);
              }
              quarter(x, s);
            }
            release_s();
          }
          float la, lb, lc, ld;
          unpack_f32x2(l2[0], la, lb);
          unpack_f32x2(l2[1], lc, ld);
          l += (la + lb) + (lc + ld);
          sm100::tmem_wait_st();
        } else {
          // A warp without rows only keeps the barriers moving, within the chunk as
          // the others: its arrival for P(j) must not fall into the phase of P(j - 2).
          if (lane == 0) {
            arrive(&bars.mu[grp][w4]);
            arrive(&bars.s_free[grp]);
          }
          if (j >= 2 && !all_wait(&bars.done[(j - 2) & 3], (j - 2) >> 2)) {
            ok = false;
            break;
          }
        }
        sm100::tc_fence_before();
        __syncwarp();
        if (lane == 0) arrive(&bars.p_full[grp]);
      }
      j = j1;
      // The item's O, unnormalised: group 0 takes the first half of its columns,
      // group 1 the second.  (PV(j1 - 5) is known done: this group's or the other's
      // last P waited for PV(j1 - 4) at least.)
      ok = ok && all_wait(&bars.done[(j1 - 1) & 3], (j1 - 1) >> 2);
      sm100::tc_fence_after();
      constexpr int kHalf = D / 2;
      uint32_t o[kHalf / 32][32];
#pragma unroll
      for (int c = 0; c < kHalf / 32; ++c) tmem_ld_32(o_col + grp * kHalf + 32 * c, o[c]);
#pragma unroll
      for (int c = 0; c < kHalf / 32; ++c) tmem_wait_ld_into(o[c]);
      const float m = s_mu[row];
      s_l[item & 1][grp][row] = mu == m ? l : l * ex2_approx(mu - m);
      sm100::tc_fence_before();
      __syncwarp();
      if (lane == 0) arrive(&bars.o_free);
      ok = !any_of<2, kSoftmaxThreads>(!ok);  // (after a wait that gave up they leave together)
      if (!ok) break;
      l = s_l[item & 1][0][row] + s_l[item & 1][1][row];
      const int64_t out_row = static_cast<int64_t>(w.t.node0 + node) * p.H + w.g * p.group + hh;
      if (s_odd[item & 7] && valid && w.k1 > w.t.prefix) {
        // Values that are not finite, of the nodes that the row sees.
        for (int t = node;;) {
          if (t / kChunk + w.t.prefix >= w.k0 && t / kChunk + w.t.prefix < w.k1) {
            const __nv_bfloat16* v = p.tree[1] + (static_cast<int64_t>(w.t.node0 + t) * p.Hkv + w.g) * D + grp * kHalf;
#pragma unroll
            for (int c = 0; c < kHalf; ++c) {
              const float f = __bfloat162float(v[c]);
              if (!isfinite(f)) o[c / 32][c % 32] = __float_as_uint(__uint_as_float(o[c / 32][c % 32]) + f);
            }
          }
          const int up = p.parents[w.t.node0 + t];
          if (up < 0 || up >= t) break;
          t = up;
        }
      }
      if (w.k0 == 0 && w.k1 == w.t.chunks) {
        if (valid) {
          const float inv = __fdividef(1.f, l);
          uint4* dst = reinterpret_cast<uint4*>(p.out + out_row * D + grp * kHalf);
#pragma unroll
          for (int c = 0; c < kHalf; c += 8) {
            uint32_t y[4];
#pragma unroll
            for (int e = 0; e < 4; ++e)
              y[e] = pack_bf16x2(__uint_as_float(o[c / 32][c % 32 + 2 * e]) * inv,
                                 __uint_as_float(o[c / 32][c % 32 + 2 * e + 1]) * inv);
            dst[c / 8] = make_uint4(y[0], y[1], y[2], y[3]);
          }
          if (grp == 0 && p.lse) p.lse[out_row] = (m + __log2f(l)) * kLn2;
        }
      } else {
        const int64_t slot = 2ll * blockIdx.x + (w.first ? 0 : 1);
        if (valid) {
          float4* dst = reinterpret_cast<float4*>(p.part_o + (slot * p.slot_rows + row) * D + grp * kHalf);
#pragma unroll
          for (int c = 0; c < kHalf; c += 4)
            dst[c / 4] = make_float4(__uint_as_float(o[c / 32][c % 32]), __uint_as_float(o[c / 32][c % 32 + 1]),
                                     __uint_as_float(o[c / 32][c % 32 + 2]), __uint_as_float(o[c / 32][c % 32 + 3]));
          if (grp == 0) p.part_ml[slot * p.slot_rows + row] = make_float2(m, l);
        }
        // The CTAs that the item's first and last chunk lie in: share c starts at
        // the largest coordinate c X / G that is not above.
        const int64_t X = s_total, G = s_grid, a = w.start + kItemCost, z = a + w.t.chunks - 1;
        const int first = static_cast<int>(((a + 1) * G - 1) / X), last = static_cast<int>(((z + 1) * G - 1) / X);
        softmax_sync();
        if (tid == 0)
          s_last = adt::atomic_add_acq_rel_gpu(p.tickets + first, 1u) == static_cast<unsigned>(last - first);
        softmax_sync();
        if (s_last) {
          // Partial rows joined: weights 2^(m_c - M) over their sum.
          const int rows = min(w.t.n * p.group - w.blk * kRows, kRows);
          const int64_t slot0 = 2ll * first + (first * X / G >= w.start ? 0 : 1);
          auto slot_of = [&](int c) { return c == first ? slot0 : 2ll * c; };
          for (int i = tid; i < rows * (D / 4); i += kSoftmaxThreads) {
            const int r = i / (D / 4), c4 = i % (D / 4);
            float M = -INFINITY;
            for (int c = first; c <= last; ++c) M = fmaxf(M, __ldcg(&p.part_ml[slot_of(c) * p.slot_rows + r]).x);
            float lt = 0.f;
            float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
            for (int c = first; c <= last; ++c) {
              const int64_t at = slot_of(c) * p.slot_rows + r;
              const float2 ml = __ldcg(&p.part_ml[at]);
              const float4 v = __ldcg(reinterpret_cast<const float4*>(p.part_o + at * D) + c4);
              const float wt = ml.x == M ? 1.f : ex2_approx(ml.x - M);
              lt += wt * ml.y;
              acc.x += wt * v.x;
              acc.y += wt * v.y;
              acc.z += wt * v.z;
              acc.w += wt * v.w;
            }
            const float inv = __fdividef(1.f, lt);
            const int idx = w.blk * kRows + r, t = idx / p.group;
            const int64_t dst = static_cast<int64_t>(w.t.node0 + t) * p.H + w.g * p.group + idx - t * p.group;
            uint2 pk;
            pk.x = pack_bf16x2(acc.x * inv, acc.y * inv);
            pk.y = pack_bf16x2(acc.z * inv, acc.w * inv);
            *reinterpret_cast<uint2*>(p.out + dst * D + c4 * 4) = pk;
            if (c4 == 0 && p.lse) p.lse[dst] = (M + __log2f(lt)) * kLn2;
          }
          if (tid == 0) p.tickets[first] = 0u;
        }
      }
    }
  }
  sm100::tc_fence_before();
  __syncthreads();
  sm100::tc_fence_after();
  if (warp == kPvWarp) sm100::tmem_dealloc(tmem, kTmemCols);
}

// ---------------------------------------------------------------- host side

// 4-D map of the K cache (d, pos, kv head, tree), boxes of 128 positions.
adt_status make_cache_map(CUtensorMap* map, const void* base, int D, int max_kv, int Hkv, int B, int64_t sh, int64_t sb) {
  const adt::EncodeTiledFn encode = adt::encode_tiled();
  if (!encode) return ADT_ERR_CUDA;
  const int64_t rows = max_kv > 0 ? max_kv : 1;
  const cuuint64_t dims[4] = {static_cast<cuuint64_t>(D), static_cast<cuuint64_t>(rows), static_cast<cuuint64_t>(Hkv),
                              static_cast<cuuint64_t>(B)};
  const cuuint64_t strides[3] = {static_cast<cuuint64_t>(D), static_cast<cuuint64_t>(Hkv > 1 ? sh : rows * D),
                                 static_cast<cuuint64_t>(B > 1 ? sb : rows * D)};
  const cuuint32_t box[4] = {static_cast<cuuint32_t>(D), kChunk, 1, 1};
  const cuuint32_t one[4] = {1, 1, 1, 1};
  const CUresult r = encode(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 4, const_cast<void*>(base), dims, strides, box, one,
                            CU_TENSOR_MAP_INTERLEAVE_NONE,
                            D == 128 ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_64B,
                            CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
  return r == CUDA_SUCCESS ? ADT_OK : ADT_ERR_INVALID_ARG;
}

struct WsLayout {
  size_t part_ml, part_o, total;
};

// Tickets at the start, for any grid; then two items' partial rows of each CTA.
WsLayout ws_layout(int grid, int rows, int D) {
  WsLayout w;
  w.part_ml = kMaxGrid * sizeof(unsigned);
  w.part_o = adt::align_up(w.part_ml + static_cast<size_t>(2 * grid) * rows * sizeof(float2), 256);
  w.total = w.part_o + static_cast<size_t>(2 * grid) * rows * D * sizeof(float);
  return w;
}

// One CTA an SM, or fewer where no lengths within the limits make as many shares.
int grid_for(int sm_count, int B, int H, int Hkv, int max_nodes, int max_kv) {
  const int64_t chunks = (static_cast<int64_t>(max_kv) + kChunk - 1) / kChunk + (max_nodes + kChunk - 1) / kChunk;
  const int64_t blocks = (static_cast<int64_t>(max_nodes) * (H / Hkv) + kRows - 1) / kRows;
  const int64_t items = blocks * B * Hkv;  // (chunks < 2^24, items <= 2^25)
  const int64_t most = (chunks + kItemCost) * items / kMinShare + 1;
  const int sms = sm_count < kMaxGrid ? sm_count : kMaxGrid;
  return most < sms ? static_cast<int>(most) : sms;
}

int slot_rows_for(int H, int Hkv, int max_nodes) {
  const int64_t rows = static_cast<int64_t>(max_nodes) * (H / Hkv);
  return rows < kRows ? static_cast<int>(rows) : kRows;
}

template <int D>
adt_status launch(const AttnParams& p, const CUtensorMap& tm, int grid, int dev, cudaStream_t st) {
  static unsigned configured[2] = {0u, 0u};  // bit per device (< 64), per instantiation
  const unsigned bit = 1u << (dev & 31);
  unsigned& word = configured[(dev >> 5) & 1];
  if (!(__atomic_load_n(&word, __ATOMIC_ACQUIRE) & bit)) {
    ADT_CUDA_TRY(cudaFuncSetAttribute(tree_attn_q8_kernel<D>, cudaFuncAttributeMaxDynamicSharedMemorySize, Cfg<D>::kDynSmem));
    __atomic_fetch_or(&word, bit, __ATOMIC_ACQ_REL);
  }
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(static_cast<unsigned>(grid), 1, 1);
  cfg.blockDim = dim3(kThreads, 1, 1);
  cfg.dynamicSmemBytes = Cfg<D>::kDynSmem;
  cfg.stream = st;
  cudaLaunchAttribute attr[1] = {adt::pdl_attribute()};
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  ADT_CUDA_TRY(cudaLaunchKernelEx(&cfg, tree_attn_q8_kernel<D>, tm, p));
  return adt::launch_status();
}

}  // namespace

extern "C" {

size_t adt_tree_attn_q8_workspace_size(int32_t B, int32_t H, int32_t Hkv, int32_t D, int32_t max_nodes, int32_t max_kv) {
  if (B < 1 || H < 1 || Hkv < 1 || H % Hkv != 0 || (D != 64 && D != 128) || max_kv < 0 || max_nodes < 1 ||
      max_nodes > kMaxTreeNodes || static_cast<int64_t>(B) * max_nodes * H > kMaxRows)
    return 0;
  adt::DeviceInfo info;
  if (adt::device_info(&info) != ADT_OK) return 0;
  return ws_layout(grid_for(info.sm_count, B, H, Hkv, max_nodes, max_kv), slot_rows_for(H, Hkv, max_nodes), D).total;
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
  adt::DeviceInfo info;
  st = adt::device_info(&info);
  if (st != ADT_OK) return st;
  const int grid = grid_for(info.sm_count, B, H, Hkv, max_nodes, max_kv), rows = slot_rows_for(H, Hkv, max_nodes);
  const WsLayout ws = ws_layout(grid, rows, D);
  if (!workspace || workspace_bytes < ws.total || !adt::aligned16(workspace)) return ADT_ERR_WORKSPACE;
  AttnParams p{};
  p.q = reinterpret_cast<const __nv_bfloat16*>(q);
  p.v_cache = v_cache;
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
  p.slot_rows = rows;
  uint8_t* base = static_cast<uint8_t*>(workspace);
  p.tickets = reinterpret_cast<unsigned*>(base);
  p.part_ml = reinterpret_cast<float2*>(base + ws.part_ml);
  p.part_o = reinterpret_cast<float*>(base + ws.part_o);
  p.wait_limit = adt::wait_limit(kWaitLimit);
  CUtensorMap tm;
  st = make_cache_map(&tm, k_cache, D, max_kv, Hkv, B, cache_stride_h, cache_stride_b);
  if (st != ADT_OK) return st;
  return D == 128 ? launch<128>(p, tm, grid, info.device, adt::as_stream(stream))
                  : launch<64>(p, tm, grid, info.device, adt::as_stream(stream));
}

}  // extern "C"
