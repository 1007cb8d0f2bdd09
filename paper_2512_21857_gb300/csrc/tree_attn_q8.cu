// adt_tree_attn_q8: tree-masked attention, and that of single tokens, whose
// prefix is the 8-bit cache.
//
// The rows of a (tree, kv head) are its nodes' query heads of that group, node
// by node, in blocks of 128 = the tensor core's M.  An item is such a block with
// its keys, in chunks of 128: the prefix, then the tree's own.  The chunks of all
// items, with kItemCost more for each item's start, are dealt to one persistent
// CTA an SM in equal contiguous shares, so ragged batches and few long sequences
// fill the device alike; an item that a share's end cuts is joined from partial
// rows (outputs of its parts, and their sums) in the workspace by the CTA that ends its
// part last.
// Two kernels share this: of up to 16 rows tree_attn_q8_few.cuh, of more this one.
//
// S = Q K^T is made of e4m3 products, K as it lies in the cache: a query row,
// scaled by a power of two to at most 448, is cut into an e4m3 row and another of
// what that leaves, and both products add up in one accumulator (as many
// instructions as one product of bf16 has).  What the two leave is below 2^-17 of
// the row's largest magnitude.  The tree's own keys are cut the same way (four
// products).  The key's scale meets the score in fp32.
//
// With z = score (in powers of two) + e, 2^e the key's value scale, a row's weights are
// P = 2^(z + kHeadroom - base), base the largest z that it has seen, rounded up (raised
// only when a row grows by more than 2^kRescaleThreshold), so that what a weight is
// rounded to goes by what it adds to O, whatever the scales of values that the row does
// not see or gives no weight.  P is rounded to fp16 and V widened to fp16 in shared
// memory, exactly: bf16 weights are three bits worse, and two e4m3 ones a weight would
// lose keys of 2^-18 of the largest one's, of which a long cache can have enough to
// matter; fp16 ends at 2^-31 of it.  Scores take e relative to `top`, the largest so far
// (a number within a chunk), and the row sum adds P 2^(top - e - kShift), against a
// level of its own for each thread.  (Values whose scale is below 2^-kSpan of the top's,
// which are zeros in earnest, are taken to be 2^-kSpan there.)
//
// Queries, trees and ancestors are prepared by a launch before (prepare_kernel).
//
// Of up to 64 rows the tile holds each twice, a copy for each half of a chunk's
// keys: a thread's softmax is half as long, and the copies are joined at the end.
//
// Warp roles (16 warps):
//   0-3, 4-7  two softmax groups that take the chunks in turn, a thread a row;
//             the running base passes from group to group through shared
//             memory, P goes to tensor memory;
//   8         K tiles by TMA into a ring, the queries, and the scales of both,
//             written a chunk after their bytes were asked for;
//   9         V tiles (packed rows: plain bulk copies) into a ring;
//   10        S products;
//   11        PV products;
//   12-15     V from e4m3 to fp16 (the rows past the prefix zeroed).
// Every wait is bounded; a timeout sets ADT_DEVERR_TIMEOUT.
//
// Bound by the turns of the softmax groups: a CTA takes 2320 cycles a chunk with 64 rows
// (each twice) and 2790 with 128, its two groups a chunk each at a time, of which waits
// for tensor memory, shared memory and the other group are more than half (issue slots
// 42 % busy, tensor cores 23 %); V's widening keeps up.  Measured: four trees of 64, 64,
// 27 and 64 nodes over 1444 to 2400 rows, 32 / 32 heads x 128, 39 us (11 at HBM's rate), 5
// of them the launch before; trees of 64 nodes over 3500 to 6001 rows, 32 / 8 heads x 128,
// 48 us (11 at the tensor cores' bf16 rate), 5 of them the joining of cut items.  (A row's
// base over scores and value scales, against one of scores alone and one reference for an
// item's value scales: 39.4 and 47.9 us for 38.7 and 46.6.)
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
constexpr int kItemCost = 4;            // chunks that an item's start and end take the time of (decode over ragged caches:
                                        // 85 us with 3 to 6 of them, 101 with 1)
constexpr int kJoinCost = 6;            // ... and that joining an item's parts takes
constexpr int kMinShare = 6;            // coordinates (see Walk) of a CTA's share, where there are few
constexpr int kSoftmaxThreads = 256;
constexpr int kKWarp = 8, kVWarp = 9, kSWarp = 10, kPvWarp = 11, kConvWarp = 12;
constexpr int kConvThreads = 128;
constexpr int kThreads = 512;
constexpr int kMaxScaleSlots = 16;
constexpr int kMaxStages = 6;
constexpr int kMaxGrid = 1024;          // tickets of the workspace
constexpr uint32_t kTmemCols = 512;
constexpr uint32_t kTiles = 3, kOCol = kTiles * kChunk;  // S tiles of 128 columns, whose first 64 P takes as it is made; O
constexpr uint32_t kWaitLimit = 1u << 22;
constexpr uint32_t kDrainLimit = 1u << 20;  // of the waits for what is in flight
constexpr float kLog2e = 1.44269504088896340736f;
constexpr float kLn2 = 0.69314718055994530942f;
constexpr float kRescaleThreshold = 8.0f;  // log2 units
constexpr float kHeadroom = 7.0f;          // weights up to 2^15: fp16 ends below 2^16
constexpr int kSpan = 96, kShift = kSpan / 2;  // (a weight 2^-24 of the largest is a normal number 2^-96 further down)

template <int D>
struct Cfg {
  static constexpr int kKStages = D == 128 ? 3 : 6;
  static constexpr int kVStages = D == 128 ? 2 : 4;
  static constexpr int kScaleSlots = D == 128 ? 8 : 16;
  static constexpr int kTile = kChunk * D;                // 128 rows of e4m3
  static constexpr int kBlock = kChunk * 128;             // one 64-column block of 128 rows of fp16
  static constexpr int kWide = D / 64 * kBlock;           // 128 rows of fp16
  static constexpr int kQOff = 0;                         // [2 items][high, low]
  static constexpr int kKOff = kQOff + 4 * kTile;
  static constexpr int kVOff = kKOff + kKStages * kTile;
  static constexpr int kWideOff = kVOff + kVStages * kTile;
  static constexpr int kScaleOff = kWideOff + 2 * kWide;  // [slots][K's scale, e - top, 2^(top - e - kShift)][128] fp32
  static constexpr int kJoinOff = kScaleOff + kScaleSlots * 3 * kChunk * 4;  // D = 64: [2 groups][128][32] fp32
  static constexpr int kDynSmem = kJoinOff + (D == 128 ? 0 : 2 * kRows * 32 * 4) + 1024;  // + alignment slack
  static_assert(D != 128 || kWide == 2 * kRows * 32 * 4, "copies are joined in a V tile");
  static_assert(kDynSmem <= 221 * 1024, "with 6 KB of the kernel's own within the 227 of an SM");
  static constexpr uint32_t kIdescO = sm100::idesc_f16_f32(kRows, D, 0, 1);
  static_assert(kKStages <= kMaxStages && kVStages <= kMaxStages && kScaleSlots <= kMaxScaleSlots && kOCol + D <= kTmemCols, "sizes");
};

// What the first launch makes of the queries and of the trees, as the second one's
// shared memory takes it.  Blocks of q_rows (<= 128) queries, chunks of t_rows
// (<= 128) nodes; (b, g) the tree and kv head.
struct Prepared {
  uint8_t* q;       // [b, g][block][high, low][q_rows x D]
  float* q_scale;   // [b, g][block][q_rows], times softmax_scale log2 e
  uint8_t* k;       // [b, g][chunk][high, low][t_rows x D]
  uint4* v;         // [b, g][chunk][D / 64][t_rows][8], fp16
  uint8_t* scale;   // [b, g][chunk][of K, of V, whether V is not finite][t_rows]
  uint4* seen;      // [b][node][chunk]: the nodes that it sees
  int q_rows, blocks, t_rows, chunks;
};

struct AttnParams {
  Prepared pre;
  const __nv_bfloat16* q;
  const uint8_t* v_cache;
  const uint8_t* scale[2];
  const int32_t* kv_len;
  const __nv_bfloat16* tree[2];
  const int32_t* parents;
  const int32_t* offs;
  int B, H, Hkv, group, max_nodes, max_kv, slot_rows;
  int copies;          // of a row in a tile: 1 or 2
  int64_t sb, sh, ssb, ssh;
  float scale_log2;
  __nv_bfloat16* out;
  float* lse;
  unsigned* tickets;   // [grid], of the items that start in a CTA's share and end in another's
  float2* part_ml;     // [2 grid][slot_rows]: row sums of a CTA's first and of its last item (part_sum)
  float4* part_o;      // [2 grid][D / 4][slot_rows]: O over the row sum
  unsigned* err;
  uint32_t wait_limit;
};

struct Tree {
  int node0, n, L, chunks, prefix, blocks;  // chunks of an item, those of the prefix, row blocks of a kv head
};

// Tree b; one that is malformed or out of range has no items.
__device__ __forceinline__ Tree tree_of(const AttnParams& p, int b, unsigned* bits) {
  Tree t;
  t.node0 = __ldcg(p.offs + b);
  t.n = __ldcg(p.offs + b + 1) - t.node0;
  t.L = __ldcg(p.kv_len + b);
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
// Where an item a CTA takes no longer than equal shares with their joining would,
// all items are padded to one width, and a share is an item.
struct Walk {
  int b, g, blk;
  Tree t;
  int64_t start, end;  // the item's first coordinate; the end of the share
  int padded;          // every item's width, or 0: its chunks and kItemCost
  int k0, k1;          // the share's chunks of the item
  bool first;          // of the share's items
  bool more;
  __device__ __forceinline__ void clip(int64_t from) {
    const int64_t base = start + kItemCost;
    k0 = from > base ? static_cast<int>(from - base) : 0;
    k1 = static_cast<int>(min(static_cast<int64_t>(t.chunks), end - base));
  }
  __device__ __forceinline__ bool some() const { return k1 > k0; }
};

// The share's next item; its `more` says whether there is one.  (One copy of this
// for all roles: the instruction cache of an SM is smaller than this kernel.)
__device__ __noinline__ Walk next_item(const AttnParams& p, Walk w) {
  w.start += w.padded ? w.padded : kItemCost + w.t.chunks;
  w.first = false;
  w.more = w.start + kItemCost < w.end;
  if (!w.more) return w;
  if (++w.blk == w.t.blocks) {
    w.blk = 0;
    if (++w.g == p.Hkv) {
      w.g = 0;
      unsigned bits = 0u;
      do {
        if (++w.b >= p.B) {
          w.more = false;
          return w;
        }
        w.t = tree_of(p, w.b, &bits);
      } while (w.t.chunks == 0);
    }
  }
  w.clip(w.start);
  w.more = w.some();
  return w;
}

// This CTA's share, by one warp: its first item, the coordinates of all items and
// the number of shares.
__device__ __forceinline__ void find_share(const AttnParams& p, int lane, Walk* walk, int64_t* all, int* count, unsigned* err) {
  unsigned bits = 0u;
  Tree t{};
  int64_t mine = 0;
  int items = 0, longest = 0;
  for (int b = lane; b < p.B; b += 32) {
    t = tree_of(p, b, &bits);
    if (!t.chunks) continue;
    items += t.blocks * p.Hkv;  // (at most 2^24 rows: no more items)
    longest = max(longest, t.chunks);
    mine += static_cast<int64_t>(t.chunks + kItemCost) * t.blocks * p.Hkv;
  }
  if (err && bits) adt::raise_error(err, bits);
  int64_t total = adt::warp_sum(mine);
  items = adt::warp_sum(items);
  longest = __reduce_max_sync(adt::kFullMask, longest);
  int64_t shares = total / kMinShare;
  shares = shares < 1 ? 1 : shares > gridDim.x ? gridDim.x : shares;
  int padded = 0;
  if (items > 0 && items <= static_cast<int>(gridDim.x) && longest + kItemCost <= total / gridDim.x + kJoinCost) {
    padded = longest + kItemCost;
    shares = items;
    total = static_cast<int64_t>(items) * padded;
  }
  auto width = [&](const Tree& t) -> int { return padded ? padded : t.chunks + kItemCost; };
  auto cost = [&](const Tree& t) -> int64_t { return t.chunks ? static_cast<int64_t>(width(t)) * t.blocks * p.Hkv : 0; };
  const int64_t c = blockIdx.x;
  const int64_t x0 = c < shares ? c * total / shares : total, x1 = c < shares ? (c + 1) * total / shares : total;
  Walk w{};
  w.first = w.more = true;
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
        const int64_t off = x0 - (before + upto - mine_here), each = width(t), item = off / each;
        w.b = b0 + lane;
        w.g = static_cast<int>(item / t.blocks);
        w.blk = static_cast<int>(item % t.blocks);
        w.t = t;
        w.start = x0 - off + item * each;
        w.end = x1;
        w.padded = padded;
        w.clip(x0);
        *walk = w;
      }
      break;
    }
    before += __shfl_sync(adt::kFullMask, upto, 31);
  }
  if (lane == 0) {
    if (x0 >= x1) *walk = w;  // (no chunks)
    *all = total;
    *count = static_cast<int>(shares);
  }
}

// The tree's values that are not finite were left out of the products: adds those
// that node t sees, of nodes t0 up to before t1, to `cols` columns of its row, as
// written (final or partial).  tree: the first node's values at the first column.
__device__ __noinline__ void add_odd(__nv_bfloat16* out, float* part, int part_step, int cols, const __nv_bfloat16* tree,
                                     const int32_t* parents, int64_t step, int t, int t0, int t1) {
  for (;;) {
    for (int i = 0; t >= t0 && t < t1 && i < cols; ++i) {
      const float f = __bfloat162float(tree[t * step + i]);
      if (isfinite(f)) continue;
      if (out)
        out[i] = __float2bfloat16(__bfloat162float(out[i]) + f);
      else
        part[(i / 4) * part_step * 4 + i % 4] += f;
    }
    const int up = parents[t];
    if (up < 0 || up >= t) return;
    t = up;
  }
}

struct Bars {
  uint64_t k_full[kMaxStages], k_free[kMaxStages];
  uint64_t v_full[kMaxStages], v_free[kMaxStages];
  uint64_t scale_full[kMaxScaleSlots];
  uint64_t wide_full[2];     // a V tile in fp16
  uint64_t q_full[2], q_free[2];
  uint64_t s_full[4], p_full[4];
  uint64_t mu[2][4];         // the running maxima after a chunk are in shared memory, per group and warp
  uint64_t done[4];          // the PV product of chunk j is done (barrier j % 4)
  uint64_t o_free;           // an item's O is read
  uint64_t join_free[2];     // its copies are joined (even and odd items: a second one may end before the first is asked for)
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

__device__ __forceinline__ uint32_t e4m3x2_to_f16(uint32_t two) {
  uint32_t r;
  asm("cvt.rn.f16x2.e4m3x2 %0, %1;\n" : "=r"(r) : "h"(static_cast<uint16_t>(two)));
  return r;
}

__device__ __forceinline__ uint32_t pack_half2(float lo, float hi) {
  const __half2 v = __floats2half2_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&v);
}

// 16 elements of a bf16 row, D / 16 neighbouring lanes to a row (all lanes of the
// warp take part): cut into e4m3 rows, each of `up` times what the ones before leave,
// whose sum (a row `up` times smaller than the one before) goes with the scale
// 2^(s - 127), s what it returns.  A row that is not finite becomes NaN.
template <int D, int kParts>
__device__ __forceinline__ uint32_t cut_row(const uint4 (&x)[2], float up, uint4 (&parts)[kParts]) {
  const uint32_t w[8] = {x[0].x, x[0].y, x[0].z, x[0].w, x[1].x, x[1].y, x[1].z, x[1].w};
  uint32_t most = 0u;
#pragma unroll
  for (int k = 0; k < 8; ++k) most = max(most, max(w[k] << 16 & 0x7fff0000u, w[k] & 0x7fff0000u));
#pragma unroll
  for (int o = D / 32; o > 0; o >>= 1) most = max(most, __shfl_xor_sync(adt::kFullMask, most, o));
  const bool finite = most < 0x7f800000u;
  const uint32_t s = finite ? adt::q8_row_scale(__uint_as_float(most)) : 127u;
  const float inv = __uint_as_float((254u - s) << 23);
  uint32_t y[kParts][4];
#pragma unroll
  for (int k = 0; k < 4; ++k) {
#pragma unroll
    for (int i = 0; i < kParts; ++i) y[i][k] = 0u;
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      const uint32_t z = w[2 * k + e];
      float a = __uint_as_float(z << 16) * inv, b = __uint_as_float(z & 0xffff0000u) * inv;
#pragma unroll
      for (int i = 0; i < kParts; ++i) {
        const uint32_t two = adt::f32x2_to_e4m3(a, b);
        const float2 back = adt::e4m3x2_to_f32(two);
        y[i][k] |= two << (16 * e);
        a = (a - back.x) * up;
        b = (b - back.y) * up;
      }
    }
#pragma unroll
    for (int i = 0; i < kParts; ++i)
      if (!finite) y[i][k] = 0x7f7f7f7fu;
  }
#pragma unroll
  for (int i = 0; i < kParts; ++i) parts[i] = make_uint4(y[i][0], y[i][1], y[i][2], y[i][3]);
  return s;
}

__device__ __forceinline__ void group_sync(int grp) {  // of the four warps of a softmax group
  if (grp == 0)
    asm volatile("bar.sync 3, 128;\n" ::: "memory");
  else
    asm volatile("bar.sync 4, 128;\n" ::: "memory");
}

constexpr int kAhead = 8;  // chunks whose scales are asked for ahead: as many as a warp's lanes prefetch at once
__device__ __forceinline__ void prefetch_l2(const void* src) { asm volatile("prefetch.global.L2 [%0];\n" ::"l"(src)); }

// A bounded wait, as short as it can be (its callers are many, and the instruction
// cache of an SM is smaller than this kernel): false after `limit` polls, or once
// another role has given up.
__device__ __forceinline__ bool poll(uint64_t* bar, uint32_t parity, volatile int* abort_flag, uint32_t limit) {
  const uint32_t a = sm100::smem_addr(bar);
#pragma unroll 1
  while (!sm100::mbar_try_wait(a, parity)) {
    if (--limit == 0 || ((limit & 255u) == 0 && *abort_flag)) return false;
  }
  return true;
}

// A query row's cut scale times softmax_scale log2 e; never 0, which would make NaN of the -inf of a masked key.
__device__ __forceinline__ float row_factor(uint32_t s, float scale_log2) {
  return fmaxf(__uint_as_float(s << 23) * scale_log2, 1e-38f);
}
__device__ __forceinline__ float power_of_two(int e) {
  return e < -126 ? 0.f : __uint_as_float(static_cast<uint32_t>(min(e, 127) + 127) << 23);
}

// 2^(a - b) for what a level's sums (or O) take on at another one's, where both may be -inf.
__device__ __forceinline__ float level_factor(float a, float b) { return a == b ? 1.f : ex2_approx(a - b); }
// O over the row sum l is O reciprocal(l), 0 of a part whose rows see none of its keys, times
// 2^e of their levels: half_power(e) twice, which stays within fp32 where 2^e may not.
__device__ __forceinline__ float half_power(float e) { return ex2_approx(0.5f * e); }
__device__ __forceinline__ float reciprocal(float l) { return l == 0.f ? 0.f : __fdividef(1.f, l); }
// A part's row sum, l 2^level, as it is stored: a level and a factor in [1, 2), or 0, or what is not finite.
__device__ __forceinline__ float2 part_sum(float level, float l) {
  const uint32_t bits = __float_as_uint(l);
  if (l == 0.f) return make_float2(-INFINITY, 0.f);
  if ((bits & 0x7f800000u) == 0x7f800000u) return make_float2(level, l);
  return make_float2(level + static_cast<float>(static_cast<int>(bits >> 23) - 127), __uint_as_float((bits & 0x7fffffu) | 0x3f800000u));
}
constexpr float kJoinScale = 0x1p-9f;  // of weights that add parts up: within fp32 whatever the values
constexpr float kJoinLevel = 9.f;

// The first launch: a row is D / 16 lanes', 16 elements each.  Of a tree the query
// rows, then its nodes' rows of every kv head (zeros up to a multiple of 16 nodes).
// Bound by its launch and two rounds of loads (four trees of 64 nodes, 32 / 32 heads x
// 128: 5 us more for a call); within the second one, every item and every share of one would do
// it anew, by warps that have other work.
constexpr int kPrepThreads = 256;

template <int D>
__global__ void __launch_bounds__(kPrepThreads) prepare_kernel(const AttnParams p) {
  constexpr int kLanes = D / 16, kPass = kPrepThreads / kLanes;
  __shared__ int16_t s_par[kMaxTreeNodes];
  asm volatile("griddepcontrol.wait;\n" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;\n" ::: "memory");
  const int b = blockIdx.y, tid = threadIdx.x;
  unsigned bits = 0u;
  const Tree t = tree_of(p, b, &bits);
  if (blockIdx.x == 0 && tid == 0 && bits) adt::raise_error(p.err, bits);
  if (t.n == 0) return;
  const Prepared& w = p.pre;
  const int queries = t.n * p.H, nodes = (t.n + 15) & ~15;
  const int unit = blockIdx.x * kPass + tid / kLanes, cl = tid % kLanes;
  if (blockIdx.x == 0) {
    // What each node sees.  Parents precede their children; anything else marks the
    // tree malformed.
    for (int i = tid; i < t.n; i += kPrepThreads) {
      const int up = p.parents[t.node0 + i];
      s_par[i] = static_cast<int16_t>(min(max(up, -1), kMaxTreeNodes));
      if ((i == 0) != (up < 0) || up >= i) adt::raise_error(p.err, ADT_DEVERR_BAD_TREE);
    }
    __syncthreads();
    for (int i = tid; i < t.n * w.chunks; i += kPrepThreads) {
      uint32_t m[4] = {0u, 0u, 0u, 0u};
      const int t0 = i % w.chunks * kChunk;
      for (int x = i / w.chunks;;) {
        const int at = x - t0;
#pragma unroll
        for (int e = 0; e < 4; ++e) m[e] |= at >> 5 == e ? 1u << (at & 31) : 0u;
        const int up = s_par[x];
        if (up < 0 || up >= x) break;
        x = up;
      }
      w.seen[static_cast<int64_t>(b) * p.max_nodes * w.chunks + i] = make_uint4(m[0], m[1], m[2], m[3]);
    }
  }
  uint4 x[2] = {}, v[2] = {};
  const bool is_q = unit < queries;
  const int rest = unit - queries, node = is_q ? unit / p.H : rest / p.Hkv;
  const bool is_t = !is_q && node < nodes;
  const int h = is_q ? unit - node * p.H : 0, g = is_q ? h / p.group : rest - node * p.Hkv;
  if (is_q) {
    const uint4* src = reinterpret_cast<const uint4*>(p.q + (static_cast<int64_t>(t.node0) * p.H + unit) * D) + cl * 2;
    x[0] = src[0];
    x[1] = src[1];
  } else if (is_t && node < t.n) {
    const int64_t at = (static_cast<int64_t>(t.node0 + node) * p.Hkv + g) * D;
    const uint4* src = reinterpret_cast<const uint4*>(p.tree[0] + at) + cl * 2;
    x[0] = src[0];
    x[1] = src[1];
    src = reinterpret_cast<const uint4*>(p.tree[1] + at) + cl * 2;
    v[0] = src[0];
    v[1] = src[1];
  }
  uint4 cut[2];
  const uint32_t s = cut_row<D>(x, 1.f, cut);
  const int64_t bg = static_cast<int64_t>(b) * p.Hkv + g;
  if (is_q) {
    const int row = node * p.group + h - g * p.group, blk = row / kRows, r = row % kRows;
    const int64_t at = bg * w.blocks + blk;
    uint8_t* dst = w.q + at * 2 * w.q_rows * D + tile_off<D>(r, cl);
    *reinterpret_cast<uint4*>(dst) = cut[0];
    *reinterpret_cast<uint4*>(dst + w.q_rows * D) = cut[1];
    if (cl == 0) w.q_scale[at * w.q_rows + r] = row_factor(s, p.scale_log2);
  }
  // Values: those that are not finite as zeros (a weight of 0 times them would
  // reach rows that do not see them), scaled as their cached rows would be, but in
  // fp16: below 448, with 2^-24 the least step, 2^-33 of the row's largest.
  uint32_t y[8] = {v[0].x, v[0].y, v[0].z, v[0].w, v[1].x, v[1].y, v[1].z, v[1].w}, most = 0u, odd = 0u;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const bool lo = (y[e] & 0x7f80u) == 0x7f80u, hi = (y[e] & 0x7f800000u) == 0x7f800000u;
    odd |= lo || hi ? 1u : 0u;
    if (lo) y[e] &= 0xffff0000u;
    if (hi) y[e] &= 0xffffu;
    most = max(most, max(y[e] << 16 & 0x7fff0000u, y[e] & 0x7fff0000u));
  }
#pragma unroll
  for (int o = kLanes / 2; o > 0; o >>= 1) {
    most = max(most, __shfl_xor_sync(adt::kFullMask, most, o));
    odd |= __shfl_xor_sync(adt::kFullMask, odd, o);
  }
  if (!is_t) return;
  const uint32_t vs = adt::q8_row_scale(__uint_as_float(most));
  const float inv = __uint_as_float((254u - vs) << 23);
#pragma unroll
  for (int e = 0; e < 8; ++e)
    y[e] = pack_half2(__uint_as_float(y[e] << 16) * inv, __uint_as_float(y[e] & 0xffff0000u) * inv);
  const int r = node % kChunk;
  const int64_t at = bg * w.chunks + node / kChunk;
  uint8_t* dst = w.k + at * 2 * w.t_rows * D + tile_off<D>(r, cl);
  *reinterpret_cast<uint4*>(dst) = cut[0];
  *reinterpret_cast<uint4*>(dst + w.t_rows * D) = cut[1];
  uint8_t* wide = reinterpret_cast<uint8_t*>(w.v + at * (D / 64) * w.t_rows * 8);
  *reinterpret_cast<uint4*>(wide + sw128_off(r, 2 * cl, w.t_rows)) = make_uint4(y[0], y[1], y[2], y[3]);
  *reinterpret_cast<uint4*>(wide + sw128_off(r, 2 * cl + 1, w.t_rows)) = make_uint4(y[4], y[5], y[6], y[7]);
  if (cl == 0) {
    uint8_t* sc = w.scale + at * 3 * w.t_rows + r;
    sc[0] = static_cast<uint8_t>(s);
    sc[w.t_rows] = static_cast<uint8_t>(vs);
    sc[2 * w.t_rows] = static_cast<uint8_t>(odd);
  }
}

// What was prepared may be read after this.  (The launch before lets this one start
// once all work before it is done, so the caller's tensors may be read at any time:
// past L1, which may hold what an earlier launch read.)
__device__ __forceinline__ void await_prepared() { asm volatile("griddepcontrol.wait;\n" ::: "memory"); }

template <int D>
__global__ void __launch_bounds__(kThreads, 1)
    tree_attn_q8_kernel(const __grid_constant__ CUtensorMap tm_k, const AttnParams p) {
  using C = Cfg<D>;
  constexpr int KS = C::kKStages, VS = C::kVStages, kScaleSlots = C::kScaleSlots;
  extern __shared__ __align__(1024) uint8_t smem_raw[];
  uint8_t* smem = smem_raw + ((1024u - (sm100::smem_addr(smem_raw) & 1023u)) & 1023u);
  __shared__ Bars bars;
  // Of an item, even or odd (one may begin before all have left the one before): the rows' bases, a group's row sums (level, sum).
  __shared__ float s_mu[2][kRows];
  __shared__ float2 s_l[2][2][kRows];
  __shared__ float s_top[kScaleSlots];    // the largest value scale up to a chunk, as a power of two
  __shared__ int s_odd[kScaleSlots];      // 1: a tree chunk has values that are not finite; 2: the item has had rows that are not
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
    init(bars.s_full, 4, 1);
    init(bars.p_full, 4, 4);
    init(bars.mu[0], 8, 1);
    init(bars.done, 4, 1);
    init(&bars.o_free, 1, 8);
    init(bars.join_free, 2, 8);
    init(bars.drain, 2, 1);
    sm100::fence_mbar_init();
  }
  if (warp == kPvWarp) {
    sm100::tmem_alloc(sm100::smem_addr(&tmem_slot), kTmemCols);
    sm100::tmem_relinquish();
  }
  if (warp == kKWarp && lane == 0) sm100::prefetch_tensormap(&tm_k);
  if (warp == 0) find_share(p, lane, &s_walk, &s_total, &s_grid, nullptr);
  sm100::tc_fence_before();
  __syncthreads();
  sm100::tc_fence_after();
  const uint32_t tmem = tmem_slot;
  Walk w = s_walk;
  if (!w.some()) {  // (all threads alike)
    await_prepared();
    __syncthreads();
    if (warp == kPvWarp) sm100::tmem_dealloc(tmem, kTmemCols);
    return;
  }
  uint8_t* sQ = smem + C::kQOff;
  uint8_t* sK = smem + C::kKOff;
  uint8_t* sV = smem + C::kVOff;
  uint8_t* sWide = smem + C::kWideOff;
  auto wait = [&](uint64_t* bar, uint32_t phase) { return poll(bar, phase & 1u, &s_abort, p.wait_limit); };
  // What a role says whose wait gave up: the others' give up too.
  auto give_up = [&]() {
    s_abort = 1;
    adt::raise_error(p.err, ADT_DEVERR_TIMEOUT);
  };
  auto all_wait = [&](uint64_t* bar, uint32_t phase) { return __all_sync(adt::kFullMask, wait(bar, phase)); };
  auto arrive = [&](uint64_t* bar) { sm100::mbar_arrive(sm100::smem_addr(bar)); };
  // Chunk j (counted over the whole share) has slot j % stages of a ring, its
  // phase there j / stages.  A wait on a parity is only meaningful to a thread
  // that knows the phase before complete; each comment below says how.
  uint32_t j = 0;

  if (warp == kKWarp) {
    // ------------------------------------------------------------ K tiles, scales
    uint32_t issued = 0, q_issued = 0;  // one past the last tile, and the last item's queries, requested
    // Scales of four keys and of their values, and a tree's values that are not finite,
    // of the chunk before.  They come byte by byte (their rows need no alignment) and
    // are written a chunk later.
    uint32_t pend[3][4] = {};
    int slot = 0, top = 0, k = w.k0;
    uint32_t item = 0;
    bool ok = true, first = true, have = false, lost = false;
    for (;; ++j) {
      const int64_t s0 = w.b * p.ssb + w.g * p.ssh, bg = static_cast<int64_t>(w.b) * p.Hkv + w.g;
      const bool tree_k = k >= w.t.prefix;
      const int64_t chunk = bg * p.pre.chunks + k - w.t.prefix;  // (of the tree's)
      const int keys = tree_k ? w.t.n - (k - w.t.prefix) * kChunk : w.t.L - k * kChunk;
      auto prefetch_scale = [&](int at, int i) {  // first and last byte of K's and of V's
        const int row = min(at * kChunk + (i & 1) * (kChunk - 1), w.t.L - 1);
        if (at * kChunk < w.t.L && at < w.k1) prefetch_l2(p.scale[i >> 1 & 1] + s0 + row);
      };
      const bool fresh = k == w.k0;
      if (w.more) {
        const int st = j % KS;
        if (lane == 0) {
          ok = !fresh || item < 2 || wait(&bars.q_free[item & 1], (item >> 1) - 1);
          ok = ok && (j < KS || wait(&bars.k_free[st], j / KS - 1));
        }
        ok = __shfl_sync(adt::kFullMask, ok ? 1 : 0, 0) != 0;
        if (!ok) break;
        if (tree_k && j == 0) await_prepared();
        if (lane == 0) {
          const uint32_t bar = sm100::smem_addr(&bars.k_full[st]), dst = sm100::smem_addr(sK + st * C::kTile);
          if (tree_k) {  // (the low part comes from warp 9 to the same barrier)
            const int bytes = min(kChunk, (keys + 15) & ~15) * D;
            sm100::mbar_arrive_expect_tx(bar, 2 * bytes);
            sm100::bulk_load(dst, p.pre.k + chunk * 2 * p.pre.t_rows * D, bytes, bar);
          } else {
            sm100::mbar_arrive_expect_tx(bar, C::kTile);
            sm100::tma_load_4d(dst, &tm_k, 0, k * kChunk, w.g, w.b, bar);
          }
        }
        if (fresh) {
          // Without a prefetch this warp waited for memory once a chunk, 2000 cycles of 2800.
          prefetch_scale(k + (lane >> 2), lane);
          if (j == 0) await_prepared();
          if (lane == 0) {  // the item's queries, `copies` times
            const int rows = (min(w.t.n * p.group - w.blk * kRows, kRows) + 7) & ~7;
            const uint32_t bar = sm100::smem_addr(&bars.q_full[item & 1]);
            sm100::mbar_arrive_expect_tx(bar, 2 * p.copies * rows * D);
            const uint8_t* src = p.pre.q + (bg * p.pre.blocks + w.blk) * 2 * p.pre.q_rows * D;
            const uint32_t dst = sm100::smem_addr(sQ + (item & 1) * 2 * C::kTile);
#pragma unroll 1
            for (int c = 0; c < p.copies; ++c) {
              sm100::bulk_load(dst + c * (C::kTile / p.copies), src, rows * D, bar);
              sm100::bulk_load(dst + C::kTile + c * (C::kTile / p.copies), src + p.pre.q_rows * D, rows * D, bar);
            }
            q_issued = item + 1;
          }
        }
        issued = j + 1;
      }
      if (have) {
        // The scales of the chunk before.  Their slot was read last for a chunk
        // kScaleSlots before, which was done with before S of three chunks on could
        // start, and S(j - KS) is done.
        static_assert(kScaleSlots >= KS + 4, "a slot that is read");
        uint32_t most = 0u;
#pragma unroll
        for (int i = 0; i < 4; ++i) most = max(most, pend[1][i] == 255u ? 0u : pend[1][i]);
        // A value that is not a number takes the outputs of all rows, which all see it, and leaves the row sums.
        lost = (lost && !first) || __any_sync(adt::kFullMask, pend[1][0] == 255u || pend[1][1] == 255u || pend[1][2] == 255u || pend[1][3] == 255u);
        most = __reduce_max_sync(adt::kFullMask, most);
        const bool odd = __any_sync(adt::kFullMask, (pend[2][0] | pend[2][1] | pend[2][2] | pend[2][3]) != 0u);
        top = first ? static_cast<int>(most) : max(top, static_cast<int>(most));
        float f[12];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int e = max((pend[1][i] == 255u ? 0 : static_cast<int>(pend[1][i])) - top, -kSpan);
          f[i] = adt::q8_scale(pend[0][i]);
          f[4 + i] = static_cast<float>(e);
          f[8 + i] = power_of_two(-e - kShift);
        }
        float4* dst = reinterpret_cast<float4*>(s_scale + slot * 3 * kChunk);
#pragma unroll
        for (int i = 0; i < 3; ++i) dst[32 * i + lane] = make_float4(f[4 * i], f[4 * i + 1], f[4 * i + 2], f[4 * i + 3]);
        if (lane == 0) {
          s_odd[slot] = (odd ? 1 : 0) | (lost ? 2 : 0);
          s_top[slot] = static_cast<float>(top - 127);
        }
        __syncwarp();
        if (lane == 0) arrive(&bars.scale_full[slot]);
      }
      if (!w.more) break;
      const uint8_t* src = (tree_k ? p.pre.scale + chunk * 3 * p.pre.t_rows : p.scale[0] + s0 + k * kChunk) + lane * 4;
      const uint8_t* vsrc = tree_k ? src + p.pre.t_rows : p.scale[1] + s0 + k * kChunk + lane * 4;
      const int left = keys - lane * 4;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        pend[0][i] = 127u;
        pend[1][i] = pend[2][i] = 0u;
        if (i < left) {
          pend[0][i] = __ldcg(src + i);
          pend[1][i] = __ldcg(vsrc + i);
          if (tree_k) pend[2][i] = vsrc[p.pre.t_rows + i];
        }
      }
      if (!tree_k && lane < 4) prefetch_scale(k + kAhead, lane);
      slot = static_cast<int>(j % kScaleSlots);
      first = fresh;
      have = true;
      if (++k == w.k1) {
        w = next_item(p, w);
        k = w.k0;
        ++item;
      }
    }
    if (!ok && lane == 0) give_up();
    asm volatile("griddepcontrol.launch_dependents;\n" ::: "memory");
    // Every copy issued lands before the CTA goes on (also after an abort).
    if (lane == 0) {
      auto landed = [&](uint64_t* bar, uint32_t n, uint32_t slots) {  // the last uses of a ring, of n in all
        for (uint32_t i = n > slots ? n - slots : 0; i < n; ++i)
          (void)sm100::mbar_wait_bounded(sm100::smem_addr(bar + i % slots), i / slots & 1u, kDrainLimit);
      };
      landed(bars.k_full, issued, KS);
      landed(bars.q_full, q_issued, 2);
    }
    __syncwarp();
  } else if (warp == kVWarp) {
    // ------------------------------------------------------------ V tiles
    if (lane == 0) {
      uint32_t issued = 0;
      bool ok = true;
      for (; ok && w.more; w = next_item(p, w)) {
        const uint8_t* v = p.v_cache + w.b * p.sb + w.g * p.sh;
        for (int k = w.k0; k < w.k1; ++k, ++j) {
          const int st = j % VS;
          const uint32_t bar = sm100::smem_addr(&bars.v_full[st]);
          if (j >= VS && !wait(&bars.v_free[st], j / VS - 1)) {
            ok = false;
            break;
          }
          if (k >= w.t.prefix) {
            await_prepared();
            // The low part of the tree's keys, once the chunk before in that slot of K
            // is done with, and its barrier's phase with it.  (S(j - 2 KS) is: V(j - VS)
            // was widened after PV(j - VS - 2).)
            static_assert(VS + 2 <= 2 * KS, "a phase of k_free that is known complete");
            if (j >= KS && !wait(&bars.k_free[j % KS], j / KS - 1)) {
              ok = false;
              break;
            }
            const int c = k - w.t.prefix, bytes = min(kChunk, (w.t.n - c * kChunk + 15) & ~15) * D;
            const int64_t chunk = (static_cast<int64_t>(w.b) * p.Hkv + w.g) * p.pre.chunks + c;
            // (Warps 12-15 do not wait for this phase: S frees the slot, and the next one
            // may be complete first.  It is before S can be.)
            sm100::mbar_arrive(bar);
            sm100::bulk_load(sm100::smem_addr(sV + st * C::kTile), p.pre.k + (chunk * 2 + 1) * p.pre.t_rows * D, bytes,
                             sm100::smem_addr(&bars.k_full[j % KS]));
          } else {
            const int rows = min(w.t.L - k * kChunk, kChunk);
            sm100::mbar_arrive_expect_tx(bar, rows * D);
            sm100::bulk_load(sm100::smem_addr(sV + st * C::kTile), v + static_cast<int64_t>(k) * kChunk * D, rows * D, bar);
          }
          issued = j + 1;
        }
      }
      if (!ok) give_up();
      if (!ok) __nanosleep(200000);  // (a tree's keys on their way, on another barrier)
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
      const uint64_t qd0 = tile_desc<D>(sm100::smem_addr(sQ)), kd0 = tile_desc<D>(sm100::smem_addr(sK)),
                     vd0 = tile_desc<D>(sm100::smem_addr(sV));
      uint32_t item = 0, phase = 0;
      int st = 0;
      for (; ok && w.more; w = next_item(p, w), ++item) {
        const uint64_t q = qd0 + (item & 1) * (2 * C::kTile / 16);
        ok = wait(&bars.q_full[item & 1], item >> 1);
        for (int k = w.k0; ok && k < w.k1; ++k, ++j) {
          // The tile was S(j - 3)'s and then P's.
          ok = wait(&bars.k_full[st], phase) && (j < kTiles || wait(&bars.done[(j - kTiles) & 3], (j - kTiles) >> 2));
          if (!ok) break;
          sm100::tc_fence_after();
          const uint32_t d = tmem + j % kTiles * kChunk;
          const int keys = k < w.t.prefix ? w.t.L - k * kChunk : w.t.n - (k - w.t.prefix) * kChunk;
          const uint32_t idesc = sm100::idesc_e4m3_f32(kRows, 0) | static_cast<uint32_t>(min(kChunk, (keys + 15) & ~15) >> 3) << 17;
          // The queries' high and low part with the keys, of a tree with their low part too.
          const int parts = k >= w.t.prefix ? 4 : 2;
          uint32_t more = 0u;
#pragma unroll 1
          for (int part = 0; part < parts; ++part) {
            const uint64_t qd = q + (part & 1) * (C::kTile / 16);
            const uint64_t kd = part < 2 ? kd0 + st * (C::kTile / 16) : vd0 + (j % VS) * (C::kTile / 16);
#pragma unroll
            for (int kk = 0; kk < D / 32; ++kk) {
              sm100::mma_f8_ss(d, qd + kk * 2, kd + kk * 2, idesc, more);
              more = 1u;
            }
          }
          if (k >= w.t.prefix) sm100::mma_commit(sm100::smem_addr(&bars.v_free[j % VS]));
          sm100::mma_commit(sm100::smem_addr(&bars.s_full[j & 3]));
          sm100::mma_commit(sm100::smem_addr(&bars.k_free[st]));
          if (++st == KS) {
            st = 0;
            phase ^= 1u;
          }
        }
        if (ok) sm100::mma_commit(sm100::smem_addr(&bars.q_free[item & 1]));
      }
      if (!ok) give_up();
      sm100::mma_commit(sm100::smem_addr(&bars.drain[0]));
      (void)sm100::mbar_wait_bounded(sm100::smem_addr(&bars.drain[0]), 0, kDrainLimit);
    }
    __syncwarp();
  } else if (warp == kPvWarp) {
    // ------------------------------------------------------------ O += P V
    if (lane == 0) {
      bool ok = true;
      const uint64_t wd0 = sm100::smem_desc_sw128(sm100::smem_addr(sWide), C::kBlock, 1024);
      uint32_t item = 0;
      for (; ok && w.more; w = next_item(p, w), ++item) {
        for (int k = w.k0; ok && k < w.k1; ++k, ++j) {
          ok = wait(&bars.p_full[j & 3], j >> 2) && wait(&bars.wide_full[j & 1], j >> 1) &&
               (k > w.k0 || item == 0 || wait(&bars.o_free, item - 1));
          if (!ok) break;
          sm100::tc_fence_after();
          const uint32_t a = tmem + j % kTiles * kChunk;
          const uint64_t vd = wd0 + (j & 1) * (C::kWide / 16);
          const int keys = k < w.t.prefix ? w.t.L - k * kChunk : w.t.n - (k - w.t.prefix) * kChunk;
          const int steps = min(kChunk / 16, (keys + 15) / 16);
          uint32_t more = k > w.k0 ? 1u : 0u;
#pragma unroll 1
          for (int kk = 0; kk < steps; ++kk) {
            sm100::mma_bf16_ts(tmem + kOCol, a + kk * 8, vd + kk * 128, C::kIdescO, more);
            more = 1u;
          }
          sm100::mma_commit(sm100::smem_addr(&bars.done[j & 3]));
        }
      }
      if (!ok) give_up();
      sm100::mma_commit(sm100::smem_addr(&bars.drain[1]));
      (void)sm100::mbar_wait_bounded(sm100::smem_addr(&bars.drain[1]), 0, kDrainLimit);
    }
    __syncwarp();
  } else if (warp >= kConvWarp) {
    // ------------------------------------------------------------ V in fp16
    constexpr int kLanes = D / 16, kPass = kConvThreads / kLanes;  // lanes of a row, rows of a pass
    const int ct = tid - kConvWarp * 32, cl = ct % kLanes, cr = ct / kLanes;
    // Eight lanes' stores fall on all banks: where they would not, the halves of 16
    // elements are taken in the other order.  A pass further the place within the
    // swizzle's eight rows is the same.
    static_assert(kPass % 8 == 0, "the swizzle repeats");
    const int swap = cl >> 2 & 1;
    constexpr int kAtOnce = 2;
    const uint32_t from = static_cast<uint32_t>(cr * D + cl * 16);
    const uint32_t to[2] = {sw128_off(cr, 2 * cl + swap, kChunk), sw128_off(cr, 2 * cl + 1 - swap, kChunk)};
    uint32_t ended = 0, joins = 0;  // ended, bit i: chunk j - 1 - i was its item's last
    bool ok = true;
    for (; ok && w.more; w = next_item(p, w)) {
      for (int k = w.k0; k < w.k1; ++k, ++j) {
        const int st = j % VS;
        uint8_t* wide = sWide + (j & 1) * C::kWide;
        // PV(j - 2) read this tile (known complete before: PV(j - 3), and so PV(j - 6)),
        // and copies of that item's rows are joined in it.  Of V's slot the phase
        // before is known complete: chunk j - VS's product is.
        const bool tree_k = k >= w.t.prefix;
        static_assert(VS >= 2, "V's slot");
        const bool join = p.copies > 1 && (ended & 2u);
        ok = (j < 2 || wait(&bars.done[(j - 2) & 3], (j - 2) >> 2)) && (tree_k || wait(&bars.v_full[st], j / VS)) &&
             (!join || wait(&bars.join_free[joins & 1], joins >> 1));
        if (!ok && lane == 0) give_up();
        ok = !any_of<1, kConvThreads>(!ok);
        if (!ok) break;
        joins += join ? 1u : 0u;
        ended = ended << 1 | (k + 1 == w.k1 ? 1u : 0u);
        if (tree_k) {  // the tree's are prepared
          if (ct == 0) {
            await_prepared();
            const int c = k - w.t.prefix, rows = min(kChunk, (w.t.n - c * kChunk + 15) & ~15);
            const int64_t chunk = (static_cast<int64_t>(w.b) * p.Hkv + w.g) * p.pre.chunks + c;
            const uint32_t bar = sm100::smem_addr(&bars.wide_full[j & 1]);
            sm100::mbar_arrive_expect_tx(bar, rows * D * 2);
            for (int x = 0; x < D / 64; ++x)
              sm100::bulk_load(sm100::smem_addr(wide + x * C::kBlock), p.pre.v + (chunk * (D / 64) + x) * p.pre.t_rows * 8,
                               rows * 128, bar);
          } else if (lane == 0) {
            arrive(&bars.wide_full[j & 1]);
          }
          continue;
        }
        const int rows = w.t.L - k * kChunk - cr;
        const uint8_t* src = sV + st * C::kTile + from;
#pragma unroll 1
        for (int i = 0; i < kChunk / kPass; i += kAtOnce) {
          uint2 v[kAtOnce][2];
#pragma unroll
          for (int y = 0; y < kAtOnce; ++y) {
#pragma unroll
            for (int x = 0; x < 2; ++x) {
              v[y][x] = make_uint2(0u, 0u);  // (rows past the prefix: anything in the cache, zeros here)
              if ((i + y) * kPass < rows) v[y][x] = *reinterpret_cast<const uint2*>(src + (i + y) * kPass * D + 8 * (x ^ swap));
            }
          }
#pragma unroll
          for (int y = 0; y < kAtOnce; ++y) {
#pragma unroll
            for (int x = 0; x < 2; ++x)
              *reinterpret_cast<uint4*>(wide + to[x] + (i + y) * kPass * 128) =
                  make_uint4(e4m3x2_to_f16(v[y][x].x), e4m3x2_to_f16(v[y][x].x >> 16), e4m3x2_to_f16(v[y][x].y),
                             e4m3x2_to_f16(v[y][x].y >> 16));
          }
        }
        sm100::fence_proxy_async_smem();
        __syncwarp();
        if (lane == 0) arrive(&bars.wide_full[j & 1]);
        conv_sync();  // all have read the e4m3 tile
        if (ct == 0) arrive(&bars.v_free[st]);
      }
    }
    if (!ok && lane == 0) give_up();
    // (A tree's values on their way: PV, or after an abort the wait here, sees them land.)
    if (ct == 0 && j > 0)
      for (uint32_t i = j > 2 ? j - 2 : 0; i < j; ++i)
        (void)sm100::mbar_wait_bounded(sm100::smem_addr(&bars.wide_full[i & 1]), i >> 1 & 1u, kDrainLimit);
    __syncwarp();
  } else {
    // ------------------------------------------------------------ softmax
    const int grp = warp >> 2, w4 = warp & 3, lrow = w4 * 32 + lane;
    const uint32_t lanes = static_cast<uint32_t>(w4 * 32) << 16;
    const uint32_t o_col = tmem + lanes + kOCol;
    // Copy c of a row takes the quarters [c, c + 1) 4 / copies of every chunk's keys, of four.
    const int copies = p.copies, span = kRows / copies, row = lrow & (span - 1);
    const int first_quarter = lrow / span * (4 / copies), end_quarter = first_quarter + 4 / copies;
    await_prepared();
    uint32_t item = 0;
    bool ok = true;
    for (; ok && w.more; w = next_item(p, w), ++item) {
      const int par = item & 1;
      const int index = w.blk * kRows + row, node = index / p.group;
      const bool valid = node < w.t.n, active = __any_sync(adt::kFullMask, valid);
      const uint32_t j0 = j, j1 = j + static_cast<uint32_t>(w.k1 - w.k0);
      float l = 0.f, level = -INFINITY;  // sum of weights at the scores' own size: l 2^(level + kShift - kHeadroom)
      const int64_t bg = static_cast<int64_t>(w.b) * p.Hkv + w.g;
      const float scale = valid ? p.pre.q_scale[(bg * p.pre.blocks + w.blk) * p.pre.q_rows + row] : 0.f;
      if ((j0 & 1) != static_cast<uint32_t>(grp)) ++j;
      for (; j < j1; j += 2) {
        const int k = w.k0 + static_cast<int>(j - j0);
        const int slot = static_cast<int>(j % kScaleSlots);
        const bool tree_j = k >= w.t.prefix;
        uint4 seen = make_uint4(0u, 0u, 0u, 0u);
        if (tree_j && valid) seen = p.pre.seen[(static_cast<int64_t>(w.b) * p.max_nodes + node) * p.pre.chunks + k - w.t.prefix];
        if (!all_wait(&bars.s_full[j & 3], j >> 2) || !all_wait(&bars.scale_full[slot], j / kScaleSlots)) {
          ok = false;
          break;
        }
        sm100::tc_fence_after();
        const int kl = tree_j ? w.t.n - (k - w.t.prefix) * kChunk : w.t.L - k * kChunk;
        const int quarters = min(end_quarter, (kl + 31) / 32);
        const uint32_t s_col = tmem + lanes + j % kTiles * kChunk;
        if (active) {
          const ulonglong2* ks = reinterpret_cast<const ulonglong2*>(s_scale + slot * 3 * kChunk);
          const ulonglong2 *ze = ks + kChunk / 4, *iv = ze + kChunk / 4;
          const float top = s_top[slot];
          const bool masked = tree_j || kl < kChunk;
          const uint64_t scale2 = pack_f32x2(scale, scale);
          float mq[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
          // Scores times their keys' scales, with their values' exponents (z - top), back in place.
#pragma unroll 1
          for (int s = 2 * first_quarter; s < 2 * quarters; ++s) {
            uint32_t x[16];
            sm100::tmem_ld_16(s_col + 16 * s, x);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const ulonglong2 f = ks[4 * s + e], z = ze[4 * s + e];
              float a, b, c, d;
              unpack_f32x2(fma_f32x2(mul_f32x2(pack_u32x2(x[4 * e], x[4 * e + 1]), f.x), scale2, z.x), a, b);
              unpack_f32x2(fma_f32x2(mul_f32x2(pack_u32x2(x[4 * e + 2], x[4 * e + 3]), f.y), scale2, z.y), c, d);
              x[4 * e] = __float_as_uint(a);
              x[4 * e + 1] = __float_as_uint(b);
              x[4 * e + 2] = __float_as_uint(c);
              x[4 * e + 3] = __float_as_uint(d);
            }
            if (masked) {  // (after the product: -inf whatever a key and its scale are)
              const int left = kl - 16 * s, q4 = s >> 1;
              const uint32_t bits = (q4 == 0 ? seen.x : q4 == 1 ? seen.y : q4 == 2 ? seen.z : seen.w) >> (16 * (s & 1));
              const uint32_t keep = tree_j ? bits : left >= 16 ? ~0u : left > 0 ? (1u << left) - 1u : 0u;
#pragma unroll
              for (int e = 0; e < 16; ++e) x[e] = (keep >> e) & 1u ? x[e] : 0xFF800000u;
            }
#pragma unroll
            for (int e = 0; e < 16; e += 2)
              mq[(e >> 1) & 3] = fmaxf(fmaxf(mq[(e >> 1) & 3], __uint_as_float(x[e])), __uint_as_float(x[e + 1]));
            tmem_st_16(s_col + 16 * s, x);
          }
          sm100::tmem_wait_st();
          const float mx = valid ? fmaxf(fmaxf(mq[0], mq[1]), fmaxf(mq[2], mq[3])) + top : -INFINITY;
          // The running base after the chunk before (the other group's).  (An
          // item's last chunk is done before the next one's: so are its maxima.)
          float prev = -INFINITY;
          if (j > j0) {
            if (!all_wait(&bars.mu[grp ^ 1][w4], (j - 1) >> 1)) {
              ok = false;
              break;
            }
            prev = s_mu[par][lrow];
          }
          // Raised only when a row grows by more than 2^8, to a whole number, which takes
          // `top` without a rounding; then O (once the chunks before are in it) is scaled.
          const float nm = mx > prev + kRescaleThreshold ? ceilf(mx) : prev;
          s_mu[par][lrow] = nm;
          __syncwarp();
          if (lane == 0) arrive(&bars.mu[grp][w4]);
          if (j > j0 && __any_sync(adt::kFullMask, nm != prev)) {
            // (PV(j - 5), whose phase comes before, is done: S(j) is, after PV(j - 3).)
            if (!all_wait(&bars.done[(j - 1) & 3], (j - 1) >> 2)) {
              ok = false;
              break;
            }
            sm100::tc_fence_after();
            const float alpha = level_factor(prev, nm);
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
          sm100::tc_fence_after();
          const float shift = nm == -INFINITY ? 0.f : top - nm + kHeadroom;
          const uint64_t shift2 = pack_f32x2(shift, shift);
          uint64_t l2[2] = {0ull, 0ull};
          // 16 scores at a time -> 8 pairs of weights in fp16.
#pragma unroll 1
          for (int s = 2 * first_quarter; s < 2 * quarters; ++s) {
            uint32_t x[16], pk[8];
            sm100::tmem_ld_16(s_col + 16 * s, x);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const ulonglong2 g = iv[4 * s + e];
#pragma unroll
              for (int h = 0; h < 2; ++h) {
                float a, b;
                unpack_f32x2(add_f32x2(pack_u32x2(x[4 * e + 2 * h], x[4 * e + 2 * h + 1]), shift2), a, b);
                a = ex2_approx(a);
                b = ex2_approx(b);
                l2[h] = fma_f32x2(pack_f32x2(a, b), h ? g.y : g.x, l2[h]);
                pk[2 * e + h] = pack_half2(a, b);
              }
            }
            sm100::tmem_st_8(s_col + 8 * s, pk);  // over scores that have been read
          }
          if (copies > 1) {  // the weights of the other copy's keys
            const uint32_t zero[16] = {};
            tmem_st_16(s_col + (first_quarter ? 0 : 32), zero);
            tmem_st_16(s_col + (first_quarter ? 16 : 48), zero);
          }
          float la, lb, lc, ld;
          unpack_f32x2(l2[0], la, lb);
          unpack_f32x2(l2[1], lc, ld);
          // (At the larger of both levels: the base may stay while the top rises.)
          const float at = nm - top, to = fmaxf(at, level);
          l = l * level_factor(level, to) + ((la + lb) + (lc + ld)) * level_factor(at, to);
          level = to;
          sm100::tmem_wait_st();
        } else {
          // A warp without rows only keeps the barriers moving.
          if (lane == 0) arrive(&bars.mu[grp][w4]);
        }
        sm100::tc_fence_before();
        __syncwarp();
        if (lane == 0) arrive(&bars.p_full[j & 3]);
      }
      j = j1;
      // The item's O, unnormalised: group 0 takes the first half of its columns,
      // group 1 the second.  (PV(j1 - 5) is known done: this group's last S, of chunk
      // j1 - 2 at least, came after it, or the item before ended later.)
      ok = ok && all_wait(&bars.done[(j1 - 1) & 3], (j1 - 1) >> 2);
      sm100::tc_fence_after();
      constexpr int kHalf = D / 2;
      const float m = s_mu[par][lrow];
      s_l[par][grp][lrow] = make_float2(level, l);
      if (!ok && lane == 0) give_up();
      ok = !any_of<2, kSoftmaxThreads>(!ok);  // (after a wait that gave up they leave together)
      if (!ok) break;
      // A thread writes its own row's columns, or, of rows in copies, parts of row r:
      // the copies' sums, with weights that bring them to one maximum.
      const int tg = tid & 127, r = copies == 1 ? row : tg / copies;
      float M = -INFINITY, G = -INFINITY, lt = 0.f;
#pragma unroll 1
      for (int c = r; c < kRows; c += span) {
        M = fmaxf(M, s_mu[par][c]);
        G = fmaxf(G, fmaxf(s_l[par][0][c].x, s_l[par][1][c].x));
      }
#pragma unroll 1
      for (int c = r; c < kRows; c += span) {
        const float2 a = s_l[par][0][c], b = s_l[par][1][c];
        lt += a.y * level_factor(a.x, G) + b.y * level_factor(b.x, G);
      }
      float mine = 1.f;
      if (copies > 1) {
        float Mr = -INFINITY;
#pragma unroll 1
        for (int c = row; c < kRows; c += span) Mr = fmaxf(Mr, s_mu[par][c]);
        mine = level_factor(m, Mr);
      }
      // O 2^M over lt 2^(G + kShift), in two steps that stay within fp32.
      const bool whole = w.k0 == 0 && w.k1 == w.t.chunks;
      const bool lost = (s_odd[(j1 - 1) % kScaleSlots] & 2) != 0;
      const float inv = lost ? NAN : reciprocal(lt), unit = M == -INFINITY ? 1.f : half_power(M - G - kShift);
      if (copies == 1) mine = inv;
      const int64_t slot = 2ll * blockIdx.x + (w.first ? 0 : 1);
      const int ri = w.blk * kRows + r, rt = ri / p.group;
      const bool there = rt < w.t.n;
      const int64_t out_row = static_cast<int64_t>(w.t.node0 + rt) * p.H + w.g * p.group + (ri - rt * p.group);
      __nv_bfloat16* out = p.out + out_row * D + grp * kHalf;
      float4* part = p.part_o + (slot * (D / 4) + grp * (kHalf / 4)) * p.slot_rows + r;
      auto put4 = [&](int c, float4 v) {
        v = make_float4(v.x * inv * unit * unit, v.y * inv * unit * unit, v.z * inv * unit * unit, v.w * inv * unit * unit);
        if (whole) {
          uint2 y;
          y.x = pack_bf16x2(v.x, v.y);
          y.y = pack_bf16x2(v.z, v.w);
          *reinterpret_cast<uint2*>(out + c) = y;
        } else {
          part[c / 4 * p.slot_rows] = v;
        }
      };
#pragma unroll 1
      for (int c0 = 0; c0 < kHalf; c0 += 32) {
        uint32_t o[32];
        tmem_ld_32(o_col + grp * kHalf + c0, o);
        tmem_wait_ld_into(o);
        if (c0 + 32 == kHalf) {
          sm100::tc_fence_before();
          __syncwarp();
          if (lane == 0) arrive(&bars.o_free);
        }
        const float once = copies == 1 ? unit : 1.f;
#pragma unroll
        for (int c = 0; c < 32; ++c) o[c] = __float_as_uint(__uint_as_float(o[c]) * mine * once * once);
        auto four = [&](int c) {
          return make_float4(__uint_as_float(o[c]), __uint_as_float(o[c + 1]), __uint_as_float(o[c + 2]), __uint_as_float(o[c + 3]));
        };
        if (copies == 1) {
          if (there && whole) {
            uint4* dst = reinterpret_cast<uint4*>(out + c0);
#pragma unroll
            for (int c = 0; c < 32; c += 8) {
              uint32_t y[4];
#pragma unroll
              for (int e = 0; e < 4; ++e)
                y[e] = pack_bf16x2(__uint_as_float(o[c + 2 * e]), __uint_as_float(o[c + 2 * e + 1]));
              dst[c / 8] = make_uint4(y[0], y[1], y[2], y[3]);
            }
          } else if (there) {
            float4* dst = part + c0 / 4 * p.slot_rows;
#pragma unroll
            for (int c = 0; c < 8; ++c) dst[c * p.slot_rows] = four(4 * c);
          }
          continue;
        }
        // Through the V tile of the item's last chunk, which warps 12-15 leave alone
        // until then (D = 64: a buffer).
        float4* buf = reinterpret_cast<float4*>(D == 128 ? sWide + ((j1 - 1) & 1) * C::kWide : smem + C::kJoinOff) + grp * kRows * 8;
        if (c0) group_sync(grp);  // the columns before are read
#pragma unroll
        for (int c = 0; c < 8; ++c) buf[lrow * 8 + (c ^ (lrow & 7))] = four(4 * c);
        group_sync(grp);
#pragma unroll 1
        for (int c = tg & (copies - 1); there && c < 8; c += copies) {
          float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 1
          for (int x = r; x < kRows; x += span) {
            const float4 y = buf[x * 8 + (c ^ (x & 7))];
            v.x += y.x;
            v.y += y.y;
            v.z += y.z;
            v.w += y.w;
          }
          put4(c0 + 4 * c, v);
        }
      }
      if (copies > 1) {
        __syncwarp();
        if (lane == 0) arrive(&bars.join_free[item & 1]);
      }
      if (there && grp == 0 && (copies == 1 || (tg & (copies - 1)) == 0)) {
        const float at = G + (kShift - kHeadroom);
        if (!whole)
          p.part_ml[slot * p.slot_rows + r] = part_sum(at, lt);
        else if (p.lse)
          p.lse[out_row] = (at + __log2f(lt)) * kLn2;
      }
      // (The slots of an item's last two chunks, of its tree's two at most, are in
      // use until the next items' S products are read.)
      bool odd = false;
#pragma unroll 1
      for (int k = max(w.k0, w.t.prefix); k < w.k1; ++k) odd |= s_odd[(j1 - static_cast<uint32_t>(w.k1 - k)) % kScaleSlots] & 1;
      if (odd) {
        group_sync(grp);  // the rows are written
        if (there && (copies == 1 || (tg & (copies - 1)) == 0))
          add_odd(whole ? out : nullptr, reinterpret_cast<float*>(part), p.slot_rows, kHalf,
                  p.tree[1] + (static_cast<int64_t>(w.t.node0) * p.Hkv + w.g) * D + grp * kHalf, p.parents + w.t.node0,
                  static_cast<int64_t>(p.Hkv) * D, rt, (w.k0 - w.t.prefix) * kChunk, (w.k1 - w.t.prefix) * kChunk);
      }
      if (!whole) {
        // The CTAs that the item's first and last chunk lie in: share c starts at
        // the largest coordinate c X / G that is not above.
        const int64_t X = s_total, G = s_grid, a = w.start + kItemCost, z = a + w.t.chunks - 1;
        const int first = static_cast<int>(((a + 1) * G - 1) / X), last = static_cast<int>(((z + 1) * G - 1) / X);
        softmax_sync();
        if (tid == 0)
          s_last = adt::atomic_add_acq_rel_gpu(p.tickets + first, 1u) == static_cast<unsigned>(last - first);
        softmax_sync();
        if (s_last) {
          // Partial rows joined by their sums.  Neighbouring lanes
          // take neighbouring rows, a thread 16 columns at a time, of four CTAs' parts.
          constexpr int kAtOnce = 4;
          const int rows = min(w.t.n * p.group - w.blk * kRows, kRows);
          const int shift = 32 - __clz(rows - 1), jr = tid & ((1 << shift) - 1);  // (rows rounded up to a power of two)
          const int slot0 = first * 2 + (first * X / G >= w.start ? 0 : 1);
          auto slot_of = [&](int c) -> int64_t { return c == first ? slot0 : 2 * c; };
          if (jr < rows) {
            float Mj = -INFINITY;
#pragma unroll 4
            for (int c = first; c <= last; ++c) Mj = fmaxf(Mj, __ldcg(&p.part_ml[slot_of(c) * p.slot_rows + jr]).x);
            const int idx = w.blk * kRows + jr, tj = idx / p.group;
            const int64_t at = static_cast<int64_t>(w.t.node0 + tj) * p.H + w.g * p.group + idx - tj * p.group;
#pragma unroll 1
            for (int c16 = tid >> shift; c16 < D / 16; c16 += kSoftmaxThreads >> shift) {
              float lj = 0.f;
              float4 acc[4] = {};
#pragma unroll 1
              for (int c = first; c <= last; c += kAtOnce) {
                float2 ml[kAtOnce];
                float4 v[kAtOnce][4];
#pragma unroll
                for (int x = 0; x < kAtOnce; ++x) {
                  const int64_t sl = slot_of(min(c + x, last));
                  ml[x] = __ldcg(&p.part_ml[sl * p.slot_rows + jr]);
#pragma unroll
                  for (int e = 0; e < 4; ++e) v[x][e] = __ldcg(p.part_o + (sl * (D / 4) + c16 * 4 + e) * p.slot_rows + jr);
                }
#pragma unroll
                for (int x = 0; x < kAtOnce; ++x) {
                  if (c + x > last) break;
                  const float wt = level_factor(ml[x].x, Mj) * ml[x].y * kJoinScale;
                  lj += wt;
#pragma unroll
                  for (int e = 0; e < 4; ++e) {
                    acc[e].x += wt * v[x][e].x;
                    acc[e].y += wt * v[x][e].y;
                    acc[e].z += wt * v[x][e].z;
                    acc[e].w += wt * v[x][e].w;
                  }
                }
              }
              const float invj = __fdividef(1.f, lj);
              uint32_t y[8];
#pragma unroll
              for (int e = 0; e < 4; ++e) {
                y[2 * e] = pack_bf16x2(acc[e].x * invj, acc[e].y * invj);
                y[2 * e + 1] = pack_bf16x2(acc[e].z * invj, acc[e].w * invj);
              }
              uint4* dst = reinterpret_cast<uint4*>(p.out + at * D) + c16 * 2;
              dst[0] = make_uint4(y[0], y[1], y[2], y[3]);
              dst[1] = make_uint4(y[4], y[5], y[6], y[7]);
              if (c16 == 0 && p.lse) p.lse[at] = (Mj + kJoinLevel + __log2f(lj)) * kLn2;
            }
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

#include "tree_attn_q8_few.cuh"

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

int slot_rows_for(int H, int Hkv, int max_nodes) {
  const int64_t rows = static_cast<int64_t>(max_nodes) * (H / Hkv);
  return rows < kRows ? static_cast<int>(rows) : kRows;
}

// Tickets at the start, for any grid; two items' partial rows of each CTA; what is
// prepared where the items have more than 16 rows.  (Offsets from `base`, which may be NULL; at most 2^24 query rows, so
// that all sizes stay below 2^50.)
size_t ws_layout(uint8_t* base, int grid, int B, int H, int Hkv, int D, int max_nodes, AttnParams* p) {
  const int rows = slot_rows_for(H, Hkv, max_nodes);
  size_t at = kMaxGrid * sizeof(unsigned);
  auto take = [&](size_t bytes) {
    uint8_t* x = base + at;
    at = adt::align_up(at + bytes, 256);
    return x;
  };
  Prepared& w = p->pre;
  w.q_rows = (rows + 7) & ~7;
  w.blocks = static_cast<int>((static_cast<int64_t>(max_nodes) * (H / Hkv) + kRows - 1) / kRows);
  w.t_rows = max_nodes < kChunk ? (max_nodes + 15) & ~15 : kChunk;
  w.chunks = (max_nodes + kChunk - 1) / kChunk;
  const size_t bg = static_cast<size_t>(B) * Hkv, slots = 2 * static_cast<size_t>(grid) * rows;
  p->slot_rows = rows;
  p->copies = rows <= 64 ? 2 : 1;
  p->tickets = reinterpret_cast<unsigned*>(base);
  p->part_ml = reinterpret_cast<float2*>(take(slots * sizeof(float2)));
  p->part_o = reinterpret_cast<float4*>(take(slots * D * sizeof(float)));
  if (rows <= kFewRows) return at;
  w.q = take(bg * w.blocks * 2 * w.q_rows * D);
  w.q_scale = reinterpret_cast<float*>(take(bg * w.blocks * w.q_rows * sizeof(float)));
  w.k = take(bg * w.chunks * 2 * w.t_rows * D);
  w.v = reinterpret_cast<uint4*>(take(bg * w.chunks * w.t_rows * D * 2));
  w.scale = take(bg * w.chunks * 3 * w.t_rows);
  w.seen = reinterpret_cast<uint4*>(take(static_cast<size_t>(B) * max_nodes * w.chunks * sizeof(uint4)));
  return at;
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

template <int D>
adt_status launch(const AttnParams& p, const CUtensorMap& tm, const CUtensorMap& tm_v, int grid, int dev, cudaStream_t st) {
  static unsigned configured[2] = {0u, 0u};  // bit per device (< 64), per instantiation
  const unsigned bit = 1u << (dev & 31);
  unsigned& word = configured[(dev >> 5) & 1];
  if (!(__atomic_load_n(&word, __ATOMIC_ACQUIRE) & bit)) {
    ADT_CUDA_TRY(cudaFuncSetAttribute(tree_attn_q8_kernel<D>, cudaFuncAttributeMaxDynamicSharedMemorySize, Cfg<D>::kDynSmem));
    ADT_CUDA_TRY(cudaFuncSetAttribute(tree_attn_q8_few_kernel<D>, cudaFuncAttributeMaxDynamicSharedMemorySize, FewCfg<D>::kDynSmem));
    __atomic_fetch_or(&word, bit, __ATOMIC_ACQ_REL);
  }
  cudaLaunchConfig_t cfg = {};
  cudaLaunchAttribute attr[1] = {adt::pdl_attribute()};
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  cfg.stream = st;
  if (p.max_nodes * p.group <= kFewRows) {
    cfg.gridDim = dim3(static_cast<unsigned>(grid), 1, 1);
    cfg.blockDim = dim3(kThreads, 1, 1);
    cfg.dynamicSmemBytes = FewCfg<D>::kDynSmem;
    ADT_CUDA_TRY(cudaLaunchKernelEx(&cfg, tree_attn_q8_few_kernel<D>, tm, tm_v, p));
    return adt::launch_status();
  }
  constexpr int kPass = kPrepThreads / (D / 16);
  const int64_t units = static_cast<int64_t>(p.max_nodes) * p.H + ((p.max_nodes + 15) & ~15) * static_cast<int64_t>(p.Hkv);
  cfg.gridDim = dim3(static_cast<unsigned>((units + kPass - 1) / kPass), static_cast<unsigned>(p.B), 1);
  cfg.blockDim = dim3(kPrepThreads, 1, 1);
  ADT_CUDA_TRY(cudaLaunchKernelEx(&cfg, prepare_kernel<D>, p));
  cfg.gridDim = dim3(static_cast<unsigned>(grid), 1, 1);
  cfg.blockDim = dim3(kThreads, 1, 1);
  cfg.dynamicSmemBytes = Cfg<D>::kDynSmem;
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
  AttnParams p{};
  return ws_layout(nullptr, grid_for(info.sm_count, B, H, Hkv, max_nodes, max_kv), B, H, Hkv, D, max_nodes, &p);
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
  const int grid = grid_for(info.sm_count, B, H, Hkv, max_nodes, max_kv);
  AttnParams p{};
  const size_t bytes = ws_layout(static_cast<uint8_t*>(workspace), grid, B, H, Hkv, D, max_nodes, &p);
  if (!workspace || workspace_bytes < bytes || !adt::aligned16(workspace)) return ADT_ERR_WORKSPACE;
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
  p.wait_limit = adt::wait_limit(kWaitLimit);
  CUtensorMap tm, tm_v;
  st = make_cache_map(&tm, k_cache, D, max_kv, Hkv, B, cache_stride_h, cache_stride_b);
  if (st == ADT_OK) st = make_cache_map(&tm_v, v_cache, D, max_kv, Hkv, B, cache_stride_h, cache_stride_b);
  if (st != ADT_OK) return st;
  return D == 128 ? launch<128>(p, tm, tm_v, grid, info.device, adt::as_stream(stream))
                  : launch<64>(p, tm, tm_v, grid, info.device, adt::as_stream(stream));
}

}  // extern "C"
