// adt_tree_attn_q8 of few query rows (up to 16 of a tree and kv head: single tokens
// with grouped heads, small trees).  Included by tree_attn_q8.cu, which holds the
// kernel of 128 rows and what both share.
//
// Products with the keys as the 128 rows of a tile: S^T = K Q^T, O^T = V^T P^T,
// both of e4m3 operands as they lie in the cache; 16 columns instead of 128 rows that
// few queries would leave empty, and no copy of V in a wider type.  A thread owns a
// key: its scales are its own registers' and its weights a row of P^T.
//
// Weights meet V in four e4m3 numbers, 2^-4 apart: p = p1 + p2 / 16 + p3 / 256 + p4 / 4096,
// each what the ones before leave, with an accumulator each (columns of one product).
// Three hold all of a weight's bits, but end at 2^-22 of the largest one (times value
// scale), and a cache of 30000 rows can have 0.7 % of its sum below; four end at 2^-26.
//
// A weight takes on its value's scale 2^ev in the exponent: 2^(x c + ev - base), x c
// the score, base the largest such exponent so far (raised only when a row grows by
// more than 2^kFewThreshold).  A value whose scale is below 2^-kSpan of the largest so
// far, 2^top (a row of zeros has the least there is), adds nothing to O, and its weight is
// made as if it were 2^-kSpan there, so that its part of the row sum is neither lost nor
// too large.  The row sum adds weights times 2^(from - ev - kFewShift): `from` is the first
// chunk's top, and follows the top 2^kFewLag below (where the top rises for a key that
// means nothing to a row, the row's base stays, and its sum grows by what `from` does).
//
// Warp roles: 0-3, 4-7 two softmax groups that take the chunks in turn; 8 K tiles, 9 V
// tiles; 10 S products; 11 PV products; 12-15 an item's start and end beside the
// chunks of the items around it: queries and, with the tree's chunk, its rows cut
// into e4m3 rows (keys into two as the queries; values into three 2^-4 apart, which hold
// each element to 2^-8 of it or 2^-27 of the row's largest), and O, which has a place for two items, read
// out and joined.
//
// Bound by HBM where caches are long: 16 sequences of 1 to 30011 rows, 32 / 8 heads x
// 128 (353 MB) 75 us, 70 % of a copy's rate; about 15 us are the shares' calculation, the
// first tiles' way and the last one's.  Short ones are a chain of waits: one sequence of
// 512 rows, 8 heads x 64, 11.5 us.
//
// The rule, 16 rows: this kernel against that of 128 rows, us, D = 64 and 128.  Four trees
// over 2400 rows, 16 / 16 heads: of 1 node 19.8 and 20.8 (27 and 29), of 16 nodes 24.2 and
// 28.8 (27.3 and 30.3).  Eight tokens over 8000 rows, 16 query heads to each of 8 kv heads:
// 36.6 and 41.5 (49.4 and 51.6).  With 32 columns it takes for trees of 17 nodes 28.9 and
// 33.7 (28.0 and 31.4), of 32 nodes 33.5 and 41.5 (28.0 and 31.7), one of 26 nodes over 512
// rows, 8 heads x 64, 19.2 (12.9); of 20 heads to a kv head 47.1 and 51.6 (49.4 and 51.9).
constexpr int kFewRows = 16;
constexpr int kTreeRows = 32;  // of a tree's tiles: keys of a product
constexpr float kFewThreshold = 4.5f, kFewHeadroom = 4.f;  // weights up to 2^8.5: e4m3 ends at 448
constexpr int kFewShift = 8, kFewLag = 80;  // row sums from 2^-84 to 2^97 a key: within fp32, their least parts too
constexpr float kUnset = -3e38f;  // the base of a row that has seen no key
constexpr int kNoScale = -1000;   // (scales are 2^-127 and more)
constexpr int kLeastScale = -127;

template <int D>
struct FewCfg {
  static constexpr int kStages = D == 128 ? 4 : 8;
  static constexpr int kTile = kChunk * D;
  static constexpr int kQ = kFewRows * D;                      // queries, high or low part
  static constexpr int kSmall = kTreeRows * D;          // a tree's keys or values, a part
  static constexpr int kQOff = 0;                       // [2 items][high, low]
  static constexpr int kTreeOff = kQOff + 4 * kQ;       // [2 items][K high, K low, V in three]
  static constexpr int kTreeBytes = 5 * kSmall;
  // Weights [128 keys][p1, p2, p3, p4: kFewRows each], the swizzle as wide as a row.
  // Two tiles a group: PV(j) is done 2000 cycles after P(j) is written.
  static constexpr int kPTiles = 4;
  static constexpr int kPBytes = kChunk * 4 * kFewRows;
  static constexpr int kPOff = kTreeOff + 2 * kTreeBytes;
  static constexpr int kKOff = kPOff + kPTiles * kPBytes;
  static constexpr int kVOff = kKOff + kStages * kTile;
  static constexpr int kDynSmem = kVOff + kStages * kTile + 1024;  // + alignment slack
  static constexpr uint32_t kIdescO = sm100::idesc_e4m3_f32(D, 4 * kFewRows) | 1u << 15 | 1u << 16;  // both MN-major
  // Tensor memory: four S tiles of kFewRows columns, O of two items (4 kFewRows), row sums [2 items][2 groups] of kFewRows.
  static constexpr uint32_t kOAt = 4 * kFewRows, kLAt = 12 * kFewRows;
  static constexpr uint32_t kCols = 16 * kFewRows;
};

struct FewBars {
  uint64_t k_full[8], k_free[8], v_full[8], v_free[8], v_tail;
  uint64_t prep_full[2], prep_free[2];
  uint64_t s_full[4], s_free[4], p_full[4], done[4], mu[2];
  uint64_t drain[2];
};

__device__ __forceinline__ uint16_t f16x2_to_e4m3(uint32_t h) {
  uint16_t r;
  asm("cvt.rn.satfinite.e4m3x2.f16x2 %0, %1;\n" : "=h"(r) : "r"(h));
  return r;
}
// (h - the e4m3 numbers in e) * 16, exact.
__device__ __forceinline__ uint32_t rest16(uint32_t h, uint16_t e) {
  const uint32_t b = e4m3x2_to_f16(e);
  const __half2 d = __hmul2(__hsub2(*reinterpret_cast<const __half2*>(&h), *reinterpret_cast<const __half2*>(&b)),
                            __float2half2_rn(16.f));
  return *reinterpret_cast<const uint32_t*>(&d);
}

// Sums of 16 values over the warp's lanes: lane l gets that of value l / 2.
__device__ __forceinline__ float transposed_sum(float (&v)[16], int lane) {
#pragma unroll
  for (int n = 8, o = 16; n >= 1; n >>= 1, o >>= 1) {
    const bool up = lane & o;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      if (i >= n) break;
      const float send = up ? v[i] : v[i + n], keep = up ? v[i + n] : v[i];
      v[i] = keep + __shfl_xor_sync(adt::kFullMask, send, o);
    }
  }
  return v[0] + __shfl_xor_sync(adt::kFullMask, v[0], 1);
}

// The largest of a warp's values; NaN counts as none.
__device__ __forceinline__ float warp_most(float v) {
  float r;
  asm("redux.sync.max.f32 %0, %1, 0xffffffff;\n" : "=f"(r) : "f"(v));
  return r;
}

template <int D>
__global__ void __launch_bounds__(kThreads, 1)
    tree_attn_q8_few_kernel(const __grid_constant__ CUtensorMap tm_k, const __grid_constant__ CUtensorMap tm_v,
                            const __grid_constant__ AttnParams p) {
  using C = FewCfg<D>;
  constexpr int NS = C::kStages, PT = C::kPTiles;
  extern __shared__ __align__(1024) uint8_t smem_raw[];
  uint8_t* smem = smem_raw + ((1024u - (sm100::smem_addr(smem_raw) & 1023u)) & 1023u);
  __shared__ FewBars bars;
  // Of an item's rows (and its tree's keys), by item.
  __shared__ __align__(16) float s_c[2][kFewRows], s_base[2][kFewRows];
  __shared__ float s_tk[2][kFewRows];
  __shared__ int s_tv[2][kFewRows], s_top[2], s_from[2], s_ver[2], s_odd[2];
  __shared__ uint32_t s_seen[2][kFewRows];                    // of a key: the rows that see it
  __shared__ __align__(16) float s_gb[2][2][kFewRows], s_alpha[2][kFewRows];  // of a group: the level its row sums are at
  __shared__ float s_most[2][4][kFewRows];
  __shared__ int s_wtop[2][4];
  __shared__ __align__(16) float s_sum[kFewRows][4];          // of a row: the warps' parts
  __shared__ int16_t s_par[kFewRows];
  __shared__ Walk s_walk;
  __shared__ int64_t s_total;
  __shared__ int s_grid;
  __shared__ uint32_t tmem_slot;
  __shared__ volatile int s_abort;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;

  if (tid == 0) {
    s_abort = 0;
    auto init = [](uint64_t* bar, int n, uint32_t count) {
      for (int i = 0; i < n; ++i) sm100::mbar_init(sm100::smem_addr(bar + i), count);
    };
    init(bars.k_full, 8, 1);
    init(bars.k_free, 8, 1);
    init(bars.v_full, 8, 1);
    init(bars.v_free, 8, 1);
    init(&bars.v_tail, 1, 1);
    init(bars.prep_full, 2, 4);
    init(bars.prep_free, 2, 1);
    init(bars.s_full, 4, 1);
    init(bars.s_free, 4, 4);
    init(bars.p_full, 4, 4);
    init(bars.mu, 2, 1);
    init(bars.done, 4, 1);
    init(bars.drain, 2, 1);
    sm100::fence_mbar_init();
  }
  if (warp == kPvWarp) {
    sm100::tmem_alloc(sm100::smem_addr(&tmem_slot), C::kCols);
    sm100::tmem_relinquish();
  }
  if (warp == kKWarp && lane < 2) sm100::prefetch_tensormap(lane ? &tm_v : &tm_k);
  asm volatile("griddepcontrol.wait;\n" ::: "memory");
  if (warp == 0) find_share(p, lane, &s_walk, &s_total, &s_grid, blockIdx.x == 0 ? p.err : nullptr);
  sm100::tc_fence_before();
  __syncthreads();
  sm100::tc_fence_after();
  const uint32_t tmem = tmem_slot;
  Walk w = s_walk;
  if (!w.some()) {
    __syncthreads();
    if (warp == kPvWarp) sm100::tmem_dealloc(tmem, C::kCols);
    return;
  }
  uint8_t* sQ = smem + C::kQOff;
  uint8_t* sT = smem + C::kTreeOff;
  uint8_t* sP = smem + C::kPOff;
  uint8_t* sK = smem + C::kKOff;
  uint8_t* sV = smem + C::kVOff;
  auto wait = [&](uint64_t* bar, uint32_t phase) { return poll(bar, phase & 1u, &s_abort, p.wait_limit); };
  auto all_wait = [&](uint64_t* bar, uint32_t phase) { return __all_sync(adt::kFullMask, wait(bar, phase)); };
  auto arrive = [&](uint64_t* bar) { sm100::mbar_arrive(sm100::smem_addr(bar)); };
  auto give_up = [&]() {
    s_abort = 1;
    adt::raise_error(p.err, ADT_DEVERR_TIMEOUT);
  };
  // Chunk j (over the whole share) is softmax group j % 2's, its scores in S tile j % 4;
  // of the prefix's chunks, i in all, tile i has slot i % NS of both rings.  (A wait on a parity is only
  // meaningful to a thread that knows the phase before complete.)
  uint32_t j = 0, i = 0, item = 0;

  if (warp == kKWarp) {
    // ------------------------------------------------------------ K tiles
    if (lane == 0) {
      bool ok = true;
      for (; ok && w.more; w = next_item(p, w)) {
        const int end = min(w.k1, w.t.prefix);
        for (int k = w.k0; k < end; ++k, ++i) {
          const int st = i % NS;
          if (i >= NS && !wait(&bars.k_free[st], i / NS - 1)) {
            ok = false;
            break;
          }
          const uint32_t bar = sm100::smem_addr(&bars.k_full[st]);
          sm100::mbar_arrive_expect_tx(bar, C::kTile);
          sm100::tma_load_4d(sm100::smem_addr(sK + st * C::kTile), &tm_k, 0, k * kChunk, w.g, w.b, bar);
        }
      }
      if (!ok) give_up();
      asm volatile("griddepcontrol.launch_dependents;\n" ::: "memory");
      // Every copy issued lands before the CTA goes on (also after an abort).
      for (uint32_t x = i > NS ? i - NS : 0; x < i; ++x)
        (void)sm100::mbar_wait_bounded(sm100::smem_addr(&bars.k_full[x % NS]), x / NS & 1u, kDrainLimit);
    }
    __syncwarp();
  } else if (warp == kVWarp) {
    // ------------------------------------------------------------ V tiles
    bool ok = true;
    uint32_t tails = 0, full = 0;  // full: one past the last tile that landed or lands on v_full
    for (; ok && w.more; w = next_item(p, w)) {
      const int end = min(w.k1, w.t.prefix);
      for (int k = w.k0; k < end; ++k, ++i) {
        const int st = i % NS, rows = w.t.L - k * kChunk;
        if (i >= NS) ok = all_wait(&bars.v_free[st], i / NS - 1);
        if (!ok) break;
        // Of the last tile the rows past the prefix hold anything, NaN among it, and
        // meet weights of zero: zeros, as far as a product reads (32 keys).
        const bool tail = rows < kChunk && (rows & 31) != 0;
        if (lane == 0) {
          const uint32_t bar = sm100::smem_addr(tail ? &bars.v_tail : &bars.v_full[st]);
          sm100::mbar_arrive_expect_tx(bar, C::kTile);
          sm100::tma_load_4d(sm100::smem_addr(sV + st * C::kTile), &tm_v, 0, k * kChunk, w.g, w.b, bar);
        }
        if (tail) {
          // (This copy has landed before the warp goes on, whatever happens elsewhere.)
          const bool landed = sm100::mbar_wait_bounded(sm100::smem_addr(&bars.v_tail), tails & 1u, kDrainLimit);
          ++tails;
          ok = __all_sync(adt::kFullMask, landed);
          if (!ok) break;
          uint4* z = reinterpret_cast<uint4*>(sV + st * C::kTile + rows * D);
          for (int x = lane; x < (32 - (rows & 31)) * (D / 16); x += 32) z[x] = make_uint4(0u, 0u, 0u, 0u);
          sm100::fence_proxy_async_smem();
          __syncwarp();
          if (lane == 0) arrive(&bars.v_full[st]);
        }
        full = i + 1;
      }
    }
    if (!ok && lane == 0) give_up();
    if (lane == 0)
      for (uint32_t x = full > NS ? full - NS : 0; x < full; ++x)
        (void)sm100::mbar_wait_bounded(sm100::smem_addr(&bars.v_full[x % NS]), x / NS & 1u, kDrainLimit);
    __syncwarp();
  } else if (warp == kSWarp) {
    // ------------------------------------------------------------ S^T = K Q^T
    if (lane == 0) {
      bool ok = true;
      const uint64_t qd0 = tile_desc<D>(sm100::smem_addr(sQ)), kd0 = tile_desc<D>(sm100::smem_addr(sK)),
                     td0 = tile_desc<D>(sm100::smem_addr(sT));
      for (; ok && w.more; w = next_item(p, w), ++item) {
        const uint32_t idesc = sm100::idesc_e4m3_f32(kChunk, kFewRows);
        ok = wait(&bars.prep_full[item & 1], item >> 1);
        for (int k = w.k0; ok && k < w.k1; ++k, ++j) {
          const bool tree_k = k >= w.t.prefix;
          const int st = i % NS;
          ok = (tree_k || wait(&bars.k_full[st], i / NS)) && (j < 4 || wait(&bars.s_free[j & 3], (j >> 2) - 1));
          if (!ok) break;
          sm100::tc_fence_after();
          // The queries' high and low part with the keys, of a tree with their low part too.
          // (A tree's tile is 128 rows from its 32 on, up to the weights at most: scores of
          // keys that there are not, which no row sees.)
          const int parts = tree_k ? 4 : 2;
          uint32_t more = 0u;
#pragma unroll 1
          for (int part = 0; part < parts; ++part) {
            const uint64_t qd = qd0 + ((item & 1) * 2 + (part & 1)) * (C::kQ / 16);
            const uint64_t kd = tree_k ? td0 + ((item & 1) * C::kTreeBytes + (part >> 1) * C::kSmall) / 16 : kd0 + st * (C::kTile / 16);
#pragma unroll
            for (int kk = 0; kk < D / 32; ++kk) {
              sm100::mma_f8_ss(tmem + (j & 3) * kFewRows, kd + kk * 2, qd + kk * 2, idesc, more);
              more = 1u;
            }
          }
          sm100::mma_commit(sm100::smem_addr(&bars.s_full[j & 3]));
          if (!tree_k) {
            sm100::mma_commit(sm100::smem_addr(&bars.k_free[st]));
            ++i;
          }
        }
      }
      if (!ok) give_up();
      sm100::mma_commit(sm100::smem_addr(&bars.drain[0]));
      (void)sm100::mbar_wait_bounded(sm100::smem_addr(&bars.drain[0]), 0, kDrainLimit);
    }
    __syncwarp();
  } else if (warp == kPvWarp) {
    // ------------------------------------------------------------ O^T += V^T P^T
    if (lane == 0) {
      bool ok = true;
      // (MN-major: columns of 8 keys 1024 bytes apart, at D = 64 512.)
      const uint64_t vd0 = tile_desc<D>(sm100::smem_addr(sV)), td0 = tile_desc<D>(sm100::smem_addr(sT)),
                     pd0 = tile_desc<4 * kFewRows>(sm100::smem_addr(sP));
      for (; ok && w.more; w = next_item(p, w), ++item) {
        for (int k = w.k0; ok && k < w.k1; ++k, ++j) {
          const bool tree_k = k >= w.t.prefix;
          const int st = i % NS;
          ok = wait(&bars.p_full[j & 3], j >> 2) && (tree_k || wait(&bars.v_full[st], i / NS));
          if (!ok) break;
          sm100::tc_fence_after();
          const uint64_t pd = pd0 + (j % PT) * (C::kPBytes / 16);
          const int steps = tree_k ? 3 : min(4, (w.t.L - k * kChunk + 31) / 32);
          uint32_t more = k > w.k0 ? 1u : 0u;
#pragma unroll 1
          for (int kk = 0; kk < steps; ++kk) {
            // Part kk of a tree's values is 2^-4kk of what it says: with p1 it belongs to
            // the accumulator of p's part kk, with p2 to the next.
            const uint64_t vd = (tree_k ? td0 + ((item & 1) * C::kTreeBytes + (2 + kk) * C::kSmall) / 16
                                        : vd0 + (st * C::kTile + kk * 32 * D) / 16);
            const int part = tree_k ? kk : 0;
            sm100::mma_f8_ss(tmem + C::kOAt + ((item & 1) * 4 + part) * kFewRows, vd, pd + (kk - part) * (32 * 4 * kFewRows / 16),
                             C::kIdescO - (static_cast<uint32_t>(part * kFewRows >> 3) << 17), more);
            more = 1u;
          }
          sm100::mma_commit(sm100::smem_addr(&bars.done[j & 3]));
          if (!tree_k) {
            sm100::mma_commit(sm100::smem_addr(&bars.v_free[st]));
            ++i;
          }
        }
        if (ok) sm100::mma_commit(sm100::smem_addr(&bars.prep_free[item & 1]));
      }
      if (!ok) give_up();
      sm100::mma_commit(sm100::smem_addr(&bars.drain[1]));
      (void)sm100::mbar_wait_bounded(sm100::smem_addr(&bars.drain[1]), 0, kDrainLimit);
    }
    __syncwarp();
  } else if (warp >= kConvWarp) {
    // ------------------------------------------------------------ an item's start and end
    // A row is D / 16 lanes', 16 elements each: the item's queries, then the tree's keys
    // and values.  One copy of the code for all, and what there is to read in flight
    // before: an item's first product waits for this.
    constexpr int kLanes = D / 16, kPass = kConvThreads / kLanes;
    const int ct = tid - kConvWarp * 32, cl = ct % kLanes, cr = ct / kLanes;
    bool ok = true;
    // (All threads are past the end of the item before the last, and so are all others.)
    auto prepare = [&]() {
      const int at = item & 1, rows = w.t.n * p.group, n = w.t.n;
      uint8_t* q = sQ + (item & 1) * 2 * C::kQ;
      uint8_t* t = sT + (item & 1) * C::kTreeBytes;
      const bool tree = w.k1 > w.t.prefix;
      const int units = tree ? rows + 2 * n : rows;
      uint4 x[2];
      int up = -1;
      auto fetch = [&](int u) {
        x[0] = x[1] = make_uint4(0u, 0u, 0u, 0u);
        if (u >= units) return;
        const __nv_bfloat16* src;
        if (u < rows) {
          const int node = u / p.group;
          src = p.q + (static_cast<int64_t>(w.t.node0 + node) * p.H + w.g * p.group + (u - node * p.group)) * D;
        } else {
          const int v = u - rows >= n;
          src = p.tree[v] + (static_cast<int64_t>(w.t.node0 + u - rows - v * n) * p.Hkv + w.g) * D;
        }
        x[0] = reinterpret_cast<const uint4*>(src)[cl * 2];
        x[1] = reinterpret_cast<const uint4*>(src)[cl * 2 + 1];
      };
      fetch(cr);
      if (tree && ct < n) up = p.parents[w.t.node0 + ct];
      any_of<1, kConvThreads>(false);
      if (ct < kFewRows) s_base[at][ct] = kUnset;
      if (tree && ct < n) {
        s_par[ct] = static_cast<int16_t>(min(max(up, -1), kMaxTreeNodes));
        if ((ct == 0) != (up < 0) || up >= ct) adt::raise_error(p.err, ADT_DEVERR_BAD_TREE);
      }
      if (ct == 0) {
        s_odd[at] = s_ver[at] = 0;
        s_top[at] = kNoScale;
      }
      any_of<1, kConvThreads>(false);
#pragma unroll 1
      for (int u = cr; u - cr < units; u += kPass) {
        const bool is_q = u < rows, is_v = u >= rows + n;
        // Values that are not finite as zeros: see add_odd.
        if (is_v) {
          uint32_t y[8] = {x[0].x, x[0].y, x[0].z, x[0].w, x[1].x, x[1].y, x[1].z, x[1].w};
          bool odd = false;
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const bool lo = (y[e] & 0x7f80u) == 0x7f80u, hi = (y[e] & 0x7f800000u) == 0x7f800000u;
            odd |= lo || hi;
            if (lo) y[e] &= 0xffff0000u;
            if (hi) y[e] &= 0xffffu;
          }
          if (odd) s_odd[at] = 1;
          x[0] = make_uint4(y[0], y[1], y[2], y[3]);
          x[1] = make_uint4(y[4], y[5], y[6], y[7]);
        }
        uint4 cut[3];
        const uint32_t s = cut_row<D>(x, is_v ? 16.f : 1.f, cut);
        fetch(u + kPass);
        if (u >= units) continue;
        const int r = is_q ? u : u - rows - (is_v ? n : 0);
        uint8_t* dst = (is_q ? q : t + (is_v ? 2 * C::kSmall : 0)) + tile_off<D>(r, cl);
        const int step = is_q ? C::kQ : C::kSmall;
        *reinterpret_cast<uint4*>(dst) = cut[0];
        *reinterpret_cast<uint4*>(dst + step) = cut[1];
        if (is_v) *reinterpret_cast<uint4*>(dst + 2 * step) = cut[2];
        if (cl != 0) continue;
        if (is_q)
          s_c[at][r] = row_factor(s, p.scale_log2);
        else if (is_v)
          s_tv[at][r] = static_cast<int>(s) - 127;
        else
          s_tk[at][r] = __uint_as_float(s << 23);
      }
      // Zeros: the queries up to kFewRows (their scores are read), values up to the 32 that a product reads.
#pragma unroll 1
      for (int i = rows * D / 16 + ct; i < kFewRows * D / 16; i += kConvThreads) {
        reinterpret_cast<uint4*>(q)[i] = reinterpret_cast<uint4*>(q + C::kQ)[i] = make_uint4(0u, 0u, 0u, 0u);
        if (i % (D / 16) == 0) s_c[at][i / (D / 16)] = 1.f;
      }
      if (tree) {
#pragma unroll 1
        for (int i = n * D / 16 + ct; i < kTreeRows * D / 16; i += kConvThreads) {
          uint4* v = reinterpret_cast<uint4*>(t + 2 * C::kSmall) + i;
          v[0] = v[C::kSmall / 16] = v[2 * C::kSmall / 16] = make_uint4(0u, 0u, 0u, 0u);
        }
      }
      if (tree && warp == kConvWarp) {
        // Row by row the keys seen, then key by key the rows that see it.
        uint32_t m = 0u;
        if (lane < rows) {
          for (int x = lane / p.group;;) {
            m |= 1u << x;
            const int up = s_par[x];
            if (up < 0 || up >= x) break;
            x = up;
          }
        }
        uint32_t mine = 0u;
#pragma unroll 1
        for (int x = 0; x < n; ++x) {
          const uint32_t b = __ballot_sync(adt::kFullMask, m >> x & 1u);
          if (x == lane) mine = b;
        }
        if (lane < n) s_seen[at][lane] = mine;
      }
      sm100::fence_proxy_async_smem();
      __syncwarp();
      if (lane == 0) arrive(&bars.prep_full[item & 1]);
    };
    // An item's rows, once its products are done: final ones, or this CTA's part.
    auto finish = [&](const Walk& w, uint32_t item, uint32_t j0) {
      ok = wait(&bars.prep_free[item & 1], item >> 1);
      if (!ok && lane == 0) give_up();
      ok = !any_of<1, kConvThreads>(!ok);
      if (!ok) return;
      sm100::tc_fence_after();
      const int at = item & 1, rows = w.t.n * p.group, w4 = warp & 3, from = s_from[at];
      const uint32_t lanes = static_cast<uint32_t>(w4 * 32) << 16;
      // Row sums over the keys' lanes, at the bases' last level; of a group that had a chunk.
#pragma unroll 1
      for (int blk = 0; blk < kFewRows / 16; ++blk) {
        float v[16] = {};
#pragma unroll 1
        for (int g = 0; g < 2; ++g) {
          if (w.k1 - w.k0 < 2 && (j0 & 1) != static_cast<uint32_t>(g)) continue;
          uint32_t r[16];
          sm100::tmem_ld_16(tmem + lanes + C::kLAt + (at * 2 + g) * kFewRows + 16 * blk, r);
#pragma unroll
          for (int e = 0; e < 16; ++e)
            v[e] = fmaf(__uint_as_float(r[e]), ex2_approx(s_gb[at][g][16 * blk + e] - (s_base[at][16 * blk + e] - from)), v[e]);
        }
        const float sum = transposed_sum(v, lane);
        if ((lane & 1) == 0) s_sum[16 * blk + (lane >> 1)][w4] = sum;
      }
      any_of<1, kConvThreads>(false);
      const bool whole = w.k0 == 0 && w.k1 == w.t.chunks;
      const int64_t slot = (2ll * blockIdx.x + (w.first ? 0 : 1)) * p.slot_rows;
      const int d = D == 128 ? ct : w4 * 16 + lane;
      auto out_row_of = [&](int r) {
        const int node = r / p.group;
        return static_cast<int64_t>(w.t.node0 + node) * p.H + w.g * p.group + (r - node * p.group);
      };
      float* part = reinterpret_cast<float*>(p.part_o) + slot * D;
      auto row_sum = [&](int r) {
        const float4 a = *reinterpret_cast<const float4*>(s_sum[r]);
        return (a.x + a.y) + (a.z + a.w);
      };
      // O, columns back to rows, over the row sum and at its size, in two steps that stay within fp32.
      const float unit = half_power(from - kFewShift);
#pragma unroll 1
      for (int r0 = 0; r0 < rows; r0 += 8) {
        uint32_t o[4][8];
#pragma unroll
        for (int x = 0; x < 4; ++x) sm100::tmem_ld_8(tmem + lanes + C::kOAt + (at * 4 + x) * kFewRows + r0, o[x]);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const int r = r0 + e;
          if (r >= rows || (D == 64 && lane >= 16)) break;
          float v = __uint_as_float(o[3][e]);
#pragma unroll
          for (int x = 2; x >= 0; --x) v = fmaf(v, 0.0625f, __uint_as_float(o[x][e]));
          v = v * reciprocal(row_sum(r)) * unit * unit;
          if (whole)
            p.out[out_row_of(r) * D + d] = __float2bfloat16(v);
          else
            part[r * D + d] = v;
        }
        __syncwarp();
      }
      sm100::tc_fence_before();
      if (ct < rows) {
        const float l = row_sum(ct), m = s_base[at][ct] - from + (kFewShift - kFewHeadroom);
        if (!whole)
          p.part_ml[slot + ct] = part_sum(m, l);
        else if (p.lse)
          p.lse[out_row_of(ct)] = (m + __log2f(l)) * kLn2;
      }
      if (s_odd[at] != 0 && w.k1 > w.t.prefix) {
        any_of<1, kConvThreads>(false);  // the rows are written
        if (ct < rows)
          add_odd(whole ? p.out + out_row_of(ct) * D : nullptr, part + ct * D, 1, D,
                  p.tree[1] + (static_cast<int64_t>(w.t.node0) * p.Hkv + w.g) * D, p.parents + w.t.node0,
                  static_cast<int64_t>(p.Hkv) * D, ct / p.group, 0, w.t.n);
      }
      if (whole) return;
      // The parts joined by the CTA that ends its own last, beside the next item's
      // chunks, by their sums.
      any_of<1, kConvThreads>(false);
      // (Which CTAs these are: as in the kernel of 128 rows.)
      const int64_t X = s_total, G = s_grid, a = w.start + kItemCost, z = a + w.t.chunks - 1;
      const int first = static_cast<int>(((a + 1) * G - 1) / X), last = static_cast<int>(((z + 1) * G - 1) / X);
      const bool mine = ct == 0 && adt::atomic_add_acq_rel_gpu(p.tickets + first, 1u) == static_cast<unsigned>(last - first);
      if (!any_of<1, kConvThreads>(mine)) return;
      const int slot0 = first * 2 + (first * X / G >= w.start ? 0 : 1);
      auto slot_of = [&](int c) -> int64_t { return static_cast<int64_t>(c == first ? slot0 : 2 * c) * p.slot_rows; };
      const float* po = reinterpret_cast<const float*>(p.part_o);
#pragma unroll 1
      for (int i = ct; i < w.t.n * p.group * (D / 4); i += kConvThreads) {
        const int r = i / (D / 4), c4 = i % (D / 4);
        const int64_t row = out_row_of(r);
        float M = -INFINITY, l = 0.f;
#pragma unroll 4
        for (int c = first; c <= last; ++c) M = fmaxf(M, __ldcg(&p.part_ml[slot_of(c) + r]).x);
        float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
        for (int c = first; c <= last; ++c) {
          const float2 ml = __ldcg(&p.part_ml[slot_of(c) + r]);
          const float4 v = __ldcg(reinterpret_cast<const float4*>(po + (slot_of(c) + r) * D) + c4);
          const float wt = level_factor(ml.x, M) * ml.y * kJoinScale;
          l += wt;
          acc.x += wt * v.x;
          acc.y += wt * v.y;
          acc.z += wt * v.z;
          acc.w += wt * v.w;
        }
        const float inv = __fdividef(1.f, l);
        uint2 y;
        y.x = pack_bf16x2(acc.x * inv, acc.y * inv);
        y.y = pack_bf16x2(acc.z * inv, acc.w * inv);
        *reinterpret_cast<uint2*>(p.out + row * D + c4 * 4) = y;
        if (c4 == 0 && p.lse) p.lse[row] = (M + kJoinLevel + __log2f(l)) * kLn2;
      }
      if (ct == 0) p.tickets[first] = 0u;
    };
    Walk before = w;
    for (;; ++item) {
      if (w.more) prepare();
      if (item > 0) {
        finish(before, item - 1, j);
        j += static_cast<uint32_t>(before.k1 - before.k0);
      }
      if (!ok || !w.more) break;
      before = w;
      w = next_item(p, w);
    }
  } else {
    // ------------------------------------------------------------ softmax
    const int grp = warp >> 2, w4 = warp & 3, key = w4 * 32 + lane;
    const uint32_t lanes = static_cast<uint32_t>(w4 * 32) << 16;
    constexpr int kBlocks = kFewRows / 16;
    const int gt = tid & 127;
    // A warp whose wait gave up goes on, without further waits, to where its group
    // leaves together.
    bool ok = true, left = false;
    for (; !left && w.more; w = next_item(p, w), ++item) {
      const int at = item & 1;
      const uint32_t o_col = tmem + lanes + C::kOAt + at * 4 * kFewRows, l_col = tmem + lanes + C::kLAt + (at * 2 + grp) * kFewRows;
      const uint32_t j0 = j, j1 = j + static_cast<uint32_t>(w.k1 - w.k0);
      // (Then the item before the last is read from tensor and shared memory, too.)
      ok = ok && all_wait(&bars.prep_full[item & 1], item >> 1);
      const int64_t s0 = w.b * p.ssb + w.g * p.ssh + key;
      const uint8_t *ksrc = p.scale[0] + s0, *vsrc = p.scale[1] + s0;
      if ((j0 & 1) != static_cast<uint32_t>(grp)) ++j;
      // The scales of this group's next chunk are on their way while one is worked on.
      uint32_t kb = 127u, vb = 127u;
      auto fetch = [&](int k) {
        kb = vb = 127u;
        if (k < w.k1 && k < w.t.prefix && k * kChunk + key < w.t.L) {
          kb = ksrc[static_cast<int64_t>(k) * kChunk];
          vb = vsrc[static_cast<int64_t>(k) * kChunk];
        }
      };
      fetch(w.k0 + static_cast<int>(j - j0));
      bool fresh = true;
      int ver = 0;
      for (; j < j1; j += 2) {
        const int k = w.k0 + static_cast<int>(j - j0);
        const bool tree_k = k >= w.t.prefix;
        const uint32_t kbyte = kb, vbyte = vb;
        fetch(k + 2);
        // The chunk before has settled its bases (another item's too: no phase of a
        // barrier is passed over).
        ok = ok && all_wait(&bars.s_full[j & 3], j >> 2) && (j == 0 || all_wait(&bars.mu[grp ^ 1], (j - 1) >> 1));
        sm100::tc_fence_after();
        const uint32_t s_col = tmem + lanes + (j & 3) * kFewRows;
        float ks = adt::q8_scale(kbyte);
        int ev = static_cast<int>(vbyte) - 127;
        const bool nan_v = !tree_k && vbyte == 255u;
        uint32_t sees = !tree_k && k * kChunk + key < w.t.L ? ~0u : 0u;
        if (tree_k && key < w.t.n) {
          ks = s_tk[at][key];
          ev = s_tv[at][key];
          sees = s_seen[at][key];
        }
        if (nan_v || sees == 0u) ev = kLeastScale;
        const bool masked = tree_k || (k + 1) * kChunk > w.t.L;
        // 16 rows' scores times the key's scale, -inf where they do not see it.
        auto load = [&](int blk, float (&x)[16]) {
          uint32_t r[16];
          sm100::tmem_ld_16(s_col + 16 * blk, r);
          const uint32_t bits = sees >> (16 * blk);
#pragma unroll
          for (int e = 0; e < 16; ++e) {
            x[e] = __uint_as_float(r[e]) * ks;
            if (masked) x[e] = bits >> e & 1u ? x[e] : -INFINITY;
          }
        };
        int top = s_top[at];
        float evf = static_cast<float>(max(ev, top - kSpan));
        bool raise = j == j0;
        if (!raise) {
          float most = -INFINITY;
#pragma unroll 1
          for (int blk = 0; blk < kBlocks; ++blk) {
            float x[16];
            load(blk, x);
            const float4* c4 = reinterpret_cast<const float4*>(s_c[at] + 16 * blk);
            const float4* b4 = reinterpret_cast<const float4*>(s_base[at] + 16 * blk);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const float4 c = c4[e], b = b4[e];
              most = fmaxf(most, fmaxf(fmaf(x[4 * e], c.x, -b.x), fmaf(x[4 * e + 1], c.y, -b.y)));
              most = fmaxf(most, fmaxf(fmaf(x[4 * e + 2], c.z, -b.z), fmaf(x[4 * e + 3], c.w, -b.w)));
            }
          }
          const bool more = !ok || most + evf > kFewThreshold;
          raise = grp == 0 ? any_of<3, 128>(more) : any_of<4, 128>(more);
        }
        if (raise) {
          // The largest scale, then every row's largest exponent over the chunk.
          const int wtop = __reduce_max_sync(adt::kFullMask, ev);
          if (lane == 0) s_wtop[grp][w4] = wtop;
          group_sync(grp);
          top = max(max(max(s_wtop[grp][0], s_wtop[grp][1]), max(s_wtop[grp][2], s_wtop[grp][3])), top);
          evf = static_cast<float>(max(ev, top - kSpan));
#pragma unroll 1
          for (int blk = 0; blk < kBlocks; ++blk) {
            float x[16];
            load(blk, x);
#pragma unroll
            for (int e = 0; e < 16; ++e) {
              const float m = warp_most(fmaf(x[e], s_c[at][16 * blk + e], evf));
              if (lane == 0) s_most[grp][w4][16 * blk + e] = m;
            }
          }
          // O is scaled once the chunks before are in it; then nothing reads the bases of
          // the chunk before either.
          // (That PV(j - 5) is, whose phase comes before, PV(j - 4) says.)
          if (ok && j > j0)
            ok = (j < 4 || all_wait(&bars.done[j & 3], (j - 4) >> 2)) && all_wait(&bars.done[(j - 1) & 3], (j - 1) >> 2);
          if (!ok && lane == 0) give_up();
          left = grp == 0 ? any_of<3, 128>(!ok) : any_of<4, 128>(!ok);
          if (left) break;
          if (gt < kFewRows) {
            const float y = fmaxf(fmaxf(s_most[grp][0][gt], s_most[grp][1][gt]), fmaxf(s_most[grp][2][gt], s_most[grp][3][gt]));
            const float old = s_base[at][gt], now = y > old + kFewThreshold ? y : old;
            s_base[at][gt] = now;
            s_alpha[grp][gt] = now == old ? 1.f : ex2_approx(old - now);
          }
          if (gt == 0) {
            s_from[at] = s_top[at] == kNoScale ? top : max(s_from[at], top - kFewLag);
            s_top[at] = top;
            ++s_ver[at];
          }
          group_sync(grp);
          if (j > j0) {
            sm100::tc_fence_after();
#pragma unroll 1
            for (int c = 0; c < 4 * kFewRows; c += 16) {
              uint32_t r[16];
              sm100::tmem_ld_16(o_col + c, r);
#pragma unroll
              for (int e = 0; e < 16; ++e)
                r[e] = __float_as_uint(__uint_as_float(r[e]) * s_alpha[grp][(c & (kFewRows - 1)) + e]);
              tmem_st_16(o_col + c, r);
            }
            sm100::tmem_wait_st();
          }
        }
        if (gt == 0) arrive(&bars.mu[grp]);
        const int now = s_ver[at];
        const int from = s_from[at];
        // The row sums of this group come to the bases' new level.
        if (fresh || now != ver) {
#pragma unroll 1
          for (int blk = 0; blk < kBlocks; ++blk) {
            uint32_t r[16];
            sm100::tmem_ld_16(l_col + 16 * blk, r);
#pragma unroll
            for (int e = 0; e < 16; ++e) {
              const float d = s_gb[at][grp][16 * blk + e] - (s_base[at][16 * blk + e] - from);
              r[e] = fresh ? 0u : __float_as_uint(__uint_as_float(r[e]) * ex2_approx(d));
            }
            tmem_st_16(l_col + 16 * blk, r);
          }
          sm100::tmem_wait_st();
          group_sync(grp);
          if (gt < kFewRows) s_gb[at][grp][gt] = s_base[at][gt] - from;
          fresh = false;
          ver = now;
        }
        // P's tile was last read by PV(j - PT).
        ok = j < PT || all_wait(&bars.done[(j - PT) & 3], (j - PT) >> 2);
        if (!ok) continue;
        const float iev = power_of_two(from - static_cast<int>(evf) - kFewShift), shift = evf + kFewHeadroom;
        const uint32_t keep = ev < top - kSpan ? 0u : ~0u;
#pragma unroll 1
        for (int blk = 0; blk < kBlocks; ++blk) {
          float x[16];
          load(blk, x);
          uint32_t r[16];
          sm100::tmem_ld_16(l_col + 16 * blk, r);
          const float4* c4 = reinterpret_cast<const float4*>(s_c[at] + 16 * blk);
          const float4* b4 = reinterpret_cast<const float4*>(s_base[at] + 16 * blk);
          uint32_t p1[4], p2[4], p3[4], p4[4];
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const float4 c = c4[e], b = b4[e];
            const float cc[4] = {c.x, c.y, c.z, c.w}, bb[4] = {b.x, b.y, b.z, b.w};
            uint32_t h[2];
#pragma unroll
            for (int f = 0; f < 4; ++f) {
              const int z = 4 * e + f;
              x[z] = ex2_approx(fmaf(x[z], cc[f], shift - bb[f]));
              r[z] = __float_as_uint(fmaf(x[z], iev, __uint_as_float(r[z])));
            }
#pragma unroll
            for (int f = 0; f < 2; ++f) h[f] = pack_half2(x[4 * e + 2 * f], x[4 * e + 2 * f + 1]);
            p1[e] = p2[e] = p3[e] = p4[e] = 0u;
#pragma unroll
            for (int f = 0; f < 2; ++f) {
              const uint16_t a1 = f16x2_to_e4m3(h[f]);
              const uint32_t r1 = rest16(h[f], a1);
              const uint16_t a2 = f16x2_to_e4m3(r1);
              const uint32_t r2 = rest16(r1, a2);
              const uint16_t a3 = f16x2_to_e4m3(r2);
              const uint16_t a4 = f16x2_to_e4m3(rest16(r2, a3));
              p1[e] |= static_cast<uint32_t>(a1) << (16 * f);
              p2[e] |= static_cast<uint32_t>(a2) << (16 * f);
              p3[e] |= static_cast<uint32_t>(a3) << (16 * f);
              p4[e] |= static_cast<uint32_t>(a4) << (16 * f);
            }
            p1[e] = nan_v ? 0x7f7f7f7fu : p1[e] & keep;
            p2[e] &= keep;
            p3[e] &= keep;
            p4[e] &= keep;
          }
          tmem_st_16(l_col + 16 * blk, r);
          uint8_t* tile_p = sP + (j % PT) * C::kPBytes;
          *reinterpret_cast<uint4*>(tile_p + tile_off<4 * kFewRows>(key, blk)) = make_uint4(p1[0], p1[1], p1[2], p1[3]);
          *reinterpret_cast<uint4*>(tile_p + tile_off<4 * kFewRows>(key, kBlocks + blk)) = make_uint4(p2[0], p2[1], p2[2], p2[3]);
          *reinterpret_cast<uint4*>(tile_p + tile_off<4 * kFewRows>(key, 2 * kBlocks + blk)) = make_uint4(p3[0], p3[1], p3[2], p3[3]);
          *reinterpret_cast<uint4*>(tile_p + tile_off<4 * kFewRows>(key, 3 * kBlocks + blk)) = make_uint4(p4[0], p4[1], p4[2], p4[3]);
        }
        sm100::fence_proxy_async_smem();
        sm100::tmem_wait_st();
        sm100::tc_fence_before();
        __syncwarp();
        if (lane == 0) {
          arrive(&bars.s_free[j & 3]);
          arrive(&bars.p_full[j & 3]);
        }
      }
      j = j1;
    }
    if (!ok && lane == 0) give_up();
  }
  sm100::tc_fence_before();
  __syncthreads();
  sm100::tc_fence_after();
  if (warp == kPvWarp) sm100::tmem_dealloc(tmem, C::kCols);
}
