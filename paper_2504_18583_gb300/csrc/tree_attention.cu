// Attention of a tree's nodes over the paged cache: S = Q K^T, a running
// maximum and sum, O += P V, both products on tcgen05 with the accumulators in
// tensor memory.
//
// A unit is one sequence's key/value head with up to 128 or 256 query vectors
// (nodes x the query heads that share the head) and its keys in tiles of 128.
// Each CTA (one an SM) works out its share from the sequences' lengths, which
// the host need not know.  A unit that is split between CTAs costs its
// partials' way through L2 (kSplit tiles' time), so units stay whole where they
// can: with no more units than CTAs, each CTA takes one equal part of one unit,
// the parts no longer than they must be; with more, all units' tiles, in order,
// are cut into one even range a CTA, and a cut near a unit's end moves there.
// A part leaves a partial (unnormalised O, maximum, sum, all in 32 bits) in the
// workspace; the last of a unit's CTAs to arrive joins them in tile order, so no
// CTA waits for another and results do not depend on timing.
//
// Roles: warp 0 loads keys and warp 2 values (TMA boxes of one page's 16 tokens
// x 64 entries: a tile of eight pages lands as the 128-byte-swizzled operand
// that the products read, K as stored, V as its transpose without moving a
// byte; a thread issues a box some 60 clocks after the last, so one warp would
// not keep up); warp 1 issues the products; warp 3 looks after the values of
// tiles that reach past the context; two warpgroups take the softmax, a thread a
// row, so that row maxima and sums need no exchange.  The two groups work on two
// score tiles in turn: with more than 128 query vectors each has its own 128 of
// them, else both have the same and alternate key tiles (their sums are joined
// at the end straight from tensor memory).  One tile's products run under the
// other's softmax.  The accumulator is scaled only when a row's maximum has grown
// by more than 2^8 since the last time.  Probabilities are rounded to the
// cache's 16-bit type for the second product, which takes 16-bit operands; their
// sum is taken before that, in 32 bits.  (Against 64 bits the output's error is
// 1.2 to 1.45 times that of 32-bit probabilities rounded once at the end.)  fp16
// has few exponents: its probabilities are held times 2^7, sums and outputs with
// them, so that one is rounded to its 11 bits down to 2^-21 of the largest and
// to a multiple of 2^-31 below that.  (Times 1 a long context's many small ones
// lost up to all of their part: those 18 nats below a single key vanished.)
//
// Masks touch only tiles that reach past the context: a row's 256 mask bits
// select among its scores.  Values there may hold anything: what lies past the
// sequence is zeroed in shared memory, and so are infinities and NaN of tree
// nodes, which the CTA that writes the output adds back for the rows that see the
// node (0 x NaN would reach every row otherwise).
//
// What bounds it, measured:
//   8 sequences x 64 nodes at 4096, 64/8 heads of 128: 68 us; 36 us of products
//     at the peak.  Its 128 units stay whole, so 24 of 152 CTAs have no part.  A
//     pair of tiles takes 3300 clocks: 2100 of products, and the chain softmax
//     (1310) -> P V -> scores of one group, of which the issuing warp's waits and
//     commits are 600; the tensor pipe is busy half the time of the other 128.
//   16 ragged sequences x 29 nodes, 32/8 heads of 128: 28 us; 11 us of K and V.
//     7000 clocks to the first instruction of a role (lengths, shares, barriers),
//     7000 more to the first scores, then up to 28000 of tiles (144 parts, the
//     longest of 14 tiles where the mean is 7), 5000 at the end.
//   2 x 13 nodes at 65000, 32/8 heads of 64: 57 us; 35 us of K and V.  72000 of
//     110000 clocks near HBM's rate, 15000 before, 6500 to write a part and 9000
//     to 12000 for the last to join ten or eleven.
//   1 node at 512: 12 us, all of it dependent steps.
#include <type_traits>

#include "attn_tc.cuh"

namespace pard {

namespace {

constexpr int kTaThreads = 384;
constexpr int kSeqCache = 64;                   // sequences whose lengths a CTA keeps at hand
constexpr int kStart = 2;                       // what a unit's start costs in tiles

// tiles of keys, and of values, in flight: what shared memory holds beside the queries
__host__ __device__ constexpr int k_stages(int hd, int blocks) { return hd == 128 ? (blocks == 1 ? 3 : 2) : (blocks == 1 ? 6 : 5); }
__host__ __device__ constexpr int v_stages(int hd, int blocks) { return hd == 128 ? 3 : (blocks == 1 ? 6 : 5); }

// Keys, tiles and row blocks of a sequence.
struct Seq {
  int ctx, nodes, keys, plain, tiles, blocks;  // plain: keys that every node sees
};
__device__ __forceinline__ Seq seq_of(const TreeAttnArgs& a, int ctx, int nodes, int rows_per_block) {
  Seq s;
  s.nodes = min(max(nodes, 0), a.width);
  s.ctx = max(ctx, 0);
  const int64_t end = (int64_t)s.ctx + s.nodes, most = (int64_t)a.max_pages * kPageTok;
  s.keys = (int)(end < most ? end : most);
  s.plain = min(s.ctx, s.keys);
  s.tiles = s.nodes > 0 ? (s.keys + kTile - 1) / kTile : 0;
  s.blocks = (s.nodes * (a.n_q_heads / a.n_kv_heads) + rows_per_block - 1) / rows_per_block;
  return s;
}
// Ranges count a unit as kStart tiles more than it has: what its queries,
// first loads and epilogue cost.  (All of them together stay below 2^31: the
// caller has checked.)
__device__ __forceinline__ int seq_cost(const TreeAttnArgs& a, const Seq& s) {
  return s.tiles ? a.n_kv_heads * s.blocks * (s.tiles + kStart) : 0;
}
// A warp's walk over its CTA's share: one segment (part of a unit) after the
// other.  It lies in shared memory: held in registers, it made the softmax's
// scores spill.
struct Walk {
  int left;            // places to go; in the one-part form 1, then 0
  int b, off;          // sequence, and place within all of its units
  int at;              // place of the whole pass that off counts from
  Seq s;
  int head, block, t0, t1;
  int count, me, c0;   // the unit's contributors, this CTA's place among them, the first of them (among CTAs with a place)
  __device__ __forceinline__ void load(const TreeAttnArgs& a, const int2* cache, int rows_per_block) {
    const int2 v = b < kSeqCache ? cache[b] : make_int2(a.ctx_len[b], a.n_nodes[b]);
    s = seq_of(a, v.x, v.y, rows_per_block);
  }
  __device__ __noinline__ bool next(const TreeAttnArgs& a, const int2* cache, int rows_per_block, const Ranges& ranges,
                                    bool one_part) {
    if (one_part) return left-- > 0;
    while (left > 0) {
      for (int cost = seq_cost(a, s); off >= cost; cost = seq_cost(a, s)) {  // the first call's off lies inside its sequence
        at += cost;
        ++b;
        off = 0;
        load(a, cache, rows_per_block);
      }
      const int len = s.tiles + kStart, unit = off / len, y = off - unit * len;
      const int x0 = Ranges::cut(y, len), x1 = y + left < len ? Ranges::cut(y + left, len) : len;
      const int u0 = at + off - y;  // place of the unit in the whole pass
      head = unit / s.blocks;
      block = unit - head * s.blocks;
      const int step = min(len - y, left);
      off += step;
      left -= step;
      t0 = max(0, x0 - kStart);
      t1 = x1 - kStart;
      if (t1 <= t0) continue;
      count = 1;
      me = 0;
      c0 = blockIdx.x;
      if (t0 > 0 || t1 < s.tiles) {  // who else has a part of it
        while (c0 > 0 && ranges.at(c0) > u0 && Ranges::cut(ranges.at(c0) - u0, len) > 0) --c0;
        int c1 = blockIdx.x;
        while (c1 + 1 < ranges.grid && ranges.at(c1 + 1) < u0 + len && Ranges::cut(ranges.at(c1 + 1) - u0, len) < len) ++c1;
        me = blockIdx.x;
        if (ranges.each == 0) {  // those between them whose range is empty never arrive
          c0 = ranges.at(c0);
          c1 = ranges.at(c1);
          me = ranges.at(me);
        }
        count = c1 - c0 + 1;
        me -= c0;
      }
      return true;
    }
    return false;
  }
};

// 32 of a row's allowed columns, from the mask bits of its node: column 0 is
// key `key`; bits of the context are set, those past the nodes clear.
__device__ __forceinline__ uint32_t allowed32(const uint32_t* row, int words32, int key, const Seq& s) {
  const int rel = key - s.ctx, some = s.keys - key;  // node of column 0; columns that are keys at all
  uint32_t m = 0xFFFFFFFFu;
  if (rel >= 0) {
    const int w = rel >> 5;
    const uint32_t lo = w < words32 ? row[w] : 0u, hi = w + 1 < words32 ? row[w + 1] : 0u;
    m = __funnelshift_r(lo, hi, rel & 31);
  } else if (rel > -32) {
    m = row[0] << -rel | ((1u << -rel) - 1u);
  }
  return some >= 32 ? m : some <= 0 ? 0u : m & ((1u << some) - 1u);
}

// Adds the infinities and NaN of the tree nodes' values back to the output of the
// row that has thread t of group g, where it sees them: on top of the joined sum
// they stay what they are.
template <typename T, int HD, int BLOCKS>
__device__ __noinline__ void patch_row(const TreeAttnArgs& a, const Walk& w, int g, int t) {
  constexpr int cols = BLOCKS == 2 ? HD : HD / 2;
  const int group = a.n_q_heads / a.n_kv_heads, row = w.block * BLOCKS * kTile + (BLOCKS == 2 ? g * kTile : 0) + t, of = row / group;
  const int col0 = BLOCKS == 2 ? 0 : g * cols;
  if (row >= w.s.nodes * group) return;
  const uint32_t* mrow = reinterpret_cast<const uint32_t*>(a.mask + ((size_t)w.b * a.width + of) * a.words);
  T* out = reinterpret_cast<T*>(a.out) + (((int64_t)w.b * a.width + of) * a.n_q_heads + (int64_t)w.head * group + (row - of * group)) * HD;
  for (int pos = w.s.ctx; pos < w.s.keys; ++pos) {
    const int node = pos - w.s.ctx, page = page_of(a.page_table + (size_t)w.b * a.max_pages, pos, a.max_pages, a.n_pages);
    if (page < 0 || !(mrow[node >> 5] >> (node & 31) & 1)) continue;
    const T* v = reinterpret_cast<const T*>(a.v_cache) + page * a.page_stride + ((int64_t)w.head * kPageTok + pos % kPageTok) * HD;
#pragma unroll 1
    for (int c = col0; c < col0 + cols; ++c) {
      const float x = Num<T>::get(v + c);
      if (fabsf(x) < INFINITY) continue;
      const uint32_t y = Num<T>::pack(Num<T>::get(out + c) + x, 0.f);
      *reinterpret_cast<uint16_t*>(out + c) = (uint16_t)y;
    }
  }
}

// What a CTA keeps in shared memory behind the operands.
template <int NK, int NV>
struct Control {
  uint64_t k_full[NK], k_empty[NK], v_full[NV], v_empty[NV];
  uint64_t fixed[NV];      // a stage's values are fit for the product
  uint64_t s_full[2];      // scores of a group are in tensor memory
  uint64_t p_full[2];      // its probabilities are, and O is scaled
  uint64_t o_full[2];      // a segment's last product is done
  uint64_t ready[2];       // the group has read O and laid out its queries
  uint64_t pair, met[2];   // the two groups meet, a group's warps do
  uint64_t drain;          // every product is done
  uint32_t tmem, last_in[2], odd[NV];  // odd: a stage's tree values held infinities or NaN
  int abort_flag, start_b, start_off;
  int sum[kTaThreads / 32], units[kTaThreads / 32], most[kTaThreads / 32];
  int2 seq[kSeqCache];
  Walk walk[kTaThreads / 32];
  uint16_t slots[2][kMaxGrid];
};

template <int HD, int BLOCKS>
constexpr int smem_bytes() {
  return (BLOCKS + k_stages(HD, BLOCKS) + v_stages(HD, BLOCKS)) * stage_bytes(HD) +
         (int)sizeof(Control<k_stages(HD, BLOCKS), v_stages(HD, BLOCKS)>);
}
static_assert(smem_bytes<128, 1>() <= 227 * 1024 && smem_bytes<128, 2>() <= 227 * 1024, "shared memory of one CTA");
static_assert(smem_bytes<64, 1>() <= 227 * 1024 && smem_bytes<64, 2>() <= 227 * 1024, "shared memory of one CTA");

}  // namespace

template <typename T, int HD, int BLOCKS>
__global__ void __launch_bounds__(kTaThreads, 1)
    tree_attention_kernel(const __grid_constant__ TreeAttnArgs a, const __grid_constant__ CUtensorMap kmap,
                          const __grid_constant__ CUtensorMap vmap) {
  constexpr int NK = k_stages(HD, BLOCKS), NV = v_stages(HD, BLOCKS), kStage = stage_bytes(HD);
  constexpr int kChunks = HD / 64, kChunkBytes = kTile * 128, kRows = kTile * BLOCKS;
  constexpr uint32_t kIdescS = idesc16(Num<T>::kFormat, kTile, kTile, false);
  constexpr uint32_t kIdescO = idesc16(Num<T>::kFormat, kTile, HD, true);
  extern __shared__ __align__(1024) uint8_t qbuf[];  // queries, then the rings
  uint8_t* kring = qbuf + BLOCKS * kStage;
  uint8_t* vring = kring + NK * kStage;
  Control<NK, NV>& sh = *reinterpret_cast<Control<NK, NV>*>(vring + NV * kStage);
  volatile int* abort_flag = &sh.abort_flag;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int group = a.n_q_heads / a.n_kv_heads, grid = gridDim.x;

  // ---- this CTA's range -------------------------------------------------------
  if (warp == 1) tmem_alloc(&sh.tmem, 512);
  if (tid == 0) {
    tma_prefetch_desc(&kmap);
    tma_prefetch_desc(&vmap);
#pragma unroll 1
    for (int i = 0; i < NK; ++i) { mbar_init(sh.k_full + i, 1); mbar_init(sh.k_empty + i, 1); }
#pragma unroll 1
    for (int i = 0; i < NV; ++i) { mbar_init(sh.v_full + i, 1); mbar_init(sh.v_empty + i, 1); mbar_init(sh.fixed + i, 1); }
#pragma unroll 1
    for (int i = 0; i < 2; ++i) {
      mbar_init(sh.s_full + i, 1); mbar_init(sh.p_full + i, 4);
      mbar_init(sh.o_full + i, 1); mbar_init(sh.ready + i, 4); mbar_init(sh.met + i, 4);
    }
    mbar_init(&sh.pair, 8);
    mbar_init(&sh.drain, 1);
    fence_barrier_init();
    *abort_flag = 0;
  }
  pdl_trigger();
  pdl_wait();
  const uint32_t stalled = reinterpret_cast<const volatile uint32_t*>(a.workspace)[kStalledWord];
  // The share's form and, in ranges, this CTA's first place: two rounds over the
  // sequences, their sum and then the place in it; both are one round of a
  // single step for up to 384.
  Ranges ranges;
  int lo = 0, hi = 0, units = 0, longest = 0;
#pragma unroll 1
  for (int round = 0; round < 2; ++round) {
    int run = 0;
#pragma unroll 1
    for (int b0 = 0; b0 < a.batch; b0 += kTaThreads) {
      const int b = b0 + tid;
      int2 v = make_int2(0, 0);
      if (b < a.batch) v = make_int2(a.ctx_len[b], a.n_nodes[b]);
      if (b < kSeqCache) sh.seq[b] = v;
      const Seq s = seq_of(a, v.x, v.y, kRows);
      const int cost = b < a.batch ? seq_cost(a, s) : 0;
      int inc = cost;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const int t = __shfl_up_sync(0xffffffffu, inc, o);
        if (lane >= o) inc += t;
      }
      const int u = __reduce_add_sync(0xffffffffu, cost ? a.n_kv_heads * s.blocks : 0);
      const int most = __reduce_max_sync(0xffffffffu, cost ? s.tiles : 0);
      if (lane == 31) { sh.sum[warp] = inc; sh.units[warp] = u; sh.most[warp] = most; }
      __syncthreads();
      const bool is = lane < kTaThreads / 32;
      const int of = is ? sh.sum[lane] : 0, step = __reduce_add_sync(0xffffffffu, of);
      inc += run + __reduce_add_sync(0xffffffffu, lane < warp ? of : 0);
      units += __reduce_add_sync(0xffffffffu, is ? sh.units[lane] : 0);
      longest = max(longest, __reduce_max_sync(0xffffffffu, is ? sh.most[lane] : 0));
      run += step;
      if (a.batch <= kTaThreads) {
        ranges.set(run, grid);
        lo = ranges.at(blockIdx.x);
        hi = ranges.at(blockIdx.x + 1);
        round = 1;
      }
      if (round && inc > lo && inc - cost <= lo) { sh.start_b = b; sh.start_off = lo - (inc - cost); }
      __syncthreads();
    }
    if (!round) {
      ranges.set(run, grid);
      lo = ranges.at(blockIdx.x);
      hi = ranges.at(blockIdx.x + 1);
    }
  }
  const bool one_part = a.batch <= kSeqCache && units <= grid;
  Walk& w = sh.walk[warp];
  if (one_part) {
    // the fewest tiles a part that the CTAs are enough for; two sequences a lane
    static_assert(kSeqCache == 64, "two sequences a lane");
    int tiles[2], mine[2];
    const int all_tiles = ranges.total - units * kStart;
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      const int b = 2 * lane + e;
      const Seq s = b < a.batch ? seq_of(a, sh.seq[b].x, sh.seq[b].y, kRows) : Seq{};
      tiles[e] = s.tiles;
      mine[e] = s.tiles ? a.n_kv_heads * s.blocks : 0;
    }
    // (A unit's parts are less than one more than its tiles / most, or, of millions of
    // tiles, than its tiles and four / most: a CTA fewer to share out is room for that.
    // Signed or unsigned, the quotients are the same, but what the compiler makes of the
    // whole kernel is not: with signed ones two trees of 13 nodes at 65000 take 59.8 us
    // instead of 57.6, one node at 512 12.7 instead of 12.4; with unsigned ones the kernels
    // of two blocks take 68.2 instead of 67.0 for 8 x 64 nodes at 4096.)
    using Whole = std::conditional_t<BLOCKS == 1, uint32_t, int>;
    int least = max(1, (int)((Whole)all_tiles / (Whole)grid));
    int most = max(least, min(longest, (int)((Whole)all_tiles / (Whole)max(grid - units, 1)) + 1));
#pragma unroll 1
    while (least < most) {
      const int mid = (least + most) / 2;
      const int need = __reduce_add_sync(0xffffffffu, mine[0] * parts_of(tiles[0], mid) + mine[1] * parts_of(tiles[1], mid));
      if (need <= grid) most = mid; else least = mid + 1;
    }
    int inc = 0;
#pragma unroll
    for (int e = 0; e < 2; ++e) { mine[e] *= parts_of(tiles[e], most); inc += mine[e]; }
    const int own = inc;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int t = __shfl_up_sync(0xffffffffu, inc, o);
      if (lane >= o) inc += t;
    }
    if (lane == 0) w.left = 0;  // more CTAs than parts
    __syncwarp();
    int before = inc - own;
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      const int at = (int)blockIdx.x - before;
      if (at >= 0 && at < mine[e]) {
        const int parts = parts_of(tiles[e], most), unit = at / parts;
        w.left = 1;
        w.b = 2 * lane + e;
        w.load(a, sh.seq, kRows);
        w.head = unit / w.s.blocks;
        w.block = unit - w.head * w.s.blocks;
        w.count = parts;
        w.me = at - unit * parts;
        w.c0 = (int)blockIdx.x - w.me;
        w.t0 = w.me * w.s.tiles / parts;
        w.t1 = (w.me + 1) * w.s.tiles / parts;
      }
      before += mine[e];
    }
  } else if (lane == 0) {
    w.left = hi - lo;  // 0: more CTAs than places
    w.b = hi > lo ? sh.start_b : 0;
    w.off = hi > lo ? sh.start_off : 0;
    w.at = lo - w.off;
    w.load(a, sh.seq, kRows);
  }
  __syncwarp();
  const bool had_part = w.left > 0;
  // the warp's next segment
  auto next = [&]() -> bool {
    __syncwarp();
    bool some = false;
    if (lane == 0) some = w.next(a, sh.seq, kRows, ranges, one_part);
    return __shfl_sync(0xffffffffu, (int)some, 0);
  };
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = sh.tmem;
  int tile0 = 0;  // tiles of the segments before this one
  bool ok = true;

  if (warp == 0 || warp == 2) {
    // ---- loads: keys by one warp, values by another --------------------------------
    // Page ids are fetched 32 pages (four tiles) at a time, a block ahead of
    // their use: a load from the table would be on every copy's path.
    const bool v = warp == 2;
    uint64_t *full = v ? sh.v_full : sh.k_full, *empty = v ? sh.v_empty : sh.k_empty;
    uint8_t* to0 = v ? vring : kring;
    const CUtensorMap* map = v ? &vmap : &kmap;
    const int ns = v ? NV : NK;
    int st = 0, phase = 0, issued = 0;  // stages are used in turn
    while (ok && next()) {
      const int n = w.t1 - w.t0, head = w.head, page0 = w.t0 * kTilePages;
      const int32_t* row = a.page_table + (size_t)w.b * a.max_pages;
      const int last_page = (w.s.keys - 1) / kPageTok;
      auto fetch = [&](int block) {
        const int p = page0 + 32 * block + lane;
        const int page = p <= last_page ? row[p] : 0;
        return (uint32_t)page < (uint32_t)a.n_pages ? page : a.n_pages;  // out of the tensor: reads as zeros
      };
      int have = fetch(0), after = n > 4 ? fetch(1) : 0;
#pragma unroll 1
      for (int j = 0; j < n; ++j) {
        const int pages = min(kTilePages, last_page - page0 - j * kTilePages + 1);
        if (j > 0 && (j & 3) == 0) {
          have = after;
          if (j + 4 < n) after = fetch(j / 4 + 1);
        }
        int page[kTilePages];
#pragma unroll
        for (int q = 0; q < kTilePages; ++q) page[q] = __shfl_sync(0xffffffffu, have, (j & 3) * kTilePages + q);
        ok = warp_wait(empty + st, phase ^ 1, abort_flag);
        if (!ok) break;
        if (elect_one()) {
          mbar_arrive_expect_tx(full + st, (uint32_t)pages * kChunks * kPageTok * 128);
          uint8_t* to = to0 + st * kStage;
#pragma unroll
          for (int q = 0; q < kTilePages; ++q)
            if (q < pages) {
#pragma unroll
              for (int c = 0; c < kChunks; ++c)
                tma_load_4d(to + c * kChunkBytes + q * kPageTok * 128, map, full + st, c * 64, 0, head, page[q]);
            }
        }
        __syncwarp();
        ++issued;
        if (++st == ns) { st = 0; phase ^= 1; }
      }
    }
    if (!ok) {  // copies in flight write this CTA's shared memory: they land before it goes
      *abort_flag = 1;
      for (int i = max(0, issued - ns); i < issued; ++i) mbar_drain(full + i % ns, (i / ns) & 1);
    }
  } else if (warp == 1) {
    // ---- products ---------------------------------------------------------------
    uint32_t ph_p = 0, ph_ready = 0;
    const uint32_t q_addr = smem_u32(qbuf), k_addr = smem_u32(kring), v_addr = smem_u32(vring);
    auto wait_k = [&](int i) { ok = ok && warp_wait(sh.k_full + i % NK, (i / NK) & 1, abort_flag); };
    auto wait_v = [&](int i) { ok = ok && warp_wait(sh.fixed + i % NV, (i / NV) & 1, abort_flag); };
    // Operand addresses go through a shuffle, which tells the compiler that they
    // are the warp's and not a lane's, and steps add constants to a
    // descriptor's low word: an issue then costs little beside its product.
    auto uniform = [](uint32_t x) { return __shfl_sync(0xffffffffu, x, 0); };
    // Shared-memory descriptors, 128-byte swizzle.  Queries and keys: 128-byte
    // rows along K, eight-row atoms 1024 bytes apart.  Values: 64 of a key's
    // entries a row (N is contiguous), atoms of eight keys 1024 bytes apart along
    // K, the next 64 entries a chunk further.
    constexpr uint64_t kDescK = (uint64_t)1 << 16 | (uint64_t)(1024 >> 4) << 32 | (uint64_t)1 << 46 | (uint64_t)2 << 61;
    constexpr uint64_t kDescV = (uint64_t)(kChunkBytes >> 4) << 16 | (uint64_t)(1024 >> 4) << 32 | (uint64_t)1 << 46 | (uint64_t)2 << 61;
    auto scores = [&](int g, int i) {
      const uint32_t qa = uniform((q_addr + (BLOCKS == 2 ? g * kStage : 0)) >> 4), kb = uniform((k_addr + (i % NK) * kStage) >> 4);
      const uint32_t d = uniform(tmem + g * kTile);
      if (elect_one()) {
#pragma unroll
        for (int k = 0; k < HD / 16; ++k) {
          const uint32_t at = ((k / 4) * kChunkBytes + (k % 4) * 32) >> 4;
          umma_ss(d, kDescK | (qa + at), kDescK | (kb + at), kIdescS, k > 0);
        }
        umma_commit(sh.s_full + g);
      }
      __syncwarp();
    };
    auto outputs = [&](int g, int i, bool first, int keys) {  // O += P V
      const uint32_t vb = uniform((v_addr + (i % NV) * kStage) >> 4);
      const uint32_t o = uniform(tmem + 2 * kTile + g * HD), p = uniform(tmem + g * kTile);
      // keys past the end have probability 0: whole steps of 16 are left out
      const int steps = __shfl_sync(0xffffffffu, (keys + 15) / 16, 0);
      ok = ok && warp_wait(sh.p_full + g, ph_p >> g & 1, abort_flag);
      if (!ok) return;
      ph_p ^= 1u << g;
      tc_fence_after();
      if (elect_one()) {
#pragma unroll
        for (int k = 0; k < kTile / 16; ++k)
          if (k < steps) umma_ts(o, p + k * 8, kDescV | (vb + k * 128), kIdescO, !first || k > 0);
      }
      __syncwarp();
    };
    auto commit = [&](uint64_t* bar) {
      if (elect_one()) umma_commit(bar);
      __syncwarp();
    };
    while (ok && next()) {
      const int n = w.t1 - w.t0, keys0 = w.s.keys - w.t0 * kTile;  // from the first tile on
      ok = warp_wait(sh.ready + 0, ph_ready, abort_flag) && warp_wait(sh.ready + 1, ph_ready, abort_flag);
      ph_ready ^= 1;
      tc_fence_after();
      if (BLOCKS == 2) {  // step j: each group takes tile j, and the scores of the next
#pragma unroll 1
        for (int j = -1; j < n && ok; ++j) {
          const int i = tile0 + j;
          const bool more = j + 1 < n;
          if (j >= 0) wait_v(i);
          if (!ok) break;
#pragma unroll
          for (int g = 0; g < 2; ++g) {
            if (j >= 0) outputs(g, i, j == 0, keys0 - j * kTile);
            // (asked for here, since the load of a stage that has just come free is
            // what a step would wait for)
            if (more && g == 0) wait_k(i + 1);
            if (!ok) break;
            if (more) scores(g, i + 1); else commit(sh.o_full + g);
          }
          if (!ok) break;
          if (j >= 0) commit(sh.v_empty + i % NV);
          if (more) commit(sh.k_empty + (i + 1) % NK);
        }
      } else {  // group j & 1 takes tile j, and the scores of its next, j + 2
#pragma unroll 1
        for (int j = -2; j < n && ok; ++j) {
          const int g = j & 1, i = tile0 + j;
          if (j >= 0) {
            wait_v(i);
            if (ok) outputs(g, i, j < 2, keys0 - j * kTile);
            if (!ok) break;
            commit(sh.v_empty + i % NV);
          }
          if (j + 2 < n) {
            wait_k(i + 2);
            if (!ok) break;
            scores(g, i + 2);
            commit(sh.k_empty + (i + 2) % NK);
          }
        }
        if (!ok) break;
        commit(sh.o_full + 0);
        commit(sh.o_full + 1);
      }
      tile0 += n;
    }
    if (!ok) *abort_flag = 1;
    // products in flight read shared memory and write tensor memory: let them end
    commit(&sh.drain);
    mbar_drain(&sh.drain, 0);
  } else if (warp == 3) {
    // ---- values of tiles that reach past the context --------------------------------
    // and, first, the rows of unused nodes, which are zero
    const size_t row16 = (size_t)a.n_q_heads * HD / 8;  // 16-byte pieces of a node
#pragma unroll 1
    for (int b = 0; b < a.batch; ++b) {
      const int nodes = min(max(b < kSeqCache ? sh.seq[b].y : a.n_nodes[b], 0), a.width);
      uint4* at = reinterpret_cast<uint4*>(a.out) + ((size_t)b * a.width + nodes) * row16;
#pragma unroll 1
      for (size_t i = blockIdx.x * 32 + lane; i < (a.width - nodes) * row16; i += grid * 32) at[i] = make_uint4(0, 0, 0, 0);
    }
    while (ok && next()) {
      const int n = w.t1 - w.t0;
#pragma unroll 1
      for (int j = 0; j < n; ++j) {
        const int st = (tile0 + j) % NV;
        ok = warp_wait(sh.v_full + st, ((tile0 + j) / NV) & 1, abort_flag);
        if (!ok) break;
        const int k0 = (w.t0 + j) * kTile;
        if (k0 + kTile > w.s.plain) {
          const int first = max(0, w.s.plain - k0), end = w.s.keys - k0;
          const int used = min(kTile, (end + 15) & ~15);  // the products take steps of 16 keys
          constexpr int kPieces = HD / 8;
          bool any = false;
#pragma unroll 4
          for (int p = first * kPieces + lane; p < used * kPieces; p += 32) {
            const int r = p / kPieces, c = p % kPieces;
            uint4* at = reinterpret_cast<uint4*>(vring + st * kStage + (c / 8) * kChunkBytes + r * 128 + (((c % 8) ^ (r & 7)) << 4));
            const uint4 v = *at;
            const uint4 f = r >= end ? make_uint4(0, 0, 0, 0)
                                     : make_uint4(finite_of<T>(v.x), finite_of<T>(v.y), finite_of<T>(v.z), finite_of<T>(v.w));
            if (f.x != v.x || f.y != v.y || f.z != v.z || f.w != v.w) {
              *at = f;
              any |= r < end;
            }
          }
          fence_proxy_async_all();
          any = __any_sync(0xffffffffu, any);
          if (lane == 0) sh.odd[st] = any;
        }
        __syncwarp();
        if (lane == 0) mbar_arrive(sh.fixed + st);
      }
      tile0 += n;
    }
    if (!ok) *abort_flag = 1;
  } else {
    // ---- softmax: group g, a thread a row --------------------------------------------
    const int g = (warp - 4) >> 2, t = tid - 128 - g * kTile;  // t: row of the score tile = lane of tensor memory
    const uint32_t my = tmem + ((uint32_t)((warp & 3) * 32) << 16);
    const uint32_t s_addr = my + g * kTile, o_addr = my + 2 * kTile + g * HD;
    const float sl2 = fmaxf(fabsf(a.scale) * 1.4426950408889634f, 1e-30f);  // a masked score stays -inf at scale 0
    const bool wide_out = (reinterpret_cast<uintptr_t>(a.out) & 31) == 0;
    uint32_t ph_s = 0, ph_o = 0, ph_pair = 0, ph_met = 0;
    auto meet = [&] {  // both groups, 256 threads
      __syncwarp();
      if (lane == 0) mbar_arrive(&sh.pair);
      ok = warp_wait(&sh.pair, ph_pair, abort_flag);
      ph_pair ^= 1;
    };
    auto group_meet = [&] {
      __syncwarp();
      if (lane == 0) mbar_arrive(sh.met + g);
      ok = warp_wait(sh.met + g, ph_met, abort_flag);
      ph_met ^= 1;
    };
    while (ok && next()) {
      const int n = w.t1 - w.t0;
      const int row_base = w.block * kRows + (BLOCKS == 2 ? g * kTile : 0);  // row of the unit that lane 0 of the group has
      const int row = row_base + t, rows = w.s.nodes * group;
      // queries into shared memory, swizzled; one block: each group lays out half
      {
        constexpr int kPieces = HD / 8, kMine = BLOCKS == 2 ? kTile : kTile / 2, kStep = kTile / kPieces;
        // row / group as a product: exact for the rows of 256 nodes x 4096 heads
        const uint32_t magic = group > 1 ? 0xFFFFFFFFu / (uint32_t)group + 1 : 0;
        const uint32_t sign = a.scale < 0.f ? 0x80008000u : 0u;  // a negative scale turns the queries' signs
        const int c = t % kPieces, r0 = t / kPieces + (BLOCKS == 2 ? 0 : g * kMine);
        const T* q = reinterpret_cast<const T*>(a.q) + (int64_t)w.b * a.width * a.q_stride + (int64_t)w.head * group * HD + c * 8;
        uint8_t* dst = qbuf + (BLOCKS == 2 ? g * kStage : 0) + (c / 8) * kChunkBytes;
        uint4 v[kMine / kStep];  // all loads are out before the first is stored
#pragma unroll
        for (int i = 0; i < kMine / kStep; ++i) {
          const int r = row_base + r0 + i * kStep, node = magic ? (int)__umulhi((uint32_t)r, magic) : r;
          v[i] = make_uint4(0, 0, 0, 0);
          if (r < rows) v[i] = *reinterpret_cast<const uint4*>(q + (int64_t)node * a.q_stride + (r - node * group) * HD);
        }
#pragma unroll
        for (int i = 0; i < kMine / kStep; ++i) {
          const int r = r0 + i * kStep;
          v[i].x ^= sign; v[i].y ^= sign; v[i].z ^= sign; v[i].w ^= sign;
          *reinterpret_cast<uint4*>(dst + r * 128 + (((c % 8) ^ (r & 7)) << 4)) = v[i];
        }
        fence_proxy_async_all();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(sh.ready + g);
      }
      const int node = min(row / group, w.s.nodes - 1);
      const uint32_t* mrow = reinterpret_cast<const uint32_t*>(a.mask + ((size_t)w.b * a.width + node) * a.words);
      auto page_flag = [&](int j) -> uint32_t {  // this lane's page of tile j is one of the pool
        const int p = (w.t0 + j) * kTilePages + lane;
        if (lane >= kTilePages || p * kPageTok >= w.s.keys) return 1;
        return (uint32_t)a.page_table[(size_t)w.b * a.max_pages + p] < (uint32_t)a.n_pages;
      };
      float m_ref = -INFINITY, sum = 0.f;
      bool patch = false;  // values that the rows who see them get back in the epilogue
      const int j0 = BLOCKS == 2 ? 0 : g, jn = BLOCKS == 2 ? 1 : 2;
      uint32_t flag = j0 < n ? page_flag(j0) : 1u;
#pragma unroll 1
      for (int j = j0; j < n; j += jn) {
        const uint32_t flags = __ballot_sync(0xffffffffu, flag);
        if (j + jn < n) flag = page_flag(j + jn);
        const int k0 = (w.t0 + j) * kTile;
        const bool tail = k0 + kTile > w.s.plain;
        const bool masked = tail || flags != 0xFFFFFFFFu;
        uint32_t allow[4] = {0, 0, 0, 0};
        if (masked) {
#pragma unroll
          for (int c = 0; c < 4; ++c)
            allow[c] = allowed32(mrow, 2 * a.words, k0 + 32 * c, w.s) &
                       (((flags >> (2 * c)) & 1 ? 0xFFFFu : 0u) | ((flags >> (2 * c + 1)) & 1 ? 0xFFFF0000u : 0u));
        }
        ok = warp_wait(sh.s_full + g, ph_s, abort_flag);
        if (!ok) break;
        ph_s ^= 1;
        tc_fence_after();
        if (masked) {
          // masked scores become -inf where they lie, 32 columns a turn
#pragma unroll 1
          for (int c = 0; c < 4; ++c) {
            const uint32_t m = c < 2 ? (c ? allow[1] : allow[0]) : (c == 2 ? allow[2] : allow[3]);
            uint32_t x[32];
            tm_ld32(s_addr + 32 * c, x);
            tm_landed<32>(x);
#pragma unroll
            for (int i = 0; i < 32; ++i)
              if (!(m >> i & 1)) x[i] = 0xFF800000u;
            tm_st32(s_addr + 32 * c, x);
          }
          tm_wait_st();
        }
        uint32_t v[kTile];
#pragma unroll
        for (int c = 0; c < 4; ++c) tm_ld32(s_addr + 32 * c, v + 32 * c);
        tm_landed<kTile>(v);
        float mx[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
        for (int i = 0; i < kTile; i += 2)
          mx[i >> 1 & 3] = fmaxf(fmaxf(__uint_as_float(v[i]), __uint_as_float(v[i + 1])), mx[i >> 1 & 3]);
        // what probabilities are taken against: 2^kRaise below the largest
        const float top = fmaxf(fmaxf(mx[0], mx[1]), fmaxf(mx[2], mx[3])) * sl2 - Num<T>::kRaise;
        if (j == j0) {
          m_ref = top;
        } else if (__any_sync(0xffffffffu, top > m_ref + kLazy)) {
          const float m_new = fmaxf(m_ref, top);
          const float alpha = m_new == m_ref ? 1.0f : ex2(m_ref - m_new);
          m_ref = m_new;
          sum *= alpha;
          scale_row<HD>(o_addr, alpha);
        }
        const float base = m_ref == -INFINITY ? 0.f : m_ref;
        const uint64_t scale2 = pair_of(__float_as_uint(sl2), __float_as_uint(sl2));
        const uint64_t base2 = pair_of(__float_as_uint(-base), __float_as_uint(-base));
        uint64_t acc[2] = {0, 0};
        // in place: the pair at 2 i becomes entry i
#pragma unroll
        for (int h = 0; h < 2; ++h) {
#pragma unroll
          for (int i = 32 * h; i < 32 * h + 32; ++i) {
            const float2 e = floats_of(fma2(pair_of(v[2 * i], v[2 * i + 1]), scale2, base2));
            const float x = ex2(e.x), y = ex2(e.y);
            acc[i & 1] = add2(acc[i & 1], pair_of(__float_as_uint(x), __float_as_uint(y)));
            v[i] = Num<T>::pack(x, y);
          }
          tm_st32(s_addr + 32 * h, v + 32 * h);
        }
        tm_wait_st();
        const float2 acc2 = floats_of(add2(acc[0], acc[1]));
        sum += acc2.x + acc2.y;
        if (tail) {  // the stage is not refilled before this group's probabilities are used
          const int st = (tile0 + j) % NV;
          ok = warp_wait(sh.fixed + st, ((tile0 + j) / NV) & 1, abort_flag);
          if (!ok) break;
          patch |= sh.odd[st] != 0;
        }
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(sh.p_full + g);
      }
      if (!ok) break;
      ok = warp_wait(sh.o_full + g, ph_o, abort_flag);
      if (!ok) break;
      ph_o ^= 1;
      tc_fence_after();
      // ---- epilogue: a group's own accumulator, or half the columns of both groups' ----
      float w0 = 1.f, w1 = 0.f;
      if (BLOCKS == 1) {
        float4* ml = reinterpret_cast<float4*>(qbuf);  // the queries have been read
        ml[g * kTile + t] = make_float4(m_ref, sum, patch ? 1.f : 0.f, 0.f);
        meet();
        if (!ok) break;
        const float4 x = ml[t], y = ml[kTile + t];
        patch = x.z + y.z > 0.f;
        m_ref = fmaxf(x.x, y.x);
        w0 = x.x == -INFINITY ? 0.f : ex2(x.x - m_ref);
        w1 = y.x == -INFINITY ? 0.f : ex2(y.x - m_ref);
        sum = x.y * w0 + y.y * w1;
      }
      constexpr int kCols = BLOCKS == 2 ? HD : HD / 2;
      const int col0 = BLOCKS == 2 ? 0 : g * kCols, in_block = (BLOCKS == 2 ? g * kTile : 0) + t;
      const bool whole = w.t0 == 0 && w.t1 == w.s.tiles, on = row < rows;
      // A unit's contributors are consecutive CTAs.  All but the last to arrive
      // leave their partial; that one joins them, in tile order.  Where two share
      // a unit, the last joins the other's partial with what it still has in
      // tensor memory; one that finds the other there already, as the owner of a
      // unit's first tile does as a rule (in ranges it came to it last of all its
      // work), leaves no partial of its own.
      const int count = whole ? 1 : w.count, me = w.me, c0 = w.c0;
      uint32_t* arrived = reinterpret_cast<uint32_t*>(a.workspace) + 2 * c0 + g;
      const Partial mine = slot_of(a, 2 * (c0 + me) + (w.t0 > 0 ? 0 : 1), HD, BLOCKS);
      bool two = false, finish = whole;  // this CTA writes the unit's output
      if (count == 2) {
        if (t == 0) sh.last_in[g] = last_of(ld_acquire(arrived), count);
        group_meet();
        if (!ok) break;
        two = finish = sh.last_in[g] != 0;
        patch |= sh.last_in[g] == 2;
      }
      T* out = reinterpret_cast<T*>(a.out) +
               (((int64_t)w.b * a.width + node) * a.n_q_heads + (int64_t)w.head * group + (row - node * group)) * HD;
      if (!two) {
        const float inv = sum > 0.f ? 1.0f / sum : 0.f;
#pragma unroll 1
        for (int c = col0; c < col0 + kCols; c += 32) {
          uint32_t o[32];
          own_columns<HD, BLOCKS>(o, my + 2 * kTile + (BLOCKS == 2 ? g * HD : 0) + c, w0, n > 1 ? w1 : 0.f, n > 1);
          if (!on) continue;
          if (whole) {
            store_columns<T>(out + c, o, inv, wide_out);
          } else {
#pragma unroll
            for (int i = 0; i < 8; ++i)
              *mine.o(c / 4 + i, in_block) = make_float4(__uint_as_float(o[4 * i]), __uint_as_float(o[4 * i + 1]),
                                                         __uint_as_float(o[4 * i + 2]), __uint_as_float(o[4 * i + 3]));
          }
        }
        if (!whole) {
          *mine.stats(HD, g, in_block) = make_float2(m_ref, sum);
          // written before the group meets, read after, and written again only when
          // all of it has been through another tile
#pragma unroll 1
          for (int i = t; i < count; i += kTile)
            sh.slots[g][i] = (uint16_t)(2 * (c0 + i) + (i == 0 ? 1 : 0));
          fence_gpu();
          group_meet();
          if (!ok) break;
          if (t == 0) sh.last_in[g] = last_of(arrive_acq_rel(arrived, patch), count);
          group_meet();
          if (!ok) break;
          patch |= sh.last_in[g] == 2;
          finish = sh.last_in[g] != 0;
          if (finish) {
            if (count == 2) {
              two = true;
            } else {
              fence_gpu();
              T* unit = reinterpret_cast<T*>(a.out) + ((int64_t)w.b * a.width * a.n_q_heads + (int64_t)w.head * group) * HD;
              const int live = min(kTile, rows - row_base);
              join<T, HD, BLOCKS>(a, sh.slots[g], count, g, t, in_block - t, live, col0 / 4, kCols / 4, unit, row_base);
              if (t == 0) *arrived = 0;  // as the next call wants it
            }
          }
        }
      }
      if (two) {
        const Partial other = slot_of(a, 2 * (c0 + 1 - me) + me, HD, BLOCKS);
        join_two<T, HD, BLOCKS>(other, my + 2 * kTile + (BLOCKS == 2 ? g * HD : 0), g, in_block, me == 0, m_ref, sum, w0,
                                n > 1 ? w1 : 0.f, n > 1, col0, on, out, wide_out);
        if (t == 0) *arrived = 0;
      }
      if (finish && patch) {
        group_meet();  // a row may have been joined by other threads
        if (!ok) break;
        patch_row<T, HD, BLOCKS>(a, w, g, t);
      }
      if (BLOCKS == 1) {  // the queries' place holds the sums, and each group reads both accumulators
        meet();
        if (!ok) break;
      }
      tile0 += n;
    }
    if (!ok) *abort_flag = 1;
  }
  tc_fence_before();
  __syncthreads();
  if (warp == 1) tmem_dealloc(tmem, 512);
  if (*abort_flag || stalled) {
    // A wait ran out, now or in an earlier call with this workspace (whose
    // arrivals are then not to be trusted): every unit of the range becomes NaN,
    // never numbers that look right, until the workspace is zeroed again.
    if (tid == 0) {
      reinterpret_cast<volatile uint32_t*>(a.workspace)[kStalledWord] = 1;
      w.left = one_part ? had_part : hi - lo;
      if (!one_part) {
        w.b = hi > lo ? sh.start_b : 0;
        w.off = hi > lo ? sh.start_off : 0;
        w.at = lo - w.off;
        w.load(a, sh.seq, kRows);
      }
    }
    __syncthreads();
    const Walk& u = sh.walk[0];
    while (true) {
      __syncthreads();
      if (tid == 0) sh.odd[0] = sh.walk[0].next(a, sh.seq, kRows, ranges, one_part);
      __syncthreads();
      if (!sh.odd[0]) break;
#pragma unroll 1
      for (int r = u.block * kRows + tid; r < min((u.block + 1) * kRows, u.s.nodes * group); r += kTaThreads) {
        const int node = r / group;
        T* out = reinterpret_cast<T*>(a.out) +
                 (((int64_t)u.b * a.width + node) * a.n_q_heads + (int64_t)u.head * group + (r - node * group)) * HD;
#pragma unroll 1
        for (int e = 0; e < HD; e += 2) *reinterpret_cast<uint32_t*>(out + e) = 0x7FFF7FFFu;
      }
    }
  }
}

namespace {

int query_blocks(int width, int group) { return width * group <= kTile ? 1 : 2; }

template <typename T, int HD, int BLOCKS>
void run_attention(const TreeAttnArgs& a, cudaStream_t s) {
  constexpr int smem = smem_bytes<HD, BLOCKS>();
  auto* kernel = tree_attention_kernel<T, HD, BLOCKS>;
  static OncePerDevice ctas;
  const int dev = current_device(), sms = ctas.get(dev, [&] {
    allow_shared(kernel, smem);
    int n = 0;
    const cudaError_t e = cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev);
    if (e != cudaSuccess) throw e;
    return n;
  });
  const int grid = sms < kMaxGrid ? sms : kMaxGrid;
  const CUtensorMap km = cache_map(a, a.k_cache), vm = cache_map(a, a.v_cache);
  launch_in_turn(kernel, dim3(grid), kTaThreads, smem, 0, s, a, km, vm);
}

template <typename T>
void run_typed(const TreeAttnArgs& a, cudaStream_t s) {
  const bool one = query_blocks(a.width, a.n_q_heads / a.n_kv_heads) == 1;
  if (a.head_dim == 128) {
    if (one) run_attention<T, 128, 1>(a, s); else run_attention<T, 128, 2>(a, s);
  } else {
    if (one) run_attention<T, 64, 1>(a, s); else run_attention<T, 64, 2>(a, s);
  }
}

}  // namespace

int64_t tree_attention_places(int batch, int width, int n_q_heads, int n_kv_heads, int max_pages) {
  const int group = n_q_heads / n_kv_heads, rows = kTile * query_blocks(width, group);
  const int64_t blocks = ((int64_t)width * group + rows - 1) / rows, tiles = ((int64_t)max_pages * kPageTok + kTile - 1) / kTile;
  return batch * blocks * n_kv_heads * (tiles + kStart);
}

size_t tree_attention_workspace(int, int width, int n_q_heads, int n_kv_heads, int head_dim) {
  return kArriveBytes + 2 * kMaxGrid * slot_floats(head_dim, query_blocks(width, n_q_heads / n_kv_heads)) * sizeof(float);
}

void launch_tree_attention(const TreeAttnArgs& a, cudaStream_t s) {
  if (a.dtype == DT_BF16) run_typed<__nv_bfloat16>(a, s); else run_typed<__half>(a, s);
}

}  // namespace pard
