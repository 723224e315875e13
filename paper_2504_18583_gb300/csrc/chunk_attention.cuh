// Attention of a chunk of new tokens a sequence over the paged cache:
//   o_i = sum_j softmax_j(s q_i . k_j) v_j    over j <= p_i, and, with a window w,
//                                             p_i - j < w or j < sinks
// p_i = ctx + i the token's position; its own keys are in the cache already.
// Both products on tcgen05 with the accumulators in tensor memory, one pass over
// the keys with a running maximum and sum.
//
// A unit is a block of up to 128 or 256 consecutive query vectors (tokens x the
// query heads that share a key/value head) of one sequence and the tiles of 128
// keys that any of its rows sees: those of the first tokens that stay visible,
// then those from the first row's window to the last row's position.  All units'
// tiles in order (sequence, head, block) are cut into one even range a CTA, or,
// where there are no more units than CTAs and a block a sequence, each CTA takes
// one equal part of one unit.  CTAs work that out from the sequences' lengths,
// which the host need not know.  Parts of a unit leave partials in the workspace
// and the last to arrive joins them, in tile order.
//
// Warp 0 loads keys and queries and warp 2 values, by tensor copies of a page's 16
// tokens; warp 1 issues the products; warp 3 works out the CTA's next segments
// (parts of units) while the others are at this one, and looks over values that not
// every row sees.  Two warpgroups take the softmax, a thread a row, half a tile (64
// keys) at a time, so that the first half's product runs under the second's softmax;
// probabilities go over the scores in tensor memory.  With more than 128 query
// vectors each group has its own 128 of them and a buffer of scores, and one group's
// products run under the other's softmax; else both have the same rows and a half of
// each tile (their sums are joined at the end), and the scores of the next tile but
// one are asked for as soon as a buffer is free.
//
// Masks touch only tiles that some row does not see whole: a row sees a run of
// columns up to its own position, less those between the first tokens and its
// window.  There values may hold anything: what lies past the last key that a tile is
// read for, and infinities and NaN of keys that not every row sees, are zeroed in
// shared memory, and the CTA that writes a unit's output adds the latter back for the
// rows that see them.
//
// An 8-bit cache (e4m3 codes, a power of two a token and head) is loaded as it lies
// into rings of its own, and four more warps turn each tile into fp16 operands, exactly
// (down to 2^-24, and held to 65504), so that everything behind them is as for a
// 16-bit cache.  Queries and probabilities are then fp16 too, whatever the queries'
// type: bf16 queries are scaled row by row by a power of two that the softmax's scale
// takes back.
//
// What bounds it, as measured with the tiles in steady state:
// - Long chunks, 256 query vectors a unit: a tile of 128 keys takes 2950 to 3140 clocks,
//   its 32 products 2052 of them and the softmax of both groups, eight warps, nearly all
//   the others': scores wait for the probabilities that lie where they go.  The clock
//   falls to 1.8 GHz under the power limit.  2048 tokens behind 30000 (64 heads on 8 of
//   128): 1.40 ms, 1.49 PFLOP/s, 1.58 ms in a long run.  A prompt of 8191: 401 us, 412 in
//   a long run.
// - Units' ends: 7000 to 8000 clocks from a unit's last scores to the next one's first
//   probabilities.  Four pieces of up to 512 tokens: 70 us; 16 sequences, most of them
//   single tokens, with a window (heads of 64): 52 us, 2800 to 3600 clocks a tile, where
//   masked tiles are many.
// - Single tokens, 16-bit cache: HBM.  32 of them over 264000 keys: 179 us, 90% of the
//   copy rate.
// - 8-bit cache: the chain copy -> conversion -> products, two tiles deep, which is what
//   fits beside the 16-bit operands: 2800 clocks a pair of tiles, where HBM would take
//   1400 and shared memory, which has the bytes four times, 1800.  No unit is full: shared
//   memory's pipe 32%, issue slots 41%, tensor pipe 34%, HBM 37%.  32 single tokens 192 us,
//   more than from a 16-bit cache; 1000 tokens behind 16001 276 us, 214 from a 16-bit one.
// - A single token with a window of 2048: 14.5 us, the chain lengths -> shares -> pages ->
//   keys -> softmax -> partial -> join, 28000 clocks.
//
// Tried and slower: 64-column score products (2048 tokens behind 30000: 1417 -> 1631 us),
// two threads a row (2075), the maximum only where the sum grows too large (8191 tokens:
// 471 -> 540), a third buffer of scores for heads of 64 (a prompt of 4096: 108 -> 119),
// the second group's products left out where it has no rows (8191 tokens: 402 -> 413),
// eight converting warps, codes turned by integer instructions (204 -> 240) or half of them
// (222); without any arithmetic the conversion takes as long.
// (A header, since 16-bit and 8-bit caches are compiled apart: a function that is
// not inlined is given the registers of the kernels that call it, and those have 168
// and 128.)
#pragma once

#include "attn_tc.cuh"
#include "serve.h"

namespace pard {

namespace {

constexpr int kSeqHeld = 64;                    // sequences whose lengths a CTA keeps at hand
constexpr int kStep = kTile / 2;                // keys of a step
// What a unit's start, and splitting it, costs in tiles.  (2 and 6: four ragged pieces 73 us instead of 70.5; but 1000 tokens
// behind 16001 202 instead of 213, in an 8-bit cache 268 instead of 276; others within 1%.)
constexpr int kUnitStart = 3, kUnitSplit = 4;
using ChunkRanges = RangesOf<kUnitSplit>;
constexpr int kConvWarps = 4;                   // warps that convert an 8-bit cache's tiles

constexpr int kAheadSegs = 4;                   // segments that are worked out ahead

__host__ __device__ constexpr int chunk_threads(bool q8) { return q8 ? 384 + 32 * kConvWarps : 384; }
// Tiles of keys, and of values, in shared memory beside the queries; of an 8-bit
// cache also as they lie, on their way into those.
__host__ __device__ constexpr int ck_stages(int hd, int blocks, bool q8) {
  return q8 ? (hd == 128 ? 2 : 3) : hd == 128 ? (blocks == 1 ? 3 : 2) : (blocks == 1 ? 6 : 5);
}
__host__ __device__ constexpr int cv_stages(int hd, int blocks, bool q8) {
  return q8 ? (hd == 128 ? 2 : 3) : hd == 128 ? 3 : (blocks == 1 ? 6 : 5);
}
__host__ __device__ constexpr int raw_stages(int hd, int blocks, bool q8) { return !q8 ? 0 : hd == 128 ? (blocks == 1 ? 2 : 1) : 4; }

// A sequence of the batch.
struct Chunk {
  int ctx, n, row0, keys, rows, blocks;  // keys: that the page table has room for; rows: query vectors a key/value head
};
__device__ __forceinline__ Chunk chunk_of(const ChunkAttnArgs& a, int ctx, int from, int to, int rows_per_block) {
  Chunk s;
  s.row0 = min(max(from, 0), a.n_tokens);
  s.n = max(min(max(to, 0), a.n_tokens) - s.row0, 0);
  s.ctx = min(max(ctx, 0), 1 << 30);
  const int64_t end = (int64_t)s.ctx + s.n, most = (int64_t)a.max_pages * kPageTok;
  s.keys = (int)(end < most ? end : most);
  s.rows = s.n * a.group;
  s.blocks = (s.rows + rows_per_block - 1) / rows_per_block;
  return s;
}
// n / group for rows of a block counted from a token's first: n below group + 256
__device__ __forceinline__ int in_group(const ChunkAttnArgs& a, int n) { return a.group_magic ? (int)__umulhi((uint32_t)n, a.group_magic) : n; }
// n / group for any n: the product passes the quotient by less than one
__device__ __forceinline__ int token_of(const ChunkAttnArgs& a, int n) {
  const int q = in_group(a, n);
  return q * a.group > n ? q - 1 : q;
}
// One block's positions and tiles: tiles [0, sink) then [sink + skip, sink + skip + tiles - sink).
struct Span {
  int token, rest;        // of the first row: its token in the chunk, and its place among that one's rows
  int p_lo, p_hi, end;    // first and last row's positions; keys that the last row may see
  int sink, skip, tiles;
  __device__ __forceinline__ int tile(int k) const { return k < sink ? k : k + skip; }
  // keys up to which a tile is looked at: of the first tokens', those
  __device__ __forceinline__ int limit(const ChunkAttnArgs& a, int k) const { return k < sink ? min(a.sinks, end) : end; }
};
__device__ __forceinline__ int window_from(const ChunkAttnArgs& a, int p) { return a.window ? max(0, p - a.window + 1) : 0; }
__device__ __forceinline__ Span span_of(const ChunkAttnArgs& a, const Chunk& s, int block, int rows_per_block) {
  Span g;
  const int r0 = block * rows_per_block;
  g.token = token_of(a, r0);
  g.rest = r0 - g.token * a.group;
  g.p_lo = s.ctx + g.token;
  g.p_hi = g.p_lo + in_group(a, g.rest + min(rows_per_block, s.rows - r0) - 1);
  g.end = min(g.p_hi + 1, s.keys);
  const int last = (g.end + kTile - 1) / kTile;  // tiles up to the end (one at least: a table has a page)
  const int first = min(window_from(a, g.p_lo) / kTile, last - 1);
  g.sink = min((min(a.sinks, g.end) + kTile - 1) / kTile, first);
  g.skip = first - g.sink;
  g.tiles = last - g.skip;
  if (g.skip == 0) g.sink = 0;
  return g;
}
// every row of the positions [lo, hi] sees these keys
__device__ __forceinline__ bool all_see(const ChunkAttnArgs& a, const Chunk& s, int lo, int hi, int key0, int key1) {
  return key1 <= min(lo + 1, s.keys) && (window_from(a, hi) <= key0 || key1 <= a.sinks);
}

// A segment, part of a unit: tiles [t0, t1) (none: there are no more).
struct Segment {
  Chunk s;
  Span g;
  int b, head, block, t0, t1;
  int count, me, c0;   // the unit's contributors, this CTA's place among them, the first of them (among CTAs with a place)
};
// The walk over a CTA's share, one segment after the other, in shared memory.
struct ChunkWalk : Segment {
  int left;            // places to go; in the one-part form 1, then 0
  int off;             // place within the unit
  int at;              // place of the whole pass where the unit begins
  __device__ __forceinline__ void load(const ChunkAttnArgs& a, const int2* held, int rows_per_block) {
    if (b < kSeqHeld) s = chunk_of(a, held[b].x, held[b].y, held[b + 1].y, rows_per_block);
    else s = chunk_of(a, a.ctx_len[b], a.starts[b], a.starts[b + 1], rows_per_block);
  }
  __device__ __noinline__ bool next(const ChunkAttnArgs& a, const int2* held, int rows_per_block, const ChunkRanges& ranges,
                                    bool one_part) {
    if (one_part) return left-- > 0;
    while (left > 0) {
      const int len = g.tiles + kUnitStart;
      if (off >= len) {  // the next unit
        at += len;
        off = 0;
        if (++block >= s.blocks) {
          block = 0;
          if (++head >= a.n_kv_heads) {
            head = 0;
            do {
              if (++b >= a.batch) return false;
              load(a, held, rows_per_block);
            } while (s.blocks == 0);
          }
        }
        g = span_of(a, s, block, rows_per_block);
        continue;
      }
      const int x0 = ChunkRanges::cut(off, len), x1 = off + left < len ? ChunkRanges::cut(off + left, len) : len;
      const int step = min(len - off, left);
      off += step;
      left -= step;
      t0 = max(0, x0 - kUnitStart);
      t1 = x1 - kUnitStart;
      if (t1 <= t0) continue;
      count = 1;
      me = 0;
      c0 = blockIdx.x;
      if (t0 > 0 || t1 < g.tiles) {  // who else has a part of it
        while (c0 > 0 && ranges.at(c0) > at && ChunkRanges::cut(ranges.at(c0) - at, len) > 0) --c0;
        int c1 = blockIdx.x;
        while (c1 + 1 < ranges.grid && ranges.at(c1 + 1) < at + len && ChunkRanges::cut(ranges.at(c1 + 1) - at, len) < len) ++c1;
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

// The lowest n of 32 bits.
__device__ __forceinline__ uint32_t low_bits(int n) { return n >= 32 ? 0xFFFFFFFFu : n <= 0 ? 0u : (1u << n) - 1u; }
// 32 columns, the first of them key `key`, that a row sees: up to `end`, from `from` on or before `sinks`.
__device__ __forceinline__ uint32_t seen32(int key, int end, int from, int sinks) {
  return low_bits(end - key) & (~low_bits(from - key) | low_bits(sinks - key));
}

// The type of the products' operands: an 8-bit cache's entries are made fp16 ones
// whatever the queries' type.
template <typename T, bool Q8> struct OperandOf { using type = T; };
template <typename T> struct OperandOf<T, true> { using type = __half; };

// A value's entry, of a 16-bit cache or an 8-bit one.
template <typename T, int HD, bool Q8>
__device__ __forceinline__ float value_at(const ChunkAttnArgs& a, int64_t page, int head, int tok, int c) {
  if (!Q8)
    return Num<T>::get(reinterpret_cast<const T*>(a.v_cache) + page * a.page_stride + ((int64_t)head * kPageTok + tok) * HD + c);
  const uint32_t code = reinterpret_cast<const uint8_t*>(a.v_cache)[page * a.page_stride + ((int64_t)head * kPageTok + tok) * HD + c];
  const uint32_t e = a.v_scale[page * a.scale_stride + (int64_t)head * kPageTok + tok];
  return (code & 0x7F) == 0x7F || e == 255u ? __int_as_float(0x7FFFFFFF) : 0.f;  // (finite: as an operand it is held to 65504)
}

// Adds the infinities and NaN of a unit's values that not every row of the block
// sees back to the output of the row that has thread t of group g, where it sees
// them: they stay what they are there.
template <typename T, int HD, int BLOCKS, bool Q8>
__device__ __noinline__ void patch_chunk(const ChunkAttnArgs& a, const Segment& w, int g, int t) {
  constexpr int cols = BLOCKS == 2 ? HD : HD / 2;
  const int r = (BLOCKS == 2 ? g * kTile : 0) + t, col0 = BLOCKS == 2 ? 0 : g * cols;
  if (w.block * BLOCKS * kTile + r >= w.s.rows) return;
  const int in_token = in_group(a, w.g.rest + r), token = w.g.token + in_token, p = w.s.ctx + token;
  const int end = min(p + 1, w.s.keys), from = window_from(a, p);
  T* out = reinterpret_cast<T*>(a.out) +
           (((int64_t)w.s.row0 + token) * a.n_q_heads + (int64_t)w.head * a.group + (w.g.rest + r - in_token * a.group)) * HD;
  for (int k = 0; k < w.g.tiles; ++k) {
    const int k0 = w.g.tile(k) * kTile;
    if (all_see(a, w.s, w.g.p_lo, w.g.p_hi, k0, k0 + kTile)) continue;
    for (int pos = k0; pos < min(k0 + kTile, end); ++pos) {
      if ((pos < from && pos >= a.sinks) || all_see(a, w.s, w.g.p_lo, w.g.p_hi, pos, pos + 1)) continue;
      const int page = page_of(a.page_table + (size_t)w.b * a.max_pages, pos, a.max_pages, a.n_pages);
      if (page < 0) continue;
#pragma unroll 1
      for (int c = col0; c < col0 + cols; ++c) {
        const float x = value_at<T, HD, Q8>(a, page, w.head, pos % kPageTok, c);
        if (fabsf(x) < INFINITY) continue;
        const uint32_t y = Num<T>::pack(Num<T>::get(out + c) + x, 0.f);
        *reinterpret_cast<uint16_t*>(out + c) = (uint16_t)y;
      }
    }
  }
}

// A unit of up to eight rows (a single token's, as a rule in many parts) leaves its
// partials row by row, and a warp joins a row: its lanes take the parts' maxima and sums
// (32 at a time) and then the row's columns, in 32 / kCols4 shares of the parts that are
// added up last.  (With O as [HD / 4][rows], a row's pieces 2048 bytes apart, sixteen
// parts of four rows took 5000 clocks to load.)
constexpr int kFewRows = 8;
template <int HD>
__device__ __forceinline__ Partial few_rows(Partial p) {
  p.c4_step = 1;
  p.row_step = HD / 4;
  return p;
}
template <typename T, int HD, int BLOCKS>
__device__ __noinline__ void join_few(const Partial first, const uint16_t* slots, int count, int g, int t, int row0, int rows,
                                      int c4_0, T* out, int row_in_token, int group, int64_t token_step) {
  constexpr int kCols4 = HD / 4 / (BLOCKS == 1 ? 2 : 1), kShares = 32 / kCols4, kBatch = 8;
  constexpr int64_t kSlot = slot_floats(HD, BLOCKS);
  const int lane = t & 31, c = lane % kCols4, share = lane / kCols4;
#pragma unroll 1
  for (int row = t >> 5; row < rows; row += 4) {
    float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
    float m = -INFINITY, l = 0.f;
    const float4* o = few_rows<HD>(first).o(c4_0 + c, row0 + row);
#pragma unroll 1
    for (int i0 = 0; i0 < count; i0 += 32) {
      const int n = min(32, count - i0), slot = lane < n ? slots[i0 + lane] : 0;
      float2 st = make_float2(-INFINITY, 0.f);
      if (lane < n) st = *reinterpret_cast<const float2*>(reinterpret_cast<const float*>(first.stats(HD, g, row0 + row)) + slot * kSlot);
      float4 v[kBatch];
      auto load = [&](int i) {
#pragma unroll
        for (int e = 0; e < kBatch; ++e) {
          const int at = i + e * kShares + share, from = __shfl_sync(0xffffffffu, slot, at & 31);
          v[e] = make_float4(0.f, 0.f, 0.f, 0.f);
          if (at < n) v[e] = o[from * (kSlot / 4)];
        }
      };
      load(0);
      float top = fmaxf(m, st.x), sum;
#pragma unroll
      for (int d = 16; d > 0; d >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, d));
      const float base = top == -INFINITY ? 0.f : top, old = ex2(m - base), w = ex2(st.x - base);
      sum = st.y * w;
#pragma unroll
      for (int d = 16; d > 0; d >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
      l = l * old + sum;
      m = top;
      acc.x *= old; acc.y *= old; acc.z *= old; acc.w *= old;
#pragma unroll 1
      for (int i = 0; i < n; i += kShares * kBatch) {
        if (i > 0) load(i);
#pragma unroll
        for (int e = 0; e < kBatch; ++e) {
          const float by = __shfl_sync(0xffffffffu, w, (i + e * kShares + share) & 31);
          acc.x = fmaf(v[e].x, by, acc.x);
          acc.y = fmaf(v[e].y, by, acc.y);
          acc.z = fmaf(v[e].z, by, acc.z);
          acc.w = fmaf(v[e].w, by, acc.w);
        }
      }
    }
#pragma unroll
    for (int d = kCols4; d < 32; d <<= 1) {
      acc.x += __shfl_xor_sync(0xffffffffu, acc.x, d);
      acc.y += __shfl_xor_sync(0xffffffffu, acc.y, d);
      acc.z += __shfl_xor_sync(0xffffffffu, acc.z, d);
      acc.w += __shfl_xor_sync(0xffffffffu, acc.w, d);
    }
    const float inv = l > 0.f ? 1.0f / l : 0.f;
    const int r = row_in_token + row, token = r / group;
    uint2 p;
    p.x = Num<T>::pack(acc.x * inv, acc.y * inv);
    p.y = Num<T>::pack(acc.z * inv, acc.w * inv);
    if (share == 0) *reinterpret_cast<uint2*>(out + token * token_step + (r - token * group) * HD + (c4_0 + c) * 4) = p;
  }
}

// ---- 8-bit entries into 16-bit ones -------------------------------------------
// A row's codes times its power of two, as fp16.  The conversion gives codes as they
// are (NaN too), and the product with a power of two from 2^-14 to 2^7 stays a normal
// fp16 power of two's, exact down to 2^-24; beyond that it is taken in 32 bits and
// held to 65504.  (As bf16, with the bits moved and two products, an entry took three
// times the instructions, and the tiles of 128 keys 14000 clocks against HBM's 1400.)
struct Widen {
  uint32_t m;
  float s;
  // one of four exponents is below 113 or above 134
  __device__ __forceinline__ static uint32_t far4(uint32_t e) { return __vcmpltu4(e, 0x71717171u) | __vcmpgtu4(e, 0x86868686u); }
  __device__ __forceinline__ void set(uint32_t e) { m = (e - 112u) * 0x04000400u; }
  __device__ __forceinline__ void set_far(uint32_t e) {
    s = e == 255u ? __int_as_float(0x7FFFFFFF) : __uint_as_float(e ? e << 23 : 1u << 22);
  }
  static __device__ __forceinline__ uint32_t codes(uint32_t two) {
    uint32_t v;
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(v) : "h"((uint16_t)two));
    return v;
  }
  __device__ __forceinline__ uint32_t near_two(uint32_t two) const {
    const uint32_t x = codes(two);
    const __half2 p = __hmul2(*reinterpret_cast<const __half2*>(&x), *reinterpret_cast<const __half2*>(&m));
    return *reinterpret_cast<const uint32_t*>(&p);
  }
  __device__ __forceinline__ uint32_t far_two(uint32_t two) const {
    const uint32_t h = codes(two);
    const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&h));
    auto held = [&](float x) { x *= s; return x > 65504.f ? 65504.f : x < -65504.f ? -65504.f : x; };  // (NaN stays)
    return Num<__half>::pack(held(f.x), held(f.y));
  }
};

// What a CTA keeps in shared memory behind the operands.
template <int NK, int NV, int NR>
struct ChunkControl {
  static constexpr bool Q8 = NR > 0;
  uint64_t k_full[NK], k_empty[NK], v_full[NV], v_empty[NV];  // stages (8-bit: v_full unused)
  uint64_t fixed[NV];      // a stage's values are fit for the product
  uint64_t raw_full[2][NR + 1], raw_empty[2][NR + 1];         // keys', values' codes
  uint64_t s_full[2];      // a tile's scores are in one of the two buffers
  uint64_t p_full[2][2];   // the probabilities of one of its halves are, and O is scaled
  uint64_t o_full[2][2];   // two blocks: a group's product with a tile's first half is done, with all of a segment's;
                           // one: the product with its probabilities of a buffer is
  uint64_t ready[2];       // the group has read O of the segment before
  uint64_t q_full, q_free; // a segment's queries are there; one block: their place is no longer read
  uint64_t seg_full[kAheadSegs], seg_free[kAheadSegs];
  uint64_t pair, met[2];   // the two groups meet, a group's warps do
  uint64_t drain;          // every product is done
  alignas(16) uint8_t scale[2][Q8 ? NR * kTile : 16];  // of the codes
  uint8_t far[2][NR + 1];  // a tile of keys or values has one that Widen::far4() tells (what lies past the last key counts)
  uint8_t back[Q8 ? 2 * kTile : 16];  // exponents of the queries' rows, which were scaled by them
  int2 seq[kSeqHeld + 1];  // sequences' context lengths and first rows
  uint32_t tmem, last_in[2], odd[NV];  // odd: a stage's values that not all rows see held infinities or NaN (a byte a warp)
  int odd_in[2];           // the last segment, counted from 1, in which a group met such
  uint8_t pages[16];       // which of a tile's pages are the pool's, tiles in turn: keys are loaded fewer than 16 ahead of the softmax
  int abort_flag, start_b, start_head, start_block, start_off;
  int sum[16], units[16], most[16];
  ChunkWalk walk;
  Segment seg[kAheadSegs];
  union {
    int tiles[kSeqHeld];            // of a sequence's block, where it has one: until the segments are worked out
    uint16_t slots[2][kMaxGrid];
  };
};
template <int HD, int BLOCKS, bool Q8>
constexpr int chunk_smem() {
  constexpr int nk = ck_stages(HD, BLOCKS, Q8), nv = cv_stages(HD, BLOCKS, Q8), nr = raw_stages(HD, BLOCKS, Q8);
  return (BLOCKS + nk + nv + nr) * stage_bytes(HD) + (int)sizeof(ChunkControl<nk, nv, nr>);
}
static_assert(chunk_smem<128, 1, false>() <= 227 * 1024 && chunk_smem<128, 2, false>() <= 227 * 1024, "shared memory of one CTA");
static_assert(chunk_smem<64, 1, false>() <= 227 * 1024 && chunk_smem<64, 2, false>() <= 227 * 1024, "shared memory of one CTA");
static_assert(chunk_smem<128, 1, true>() <= 227 * 1024 && chunk_smem<128, 2, true>() <= 227 * 1024, "shared memory of one CTA");
static_assert(chunk_smem<64, 1, true>() <= 227 * 1024 && chunk_smem<64, 2, true>() <= 227 * 1024, "shared memory of one CTA");

// orders this thread's accesses to shared memory with copies' and products' ones
__device__ __forceinline__ void fence_proxy_shared() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }

__device__ __forceinline__ void tma_load_3d(void* dst, const CUtensorMap* m, uint64_t* bar, int c0, int c1, int c2) {
  asm volatile(
      "cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];" ::"r"(
          smem_u32(dst)),
      "l"(reinterpret_cast<uint64_t>(m)), "r"(c0), "r"(c1), "r"(c2), "r"(smem_u32(bar))
      : "memory");
}

}  // namespace

// by_tma: queries come by tensor copies (qmap), else by the softmax warps' loads
template <typename T, int HD, int BLOCKS, bool Q8>
__global__ void __launch_bounds__(chunk_threads(Q8), 1)
    chunk_attention_kernel(const __grid_constant__ ChunkAttnArgs a, const __grid_constant__ CUtensorMap kmap,
                           const __grid_constant__ CUtensorMap vmap, const __grid_constant__ CUtensorMap qmap) {
  constexpr int NK = ck_stages(HD, BLOCKS, Q8), NV = cv_stages(HD, BLOCKS, Q8), NR = raw_stages(HD, BLOCKS, Q8);
  constexpr int kStage = stage_bytes(HD), kRaw = kStage / 2, kConsumers = Q8 ? 11 + kConvWarps : 11;
  constexpr int kChunks = HD / 64, kChunkBytes = kTile * 128, kRows = kTile * BLOCKS, kThreads = chunk_threads(Q8);
  using M = typename OperandOf<T, Q8>::type;
  constexpr bool kRaised = Num<T>::kFormat != Num<M>::kFormat;  // bf16 queries become fp16 ones, row by row scaled
  constexpr uint32_t kIdescS = idesc16(Num<M>::kFormat, kTile, kTile, false);
  constexpr uint32_t kIdescO = idesc16(Num<M>::kFormat, kTile, HD, true);
  extern __shared__ __align__(1024) uint8_t qbuf[];  // queries, then the rings
  uint8_t* kring = qbuf + BLOCKS * kStage;
  uint8_t* vring = kring + NK * kStage;
  uint8_t* raw_rings = vring + NV * kStage;  // keys' codes, values' codes
  using Control = ChunkControl<NK, NV, NR>;
  Control& sh = *reinterpret_cast<Control*>(raw_rings + NR * kStage);
  volatile int* abort_flag = &sh.abort_flag;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int group = a.group, grid = gridDim.x;
  const bool by_tma = !Q8 && a.q_by_tma;

  // ---- this CTA's range -------------------------------------------------------
  if (warp == 1) tmem_alloc(&sh.tmem, 512);
  if (tid == 0) {
    tma_prefetch_desc(&kmap);
    tma_prefetch_desc(&vmap);
    if (by_tma) tma_prefetch_desc(&qmap);
#pragma unroll 1
    for (int i = 0; i < NK; ++i) { mbar_init(sh.k_full + i, Q8 ? kConvWarps / 2 : 1); mbar_init(sh.k_empty + i, 1); }
#pragma unroll 1
    for (int i = 0; i < NV; ++i) { mbar_init(sh.v_full + i, 1); mbar_init(sh.v_empty + i, 1); mbar_init(sh.fixed + i, Q8 ? kConvWarps / 2 : 1); sh.odd[i] = 0; }
#pragma unroll 1
    for (int i = 0; i < NR; ++i) {
      mbar_init(sh.raw_full[0] + i, 1); mbar_init(sh.raw_full[1] + i, 1);
      mbar_init(sh.raw_empty[0] + i, kConvWarps / 2); mbar_init(sh.raw_empty[1] + i, kConvWarps / 2);
    }
#pragma unroll 1
    for (int i = 0; i < 2; ++i) {
      mbar_init(sh.s_full + i, 1); mbar_init(sh.p_full[i], 4); mbar_init(sh.p_full[i] + 1, 4);
      mbar_init(sh.o_full[i], 1); mbar_init(sh.o_full[i] + 1, 1); mbar_init(sh.ready + i, 4); mbar_init(sh.met + i, 4);
    }
#pragma unroll 1
    for (int i = 0; i < kAheadSegs; ++i) { mbar_init(sh.seg_full + i, 1); mbar_init(sh.seg_free + i, kConsumers); }
    mbar_init(&sh.q_full, by_tma ? 1 : 8);
    mbar_init(&sh.q_free, 8);
    mbar_init(&sh.pair, 8);
    mbar_init(&sh.drain, 1);
    fence_barrier_init();
    *abort_flag = sh.odd_in[0] = sh.odd_in[1] = 0;
    sh.start_b = sh.start_head = sh.start_block = sh.start_off = 0;  // (starts that decrease may leave them: in bounds then)
  }
  pdl_trigger();
  pdl_wait();
  const uint32_t stalled = reinterpret_cast<const volatile uint32_t*>(a.workspace)[kStalledWord];
  // The share's form and, in ranges, this CTA's first place: two rounds over the
  // sequences, their sum and then the place in it; both are one round of a
  // single step for up to as many sequences as threads.
  ChunkRanges ranges;
  int lo = 0, hi = 0, units = 0, longest = 0;
  bool single = true;  // no sequence has more than one block
#pragma unroll 1
  for (int round = 0; round < 2; ++round) {
    int run = 0;
#pragma unroll 1
    for (int b0 = 0; b0 < a.batch; b0 += kThreads) {
      const int b = b0 + tid;
      int3 v = make_int3(0, 0, 0);
      if (b < a.batch) v = make_int3(a.ctx_len[b], a.starts[b], a.starts[b + 1]);
      if (b < kSeqHeld && b < a.batch) {
        sh.seq[b] = make_int2(v.x, v.y);
        if (b == kSeqHeld - 1 || b == a.batch - 1) sh.seq[b + 1] = make_int2(0, v.z);
      }
      const Chunk s = chunk_of(a, v.x, v.y, v.z, kRows);
      int places = 0, tiles = 0;  // of a head
      if (s.blocks == 1) {
        tiles = span_of(a, s, 0, kRows).tiles;
        places = tiles + kUnitStart;
      }
      for (uint32_t m = __ballot_sync(0xffffffffu, s.blocks > 1); m; m &= m - 1) {  // the warp adds up one's blocks
        const int from = __ffs(m) - 1;
        const Chunk o = chunk_of(a, __shfl_sync(0xffffffffu, v.x, from), __shfl_sync(0xffffffffu, v.y, from),
                                 __shfl_sync(0xffffffffu, v.z, from), kRows);
        int part = 0;
        for (int i = lane; i < o.blocks; i += 32) part += span_of(a, o, i, kRows).tiles + kUnitStart;
        part = __reduce_add_sync(0xffffffffu, part);
        if (lane == from) places = part;
      }
      if (b < kSeqHeld) sh.tiles[b] = tiles;
      const int cost = places * a.n_kv_heads;
      int inc = cost;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const int t = __shfl_up_sync(0xffffffffu, inc, o);
        if (lane >= o) inc += t;
      }
      const int u = __reduce_add_sync(0xffffffffu, a.n_kv_heads * s.blocks);
      const int most = __reduce_max_sync(0xffffffffu, tiles);
      if (lane == 31) { sh.sum[warp] = inc; sh.units[warp] = u; sh.most[warp] = most; }
      single &= !__syncthreads_or(s.blocks > 1);
      const bool is = lane < kThreads / 32;
      const int of = is ? sh.sum[lane] : 0, step = __reduce_add_sync(0xffffffffu, of);
      inc += run + __reduce_add_sync(0xffffffffu, lane < warp ? of : 0);
      units += __reduce_add_sync(0xffffffffu, is ? sh.units[lane] : 0);
      longest = max(longest, __reduce_max_sync(0xffffffffu, is ? sh.most[lane] : 0));
      run += step;
      if (a.batch <= kThreads) {
        ranges.set(run, grid);
        lo = ranges.at(blockIdx.x);
        hi = ranges.at(blockIdx.x + 1);
        round = 1;
      }
      if (round && inc > lo && inc - cost <= lo) {
        const int off = lo - (inc - cost);
        sh.start_b = b;
        sh.start_head = off / places;
        sh.start_off = off % places;
      }
      if (a.batch > kThreads) __syncthreads();  // what the next step writes has been read
    }
    if (!round) {
      ranges.set(run, grid);
      lo = ranges.at(blockIdx.x);
      hi = ranges.at(blockIdx.x + 1);
    }
  }
  const bool one_part = single && a.batch <= kSeqHeld && units <= grid;
  ChunkWalk& w = sh.walk;
  auto begin = [&] {  // the walk in ranges, from its first place
    w.left = hi - lo;  // 0: more CTAs than places
    w.b = hi > lo ? sh.start_b : 0;
    w.head = hi > lo ? sh.start_head : 0;
    w.block = hi > lo ? sh.start_block : 0;
    w.off = hi > lo ? sh.start_off : 0;
    w.at = lo - w.off;
    w.load(a, sh.seq, kRows);
    if (hi > lo) w.g = span_of(a, w.s, w.block, kRows);
  };
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = sh.tmem;
  int tile0 = 0;  // tiles of the segments before this one
  bool ok = true;
  // a warp's next segment: what it has read of the one before may be written over
  int taken = 0;
  auto next = [&]() -> bool {
    __syncwarp();
    if (taken > 0 && lane == 0) mbar_arrive(sh.seg_free + (taken - 1) % kAheadSegs);
    ok = ok && warp_wait(sh.seg_full + taken % kAheadSegs, (taken / kAheadSegs) & 1, abort_flag);
    ++taken;
    return ok && sh.seg[(taken - 1) % kAheadSegs].t1 > 0;
  };
  auto segment = [&]() -> const Segment& { return sh.seg[(taken - 1) % kAheadSegs]; };
  // pages of a tile that hold keys the block may see
  auto pages_of = [&](const Segment& u, int k) { return min(kTilePages, (u.g.limit(a, k) - 1) / kPageTok - u.g.tile(k) * kTilePages + 1); };

  if (warp == 0 || warp == 2) {
    // ---- loads: keys by one warp, values by another ------------------------------------
    // Page ids are fetched 32 pages (four tiles) at a time, a block ahead of
    // their use: a load from the table would be on every copy's path.
    const bool v = warp == 2;
    uint64_t* full = Q8 ? sh.raw_full[v] : (v ? sh.v_full : sh.k_full);
    uint64_t* empty = Q8 ? sh.raw_empty[v] : (v ? sh.v_empty : sh.k_empty);
    uint8_t* to0 = Q8 ? raw_rings + (v ? NR * kRaw : 0) : (v ? vring : kring);
    const CUtensorMap* map = v ? &vmap : &kmap;
    const int ns = Q8 ? NR : v ? NV : NK;
    int st = 0, phase = 0, issued = 0, last = 0;  // stages are used in turn
    int q_out = 0;  // segments whose queries were asked for
    while (next()) {
      const Segment& u = segment();
      const int n = u.t1 - u.t0, head = u.head;
      const int32_t* row = a.page_table + (size_t)u.b * a.max_pages;
      const int last_page = (u.g.end - 1) / kPageTok;
      auto fetch = [&](int block) {
        const int j = 4 * block + lane / kTilePages;
        const int p = j < n ? u.g.tile(u.t0 + j) * kTilePages + lane % kTilePages : last_page + 1;
        const int page = p <= last_page ? row[p] : 0;
        return (uint32_t)page < (uint32_t)a.n_pages ? page : a.n_pages;  // out of the tensor: reads as zeros
      };
      // The segment's queries, once the products of the one before have read theirs:
      // two blocks, when its last scores are there; one, when the softmax no longer
      // uses their place.
      auto queries = [&] {
        if (taken > 1) {
          if (BLOCKS == 1) ok = ok && warp_wait(&sh.q_free, taken & 1, abort_flag);
          else ok = ok && warp_wait(empty + last % ns, (last / ns) & 1, abort_flag);
        }
        if (ok && elect_one()) {
          mbar_arrive_expect_tx(&sh.q_full, BLOCKS * kStage);
#pragma unroll
          for (int i = 0; i < BLOCKS; ++i)
#pragma unroll
            for (int c = 0; c < kChunks; ++c)
              tma_load_3d(qbuf + i * kStage + c * kChunkBytes, &qmap, &sh.q_full, c * 64, head * group,
                          u.s.row0 + u.g.token + i * (kTile / group));
        }
        __syncwarp();
        ++q_out;
      };
      if (!Q8 && by_tma && !v && taken == 1) queries();
      const int last_before = last;
      int have = fetch(0), after = n > 4 ? fetch(1) : 0;
      auto exponents_of = [&](int page) {
        const uint8_t* from = (v ? a.v_scale : a.k_scale) + page * a.scale_stride + (int64_t)head * kPageTok;
        return lane < kTilePages && page < a.n_pages ? __ldg(reinterpret_cast<const uint4*>(from)) : make_uint4(0, 0, 0, 0);
      };
      uint4 exponents = Q8 ? exponents_of(__shfl_sync(0xffffffffu, have, lane & 7)) : make_uint4(0, 0, 0, 0);
#pragma unroll 1
      for (int j = 0; j < n && ok; ++j) {
        const int pages = pages_of(u, u.t0 + j);
        if (j > 0 && (j & 3) == 0) {
          have = after;
          if (j + 4 < n) after = fetch(j / 4 + 1);
        }
        ok = ok && warp_wait(empty + st, phase ^ 1, abort_flag);
        if (!ok) break;
        const uint32_t in_pool = __ballot_sync(0xffffffffu, have < a.n_pages) >> ((j & 3) * kTilePages);
        uint8_t* to = to0 + st * (Q8 ? kRaw : kStage);
        if constexpr (Q8) {
          // codes by tensor copies, 16 bytes of exponents a page through registers, asked
          // for a tile ahead
          uint8_t* scale = sh.scale[v] + st * kTile;
          constexpr int kCodes = HD * kPageTok;
          if (lane < pages) *reinterpret_cast<uint4*>(scale + lane * kPageTok) = exponents;
          const bool far = __any_sync(0xffffffffu, lane < pages && (Widen::far4(exponents.x) | Widen::far4(exponents.y) |
                                                                    Widen::far4(exponents.z) | Widen::far4(exponents.w)));
          if (j + 1 < n) {
            const int ahead = (j + 1) & 3;
            exponents = exponents_of(__shfl_sync(0xffffffffu, ahead == 0 ? after : have, ahead * kTilePages + (lane & 7)));
          }
          int page[kTilePages];
#pragma unroll
          for (int q = 0; q < kTilePages; ++q) page[q] = __shfl_sync(0xffffffffu, have, (j & 3) * kTilePages + q);
          __syncwarp();
          if (elect_one()) {
            if (!v) sh.pages[issued & 15] = (uint8_t)in_pool;
            sh.far[v][st] = far;
            mbar_arrive_expect_tx(full + st, (uint32_t)pages * kCodes);
#pragma unroll
            for (int q = 0; q < kTilePages; ++q)
              if (q < pages) tma_load_4d(to + q * kCodes, map, full + st, 0, 0, head, page[q]);
          }
        } else {
          int page[kTilePages];
#pragma unroll
          for (int q = 0; q < kTilePages; ++q) page[q] = __shfl_sync(0xffffffffu, have, (j & 3) * kTilePages + q);
          if (elect_one()) {
            if (!v) sh.pages[issued & 15] = (uint8_t)in_pool;
            mbar_arrive_expect_tx(full + st, (uint32_t)pages * kChunks * kPageTok * 128);
#pragma unroll
            for (int q = 0; q < kTilePages; ++q)
              if (q < pages) {
#pragma unroll
                for (int c = 0; c < kChunks; ++c)
                  tma_load_4d(to + c * kChunkBytes + q * kPageTok * 128, map, full + st, c * 64, 0, head, page[q]);
              }
          }
        }
        __syncwarp();
        last = issued++;
        if (++st == ns) { st = 0; phase ^= 1; }
        if (!Q8 && by_tma && !v && j == 0 && taken > 1) {  // a tile first: its place came free before the queries'
          const int mine = last;
          last = last_before;
          queries();
          last = mine;
        }
      }
    }
    if (!ok) {  // copies in flight write this CTA's shared memory: they land before it goes
      *abort_flag = 1;
      for (int i = max(0, issued - ns); i < issued; ++i) mbar_drain(full + i % ns, (i / ns) & 1);
      if (q_out) mbar_drain(&sh.q_full, (q_out - 1) & 1);
    }
  } else if (warp == 1) {
    // ---- products ---------------------------------------------------------------------
    // One lane issues, all wait.  A tile takes 32 products (128 columns: 2048 clocks),
    // and what lies between them is the warp's own time, so it is kept short: stages
    // and phases are counted along, addresses made the warp's (by a shuffle: the
    // compiler then keeps them in uniform registers) once a tile, and steps add
    // constants to a descriptor's low word.
    uint32_t ph_p = 0;
    int kst = 0, vst = 0;
    uint32_t kph = 0, vph = 0;
    const uint32_t q_addr = smem_u32(qbuf) >> 4, k_addr = smem_u32(kring) >> 4, v_addr = smem_u32(vring) >> 4;
    const bool leader = elect_one();
    auto uniform = [](uint32_t x) { return __shfl_sync(0xffffffffu, x, 0); };
    const uint32_t tm = uniform(tmem);
    // Shared-memory descriptors, 128-byte swizzle.  Queries and keys: 128-byte
    // rows along K, eight-row atoms 1024 bytes apart.  Values: 64 of a key's
    // entries a row (N is contiguous), atoms of eight keys 1024 bytes apart along
    // K, the next 64 entries a chunk further.
    constexpr uint64_t kDescK = (uint64_t)1 << 16 | (uint64_t)(1024 >> 4) << 32 | (uint64_t)1 << 46 | (uint64_t)2 << 61;
    constexpr uint64_t kDescV = (uint64_t)(kChunkBytes >> 4) << 16 | (uint64_t)(1024 >> 4) << 32 | (uint64_t)1 << 46 | (uint64_t)2 << 61;
    // tensor memory: two buffers of scores (two blocks: a group each; one: tiles in
    // turn), then the groups' accumulators
    auto scores = [&](int x, uint32_t kb) {  // of the keys at kb into buffer x
      const uint32_t qa = q_addr + (BLOCKS == 2 ? x * (kStage >> 4) : 0), d = tm + x * kTile;
      if (leader) {
#pragma unroll
        for (int k = 0; k < HD / 16; ++k) {
          const uint32_t at = ((k / 4) * kChunkBytes + (k % 4) * 32) >> 4;
          umma_ss(d, kDescK | (qa + at), kDescK | (kb + at), kIdescS, k > 0);
        }
        umma_commit(sh.s_full + x);
      }
    };
    // O += P V of half h, whose probabilities are in buffer x.  Keys past the end have
    // probability 0: whole steps of 16 are left out, but for the first, which leaves
    // zeros where there were none yet.
    auto outputs = [&](int g, int x, int h, uint32_t vb, bool first, int keys) {
      const uint32_t o = tm + 2 * kTile + g * HD, p = tm + x * kTile + h * kStep, bit = 2 * x + h;
      ok = ok && warp_wait(&sh.p_full[x][h], ph_p >> bit & 1, abort_flag);
      if (!ok) return;
      ph_p ^= 1u << bit;
      tc_fence_after();
      if (leader) {
        umma_ts(o, p, kDescV | (vb + h * 4 * 128), kIdescO, !first);
        if (keys >= (h + 1) * kStep) {
#pragma unroll
          for (int k = 1; k < kStep / 16; ++k) umma_ts(o, p + k * 8, kDescV | (vb + (h * 4 + k) * 128), kIdescO, 1);
        } else {
#pragma unroll 1
          for (int k = 1; k < kStep / 16; ++k)
            if (keys > h * kStep + k * 16) umma_ts(o, p + k * 8, kDescV | (vb + (h * 4 + k) * 128), kIdescO, 1);
        }
        if (BLOCKS == 1) umma_commit(&sh.o_full[g][x]); else if (h == 0) umma_commit(&sh.o_full[g][0]);
      }
    };
    auto commit = [&](uint64_t* bar) {
      if (leader) umma_commit(bar);
    };
    while (next()) {
      const Segment& u = segment();
      const int n = u.t1 - u.t0;
      const uint32_t turn = (taken - 1) & 1;
      ok = ok && warp_wait(&sh.q_full, turn, abort_flag);
      if (!by_tma) tc_fence_after();
      // tile j's outputs, and the scores that go where its probabilities were: two
      // blocks, of the next tile; one, of the tile after the next.  The first scores
      // need nothing of the segment before, the first outputs that its own were read.
      constexpr int kAhead = BLOCKS == 2 ? 1 : 2;
#pragma unroll 1
      for (int j = -kAhead; j < n && ok; ++j) {
        const bool more = j + kAhead < n;
        // Keys of tile j, all tiles by one formula.  (As a choice by j, of the last tile's
        // count, that of the first tokens' last and kTile, CUDA 13.0.88 compiles the kernels
        // of one block to kTile where a traced j equals the first tokens' index: stale rows of
        // shared memory are multiplied then, which test_tiles_that_are_not_loaded_whole sees.)
        const int keys = min(kTile, u.g.limit(a, u.t0 + j) - u.g.tile(u.t0 + j) * kTile);
        const uint32_t kb = uniform(k_addr + kst * (kStage >> 4)), vb = uniform(v_addr + vst * (kStage >> 4));
        if (j >= 0) ok = warp_wait(sh.fixed + vst, vph, abort_flag);
        if (BLOCKS == 1 && j == 0) ok = ok && warp_wait(sh.ready + 0, turn, abort_flag) && warp_wait(sh.ready + 1, turn, abort_flag);
        if (!ok) break;
#pragma unroll
        for (int e = 0; e < BLOCKS; ++e) {
          const int x = BLOCKS == 2 ? e : j & 1;
          if (BLOCKS == 2 && j == 0) ok = ok && warp_wait(sh.ready + e, turn, abort_flag);
#pragma unroll
          for (int h = 0; h < 2; ++h)
            if (j >= 0) outputs(BLOCKS == 2 ? e : h, x, h, vb, j == 0 && (BLOCKS == 1 || h == 0), keys);
          // (asked for here, since the load of a stage that has just come free is
          // what a step would wait for)
          if (more && e == 0) ok = ok && warp_wait(sh.k_full + kst, kph, abort_flag);
          if (!ok) break;
          if (more) scores(x, kb);
        }
        if (!ok) break;
        if (j >= 0) {
          commit(sh.v_empty + vst);
          if (++vst == NV) { vst = 0; vph ^= 1; }
        }
        if (more) {
          commit(sh.k_empty + kst);
          if (++kst == NK) { kst = 0; kph ^= 1; }
        }
      }
      if (BLOCKS == 2 && ok) {
        commit(&sh.o_full[0][1]);
        commit(&sh.o_full[1][1]);
      }
    }
    if (!ok) *abort_flag = 1;
    // products in flight read shared memory and write tensor memory: let them end
    __syncwarp();
    commit(&sh.drain);
    mbar_drain(&sh.drain, 0);
  } else if (warp == 3) {
    // ---- segments, worked out ahead of their use -----------------------------------------
    if (one_part) {
      // the fewest tiles a part that the CTAs are enough for; two sequences a lane
      static_assert(kSeqHeld == 64, "two sequences a lane");
      int tiles[2], mine[2];
      const int all_tiles = ranges.total - units * kUnitStart;
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        tiles[e] = sh.tiles[2 * lane + e];
        mine[e] = tiles[e] ? a.n_kv_heads : 0;
      }
      // (a unit's parts are less than one more than its tiles / most, or, of millions of
      // tiles, than its tiles and four / most)
      int least = max(1, all_tiles / grid), most = max(least, min(longest, all_tiles / (grid - units + 1) + 5));
#pragma unroll 1
      while (least < most) {
        const int mid = (least + most) / 2;
        const int need = __reduce_add_sync(0xffffffffu, mine[0] * parts_of<kUnitSplit>(tiles[0], mid) + mine[1] * parts_of<kUnitSplit>(tiles[1], mid));
        if (need <= grid) most = mid; else least = mid + 1;
      }
      int inc = 0;
#pragma unroll
      for (int e = 0; e < 2; ++e) { mine[e] *= parts_of<kUnitSplit>(tiles[e], most); inc += mine[e]; }
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
          const int parts = parts_of<kUnitSplit>(tiles[e], most);
          w.left = 1;
          w.b = 2 * lane + e;
          w.load(a, sh.seq, kRows);
          w.g = span_of(a, w.s, 0, kRows);
          w.head = at / parts;
          w.block = 0;
          w.count = parts;
          w.me = at - w.head * parts;
          w.c0 = (int)blockIdx.x - w.me;
          w.t0 = w.me * w.g.tiles / parts;
          w.t1 = (w.me + 1) * w.g.tiles / parts;
        }
        before += mine[e];
      }
    } else {
      if (hi > lo) {  // the block that the first place lies in
        const int b = sh.start_b, rest = sh.start_off;
        if (lane == 0) w.b = b;
        __syncwarp();
        w.load(a, sh.seq, kRows);
        __syncwarp();
        const Chunk s = w.s;
        int before = 0;
#pragma unroll 1
        for (int i0 = 0; i0 < s.blocks; i0 += 32) {
          const int len = i0 + lane < s.blocks ? span_of(a, s, i0 + lane, kRows).tiles + kUnitStart : 0;
          int inc = len;
#pragma unroll
          for (int o = 1; o < 32; o <<= 1) {
            const int t = __shfl_up_sync(0xffffffffu, inc, o);
            if (lane >= o) inc += t;
          }
          const uint32_t past = __ballot_sync(0xffffffffu, before + inc > rest);
          if (past) {
            if (lane == __ffs(past) - 1) { sh.start_block = i0 + lane; sh.start_off = rest - (before + inc - len); }
            break;
          }
          before += __shfl_sync(0xffffffffu, inc, 31);
        }
        __syncwarp();
      }
      if (lane == 0) begin();
    }
    int made = 0;
    bool more = true;
    auto make = [&] {
      if (!more || !ok) return;
      const int slot = made % kAheadSegs;
      if (made >= kAheadSegs) {
        // An 8-bit cache's tiles pass this warp by, and it waits for as long as the others
        // take for a segment: up to 10 min, since a wait of theirs that runs out ends this one.
        const int tries = Q8 ? 300 : 1;
        for (int i = 1;; ++i) {  // (all lanes leave together)
          ok = warp_wait(sh.seg_free + slot, (made / kAheadSegs - 1) & 1, abort_flag);
          if (ok || i == tries || __any_sync(0xffffffffu, *abort_flag)) break;
        }
      }
      if (!ok) return;
      __syncwarp();
      int some = 0;
      if (lane == 0) {
        some = w.next(a, sh.seq, kRows, ranges, one_part);
        sh.seg[slot] = w;
        if (!some) sh.seg[slot].t1 = 0;
        mbar_arrive(sh.seg_full + slot);
      }
      __syncwarp();
      more = __shfl_sync(0xffffffffu, some, 0) != 0;
      ++made;
    };
    for (int cur = 0; ok; ++cur) {
      while (ok && more && made < cur + kAheadSegs - 1) make();
      if (!ok || cur >= made) break;
      const Segment& u = sh.seg[cur % kAheadSegs];
      const int n = u.t1 - u.t0;
      if (u.t1 <= 0) break;
      // ---- values of tiles that some row does not see whole ------------------------------
#pragma unroll 1
      for (int j = 0; j < n && !Q8; ++j) {
        const int st = (tile0 + j) % NV;
        ok = warp_wait(sh.v_full + st, ((tile0 + j) / NV) & 1, abort_flag);
        if (!ok) break;
        const int k0 = u.g.tile(u.t0 + j) * kTile;
        if (!all_see(a, u.s, u.g.p_lo, u.g.p_hi, k0, k0 + kTile)) {
          const int end = u.g.limit(a, u.t0 + j) - k0;  // keys of the tile
          constexpr int kPieces = HD / 8, kBatch = 4;
          auto place = [&](int p) {
            const int r = p / kPieces, c = p % kPieces;
            return reinterpret_cast<uint4*>(vring + st * kStage + (c / 8) * kChunkBytes + r * 128 + (((c % 8) ^ (r & 7)) << 4));
          };
          // Rows that the last of the block's rows has in its window, or that are among the
          // first tokens, and that the first row's position reaches, are left alone; the
          // others, and those past the end that the products read too (16 keys at a time and
          // each half's first 16 in any case), lose what is not finite.  As a rule there is
          // nothing: times zero, summed, it would be NaN.
          bool any = false, wrote = false;
          auto clean = [&](int r0, int r1) {
            if (r0 >= r1) return;
            uint32_t acc[4] = {0, 0, 0, 0};
#pragma unroll 1
            for (int p0 = r0 * kPieces + lane; p0 < r1 * kPieces; p0 += 32 * kBatch) {
              uint4 x[kBatch];
#pragma unroll
              for (int i = 0; i < kBatch; ++i) x[i] = *place(min(p0 + 32 * i, r1 * kPieces - 1));
#pragma unroll
              for (int i = 0; i < kBatch; ++i) {
                acc[0] = Num<M>::times_zero(x[i].x, acc[0]);
                acc[1] = Num<M>::times_zero(x[i].y, acc[1]);
                acc[2] = Num<M>::times_zero(x[i].z, acc[2]);
                acc[3] = Num<M>::times_zero(x[i].w, acc[3]);
              }
            }
            if (!__any_sync(0xffffffffu, ((acc[0] | acc[1] | acc[2] | acc[3]) & 0x7FFF7FFFu) != 0)) return;
            wrote = true;
#pragma unroll 1
            for (int p = r0 * kPieces + lane; p < r1 * kPieces; p += 32) {
              const uint4 x = *place(p), f = make_uint4(finite_of<M>(x.x), finite_of<M>(x.y), finite_of<M>(x.z), finite_of<M>(x.w));
              if (f.x == x.x && f.y == x.y && f.z == x.z && f.w == x.w) continue;
              *place(p) = f;
              any |= p < end * kPieces;
            }
          };
          const int reach = min(max(min(u.g.p_lo + 1, u.s.keys) - k0, 0), min(end, kTile));
          const int from = min(max(window_from(a, u.g.p_hi) - k0, 0), reach), sinks = min(max(a.sinks - k0, 0), from);
          clean(sinks, from);
          clean(reach, min(kTile, (end + 15) & ~15));
          if (end <= kStep) clean(kStep, kStep + 16);
          if (wrote) fence_proxy_shared();
          any = __any_sync(0xffffffffu, any);
          if (lane == 0) sh.odd[st] = any;
        }
        __syncwarp();
        if (lane == 0) mbar_arrive(sh.fixed + st);
      }
      tile0 += n;
    }
    if (!ok) *abort_flag = 1;
  } else if (warp < 12) {
    // ---- softmax: group g, a thread a row --------------------------------------------
    const int g = (warp - 4) >> 2, t = tid - 128 - g * kTile;  // t: row of the score tile = lane of tensor memory
    const uint32_t my = tmem + ((uint32_t)((warp & 3) * 32) << 16);
    const uint32_t o_addr = my + 2 * kTile + g * HD;
    const float sl2_all = fmaxf(fabsf(a.scale) * 1.4426950408889634f, 1.2e-38f);  // a masked score stays -inf at scale 0
    const bool wide_out = (reinterpret_cast<uintptr_t>(a.out) & 31) == 0;
    uint32_t ph_s = 0, ph_pair = 0, ph_met = 0;
    uint32_t ph_o[2] = {0, 0};  // phases of o_full that come next
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
    auto arrive = [&](uint64_t* bar) {
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(bar);
    };
    while (next()) {
      const Segment& u = segment();
      arrive(sh.ready + g);  // O of the segment before has been read
      const int n = u.t1 - u.t0;
      const int row_base = u.block * kRows + (BLOCKS == 2 ? g * kTile : 0);  // row of the unit that lane 0 of the group has
      const int row = row_base + t, rows = u.s.rows;
      const bool live = row_base + (warp & 3) * 32 < rows;  // the warp has a row at all
      // queries into shared memory, swizzled; one block: each group lays out half
      if (!by_tma) {
        constexpr int kPieces = HD / 8, kMine = BLOCKS == 2 ? kTile : kTile / 2, kEach = kTile / kPieces;
        const uint32_t sign = a.scale < 0.f ? 0x80008000u : 0u;  // a negative scale turns the queries' signs
        const int c = t % kPieces, r0 = t / kPieces + (BLOCKS == 2 ? 0 : g * kMine), in_unit = BLOCKS == 2 ? g * kTile : 0;
        const T* q = reinterpret_cast<const T*>(a.q) + ((int64_t)u.s.row0 + u.g.token) * a.q_stride + (int64_t)u.head * group * HD + c * 8;
        uint8_t* dst = qbuf + (BLOCKS == 2 ? g * kStage : 0) + (c / 8) * kChunkBytes;
        uint4 v[kMine / kEach];  // all loads are out before the first is stored
#pragma unroll
        for (int i = 0; i < kMine / kEach; ++i) {
          const int n_row = u.g.rest + in_unit + r0 + i * kEach, tok = in_group(a, n_row);
          v[i] = make_uint4(0, 0, 0, 0);
          if (row_base + r0 + i * kEach < rows) v[i] = *reinterpret_cast<const uint4*>(q + (int64_t)tok * a.q_stride + (n_row - tok * group) * HD);
        }
#pragma unroll
        for (int i = 0; i < kMine / kEach; ++i) {
          const int r = r0 + i * kEach;
          if constexpr (kRaised) {
            // bf16 queries as fp16, each row times the power of two that brings its
            // largest entry into [2^14, 2^15): exact down to 2^-39 of it
            float most = 0.f, f[8];
            const uint32_t in[4] = {v[i].x, v[i].y, v[i].z, v[i].w};
#pragma unroll
            for (int k = 0; k < 8; ++k) {
              f[k] = __uint_as_float(k & 1 ? in[k / 2] & 0xFFFF0000u : in[k / 2] << 16);
              const float m = fabsf(f[k]);
              if (m < INFINITY) most = fmaxf(most, m);
            }
#pragma unroll
            for (int d = kPieces / 2; d > 0; d >>= 1) most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, d));
            const int e = max((int)(__float_as_uint(most) >> 23), 15);  // biased exponent of the largest
            const float up = __uint_as_float((uint32_t)(268 - e) << 23);  // 2^(14 - (e - 127))
#pragma unroll
            for (int k = 0; k < 8; ++k) f[k] *= up;
            v[i] = make_uint4(Num<__half>::pack(f[0], f[1]), Num<__half>::pack(f[2], f[3]), Num<__half>::pack(f[4], f[5]), Num<__half>::pack(f[6], f[7]));
            if (c == 0) sh.back[in_unit + r] = (uint8_t)e;
          }
          v[i].x ^= sign; v[i].y ^= sign; v[i].z ^= sign; v[i].w ^= sign;
          *reinterpret_cast<uint4*>(dst + r * 128 + (((c % 8) ^ (r & 7)) << 4)) = v[i];
        }
        fence_proxy_shared();
        arrive(&sh.q_full);
      }
      float sl2 = sl2_all;
      if constexpr (kRaised) {
        if (BLOCKS == 1) meet(); else group_meet();  // the rows' exponents are there
        if (!ok) break;
        sl2 = fmaxf(sl2_all * __uint_as_float((uint32_t)max((int)sh.back[BLOCKS == 2 ? g * kTile + t : t] - 14, 1) << 23), 1.2e-38f);
      }
      const int n_row = u.g.rest + min(row, rows - 1) - u.block * kRows, in_token = in_group(a, n_row);  // of the block's first token on
      const int token = u.g.token + in_token, p = u.s.ctx + token;
      const int see_end = min(p + 1, u.s.keys), see_from = window_from(a, p);
      // positions of the group's first and last rows
      auto position = [&](int r) { return u.g.p_lo + in_group(a, u.g.rest + min(r, rows - 1) - u.block * kRows); };
      const int g_lo = position(row_base), g_hi = position(row_base + kTile - 1);
      float m_ref = -INFINITY, sum = 0.f;
      const uint64_t scale2 = pair_of(__float_as_uint(sl2), __float_as_uint(sl2));
      // all_see() of a tile that begins at k0: k0 <= whole and (from <= k0 or the tile lies
      // among the first tokens), of the block's rows and of the group's
      const int whole_block = min(u.g.p_lo + 1, u.s.keys) - kTile, from_block = window_from(a, u.g.p_hi);
      const int whole_group = min(g_lo + 1, u.s.keys) - kTile, from_group = window_from(a, g_hi);
      const int first_tile = u.t0, sink_tiles = u.g.sink, skip = u.g.skip;
#pragma unroll 1
      for (int j = 0; j < n; ++j) {
        const int k = first_tile + j, k0 = (k < sink_tiles ? k : k + skip) * kTile, x = BLOCKS == 2 ? g : j & 1;
        const bool among = k0 + kTile <= a.sinks;
        const bool partly = k0 > whole_block || (from_block > k0 && !among);  // some row of the block does not see all of the tile,
        bool masked = k0 > whole_group || (from_group > k0 && !among);        // some row of the group
        ok = warp_wait(sh.s_full + x, ph_s >> x & 1, abort_flag);
        if (!ok) break;
        const uint32_t flags = sh.pages[(tile0 + j) & 15];
        masked |= flags != 0xFFu;
        ph_s ^= 1u << x;
        tc_fence_after();
#pragma unroll
        for (int e = 0; e < BLOCKS; ++e) {
          const int h = BLOCKS == 2 ? e : g;
          const uint32_t s_at = my + x * kTile + h * kStep;
          if (live) {
            uint32_t v[kStep];
            tm_ld32(s_at, v);
            tm_ld32(s_at + 32, v + 32);
            tm_landed<kStep>(v);
            if (masked) {
#pragma unroll
              for (int c = 0; c < 2; ++c) {
                const uint32_t there = flags >> (4 * h + 2 * c);
                const uint32_t m = seen32(k0 + h * kStep + 32 * c, see_end, see_from, a.sinks) &
                                   ((there & 1 ? 0xFFFFu : 0u) | (there & 2 ? 0xFFFF0000u : 0u));
#pragma unroll
                for (int i = 0; i < 32; ++i)
                  if (!(m >> i & 1)) v[32 * c + i] = 0xFF800000u;
              }
            }
            float mx[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
            for (int i = 0; i < kStep; i += 2)
              mx[i >> 1 & 3] = fmaxf(fmaxf(__uint_as_float(v[i]), __uint_as_float(v[i + 1])), mx[i >> 1 & 3]);
            // what probabilities are taken against: 2^kRaise below the largest
            const float top = fmaxf(fmaxf(mx[0], mx[1]), fmaxf(mx[2], mx[3])) * sl2 - Num<M>::kRaise;
            if (j == 0 && e == 0) {
              m_ref = top;
            } else if (__any_sync(0xffffffffu, top > m_ref + kLazy)) {
              const float m_new = fmaxf(m_ref, top);
              const float alpha = m_new == m_ref ? 1.0f : ex2(m_ref - m_new);
              m_ref = m_new;
              sum *= alpha;
              // The products before this one are done: two blocks, those of earlier tiles
              // when the scores came, this tile's first half's by its barrier; one, those of
              // the buffer when its scores came again, the other's by that one's barrier.
              if (BLOCKS == 2 ? e == 1 : j > 0) {
                ok = BLOCKS == 2 ? warp_wait(&sh.o_full[g][0], ph_o[0], abort_flag) : warp_wait(&sh.o_full[g][x ^ 1], (x ? ph_o[0] : ph_o[1]) ^ 1, abort_flag);
                tc_fence_after();
                if (!ok) break;
              }
              scale_row<HD>(o_addr, alpha);
            }
            const float base = m_ref == -INFINITY ? 0.f : m_ref;
            const uint64_t base2 = pair_of(__float_as_uint(-base), __float_as_uint(-base));
            uint64_t acc[2] = {0, 0};
            // in place: the pair at 2 i becomes entry i
#pragma unroll
            for (int i = 0; i < kStep / 2; ++i) {
              const float2 f = floats_of(fma2(pair_of(v[2 * i], v[2 * i + 1]), scale2, base2));
              const float y = ex2(f.x), z = ex2(f.y);
              acc[i & 1] = add2(acc[i & 1], pair_of(__float_as_uint(y), __float_as_uint(z)));
              v[i] = Num<M>::pack(y, z);
            }
            tm_st32(s_at, v);
            tm_wait_st();
            const float2 acc2 = floats_of(add2(acc[0], acc[1]));
            sum += acc2.x + acc2.y;
          }
          if (partly && e == BLOCKS - 1) {  // the stage is not refilled before these probabilities are used
            const int st = (tile0 + j) % NV;
            ok = warp_wait(sh.fixed + st, ((tile0 + j) / NV) & 1, abort_flag);
            if (!ok) break;
            if (sh.odd[st]) sh.odd_in[g] = taken;  // the rows who see them get them back in the epilogue
          }
          arrive(&sh.p_full[x][h]);
        }
        if (!ok) break;
        // a product more of its kind is on the way
        if (BLOCKS == 2 || x == 0) ph_o[0] ^= 1; else ph_o[1] ^= 1;
      }
      if (!ok) break;
      // all of the segment's products
      if (BLOCKS == 2) {
        ok = warp_wait(&sh.o_full[g][1], ph_o[1], abort_flag);
        ph_o[1] ^= 1;
      } else {
        ok = warp_wait(&sh.o_full[g][0], ph_o[0] ^ 1, abort_flag) && (n == 1 || warp_wait(&sh.o_full[g][1], ph_o[1] ^ 1, abort_flag));
      }
      if (!ok) break;
      tc_fence_after();
      // ---- epilogue: a group's own accumulator, or half the columns of both groups' ----
      float w0 = 1.f, w1 = 0.f;
      if (BLOCKS == 1) {
        float2* ml = reinterpret_cast<float2*>(qbuf);  // the queries have been read
        ml[g * kTile + t] = make_float2(m_ref, sum);
        meet();
        if (!ok) break;
        const float2 y = ml[t], z = ml[kTile + t];
        m_ref = fmaxf(y.x, z.x);
        w0 = y.x == -INFINITY ? 0.f : ex2(y.x - m_ref);
        w1 = z.x == -INFINITY ? 0.f : ex2(z.x - m_ref);
        sum = y.y * w0 + z.y * w1;
        fence_proxy_shared();  // (a copy may write there next)
        meet();
        if (!ok) break;
        arrive(&sh.q_free);
      }
      constexpr int kCols = BLOCKS == 2 ? HD : HD / 2;
      const int col0 = BLOCKS == 2 ? 0 : g * kCols, in_block = (BLOCKS == 2 ? g * kTile : 0) + t;
      const bool whole = u.t0 == 0 && u.t1 == u.g.tiles, on = row < rows;
      // A unit's contributors are consecutive CTAs.  All but the last to arrive
      // leave their partial; that one joins them, in tile order.
      const int count = whole ? 1 : u.count, me = u.me, c0 = u.c0;
      uint32_t* arrived = reinterpret_cast<uint32_t*>(a.workspace) + 2 * c0 + g;
      const bool few = rows - u.block * kRows <= kFewRows;
      auto slot = [&](int i) { const Partial s = slot_of(a, i, HD, BLOCKS); return few ? few_rows<HD>(s) : s; };
      const Partial mine = slot(2 * (c0 + me) + (u.t0 > 0 ? 0 : 1));
      bool two = false;
      auto odd = [&] { return sh.odd_in[g] == taken; };
      if (count == 2) {
        if (t == 0) sh.last_in[g] = last_of(ld_acquire(arrived), count);
        group_meet();
        if (!ok) break;
        two = sh.last_in[g] != 0;
      }
      T* unit = reinterpret_cast<T*>(a.out) + ((int64_t)u.s.row0 * a.n_q_heads + (int64_t)u.head * group) * HD;
      const int in_chunk = row - u.block * kRows + u.g.rest - in_token * group;  // this row among its token's
      T* out = unit + ((int64_t)token * a.n_q_heads + in_chunk) * HD;
      const int unit_row0 = row_base;
      if (!two) {
        const float inv = sum > 0.f ? 1.0f / sum : 0.f;
#pragma unroll 1
        for (int c = col0; c < col0 + kCols; c += 32) {
          if (!live) break;
          uint32_t o[32];
          own_columns<HD, BLOCKS>(o, my + 2 * kTile + (BLOCKS == 2 ? g * HD : 0) + c, w0, w1, true);
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
          if (t == 0) sh.last_in[g] = last_of(arrive_acq_rel(arrived, odd()), count);
          group_meet();
          if (!ok) break;
          if (sh.last_in[g]) {
            if (count == 2) {
              two = true;
            } else {
              fence_gpu();
              const int live_rows = min(kTile, rows - row_base);
              if (few) join_few<T, HD, BLOCKS>(slot_of(a, 0, HD, BLOCKS), sh.slots[g], count, g, t, in_block - t, live_rows, col0 / 4, unit, unit_row0, group, (int64_t)a.n_q_heads * HD);
              else join<T, HD, BLOCKS>(a, sh.slots[g], count, g, t, in_block - t, live_rows, col0 / 4, kCols / 4, unit, unit_row0);
              if (t == 0) *arrived = 0;  // as the next call wants it
            }
          }
        }
      }
      if (two) {
        const Partial other = slot(2 * (c0 + 1 - me) + me);
        join_two<T, HD, BLOCKS>(other, my + 2 * kTile + (BLOCKS == 2 ? g * HD : 0), g, in_block, me == 0, m_ref, sum, w0,
                                w1, true, col0, on, out, wide_out);
        if (t == 0) *arrived = 0;
      }
      if (whole ? odd() : sh.last_in[g] == 2 || (sh.last_in[g] == 1 && odd())) {
        group_meet();  // a row may have been joined by other threads
        if (!ok) break;
        patch_chunk<T, HD, BLOCKS, Q8>(a, segment(), g, t);
      }
      if (BLOCKS == 1) {  // each group reads both accumulators
        meet();
        if (!ok) break;
      }
      tile0 += n;
    }
    if (!ok) *abort_flag = 1;
  } else if constexpr (Q8) {
    // ---- codes into 16-bit entries: two warps for keys, two for values ----------------------
    constexpr int kCodes = HD * kPageTok, kHeld = kCodes / 512, kRowPieces = HD / 16;
    const int v = (warp - 12) / (kConvWarps / 2), cw = (warp - 12) % (kConvWarps / 2), ns = v ? NV : NK;
    uint8_t *from0 = raw_rings + v * NR * kRaw, *to0 = v ? vring : kring;
    uint64_t *empty = v ? sh.v_empty : sh.k_empty, *full = v ? sh.fixed : sh.k_full;
    int st = 0, rs = 0;
    uint32_t ph = 0, rph = 0;
    while (next()) {
      const Segment& u = segment();
      const int n = u.t1 - u.t0;
#pragma unroll 1
      for (int j = 0; j < n; ++j) {
        const int tile = u.g.tile(u.t0 + j), k0 = tile * kTile;
        ok = warp_wait(sh.raw_full[v] + rs, rph, abort_flag) && warp_wait(empty + st, ph ^ 1, abort_flag);
        if (!ok) break;
        uint8_t* stage = to0 + st * kStage;
        const uint8_t *raw = from0 + rs * kRaw, *scale = sh.scale[v] + rs * kTile;
        const bool clean = v && !all_see(a, u.s, u.g.p_lo, u.g.p_hi, k0, k0 + kTile);
        const int pages = pages_of(u, u.t0 + j), end = u.g.limit(a, u.t0 + j);
        bool any = false;
        // eight entries of row r: two pieces of a row's sixteen codes, and the lanes of a
        // row's second half write theirs the other way round, so that eight lanes reach
        // all banks
        const int c16 = lane % kRowPieces, turn = HD == 128 ? c16 / 4 : 0;
        uint8_t* to = stage + (c16 / 4) * kChunkBytes + lane / kRowPieces * 128;
        auto put = [&](int q, int e, const uint32_t (&y)[8]) {
          const int r = lane / kRowPieces + e * (32 / kRowPieces), c = (2 * c16) % 8;
          uint8_t* at = to + (q * kPageTok + e * (32 / kRowPieces)) * 128;
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            const bool second = (h ^ turn) != 0;
            *reinterpret_cast<uint4*>(at + (((c + (second ? 1 : 0)) ^ (r & 7)) << 4)) =
                second ? make_uint4(y[4], y[5], y[6], y[7]) : make_uint4(y[0], y[1], y[2], y[3]);
          }
        };
        if (!clean && !sh.far[v][rs]) {
#pragma unroll 1
          for (int q = cw; q < pages; q += kConvWarps / 2) {
            uint4 x[kHeld];
            uint32_t by[kHeld];
#pragma unroll
            for (int e = 0; e < kHeld; ++e) {
              x[e] = reinterpret_cast<const uint4*>(raw + q * kCodes)[e * 32 + lane];
              by[e] = scale[q * kPageTok + (e * 32 + lane) / kRowPieces];
            }
#pragma unroll
            for (int e = 0; e < kHeld; ++e) {
              Widen w8;
              w8.set(by[e]);
              const uint32_t y[8] = {w8.near_two(x[e].x), w8.near_two(x[e].x >> 16), w8.near_two(x[e].y), w8.near_two(x[e].y >> 16),
                                     w8.near_two(x[e].z), w8.near_two(x[e].z >> 16), w8.near_two(x[e].w), w8.near_two(x[e].w >> 16)};
              put(q, e, y);
            }
          }
        } else {
#pragma unroll 1
          for (int qe = 0; qe < kHeld * ((pages - cw + kConvWarps / 2 - 1) / (kConvWarps / 2)); ++qe) {
            const int q = cw + qe / kHeld * (kConvWarps / 2), e = qe % kHeld;
            Widen w8;
            const uint4 xe = reinterpret_cast<const uint4*>(raw + q * kCodes)[e * 32 + lane];
            w8.set_far(scale[q * kPageTok + (e * 32 + lane) / kRowPieces]);
            uint32_t y[8] = {w8.far_two(xe.x), w8.far_two(xe.x >> 16), w8.far_two(xe.y), w8.far_two(xe.y >> 16),
                             w8.far_two(xe.z), w8.far_two(xe.z >> 16), w8.far_two(xe.w), w8.far_two(xe.w >> 16)};
            const int key = k0 + q * kPageTok + lane / kRowPieces + e * (32 / kRowPieces);
            if (clean && !all_see(a, u.s, u.g.p_lo, u.g.p_hi, key, key + 1)) {
#pragma unroll
              for (int k = 0; k < 8; ++k) {
                const uint32_t f = key >= end ? 0u : finite_of<__half>(y[k]);
                any |= key < end && f != y[k];
                y[k] = f;
              }
            }
            put(q, e, y);
          }
        }
        if (v && cw == 0 && pages <= kTilePages / 2) {  // the second half's first 16, which are multiplied in any case
#pragma unroll 1
          for (int e = lane; e < kPageTok * HD / 8; e += 32)
            *reinterpret_cast<uint4*>(stage + (e / (kPageTok * 8)) * kChunkBytes + kStep * 128 + e % (kPageTok * 8) * 16) = make_uint4(0, 0, 0, 0);
        }
        fence_proxy_shared();
        any = __any_sync(0xffffffffu, any);
        if (lane == 0) {
          if (v) reinterpret_cast<uint8_t*>(sh.odd + st)[cw] = any;
          mbar_arrive(full + st);
          mbar_arrive(sh.raw_empty[v] + rs);
        }
        if (++st == ns) { st = 0; ph ^= 1; }
        if (++rs == NR) { rs = 0; rph ^= 1; }
      }
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
    const bool part = sh.seg[0].t1 > 0;
    __syncthreads();
    if (tid == 0) {
      reinterpret_cast<volatile uint32_t*>(a.workspace)[kStalledWord] = 1;
      if (one_part) w.left = part; else begin();
    }
    while (true) {
      __syncthreads();
      if (tid == 0) sh.odd[0] = w.next(a, sh.seq, kRows, ranges, one_part);
      __syncthreads();
      if (!sh.odd[0]) break;
#pragma unroll 1
      for (int r = w.block * kRows + tid; r < min((w.block + 1) * kRows, w.s.rows); r += kThreads) {
        const int token = r / group;
        T* out = reinterpret_cast<T*>(a.out) +
                 (((int64_t)w.s.row0 + token) * a.n_q_heads + (int64_t)w.head * group + (r - token * group)) * HD;
#pragma unroll 1
        for (int e = 0; e < HD; e += 2) *reinterpret_cast<uint32_t*>(out + e) = 0x7FFF7FFFu;
      }
    }
  }
}

namespace {

// Blocks of 256 query vectors where a sequence has more than 128 of them on average:
// two groups with rows of their own use each tile twice.  With fewer, both work on
// the same rows.  8 sequences of 8000 keys, four query heads a key/value head, 32
// tokens each: 64 us in blocks of 128 and 69 of 256; 40 tokens: 90 and 70 (8-bit
// caches: 65 and 94; 106 and 97).
int chunk_blocks(int n_tokens, int batch, int group) { return (int64_t)n_tokens * group <= (int64_t)batch * kTile ? 1 : 2; }

// An 8-bit cache's codes as [page][head][token][entry], boxes of a page's 16 tokens of a head.
inline CUtensorMap codes_map(const ChunkAttnArgs& a, const void* base) {
  CUtensorMap m;
  std::memset(&m, 0, sizeof(m));
  auto enc = encoder();
  if (!enc) throw cudaErrorNotSupported;
  const cuuint64_t hd = a.head_dim;
  const cuuint64_t dims[4] = {hd, (cuuint64_t)kPageTok, (cuuint64_t)a.n_kv_heads, (cuuint64_t)a.n_pages};
  const cuuint64_t strides[3] = {hd, hd * kPageTok, (cuuint64_t)a.page_stride};
  const cuuint32_t box[4] = {(cuuint32_t)hd, (cuuint32_t)kPageTok, 1, 1}, es[4] = {1, 1, 1, 1};
  const CUresult r = enc(&m, CU_TENSOR_MAP_DATA_TYPE_UINT8, 4, const_cast<void*>(base), dims, strides, box, es,
                         CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_NONE, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                         CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
  if (r != CUDA_SUCCESS) throw cudaErrorInvalidValue;
  return m;
}

// The queries as [token][head][entry], boxes of some tokens x a key/value head's query heads x 64 entries.
inline CUtensorMap query_map(const ChunkAttnArgs& a, int tokens) {
  CUtensorMap m;
  std::memset(&m, 0, sizeof(m));
  auto enc = encoder();
  if (!enc) throw cudaErrorNotSupported;
  const cuuint64_t hd = a.head_dim;
  const cuuint64_t dims[3] = {hd, (cuuint64_t)a.n_q_heads, (cuuint64_t)a.n_tokens};
  const cuuint64_t strides[2] = {hd * 2, (cuuint64_t)a.q_stride * 2};
  const cuuint32_t box[3] = {64, (cuuint32_t)(a.n_q_heads / a.n_kv_heads), (cuuint32_t)tokens}, es[3] = {1, 1, 1};
  const CUresult r = enc(&m, a.dtype == DT_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 3,
                         const_cast<void*>(a.q), dims, strides, box, es, CU_TENSOR_MAP_INTERLEAVE_NONE,
                         CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
  if (r != CUDA_SUCCESS) throw cudaErrorInvalidValue;
  return m;
}

template <typename T, int HD, int BLOCKS, bool Q8>
void run_chunk(const ChunkAttnArgs& a, cudaStream_t s) {
  constexpr int smem = chunk_smem<HD, BLOCKS, Q8>();
  auto* kernel = chunk_attention_kernel<T, HD, BLOCKS, Q8>;
  static OncePerDevice ctas;
  const int dev = current_device(), sms = ctas.get(dev, [&] {
    allow_shared(kernel, smem);
    int n = 0;
    const cudaError_t e = cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev);
    if (e != cudaSuccess) throw e;
    return n;
  });
  const int grid = sms < kMaxGrid ? sms : kMaxGrid;
  CUtensorMap km, vm, qm;
  std::memset(&km, 0, sizeof(km));
  vm = qm = km;
  ChunkAttnArgs args = a;
  const int group = a.n_q_heads / a.n_kv_heads;
  args.group = group;
  args.group_magic = group > 1 ? 0xFFFFFFFFu / (uint32_t)group + 1 : 0;
  if (Q8) {
    km = codes_map(a, a.k_cache);
    vm = codes_map(a, a.v_cache);
  } else {
    km = cache_map(a, a.k_cache);
    vm = cache_map(a, a.v_cache);
    // Queries come by tensor copies where a block's rows are whole tokens and need
    // no other sign; the softmax warps' own loads take 4000 clocks before a unit's first scores.
    args.q_by_tma = kTile % group == 0 && !(a.scale < 0.f);
    if (args.q_by_tma) qm = query_map(a, kTile / group);
  }
  launch_in_turn(kernel, dim3(grid), chunk_threads(Q8), smem, 0, s, args, km, vm, qm);
}

// The caches' width is the translation unit's.
template <typename T, int HD, bool Q8>
void run_chunk_sized(const ChunkAttnArgs& a, cudaStream_t s) {
  if (chunk_blocks(a.n_tokens, a.batch, a.n_q_heads / a.n_kv_heads) == 1) run_chunk<T, HD, 1, Q8>(a, s);
  else run_chunk<T, HD, 2, Q8>(a, s);
}
template <bool Q8>
void run_chunk_attention(const ChunkAttnArgs& a, cudaStream_t s) {
  if (a.dtype == DT_BF16) {
    if (a.head_dim == 128) run_chunk_sized<__nv_bfloat16, 128, Q8>(a, s); else run_chunk_sized<__nv_bfloat16, 64, Q8>(a, s);
  } else {
    if (a.head_dim == 128) run_chunk_sized<__half, 128, Q8>(a, s); else run_chunk_sized<__half, 64, Q8>(a, s);
  }
}

}  // namespace

}  // namespace pard
