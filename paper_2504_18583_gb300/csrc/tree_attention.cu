// Attention of a tree's nodes over the paged cache: S = Q K^T, a running
// maximum and sum, O += P V, both products on tcgen05 with the accumulators in
// tensor memory.
//
// A unit is one sequence's key/value head with up to 128 or 256 query vectors
// (nodes x the query heads that share the head) and its keys in tiles of 128.
// All units' tiles, in order, are cut into one even range a CTA (one CTA an SM,
// persistent): contexts may differ by any factor, the host need not know them,
// and no SM waits for a long sequence.  A range that begins or ends inside a
// unit leaves a partial (unnormalised O, maximum, sum, all in 32 bits) in the
// workspace; the combine kernel joins a unit's partials in tile order, so
// results do not depend on timing.
//
// Roles: warp 0 loads (TMA boxes of one page's 16 tokens x 64 entries: a tile
// of eight pages lands as the 128-byte-swizzled operand that the products
// read, K as stored, V as its transpose without moving a byte); warp 1 issues
// the products; warps 2-3 look after the values of tiles that reach past the
// context; two warpgroups take the softmax, a thread a row, so that row
// maxima and sums need no exchange.  The two groups work on two score tiles in
// turn: with more than 128 query vectors each has its own 128 of them, else
// both have the same and alternate key tiles (their sums are joined at the end
// straight from tensor memory).  One tile's products run under the other's
// softmax.  The accumulator is scaled only when a row's maximum has grown by
// more than 2^8 since the last time.
//
// Masks touch only tiles that reach past the context: a row's 256 mask bits
// select among its scores.  Values there may hold anything: what lies past the
// sequence is zeroed in shared memory, and so are infinities and NaN of tree
// nodes, which the epilogue adds back for the rows that see the node (0 x NaN
// would reach every row otherwise).
#include <cuda_fp16.h>

#include <cstring>
#include <mutex>

#include <cudaTypedefs.h>

#include "common.cuh"
#include "tree.h"

namespace pard {

namespace {

constexpr int kTile = 128;                      // keys a tile, rows a score tile
constexpr int kTilePages = kTile / kPageTok;
constexpr int kTaThreads = 384;
constexpr int kMaxGrid = 160;                   // workspace slots are sized for this many CTAs
constexpr float kLazy = 8.0f;                   // growth of a maximum, in powers of two, that is let pass

__host__ __device__ constexpr int stage_bytes(int hd) { return kTile * hd * 2; }
__host__ __device__ constexpr int stages(int hd, int blocks) { return (hd == 128 ? 7 : 14) - (hd == 128 ? blocks : 2 * blocks); }
__host__ __device__ constexpr int bar_bytes(int hd, int blocks) { return (8 * (3 * stages(hd, blocks) + 10) + 16 + 8 * stages(hd, blocks) + 127) / 128 * 128; }
__host__ __device__ constexpr int smem_bytes(int hd, int blocks) {
  return 1024 + (blocks + stages(hd, blocks)) * stage_bytes(hd) + bar_bytes(hd, blocks);
}
static_assert(smem_bytes(128, 1) <= 227 * 1024 && smem_bytes(128, 2) <= 227 * 1024, "shared memory of one CTA");
static_assert(smem_bytes(64, 1) <= 227 * 1024 && smem_bytes(64, 2) <= 227 * 1024, "shared memory of one CTA");

template <typename T> struct Num;
template <> struct Num<__nv_bfloat16> {
  static constexpr uint32_t kFormat = 1;        // of the instruction descriptor
  static constexpr uint32_t kExponent = 0x7F80; // all ones: infinity or NaN
  static __device__ __forceinline__ uint32_t pack(float x, float y) {
    __nv_bfloat162 p = __floats2bfloat162_rn(x, y);
    return *reinterpret_cast<uint32_t*>(&p);
  }
  static __device__ __forceinline__ float get(const void* p) { return __bfloat162float(*reinterpret_cast<const __nv_bfloat16*>(p)); }
};
template <> struct Num<__half> {
  static constexpr uint32_t kFormat = 0;
  static constexpr uint32_t kExponent = 0x7C00;
  static __device__ __forceinline__ uint32_t pack(float x, float y) {
    __half2 p = __floats2half2_rn(x, y);
    return *reinterpret_cast<uint32_t*>(&p);
  }
  static __device__ __forceinline__ float get(const void* p) { return __half2float(*reinterpret_cast<const __half*>(p)); }
};

// Instruction descriptor, kind::f16, fp32 accumulator, A K-major; `flip`: B
// lies with its N entries contiguous.
__host__ __device__ constexpr uint32_t idesc16(uint32_t fmt, int M, int N, bool flip) {
  return (1u << 4) | (fmt << 7) | (fmt << 10) | ((flip ? 1u : 0u) << 16) | ((uint32_t)(N >> 3) << 17) |
         ((uint32_t)(M >> 4) << 24);
}
// Descriptor of a 128-byte-swizzled operand whose N (or M) entries are
// contiguous: 64 of them a 128-byte row, eight K rows an atom; atoms 1024 bytes
// apart along K, `chunk` bytes along N.
__device__ __forceinline__ uint64_t sw128_flip_desc(uint32_t addr, uint32_t chunk) {
  uint64_t d = 0;
  d |= (uint64_t)((addr & 0x3FFFFu) >> 4);
  d |= (uint64_t)(chunk >> 4) << 16;
  d |= (uint64_t)(1024 >> 4) << 32;
  d |= (uint64_t)1 << 46;
  d |= (uint64_t)2 << 61;
  return d;
}

__device__ __forceinline__ void umma_ss(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t accumulate) {
  umma_bf16(d, a, b, idesc, accumulate);  // the descriptor names the type
}
__device__ __forceinline__ void umma_ts(uint32_t d, uint32_t a_tmem, uint64_t b, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}" ::"r"(d),
      "r"(a_tmem), "l"(b), "r"(idesc), "r"(accumulate)
      : "memory");
}
__device__ __forceinline__ void tma_load_4d(void* dst, const CUtensorMap* m, uint64_t* bar, int c0, int c1, int c2,
                                            int c3) {
  asm volatile(
      "cp.async.bulk.tensor.4d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5}], [%6];" ::"r"(
          smem_u32(dst)),
      "l"(reinterpret_cast<uint64_t>(m)), "r"(c0), "r"(c1), "r"(c2), "r"(c3), "r"(smem_u32(bar))
      : "memory");
}
// 32 lanes x 32 columns without a wait, to and from tensor memory
__device__ __forceinline__ void tm_ld32(uint32_t addr, uint32_t* r) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 "
      "{%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,"
      "%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]),
        "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]),
        "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]),
        "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
      : "r"(addr)
      : "memory");
}
__device__ __forceinline__ void tm_st32(uint32_t addr, const uint32_t* r) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x32.b32 [%32], "
      "{%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,"
      "%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31};" ::"r"(r[0]),
      "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]),
      "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(r[16]), "r"(r[17]), "r"(r[18]), "r"(r[19]),
      "r"(r[20]), "r"(r[21]), "r"(r[22]), "r"(r[23]), "r"(r[24]), "r"(r[25]), "r"(r[26]), "r"(r[27]), "r"(r[28]),
      "r"(r[29]), "r"(r[30]), "r"(r[31]), "r"(addr)
      : "memory");
}
__device__ __forceinline__ void tm_wait_ld() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void tm_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
// Two 16-bit values with infinities and NaN replaced by zero.
template <typename T>
__device__ __forceinline__ uint32_t finite_of(uint32_t v) {
  constexpr uint32_t e = Num<T>::kExponent;
  if ((v & e) == e) v &= 0xFFFF0000u;
  if ((v >> 16 & e) == e) v &= 0x0000FFFFu;
  return v;
}
// A bounded wait that all lanes of a warp leave with the same answer.
__device__ __forceinline__ bool warp_wait(uint64_t* bar, uint32_t parity, volatile int* abort) {
  return __all_sync(0xffffffffu, mbar_wait(bar, parity, abort));
}

// Keys, tiles and row blocks of a sequence.
struct Seq {
  int ctx, nodes, keys, plain, tiles, blocks;  // plain: keys that every node sees
};
__device__ __forceinline__ Seq seq_of(const TreeAttnArgs& a, int b, int rows_per_block) {
  Seq s;
  s.nodes = min(max(a.n_nodes[b], 0), a.width);
  s.ctx = max(a.ctx_len[b], 0);
  const int64_t end = (int64_t)s.ctx + s.nodes, most = (int64_t)a.max_pages * kPageTok;
  s.keys = (int)(end < most ? end : most);
  s.plain = min(s.ctx, s.keys);
  s.tiles = s.nodes > 0 ? (s.keys + kTile - 1) / kTile : 0;
  s.blocks = (s.nodes * (a.n_q_heads / a.n_kv_heads) + rows_per_block - 1) / rows_per_block;
  return s;
}
__device__ __forceinline__ int64_t seq_cost(const TreeAttnArgs& a, const Seq& s) {
  return (int64_t)a.n_kv_heads * s.blocks * s.tiles;
}
__device__ __forceinline__ int64_t range_at(int c, int64_t total, int grid) { return c * total / grid; }

// A CTA's walk over its range: one segment (part of a unit) after the other.
struct Walk {
  int64_t left;        // tiles to go
  int b, off;          // sequence, and tile within all of its units
  Seq s;
  int head, block, t0, t1;
  __device__ __forceinline__ bool next(const TreeAttnArgs& a, int rows_per_block) {
    if (left <= 0) return false;
    while (off >= seq_cost(a, s)) {  // the first call's off lies inside its sequence
      ++b;
      off = 0;
      s = seq_of(a, b, rows_per_block);
    }
    const int unit = off / s.tiles;
    t0 = off - unit * s.tiles;
    t1 = (int)min((int64_t)s.tiles, t0 + left);
    head = unit / s.blocks;
    block = unit - head * s.blocks;
    off += t1 - t0;
    left -= t1 - t0;
    return true;
  }
};

// Order in which a segment's n tiles are loaded (K and V are an item each).
// Two query blocks: K0 V0 K1 V1 ...; one: K0 K1 V0 K2 V1 ..., the order in
// which two alternating tiles are consumed.
template <int BLOCKS> __device__ __forceinline__ int item_k(int j) { return BLOCKS == 2 ? 2 * j : (j ? 2 * j - 1 : 0); }
template <int BLOCKS> __device__ __forceinline__ int item_v(int j, int n) {
  return BLOCKS == 2 ? 2 * j + 1 : (j < n - 1 ? 2 * j + 2 : 2 * n - 1);
}
// which tile item i is of, and whether it is its values
template <int BLOCKS> __device__ __forceinline__ int tile_of(int i, int n, bool& v) {
  if (BLOCKS == 2) { v = i & 1; return i >> 1; }
  if (i == 0) { v = false; return 0; }
  if (i == 2 * n - 1) { v = true; return n - 1; }
  v = !(i & 1);
  return v ? (i - 2) >> 1 : (i + 1) >> 1;
}

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

struct Partial {  // of one slot, rows = 128 * blocks: O as [HD / 4][rows] float4, then maxima, sums
  float* base;
  int rows;
  __device__ __forceinline__ float4* o(int c4, int row) const { return reinterpret_cast<float4*>(base) + (size_t)c4 * rows + row; }
  __device__ __forceinline__ float* max_of(int hd, int row) const { return base + (size_t)hd * rows + row; }
  __device__ __forceinline__ float* sum_of(int hd, int row) const { return base + (size_t)(hd + 1) * rows + row; }
};
__host__ __device__ constexpr size_t slot_floats(int hd, int blocks) { return (size_t)(hd + 2) * kTile * blocks; }
constexpr size_t kStatusBytes = kMaxGrid * 4;
__device__ __forceinline__ Partial slot_of(const TreeAttnArgs& a, int slot, int hd, int blocks) {
  return Partial{reinterpret_cast<float*>(reinterpret_cast<uint8_t*>(a.workspace) + kStatusBytes) +
                     (size_t)slot * slot_floats(hd, blocks),
                 kTile * blocks};
}

}  // namespace

template <typename T, int HD, int BLOCKS>
__global__ void __launch_bounds__(kTaThreads, 1)
    tree_attention_kernel(const TreeAttnArgs a, const __grid_constant__ CUtensorMap kmap,
                          const __grid_constant__ CUtensorMap vmap) {
  constexpr int NS = stages(HD, BLOCKS), kStage = stage_bytes(HD), kChunks = HD / 64, kChunkBytes = kTile * 128;
  constexpr int kRows = kTile * BLOCKS;
  constexpr uint32_t kIdescS = idesc16(Num<T>::kFormat, kTile, kTile, false);
  constexpr uint32_t kIdescO = idesc16(Num<T>::kFormat, kTile, HD, true);
  extern __shared__ uint8_t smem_raw[];
  uint8_t* qbuf = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  uint8_t* ring = qbuf + BLOCKS * kStage;
  uint64_t* full = reinterpret_cast<uint64_t*>(ring + NS * kStage);
  uint64_t* fixed = full + NS;     // [NS], by tiles: a tile's values are fit for the product
  uint64_t* empty = fixed + NS;
  uint64_t* s_full = empty + NS;   // [2] scores of a group are in tensor memory
  uint64_t* p_full = s_full + 2;   // [2] probabilities are, and O is scaled
  uint64_t* o_full = p_full + 2;   // [2] a segment's last product is done
  uint64_t* ready = o_full + 2;    // [2] the group has read O and laid out its queries
  uint64_t* pair = ready + 2;      // the two groups meet
  uint64_t* drain = pair + 1;      // every product is done
  uint32_t* misc = reinterpret_cast<uint32_t*>(drain + 1);
  uint32_t* tmem_slot = misc;
  volatile int* abort_flag = reinterpret_cast<volatile int*>(misc + 1);
  int* start_b = reinterpret_cast<int*>(misc + 2);
  int* start_off = start_b + 1;
  uint32_t* odd = misc + 4;        // [NS][2], by tiles: its tree values held infinities or NaN
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int group = a.n_q_heads / a.n_kv_heads;

  // ---- this CTA's range -------------------------------------------------------
  __shared__ int64_t s_sum[kTaThreads / 32];
  int64_t total = 0;
  for (int b0 = 0; b0 < a.batch; b0 += kTaThreads)
    if (b0 + tid < a.batch) total += seq_cost(a, seq_of(a, b0 + tid, kRows));
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) total += __shfl_xor_sync(0xffffffffu, total, o);
  if (lane == 0) s_sum[warp] = total;
  if (tid == 0) {
    for (int i = 0; i < NS; ++i) { mbar_init(full + i, 1); mbar_init(fixed + i, 2); mbar_init(empty + i, 1); }
    for (int i = 0; i < 2; ++i) { mbar_init(s_full + i, 1); mbar_init(p_full + i, 4); mbar_init(o_full + i, 1); mbar_init(ready + i, 4); }
    mbar_init(pair, 8);
    mbar_init(drain, 1);
    fence_barrier_init();
    *abort_flag = 0;
  }
  __syncthreads();
  total = 0;
  for (int i = 0; i < kTaThreads / 32; ++i) total += s_sum[i];
  const int64_t lo = range_at(blockIdx.x, total, gridDim.x), hi = range_at(blockIdx.x + 1, total, gridDim.x);
  if (tid == 0) reinterpret_cast<uint32_t*>(a.workspace)[blockIdx.x] = 0;  // status: raised where a wait runs out
  pdl_trigger();
  if (lo >= hi) return;
  int64_t run = 0;
  for (int b0 = 0; b0 < a.batch && run <= lo; b0 += kTaThreads) {
    const int64_t cost = b0 + tid < a.batch ? seq_cost(a, seq_of(a, b0 + tid, kRows)) : 0;
    int64_t inc = cost;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int64_t t = __shfl_up_sync(0xffffffffu, inc, o);
      if (lane >= o) inc += t;
    }
    __syncthreads();
    if (lane == 31) s_sum[warp] = inc;
    __syncthreads();
    for (int i = 0; i < kTaThreads / 32; ++i) {
      if (i < warp) inc += s_sum[i];
    }
    inc += run;
    if (inc > lo && inc - cost <= lo) { *start_b = b0 + tid; *start_off = (int)(lo - (inc - cost)); }
    for (int i = 0; i < kTaThreads / 32; ++i) run += s_sum[i];
  }
  if (warp == 1) tmem_alloc(tmem_slot, 512);
  if (tid == 0) { tma_prefetch_desc(&kmap); tma_prefetch_desc(&vmap); }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = *tmem_slot;
  Walk w;
  w.left = hi - lo;
  w.b = *start_b;
  w.off = *start_off;
  w.s = seq_of(a, w.b, kRows);
  int item0 = 0;  // items of the segments before this one
  bool ok = true;

  if (warp == 0) {
    // ---- loads ------------------------------------------------------------------
    int issued = 0;
    while (ok && w.next(a, kRows)) {
      const int n = w.t1 - w.t0;
      const int32_t* row = a.page_table + (size_t)w.b * a.max_pages;
      const int last_page = (w.s.keys - 1) / kPageTok;
      for (int i = 0; i < 2 * n && ok; ++i) {
        bool v;
        const int j = tile_of<BLOCKS>(i, n, v);
        const int item = item0 + i, st = item % NS;
        const int p0 = (w.t0 + j) * kTilePages, pages = min(kTilePages, last_page - p0 + 1);
        int page = 0;
        if (lane < kTilePages * kChunks) {
          const int q = lane / kChunks;
          if (q < pages) {
            page = row[p0 + q];
            if ((uint32_t)page >= (uint32_t)a.n_pages) page = a.n_pages;  // out of the tensor: reads as zeros
          }
        }
        ok = warp_wait(empty + st, ((item / NS) & 1) ^ 1, abort_flag);
        if (!ok) break;
        if (elect_one()) mbar_arrive_expect_tx(full + st, (uint32_t)pages * kChunks * kPageTok * 128);
        __syncwarp();
        const int q = lane / kChunks, c = lane % kChunks;
        if (lane < pages * kChunks)
          tma_load_4d(ring + st * kStage + c * kChunkBytes + q * kPageTok * 128, v ? &vmap : &kmap, full + st, c * 64, 0,
                      w.head, page);
        __syncwarp();
        issued = item + 1;
      }
      item0 += 2 * n;
    }
    if (!ok) {  // let the copies in flight land before the CTA goes
      *abort_flag = 1;
      for (int it = max(0, issued - NS); it < issued; ++it) mbar_drain(full + it % NS, (it / NS) & 1);
    }
  } else if (warp == 1) {
    // ---- products ---------------------------------------------------------------
    uint32_t ph_p[2] = {0, 0}, ph_ready = 0;
    const uint32_t q_addr = smem_u32(qbuf), r_addr = smem_u32(ring);
    auto wait_full = [&](uint64_t* bars, int item) { ok = ok && warp_wait(bars + item % NS, (item / NS) & 1, abort_flag); };
    auto scores = [&](int g, int item) {
      const uint32_t qa = q_addr + (BLOCKS == 2 ? g * kStage : 0), kb = r_addr + (item % NS) * kStage;
      if (elect_one()) {
#pragma unroll
        for (int k = 0; k < HD / 16; ++k) {
          const uint32_t at = (k / 4) * kChunkBytes + (k % 4) * 32;
          umma_ss(tmem + g * kTile, sw128_desc(qa + at), sw128_desc(kb + at), kIdescS, k > 0);
        }
        umma_commit(s_full + g);
      }
      __syncwarp();
    };
    auto outputs = [&](int g, int item, bool first, int keys) {
      const uint32_t vb = r_addr + (item % NS) * kStage;
      // keys past the end have probability 0: whole steps of 16 are left out
      const int steps = min(kTile / 16, (keys + 15) / 16);
      if (elect_one()) {
        for (int k = 0; k < steps; ++k)
          umma_ts(tmem + 2 * kTile + g * HD, tmem + g * kTile + k * 8, sw128_flip_desc(vb + k * 2048, kChunkBytes), kIdescO,
                  !(first && k == 0));
      }
      __syncwarp();
    };
    auto commit = [&](uint64_t* bar) {
      if (elect_one()) umma_commit(bar);
      __syncwarp();
    };
    auto wait_p = [&](int g) {
      ok = ok && warp_wait(p_full + g, ph_p[g], abort_flag);
      ph_p[g] ^= 1;
      tc_fence_after();
    };
    while (ok && w.next(a, kRows)) {
      const int n = w.t1 - w.t0;
      auto left = [&](int j) { return w.s.keys - (w.t0 + j) * kTile; };
      ok = ok && warp_wait(ready + 0, ph_ready, abort_flag) && warp_wait(ready + 1, ph_ready, abort_flag);
      ph_ready ^= 1;
      tc_fence_after();
      wait_full(full, item0 + item_k<BLOCKS>(0));
      if (!ok) break;
      scores(0, item0 + item_k<BLOCKS>(0));
      if (BLOCKS == 2) {
        scores(1, item0 + item_k<BLOCKS>(0));
        commit(empty + (item0 + item_k<BLOCKS>(0)) % NS);
        for (int j = 0; j < n && ok; ++j) {
          const int iv = item0 + item_v<BLOCKS>(j, n), ik = item0 + item_k<BLOCKS>(j + 1);
          const bool more = j + 1 < n;
          wait_full(fixed, item0 / 2 + j);
          if (more) wait_full(full, ik);
#pragma unroll
          for (int g = 0; g < 2; ++g) {
            wait_p(g);
            if (!ok) break;
            outputs(g, iv, j == 0, left(j));
            if (more) scores(g, ik); else commit(o_full + g);
          }
          if (!ok) break;
          commit(empty + iv % NS);
          if (more) commit(empty + ik % NS);
        }
      } else {
        commit(empty + (item0 + item_k<BLOCKS>(0)) % NS);
        if (n > 1) {
          const int ik = item0 + item_k<BLOCKS>(1);
          wait_full(full, ik);
          if (!ok) break;
          scores(1, ik);
          commit(empty + ik % NS);
        }
        for (int j = 0; j < n && ok; ++j) {
          const int g = j & 1, iv = item0 + item_v<BLOCKS>(j, n);
          wait_full(fixed, item0 / 2 + j);
          wait_p(g);
          if (!ok) break;
          outputs(g, iv, j < 2, left(j));
          commit(empty + iv % NS);
          if (j + 2 < n) {
            const int ik = item0 + item_k<BLOCKS>(j + 2);
            wait_full(full, ik);
            if (!ok) break;
            scores(g, ik);
            commit(empty + ik % NS);
          }
        }
        if (!ok) break;
        commit(o_full + 0);
        commit(o_full + 1);
      }
      item0 += 2 * n;
    }
    if (!ok) *abort_flag = 1;
    // products in flight read shared memory and write tensor memory: let them end
    commit(drain);
    mbar_drain(drain, 0);
  } else if (warp < 4) {
    // ---- values of tiles that reach past the context -------------------------------
    while (ok && w.next(a, kRows)) {
      const int n = w.t1 - w.t0;
      for (int j = 0; j < n && ok; ++j) {
        const int item = item0 + item_v<BLOCKS>(j, n), st = item % NS, vc = item0 / 2 + j;
        ok = warp_wait(full + st, (item / NS) & 1, abort_flag);
        if (!ok) break;
        const int k0 = (w.t0 + j) * kTile;
        if (k0 + kTile > w.s.plain) {
          const int first = max(0, w.s.plain - k0), end = w.s.keys - k0;
          constexpr int kPieces = HD / 8;
          bool any = false;
          for (int p = first * kPieces + tid - 64; p < kTile * kPieces; p += 64) {
            const int r = p / kPieces, c = p % kPieces;
            uint4* at = reinterpret_cast<uint4*>(ring + st * kStage + (c / 8) * kChunkBytes + r * 128 + (((c % 8) ^ (r & 7)) << 4));
            if (r >= end) { *at = make_uint4(0, 0, 0, 0); continue; }
            const uint4 v = *at;
            const uint4 f = make_uint4(finite_of<T>(v.x), finite_of<T>(v.y), finite_of<T>(v.z), finite_of<T>(v.w));
            if (f.x != v.x || f.y != v.y || f.z != v.z || f.w != v.w) { *at = f; any = true; }
          }
          fence_proxy_async_all();
          any = __any_sync(0xffffffffu, any);
          if (lane == 0) odd[2 * (vc % NS) + warp - 2] = any;
        }
        __syncwarp();
        if (lane == 0) mbar_arrive(fixed + vc % NS);
      }
      item0 += 2 * n;
    }
    if (!ok) *abort_flag = 1;
  } else {
    // ---- softmax: group g, a thread a row --------------------------------------------
    const int g = (warp - 4) >> 2, t = tid - 128 - g * kTile;  // t: row of the score tile = lane of tensor memory
    const uint32_t my = tmem + ((uint32_t)((warp & 3) * 32) << 16);
    const uint32_t s_addr = my + g * kTile, o_addr = my + 2 * kTile + g * HD;
    const float sl2 = fmaxf(fabsf(a.scale) * 1.4426950408889634f, 1e-30f);  // a masked score stays -inf at scale 0
    const uint32_t sign = a.scale < 0.f ? 0x80008000u : 0u;  // a negative scale turns the queries' signs
    uint32_t ph_s = 0, ph_o = 0, ph_pair = 0;
    auto meet = [&] {  // both groups, 256 threads
      __syncwarp();
      if (lane == 0) mbar_arrive(pair);
      ok = warp_wait(pair, ph_pair, abort_flag);
      ph_pair ^= 1;
    };
    while (ok && w.next(a, kRows)) {
      const int n = w.t1 - w.t0, row0 = w.block * kRows, live = w.s.nodes * group - row0;
      // queries into shared memory, swizzled; one block: each group lays out half
      {
        constexpr int kPieces = HD / 8, kMine = BLOCKS == 2 ? kTile : kTile / 2;
        uint8_t* dst = qbuf + (BLOCKS == 2 ? g * kStage : 0);
        const T* q = reinterpret_cast<const T*>(a.q) + (int64_t)w.b * a.width * a.q_stride + (int64_t)w.head * group * HD;
        for (int p = t; p < kMine * kPieces; p += kTile) {
          const int r = p / kPieces + (BLOCKS == 2 ? 0 : g * kMine), c = p % kPieces;
          const int gr = r + (BLOCKS == 2 ? g * kTile : 0);  // row of the unit's block
          uint4 v = make_uint4(0, 0, 0, 0);
          if (gr < live) {
            const int node = (row0 + gr) / group, h = (row0 + gr) - node * group;
            v = *reinterpret_cast<const uint4*>(q + (int64_t)node * a.q_stride + h * HD + c * 8);
            v.x ^= sign; v.y ^= sign; v.z ^= sign; v.w ^= sign;
          }
          *reinterpret_cast<uint4*>(dst + (c / 8) * kChunkBytes + r * 128 + (((c % 8) ^ (r & 7)) << 4)) = v;
        }
        fence_proxy_async_all();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(ready + g);
      }
      const int row = row0 + (BLOCKS == 2 ? g * kTile : 0) + t;  // of the unit
      const int node = min(row / group, w.s.nodes - 1);
      const uint32_t* mrow = reinterpret_cast<const uint32_t*>(a.mask + ((size_t)w.b * a.width + node) * a.words);
      const int32_t* pages = a.page_table + (size_t)w.b * a.max_pages;
      const int n_pg = (w.s.keys + kPageTok - 1) / kPageTok;
      const int j0 = BLOCKS == 2 ? 0 : g, jn = BLOCKS == 2 ? 1 : 2;
      auto page_flag = [&](int j) -> uint32_t {  // this lane's page of tile j is one of the pool
        const int p = (w.t0 + j) * kTilePages + lane;
        return lane >= kTilePages || p >= n_pg || (uint32_t)pages[p] < (uint32_t)a.n_pages;
      };
      float m_ref = -INFINITY, sum = 0.f;
      bool patch = false;  // values that the rows who see them get back in the epilogue
      uint32_t flag = j0 < n ? page_flag(j0) : 1u;
      for (int j = j0; j < n; j += jn) {
        const uint32_t flags = __ballot_sync(0xffffffffu, flag);
        if (j + jn < n) flag = page_flag(j + jn);
        ok = warp_wait(s_full + g, ph_s, abort_flag);
        if (!ok) break;
        ph_s ^= 1;
        tc_fence_after();
        uint32_t v[kTile];
#pragma unroll
        for (int c = 0; c < 4; ++c) tm_ld32(s_addr + 32 * c, v + 32 * c);
        tm_wait_ld();
        const int k0 = (w.t0 + j) * kTile;
        const bool tail = k0 + kTile > w.s.plain;
        if (tail || flags != 0xFFFFFFFFu) {
#pragma unroll
          for (int c = 0; c < 4; ++c) {
            uint32_t m = allowed32(mrow, 2 * a.words, k0 + 32 * c, w.s);
            m &= ((flags >> (2 * c)) & 1 ? 0xFFFFu : 0u) | ((flags >> (2 * c + 1)) & 1 ? 0xFFFF0000u : 0u);
#pragma unroll
            for (int i = 0; i < 32; ++i)
              if (!(m >> i & 1)) v[32 * c + i] = 0xFF800000u;
          }
        }
        float mx[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
        for (int i = 0; i < kTile; ++i) mx[i & 3] = fmaxf(mx[i & 3], __uint_as_float(v[i]));
        const float top = fmaxf(fmaxf(mx[0], mx[1]), fmaxf(mx[2], mx[3])) * sl2;
        if (j == j0) {
          m_ref = top;
        } else if (__any_sync(0xffffffffu, top > m_ref + kLazy)) {
          const float m_new = fmaxf(m_ref, top);
          const float alpha = m_new == m_ref ? 1.0f : ex2(m_ref - m_new);
          m_ref = m_new;
          sum *= alpha;
#pragma unroll
          for (int c = 0; c < HD / 32; ++c) {
            uint32_t o[32];
            tm_ld32(o_addr + 32 * c, o);
            tm_wait_ld();
#pragma unroll
            for (int i = 0; i < 32; ++i) o[i] = __float_as_uint(__uint_as_float(o[i]) * alpha);
            tm_st32(o_addr + 32 * c, o);
          }
        }
        const float base = m_ref == -INFINITY ? 0.f : m_ref;
        float acc[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          uint32_t p[32];
#pragma unroll
          for (int i = 0; i < 32; ++i) {
            const float x = ex2(fmaf(__uint_as_float(v[64 * h + 2 * i]), sl2, -base));
            const float y = ex2(fmaf(__uint_as_float(v[64 * h + 2 * i + 1]), sl2, -base));
            acc[2 * (i & 1)] += x;
            acc[2 * (i & 1) + 1] += y;
            p[i] = Num<T>::pack(x, y);
          }
          tm_st32(s_addr + 32 * h, p);
        }
        tm_wait_st();
        sum += (acc[0] + acc[1]) + (acc[2] + acc[3]);
        if (tail) {  // the stage is not refilled before this group's probabilities are used
          const int vc = item0 / 2 + j;
          ok = warp_wait(fixed + vc % NS, (vc / NS) & 1, abort_flag);
          if (!ok) break;
          patch |= (odd[2 * (vc % NS)] | odd[2 * (vc % NS) + 1]) != 0;
        }
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(p_full + g);
      }
      if (!ok) break;
      ok = warp_wait(o_full + g, ph_o, abort_flag);
      if (!ok) break;
      ph_o ^= 1;
      tc_fence_after();
      // ---- epilogue: a group's own accumulator, or half the columns of both groups' ----
      float m_row = m_ref, l_row = sum, w0 = 1.f, w1 = 0.f;
      if (BLOCKS == 1) {
        float4* ml = reinterpret_cast<float4*>(qbuf);  // the queries have been read
        ml[g * kTile + t] = make_float4(m_ref, sum, patch ? 1.f : 0.f, 0.f);
        meet();
        if (!ok) break;
        const float4 x = ml[t], y = ml[kTile + t];
        patch = x.z + y.z > 0.f;
        m_row = fmaxf(x.x, y.x);
        w0 = x.x == -INFINITY ? 0.f : ex2(x.x - m_row);
        w1 = y.x == -INFINITY ? 0.f : ex2(y.x - m_row);
        l_row = x.y * w0 + y.y * w1;
      }
      constexpr int kCols = BLOCKS == 2 ? HD : HD / 2;
      const int col0 = BLOCKS == 2 ? 0 : g * kCols;
      const bool whole = w.t0 == 0 && w.t1 == w.s.tiles, on = row < w.s.nodes * group;
      const float inv = whole ? (l_row > 0.f ? 1.0f / l_row : 0.f) : 1.f;
      const int in_block = (BLOCKS == 2 ? g * kTile : 0) + t;
      const Partial part = slot_of(a, 2 * blockIdx.x + (w.t0 > 0 ? 0 : 1), HD, BLOCKS);
      T* out = reinterpret_cast<T*>(a.out) +
               (((int64_t)w.b * a.width + node) * a.n_q_heads + (int64_t)w.head * group + (row - node * group)) * HD;
#pragma unroll
      for (int c = 0; c < kCols / 32; ++c) {
        uint32_t o[32];
        if (BLOCKS == 2) {
          tm_ld32(o_addr + 32 * c, o);
          tm_wait_ld();
        } else {
          uint32_t o1[32];
          tm_ld32(my + 2 * kTile + col0 + 32 * c, o);
          tm_ld32(my + 2 * kTile + HD + col0 + 32 * c, o1);
          tm_wait_ld();
          // a group without a tile has written nothing there
#pragma unroll
          for (int i = 0; i < 32; ++i)
            o[i] = __float_as_uint((n > 1 ? __uint_as_float(o1[i]) * w1 : 0.f) + __uint_as_float(o[i]) * w0);
        }
        if (patch && on) {
          for (int i = 0; i < w.s.nodes; ++i) {
            const int pos = w.s.ctx + i;
            if (pos < w.t0 * kTile || pos >= min(w.t1 * kTile, w.s.keys) || !(mrow[i >> 5] >> (i & 31) & 1)) continue;
            const int page = pages[pos / kPageTok];
            if ((uint32_t)page >= (uint32_t)a.n_pages) continue;
            const T* vp = reinterpret_cast<const T*>(a.v_cache) + page * a.page_stride +
                          ((int64_t)w.head * kPageTok + pos % kPageTok) * HD + col0 + 32 * c;
#pragma unroll
            for (int e = 0; e < 32; ++e) {
              const float x = Num<T>::get(vp + e);
              if (!(fabsf(x) < INFINITY)) o[e] = __float_as_uint(__uint_as_float(o[e]) + x);
            }
          }
        }
        if (!on) continue;
        if (whole) {
#pragma unroll
          for (int i = 0; i < 32; ++i) o[i] = __float_as_uint(__uint_as_float(o[i]) * inv);
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            uint4 p;
            p.x = Num<T>::pack(__uint_as_float(o[8 * i]), __uint_as_float(o[8 * i + 1]));
            p.y = Num<T>::pack(__uint_as_float(o[8 * i + 2]), __uint_as_float(o[8 * i + 3]));
            p.z = Num<T>::pack(__uint_as_float(o[8 * i + 4]), __uint_as_float(o[8 * i + 5]));
            p.w = Num<T>::pack(__uint_as_float(o[8 * i + 6]), __uint_as_float(o[8 * i + 7]));
            *reinterpret_cast<uint4*>(out + col0 + 32 * c + 8 * i) = p;
          }
        } else {
#pragma unroll
          for (int i = 0; i < 8; ++i)
            *part.o((col0 + 32 * c) / 4 + i, in_block) =
                make_float4(__uint_as_float(o[4 * i]), __uint_as_float(o[4 * i + 1]), __uint_as_float(o[4 * i + 2]),
                            __uint_as_float(o[4 * i + 3]));
        }
      }
      if (!whole && on && (BLOCKS == 2 || g == 0)) {
        *part.max_of(HD, in_block) = m_row;
        *part.sum_of(HD, in_block) = l_row;
      }
      if (BLOCKS == 1) {  // the queries' place holds the sums, and each group reads both accumulators
        meet();
        if (!ok) break;
      }
      item0 += 2 * n;
    }
    if (!ok) *abort_flag = 1;
  }
  tc_fence_before();
  __syncthreads();
  if (tid == 0 && *abort_flag) reinterpret_cast<uint32_t*>(a.workspace)[blockIdx.x] = 1;
  if (warp == 1) tmem_dealloc(tmem, 512);
}

// Joins the partials of units that several CTAs shared, in tile order, and
// zeroes the rows of unused nodes.  A lane takes a row, a warp HD / 32 groups
// of four columns.  A stalled pipeline in any CTA turns the output into NaN:
// never into numbers that look right.
constexpr int kCombineThreads = 256, kCombineRows = 32;

template <typename T, int HD, int BLOCKS>
__global__ void __launch_bounds__(kCombineThreads) tree_combine_kernel(const TreeAttnArgs a, int grid) {
  constexpr int kRows = kTile * BLOCKS, kC4 = HD / 32;
  __shared__ int64_t s_sum[2][kCombineThreads / 32];
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int b = blockIdx.z, head = blockIdx.y, group = a.n_q_heads / a.n_kv_heads;
  const int row = blockIdx.x * kCombineRows + lane;
  int64_t total = 0, before = 0;
  for (int i = tid; i < a.batch; i += kCombineThreads) {
    const int64_t c = seq_cost(a, seq_of(a, i, kRows));
    total += c;
    if (i < b) before += c;
  }
  const Seq s = seq_of(a, b, kRows);
  pdl_wait();
  const int stalled = __syncthreads_or(tid < grid && reinterpret_cast<const uint32_t*>(a.workspace)[tid] != 0);
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    total += __shfl_xor_sync(0xffffffffu, total, o);
    before += __shfl_xor_sync(0xffffffffu, before, o);
  }
  if (lane == 0) { s_sum[0][warp] = total; s_sum[1][warp] = before; }
  __syncthreads();
  total = before = 0;
  for (int i = 0; i < kCombineThreads / 32; ++i) { total += s_sum[0][i]; before += s_sum[1][i]; }
  if (row >= a.width * group) return;
  const int node = row / group;
  T* out = reinterpret_cast<T*>(a.out) +
           (((int64_t)b * a.width + node) * a.n_q_heads + (int64_t)head * group + (row - node * group)) * HD;
  float4 acc[kC4];
  float scale = 0.f;
#pragma unroll
  for (int e = 0; e < kC4; ++e) acc[e] = make_float4(0.f, 0.f, 0.f, 0.f);
  if (stalled) {
    scale = __int_as_float(0x7FC00000);
  } else if (node < s.nodes) {
    const int block = row / kRows, r = row % kRows;
    const int64_t t0 = before + (int64_t)(head * s.blocks + block) * s.tiles;
    const int first = (int)(((t0 + 1) * grid - 1) / total), last = (int)(((t0 + s.tiles) * grid - 1) / total);
    if (first == last) return;  // written whole
    float m = -INFINITY, l = 0.f;
    for (int c = first; c <= last; ++c) {
      if (range_at(c, total, grid) == range_at(c + 1, total, grid)) continue;  // a CTA without a tile
      m = fmaxf(m, *slot_of(a, 2 * c + (c == first ? 1 : 0), HD, BLOCKS).max_of(HD, r));
    }
    for (int c = first; c <= last; ++c) {
      if (range_at(c, total, grid) == range_at(c + 1, total, grid)) continue;
      const Partial p = slot_of(a, 2 * c + (c == first ? 1 : 0), HD, BLOCKS);
      const float mc = *p.max_of(HD, r), w = mc == -INFINITY ? 0.f : ex2(mc - m);
      l = fmaf(*p.sum_of(HD, r), w, l);
#pragma unroll
      for (int e = 0; e < kC4; ++e) {
        const float4 v = *p.o(warp * kC4 + e, r);
        acc[e].x = fmaf(v.x, w, acc[e].x);
        acc[e].y = fmaf(v.y, w, acc[e].y);
        acc[e].z = fmaf(v.z, w, acc[e].z);
        acc[e].w = fmaf(v.w, w, acc[e].w);
      }
    }
    scale = l > 0.f ? 1.0f / l : 0.f;
  }
#pragma unroll
  for (int e = 0; e < kC4; ++e) {
    uint2 p;
    p.x = Num<T>::pack(acc[e].x * scale, acc[e].y * scale);
    p.y = Num<T>::pack(acc[e].z * scale, acc[e].w * scale);
    *reinterpret_cast<uint2*>(out + (warp * kC4 + e) * 4) = p;
  }
}

namespace {

PFN_cuTensorMapEncodeTiled_v12000 encoder() {
  static PFN_cuTensorMapEncodeTiled_v12000 fn = [] {
    void* p = nullptr;
    cudaDriverEntryPointQueryResult q;
    if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &p, 12000, cudaEnableDefault, &q) != cudaSuccess ||
        q != cudaDriverEntryPointSuccess)
      p = nullptr;
    return reinterpret_cast<PFN_cuTensorMapEncodeTiled_v12000>(p);
  }();
  return fn;
}

// The cache as [page][head][token][entry], boxes of 16 tokens x 64 entries.
CUtensorMap cache_map(const TreeAttnArgs& a, const void* base) {
  CUtensorMap m;
  std::memset(&m, 0, sizeof(m));
  auto enc = encoder();
  if (!enc) throw cudaErrorNotSupported;
  const cuuint64_t hd = a.head_dim;
  const cuuint64_t dims[4] = {hd, (cuuint64_t)kPageTok, (cuuint64_t)a.n_kv_heads, (cuuint64_t)a.n_pages};
  const cuuint64_t strides[3] = {hd * 2, hd * 2 * kPageTok, (cuuint64_t)a.page_stride * 2};
  const cuuint32_t box[4] = {64, (cuuint32_t)kPageTok, 1, 1}, es[4] = {1, 1, 1, 1};
  const CUresult r = enc(&m, a.dtype == DT_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 4,
                         const_cast<void*>(base), dims, strides, box, es, CU_TENSOR_MAP_INTERLEAVE_NONE,
                         CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
  if (r != CUDA_SUCCESS) throw cudaErrorInvalidValue;
  return m;
}

int query_blocks(int width, int group) { return width * group <= kTile ? 1 : 2; }

template <typename T, int HD, int BLOCKS>
void run_attention(const TreeAttnArgs& a, cudaStream_t s) {
  constexpr int smem = smem_bytes(HD, BLOCKS);
  auto* kernel = tree_attention_kernel<T, HD, BLOCKS>;
  static const cudaError_t configured = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
  if (configured != cudaSuccess) throw configured;
  static const int sms = [] {
    int dev = 0, n = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess) n = 1;
    return n;
  }();
  const int grid = sms < kMaxGrid ? sms : kMaxGrid, group = a.n_q_heads / a.n_kv_heads;
  const CUtensorMap km = cache_map(a, a.k_cache), vm = cache_map(a, a.v_cache);
  kernel<<<grid, kTaThreads, smem, s>>>(a, km, vm);
  cudaError_t e = cudaGetLastError();
  if (e != cudaSuccess) throw e;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((a.width * group + kCombineRows - 1) / kCombineRows, a.n_kv_heads, a.batch);
  cfg.blockDim = dim3(kCombineThreads);
  cfg.stream = s;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  e = cudaLaunchKernelEx(&cfg, tree_combine_kernel<T, HD, BLOCKS>, a, grid);
  if (e != cudaSuccess) throw e;
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

size_t tree_attention_workspace(int, int width, int n_q_heads, int n_kv_heads, int head_dim) {
  return kStatusBytes + 2 * kMaxGrid * slot_floats(head_dim, query_blocks(width, n_q_heads / n_kv_heads)) * sizeof(float);
}

void launch_tree_attention(const TreeAttnArgs& a, cudaStream_t s) {
  if (a.dtype == DT_BF16) run_typed<__nv_bfloat16>(a, s); else run_typed<__half>(a, s);
}

}  // namespace pard
