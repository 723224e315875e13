// What the attention kernels over the paged cache share: types, tcgen05 and
// tensor-memory access beyond common.cuh, pairs of floats, the cache's tensor
// map, and how a unit's parts are cut and joined (partials in the workspace,
// arrivals at its beginning).
#pragma once

#include <cuda_fp16.h>

#include <cstring>

#include <cudaTypedefs.h>

#include "common.cuh"
#include "per_device.h"
#include "tree.h"
#include "warp_wait.cuh"

namespace pard {

namespace {

constexpr int kTile = 128;                      // keys a tile, rows a score tile
constexpr int kTilePages = kTile / kPageTok;
constexpr int kSplit = 6;                       // what splitting a unit costs in tiles
constexpr int kMaxGrid = 160;                   // workspace slots are sized for this many CTAs
constexpr float kLazy = 8.0f;                   // growth of a maximum, in powers of two, that is let pass

__host__ __device__ constexpr int stage_bytes(int hd) { return kTile * hd * 2; }
template <typename T> struct Num;
template <> struct Num<__nv_bfloat16> {
  static constexpr uint32_t kFormat = 1;        // of the instruction descriptor
  static constexpr uint32_t kExponent = 0x7F80; // all ones: infinity or NaN
  static constexpr float kRaise = 0.f;          // probabilities are held times 2^kRaise
  static __device__ __forceinline__ uint32_t pack(float x, float y) {
    __nv_bfloat162 p = __floats2bfloat162_rn(x, y);
    return *reinterpret_cast<uint32_t*>(&p);
  }
  static __device__ __forceinline__ float get(const void* p) { return __bfloat162float(*reinterpret_cast<const __nv_bfloat16*>(p)); }
  // two values times zero, added: NaN where one was infinite or NaN
  static __device__ __forceinline__ uint32_t times_zero(uint32_t x, uint32_t sum) {
    asm("fma.rn.bf16x2 %0, %1, %2, %0;" : "+r"(sum) : "r"(x), "r"(0u));
    return sum;
  }
};
template <> struct Num<__half> {
  static constexpr uint32_t kFormat = 0;
  static constexpr uint32_t kExponent = 0x7C00;
  static constexpr float kRaise = 7.f;          // times 2^kLazy still below 65504
  static __device__ __forceinline__ uint32_t pack(float x, float y) {
    __half2 p = __floats2half2_rn(x, y);
    return *reinterpret_cast<uint32_t*>(&p);
  }
  static __device__ __forceinline__ float get(const void* p) { return __half2float(*reinterpret_cast<const __half*>(p)); }
  static __device__ __forceinline__ uint32_t times_zero(uint32_t x, uint32_t sum) {
    asm("fma.rn.f16x2 %0, %1, %2, %0;" : "+r"(sum) : "r"(x), "r"(0u));
    return sum;
  }
};

// Instruction descriptor, kind::f16, fp32 accumulator, A K-major; `flip`: B
// lies with its N entries contiguous.
__host__ __device__ constexpr uint32_t idesc16(uint32_t fmt, int M, int N, bool flip) {
  return (1u << 4) | (fmt << 7) | (fmt << 10) | ((flip ? 1u : 0u) << 16) | ((uint32_t)(N >> 3) << 17) |
         ((uint32_t)(M >> 4) << 24);
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
// ... after which registers hold what was loaded: nothing moves their uses before it
template <int N>
__device__ __forceinline__ void tm_landed(uint32_t* r) {
  tm_wait_ld();
#pragma unroll
  for (int i = 0; i < N; ++i) asm volatile("" : "+r"(r[i]));
}
__device__ __forceinline__ void tm_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
// two 32-bit floats at a time
__device__ __forceinline__ uint64_t pair_of(uint32_t x, uint32_t y) {
  uint64_t p;
  asm("mov.b64 %0, {%1, %2};" : "=l"(p) : "r"(x), "r"(y));
  return p;
}
__device__ __forceinline__ float2 floats_of(uint64_t p) {
  uint32_t x, y;
  asm("mov.b64 {%0, %1}, %2;" : "=r"(x), "=r"(y) : "l"(p));
  return make_float2(__uint_as_float(x), __uint_as_float(y));
}
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c) {
  uint64_t d;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d) : "l"(a), "l"(b), "l"(c));
  return d;
}
__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b) {
  uint64_t d;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
  return d;
}
// This row's accumulator times alpha, 16 columns a turn: the scores stay in
// their registers meanwhile.
template <int HD>
__device__ __forceinline__ void scale_row(uint32_t o_addr, float alpha) {
#pragma unroll 1
  for (int c = 0; c < HD; c += 16) {
    uint32_t o[16];
    tmem_ld16(o_addr + c, o);
#pragma unroll
    for (int i = 0; i < 16; ++i) o[i] = __float_as_uint(__uint_as_float(o[i]) * alpha);
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x16.b32 [%16], {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15};" ::"r"(o[0]),
        "r"(o[1]), "r"(o[2]), "r"(o[3]), "r"(o[4]), "r"(o[5]), "r"(o[6]), "r"(o[7]), "r"(o[8]), "r"(o[9]), "r"(o[10]),
        "r"(o[11]), "r"(o[12]), "r"(o[13]), "r"(o[14]), "r"(o[15]), "r"(o_addr + c)
        : "memory");
  }
}
// 32 bytes of an output row: rows lie apart, so what a warp writes at once are
// pieces of 32 rows, and whole 32-byte sectors take half the passes of 16 bytes.
__device__ __forceinline__ void store32(void* to, const uint32_t* v, bool wide) {
  if (wide) {
    asm volatile("st.global.v8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};" ::"l"(to), "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]),
                 "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7])
                 : "memory");
  } else {
    reinterpret_cast<uint4*>(to)[0] = make_uint4(v[0], v[1], v[2], v[3]);
    reinterpret_cast<uint4*>(to)[1] = make_uint4(v[4], v[5], v[6], v[7]);
  }
}
// Two 16-bit values with infinities and NaN replaced by zero.
template <typename T>
__device__ __forceinline__ uint32_t finite_of(uint32_t v) {
  constexpr uint32_t e = Num<T>::kExponent;
  if ((v & e) == e) v &= 0xFFFF0000u;
  if ((v >> 16 & e) == e) v &= 0x0000FFFFu;
  return v;
}
// Parts of a unit of so many tiles where a part has `most`: one that is longer
// by less than a split costs stays whole.
template <int SPLIT = kSplit>
__device__ __forceinline__ int parts_of(int tiles, int most) {
  // Exact below 2^21 tiles: the quotient is 0.5 / most off any whole number, and
  // __fdividef off by two units in the last place at most, 2^-22 (tiles + most) / most.
  // Above, with the numerator's own rounding, it is off by up to 4 / most: a part more or
  // less, which those who look for `most` leave room for.
  return tiles <= most + SPLIT ? 1 : (int)__fdividef((float)(tiles + most) - 0.5f, (float)most);
}
// Where CTA c's range begins: floor(total c / grid).  With fewer places than
// CTAs a range is one place or none, and its beginning is then also the number
// of CTAs before c that have one.
template <int SPLIT>
struct RangesOf {
  int total, grid, each, rest;
  uint32_t magic;  // 2^32 / grid, rounded up: c rest < grid^2
  __device__ __forceinline__ void set(int n, int g) {
    magic = 0xFFFFFFFFu / (uint32_t)g + 1;
    total = n;
    grid = g;
    each = n / g;
    rest = n - each * g;
  }
  __device__ __forceinline__ int at(int c) const { return c * each + (int)__umulhi((uint32_t)(c * rest), magic); }
  // a cut at place x of a unit of `len` places: near an end it moves there
  static __device__ __forceinline__ int cut(int x, int len) {
    return x <= SPLIT ? 0 : x >= len - SPLIT ? len : x;
  }
};
using Ranges = RangesOf<kSplit>;

// A slot holds one partial, rows = 128 * blocks: O as [HD / 4][rows] float4,
// then each softmax group's maxima and sums.  Before the slots: arrivals at a
// unit, by the CTA that has its first tile, for each group.
struct Partial {
  float* base;
  int rows, c4_step, row_step = 1;  // steps: of O
  __device__ __forceinline__ float4* o(int c4, int row) const { return reinterpret_cast<float4*>(base) + (size_t)c4 * c4_step + (size_t)row * row_step; }
  __device__ __forceinline__ float2* stats(int hd, int g, int row) const {
    return reinterpret_cast<float2*>(base + (size_t)hd * rows) + (size_t)g * rows + row;
  }
};
__host__ __device__ constexpr size_t slot_floats(int hd, int blocks) { return (size_t)(hd + 4) * kTile * blocks; }
// Values that not every row sees are taken out of the products where they are infinite
// or NaN; who has such says so as it arrives, and the last to arrive adds the whole
// unit's to the output, behind the join: in a partial, a weight of zero would turn an
// infinity into NaN.
constexpr uint32_t kOddArrival = 1u << 16;       // in an arrival, beside the one that counts it
// 1: those who have arrived are all of a unit's contributors but one, who is the last; 2: and one of them said so; else 0
__device__ __forceinline__ uint32_t last_of(uint32_t arrived, int count) {
  return (arrived & (kOddArrival - 1)) != (uint32_t)count - 1 ? 0u : arrived < kOddArrival ? 1u : 2u;
}
constexpr int kStalledWord = 2 * kMaxGrid;       // after the arrivals: a wait has run out in some call
constexpr size_t kArriveBytes = (kStalledWord + 4) * sizeof(uint32_t);
template <typename Args>
__device__ __forceinline__ Partial slot_of(const Args& a, int slot, int hd, int blocks) {
  return Partial{reinterpret_cast<float*>(reinterpret_cast<uint8_t*>(a.workspace) + kArriveBytes) +
                     (size_t)slot * slot_floats(hd, blocks),
                 kTile * blocks, kTile * blocks};
}
__device__ __forceinline__ uint32_t ld_acquire(const uint32_t* p) {
  uint32_t v;
  asm volatile("ld.acquire.gpu.global.u32 %0, [%1];" : "=r"(v) : "l"(p) : "memory");
  return v;
}
__device__ __forceinline__ void fence_gpu() { asm volatile("fence.acq_rel.gpu;" ::: "memory"); }
__device__ __forceinline__ uint32_t arrive_acq_rel(uint32_t* p, bool odd) {
  uint32_t old;
  asm volatile("atom.acq_rel.gpu.global.add.u32 %0, [%1], %2;" : "=r"(old) : "l"(p), "r"(odd ? kOddArrival + 1 : 1u) : "memory");
  return old;
}

// Joins a unit's partials, in order, for one group's rows and columns.  Threads
// take rows (32, 64 or 128 of them) and share a row's columns out; the loads of
// four partials' four pieces go out together.  It runs once a unit: its code
// comes from L2 as its data do, so it is kept short.
template <typename T, int HD, int BLOCKS, typename Args>
__device__ __noinline__ void join(const Args& a, const uint16_t* slots, int count, int g, int t, int row0, int rows,
                                  int c4_0, int n_c4, T* unit_out, int unit_row0) {
  const int span = rows <= 32 ? 32 : rows <= 64 ? 64 : 128, row = t & (span - 1), step = kTile / span;
  if (row >= rows) return;
  const int group = a.n_q_heads / a.n_kv_heads, r = unit_row0 + row, node = r / group;
  T* out = unit_out + ((int64_t)node * a.n_q_heads + (r - node * group)) * HD + c4_0 * 4;
#pragma unroll 1
  for (int c = t / span; c < n_c4; c += 4 * step) {
    float4 acc[4];
    float m = -INFINITY, l = 0.f;
#pragma unroll
    for (int e = 0; e < 4; ++e) acc[e] = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 1
    for (int i0 = 0; i0 < count; i0 += 4) {
      float4 v[4][4];
      float2 st[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        st[i] = make_float2(-INFINITY, 0.f);
#pragma unroll
        for (int e = 0; e < 4; ++e) v[i][e] = make_float4(0.f, 0.f, 0.f, 0.f);
        if (i0 + i < count) {
          const Partial p = slot_of(a, slots[i0 + i], HD, BLOCKS);
          st[i] = *p.stats(HD, g, row0 + row);
#pragma unroll
          for (int e = 0; e < 4; ++e) v[i][e] = *p.o(c4_0 + min(c + e * step, n_c4 - 1), row0 + row);
        }
      }
      const float top = fmaxf(fmaxf(m, fmaxf(st[0].x, st[1].x)), fmaxf(st[2].x, st[3].x)), base = top == -INFINITY ? 0.f : top;
      const float old = ex2(m - base);
      m = top;
      l *= old;
#pragma unroll
      for (int e = 0; e < 4; ++e) { acc[e].x *= old; acc[e].y *= old; acc[e].z *= old; acc[e].w *= old; }
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float w = ex2(st[i].x - base);
        l = fmaf(st[i].y, w, l);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          acc[e].x = fmaf(v[i][e].x, w, acc[e].x);
          acc[e].y = fmaf(v[i][e].y, w, acc[e].y);
          acc[e].z = fmaf(v[i][e].z, w, acc[e].z);
          acc[e].w = fmaf(v[i][e].w, w, acc[e].w);
        }
      }
    }
    const float inv = l > 0.f ? 1.0f / l : 0.f;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      uint2 p;
      p.x = Num<T>::pack(acc[e].x * inv, acc[e].y * inv);
      p.y = Num<T>::pack(acc[e].z * inv, acc[e].w * inv);
      if (c + e * step < n_c4) *reinterpret_cast<uint2*>(out + (c + e * step) * 4) = p;
    }
  }
}

// 32 columns of this row's sum, unnormalised: a group's own accumulator, or both
// groups' (the second's only if it had a tile: it has written nothing else there).
template <int HD, int BLOCKS>
__device__ __forceinline__ void own_columns(uint32_t (&o)[32], uint32_t addr, float w0, float w1, bool second) {
  tm_ld32(addr, o);
  if (BLOCKS == 1) {
    uint32_t o1[32];
    tm_ld32(addr + HD, o1);
    tm_landed<32>(o1);
    tm_landed<32>(o);
#pragma unroll
    for (int i = 0; i < 32; ++i)
      o[i] = __float_as_uint((second ? __uint_as_float(o1[i]) * w1 : 0.f) + __uint_as_float(o[i]) * w0);
  } else {
    tm_landed<32>(o);
  }
}
template <typename T>
__device__ __forceinline__ void store_columns(T* out, const uint32_t (&o)[32], float inv, bool wide) {
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    uint32_t y[8];
#pragma unroll
    for (int e = 0; e < 8; ++e)
      y[e] = Num<T>::pack(__uint_as_float(o[16 * i + 2 * e]) * inv, __uint_as_float(o[16 * i + 2 * e + 1]) * inv);
    store32(out + 16 * i, y, wide);
  }
}
// Joins the other part's partial with this CTA's own, still in tensor memory,
// with join()'s arithmetic: the first part's product, then the second's.  All
// threads of a warp take part; 64 columns' loads go out together.
template <typename T, int HD, int BLOCKS>
__device__ __noinline__ void join_two(const Partial other, uint32_t addr, int g, int row, bool first, float m, float sum,
                                      float w0, float w1, bool second, int col0, bool on, T* out, bool wide) {
  constexpr int kCols = BLOCKS == 2 ? HD : HD / 2, kPieces = kCols < 64 ? 8 : 16;
  fence_gpu();
  const float2 st = *other.stats(HD, g, row);
  float x_mine = 0.f, x_other = 0.f, inv = 0.f;
#pragma unroll 1
  for (int c0 = col0; c0 < col0 + kCols; c0 += 4 * kPieces) {
    float4 v[kPieces];
#pragma unroll
    for (int i = 0; i < kPieces; ++i) v[i] = *other.o(c0 / 4 + i, row);
    if (c0 == col0) {
      const float top = fmaxf(m, st.x), base = top == -INFINITY ? 0.f : top;
      x_mine = ex2(m - base);
      x_other = ex2(st.x - base);
      const float l = first ? fmaf(st.y, x_other, sum * x_mine) : fmaf(sum, x_mine, st.y * x_other);
      inv = l > 0.f ? 1.0f / l : 0.f;
    }
#pragma unroll
    for (int h = 0; h < kPieces / 8; ++h) {
      uint32_t o[32];
      own_columns<HD, BLOCKS>(o, addr + c0 + 32 * h, w0, w1, second);
#pragma unroll
      for (int i = 0; i < 32; ++i) {
        const float4 q = v[8 * h + i / 4];
        const float x = __uint_as_float(o[i]), y = i % 4 == 0 ? q.x : i % 4 == 1 ? q.y : i % 4 == 2 ? q.z : q.w;
        o[i] = __float_as_uint(first ? fmaf(y, x_other, x * x_mine) : fmaf(x, x_mine, y * x_other));
      }
      if (on) store_columns(out + c0 + 32 * h, o, inv, wide);
    }
  }
}

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
template <typename Args>
CUtensorMap cache_map(const Args& a, const void* base) {
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

}  // namespace

}  // namespace pard
