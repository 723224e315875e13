// What a request asks of its logits before a token is drawn: penalties for
// tokens that are there already, biases, and a grammar's mask.
//
//   z1 = z / r where z > 0, else z r          tokens seen (prompt, generated or on the row's branch)
//   z2 = z1 - f c - p [c > 0]                 c: how often the token was generated, the branch's among it
//   z3 = z2 + the token's biases
//   z4 = z3 where the row's mask allows the token, else -inf
//
// in 32 bits, rounded once to the logits' type.
//
// A CTA has one sequence's slice of the vocabulary for some of its rows.  The
// history is counted into a table of a word an entry in shared memory (whole
// numbers: no order), which then stays for all rows; a row of a tree adds its
// branch's tokens before it is worked on and takes them out after.  Biases are
// numbered in the same word, those of one token summed in the list's order by
// one thread.  So a row costs its own reading and writing, and each slice reads
// the whole history from L2, 4 bytes a token.
//
// What bounds it: HBM for many rows, and for one the chain history -> table ->
// row; a row's loads go out before the history's are looked at, and the next
// row's before this one is worked on.
#include <cuda_fp16.h>

#include "common.cuh"
#include "serve.h"

namespace pard {

namespace {

constexpr int kAdjThreads = 256;
constexpr int kAdjVectors = 4;                // 16-byte pieces of a row's slice that a thread has
constexpr uint32_t kCount = (1u << 20) - 1;   // of a table's word: how often the token was generated,
constexpr uint32_t kInPrompt = 1u << 20;      // whether the prompt has it,
constexpr int kBiasShift = 21;                // and the number of its bias (0: none)
static_assert(kMaxHistory + kTreeMaxNodes < (1 << 20) && kMaxBiases < (1 << 11), "fields of a table's word");

template <typename T> struct Entries;  // of 16 bytes
template <> struct Entries<float> {
  static constexpr int kN = 4;
  static __device__ __forceinline__ float get(const uint32_t (&w)[4], int i) { return __uint_as_float(w[i]); }
  static __device__ __forceinline__ void put(uint32_t (&w)[4], int i, float x) { w[i] = __float_as_uint(x); }
  static __device__ __forceinline__ float one(const float* p) { return *p; }
  static __device__ __forceinline__ float round(float x) { return x; }
};
template <> struct Entries<__nv_bfloat16> {
  static constexpr int kN = 8;
  static __device__ __forceinline__ float get(const uint32_t (&w)[4], int i) {
    return __uint_as_float(i & 1 ? w[i / 2] & 0xFFFF0000u : w[i / 2] << 16);
  }
  static __device__ __forceinline__ void put(uint32_t (&w)[4], int i, float x) {
    const uint32_t v = __bfloat16_as_ushort(__float2bfloat16_rn(x));
    w[i / 2] = i & 1 ? (w[i / 2] & 0x0000FFFFu) | v << 16 : (w[i / 2] & 0xFFFF0000u) | v;
  }
  static __device__ __forceinline__ float one(const __nv_bfloat16* p) { return __bfloat162float(*p); }
  static __device__ __forceinline__ __nv_bfloat16 round(float x) { return __float2bfloat16_rn(x); }
};
template <> struct Entries<__half> {
  static constexpr int kN = 8;
  static __device__ __forceinline__ float get(const uint32_t (&w)[4], int i) {
    return __half2float(__ushort_as_half((uint16_t)(i & 1 ? w[i / 2] >> 16 : w[i / 2])));
  }
  static __device__ __forceinline__ void put(uint32_t (&w)[4], int i, float x) {
    const uint32_t v = __half_as_ushort(__float2half_rn(x));
    w[i / 2] = i & 1 ? (w[i / 2] & 0x0000FFFFu) | v << 16 : (w[i / 2] & 0xFFFF0000u) | v;
  }
  static __device__ __forceinline__ float one(const __half* p) { return __half2float(*p); }
  static __device__ __forceinline__ __half round(float x) { return __float2half_rn(x); }
};

// One sequence's penalties and biases.
struct Asked {
  float repetition, frequency, presence;
  const float* sums;  // of the biases, by their numbers
  // the value of an entry whose table word is t
  __device__ __forceinline__ float of(float z, uint32_t t) const {
    if (t & (kCount | kInPrompt)) z = z > 0.f ? __fdiv_rn(z, repetition) : z * repetition;
    if (t & kCount) z = (z - frequency * (float)(t & kCount)) - presence;
    if (t >> kBiasShift) z += sums[(t >> kBiasShift) - 1];
    return z;
  }
};

// Where a row's slice begins, in entries from a 16-byte boundary, and what lies behind it.
template <typename T>
struct Piece {
  const T* in;
  T* out;
  int head, vectors;  // entries before the first boundary, whole 16-byte pieces after it
  __device__ __forceinline__ Piece(const AdjustArgs& a, int64_t row, int lo, int n) {
    in = reinterpret_cast<const T*>(a.logits) + row * a.stride + lo;
    out = reinterpret_cast<T*>(a.out) + row * a.out_stride + lo;
    const uint32_t at = (uint32_t)reinterpret_cast<uintptr_t>(in) & 15, to = (uint32_t)reinterpret_cast<uintptr_t>(out) & 15;
    head = at != to ? n : min(n, (int)((16 - at) & 15) / (int)sizeof(T));  // apart from each other: entry by entry
    vectors = (n - head) / Entries<T>::kN;
  }
};

}  // namespace

template <typename T, bool MASK>
__global__ void __launch_bounds__(kAdjThreads, 4) adjust_kernel(const __grid_constant__ AdjustArgs a, int slice) {
  constexpr int kN = Entries<T>::kN;
  extern __shared__ __align__(16) uint32_t table[];  // a word an entry, the biases' sums, their doubles' marks
  float* sums = reinterpret_cast<float*>(table + slice);
  uint8_t* twice = reinterpret_cast<uint8_t*>(sums + a.n_bias);
  const int tid = threadIdx.x, b = blockIdx.y, lo = blockIdx.x * slice, n = min(slice, a.vocab - lo);
  const int words = (a.vocab + 31) / 32;
  pdl_trigger();
#pragma unroll 4
  for (int i = tid; i < slice / 4; i += kAdjThreads) reinterpret_cast<uint4*>(table)[i] = make_uint4(0, 0, 0, 0);
  for (int i = tid; i < a.n_bias; i += kAdjThreads) twice[i] = 0;
  pdl_wait();
  // a row's pieces that this thread has, and the mask's words that cover them
  struct Held {
    uint4 x[kAdjVectors];
    uint32_t w0[kAdjVectors], w1[kAdjVectors];
  };
  auto load = [&](int i, Held& h) {
    const int64_t row = (int64_t)b * a.width + i;
    const Piece<T> p(a, row, lo, n);
    const uint32_t* allowed = a.allowed + row * words;
#pragma unroll
    for (int e = 0; e < kAdjVectors; ++e) {
      const int v = tid + e * kAdjThreads;
      if (v >= p.vectors) break;
      h.x[e] = __ldcs(reinterpret_cast<const uint4*>(p.in + p.head) + v);
      if (MASK) {
        const int at = lo + p.head + v * kN;
        h.w0[e] = allowed[at >> 5];
        h.w1[e] = allowed[(at + kN - 1) >> 5];
      }
    }
  };
  Held now;
  load(blockIdx.z, now);
  Asked ask{1.f, 0.f, 0.f, sums};
  if (a.repetition) ask.repetition = a.repetition[b];
  if (a.frequency) ask.frequency = a.frequency[b];
  if (a.presence) ask.presence = a.presence[b];
  const int length = a.history ? min(max(a.hist_len[b], 0), a.max_history) : 0;
  const int prompt = a.prompt_len ? a.prompt_len[b] : 0;
  __syncthreads();
  if (a.n_bias) {
    // the first of a token's biases gets the highest number; it sums them all
    const int32_t* ids = a.bias_ids + (int64_t)b * a.n_bias;
    const float* bias = a.bias + (int64_t)b * a.n_bias;
    for (int j = tid; j < a.n_bias; j += kAdjThreads) {
      const uint32_t at = (uint32_t)ids[j] - (uint32_t)lo;
      if (at < (uint32_t)n) atomicMax(table + at, (uint32_t)(a.n_bias - j) << kBiasShift);
    }
    __syncthreads();
    for (int j = tid; j < a.n_bias; j += kAdjThreads) {
      const uint32_t at = (uint32_t)ids[j] - (uint32_t)lo;
      if (at < (uint32_t)n && table[at] >> kBiasShift != (uint32_t)(a.n_bias - j)) twice[(table[at] >> kBiasShift) - 1] = 1;
    }
    __syncthreads();
    for (int j = tid; j < a.n_bias; j += kAdjThreads) {
      const int number = a.n_bias - j;
      const uint32_t at = (uint32_t)ids[j] - (uint32_t)lo;
      if (at >= (uint32_t)n || table[at] >> kBiasShift != (uint32_t)number) continue;
      float sum = bias[j];
      if (twice[number - 1])
        for (int i = j + 1; i < a.n_bias; ++i)
          if (ids[i] == ids[j]) sum += bias[i];
      sums[number - 1] = sum;
    }
    __syncthreads();
  }
  {
    const int32_t* said = a.history + (int64_t)b * a.max_history;
#pragma unroll 8
    for (int i = tid; i < length; i += kAdjThreads) {
      const uint32_t at = (uint32_t)said[i] - (uint32_t)lo;
      if (at < (uint32_t)n) {
        if (i < prompt) atomicOr(table + at, kInPrompt); else atomicAdd(table + at, 1u);
      }
    }
  }
  // the branch's token that this thread adds, if it lies in the slice
  uint32_t mine = 0xFFFFFFFFu;
  if (a.tokens && tid < a.width) {
    const uint32_t at = (uint32_t)a.tokens[(int64_t)b * a.width + tid] - (uint32_t)lo;
    if (at < (uint32_t)n) mine = at;
  }
  const bool branches = __syncthreads_or(mine != 0xFFFFFFFFu);
  const int mask_words = (a.width + 63) / 64;
  auto on_branch = [&](int i) -> bool {
    return mine != 0xFFFFFFFFu && (a.mask[((int64_t)b * a.width + i) * mask_words + (tid >> 6)] >> (tid & 63) & 1);
  };
#pragma unroll 1
  for (int i = blockIdx.z; i < a.width; i += gridDim.z) {
    const int64_t row = (int64_t)b * a.width + i;
    Held next;
    if (i + (int)gridDim.z < a.width) load(i + gridDim.z, next);
    bool added = false;
    if (branches) {
      added = on_branch(i);
      if (added) atomicAdd(table + mine, 1u);
      __syncthreads();
    }
    const Piece<T> p(a, row, lo, n);
    const bool even = (p.head & 3) == 0;  // the table's words of a piece lie on 16-byte boundaries too
#pragma unroll
    for (int e = 0; e < kAdjVectors; ++e) {
      const int v = tid + e * kAdjThreads;
      if (v >= p.vectors) break;
      const int at = p.head + v * kN;
      uint32_t x[4] = {now.x[e].x, now.x[e].y, now.x[e].z, now.x[e].w}, t[kN], any = 0;
      if (even) {
#pragma unroll
        for (int k = 0; k < kN / 4; ++k) {
          const uint4 q = *reinterpret_cast<const uint4*>(table + at + 4 * k);
          t[4 * k] = q.x; t[4 * k + 1] = q.y; t[4 * k + 2] = q.z; t[4 * k + 3] = q.w;
        }
      } else {
#pragma unroll
        for (int k = 0; k < kN; ++k) t[k] = table[at + k];
      }
#pragma unroll
      for (int k = 0; k < kN; ++k) any |= t[k];
      if (any) {
#pragma unroll
        for (int k = 0; k < kN; ++k)
          if (t[k]) Entries<T>::put(x, k, ask.of(Entries<T>::get(x, k), t[k]));
      }
      if (MASK) {
        const uint32_t bits = __funnelshift_r(now.w0[e], now.w1[e], (lo + at) & 31);
#pragma unroll
        for (int k = 0; k < kN; ++k)
          if (!(bits >> k & 1)) Entries<T>::put(x, k, -INFINITY);
      }
      __stcs(reinterpret_cast<uint4*>(p.out + p.head) + v, make_uint4(x[0], x[1], x[2], x[3]));
    }
    // the entries before the first boundary and behind the last piece
    const int tail0 = p.head + p.vectors * kN, loose = p.head + n - tail0;
    for (int k = tid; k < loose; k += kAdjThreads) {
      const int at = k < p.head ? k : tail0 + k - p.head;
      float z = Entries<T>::one(p.in + at);
      const uint32_t t = table[at];
      if (MASK && !(a.allowed[row * words + ((lo + at) >> 5)] >> ((lo + at) & 31) & 1)) p.out[at] = Entries<T>::round(-INFINITY);
      else if (t) p.out[at] = Entries<T>::round(ask.of(z, t));
      else p.out[at] = p.in[at];
    }
    if (branches) {
      __syncthreads();
      if (added) atomicSub(table + mine, 1u);
    }
    now = next;
  }
}

template <typename T>
static void run_adjust(const AdjustArgs& a, cudaStream_t s) {
  // Slices as long as a thread's pieces allow, shorter where that gives fewer CTAs
  // than four an SM, down to one piece a thread; then rows are shared out too.
  const int piece = kAdjThreads * Entries<T>::kN, want = 4 * 152;
  int slice = kAdjVectors * piece;
  while (slice > piece && (int64_t)a.batch * ((a.vocab + slice - 1) / slice) < want) slice /= 2;
  const int slices = (a.vocab + slice - 1) / slice;
  const int64_t ctas = (int64_t)a.batch * slices;
  const int shares = ctas >= want ? 1 : (int)((want + ctas - 1) / ctas);
  const dim3 grid(slices, a.batch, shares < a.width ? shares : a.width);
  const size_t smem = (size_t)slice * 4 + (size_t)a.n_bias * 5;
  if (a.allowed) launch_in_turn(adjust_kernel<T, true>, grid, kAdjThreads, smem, 0, s, a, slice);
  else launch_in_turn(adjust_kernel<T, false>, grid, kAdjThreads, smem, 0, s, a, slice);
}

void launch_adjust_logits(const AdjustArgs& a, cudaStream_t s) {
  if (a.dtype == DT_F32) run_adjust<float>(a, s);
  else if (a.dtype == DT_BF16) run_adjust<__nv_bfloat16>(a, s);
  else run_adjust<__half>(a, s);
}

}  // namespace pard
