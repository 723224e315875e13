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
// numbers: no order), biases are numbered in the same words, those of one token
// summed in the list's order by one thread, and the entries that have something
// become a list.  That is done once; a row is then copied, with its mask, and the
// list's entries are worked out from its logits and written over the copy.  (With
// the table looked up for every entry instead, nearly every warp had an entry to
// change in each of its pieces: 64 rows with 8000 tokens took 28.5 us, 464 rows of
// trees, which also added and removed each branch's tokens in the table, 159.)  A
// tree's tokens are in the list too; how often a row's branch has one is counted
// where it is needed.
//
// What bounds it: HBM for many rows (464 of 128256 in fp32, of 16 trees, with
// penalties, biases and masks: 86 us, 5.6 TB/s), and for few the chain history ->
// table -> list -> row (64 of 128256 in bf16 with 8000 tokens each: 17.4 us, 9 of them
// without the tokens; one: 4.2); a row's loads go out before the history's are looked
// at, and the next row's before this one is worked on.  Slices are as long as they may
// be while the CTAs come out as whole waves of four an SM.
#include <cuda_fp16.h>

#include "common.cuh"
#include "per_device.h"
#include "serve.h"

namespace pard {

namespace {

constexpr int kAdjThreads = 256;
constexpr int kAdjCtas = 4;                   // CTAs an SM
constexpr int kAdjLongest = 6912;             // entries of a slice, six bytes of shared memory each
constexpr int kAdjVectors = 4;                // 16-byte pieces of a row's slice that a thread has
constexpr uint32_t kCount = (1u << 19) - 1;   // of a table's word: how often the token was generated,
constexpr uint32_t kOnTree = 1u << 19;        // whether a node of the tree has it,
constexpr uint32_t kInPrompt = 1u << 20;      // whether the prompt has it,
constexpr int kBiasShift = 21;                // and the number of its bias (0: none)
static_assert(kMaxHistory + kTreeMaxNodes < (1 << 19) && kMaxBiases < (1 << 11), "fields of a table's word");

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
__global__ void __launch_bounds__(kAdjThreads, kAdjCtas) adjust_kernel(const __grid_constant__ AdjustArgs a, int slice) {
  constexpr int kN = Entries<T>::kN;
  // a word an entry, the biases' sums, the list, the marks of biases that come again
  extern __shared__ __align__(16) uint32_t table[];
  float* sums = reinterpret_cast<float*>(table + slice);
  uint16_t* list = reinterpret_cast<uint16_t*>(sums + a.n_bias);
  uint8_t* twice = reinterpret_cast<uint8_t*>(list + slice);
  __shared__ int s_listed;
  __shared__ uint32_t s_words[2][kAdjLongest / 32 + 1];  // a row's mask, and the next one's
  __shared__ int32_t s_tokens[kTreeMaxNodes];  // a tree's tokens, as places in the slice (others: -1)
  const int tid = threadIdx.x, b = blockIdx.y, lo = blockIdx.x * slice, n = min(slice, a.vocab - lo);
  const int words = (a.vocab + 31) / 32;
  pdl_trigger();
#pragma unroll 4
  for (int i = tid; i < slice / 4; i += kAdjThreads) reinterpret_cast<uint4*>(table)[i] = make_uint4(0, 0, 0, 0);
  for (int i = tid; i < a.n_bias; i += kAdjThreads) twice[i] = 0;
  if (tid == 0) s_listed = 0;
  pdl_wait();
  // a row's pieces that this thread has, and a word of its mask, which goes to all
  // through shared memory (each thread's own words from L1: 40 us of 128 for 464 rows)
  struct Held {
    uint4 x[kAdjVectors];
    uint32_t word;
  };
  static_assert(kAdjLongest / 32 <= kAdjThreads, "a word a thread");
  auto load = [&](int i, Held& h) {
    const int64_t row = (int64_t)b * a.width + i;
    const Piece<T> p(a, row, lo, n);
    if (MASK && tid < (n + 31) / 32) h.word = __ldg(a.allowed + row * words + lo / 32 + tid);
#pragma unroll
    for (int e = 0; e < kAdjVectors; ++e) {
      const int v = tid + e * kAdjThreads;
      if (v >= p.vectors) break;
      h.x[e] = __ldcs(reinterpret_cast<const uint4*>(p.in + p.head) + v);
    }
  };
  Held now;
  load(blockIdx.z, now);
  // the first to touch an entry puts it on the list
  auto touched = [&](uint32_t old, uint32_t at) {
    if (old == 0) list[atomicAdd(&s_listed, 1)] = (uint16_t)at;
  };
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
      if (at < (uint32_t)n) touched(atomicMax(table + at, (uint32_t)(a.n_bias - j) << kBiasShift), at);
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
    // Sixteen tokens a thread at a time, 16 bytes a load between the history's first and
    // last boundary.  Few of them lie in the slice: first which ones do is noted in a
    // mask, three instructions a token, then those are counted.  (Nearly every 32 tokens
    // have one: counted on the way, each 32 waited for a counter's old value, 28.5 us for
    // the 64 rows above; gathered by ballots and counts of bits, those took most of 18.)
    const int32_t* said = a.history + (int64_t)b * a.max_history;
    const int head = min(length, (int)((16 - (reinterpret_cast<uintptr_t>(said) & 15)) & 15) / 4), pieces = (length - head) / 4;
    auto count = [&](int i) {
      const uint32_t at = (uint32_t)__ldg(said + i) - (uint32_t)lo;
      if (at < (uint32_t)n) touched(i < prompt ? atomicOr(table + at, kInPrompt) : atomicAdd(table + at, 1u), at);
    };
    for (int p0 = tid; p0 < pieces; p0 += 4 * kAdjThreads) {
      int4 q[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int v = p0 + e * kAdjThreads;
        q[e] = v < pieces ? __ldg(reinterpret_cast<const int4*>(said + head) + v) : make_int4(-1, -1, -1, -1);
      }
      uint32_t in = 0;
      auto note = [&](int k, int32_t id) { if ((uint32_t)id - (uint32_t)lo < (uint32_t)n) in |= 1u << k; };
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        note(4 * e, q[e].x);
        note(4 * e + 1, q[e].y);
        note(4 * e + 2, q[e].z);
        note(4 * e + 3, q[e].w);
      }
      for (; in; in &= in - 1) {
        const int k = __ffs(in) - 1;
        count(head + 4 * (p0 + (k >> 2) * kAdjThreads) + (k & 3));
      }
    }
    const int loose = length - 4 * pieces;  // before the first boundary and behind the last
    if (tid < loose) count(tid < head ? tid : 4 * pieces + tid);
  }
  const int nodes = a.tokens ? a.width : 0;
  if (tid < nodes) {
    const uint32_t at = (uint32_t)a.tokens[(int64_t)b * a.width + tid] - (uint32_t)lo;
    s_tokens[tid] = at < (uint32_t)n ? (int)at : -1;
    if (at < (uint32_t)n) touched(atomicOr(table + at, kOnTree), at);
  }
  if (MASK && tid < (n + 31) / 32) s_words[0][tid] = now.word;
  __syncthreads();
  const int listed = s_listed, mask_words = (a.width + 63) / 64;
  // One entry of the list a thread, as a rule: its logit is asked for with the row's
  // pieces, and which of the tree's nodes have it is found once.
  const bool own = listed <= kAdjThreads, has = own && tid < listed;
  const int mine = has ? list[tid] : 0;
  const uint32_t held = has ? table[mine] : 0;
  uint64_t nodes_with[kTreeMaxWords] = {0, 0, 0, 0};
  if (held & kOnTree)
    for (int j = 0; j < nodes; ++j)
#pragma unroll
      for (int w = 0; w < kTreeMaxWords; ++w)
        if (s_tokens[j] == mine && j >> 6 == w) nodes_with[w] |= (uint64_t)1 << (j & 63);
  auto load_own = [&](int i, T& z) {
    if (has) z = reinterpret_cast<const T*>(a.logits)[((int64_t)b * a.width + i) * a.stride + lo + mine];
  };
  T z{};
  load_own(blockIdx.z, z);
#pragma unroll 1
  for (int i = blockIdx.z, buf = 0; i < a.width; i += gridDim.z, buf ^= 1) {
    const int64_t row = (int64_t)b * a.width + i;
    const Piece<T> p(a, row, lo, n);
    const uint32_t* allowed = s_words[buf];
    auto allows = [&](int at) { return !MASK || (allowed[at >> 5] >> (at & 31) & 1); };
    const bool mine_allowed = has && allows(mine);
    uint32_t t = held;
    if (held & kOnTree) {
#pragma unroll
      for (int w = 0; w < kTreeMaxWords; ++w)
        if (w < mask_words) t += __popcll(a.mask[row * mask_words + w] & nodes_with[w]);
    }
    Held next;
    T z_next{};
    if (i + (int)gridDim.z < a.width) {
      load(i + gridDim.z, next);
      load_own(i + gridDim.z, z_next);
    }
#pragma unroll
    for (int e = 0; e < kAdjVectors; ++e) {
      const int v = tid + e * kAdjThreads;
      if (v >= p.vectors) break;
      uint32_t x[4] = {now.x[e].x, now.x[e].y, now.x[e].z, now.x[e].w};
      if (MASK) {
        const int at = p.head + v * kN;
        const uint32_t bits = __funnelshift_r(allowed[at >> 5], allowed[(at + kN - 1) >> 5], at & 31);
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
      const T x = p.in[at];
      p.out[at] = allows(at) ? x : Entries<T>::round(-INFINITY);
    }
    if (MASK && tid < (n + 31) / 32) s_words[buf ^ 1][tid] = next.word;
    __syncthreads();  // the copy is there
    if (own) {
      if (mine_allowed) p.out[mine] = Entries<T>::round(ask.of(Entries<T>::one(&z), t));
    } else {
      // (in place, the copy has left what is allowed as it was)
      for (int k = tid; k < listed; k += kAdjThreads) {
        const int at = list[k];
        if (MASK && !(a.allowed[row * words + ((lo + at) >> 5)] >> (at & 31) & 1)) continue;  // (the row after the next may be in `allowed`)
        uint32_t tk = table[at];
        if (tk & kOnTree)
          for (int j = 0; j < nodes; ++j)
            if (s_tokens[j] == at) tk += (uint32_t)(a.mask[row * mask_words + (j >> 6)] >> (j & 63) & 1);
        p.out[at] = Entries<T>::round(ask.of(Entries<T>::one(p.in + at), tk));
      }
    }
    now = next;
    z = z_next;
  }
}

template <typename T>
static void run_adjust(const AdjustArgs& a, cudaStream_t s) {
  // Slices as long as a thread's pieces and shared memory allow, shortened until the
  // CTAs are whole waves, down to one piece a thread; where that leaves SMs
  // without a CTA, rows are shared out too.
  const int piece = kAdjThreads * Entries<T>::kN, wave = kAdjCtas * 152;
  const int longest = kAdjVectors * piece < kAdjLongest ? kAdjVectors * piece : kAdjLongest;
  const int64_t least = (int64_t)a.batch * ((a.vocab + longest - 1) / longest), waves = (least + wave - 1) / wave;
  const int64_t slices_wanted = waves * wave / a.batch;
  int64_t slice64 = slices_wanted > 0 ? (a.vocab + slices_wanted - 1) / slices_wanted : longest;
  slice64 = (slice64 + 31) / 32 * 32;
  const int slice = (int)(slice64 < piece ? piece : slice64 > longest ? longest : slice64);
  const int slices = (a.vocab + slice - 1) / slice;
  const int64_t ctas = (int64_t)a.batch * slices;
  const int shares = ctas >= wave ? 1 : (int)(wave / ctas);
  const dim3 grid(slices, a.batch, shares < a.width ? shares : a.width);
  const size_t smem = (size_t)slice * 6 + (size_t)a.n_bias * 5;
  auto* kernel = a.allowed ? adjust_kernel<T, true> : adjust_kernel<T, false>;
  static OncePerDevice allowed[2];
  allowed[a.allowed ? 1 : 0].get(current_device(), [&] { return allow_shared(kernel, kAdjLongest * 6 + kMaxBiases * 5); });
  launch_in_turn(kernel, grid, kAdjThreads, smem, 0, s, a, slice);
}

void launch_adjust_logits(const AdjustArgs& a, cudaStream_t s) {
  if (a.dtype == DT_F32) run_adjust<float>(a, s);
  else if (a.dtype == DT_BF16) run_adjust<__nv_bfloat16>(a, s);
  else run_adjust<__half>(a, s);
}

}  // namespace pard
