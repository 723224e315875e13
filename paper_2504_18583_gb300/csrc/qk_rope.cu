// Per-head RMS norm of queries and keys, rotary positions and the write of keys
// and values into the paged cache, in one pass over the QKV projection's rows.
//
//   x' = x * rsqrt(mean(x^2) + eps) * gain          (each head of q and k; optional)
//   (a, b) -> amplitude * (a cos t - b sin t, a sin t + b cos t),  t = position * inv_freq[i]
//
// on the pairs (i, i + rot/2) or (2i, 2i + 1) of a head's first rot entries.
// All arithmetic is in 32 bits, rounded once to the output's type.
//
// What bounds it: HBM (each entry is read and written once) and, next to it, the
// instructions, about 150 for a warp's 256 entries.  A lane holds eight entries
// (16 bytes), a head is 8 or 16 lanes, so the norm is three or four shuffles and
// a half-split pair's other entries are rot/16 lanes away: they are exchanged as
// the packed input, four shuffles for eight entries.  Gains and rotation are
// multiplied together once a token, by all threads, into two factors an entry.
// The loads of the next token's heads are out while a CTA works on one's.
// Measured, 8191 tokens of 48 heads of 128: 39 us, 5.1 TB/s (67 us with a CTA a
// token and the gains applied to every head; 48 with 64-bit divisions for the
// place of an item).
//
// Angles.  position * inv_freq in 32 bits is off by 2^-24 of itself: 4e-3 at
// position 65536.  Here each frequency becomes a whole number of 2^-64 turns,
// once a thread, and the product with the position, modulo 2^64, is the exact
// phase of that number; its top 32 bits go through sincospif.  For the keys of an 8-bit
// cache, where a last bit may decide over a whole step, what lies beyond the nearest
// quarter turn does, which is up to eight times as exact: keys are then about 1.6
// units of 2^-24 off in the mean instead of 2.2, as with torch's 32-bit operations and
// 64-bit angles (on four inputs 8, 10, 17 and 9 of 8.4 million codes are not the nearest
// to the value in 64 bits, with torch's 10, 4, 13 and 16), for 0.2 us of 45.
//
// An 8-bit cache holds e4m3 codes and, for each token's head, the biased exponent
// of a power of two: the smallest under which no finite entry passes 448, e4m3's
// largest.  Codes are rounded from the 32-bit values, so an entry is rounded once;
// a power of two moves no bit, so a reader's 16-bit copy of an entry is exact.
// Infinities and NaN become NaN and do not count for the exponent.  It costs the
// row's largest entry (three or four shuffles) and four conversions a lane, and
// saves half of the caches' bytes; instructions bound it (8191 tokens as above: 44.4
// us, 4.2 TB/s, 72% of the issue slots; what is not finite is looked for once a row,
// not once an entry: 46.4 -> 45.3).  16 tokens: 4.6 us, latency.
#include <cuda_fp16.h>

#include "common.cuh"
#include "tree.h"

namespace pard {

namespace {

constexpr int kRopeThreads = 256;
static_assert(kPageTok == 16, "slots are taken apart by shifts");
constexpr int kRopeHeads = 3;  // heads a lane group has in flight

template <typename T> struct Pack;
template <> struct Pack<__nv_bfloat16> {
  static __device__ __forceinline__ float2 to(uint32_t v) {
    return __bfloat1622float2(*reinterpret_cast<__nv_bfloat162*>(&v));
  }
  static __device__ __forceinline__ uint32_t from(float x, float y) {
    __nv_bfloat162 p = __floats2bfloat162_rn(x, y);
    return *reinterpret_cast<uint32_t*>(&p);
  }
};
template <> struct Pack<__half> {
  static __device__ __forceinline__ float2 to(uint32_t v) { return __half22float2(*reinterpret_cast<__half2*>(&v)); }
  static __device__ __forceinline__ uint32_t from(float x, float y) {
    __half2 p = __floats2half2_rn(x, y);
    return *reinterpret_cast<uint32_t*>(&p);
  }
};

template <typename T>
__device__ __forceinline__ void unpack(const uint4& p, float (&v)[8]) {
  const uint32_t w[4] = {p.x, p.y, p.z, p.w};
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const float2 f = Pack<T>::to(w[e]);
    v[2 * e] = f.x;
    v[2 * e + 1] = f.y;
  }
}

// f / (2 pi) turns as a whole number of 2^-64 turns, modulo one turn.  f is
// m * 2^e with a 24-bit m; the constant is floor(2^66 / (2 pi)).
__device__ __forceinline__ uint64_t turns_per_position(float f) {
  int e;
  const float m = frexpf(fabsf(f), &e);  // [0.5, 1)
  const uint64_t p = __umul64hi((uint64_t)(uint32_t)(m * 16777216.0f) << 40, 0xa2f9836e4e441529ull);  // m * 2^64 * 2^66 / (2 pi) >> 64
  e -= 2;
  const uint64_t t = e >= 64 || e <= -64 ? 0 : (e >= 0 ? p << e : p >> -e);
  return f < 0.f ? 0 - t : t;
}

// The biased exponent of the smallest power of two p with most <= 448 p, in [1, 254].
__device__ __forceinline__ uint32_t scale_exponent(float most) {
  const uint32_t u = __float_as_uint(most);  // 448 is 1.75 * 2^8
  const int e = (int)(u >> 23) - 8 + ((u & 0x7FFFFF) > 0x600000 ? 1 : 0);
  return (uint32_t)max(e, 1);
}
// Two values as e4m3 codes, x in the low byte; what is not finite becomes NaN.
__device__ __forceinline__ uint32_t e4m3_pair(float x, float y) {
  uint16_t v;
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %2, %1;" : "=h"(v) : "f"(x), "f"(y));
  return v;
}

__device__ __forceinline__ float to_float(__nv_bfloat16 v) { return __bfloat162float(v); }
__device__ __forceinline__ float to_float(__half v) { return __half2float(v); }

}  // namespace

// A CTA has U heads of every lane group, those of its blockIdx.y, and walks over
// tokens: the next one's loads are out while it works on one.
template <typename T, int HD, int U, bool Q8>
__global__ void __launch_bounds__(kRopeThreads, U == 1 ? 5 : 4) qk_rope_kernel(const __grid_constant__ QkRopeArgs a) {
  constexpr int kGroup = HD / 8;                      // lanes of one head
  constexpr int kGroups = kRopeThreads / kGroup;      // heads a CTA takes at once
  // Each entry's factors of a token, queries' and keys': gain and rotation in
  // one, out = norm * (own * x + other * y), pair i of all lanes side by side (in
  // entry order a lane's were 64 bytes from the next lane's: four-way bank
  // conflicts, 61 us against 48 for 8191 tokens).  Two tokens in turn.
  __shared__ float4 s_turn[2][2][HD / 2];
  const int tid = threadIdx.x, g = tid / kGroup, l = tid % kGroup, lane = tid & 31;
  const int heads = a.n_q_heads + 2 * a.n_kv_heads, half = a.rot_dim / 2, e0 = l * 8;
  const int h0 = blockIdx.y * U * kGroups + g;
  // this lane's entries: out = own * cos + other * sin', with the half-split
  // layout's other entries `away` lanes off
  const bool rotates = e0 < a.rot_dim, upper = !a.interleaved && e0 >= half;
  const int away = a.interleaved || !rotates ? 0 : (upper ? -(half / 8) : half / 8);
  const int far_lane = lane + away;
  // the entry whose factors this thread computes
  const int te = tid % HD, tk = tid / HD;  // tk 0: queries, 1: keys, else none
  const bool t_turns = te < a.rot_dim, t_odd = a.interleaved ? te & 1 : te >= half;
  pdl_trigger();
  pdl_wait();
  uint64_t per_pos = 0;
  float t_own = 1.f, t_far = 1.f;
  if (tk < 2) {
    const T* gain = reinterpret_cast<const T*>(tk ? a.k_gain : a.q_gain);
    if (t_turns) per_pos = turns_per_position(a.inv_freq[a.interleaved ? te / 2 : (t_odd ? te - half : te)]);
    if (gain) {
      t_own = to_float(gain[te]);
      if (t_turns) t_far = to_float(gain[a.interleaved ? te ^ 1 : (t_odd ? te - half : te + half)]);
    }
  }
  const bool q_norm = a.q_gain != nullptr, k_norm = a.k_gain != nullptr;
  const T* qkv = reinterpret_cast<const T*>(a.qkv) + (int64_t)h0 * HD + e0;
  T* q = reinterpret_cast<T*>(a.q) + (int64_t)h0 * HD + e0;
  auto load = [&](int tok, uint4 (&x)[U]) {
    const T* row = qkv + (int64_t)tok * a.qkv_stride;
#pragma unroll
    for (int e = 0; e < U; ++e) {
      x[e] = make_uint4(0, 0, 0, 0);
      if (h0 + e * kGroups < heads) x[e] = __ldcs(reinterpret_cast<const uint4*>(row + e * kGroups * HD));
    }
  };
  int tok = blockIdx.x;
  uint4 x[U];
  load(tok, x);
  int pos = a.pos[tok];
  int64_t slot = a.slots[tok];
  for (int buf = 0; tok < a.n_tokens; buf ^= 1) {
    if (tk < 2) {
      const uint64_t phase = per_pos * (uint64_t)(int64_t)pos;
      float sn, cs;
      if (Q8 && tk == 1) {
        const uint32_t quarters = (uint32_t)((phase + (1ull << 61)) >> 62);
        const int64_t rest = (int64_t)(phase - ((uint64_t)quarters << 62));  // of the nearest quarter turn, up to an eighth
        float a, b;
        sincospif((float)(int32_t)(rest >> 30) * 1.1641532182693481e-10f, &a, &b);  // 2^-33: half turns
        sn = quarters & 1 ? b : a;
        cs = quarters & 1 ? a : b;
        if (quarters & 2) sn = -sn;
        if ((quarters + 1) & 2) cs = -cs;
      } else {
        sincospif((float)(int32_t)(phase >> 32) * 4.656612873077393e-10f, &sn, &cs);  // 2^-31: half turns
      }
      reinterpret_cast<float2*>(s_turn[buf][tk])[((te % 8 / 2) * kGroup + te / 8) * 2 + (te & 1)] =
          t_turns ? make_float2(t_own * (a.amplitude * cs), (t_odd ? t_far : -t_far) * (a.amplitude * sn)) : make_float2(t_own, 0.f);
    }
    const int64_t slot_now = slot;
    const bool write = slot >= 0 && slot < (int64_t)a.n_pages * kPageTok;
    const int64_t cache_at = (int64_t)(uint32_t)(slot >> 4) * a.page_stride + (int)(slot & (kPageTok - 1)) * HD + e0;
    __syncthreads();  // (the other buffer's readers are past it: they arrived here)
    uint4 ahead[U];
    const int after = tok + gridDim.x;
    if (after < a.n_tokens) {
      load(after, ahead);
      pos = a.pos[after];
      slot = a.slots[after];
    }
    T* q_row = q + (int64_t)tok * a.q_stride;
#pragma unroll
    for (int e = 0; e < U; ++e) {
      const int h = h0 + e * kGroups;
      const bool on = h < heads;
      const bool is_q = h < a.n_q_heads, is_v = h >= a.n_q_heads + a.n_kv_heads;
      const uint4 raw = x[e];
      uint4 out = raw;
      float v[8];
      if (Q8) unpack<T>(raw, v);
      if (__any_sync(0xffffffffu, on && !is_v)) {
        float t[8];
        if (!Q8) unpack<T>(raw, v);
        float r = 1.f;
        if (__any_sync(0xffffffffu, is_q ? q_norm : k_norm)) {
          float ss = 0.f;
#pragma unroll
          for (int i = 0; i < 8; ++i) ss = fmaf(v[i], v[i], ss);
#pragma unroll
          for (int d = kGroup / 2; d > 0; d >>= 1) ss += __shfl_xor_sync(0xffffffffu, ss, d);
          if (is_q ? q_norm : k_norm) r = rsqrtf(ss * (1.0f / HD) + a.eps);
        }
        const float4* turn = &s_turn[buf][is_q ? 0 : 1][l];
        if (a.interleaved) {
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const float4 c = turn[i * kGroup];
            t[2 * i] = v[2 * i] * c.x;
            t[2 * i + 1] = v[2 * i + 1] * c.z;
            if (rotates) {
              t[2 * i] = fmaf(v[2 * i + 1], c.y, t[2 * i]);
              t[2 * i + 1] = fmaf(v[2 * i], c.w, t[2 * i + 1]);
            }
          }
        } else {
          uint4 far;
          far.x = __shfl_sync(0xffffffffu, raw.x, far_lane);
          far.y = __shfl_sync(0xffffffffu, raw.y, far_lane);
          far.z = __shfl_sync(0xffffffffu, raw.z, far_lane);
          far.w = __shfl_sync(0xffffffffu, raw.w, far_lane);
          float o[8];
          unpack<T>(far, o);
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const float4 c = turn[i * kGroup];
            t[2 * i] = v[2 * i] * c.x;
            t[2 * i + 1] = v[2 * i + 1] * c.z;
            if (rotates) {
              t[2 * i] = fmaf(o[2 * i], c.y, t[2 * i]);
              t[2 * i + 1] = fmaf(o[2 * i + 1], c.w, t[2 * i + 1]);
            }
          }
        }
#pragma unroll
        for (int i = 0; i < 8; ++i)
          if (!Q8 || !is_v) v[i] = t[i] * r;
        if (!is_v)
          out = make_uint4(Pack<T>::from(v[0], v[1]), Pack<T>::from(v[2], v[3]), Pack<T>::from(v[4], v[5]),
                           Pack<T>::from(v[6], v[7]));
      }
      const uint4 q_out = out;
      if (Q8 && __any_sync(0xffffffffu, on && !is_q)) {
        float most = 0.f;  // (a NaN is no maximum, and its code is NaN)
#pragma unroll
        for (int i = 0; i < 8; ++i) most = fmaxf(most, fabsf(v[i]));
        if (__any_sync(0xffffffffu, most == INFINITY)) {
          most = 0.f;
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            const float m = fabsf(v[i]);
            if (m < INFINITY) most = fmaxf(most, m); else v[i] = __int_as_float(0x7FFFFFFF);
          }
        }
#pragma unroll
        for (int d = kGroup / 2; d > 0; d >>= 1) most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, d));
        const uint32_t code = scale_exponent(most);
        const float inv = __uint_as_float((254u - code) << 23);
        out.x = e4m3_pair(v[0] * inv, v[1] * inv) | e4m3_pair(v[2] * inv, v[3] * inv) << 16;
        out.y = e4m3_pair(v[4] * inv, v[5] * inv) | e4m3_pair(v[6] * inv, v[7] * inv) << 16;
        out.z = code;
      }
      if (on && is_q) {
        *reinterpret_cast<uint4*>(q_row + e * kGroups * HD) = q_out;
      } else if (Q8 && on && write) {
        const int kh = h - a.n_q_heads - (is_v ? a.n_kv_heads : 0);
        uint8_t* cache = reinterpret_cast<uint8_t*>(is_v ? a.v_cache : a.k_cache);
        *reinterpret_cast<uint2*>(cache + cache_at + kh * (kPageTok * HD)) = make_uint2(out.x, out.y);
        if (l == 0) (is_v ? a.v_scale : a.k_scale)[(slot_now >> 4) * a.scale_stride + kh * kPageTok + (slot_now & (kPageTok - 1))] = (uint8_t)out.z;
      } else if (on && write) {
        const int kh = h - a.n_q_heads - (is_v ? a.n_kv_heads : 0);
        T* cache = reinterpret_cast<T*>(is_v ? a.v_cache : a.k_cache);
        *reinterpret_cast<uint4*>(cache + cache_at + kh * (kPageTok * HD)) = out;
      }
    }
#pragma unroll
    for (int e = 0; e < U; ++e) x[e] = ahead[e];
    tok = after;
  }
}

template <typename T, int HD, int U, bool Q8>
static void launch_items(const QkRopeArgs& a, int most, cudaStream_t s) {
  constexpr int kTake = U * kRopeThreads / (HD / 8);
  const int chunks = (a.n_q_heads + 2 * a.n_kv_heads + kTake - 1) / kTake;
  const int across = most / chunks < 1 ? 1 : most / chunks;
  launch_in_turn(qk_rope_kernel<T, HD, U, Q8>, dim3(a.n_tokens < across ? a.n_tokens : across, chunks), kRopeThreads, 0, 0, s, a);
}

template <typename T, int HD, bool Q8>
static void run_rope(const QkRopeArgs& a, cudaStream_t s) {
  // few tokens: a head a lane group, so that no thread works in turns; many: as
  // many as a lane can have in flight
  if (a.n_tokens <= 304) launch_items<T, HD, 1, Q8>(a, 152 * 5, s); else launch_items<T, HD, kRopeHeads, Q8>(a, 152 * 4, s);
}

template <typename T, int HD>
static void run_cache(const QkRopeArgs& a, cudaStream_t s) {
  if (a.k_scale) run_rope<T, HD, true>(a, s); else run_rope<T, HD, false>(a, s);
}

void launch_qk_rope(const QkRopeArgs& a, cudaStream_t s) {
  if (a.dtype == DT_BF16) {
    if (a.head_dim == 128) run_cache<__nv_bfloat16, 128>(a, s); else run_cache<__nv_bfloat16, 64>(a, s);
  } else {
    if (a.head_dim == 128) run_cache<__half, 128>(a, s); else run_cache<__half, 64>(a, s);
  }
}

}  // namespace pard
