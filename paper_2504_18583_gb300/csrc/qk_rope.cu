// Per-head RMS norm of queries and keys, rotary positions and the write of keys
// and values into the paged cache, in one pass over the QKV projection's rows.
//
//   x' = x * rsqrt(mean(x^2) + eps) * gain          (each head of q and k; optional)
//   (a, b) -> amplitude * (a cos t - b sin t, a sin t + b cos t),  t = position * inv_freq[i]
//
// on the pairs (i, i + rot/2) or (2i, 2i + 1) of a head's first rot entries.
// All arithmetic is in 32 bits, rounded once to the output's type.
//
// What bounds it: HBM (each entry is read and written once).  A lane holds
// eight entries (16 bytes), a head is 8 or 16 lanes, so the norm is three or
// four shuffles and a half-split pair's other entries are rot/16 lanes away:
// they are exchanged as the packed input, four shuffles for eight entries.
// One CTA takes one token (or, where tokens are few, part of its heads); the
// loads go out before the angles are computed.
//
// Angles.  position * inv_freq in 32 bits is off by 2^-24 of itself: 4e-3 at
// position 65536.  Here each frequency becomes a whole number of 2^-64 turns,
// once a thread, and the product with the position, modulo 2^64, is the exact
// phase of that number; its top 32 bits go through sincospif.
#include <cuda_fp16.h>

#include "common.cuh"
#include "tree.h"

namespace pard {

namespace {

constexpr int kRopeThreads = 256;
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

}  // namespace

template <typename T, int HD>
__global__ void __launch_bounds__(kRopeThreads) qk_rope_kernel(const QkRopeArgs a, int heads_per_cta) {
  constexpr int kGroup = HD / 8;                      // lanes of one head
  constexpr int kGroups = kRopeThreads / kGroup;      // heads a CTA takes at once
  __shared__ float2 s_turn[HD / 2];                   // amplitude * (cos, sin) of this token's pairs
  const int tok = blockIdx.x, tid = threadIdx.x;
  const int g = tid / kGroup, l = tid % kGroup, lane = tid & 31;
  const int heads = a.n_q_heads + 2 * a.n_kv_heads;
  const int h0 = blockIdx.y * heads_per_cta, h1 = min(heads, h0 + heads_per_cta);
  const T* row = reinterpret_cast<const T*>(a.qkv) + (int64_t)tok * a.qkv_stride + l * 8;
  uint4 x[kRopeHeads];
#pragma unroll
  for (int e = 0; e < kRopeHeads; ++e) {
    const int h = h0 + e * kGroups + g;
    if (h < h1) x[e] = *reinterpret_cast<const uint4*>(row + (int64_t)h * HD);
  }
  const int half = a.rot_dim / 2;
  if (tid < half) {
    const uint64_t f = turns_per_position(a.inv_freq[tid]);
    const uint64_t phase = f * (uint64_t)(int64_t)a.pos[tok];
    float sn, cs;
    sincospif((float)(int32_t)(phase >> 32) * 4.656612873077393e-10f, &sn, &cs);  // 2^-31: half turns
    s_turn[tid] = make_float2(a.amplitude * cs, a.amplitude * sn);
  }
  const int64_t slot = a.slots[tok];
  const int64_t page = slot >= 0 ? slot / kPageTok : -1;
  const bool write = page >= 0 && page < a.n_pages;
  const int64_t cache_at = page * a.page_stride + (slot % kPageTok) * HD + l * 8;
  __syncthreads();
  // this lane's factors: out = own * cos + other * sin', with the half-split
  // layout's other entries `away` lanes off
  const int e0 = l * 8;
  const bool rotates = e0 < a.rot_dim, upper = !a.interleaved && e0 >= half;
  const int away = a.interleaved || !rotates ? 0 : (upper ? -(half / 8) : half / 8);
  float cs[8], sn[8];
  if (rotates) {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const int i = a.interleaved ? (e0 + e) / 2 : (upper ? e0 + e - half : e0 + e);
      const float2 t = s_turn[i];
      cs[e] = t.x;
      sn[e] = (a.interleaved ? (e & 1) != 0 : upper) ? t.y : -t.y;
    }
  }
  for (int base = h0; base < h1; base += kRopeHeads * kGroups) {
    if (base > h0) {
#pragma unroll
      for (int e = 0; e < kRopeHeads; ++e) {
        const int h = base + e * kGroups + g;
        if (h < h1) x[e] = *reinterpret_cast<const uint4*>(row + (int64_t)h * HD);
      }
    }
#pragma unroll
    for (int e = 0; e < kRopeHeads; ++e) {
      const int h = base + e * kGroups + g;
      // shuffles below: a warp's groups leave the loop together or sit out
      const bool on = h < h1;
      if (!__any_sync(0xffffffffu, on)) continue;
      const bool is_q = h < a.n_q_heads, is_v = h >= a.n_q_heads + a.n_kv_heads;
      const uint4 raw = on ? x[e] : make_uint4(0, 0, 0, 0);
      uint4 out = raw;
      if (__any_sync(0xffffffffu, on && !is_v)) {
        uint4 far;
        const int from = lane + away;
        far.x = __shfl_sync(0xffffffffu, raw.x, from);
        far.y = __shfl_sync(0xffffffffu, raw.y, from);
        far.z = __shfl_sync(0xffffffffu, raw.z, from);
        far.w = __shfl_sync(0xffffffffu, raw.w, from);
        float v[8], o[8];
        unpack<T>(raw, v);
        unpack<T>(far, o);
        const T* gain = reinterpret_cast<const T*>(is_q ? a.q_gain : a.k_gain);
        float ss = 0.f;
#pragma unroll
        for (int i = 0; i < 8; ++i) ss = fmaf(v[i], v[i], ss);
#pragma unroll
        for (int d = kGroup / 2; d > 0; d >>= 1) ss += __shfl_xor_sync(0xffffffffu, ss, d);
        if (gain && !is_v) {
          const float r = rsqrtf(ss * (1.0f / HD) + a.eps);
          float gn[8], gf[8];
          unpack<T>(*reinterpret_cast<const uint4*>(gain + e0), gn);
          unpack<T>(*reinterpret_cast<const uint4*>(gain + e0 + away * 8), gf);
#pragma unroll
          for (int i = 0; i < 8; ++i) { v[i] *= r * gn[i]; o[i] *= r * gf[i]; }
        }
        if (rotates) {
          float t[8];
#pragma unroll
          for (int i = 0; i < 8; ++i) t[i] = fmaf(a.interleaved ? v[i ^ 1] : o[i], sn[i], v[i] * cs[i]);
#pragma unroll
          for (int i = 0; i < 8; ++i) v[i] = t[i];
        }
        if (!is_v)
          out = make_uint4(Pack<T>::from(v[0], v[1]), Pack<T>::from(v[2], v[3]), Pack<T>::from(v[4], v[5]),
                           Pack<T>::from(v[6], v[7]));
      }
      if (!on) continue;
      if (is_q) {
        *reinterpret_cast<uint4*>(reinterpret_cast<T*>(a.q) + (int64_t)tok * a.q_stride + (int64_t)h * HD + e0) = out;
      } else if (write) {
        const int kh = h - a.n_q_heads - (is_v ? a.n_kv_heads : 0);
        T* cache = reinterpret_cast<T*>(is_v ? a.v_cache : a.k_cache);
        *reinterpret_cast<uint4*>(cache + cache_at + (int64_t)kh * kPageTok * HD) = out;
      }
    }
  }
}

template <typename T, int HD>
static void run_rope(const QkRopeArgs& a, cudaStream_t s) {
  constexpr int kGroups = kRopeThreads / (HD / 8);
  const int heads = a.n_q_heads + 2 * a.n_kv_heads;
  const int rounds = (heads + kGroups - 1) / kGroups;
  // few tokens: one round of heads a CTA, so that no thread works in turns
  const int per_cta = a.n_tokens <= 304 ? kGroups : rounds * kGroups;
  qk_rope_kernel<T, HD><<<dim3(a.n_tokens, (heads + per_cta - 1) / per_cta), kRopeThreads, 0, s>>>(a, per_cta);
}

void launch_qk_rope(const QkRopeArgs& a, cudaStream_t s) {
  if (a.dtype == DT_BF16) {
    if (a.head_dim == 128) run_rope<__nv_bfloat16, 128>(a, s); else run_rope<__nv_bfloat16, 64>(a, s);
  } else {
    if (a.head_dim == 128) run_rope<__half, 128>(a, s); else run_rope<__half, 64>(a, s);
  }
  const cudaError_t e = cudaGetLastError();
  if (e != cudaSuccess) throw e;
}

}  // namespace pard
