// Attention of a tree's nodes over the paged cache (first form: one warp a
// (sequence, node, query head), lanes over keys, running maximum and sum).
#include <cuda_fp16.h>

#include "common.cuh"
#include "tree.h"

namespace pard {

namespace {
__device__ __forceinline__ float f32(__nv_bfloat16 v) { return __bfloat162float(v); }
__device__ __forceinline__ float f32(__half v) { return __half2float(v); }
__device__ __forceinline__ void put(__nv_bfloat16* p, float v) { *p = __float2bfloat16_rn(v); }
__device__ __forceinline__ void put(__half* p, float v) { *p = __float2half_rn(v); }
}  // namespace

template <typename T, int HD>
__global__ void __launch_bounds__(32) tree_attention_kernel(const TreeAttnArgs a) {
  __shared__ float s_q[HD];
  const int h = blockIdx.x, i = blockIdx.y, b = blockIdx.z, lane = threadIdx.x;
  const int kh = h / (a.n_q_heads / a.n_kv_heads);
  const int n = min(max(a.n_nodes[b], 0), a.width), ctx = max(a.ctx_len[b], 0);
  const int keys = min(ctx + n, a.max_pages * kPageTok);
  T* out = reinterpret_cast<T*>(a.out) + (((int64_t)b * a.width + i) * a.n_q_heads + h) * HD;
  const T* q = reinterpret_cast<const T*>(a.q) + ((int64_t)b * a.width + i) * a.q_stride + h * HD;
  for (int d = lane; d < HD; d += 32) s_q[d] = f32(q[d]);
  __syncwarp();
  float top = -INFINITY, sum = 0.f, o[HD / 32] = {};
  for (int j0 = 0; i < n && j0 < keys; j0 += 32) {
    const int j = j0 + lane, node = j - ctx;
    const int page = page_of(a.page_table + (size_t)b * a.max_pages, j, a.max_pages, a.n_pages);
    bool on = j < keys && page >= 0;
    if (on && node >= 0) on = a.mask[((size_t)b * a.width + i) * a.words + node / 64] >> (node % 64) & 1;
    const int64_t at = page * a.page_stride + ((int64_t)kh * kPageTok + j % kPageTok) * HD;
    float s = -INFINITY;
    if (on) {
      s = 0.f;
      const T* kp = reinterpret_cast<const T*>(a.k_cache) + at;
      for (int d = 0; d < HD; ++d) s = fmaf(s_q[d], f32(kp[d]), s);
      s *= a.scale;
    }
    const float m = fmaxf(top, warp_max(s));
    if (m == -INFINITY) continue;
    const float p = on ? expf(s - m) : 0.f, c = expf(top - m);
    sum = sum * c + warp_sum(p);
    for (int e = 0; e < HD / 32; ++e) o[e] *= c;
    for (int t = 0; t < 32; ++t) {
      const float w = __shfl_sync(0xffffffffu, p, t);
      const int64_t va = __shfl_sync(0xffffffffu, at, t);
      if (!__shfl_sync(0xffffffffu, (int)on, t)) continue;
      const T* vp = reinterpret_cast<const T*>(a.v_cache) + va;
      for (int e = 0; e < HD / 32; ++e) o[e] = fmaf(w, f32(vp[e * 32 + lane]), o[e]);
    }
    top = m;
  }
  for (int e = 0; e < HD / 32; ++e) put(out + e * 32 + lane, sum > 0.f ? o[e] / sum : 0.f);
}

size_t tree_attention_workspace(int, int, int, int, int) { return 16; }

void launch_tree_attention(const TreeAttnArgs& a, cudaStream_t s) {
  const dim3 grid(a.n_q_heads, a.width, a.batch);
  if (a.dtype == DT_BF16) {
    if (a.head_dim == 128) tree_attention_kernel<__nv_bfloat16, 128><<<grid, 32, 0, s>>>(a);
    else tree_attention_kernel<__nv_bfloat16, 64><<<grid, 32, 0, s>>>(a);
  } else {
    if (a.head_dim == 128) tree_attention_kernel<__half, 128><<<grid, 32, 0, s>>>(a);
    else tree_attention_kernel<__half, 64><<<grid, 32, 0, s>>>(a);
  }
  const cudaError_t e = cudaGetLastError();
  if (e != cudaSuccess) throw e;
}

}  // namespace pard
