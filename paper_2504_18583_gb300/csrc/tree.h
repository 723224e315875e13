// Arguments and launchers of the tree decode step's operators (tree.cu,
// qk_rope.cu, tree_attention.cu, sample.cu), called by tree_api.cu after it
// has checked them.
#pragma once

#include <cuda_runtime.h>
#include <stddef.h>
#include <stdint.h>

namespace pard {

constexpr int kPageTok = 16;          // tokens a page of every paged cache holds
constexpr int kTreeMaxNodes = 256;    // nodes of one sequence's tree
constexpr int kTreeMaxWords = kTreeMaxNodes / 64;
constexpr int kSampleMaxVocab = 262144;
enum : int { DT_BF16 = 0, DT_F16 = 1, DT_F32 = 2 };

// Where position `pos` of a sequence lies: page id (or -1: no such page, or an
// id outside the pool) of its page-table row.
__device__ __forceinline__ int page_of(const int32_t* row, int pos, int max_pages, int n_pages) {
  const int i = pos / kPageTok;
  if (pos < 0 || i >= max_pages) return -1;
  const int p = row[i];
  return (uint32_t)p < (uint32_t)n_pages ? p : -1;
}

// A launch that may begin while the grid before it on the stream ends: each of
// these kernels sets itself up, waits for that grid (pdl_wait) before it touches
// memory, and lets the next one begin the same way.  (Back to back, one node's
// attention 14.7 -> 12.6 us, one sampled row 12.4 -> 10.4, 8191 rotated tokens
// 41.6 -> 39.1.)
template <typename Args, typename... More>
inline void launch_in_turn(void (*kernel)(Args, More...), dim3 grid, int threads, size_t smem, int cluster, cudaStream_t s,
                           const Args& a, const More&... more) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = grid;
  cfg.blockDim = dim3((unsigned)threads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = s;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = (unsigned)cluster;
  attr[1].val.clusterDim.y = 1;
  attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = cluster ? 2 : 1;
  const cudaError_t e = cudaLaunchKernelEx(&cfg, kernel, a, more...);
  if (e != cudaSuccess) throw e;
}

struct TreePlanArgs {
  const int32_t *parents, *n_nodes, *ctx_len, *page_table;
  int batch, width, words, max_pages, n_pages;
  uint64_t* mask;
  int32_t* pos;
  int64_t* slots;
};
void launch_tree_plan(const TreePlanArgs& a, cudaStream_t s);

struct TreeCommitArgs {
  const int32_t *sampled, *tokens, *parents, *n_nodes, *ctx_len, *page_table;
  int batch, width, max_pages, n_pages, n_layers, n_kv_heads, head_dim;
  uint16_t* pool;
  int64_t layer_stride, kv_stride, page_stride;  // in elements
  int32_t *accept_len, *emitted, *new_len;
};
void launch_tree_commit(const TreeCommitArgs& a, cudaStream_t s);

struct QkRopeArgs {
  const void* qkv;
  int64_t qkv_stride;
  int dtype, n_tokens, n_q_heads, n_kv_heads, head_dim, rot_dim, interleaved, n_pages;
  const void *q_gain, *k_gain;
  float eps, amplitude;
  const int32_t* pos;
  const int64_t* slots;
  const float* inv_freq;
  void *q, *k_cache, *v_cache;
  int64_t q_stride, page_stride;
};
void launch_qk_rope(const QkRopeArgs& a, cudaStream_t s);

struct TreeAttnArgs {
  const void *q, *k_cache, *v_cache;
  int64_t q_stride, page_stride;
  const int32_t *page_table, *ctx_len, *n_nodes;
  const uint64_t* mask;
  int dtype, batch, width, words, n_q_heads, n_kv_heads, head_dim, max_pages, n_pages;
  float scale;
  void* out;
  void* workspace;
};
size_t tree_attention_workspace(int batch, int width, int n_q_heads, int n_kv_heads, int head_dim);
// places of the work ranges that a pass may have: below 2^31
int64_t tree_attention_places(int batch, int width, int n_q_heads, int n_kv_heads, int max_pages);
void launch_tree_attention(const TreeAttnArgs& a, cudaStream_t s);

struct SampleArgs {
  const void* logits;
  int64_t stride;
  int dtype, rows, vocab;
  const float *u, *temperature, *top_p, *min_p;
  const int32_t* top_k;
  int32_t* token;
  float* logprob;
};
void launch_sample(const SampleArgs& a, cudaStream_t s);

}  // namespace pard
