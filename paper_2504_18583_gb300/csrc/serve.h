// Arguments and launchers of the operators of a serving loop around the decode
// step (chunk_attention.cu, adjust_logits.cu), called by serve_api.cu after it
// has checked them.  The 8-bit cache's write is qk_rope.cu's.
#pragma once

#include "tree.h"

namespace pard {

constexpr int kMaxHistory = 524000;   // tokens of a sequence that penalties count: 19 bits hold them and a branch's
constexpr int kMaxBiases = 2047;      // biases of a sequence: 11 bits number them

struct AdjustArgs {
  const void* logits;
  int64_t stride, out_stride;
  int dtype, batch, width, vocab, max_history, n_bias;
  const int32_t *history, *hist_len, *prompt_len;
  const float *repetition, *frequency, *presence;
  const int32_t* bias_ids;
  const float* bias;
  const uint32_t* allowed;
  const int32_t* tokens;
  const uint64_t* mask;
  void* out;
};
void launch_adjust_logits(const AdjustArgs& a, cudaStream_t s);

struct ChunkAttnArgs {
  const void *q, *k_cache, *v_cache;
  const uint8_t *k_scale, *v_scale;  // an 8-bit cache's exponents (null: the caches are of `dtype`)
  int64_t q_stride, page_stride, scale_stride;
  const int32_t *page_table, *starts, *ctx_len;
  int dtype, n_tokens, batch, n_q_heads, n_kv_heads, head_dim, max_pages, n_pages, window, sinks;
  float scale;
  void* out;
  void* workspace;
  // the launcher's
  int group = 1;             // query heads a key/value head
  uint32_t group_magic = 0;  // 2^32 / (query heads a key/value head), rounded up; 0 for one
  bool q_by_tma = false;
};
size_t chunk_attention_workspace(int n_tokens, int batch, int n_q_heads, int n_kv_heads, int head_dim);
// places of the work ranges that a pass may have: below 2^31
int64_t chunk_attention_places(int n_tokens, int batch, int n_q_heads, int n_kv_heads, int max_pages);
void launch_chunk_attention(const ChunkAttnArgs& a, cudaStream_t s);

}  // namespace pard
