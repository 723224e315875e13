// Attention of chunks over a cache of 16-bit entries, and the launches' choice.
#include "chunk_attention.cuh"

namespace pard {

int64_t chunk_attention_places(int n_tokens, int batch, int n_q_heads, int n_kv_heads, int max_pages) {
  const int group = n_q_heads / n_kv_heads, rows = kTile * chunk_blocks(n_tokens, batch, group);
  const int64_t blocks = (int64_t)n_tokens * group / rows + batch, tiles = ((int64_t)max_pages * kPageTok + kTile - 1) / kTile;
  return blocks * n_kv_heads * (tiles + kUnitStart);  // as the kernel counts them: its sums are 32-bit ones
}

size_t chunk_attention_workspace(int n_tokens, int batch, int n_q_heads, int n_kv_heads, int head_dim) {
  return kArriveBytes + 2 * kMaxGrid * slot_floats(head_dim, chunk_blocks(n_tokens, batch, n_q_heads / n_kv_heads)) * sizeof(float);
}

void launch_chunk_attention_8bit(const ChunkAttnArgs& a, cudaStream_t s);  // chunk_attention_8bit.cu

void launch_chunk_attention(const ChunkAttnArgs& a, cudaStream_t s) {
  if (a.k_scale) launch_chunk_attention_8bit(a, s); else run_chunk_attention<false>(a, s);
}

}  // namespace pard
