// Attention of chunks over a cache of 8-bit entries.
#include "chunk_attention.cuh"

namespace pard {

void launch_chunk_attention_8bit(const ChunkAttnArgs& a, cudaStream_t s) { run_chunk_attention<true>(a, s); }

}  // namespace pard
