// C ABI of the tree decode step's operators: argument checks and launches.
// None of them takes a context; all work is enqueued on the caller's stream.
#include <cmath>
#include <exception>
#include <string>

#include "pard.h"
#include "tree.h"

namespace pard {
void set_error(const std::string& msg);  // api.cu

namespace {

pard_status refuse(pard_status code, const char* why) {
  set_error(why);
  return code;
}

template <typename F>
pard_status launched(F&& f) {
  try {
    f();
    return PARD_OK;
  } catch (cudaError_t e) {
    set_error(std::string("kernel launch: ") + cudaGetErrorString(e));
  } catch (const std::exception& e) {
    set_error(e.what());
  }
  return PARD_ERR_CUDA;
}

bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }
bool two_byte(int dtype) { return dtype == DT_BF16 || dtype == DT_F16; }

// the paged cache's shape; pages of `page_stride` entries hold [head][16][head_dim]
const char* bad_cache(int n_kv_heads, int head_dim, int64_t page_stride, int n_pages) {
  if (head_dim != 64 && head_dim != 128) return "head_dim must be 64 or 128";
  if (n_kv_heads < 1 || n_kv_heads > 1024) return "key/value heads outside [1, 1024]";
  if (n_pages < 1) return "the cache has no pages";
  if (page_stride < (int64_t)n_kv_heads * kPageTok * head_dim) return "pages overlap: page stride too small";
  if (page_stride % 8) return "page stride must be a multiple of 8 entries";
  return nullptr;
}
const char* bad_tree(int batch, int width, int max_pages) {
  if (batch < 1 || batch > 65535) return "batch outside [1, 65535]";
  if (width < 1 || width > kTreeMaxNodes) return "tree width outside [1, 256]";
  if (max_pages < 1 || max_pages > (1 << 26)) return "page table width outside [1, 2^26]";
  return nullptr;
}

}  // namespace
}  // namespace pard

using namespace pard;

extern "C" {

pard_status pard_tree_plan(const int32_t* d_parents, const int32_t* d_n_nodes, const int32_t* d_ctx_len,
                           const int32_t* d_page_table, int32_t batch, int32_t width, int32_t max_pages,
                           int32_t n_pages, uint64_t* d_mask, int32_t* d_pos, int64_t* d_slots, void* stream) {
  if (!d_parents || !d_n_nodes || !d_ctx_len || !d_page_table || !d_mask || !d_pos || !d_slots)
    return refuse(PARD_ERR_ARG, "tree plan: null pointer");
  if (const char* why = bad_tree(batch, width, max_pages)) return refuse(PARD_ERR_ARG, why);
  if (n_pages < 1) return refuse(PARD_ERR_ARG, "the cache has no pages");
  const TreePlanArgs a{d_parents, d_n_nodes, d_ctx_len, d_page_table, batch, width, (width + 63) / 64,
                       max_pages, n_pages, d_mask, d_pos, d_slots};
  return launched([&] { launch_tree_plan(a, reinterpret_cast<cudaStream_t>(stream)); });
}

pard_status pard_qk_norm_rope(const void* d_qkv, int64_t qkv_stride, int32_t dtype, int32_t n_tokens,
                              int32_t n_q_heads, int32_t n_kv_heads, int32_t head_dim, const void* d_q_gain,
                              const void* d_k_gain, float eps, const int32_t* d_pos, const int64_t* d_slots,
                              const float* d_inv_freq, int32_t rot_dim, int32_t interleaved, float amplitude,
                              void* d_q, int64_t q_stride, void* d_k_cache, void* d_v_cache, int64_t page_stride,
                              int32_t n_pages, void* stream) {
  if (n_tokens == 0) return PARD_OK;
  if (!d_qkv || !d_pos || !d_slots || !d_q || !d_k_cache || !d_v_cache || (rot_dim > 0 && !d_inv_freq))
    return refuse(PARD_ERR_ARG, "qk_norm_rope: null pointer");
  if (n_tokens < 0) return refuse(PARD_ERR_ARG, "qk_norm_rope: negative token count");
  if (!two_byte(dtype)) return refuse(PARD_ERR_SHAPE, "qk_norm_rope: type must be bf16 or fp16");
  if (const char* why = bad_cache(n_kv_heads, head_dim, page_stride, n_pages)) return refuse(PARD_ERR_SHAPE, why);
  if (n_q_heads < 1 || n_q_heads > 4096) return refuse(PARD_ERR_SHAPE, "query heads outside [1, 4096]");
  if (rot_dim < 0 || rot_dim > head_dim || rot_dim % 16)
    return refuse(PARD_ERR_SHAPE, "rotated entries must be a multiple of 16, at most head_dim");
  if (qkv_stride < (int64_t)(n_q_heads + 2 * n_kv_heads) * head_dim || q_stride < (int64_t)n_q_heads * head_dim)
    return refuse(PARD_ERR_ARG, "rows overlap: row stride too small");
  if (qkv_stride % 8 || q_stride % 8 || !aligned16(d_qkv) || !aligned16(d_q) || !aligned16(d_k_cache) ||
      !aligned16(d_v_cache) || !aligned16(d_q_gain) || !aligned16(d_k_gain))
    return refuse(PARD_ERR_ARG, "rows, gains and caches must start on 16-byte boundaries");
  if (!(eps >= 0.f)) return refuse(PARD_ERR_ARG, "eps must not be negative");
  const QkRopeArgs a{d_qkv, qkv_stride, dtype, n_tokens, n_q_heads, n_kv_heads, head_dim, rot_dim, interleaved != 0,
                     n_pages, d_q_gain, d_k_gain, eps, amplitude, d_pos, d_slots, d_inv_freq, d_q, d_k_cache,
                     d_v_cache, q_stride, page_stride};
  return launched([&] { launch_qk_rope(a, reinterpret_cast<cudaStream_t>(stream)); });
}

size_t pard_tree_attention_workspace_bytes(int32_t batch, int32_t width, int32_t n_q_heads, int32_t n_kv_heads,
                                           int32_t head_dim) {
  if (bad_tree(batch, width, 1) || bad_cache(n_kv_heads, head_dim, (int64_t)n_kv_heads * kPageTok * head_dim, 1) ||
      n_q_heads < 1 || n_q_heads > 4096 || n_q_heads % n_kv_heads)
    return 0;
  return tree_attention_workspace(batch, width, n_q_heads, n_kv_heads, head_dim);
}

pard_status pard_tree_attention(const void* d_q, int64_t q_stride, int32_t dtype, int32_t batch, int32_t width,
                                int32_t n_q_heads, int32_t n_kv_heads, int32_t head_dim, const void* d_k_cache,
                                const void* d_v_cache, int64_t page_stride, int32_t n_pages,
                                const int32_t* d_page_table, int32_t max_pages, const int32_t* d_ctx_len,
                                const int32_t* d_n_nodes, const uint64_t* d_mask, float scale, void* d_out,
                                void* d_workspace, size_t workspace_bytes, void* stream) {
  if (!d_q || !d_k_cache || !d_v_cache || !d_page_table || !d_ctx_len || !d_n_nodes || !d_mask || !d_out ||
      !d_workspace)
    return refuse(PARD_ERR_ARG, "tree attention: null pointer");
  if (!two_byte(dtype)) return refuse(PARD_ERR_SHAPE, "tree attention: type must be bf16 or fp16");
  if (const char* why = bad_tree(batch, width, max_pages)) return refuse(PARD_ERR_ARG, why);
  if (const char* why = bad_cache(n_kv_heads, head_dim, page_stride, n_pages)) return refuse(PARD_ERR_SHAPE, why);
  if (n_q_heads < 1 || n_q_heads > 4096 || n_q_heads % n_kv_heads)
    return refuse(PARD_ERR_SHAPE, "query heads must be a multiple of the key/value heads, at most 4096");
  if (q_stride < (int64_t)n_q_heads * head_dim) return refuse(PARD_ERR_ARG, "rows overlap: row stride too small");
  if (q_stride % 8 || !aligned16(d_q) || !aligned16(d_k_cache) || !aligned16(d_v_cache) || !aligned16(d_out) ||
      !aligned16(d_workspace))
    return refuse(PARD_ERR_ARG, "rows, caches, output and workspace must start on 16-byte boundaries");
  if (!std::isfinite(scale)) return refuse(PARD_ERR_ARG, "the scale must be finite");
  if (tree_attention_places(batch, width, n_q_heads, n_kv_heads, max_pages) >= ((int64_t)1 << 31))
    return refuse(PARD_ERR_SHAPE, "more than 2^31 tiles of 128 keys: shorter page tables or a smaller batch");
  if (workspace_bytes < tree_attention_workspace(batch, width, n_q_heads, n_kv_heads, head_dim))
    return refuse(PARD_ERR_ARG, "workspace smaller than pard_tree_attention_workspace_bytes");
  const TreeAttnArgs a{d_q, d_k_cache, d_v_cache, q_stride, page_stride, d_page_table, d_ctx_len, d_n_nodes, d_mask,
                       dtype, batch, width, (width + 63) / 64, n_q_heads, n_kv_heads, head_dim, max_pages, n_pages,
                       scale, d_out, d_workspace};
  return launched([&] { launch_tree_attention(a, reinterpret_cast<cudaStream_t>(stream)); });
}

pard_status pard_sample(const void* d_logits, int64_t row_stride, int32_t dtype, int32_t rows, int32_t vocab,
                        const float* d_u, const float* d_temperature, const int32_t* d_top_k, const float* d_top_p,
                        const float* d_min_p, int32_t* d_token, float* d_logprob, void* stream) {
  if (rows == 0) return PARD_OK;
  if (!d_logits || !d_u || !d_token || !d_logprob) return refuse(PARD_ERR_ARG, "sample: null pointer");
  if (dtype != DT_F32 && !two_byte(dtype)) return refuse(PARD_ERR_SHAPE, "sample: type must be fp32, bf16 or fp16");
  if (rows < 0 || rows > (1 << 24)) return refuse(PARD_ERR_ARG, "sample: rows outside [0, 2^24]");
  if (vocab < 1 || vocab > kSampleMaxVocab) return refuse(PARD_ERR_SHAPE, "sample: vocabulary outside [1, 262144]");
  if (row_stride < vocab) return refuse(PARD_ERR_ARG, "rows overlap: row stride too small");
  if (reinterpret_cast<uintptr_t>(d_logits) % (dtype == DT_F32 ? 4 : 2))
    return refuse(PARD_ERR_ARG, "sample: logits not aligned to their type");
  const SampleArgs a{d_logits, row_stride, dtype, rows, vocab, d_u, d_temperature, d_top_p, d_min_p, d_top_k,
                     d_token, d_logprob};
  return launched([&] { launch_sample(a, reinterpret_cast<cudaStream_t>(stream)); });
}

pard_status pard_tree_commit(const int32_t* d_sampled, const int32_t* d_tokens, const int32_t* d_parents,
                             const int32_t* d_n_nodes, const int32_t* d_ctx_len, const int32_t* d_page_table,
                             int32_t batch, int32_t width, int32_t max_pages, void* d_pool, int64_t layer_stride,
                             int64_t kv_stride, int64_t page_stride, int32_t n_layers, int32_t n_kv_heads,
                             int32_t head_dim, int32_t n_pages, int32_t* d_accept_len, int32_t* d_emitted,
                             int32_t* d_new_len, void* stream) {
  if (!d_sampled || !d_tokens || !d_parents || !d_n_nodes || !d_ctx_len || !d_page_table || !d_pool ||
      !d_accept_len || !d_emitted || !d_new_len)
    return refuse(PARD_ERR_ARG, "tree commit: null pointer");
  if (const char* why = bad_tree(batch, width, max_pages)) return refuse(PARD_ERR_ARG, why);
  if (const char* why = bad_cache(n_kv_heads, head_dim, page_stride, n_pages)) return refuse(PARD_ERR_SHAPE, why);
  if (n_layers < 1 || n_layers > 4096) return refuse(PARD_ERR_SHAPE, "layers outside [1, 4096]");
  if (layer_stride % 8 || kv_stride % 8 || !aligned16(d_pool))
    return refuse(PARD_ERR_ARG, "the pool's layers, keys and values must start on 16-byte boundaries");
  const TreeCommitArgs a{d_sampled, d_tokens, d_parents, d_n_nodes, d_ctx_len, d_page_table, batch, width, max_pages,
                         n_pages, n_layers, n_kv_heads, head_dim, static_cast<uint16_t*>(d_pool), layer_stride,
                         kv_stride, page_stride, d_accept_len, d_emitted, d_new_len};
  return launched([&] { launch_tree_commit(a, reinterpret_cast<cudaStream_t>(stream)); });
}

}  // extern "C"
