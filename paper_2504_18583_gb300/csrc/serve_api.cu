// C ABI of the operators of a serving loop around the decode step: argument
// checks and launches.  None of them takes a context; all work is enqueued on the
// caller's stream.
#include "pard_serve.h"

#include "api_checks.h"
#include "serve.h"

namespace pard {
namespace {

// the exponents of an 8-bit cache; pages of `scale_stride` bytes hold [head][16]
const char* bad_scales(const void* k_scale, const void* v_scale, int64_t scale_stride, int64_t page_stride, int n_kv_heads) {
  if (!k_scale || !v_scale) return "an 8-bit cache needs both its exponents";
  if (scale_stride < (int64_t)n_kv_heads * kPageTok) return "pages overlap: exponents' stride too small";
  if (scale_stride % 16 || !aligned16(k_scale) || !aligned16(v_scale)) return "a page's exponents must start on 16-byte boundaries";
  if (page_stride % 16) return "page stride must be a multiple of 16 entries";
  return nullptr;
}
const char* bad_chunks(int n_tokens, int batch, int n_q_heads, int n_kv_heads) {
  if (n_tokens < 0) return "negative token count";
  if (batch < 1 || batch > 65535) return "batch outside [1, 65535]";
  if (n_kv_heads < 1 || n_q_heads < 1 || n_q_heads > 4096 || n_q_heads % n_kv_heads)
    return "query heads must be a multiple of the key/value heads, at most 4096";
  if ((int64_t)n_tokens * (n_q_heads / n_kv_heads) >= (int64_t)1 << 30) return "more than 2^30 query vectors a key/value head";
  return nullptr;
}

// a contiguous output of n_tokens rows lies over one of the queries' rows
bool overlap(const void* out, const void* q, int64_t q_stride, int64_t row, int64_t n_tokens) {
  const int64_t o = (int64_t)reinterpret_cast<uintptr_t>(out), at = (int64_t)reinterpret_cast<uintptr_t>(q), step = 2 * q_stride;
  const int64_t before = o - at - 2 * row, first = before < 0 ? 0 : before / step + 1;  // the first row that ends behind `out`
  return first < n_tokens && at + first * step < o + 2 * row * n_tokens;
}

// rows of `row` bytes, each side's a step of its own (at least a row) apart, share a byte
bool overlap_apart(const void* x, int64_t x_step, const void* y, int64_t y_step, int64_t row, int64_t rows) {
  const int64_t a = (int64_t)reinterpret_cast<uintptr_t>(x), b = (int64_t)reinterpret_cast<uintptr_t>(y);
  if (x_step == y_step) {  // y's row i ends or begins in the nearest of x's rows, or the next
    const int64_t d = b < a ? a - b : b - a, k = d / x_step, r = d - k * x_step;
    return (r < row && k < rows) || (x_step - r < row && k + 1 < rows);
  }
  for (int64_t i = 0, j = 0; i < rows && j < rows;) {
    const int64_t p = a + i * x_step, q = b + j * y_step;
    if (p + row <= q) i += (q - row - p) / x_step + 1;  // the first row that ends behind q
    else if (q + row <= p) j += (p - row - q) / y_step + 1;
    else return true;
  }
  return false;
}

}  // namespace
}  // namespace pard

using namespace pard;

extern "C" {

pard_status pard_qk_norm_rope_quantized(const void* d_qkv, int64_t qkv_stride, int32_t dtype, int32_t n_tokens,
                                        int32_t n_q_heads, int32_t n_kv_heads, int32_t head_dim, const void* d_q_gain,
                                        const void* d_k_gain, float eps, const int32_t* d_pos, const int64_t* d_slots,
                                        const float* d_inv_freq, int32_t rot_dim, int32_t interleaved, float amplitude,
                                        void* d_q, int64_t q_stride, void* d_k_cache, void* d_v_cache, int64_t page_stride,
                                        uint8_t* d_k_scale, uint8_t* d_v_scale, int64_t scale_stride, int32_t n_pages,
                                        void* stream) {
  if (n_tokens == 0) return PARD_OK;
  if (!d_qkv || !d_pos || !d_slots || !d_q || !d_k_cache || !d_v_cache || (rot_dim > 0 && !d_inv_freq))
    return refuse(PARD_ERR_ARG, "qk_norm_rope_quantized: null pointer");
  if (n_tokens < 0) return refuse(PARD_ERR_ARG, "qk_norm_rope_quantized: negative token count");
  if (!two_byte(dtype)) return refuse(PARD_ERR_SHAPE, "qk_norm_rope_quantized: type must be bf16 or fp16");
  if (const char* why = bad_cache(n_kv_heads, head_dim, page_stride, n_pages)) return refuse(PARD_ERR_SHAPE, why);
  if (const char* why = bad_scales(d_k_scale, d_v_scale, scale_stride, page_stride, n_kv_heads)) return refuse(PARD_ERR_ARG, why);
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
                     d_v_cache, q_stride, page_stride, d_k_scale, d_v_scale, scale_stride};
  return launched([&] { launch_qk_rope(a, reinterpret_cast<cudaStream_t>(stream)); });
}

size_t pard_chunk_attention_workspace_bytes(int32_t n_tokens, int32_t batch, int32_t n_q_heads, int32_t n_kv_heads,
                                            int32_t head_dim) {
  if (bad_chunks(n_tokens, batch, n_q_heads, n_kv_heads) ||
      bad_cache(n_kv_heads, head_dim, (int64_t)n_kv_heads * kPageTok * head_dim, 1))
    return 0;
  // as few sequences as the call may have: the same tokens in fewer of them may take larger blocks
  return chunk_attention_workspace(n_tokens, 1, n_q_heads, n_kv_heads, head_dim);
}

pard_status pard_chunk_attention(const void* d_q, int64_t q_stride, int32_t dtype, int32_t n_tokens, int32_t batch,
                                 int32_t n_q_heads, int32_t n_kv_heads, int32_t head_dim, const void* d_k_cache,
                                 const void* d_v_cache, int64_t page_stride, const uint8_t* d_k_scale,
                                 const uint8_t* d_v_scale, int64_t scale_stride, int32_t n_pages,
                                 const int32_t* d_page_table, int32_t max_pages, const int32_t* d_starts,
                                 const int32_t* d_ctx_len, int32_t window, int32_t sinks, float scale, void* d_out,
                                 void* d_workspace, size_t workspace_bytes, void* stream) {
  if (n_tokens == 0) return PARD_OK;
  if (!d_q || !d_k_cache || !d_v_cache || !d_page_table || !d_starts || !d_ctx_len || !d_out || !d_workspace)
    return refuse(PARD_ERR_ARG, "chunk attention: null pointer");
  if (!two_byte(dtype)) return refuse(PARD_ERR_SHAPE, "chunk attention: type must be bf16 or fp16");
  if (const char* why = bad_cache(n_kv_heads, head_dim, page_stride, n_pages)) return refuse(PARD_ERR_SHAPE, why);
  if (const char* why = bad_chunks(n_tokens, batch, n_q_heads, n_kv_heads)) return refuse(PARD_ERR_SHAPE, why);
  if (d_k_scale || d_v_scale)
    if (const char* why = bad_scales(d_k_scale, d_v_scale, scale_stride, page_stride, n_kv_heads)) return refuse(PARD_ERR_ARG, why);
  if (max_pages < 1 || max_pages > (1 << 26)) return refuse(PARD_ERR_ARG, "page table width outside [1, 2^26]");
  if (window < 0 || sinks < 0) return refuse(PARD_ERR_ARG, "chunk attention: window and sinks must not be negative");
  if (q_stride < (int64_t)n_q_heads * head_dim) return refuse(PARD_ERR_ARG, "rows overlap: row stride too small");
  if (q_stride % 8 || !aligned16(d_q) || !aligned16(d_k_cache) || !aligned16(d_v_cache) || !aligned16(d_out) ||
      !aligned16(d_workspace))
    return refuse(PARD_ERR_ARG, "rows, caches, output and workspace must start on 16-byte boundaries");
  if (overlap(d_out, d_q, q_stride, (int64_t)n_q_heads * head_dim, n_tokens))
    return refuse(PARD_ERR_ARG, "chunk attention: the output lies over the queries");
  if (!std::isfinite(scale)) return refuse(PARD_ERR_ARG, "the scale must be finite");
  if (chunk_attention_places(n_tokens, batch, n_q_heads, n_kv_heads, max_pages) >= ((int64_t)1 << 31))
    return refuse(PARD_ERR_SHAPE, "more than 2^31 tiles of 128 keys: shorter page tables, chunks or a smaller batch");
  if (workspace_bytes < chunk_attention_workspace(n_tokens, batch, n_q_heads, n_kv_heads, head_dim))
    return refuse(PARD_ERR_ARG, "workspace smaller than pard_chunk_attention_workspace_bytes");
  const ChunkAttnArgs a{d_q, d_k_cache, d_v_cache, d_k_scale, d_v_scale, q_stride, page_stride, scale_stride, d_page_table,
                        d_starts, d_ctx_len, dtype, n_tokens, batch, n_q_heads, n_kv_heads, head_dim, max_pages, n_pages,
                        window, sinks, scale, d_out, d_workspace};
  return launched([&] { launch_chunk_attention(a, reinterpret_cast<cudaStream_t>(stream)); });
}

pard_status pard_adjust_logits(const void* d_logits, int64_t row_stride, int32_t dtype, int32_t batch, int32_t width,
                               int32_t vocab, const int32_t* d_history, int32_t max_history, const int32_t* d_hist_len,
                               const int32_t* d_prompt_len, const float* d_repetition, const float* d_frequency,
                               const float* d_presence, const int32_t* d_bias_ids, const float* d_bias, int32_t n_bias,
                               const uint32_t* d_allowed, const int32_t* d_tokens, const uint64_t* d_mask, void* d_out,
                               int64_t out_stride, void* stream) {
  if (batch == 0 || width == 0) return PARD_OK;
  if (!d_logits || !d_out) return refuse(PARD_ERR_ARG, "adjust_logits: null pointer");
  if (dtype != DT_F32 && !two_byte(dtype)) return refuse(PARD_ERR_SHAPE, "adjust_logits: type must be fp32, bf16 or fp16");
  if (batch < 0 || batch > 65535 || width < 0 || (int64_t)batch * width > (1 << 24))
    return refuse(PARD_ERR_ARG, "adjust_logits: batch outside [0, 65535] or more than 2^24 rows");
  if (vocab < 1 || vocab > kSampleMaxVocab) return refuse(PARD_ERR_SHAPE, "adjust_logits: vocabulary outside [1, 262144]");
  if (max_history < 0 || max_history > kMaxHistory) return refuse(PARD_ERR_ARG, "adjust_logits: history outside [0, 524000]");
  if (max_history > 0 && (!d_history || !d_hist_len)) return refuse(PARD_ERR_ARG, "adjust_logits: a history needs its tokens and lengths");
  if (n_bias < 0 || n_bias > kMaxBiases) return refuse(PARD_ERR_ARG, "adjust_logits: biases outside [0, 2047]");
  if (n_bias > 0 && (!d_bias_ids || !d_bias)) return refuse(PARD_ERR_ARG, "adjust_logits: biases need their tokens and values");
  if (row_stride < vocab || out_stride < vocab) return refuse(PARD_ERR_ARG, "rows overlap: row stride too small");
  const int64_t size = dtype == DT_F32 ? 4 : 2, rows = (int64_t)batch * width;
  if (!(d_out == d_logits && (out_stride == row_stride || rows == 1)) &&
      overlap_apart(d_logits, row_stride * size, d_out, out_stride * size, vocab * size, rows))
    return refuse(PARD_ERR_ARG, "adjust_logits: the output lies over the logits, but not in place");
  if (!d_tokens != !d_mask) return refuse(PARD_ERR_ARG, "adjust_logits: a tree needs its tokens and its mask");
  if (d_tokens && width > kTreeMaxNodes) return refuse(PARD_ERR_ARG, "tree width outside [1, 256]");
  if (reinterpret_cast<uintptr_t>(d_logits) % size || reinterpret_cast<uintptr_t>(d_out) % size)
    return refuse(PARD_ERR_ARG, "adjust_logits: logits not aligned to their type");
  const AdjustArgs a{d_logits, row_stride, out_stride, dtype, batch, width, vocab, max_history, n_bias,
                     max_history ? d_history : nullptr, d_hist_len, d_prompt_len, d_repetition, d_frequency, d_presence,
                     d_bias_ids, d_bias, d_allowed, d_tokens, d_mask, d_out};
  return launched([&] { launch_adjust_logits(a, reinterpret_cast<cudaStream_t>(stream)); });
}

}  // extern "C"
