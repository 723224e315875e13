/* Operators of a serving loop around the decode step (see pard.h): attention of
 * chunks of new tokens over the paged cache, an 8-bit form of that cache, and
 * what requests ask of their logits.  Conventions, types and caches are those of
 * pard.h's tree operators: no context, all device memory the caller's, work
 * enqueued on `stream`, 16 tokens a page, page ids outside [0, n_pages) never
 * accessed. */
#ifndef PARD_SERVE_H
#define PARD_SERVE_H

#include "pard.h"

#ifdef __cplusplus
extern "C" {
#endif

/* pard_qk_norm_rope into an 8-bit cache.  A page of d_k_cache or d_v_cache holds
 * [n_kv_heads][16][head_dim] codes (e4m3, one byte; page_stride, a multiple of 16,
 * counts them), and of d_k_scale or d_v_scale [n_kv_heads][16] biased exponents
 * (e8m0: b stands for 2^(b - 127); pages scale_stride bytes apart, a multiple of
 * 16).  For each token and head b is the smallest in [1, 254] with |x| <= 448 *
 * 2^(b - 127) for all its finite entries, and a code is x / 2^(b - 127) rounded
 * to the nearest, ties to even, from the 32-bit x (queries are rounded to `dtype`
 * as there).  Infinities and NaN are stored as NaN.  The cache holds what fp32
 * does, but pard_chunk_attention reads entries as fp16: larger ones than 65504 come
 * back as 65504, and what lies between multiples of 2^-24 rounded to them.  No two
 * tokens of a call may have the same slot (but negative ones). */
pard_status pard_qk_norm_rope_quantized(const void* d_qkv, int64_t qkv_stride, int32_t dtype, int32_t n_tokens,
                                        int32_t n_q_heads, int32_t n_kv_heads, int32_t head_dim, const void* d_q_gain,
                                        const void* d_k_gain, float eps, const int32_t* d_pos, const int64_t* d_slots,
                                        const float* d_inv_freq, int32_t rot_dim, int32_t interleaved, float amplitude,
                                        void* d_q, int64_t q_stride, void* d_k_cache, void* d_v_cache, int64_t page_stride,
                                        uint8_t* d_k_scale, uint8_t* d_v_scale, int64_t scale_stride, int32_t n_pages,
                                        void* stream);

/* Attention of the new tokens of a batch (pieces of prompts, single tokens, or
 * both) over their sequences' caches:
 *   o = sum_j softmax_j(scale q . k_j) v_j
 * d_q [n_tokens][q_stride]: rows d_starts[b] .. d_starts[b + 1] - 1 are sequence
 * b's (d_starts [batch + 1] does not decrease; rows outside [0, n_tokens) do not
 * exist), at positions d_ctx_len[b], d_ctx_len[b] + 1, ...; their own keys and
 * values are in the cache already.  A token at position p sees the keys j <= p,
 * and, with window > 0, of those only p - window < j and j < sinks (without a
 * window sinks has no effect).  Query head h reads key/value head
 * h / (n_q_heads / n_kv_heads).  d_out [n_tokens][n_q_heads][head_dim]; rows of no
 * sequence are left as they were, a token none of whose keys lies in a page of
 * the pool gets zeros.  Masked keys and values may hold infinities or NaN.
 * Caches of `dtype` (d_k_scale and d_v_scale null), or 8-bit ones as
 * pard_qk_norm_rope_quantized writes them: an entry is then its code times its
 * power of two, held to +-65504 and to multiples of 2^-24.  Scores and sums are
 * held in 32 bits; probabilities are rounded to `dtype` (with an 8-bit cache to
 * fp16) before they multiply the values.  An infinity in a value makes the outputs
 * of the tokens that see it infinite, or NaN where its weight is 0 in 32 bits.
 * d_out must not overlap d_q.  d_workspace: pard_chunk_attention_workspace_bytes
 * (0: invalid arguments) bytes, which are enough for all calls with these heads and
 * no more tokens and sequences, the first 4096 of them zero before the first call;
 * each call leaves them fit for the next, of any sizes that they are enough for,
 * and for pard_tree_attention (whose workspace fits here too).  Calls that may overlap on the GPU need one
 * each.  Should a wait inside the kernel ever run out (2 s), the output is NaN,
 * and so is that of later calls until those bytes are zeroed again. */
size_t pard_chunk_attention_workspace_bytes(int32_t n_tokens, int32_t batch, int32_t n_q_heads, int32_t n_kv_heads,
                                            int32_t head_dim);
pard_status pard_chunk_attention(const void* d_q, int64_t q_stride, int32_t dtype, int32_t n_tokens, int32_t batch,
                                 int32_t n_q_heads, int32_t n_kv_heads, int32_t head_dim, const void* d_k_cache,
                                 const void* d_v_cache, int64_t page_stride, const uint8_t* d_k_scale,
                                 const uint8_t* d_v_scale, int64_t scale_stride, int32_t n_pages,
                                 const int32_t* d_page_table, int32_t max_pages, const int32_t* d_starts,
                                 const int32_t* d_ctx_len, int32_t window, int32_t sinks, float scale, void* d_out,
                                 void* d_workspace, size_t workspace_bytes, void* stream);

/* What requests ask of their logits before a token is drawn.  d_logits [batch *
 * width][row_stride]: `width` rows a sequence (1, or the nodes of its tree), fp32,
 * bf16 or fp16; d_out the same type and rows out_stride apart, may be d_logits
 * row for row (other overlaps are refused).  In 32 bits, in this order, rounded once:
 *   z = z / r where z > 0, else z r       tokens of the row's history
 *   z = z - f c - p [c > 0]               c: how often the token was generated
 *   z = z + its biases                    summed in the list's order
 *   z = -infinity                         where the row's mask has a clear bit
 * The history: d_history [batch][max_history], the first d_hist_len[b] entries
 * (clamped to [0, max_history]); the first d_prompt_len[b] of them (null: none)
 * are the prompt, which counts for r alone, the others are generated.  For a tree,
 * d_tokens [batch][width] and d_mask [batch][width][ceil(width / 64)] of
 * pard_tree_plan: the tokens of a row's set bits are generated too (width <= 256).
 * r, f, p: d_repetition, d_frequency, d_presence [batch] (null: 1, 0, 0).  Biases:
 * d_bias_ids, d_bias [batch][n_bias] (at most 2047).  d_allowed [batch * width]
 * [ceil(vocab / 32)] (null: all): bit v mod 32 of word v / 32.  Tokens outside
 * [0, vocab) are passed over.  vocab <= 262144, max_history <= 524000, batch <=
 * 65535, batch * width <= 2^24. */
pard_status pard_adjust_logits(const void* d_logits, int64_t row_stride, int32_t dtype, int32_t batch, int32_t width,
                               int32_t vocab, const int32_t* d_history, int32_t max_history, const int32_t* d_hist_len,
                               const int32_t* d_prompt_len, const float* d_repetition, const float* d_frequency,
                               const float* d_presence, const int32_t* d_bias_ids, const float* d_bias, int32_t n_bias,
                               const uint32_t* d_allowed, const int32_t* d_tokens, const uint64_t* d_mask, void* d_out,
                               int64_t out_stride, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* PARD_SERVE_H */
