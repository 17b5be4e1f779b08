/*
 * swarm_cache.h - C ABI of token-by-token generation with a trained stage (MI355X, gfx950).
 *
 * Once a model has been trained, a stage continues sequences: it keeps the keys and values of the tokens it has seen and runs its
 * blocks on the new ones only.  A long sequence costs a peer 4 d bytes per token and block application in bf16, and a shared block
 * has a cache for each of its applications, so keys and values are kept in the number format that the stage boundaries use
 * (swarm_codec_encode / swarm_codec_encode_s16 in swarm_stage.h): int8 codes with one scale per 64 consecutive elements.
 *
 * The cache of ONE block application is a pool of pages of `page_tokens` tokens:
 *     k_codes  int8  [n_pages, n_kv_heads, page_tokens, d_head]      v_codes  int8  [n_pages, n_kv_heads, d_head, page_tokens]
 *     k_scales, v_scales  [n_pages, n_kv_heads, d_head / 64, page_tokens]  fp32 (scale_bits 32) or bf16 bit patterns (16)
 * (values lie transposed, because attention contracts them over tokens).  page_table [batch, table_pages] holds the page of the
 * tokens i * page_tokens .. (i + 1) * page_tokens - 1 of every sequence; the pools of a stage's applications may share one.  A page
 * of as many tokens as a sequence may have is a contiguous cache.
 *
 * A call works on rows b * tokens + t, t < tokens: token t of the new ones of sequence b.  Device arrays say how many there are:
 *     past  [batch]  tokens that the cache holds before them         fresh [batch]  new tokens, 0 .. tokens; NULL: `tokens` of each
 * The library cannot check device data.  What it finds out of range is never used as an address: a sequence with past < 0, fresh
 * outside 0 .. tokens or past + fresh beyond its table_pages * page_tokens tokens is left out of the call (none of its cache, none of its output
 * rows is written), and a page outside 0 .. n_pages - 1 is not written, is read as zeros, and is not attended to.  Output rows
 * t >= fresh are left as they were.  Two sequences of one call must not write to the same page.
 *
 * General rules: those of swarm_stage.h.  Row pitches are in elements; rows start on 16 bytes.
 */
#ifndef SWARM_CACHE_H
#define SWARM_CACHE_H

#include "swarm_stage.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Constraints: 1 <= n_kv_heads, n_heads % n_kv_heads == 0, n_heads <= 1024; d_head 64 or 128; page_tokens a power of two, 16 to 65536;
 * n_pages, batch, table_pages >= 1; table_pages * page_tokens <= 2^30; batch * tokens <= 2^24 in every call. */
typedef struct {
  int32_t n_heads;      /* query heads; heads g * n_heads / n_kv_heads .. of them share key / value head g */
  int32_t n_kv_heads;
  int32_t d_head;
  int32_t page_tokens;
  int32_t n_pages;      /* pages of the pool                            */
  int32_t batch;        /* sequences                                    */
  int32_t table_pages;  /* pages that one sequence may have             */
  int32_t dtype;        /* swarm_dtype of queries, keys, values, outputs */
  int32_t scale_bits;   /* 32 or 16                                     */
} swarm_cache_config;

typedef struct { int8_t *k_codes, *v_codes; void *k_scales, *v_scales; } swarm_cache;   /* 16-byte aligned */

/* Appends the new tokens: rows of k and v (n_kv_heads * d_head elements each, `row_pitch` apart, as in a fused q | k | v product)
 * are quantised into the pages of the tokens past .. past + fresh - 1.
 * rotary != 0: the pairs (x[2i], x[2i+1]) of every head of k are rotated by pos * 10000^(-2i/d_head) first, and so are those of q
 * (n_heads * d_head elements, the same row_pitch), which go to q_out (rows q_out_pitch apart; may be q itself).  pos =
 * positions[b * tokens + t], or past + t where positions is NULL.  Angles and products are held in
 * 64 bits and rounded to fp32, which the codec quantises, and from there to the dtype in q_out.  rotary == 0: q, q_out and positions are NULL. */
swarm_status swarm_cache_append(const swarm_cache_config *cfg, const swarm_cache *cache, const int32_t *page_table,
                                const int32_t *past, const int32_t *fresh, int32_t tokens, const void *q, const void *k,
                                const void *v, size_t row_pitch, const int32_t *positions, int32_t rotary, void *q_out,
                                size_t q_out_pitch, void *hip_stream);

/* Reads the tokens first .. first + count - 1 back (count NULL: `tokens` of each sequence): code * scale, rounded to the dtype, into
 * rows of k_out and v_out (n_kv_heads * d_head elements, contiguous).  first and count have the bounds of past and fresh. */
swarm_status swarm_cache_read(const swarm_cache_config *cfg, const swarm_cache *cache, const int32_t *page_table,
                              const int32_t *first, const int32_t *count, int32_t tokens, void *k_out, void *v_out,
                              void *hip_stream);

/* Keeps n_kept[b] of the `tokens` (at most 64) drafted tokens that lie behind the first past[b]: draft token kept[b * tokens + j]
 * moves to place j, in any order, the same one more than once if asked (keys keep the rotation they were written with, which is
 * that of their depth).  An index outside 0 .. tokens - 1 leaves place j as it is, and so does a page out of range on either side.
 * n_kept has the bounds of fresh.
 * Places from n_kept on are not defined after the call: the next append writes them. */
swarm_status swarm_cache_keep(const swarm_cache_config *cfg, const swarm_cache *cache, const int32_t *page_table,
                              const int32_t *past, const int32_t *kept, const int32_t *n_kept, int32_t tokens,
                              void *hip_stream);

/* Attention of the new tokens, which have been appended, over the cache: for row (b, t) and query head h with key / value head g
 *     out = sum_j p_j v_j / sum_j p_j,   p_j = exp(q . k_j / sqrt(d_head)),
 * over the tokens j < past, and over those new tokens u < fresh (j = past + u) that tree[b * tokens + t] has bit u set for; tree NULL:
 * u <= t.  With a tree, tokens <= 64; tokens * n_heads / n_kv_heads <= 2^24.  A row that sees no token at all is zeros.
 * What a row does not see has no part in it.  Sums are held in 32 bits.  In bf16 a p_j may be off by 2^-11 of itself or by 2^-22 of the row's
 * largest, whichever is more, in the sum of v_j.  p_j times a value's scale may be left out there where it is below 2^-50 of the row's
 * largest in that block of 64 elements.  A value's scale that is infinite or no number makes that block NaN in
 * the rows that see it; a key's scale or an element of q that is makes the row NaN.
 * q rows (n_heads * d_head elements) are q_pitch apart, out rows out_pitch.  max_len: a bound on past + fresh that the caller knows
 * (0: what page_table can hold); it decides over how many workgroups a sequence is spread, and the workspace; a longer sequence
 * is right too, only slower.  workspace: swarm_cache_attention_workspace_bytes, 256-byte aligned, or NULL where that is 0. */
size_t swarm_cache_attention_workspace_bytes(const swarm_cache_config *cfg, int32_t tokens, int32_t max_len);
swarm_status swarm_cache_attention(const swarm_cache_config *cfg, const swarm_cache *cache, const int32_t *page_table,
                                   const int32_t *past, const int32_t *fresh, int32_t tokens, int32_t max_len, const void *q,
                                   size_t q_pitch, const uint64_t *tree, void *out, size_t out_pitch, void *workspace,
                                   size_t workspace_bytes, void *hip_stream);

/* The stage on the new tokens of cfg->batch sequences, cfg->seq of them each (rows as above): as swarm_stage_forward, with every
 * application's attention over its own cache, to which the tokens are appended.  caches: host array of n_layers * n_repeat pools, in
 * the order of the applications; cache_cfg: batch, dtype, n_heads and d_head as the stage's, n_kv_heads = n_heads.  The rotary block's
 * positions are `positions`, or past + t; with the GeLU block positions is NULL.  x_in, x_out [batch * seq, d_model]; rows of x_out
 * that `fresh` leaves out hold no defined values, and what x_in holds there reaches no other row. */
size_t swarm_stage_extend_workspace_bytes(const swarm_stage_config *cfg, const swarm_cache_config *cache_cfg, int32_t max_len);
swarm_status swarm_stage_extend(const swarm_stage_config *cfg, const swarm_block_params *params, const swarm_cache_config *cache_cfg,
                                const swarm_cache *caches, const int32_t *page_table, const int32_t *past, const int32_t *fresh,
                                const int32_t *positions, const uint64_t *tree, int32_t max_len, const void *x_in, void *x_out,
                                void *workspace, size_t workspace_bytes, void *hip_stream);

#ifdef __cplusplus
}
#endif
#endif /* SWARM_CACHE_H */
