/*
 * pearl_latent.h -- attention whose keys and values come from one latent vector a token, over a paged
 * cache of those vectors (paper, Background and section 4.3, Eq. 1: the context grows with every turn and its cache is what
 * decode reads; a latent cache holds one short row a token for all heads).
 *
 * A token caches c (latent_dim channels) and r (rope_dim channels, rotated by its position).  With the projections that
 * expand c into a head's keys and values absorbed into the queries and into what follows the attention, a query
 * head is q = (q_c, q_r) of latent_dim + rope_dim channels, and for new token i of sequence b at position
 * p = ctx_lens[b] + i
 *     s_j = scale * (q_c . c_j + q_r . r_j)   for j = 0 .. p,
 *     o   = sum_j softmax(s)_j c_j,            lse = ln sum_j exp(s_j):
 * every head reads the same row of the cache as key and its latent part as value.
 *
 * Conventions are those of pearl_attn.h, with these tensors:
 *   cache: bf16 [num_pages][page_size][latent_dim + rope_dim]; position p of sequence b is row p % page_size of page
 *          block_table[b*bt_stride + p/page_size].  Any bytes are valid in rows that no attended position owns.
 *   q: bf16 [total_q][num_q_heads][latent_dim + rope_dim]; out: bf16 [total_q][num_q_heads][latent_dim];
 *   lse: fp32 [total_q][num_q_heads] or NULL.
 * Scores, softmax state and sums are held in 32 bits; weights enter the second product in bf16, outputs are rounded to bf16.
 * A row of the cache with infinite or NaN channels reaches only the tokens that attend to it.  A token whose score of the row is NaN or
 * plus infinity has NaN in all channels and in lse.  Where the score is minus infinity the row has weight 0: the output is NaN in those latent channels
 * that are infinite in the row (in none, if all of them are in its rotated part) and lse is without it.  Where all of a token's scores are minus
 * infinity its output is NaN and lse minus infinity.
 * Supported: (latent_dim, rope_dim) (512, 64) and (256, 32); page_size 16; 1 .. 128 query heads;
 * max_q_len <= 2^21, max_kv_len <= 2^25.
 */
#ifndef PEARL_LATENT_H
#define PEARL_LATENT_H

#include "pearl_attn.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef struct {
  int32_t num_q_heads;   /* 1 .. 128 */
  int32_t latent_dim;    /* 512 or 256 */
  int32_t rope_dim;      /* 64 with 512, 32 with 256 */
  int32_t page_size;     /* tokens per page: 16 */
  int32_t num_pages;     /* physical pages of the cache */
} pearl_latent_shape;

/*
 * Appends the new tokens' rows: c normalised (RMS norm with rope->k_weight [latent_dim]; NULL: as it is), r rotated
 * (pearl_rope with rotary_dim == rope_dim), into their slots; and rotates the queries' part into the tails of the
 * absorbed queries.  rope->q_weight must be NULL.
 *   q_rope: bf16 [total_q][num_q_heads][rope_dim] (read), q_rope_stride elements from one head's row to the next
 *           one's, a token's last head's to the next token's first alike (a multiple of 8, >= rope_dim);
 *   rows_new: bf16 [total_q][latent_dim + rope_dim] (read): c, then r; rows_stride elements from a token to the next (a multiple
 *           of 8, >= latent_dim + rope_dim);
 *   q: the last rope_dim channels of every head are written, the others left as they are; cache: written.
 * q_rope may be the tails of q themselves (their rows are then rotated in place); otherwise it and rows_new must not overlap q or
 * the cache.  No other byte of the cache changes; rows whose page id is outside [0, num_pages) or
 * whose logical page is beyond bt_stride are skipped (their queries are written all the same).
 */
pearl_status pearl_latent_append(const pearl_latent_shape* shape, const pearl_seq_desc* seqs, const pearl_rope* rope,
                                 const void* q_rope, int64_t q_rope_stride, const void* rows_new, int64_t rows_stride,
                                 void* q, void* cache, void* stream);

/*
 * Bytes of device workspace that an attention call below needs for (shape, seqs): the list of tiles that are cut along the
 * keys, and their partial results (fp32), 512 of at most 64 rows: up to 67 MB.  A function of the shape and the host
 * bounds only; needs no initialisation.  0 if the arguments are invalid (pearl_last_error() says why).
 */
size_t pearl_latent_workspace_bytes(const pearl_latent_shape* shape, const pearl_seq_desc* seqs);

/*
 * Batched single-token decode: seqs->cu_q_lens must be NULL; row b of q and out is sequence b's new token at position
 * ctx_lens[b], whose row the cache already holds (pearl_latent_append first, on the same stream).
 * Contexts are cut into shares that run in parallel and are joined by log-sum-exp.
 * out must not overlap q or the cache.
 */
pearl_status pearl_attn_latent_decode(const pearl_latent_shape* shape, const pearl_seq_desc* seqs, const void* q,
                                      const void* cache, float softmax_scale, void* out, float* lse, void* workspace,
                                      size_t workspace_bytes, void* stream);

/*
 * Prefill-append: every new token of every sequence attends to its context and causally to the new ones, whose rows the
 * cache already holds.  Sequences without new tokens are skipped; rows behind the last sequence are left as they
 * were.  A batch of single tokens, or of a few each (drafted tokens that are verified), can take this call too.  A colocated batch, of large turns
 * and of single tokens on long contexts, is better served by two calls, pearl_attn_latent_decode for the latter: the cut goes by the batch's longest
 * and average turn (63 single tokens on 2K to 16K and a turn of 2000 on 9K, 16 heads: 901 us in one call, 746 in two; 56 single tokens and 8 turns of 1000: 1840
 * and 1504; with 128 heads 3% apart).
 */
pearl_status pearl_attn_latent_prefill_append(const pearl_latent_shape* shape, const pearl_seq_desc* seqs, const void* q,
                                              const void* cache, float softmax_scale, void* out, float* lse, void* workspace,
                                              size_t workspace_bytes, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* PEARL_LATENT_H */
