/*
 * gblatent.h - C ABI of latent attention on GB300 (sm_103a): attention whose
 * keys and values are, for all heads, one latent vector a token and one rotary
 * key beside it. It takes the place of attn_append, attn_prompt and attn_cached
 * (gbattn.h) in a decoder layer and stands before the MoE layer of gbmoe.h
 * (same library, status codes, gbmoe_status_string, gbmoe_last_cuda_error).
 * The paper names the DeepSeek path only (Section 6.2), without its attention.
 *
 * A token's row [latent c (R) | rotary key k_r (P)] is what the cache holds. The
 * keys and values of head h are linear in c: k_h = W_k,h c (N elements), v_h =
 * W_v,h c (V elements), which are plain products left to the caller. Two forms of
 * the same attention follow.
 *   expanded (latent_prompt): k_h, v_h for every token, the shared k_r beside k_h:
 *     score = scale (q_n . k_h + q_r . k_r), out_h = sum_j softmax_j v_h,j
 *   absorbed (latent_cached): W_k,h goes into the query, W_v,h behind the sum:
 *     score = scale (W_k,h^T q_n . c + q_r . k_r), out_h = sum_j softmax_j c_j,
 *     so the cached rows serve all heads as they are: R + P elements a token
 *     instead of heads (N + P + V).
 *
 * Conventions: those of gbattn.h (device pointers, no allocation, no
 * synchronisation, host-side refusals, packed sequences and offsets clamped to the
 * batch, which keys a query sees, a query without keys gives 0 and -inf). Rows
 * without heads are a gbattn_rows whose head_stride is not read.
 * A latent or value that is no number makes its elements so for the queries that
 * see it, whatever its weight (latent_cached on the tensor cores: others of the
 * query's elements too), and does nothing to queries that do not see it.
 */
#ifndef GBLATENT_H
#define GBLATENT_H

#include "gbattn.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef struct gblatent_config {
    int32_t heads;         /* query heads, up to 4096                                          */
    int32_t latent_dim;    /* R: a multiple of 8, up to 512                                    */
    int32_t rope_dim;      /* P: a multiple of 16, up to 128, or 0                             */
    int32_t nope_dim;      /* N: elements of a head's own key, a multiple of 8, up to 128      */
    int32_t value_dim;     /* V: a multiple of 8, up to 128                                    */
    int32_t act_dtype;     /* everything but tables, lengths and lse: GBMOE_F32 or GBMOE_BF16  */
    int32_t causal;        /* 1: keys up to the query's position; 0: all of them               */
    float scale;           /* multiplies the products (1/sqrt(N + P) as a rule)                */
    int32_t rotary_layout; /* GBATTN_HALF or GBATTN_INTERLEAVED: all P elements turn           */
    float rotary_scale;    /* multiplies cos and sin (1: a plain rotation)                     */
    float norm_eps;        /* of the latent's RMS norm                                         */
    int32_t page;          /* tokens of a cache page: 16, 32, 64 or 128                        */
} gblatent_config;

/* A pool of cache pages [n_pages, page, R + P] of act_dtype, 16-byte aligned. */
typedef struct gblatent_cache {
    void* rows;
    int32_t n_pages;
} gblatent_cache;

/* GBMOE_OK if the config is valid and covered, else the status a call with it
 * would return. */
int latent_check_config(const gblatent_config* cfg);

/* Workspace bytes of latent_prompt and latent_cached for up to T query tokens of
 * B sequences (0: invalid config or sizes). Scratch only; its first word is the
 * device error word that moe_device_status reads and clears (set it to 0 once
 * before the first call: the calls only add to it). 256-byte aligned. */
size_t latent_workspace_size(const gblatent_config* cfg, int32_t T, int32_t B);

/*
 * Appends T new tokens' rows kv [T, R + P] to the cache: token i of sequence b is
 * its token p = kv_len[b] - n + i (n new tokens) and goes to slot p % page of page
 * page_table[b][p / page]. On the way
 *   c' = c / sqrt(mean(c^2) + norm_eps) * gamma   (gamma [R], or NULL: c' = c)
 *   k_r' = k_r turned by its position             (positions [T] int32 or NULL: p)
 * in fp32, rounded once. Optional outputs: kv_out [T, R + P], the same rows (what
 * the expansion to keys and values takes; kv_out may be kv), and q_out, the
 * rotary parts of the queries q [T, heads, P] turned likewise (q_out may be q).
 * table: attn_rope_table of P. Tokens whose place p is negative or beyond the
 * page table, or whose page is outside the pool, are not stored; their outputs are
 * written. Two sequences may not append to the same slot in one call. Only the
 * rows of kv and q may be written by it, each in its own place (kv_out, q_out).
 */
int latent_append(const gblatent_config* cfg, int32_t T, const gbattn_batch* batch, const gbattn_rows* kv,
                  const void* gamma, const gbattn_rows* q, const int32_t* positions, const uint64_t* table,
                  const gblatent_cache* cache, const gbattn_rows* kv_out, const gbattn_rows* q_out, void* stream);

/*
 * Expanded form over packed sequences: q [Tq, heads, N + P], k [Tk, heads, N],
 * k_rope [Tk, P] (already turned, one for all heads), v [Tk, heads, V], out [Tq,
 * heads, V], cu_q and cu_k [B+1] (equal for whole prompts; a sequence with more
 * keys than queries has its queries at the end), lse [Tq, heads] fp32 or NULL.
 * k_rope is not read when P is 0. out may not overlap the inputs. bf16 runs on the
 * tensor cores (weights rounded to bf16: off by 2^-8 of themselves) where P is up
 * to 64, scale is above 0 and no stride that is used is 0 (or 2^39 elements and
 * more), else on CUDA cores, which are far slower. On the tensor cores a value that
 * is no number costs time in queries that do not see it but lie in a tile that
 * reaches its 128 keys (one behind a sequence's end, say): they are computed once
 * more, 0.13 us a key and up to 32 after each other, so that past some 400 000 keys
 * the waits may run out. Set such rows to something finite where that counts.
 */
int latent_prompt(const gblatent_config* cfg, int32_t Tq, int32_t Tk, int32_t B, const gbattn_rows* q,
                  const gbattn_rows* k, const gbattn_rows* k_rope, const gbattn_rows* v, const int32_t* cu_q,
                  const int32_t* cu_k, const gbattn_rows* out, float* lse, void* workspace, size_t workspace_bytes,
                  void* stream);

/*
 * Absorbed form of the batch's query tokens over their cached rows (the queries'
 * own tokens already appended): q [T, heads, R + P], out [T, heads, R], lse [T,
 * heads] fp32 or NULL. Meant for few query tokens per sequence (decoding, draft
 * tokens); any number works. Long contexts are split over CTAs and joined by a
 * second launch, deterministically; how many rows a CTA has follows from T, B and
 * max_pages * page, so a table no wider than the longest context is fastest where
 * keys are few. bf16 with R a multiple of 128 and P up to 64
 * runs on the tensor cores (weights rounded to bf16: off by 2^-8 of themselves),
 * else on CUDA cores. A token whose page is outside the pool is masked. out may
 * not overlap the inputs. T * heads, max_pages * page and n_pages * page up to
 * 2^30, else GBMOE_EUNSUPPORTED.
 */
int latent_cached(const gblatent_config* cfg, int32_t T, const gbattn_batch* batch, const gbattn_rows* q,
                  const gblatent_cache* cache, const gbattn_rows* out, float* lse, void* workspace,
                  size_t workspace_bytes, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* GBLATENT_H */
