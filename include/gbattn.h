/*
 * gbattn.h - C ABI of the attention half of a decoder layer on GB300 (sm_103a):
 * rotary positions, appending keys and values to a paged cache, causal
 * attention over packed prompts, and attention of few query tokens per
 * sequence over the paged cache. They stand before the MoE layer of gbmoe.h
 * (same library, same status codes, gbmoe_status_string, gbmoe_last_cuda_error).
 * The paper has no counterpart: its running example is the MoE layer alone.
 *
 * Conventions (as in gbmoe.h)
 *  - Pointers are DEVICE pointers owned by the caller unless a parameter says
 *    host. The library never allocates, frees or synchronises; calls are
 *    asynchronous on `stream` and run on the current device.
 *  - Argument errors are found on the host before anything is launched and
 *    return a negative status; nothing is written then. Lengths, offsets and
 *    page ids live on the device and are not checked there as errors: offsets
 *    are clamped to the batch, and pages outside the pool are left out.
 *  - Tables are 16-byte aligned, int32 and fp32 arrays 4-byte aligned.
 *  - q, k, v, out are [tokens, heads, head_dim] with strides (gbattn_rows):
 *    slices of one projection's rows are fine. The head_dim elements are
 *    contiguous; base and strides are multiples of 16 bytes.
 *  - Sequences are packed: sequence b's tokens are rows cu[b] .. cu[b+1]-1
 *    (cu [B+1] int32, not decreasing, cu[0] >= 0, cu[B] <= T).
 *  - Names: T tokens, B sequences, D head_dim, G = heads_q / heads_kv.
 *
 * Which keys a query sees: sequence b has n queries and m keys, its i-th
 * query stands at position p = m - n + i and sees keys j with j < m, j <= p
 * (causal) and j > p - window (window > 0). A query that sees no key gives 0
 * (and -inf as its log sum). Keys and values that no query sees, other
 * sequences' rows and unwritten cache slots may hold anything, NaN included.
 *   out = sum_j softmax_j(scale * q.k_j) v_j; lse = ln sum_j exp(scale * q.k_j)
 * fp32 sums and softmax statistics; out rounded once to act_dtype. Where the
 * tensor cores do it (see attn_prompt, attn_cached) the softmax weights are
 * rounded to 16 bits before the second product, their sum is not.
 * A value that is no number makes its column so for the queries that see it,
 * whatever its weight; a query that sees keys, all with scores of -inf, is 0 / 0.
 */
#ifndef GBATTN_H
#define GBATTN_H

#include "gbmoe.h"

#ifdef __cplusplus
extern "C" {
#endif

/* rotary_layout: the pairs that turn together, i = 0 .. rotary_dim/2 - 1 */
enum {
    GBATTN_HALF = 0,       /* elements i and i + rotary_dim/2 */
    GBATTN_INTERLEAVED = 1 /* elements 2i and 2i + 1          */
};

/* cache_dtype */
enum {
    GBATTN_CACHE_ACT = 0, /* act_dtype values                                              */
    GBATTN_CACHE_E4M3 = 1 /* e4m3 codes, one E8M0 scale 2^(s-127) per page and kv head     */
};

typedef struct gbattn_config {
    int32_t heads_q, heads_kv; /* heads_q a multiple of heads_kv; query head h reads kv head h / G */
    int32_t head_dim;          /* D: a multiple of 8, up to 256                             */
    int32_t act_dtype;         /* q, k, v, out: GBMOE_F32 or GBMOE_BF16                     */
    int32_t causal;            /* 1: keys up to the query's position; 0: all of them        */
    int32_t window;            /* > 0: only the last `window` keys up to the position       */
    float scale;               /* multiplies q.k (1/sqrt(D) as a rule)                      */
    int32_t rotary_dim;        /* leading elements of a head that turn: a multiple of 16, or 0 */
    int32_t rotary_layout;     /* GBATTN_HALF or GBATTN_INTERLEAVED                         */
    float rotary_scale;        /* multiplies cos and sin (1: a plain rotation)              */
    int32_t cache_dtype;       /* GBATTN_CACHE_*                                            */
    int32_t page;              /* tokens of a cache page: 16, 32, 64 or 128                 */
} gbattn_config;

/* Rows [tokens, heads, head_dim] at data; strides in elements. */
typedef struct gbattn_rows {
    void* data;
    int64_t token_stride, head_stride;
} gbattn_rows;

/* A pool of cache pages: k, v [n_pages, heads_kv, page, head_dim], e4m3 bytes or
 * act_dtype values, 16-byte aligned; k_scale, v_scale [n_pages, heads_kv] E8M0
 * bytes (E4M3 only, else NULL). Element: e4m3(code) * 2^(scale - 127). */
typedef struct gbattn_cache {
    void *k, *v;
    uint8_t *k_scale, *v_scale;
    int32_t n_pages;
} gbattn_cache;

/* A batch of B sequences over the cache: cu_q [B+1] offsets of their query (or
 * new) tokens, kv_len [B] their keys (the new ones among them, which are the
 * last), page_table [B, max_pages] the pool pages of tokens 0.., page, 2*page..
 * of each sequence. attn_cached cuts lengths beyond max_pages * page to it. */
typedef struct gbattn_batch {
    int32_t B, max_pages;
    const int32_t *cu_q, *kv_len, *page_table;
} gbattn_batch;

/* GBMOE_OK if the config is valid and covered, else the status a call with it
 * would return. */
int attn_check_config(const gbattn_config* cfg);

/* Workspace bytes of attn_prompt and attn_cached for up to T query tokens of B
 * sequences (0: invalid config or sizes). Scratch only; its first word is the
 * device error word that moe_device_status reads and clears (set it to 0 once
 * before the first call: the calls only add to it). 256-byte aligned. */
size_t attn_workspace_size(const gbattn_config* cfg, int32_t T, int32_t B);

/* Frequency scaling of attn_rope_table for contexts beyond the trained one. */
enum {
    GBATTN_ROPE_PLAIN = 0, /* f_i = base^(-2i/rotary_dim) radians per position           */
    GBATTN_ROPE_LINEAR = 1, /* f_i / factor                                              */
    GBATTN_ROPE_NTK = 2,   /* base times factor^(rotary_dim / (rotary_dim - 2))          */
    GBATTN_ROPE_RAMP = 3   /* f_i kept where it turns more than `fast` times within the
                              original context, divided by factor where it turns less than
                              `slow` times, a linear ramp over i between; the usual
                              rotary_scale with it is 0.1 ln(factor) + 1                 */
};

/*
 * Host function: the table that attn_rope and attn_append take, rotary_dim/2
 * entries of 64 bits in HOST memory (the caller copies them to the device).
 * Entry i is f_i / (2 pi) turns per position as a binary fraction of 2^64, so
 * that position * entry mod 2^64 is the exact fraction of a turn: angles do
 * not lose accuracy at long positions. original_ctx, slow and fast are read by
 * GBATTN_ROPE_RAMP only.
 */
int attn_rope_table(int32_t rotary_dim, double base, int32_t scaling, double factor, double original_ctx, double slow,
                    double fast, uint64_t* table);

/*
 * Rotary positions: for every token t and head, the first rotary_dim elements
 * turn by angle positions[t] * f_i (pairs as rotary_layout says),
 *   a' = rotary_scale * (a cos - b sin), b' = rotary_scale * (a sin + b cos),
 * the others are copied; fp32, rounded once. inverse = 1 turns back (-angle,
 * the same rotary_scale), which is also the gradient's map. q (heads_q) and k
 * (heads_kv) are both optional: a pair is left out when its data pointers
 * are NULL. Outputs may be their inputs (same pointer and strides) but not
 * overlap otherwise. positions [T] int32 (negative ones turn backwards).
 */
int attn_rope(const gbattn_config* cfg, int32_t T, const gbattn_rows* q, const gbattn_rows* k,
              const int32_t* positions, const uint64_t* table, int32_t inverse, const gbattn_rows* q_out,
              const gbattn_rows* k_out, void* stream);

/*
 * Appends T new tokens' keys and values to the cache: token i of sequence b is
 * its token p = kv_len[b] - n + i (n new tokens) and goes to slot p % page of
 * page page_table[b][p / page]. Keys turn by their position on the way
 * (rotary_dim 0: as they are; positions [T] int32 or NULL: p). Optional outputs:
 * q_out, the rotated queries (q [T, heads_q]), and k_out, the rotated keys in
 * act_dtype, which attn_prompt takes (k_out may be k, q_out may be q).
 * E4M3: the scale of a page and head covers all its tokens: the smallest
 * power of two 2^e >= 2^-127 with max |new values in the page| <= 448 * 2^e,
 * and, when the page holds earlier tokens, at least the old scale. When the
 * scale grows the earlier codes are rescaled by the power of two and rounded
 * (exact but for e4m3 subnormals). Values are rounded from fp32 to the nearest
 * code, ties to even; a NaN gives the NaN code and an infinity +-448 (both are
 * left out of the maximum). Tokens whose position is negative or beyond the
 * table, or whose page is outside the pool, are not stored. Two sequences
 * may not append to the same page in one call.
 */
int attn_append(const gbattn_config* cfg, int32_t T, const gbattn_batch* batch, const gbattn_rows* q,
                const gbattn_rows* k, const gbattn_rows* v, const int32_t* positions, const uint64_t* table,
                const gbattn_cache* cache, const gbattn_rows* q_out, const gbattn_rows* k_out, void* stream);

/*
 * Attention over packed sequences: q, out [Tq, heads_q, D], k, v [Tk,
 * heads_kv, D], cu_q and cu_k [B+1] (equal for whole prompts; a sequence with
 * more keys than queries has its queries at the end). lse [Tq, heads_q] fp32
 * or NULL. bf16 with D up to 128 runs on the tensor cores (weights rounded to
 * bf16: off by 2^-8 of themselves), else on CUDA cores. out may not overlap
 * the inputs. (A query whose tile of up to 256 tokens and the keys they see,
 * rounded up to 128, holds a value that is no number at a key that this query
 * does not see takes 0.15 us for each of its own keys, up to 32 queries and
 * heads after each other.)
 */
int attn_prompt(const gbattn_config* cfg, int32_t Tq, int32_t Tk, int32_t B, const gbattn_rows* q,
                const gbattn_rows* k, const gbattn_rows* v, const int32_t* cu_q, const int32_t* cu_k,
                const gbattn_rows* out, float* lse, void* workspace, size_t workspace_bytes, void* stream);

/*
 * Attention of the batch's query tokens over their cached keys (the queries'
 * own keys already appended): q, out [T, heads_q, D], lse [T, heads_q] fp32 or
 * NULL. Meant for few query tokens per sequence (decoding, draft tokens); any
 * number works. Long contexts are split over CTAs and joined by a second
 * launch, deterministically. bf16 with D 64, 96 or 128 runs on the tensor
 * cores, else on CUDA cores. There the weights are rounded to bf16 (bf16 cache:
 * off by 2^-8 of themselves) or fp16 (e4m3: by 2^-11, or by 2^-34 of the row's
 * largest), and with an e4m3 cache the queries to fp16 relative to the largest
 * of their row (exact down to 2^-14 of it). A token whose page is outside the
 * pool is masked.
 * T * G and max_pages * page up to 2^30, else GBMOE_EUNSUPPORTED.
 */
int attn_cached(const gbattn_config* cfg, int32_t T, const gbattn_batch* batch, const gbattn_rows* q,
                const gbattn_cache* cache, const gbattn_rows* out, float* lse, void* workspace,
                size_t workspace_bytes, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* GBATTN_H */
