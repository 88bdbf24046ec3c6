/*
 * attention_cache.h -- a cache of keys and values in 4 bits, in the same
 * library as attention.h: tokens are quantised as they are written, read back
 * as rows, and attended to where they lie.
 *
 * The tokens of a sequence get their keys and values once and are read by
 * every later token; a run of one token at a time is bound by the bytes of
 * that cache.  Here a value takes 4.5 bits instead of 16.
 *
 * Stored form.  Up to 64 channels of a (token, head) are a group with two bf16
 * numbers, a step s and a least value m:
 *
 *     m = the least value x, rounded down (0, not -0)
 *     s = (the largest x - m) / 15, rounded to nearest; below 2^-126: 0
 *     code = (x - m) / s to the nearest whole number, ties to even, in 0 .. 15
 *            (0 where s = 0)
 *     value = m + s code
 *
 * where x - m, the largest x - m and the quotient by 15 are rounded to float32
 * and everything else is exact.  A group with a NaN or an infinity in it, or
 * whose s is not finite, has s = m = NaN and codes 0: it reads back as NaN.
 *
 * The cache is one array of bytes: pages x heads x blocks.  A block is 16
 * tokens of one head, GS_CACHE_BLOCK_BYTES(D, C) bytes:
 *
 *     16 rows of key codes      16 ceil(D / 32) bytes each
 *     16 rows of value codes    16 ceil(C / 32) bytes each
 *     16 rows of key groups     4 ceil(D / 64) bytes each: s, m per group
 *     16 rows of value groups   4 ceil(C / 64) bytes each
 *
 * A key row is four chunks t = 0 .. 3, each with one little-endian 32-bit word
 * per 32 channels j: channel 32 j + 8 t + p in bits 4 p .. 4 p + 3.  A value row
 * is eight chunks g = 0 .. 7, each with one 16-bit word per 32 channels j:
 * channel 32 j + 4 g + p in bits 4 p .. 4 p + 3.  (So a lane of a warp finds the
 * codes that it needs as operands of a matrix product in one run.)  Channels
 * past D or C have code 0.
 *
 * Conventions (those of attention.h where nothing else is said):
 *  - A page holds `tokens` tokens of every head, a multiple of 16.  Token n of
 *    problem b lies in page page_table[b, n / tokens] (int32 on the device), or
 *    without a table in page b.  N, the tokens a problem has room for, is
 *    tokens x table_pages, or tokens.
 *  - Problem b has k_lengths[b] tokens in the cache (clamped to 0 .. N), of which
 *    the calls concern the last q_lengths[b] (clamped to 0 .. M): row m of problem
 *    b is token m + k_length - q_length.  Rows m >= q_length are padding; rows of
 *    a token below 0 have no place.  So one pair of lengths serves a step:
 *    write the new tokens, then attend to all of them.
 *  - A table entry outside 0 .. pages - 1 is no page.  What is written there is
 *    dropped, what is read from there is NaN (in attention: the results of
 *    every query that sees such a token, and those of queries of the same head
 *    that it is hidden from may be NaN).  Entries past the tokens that
 *    k_lengths counts are not looked at, nor is anything else there.
 *  - The tokens that one call writes must lie in places of their own: no two
 *    problems may share the page that both write to.
 *  - D, C <= 256.  `data` must be on a 16-byte boundary and strides multiples of
 *    16 bytes.
 *  - Attention is computed in three ways, all with fp32 sums and maxima:
 *      codes as they are, for at most 16 rows a key head (M x H / heads; fp32 queries: any
 *        number): only probabilities times steps are rounded, to 11 bits (fp32: 22);
 *      tiles, for more rows of fp16 or bf16 queries, up to 512, up to as many as the card
 *        takes at once (room for at most 8192 tokens), or any number (room for at most 256
 *        tokens): keys are exact (steps down to 2^-9 of the largest of 128 tokens),
 *        probabilities and values rounded to fp16 numbers times a power of two, 11 bits;
 *      rows read back first, for the rest: keys are rounded to 11 bits too, which leaves the
 *        log-sum-exp of a row over n keys of normal size off by some 5e-4 / sqrt(n).
 *    Caches whose D or C is above 128, or (fp32) that have other numbers of 32-channel
 *    words for keys and for values, are read back in the queries' type (fp16: times a
 *    power of two of each head).
 *    Rows are read back for all tokens that there is room for at a time (workspace up to
 *    2 GiB), and tiles are split along the keys by that room: calls of more than 16 rows
 *    want no more columns of the page table than their longest sequence fills.
 *    Queries are good for magnitudes up to 2^115, keys and values up to 2^102.
 */
#ifndef GAUSS_SUM_ATTENTION_CACHE_H
#define GAUSS_SUM_ATTENTION_CACHE_H

#include "attention.h"

#ifdef __cplusplus
extern "C" {
#endif

#define GS_CACHE_BLOCK_TOKENS 16
#define GS_CACHE_ROW_BYTES(W) (((W) + 31) / 32 * 16)
#define GS_CACHE_GROUP_BYTES(W) (((W) + 63) / 64 * 4)
#define GS_CACHE_BLOCK_BYTES(D, C) \
    (16 * (GS_CACHE_ROW_BYTES(D) + GS_CACHE_ROW_BYTES(C) + GS_CACHE_GROUP_BYTES(D) + GS_CACHE_GROUP_BYTES(C)))

/* A cache and how its pages make up sequences.  Every member is 8 bytes wide. */
typedef struct gs_cache {
    void* data;
    int64_t stride_page, stride_head;   /* bytes; the blocks of a (page, head) are contiguous */
    int64_t pages, tokens, heads, D, C;
    const int32_t* page_table;          /* B x table_pages, rows stride_table apart; or NULL */
    int64_t table_pages, stride_table;
} gs_cache;

/* Rows of tokens, as 16-bit or 32-bit numbers: k (B, M, heads, D), v (B, M, heads, C). */
typedef struct gs_cache_rows {
    int64_t dtype;                      /* a gs_dtype */
    int64_t B, M;
    const int32_t* q_lengths;           /* B, or NULL: M */
    const int32_t* k_lengths;           /* B, or NULL: N */
    gs_array k, v;
} gs_cache_rows;

/* Queries on a cache. */
typedef struct gs_cached_attention {
    int64_t dtype;                      /* a gs_dtype: of q and out */
    int64_t B, M, H;                    /* H a multiple of the cache's heads */
    double tau;                         /* finite, > 0 */
    int64_t causal;                     /* 0 or 1 */
    const int32_t* q_lengths;           /* B, or NULL: M */
    const int32_t* k_lengths;           /* B, or NULL: N */
    gs_array q, out;                    /* (B, M, H, D), (B, M, H, C) */
    float* lse;                         /* B x H x M contiguous, or NULL */
} gs_cached_attention;

/* Quantises rows k and v into the cache. */
gs_status gauss_sum_cache_write(const gs_cache* c, const gs_cache_rows* r, void* stream);

/* Writes the values of tokens to rows k and v (data NULL: not wanted), rounded
 * once; zeros in padding and in rows without a place. */
gs_status gauss_sum_cache_read(const gs_cache* c, const gs_cache_rows* r, void* stream);

/*
 * Softmax attention and its log-sum-exp, as gauss_sum_attention, over the
 * values that the cache holds.
 */
gs_status gauss_sum_attention_cached(const gs_cached_attention* a, const gs_cache* c, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* GAUSS_SUM_ATTENTION_CACHE_H */
