/*
 * attention.h -- softmax attention, its vector-Jacobian product and rotary
 * positions, in the same library as gauss_sum.h.
 *
 * The Gauss sum of Eq. 1 is softmax attention without its normalisation: with
 *
 *     lse_m = log sum_n exp(tau q_m . k_n),
 *     out_m = sum_n exp(tau q_m . k_n - lse_m) v_n,
 *
 * and values scaled by exp(-tau/2 ||k_n||^2), s_m = out_m exp(lse_m)
 * exp(-tau/2 ||q_m||^2) (Alg. 1).  The entry points here evaluate out and
 * lse for batches of heads, the gradients of both, and the rotation of
 * queries and keys by their positions that precedes them in a network.
 *
 * Conventions (those of gauss_sum.h where nothing else is said):
 *  - Arrays are 4-D, (B, rows, heads, width): problem, token, head, channel.
 *    The channels of one (problem, token, head) are contiguous; the other
 *    three strides are free (in elements, >= 0), so both (B, rows, heads, .)
 *    and (B, heads, rows, .) storage, slices and broadcast inputs are
 *    passed as they are.  Outputs must not overlap themselves or the inputs.
 *  - q has H heads, k and v have Hk, H a multiple of Hk: query head h reads
 *    key head h / (H / Hk).  D channels in q and k, C in v and out.
 *  - Inputs and outputs have one element type (dtype); lse, g_lse and all
 *    arithmetic are float32.  Each output is rounded once, at the end;
 *    for fp16 / bf16 the probabilities (and their gradients) are also
 *    rounded to that type as operands of the tensor-core products.
 *    fp16 gradients keep that type's precision for p (g . v - delta) down to
 *    2^-29 of the largest |g||v| + |delta| among the pairs that the masks
 *    leave of the same query (grad_q) or of the same key (grad_k), and are
 *    rounded to multiples of 2^-38 of it below.
 *  - Sizes: D, C <= 256, M, N < 2^31 / (H / Hk).  Base pointers need the
 *    alignment of one element.  fp16 / bf16 arrays with D, C <= 128 whose
 *    base addresses and strides are multiples of 16 bytes run on the tensor
 *    cores; everything else runs on the fp32 pipe with the same results up
 *    to rounding, at 12 to 20 TFLOP/s against several hundred.
 *  - Masks.  Problem b has q_lengths[b] queries and k_lengths[b] keys (device
 *    arrays of B int32, NULL: M and N; values are clamped to 0..M, 0..N).
 *    Rows past a length are padding: they are never part of any result,
 *    whatever they hold (NaN included).  causal != 0: query m sees the keys
 *    n <= m + k_length - q_length (the last query sees every key).  Among
 *    the keys inside the length, a non-finite one that the causal mask hides
 *    from some queries may make their results NaN too.
 *  - A query that sees no key, and a padding query, has out = 0,
 *    lse = -infinity and zero gradients; padding keys have zero gradients.
 *  - Results are the same from call to call (no atomic additions).
 *  - Workspaces are allocated on `stream` from the library's pool, as for
 *    gauss_sum.
 */
#ifndef GAUSS_SUM_ATTENTION_H
#define GAUSS_SUM_ATTENTION_H

#include "gauss_sum.h"

#ifdef __cplusplus
extern "C" {
#endif

/* A (B, rows, heads, width) array; strides in elements, width contiguous. */
typedef struct gs_array {
    void* data;
    int64_t stride_b, stride_row, stride_head;
} gs_array;

/* One attention problem batch.  Every member is 8 bytes wide. */
typedef struct gs_attention {
    int64_t dtype;                    /* a gs_dtype */
    int64_t B, M, N, H, Hk, D, C;
    double tau;                       /* finite, > 0 */
    int64_t causal;                   /* 0 or 1 */
    const int32_t* q_lengths;         /* B, or NULL */
    const int32_t* k_lengths;         /* B, or NULL */
    gs_array q, k, v, out;            /* out: written by the forward call, read by the VJP */
    float* lse;                       /* B x H x M contiguous; forward: may be NULL */
} gs_attention;

/* Upstream gradients and outputs of the vector-Jacobian product. */
typedef struct gs_attention_grad {
    gs_array g;                       /* dL/dout, like out */
    const float* g_lse;               /* dL/dlse, B x H x M contiguous, or NULL (zero) */
    gs_array grad_q, grad_k, grad_v;  /* like q, k, v; data NULL: not wanted */
} gs_attention_grad;

/* out and lse. */
gs_status gauss_sum_attention(const gs_attention* a, void* stream);

/*
 * Gradients of L with respect to q, k and v, given out and lse of the
 * forward call (the probabilities are recomputed from lse):
 *
 *     p_mn   = exp(tau q_m . k_n - lse_m)
 *     ds_mn  = p_mn (g_m . v_n - g_m . out_m + g_lse_m)
 *     grad_q[m] = tau sum_n ds_mn k_n
 *     grad_k[n] = tau sum_m ds_mn q_m       (sums over the query heads that
 *     grad_v[n] =     sum_m p_mn  g_m        share the key head as well)
 *
 * g_m . out_m carries the rounding of a 16-bit out, except in rows of at most
 * 24 keys, which sum it over their keys.
 */
gs_status gauss_sum_attention_vjp(const gs_attention* a, const gs_attention_grad* d,
                                  void* stream);

/*
 * Rotary positions of q (B, M, H, D) and, in the same launch, k (B, M, Hk, D;
 * k.data NULL: none): the first R channels of every head are R/2 pairs, pair
 * i being channels (i, i + R/2), or (2i, 2i + 1) with interleaved; token m of
 * problem b turns pair i by positions[b, m] x frequency i:
 *
 *     (y_a, y_b) = scale (x_a cos - x_b sin, x_a sin + x_b cos),
 *
 * and channels R .. D - 1 are copied.  transpose != 0 turns by the negative
 * angle with the same scale: the gradient of the rotation.  A frequency is a
 * fraction of a turn per position in units of 2^-64 turns (int64, modulo
 * 2^64), so that position x frequency, a wrapping integer product, is the
 * exact angle modulo one turn at any position.  Outputs may be the inputs
 * themselves (same data and strides), not otherwise overlap them.
 */
typedef struct gs_rotary {
    int64_t dtype;                    /* a gs_dtype */
    int64_t B, M, H, Hk, D, R;        /* R even, 0 <= R <= D, R <= 4096; Hk ignored without k */
    double scale;                     /* finite */
    int64_t interleaved, transpose;   /* 0 or 1 each */
    const void* positions;            /* int32 or int64, by strides */
    int64_t positions_64;             /* 1: int64, 0: int32 */
    int64_t stride_pos_b, stride_pos_m;
    const int64_t* frequencies;       /* R / 2, contiguous */
    gs_array q, k, q_out, k_out;
} gs_rotary;

gs_status gauss_sum_rotary(const gs_rotary* a, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* GAUSS_SUM_ATTENTION_H */
