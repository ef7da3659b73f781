/*
 * hgemm_few_tokens.h -- a layer of experts for the few tokens of a decoding step.
 *
 *     h[t,j] = act(W1[e] x[t])            e = indices[t,j]:  the experts that token t's router chose (hgemm_route)
 *     y[t]   = sum over j of  weights[t,j] * (W2[e] h[t,j])
 *
 * with act(u) = u / (1 + exp(-u)) (SILU; W1[e] has `inner` rows), or act(g, u) = g / (1 + exp(-g)) * u (SWIGLU; W1[e] has 2 * inner rows, those of g first).
 * W1 is experts x (inner or 2 * inner) x hidden, W2 is experts x hidden x inner.  Only the chosen experts' weights are read, each once for up to 8 of its
 * choices.  Weights are fp16 or bf16, of x's type, or 4-bit row copies with block scales (hgemm_fp4.h) with x of either type.
 *
 * All sums are in fp32, and the result is rounded once; a token's choices are added up in their order, so that results do not depend on scheduling.
 *     16-bit weights    two launches; x and the weights enter the products as they are, h to 16 bits of mantissa (against fp16 weights too: the products of both second parts, 2^-16
 *                       of the whole, are left out).  An infinity in x or in a weight makes the results that it reaches infinite or NaN
 *     4-bit weights     five launches; the weights enter the products as they are, x and h as sums of 4-bit digits: off by at most 2^-19 (NVFP4) or 2^-22 (MXFP4) of the token's
 *                       (the choice's) largest magnitude, or by 2^-127 where that is more.  With NVFP4 small elements beside a large one keep fewer bits: e4m3 scales
 *                       end at 2^-9; MXFP4's lose no more than 2^-22 of their block's largest.  A NaN or an infinity in x makes its token's results NaN
 *
 * Choices with an index outside [0, experts) count as zero.  A token may choose an expert twice.
 *
 * Conventions are those of hgemm.h: status codes, device pointers, everything asynchronous on the caller's stream, nothing allocated or
 * synchronised, the context's device current.  The scratch memory belongs to one call at a time: calls that may overlap (on several streams, or in
 * graphs that may run at once) take one each.
 */
#ifndef HGEMM_FEW_TOKENS_H_
#define HGEMM_FEW_TOKENS_H_

#include "hgemm_fp4.h"

#ifdef __cplusplus
extern "C" {
#endif

enum { HGEMM_ACT_SILU = 0, HGEMM_ACT_SWIGLU = 1 };
enum { HGEMM_WEIGHTS_F16 = 1, HGEMM_WEIGHTS_BF16 = 2, HGEMM_WEIGHTS_NVFP4 = 16, HGEMM_WEIGHTS_MXFP4 = 17 };

typedef struct {
    int32_t hidden, inner;     /* 1 .. 2^20 each */
    int32_t experts;           /* 1 .. 1024 */
    int32_t top_k;             /* 1 .. 32 */
    int32_t weights;           /* HGEMM_WEIGHTS_* */
    int32_t activation;        /* HGEMM_ACT_* */
    int32_t type;              /* of x and y: HGEMM_TYPE_F16, _BF16; the weights' own type where they have 16 bits */
    int32_t reserved;
} hgemm_few_tokens_t;

/* One matrix for each expert, one after the other. */
typedef struct {
    const void *values;        /* 16-bit: ld elements between rows, any ld >= the row's length (rows at multiples of 16 bytes are faster); 4-bit: ld bytes, a multiple of 16 */
    int64_t ld;
    const void *scales;        /* 4-bit: the scale tiles; 16-bit: NULL */
    const float *factor;       /* NV: one for each expert; else NULL */
} hgemm_expert_weights_t;

enum { HGEMM_FEW_TOKENS_MAX = 64 };

/* Bytes of scratch memory for up to `tokens` tokens (16-byte aligned); -1 if the description or the number (0 .. 64) is not legal. */
int64_t hgemm_few_tokens_scratch(const hgemm_few_tokens_t *layer, int64_t tokens);

/* tokens: 0 .. 64.  x: tokens x hidden, ldx elements between rows; y likewise; indices (int32), weights (fp32): tokens x top_k, dense. */
hgemm_status_t hgemm_few_tokens(hgemm_ctx_t *ctx, const hgemm_few_tokens_t *layer, int64_t tokens, const void *x, int64_t ldx, const hgemm_expert_weights_t *w1,
                                const hgemm_expert_weights_t *w2, const int32_t *indices, const float *weights, void *y, int64_t ldy, void *scratch, int64_t scratch_bytes, void *stream);

#ifdef __cplusplus
}
#endif

#endif /* HGEMM_FEW_TOKENS_H_ */
