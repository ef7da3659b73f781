/*
 * hgemm_routing.h -- routing of tokens to experts: choice, weights, expert order, gradient.
 *
 * For a token's logits l[0 .. experts-1] (fp32, fp16 or bf16; all arithmetic in fp32):
 *     s   = softmax(l)  or  1 / (1 + exp(-l))                         the scores
 *     v   = s + bias                                                  what the choice goes by (the bias balances the
 *                                                                     experts' load; it is not part of the weights);
 *                                                                     softmax without a bias: v = l, the same order
 *     groups > 1: experts come in `groups` equal consecutive groups; a group's value is its largest v, or the sum of
 *                 its two largest; only the `top_groups` best groups stay eligible
 *     indices = the top_k largest eligible v, largest first
 *     weights = scale * s[indices],  renormalize: scale * s[indices] / (sum of s[indices] + 1e-20)
 * Equal values go to the lowest index.  A NaN counts as -infinity; experts of other groups count as -infinity too.  A
 * token whose logits are all -infinity (softmax) has scores 0.
 *
 * Conventions are those of hgemm.h.  Nothing is allocated; every result is independent of scheduling.
 */
#ifndef HGEMM_ROUTING_H_
#define HGEMM_ROUTING_H_

#include "hgemm_fp8.h"

#ifdef __cplusplus
extern "C" {
#endif

enum { HGEMM_SCORE_SOFTMAX = 0, HGEMM_SCORE_SIGMOID = 1 };
enum { HGEMM_GROUP_MAX = 0, HGEMM_GROUP_TOP2 = 1 };

typedef struct {
    int32_t experts;      /* 1 .. 512 */
    int32_t top_k;        /* 1 .. 32, at most top_groups * experts / groups */
    int32_t score;        /* HGEMM_SCORE_* */
    int32_t groups;       /* 1 .. 32, divides experts */
    int32_t top_groups;   /* 1 .. groups */
    int32_t group_score;  /* HGEMM_GROUP_*; _TOP2 needs two experts in a group, and scores v = s (+ bias): not softmax without a bias */
    int32_t renormalize;  /* 0 or 1 */
    float scale;          /* finite */
} hgemm_routing_t;

/* tokens x experts logits with `ld` elements between rows; bias: experts fp32 values or NULL; weights (fp32) and indices
 * (int32): tokens x top_k, dense. */
hgemm_status_t hgemm_route(hgemm_ctx_t *ctx, const hgemm_routing_t *routing, int64_t tokens, const void *logits, int32_t type, int64_t ld, const float *bias,
                           float *weights, int32_t *indices, void *stream);

/* Gradient of the logits (same type; ldd elements between rows) from that of the weights (fp32, tokens x top_k).  The choice
 * itself is held fixed.  Every element of every row is written.  Indices outside 0 .. experts-1 are left out; a row's
 * indices are distinct. */
hgemm_status_t hgemm_route_backward(hgemm_ctx_t *ctx, const hgemm_routing_t *routing, int64_t tokens, const void *logits, int32_t type, int64_t ld,
                                    const int32_t *indices, const float *dweights, void *dlogits, int64_t ldd, void *stream);

/* Expert order of `count` choices (tokens x top_k indices, flat; count <= 2^26, experts <= 1024): offsets (experts + 1): first place of each expert;
 * order[place] = flat number of the choice there; position[choice] = its place.  Stable: an expert's choices keep their
 * order.  Choices with an index outside 0 .. experts-1 have position -1 and no place; places from offsets[experts]
 * on hold -1. */
hgemm_status_t hgemm_route_sort(hgemm_ctx_t *ctx, const int32_t *indices, int64_t count, int32_t experts, int32_t *offsets, int32_t *order, int32_t *position,
                                void *stream);

#ifdef __cplusplus
}
#endif

#endif /* HGEMM_ROUTING_H_ */
