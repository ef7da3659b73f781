/*
 * hgemm_fp4.h -- 4-bit products with block scales, for a linear layer or one layer per expert; their quantiser.
 *
 * A 4-bit value (e2m1) is 0, 0.5, 1, 1.5, 2, 3, 4 or 6, or the negative of one.  Two formats give it a range:
 *
 *     NV    blocks of 16 elements with an e4m3 scale each, and one fp32 factor for the whole tensor (for each matrix of a stack)
 *     MX    blocks of 32 elements with a power of two each (e8m0: 2^(byte - 127)); no factor
 *
 * A layer has a weight W of N outputs x K inputs; M rows (tokens) go through it.  The blocks lie along the contracted dimension, so each matrix is
 * needed in a ROW copy (blocks along its rows) or in a COLUMN copy (the transposed matrix, blocks along its columns):
 *
 *     forward       Y  (M x N) = X  (M x K) . W^T       X: row copy (M x K)        W: row copy (N x K)
 *     input grad    dX (M x K) = dY (M x N) . W         dY: row copy (M x N)       W: column copy (K x N)
 *     weight grad   dW (N x K) = dY^T . X               dY: column copy (N x M)    X: column copy (K x M)
 *
 * Each result is  factorA * factorB * sum over the contraction of  scaleA * A * scaleB * B, summed in fp32, rounded once to the result's type.
 *
 * Layouts (device memory)
 *   - Values: two to a byte, the first in the low half; ceil(cols / 2) bytes a row, rows `ld` BYTES apart (a multiple of 16), 16-byte aligned base.  The
 *     second value of an odd row's last byte is 0.  Bytes between a row's end and ld are never read as values or written.
 *   - Scales: tiles of 128 rows x 4 blocks, 512 bytes each.  The scale of row r, block b is byte 16 (r % 32) + 4 (r % 128 / 32) + b % 4 of tile
 *     (r / 128, b / 4); the tiles of 128 rows follow one another (ceil(blocks / 4) of them), then those of the next 128 rows.  Scales of rows and
 *     blocks that the matrix does not have are 0.  16-byte aligned.  hgemm_fp4_scale_bytes() says how many bytes a matrix has.
 *   - Stacks (one weight per expert): dense matrices one after the other with `ld` between rows, their scale tiles one matrix after the other.
 *   - Results: fp32, fp16 or bf16, row-major with any ld (elements) >= their width; 16-byte aligned bases and rows are faster.
 *
 * Products over experts (groups >= 1): the M rows are sorted by group, rows offsets[g] .. offsets[g+1]-1 belong to group g (int32, groups + 1 values
 * on the DEVICE, non-decreasing, offsets[0] = 0, offsets[groups] <= M; values outside [0, M] are clamped, and one that is smaller than one before it
 * counts as that one, here and in the quantiser).  A group's scale tiles start at a tile of their own: the scales of its row i are those of "row"
 * 128 * sum_{h < g} ceil(count_h / 128) + i, in hgemm_fp8_padded_rows(M, groups) rows of them.  Its column copy starts at the same "row" of
 * hgemm_fp8_padded_rows(M, groups) contracted elements; those up to the next multiple of 128 are zero, with scales of zero.  A group without rows is
 * legal (its weight gradient is zeros); result rows of no group are not written.
 *
 * Conventions are those of hgemm.h: status codes, device pointers, everything asynchronous on the caller's stream, nothing allocated or
 * synchronised by a run, the context's device current.  A plan holds no device memory and may be run on several streams at once.  Sizes: 0 <= M <= 2^22
 * (0 rows: nothing to do, the weight gradient is zeros), 1 <= N, K <= 2^22, groups <= 1024.
 */
#ifndef HGEMM_FP4_H_
#define HGEMM_FP4_H_

#include "hgemm_fp8.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef struct hgemm_fp4_plan_s hgemm_fp4_plan_t; /* opaque; owned by its context */

enum { HGEMM_FP4_NV = 0, HGEMM_FP4_MX = 1 };
enum { HGEMM_FP4_ROWS = 1, HGEMM_FP4_COLS = 2 };

/* Bytes of the scale tiles of `rows` x `cols` values (one matrix); -1 if a size or the format is not legal. */
int64_t hgemm_fp4_scale_bytes(int64_t rows, int64_t cols, int32_t format);

/* factor[i] (fp32) of each of `matrices` matrices of rows x cols (one after the other, ldx between rows): the smallest power of two that is at least
 * max |x| / 2688 over its finite elements (2688 = 6 * 448: the largest value times the largest scale); 0 where that maximum is 0. */
hgemm_status_t hgemm_fp4_tensor_factor(hgemm_ctx_t *ctx, int32_t x_type, int64_t matrices, int64_t rows, int64_t cols, const void *x, int64_t ldx, float *factor,
                                       void *stream);

/* What hgemm_fp4_quantize reads and writes.  For every block, with a = max |x| over it, everything in fp32 and to nearest even:
 *     NV:  scale = e4m3(a * (1 / factor) * (1 / 6)), at most 448;   value = e2m1(x / (scale * factor)), at most 6
 *          (scale 0: values 0; a factor below 2^-100 counts as 0: all scales 0)
 *     MX:  scale = the smallest power of two with a <= 6 * scale (at least 2^-127);   value = e2m1(x / scale)
 * A block with a NaN or an infinity has the scale NaN (its values mean nothing). */
typedef struct {
    int32_t blocks;            /* HGEMM_FP4_ROWS, _COLS, or both of them (one pass over x) */
    int32_t x_type;            /* HGEMM_TYPE_F32, _F16, _BF16 */
    int32_t format;            /* HGEMM_FP4_NV, _MX */
    int32_t matrices;          /* 1, or a stack's number (<= 1024; no row_index, no offsets) */
    int64_t rows, cols;        /* of one matrix to quantise */
    int64_t ldx;               /* elements between rows of x */
    const void *x;
    const int32_t *row_index;  /* NULL, or `rows` numbers: row r of the result is row row_index[r] of x, zeros if that is outside [0, x_rows) */
    int64_t x_rows;            /* rows of x (row_index only); 0: x may be NULL */
    const int32_t *offsets;    /* NULL, or the groups + 1 offsets: scale tiles and column copy per group.  Rows of no group are not written */
    int32_t groups;            /* with offsets: their groups; else 0 */
    int32_t reserved;
    const float *factor;       /* NV: one for each matrix, on the device; MX: NULL */
    void *q;                   /* row copy */
    int64_t ldq;               /* bytes */
    void *scales;
    void *q_cols;              /* column copy: cols rows of `rows` (or hgemm_fp8_padded_rows(rows, groups)) values */
    int64_t ldq_cols;          /* bytes */
    void *scales_cols;
} hgemm_fp4_quantize_t;

hgemm_status_t hgemm_fp4_quantize(hgemm_ctx_t *ctx, const hgemm_fp4_quantize_t *desc, void *stream);

/* out (fp32, fp16 or bf16; ldo elements between rows) = what rows x cols values stand for: value * (scale * factor) in fp32, rounded to out's type.  offsets:
 * as in the quantiser, for a row copy with scale tiles per group (rows of no group are not written). */
hgemm_status_t hgemm_fp4_dequantize(hgemm_ctx_t *ctx, int32_t format, int32_t out_type, int64_t matrices, int64_t rows, int64_t cols, const void *q, int64_t ldq, const void *scales,
                                    const float *factor, const int32_t *offsets, int32_t groups, void *out, int64_t ldo, void *stream);

/* A plan for one layer's product (form: HGEMM_FP8_FORWARD, _INPUT_GRAD, _WEIGHT_GRAD).  groups = 0: one weight; >= 1: one per group. */
hgemm_status_t hgemm_fp4_plan(hgemm_ctx_t *ctx, int32_t form, int64_t M, int64_t N, int64_t K, int32_t groups, int32_t format, int32_t out_type, hgemm_fp4_plan_t **out);
hgemm_status_t hgemm_fp4_plan_destroy(hgemm_fp4_plan_t *plan);

/* One product.  A is X (forward) or dY, B is W (forward, input grad) or X (weight grad), each in the copy that the form takes; lda, ldb in bytes, ldc in
 * elements.  a_factor, b_factor (device; MX: NULL): one value each, b_factor one per group where B is a stack.  accumulate != 0 (fp32 results only):
 * C += the product, where C has values of its own.  offsets: NULL exactly if the plan has no groups. */
hgemm_status_t hgemm_fp4_run(hgemm_fp4_plan_t *plan, const void *A, int64_t lda, const void *a_scales, const float *a_factor, const void *B, int64_t ldb, const void *b_scales,
                             const float *b_factor, void *C, int64_t ldc, const int32_t *offsets, int32_t accumulate, void *stream);

/* As hgemm_last_device_status, for this plan: whether a bounded wait of its launches ran out.  A plan may be destroyed while its
 * launches are under way; what they report then shows in hgemm_ctx_last_device_status. */
hgemm_status_t hgemm_fp4_last_device_status(hgemm_fp4_plan_t *plan, uint32_t *code);
/* Test hook: hgemm_debug_timeout_probe, reporting to this plan's status word. */
hgemm_status_t hgemm_fp4_debug_timeout_probe(hgemm_fp4_plan_t *plan, void *stream);

/* How a plan runs; as hgemm_fp8_config_t, with other tiles. */
typedef struct {
    int32_t cta_group;         /* 2: CTA pairs, tiles of 256 x block_q; 1: one CTA, tiles of 128 x block_q with the operands swapped */
    int32_t block_q;           /* 256 or 128 (pairs); 128 or 64 (one CTA) */
    int32_t split_k;           /* 1, 2, 4 or 8 CTAs of a cluster share the contraction (one CTA only) */
    int32_t reserved;
} hgemm_fp4_config_t;

hgemm_status_t hgemm_fp4_plan_get_config(const hgemm_fp4_plan_t *plan, hgemm_fp4_config_t *out);
hgemm_status_t hgemm_fp4_plan_set_config(hgemm_fp4_plan_t *plan, const hgemm_fp4_config_t *cfg);
/* What the planner would choose for 16-bit results (host only). */
hgemm_status_t hgemm_fp4_planned_config(int32_t form, int64_t M, int64_t N, int64_t K, int32_t groups, int32_t num_sms, hgemm_fp4_config_t *out);

#ifdef __cplusplus
}
#endif

#endif /* HGEMM_FP4_H_ */
