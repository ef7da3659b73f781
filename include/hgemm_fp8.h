/*
 * hgemm_fp8.h -- 8-bit products with one fp32 scale per block of 128, for a linear layer or one layer per expert.
 *
 * A layer has a weight W of N outputs x K inputs; M rows (tokens) go through it.  The three products of a
 * training step, on 8-bit operands (e4m3 or e5m2) with scales:
 *
 *     forward       Y  (M x N) = X  (M x K) . W^T       X, dY: one scale per 1 x 128 block of a row
 *     input grad    dX (M x K) = dY (M x N) . W         W:     one scale per 128 x 128 tile (the same W for both)
 *     weight grad   dW (N x K) = dY^T . X               dY, X: one scale per 128 x 1 block of a column
 *
 * Each result is  sum over blocks b of 128 along the contracted dimension of
 *     scaleP[i][b] * scaleQ[j][b] * sum_{k in b} P[i][k] * Q[j][k]
 * with both sums in fp32 and one rounding to the result's type.  Operands stay as they are stored: the kernels read
 * the contracted dimension down the columns where a product needs it (no transposed copies).
 *
 * Layouts (device memory)
 *   - 8-bit matrices are row-major; the distance between rows (ld, in elements) is a multiple of 16 and the base is
 *     16-byte aligned.  Columns between the matrix's width and ld are never read as values or written.
 *   - Row scales: rows x ceil(cols/128) fp32.  Column scales: ceil(rows/128) x cols.  Tile scales: ceil(rows/128) x
 *     ceil(cols/128) per matrix.  Dense, 4-byte aligned.
 *   - Results: fp32, fp16 or bf16, row-major with any ld >= their width; 16-byte aligned bases and rows are faster.
 *
 * Products over experts (groups >= 1): the M rows are sorted by group, rows offsets[g] .. offsets[g+1]-1 belong to
 * group g (int32, groups + 1 values on the DEVICE, non-decreasing, offsets[0] = 0, offsets[groups] <= M; values outside
 * [0, M] are clamped, and one that is smaller than one before it counts as that one, here and in the quantiser).  W and
 * its scales are groups x N x K, dense matrices one after the other with `ld` between rows.  A group without rows is legal; rows from offsets[groups] on are not written.  For the weight gradient (result groups x N x K, zeros for an
 * empty group) the operands are the column-quantised copies that hgemm_fp8_quantize makes when it is given the
 * offsets: group g's rows start at row 128 * sum_{h < g} ceil(count_h / 128) of the copy, the rows up to the next
 * multiple of 128 are zero, and the copy has hgemm_fp8_padded_rows(M, groups) rows.
 *
 * Conventions are those of hgemm.h: status codes, device pointers, everything asynchronous on the caller's stream,
 * nothing allocated or synchronised by a run, the context's device current.  A plan holds no device memory and may be
 * run on several streams at once.  Sizes: 0 <= M <= 2^22 (0 rows: nothing to do, the weight gradient is zeros),
 * 1 <= N, K <= 2^22, groups <= 1024.
 */
#ifndef HGEMM_FP8_H_
#define HGEMM_FP8_H_

#include "hgemm.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef struct hgemm_fp8_plan_s hgemm_fp8_plan_t; /* opaque; owned by its context */

enum { HGEMM_TYPE_F32 = 0, HGEMM_TYPE_F16 = 1, HGEMM_TYPE_BF16 = 2, HGEMM_TYPE_E4M3 = 3, HGEMM_TYPE_E5M2 = 4 };
enum { HGEMM_FP8_FORWARD = 0, HGEMM_FP8_INPUT_GRAD = 1, HGEMM_FP8_WEIGHT_GRAD = 2 };
enum { HGEMM_FP8_ROWS = 1, HGEMM_FP8_COLS = 2, HGEMM_FP8_TILES = 4 };

/* What hgemm_fp8_quantize reads and writes.  For every block with a = max |x| over its finite elements:
 *     a <  2^-100:  scale = 1, values 0
 *     otherwise:    scale = a / m, value = round(x * (m / a)), m the type's largest value (448 or 57344);
 *                   pow2: scale = the smallest power of two >= a / m, value = round(x / scale)
 * to nearest even, clamped to +-m.  NaN and infinities become NaN (and only they). */
typedef struct {
    int32_t blocks;            /* HGEMM_FP8_ROWS, _COLS, both of them (one pass over x), or _TILES */
    int32_t x_type;            /* HGEMM_TYPE_F32, _F16, _BF16 */
    int32_t q_type;            /* HGEMM_TYPE_E4M3, _E5M2 */
    int32_t pow2;              /* 0 or 1 */
    int64_t rows, cols;        /* of the quantised matrix (of one matrix, for _TILES) */
    int64_t ldx;               /* elements between rows of x */
    const void *x;
    const int32_t *row_index;  /* NULL, or `rows` numbers: row r of the result is row row_index[r] of x, zeros if that is outside [0, x_rows) (not for _TILES) */
    int64_t x_rows;            /* rows of x (row_index only); 0: x may be NULL */
    const int32_t *offsets;    /* NULL, or the groups + 1 offsets: the column-quantised copy is laid out per group (_COLS; what lies behind its last
                                  group is not written).  A row copy made in the same pass has every row, those of no group too */
    int32_t groups;            /* with offsets: their groups; for _TILES: the number of matrices (x holds groups * rows rows); else 0 */
    int32_t reserved;
    void *q;                   /* row- or tile-quantised values */
    int64_t ldq;
    float *scales;             /* row or tile scales */
    void *q_cols;              /* column-quantised values (rows, or hgemm_fp8_padded_rows(rows, groups) rows) */
    int64_t ldq_cols;
    float *scales_cols;
} hgemm_fp8_quantize_t;

hgemm_status_t hgemm_fp8_quantize(hgemm_ctx_t *ctx, const hgemm_fp8_quantize_t *desc, void *stream);

/* Rows of a column-quantised copy laid out per group: an upper bound that depends on M and groups alone. */
int64_t hgemm_fp8_padded_rows(int64_t M, int32_t groups);

/* A plan for one layer's product.  groups = 0: one weight; >= 1: one per group.  a_type is the type of X or dY,
 * b_type that of W (of X for the weight gradient). */
hgemm_status_t hgemm_fp8_plan(hgemm_ctx_t *ctx, int32_t form, int64_t M, int64_t N, int64_t K, int32_t groups, int32_t a_type, int32_t b_type,
                              int32_t out_type, hgemm_fp8_plan_t **out);
hgemm_status_t hgemm_fp8_plan_destroy(hgemm_fp8_plan_t *plan);

/* One product.  A is X (forward) or dY, B is W (forward, input grad) or X (weight grad); lda, ldb, ldc in elements.
 * accumulate != 0 (fp32 results only): C += the product, where C has values of its own.  offsets: NULL exactly if the
 * plan has no groups. */
hgemm_status_t hgemm_fp8_run(hgemm_fp8_plan_t *plan, const void *A, int64_t lda, const float *a_scales, const void *B, int64_t ldb,
                             const float *b_scales, void *C, int64_t ldc, const int32_t *offsets, int32_t accumulate, void *stream);

/* As hgemm_last_device_status, for this plan: whether a bounded wait of its launches ran out.  A plan may be destroyed while its
 * launches are under way; what they report then shows in hgemm_ctx_last_device_status. */
hgemm_status_t hgemm_fp8_last_device_status(hgemm_fp8_plan_t *plan, uint32_t *code);
/* Test hook: hgemm_debug_timeout_probe, reporting to this plan's status word. */
hgemm_status_t hgemm_fp8_debug_timeout_probe(hgemm_fp8_plan_t *plan, void *stream);

/* How a plan runs: CTAs per tile (which also says whether the kernel's operands are swapped), the tile's extent along the
 * kernel's second operand, and the CTAs that share one tile's contraction.  hgemm_fp8_plan_set_config takes what
 * hgemm_fp8_plan_get_config gives, or another combination that the plan's product has kernels for (HGEMM_ERR_UNSUPPORTED
 * otherwise). */
typedef struct {
    int32_t cta_group;         /* 2: CTA pairs, tiles of 256 x 256; 1: one CTA, tiles of 128 x block_q with the operands swapped */
    int32_t block_q;           /* 256 (pairs); 16, 32, 64 or 128 (one CTA; 128 only for the weight gradient) */
    int32_t split_k;           /* 1, 2, 4 or 8 CTAs of a cluster share the contraction (one CTA only) */
    int32_t reserved;
} hgemm_fp8_config_t;

hgemm_status_t hgemm_fp8_plan_get_config(const hgemm_fp8_plan_t *plan, hgemm_fp8_config_t *out);
hgemm_status_t hgemm_fp8_plan_set_config(hgemm_fp8_plan_t *plan, const hgemm_fp8_config_t *cfg);
/* What the planner would choose (host only). */
hgemm_status_t hgemm_fp8_planned_config(int32_t form, int64_t M, int64_t N, int64_t K, int32_t groups, int32_t num_sms, hgemm_fp8_config_t *out);

#ifdef __cplusplus
}
#endif

#endif /* HGEMM_FP8_H_ */
