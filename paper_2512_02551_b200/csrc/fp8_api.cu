// C ABI of the 8-bit products with block scales (see include/hgemm_fp8.h): quantisation, plans, launches.
#include <cuda.h>
#include <cuda_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstring>
#include <new>

#include "../../include/hgemm_fp8.h"
#include "fp8_product_kernel.cuh"
#include "fp8_quantize_kernel.cuh"
#include "hgemm_context.h"

using hgemm_dev::Fp8Params;

struct hgemm_fp8_plan_s {
    hgemm_ctx_s *ctx = nullptr;
    int32_t form = 0;
    int64_t M = 0, N = 0, K = 0;
    int32_t groups = 0, a_type = 0, b_type = 0, out_type = 0;
    hgemm_fp8_config_t cfg{};
    int status_slot = 0;
};

namespace {

constexpr int64_t kMaxDim = int64_t(1) << 22;
constexpr int kSmemOptIn = 232448;

int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

bool is_fp8(int32_t t) { return t == HGEMM_TYPE_E4M3 || t == HGEMM_TYPE_E5M2; }
bool is_wide(int32_t t) { return t == HGEMM_TYPE_F32 || t == HGEMM_TYPE_F16 || t == HGEMM_TYPE_BF16; }
int type_bytes(int32_t t) { return t == HGEMM_TYPE_F32 ? 4 : t == HGEMM_TYPE_F16 || t == HGEMM_TYPE_BF16 ? 2 : 1; }

bool legal_shape(int32_t form, int64_t M, int64_t N, int64_t K, int32_t groups)
{
    return form >= HGEMM_FP8_FORWARD && form <= HGEMM_FP8_WEIGHT_GRAD && M >= 0 && M <= kMaxDim && N >= 1 && N <= kMaxDim && K >= 1 && K <= kMaxDim &&
           groups >= 0 && groups <= hgemm_dev::kFp8MaxGroups;
}

bool legal_config(int32_t form, const hgemm_fp8_config_t &c)
{
    if (c.cta_group == 2) return c.block_q == 256 && c.split_k == 1;
    if (c.cta_group != 1) return false;
    if (c.split_k != 1 && c.split_k != 2 && c.split_k != 4 && c.split_k != 8) return false;
    if (form == HGEMM_FP8_WEIGHT_GRAD) return c.block_q == 128;
    return c.block_q == 16 || c.block_q == 32 || c.block_q == 64 || c.block_q == 128;
}

// Tiles of a configuration, over all groups (for groups that follow offsets on the device: at most).
int64_t tiles_of(int32_t form, int64_t M, int64_t N, int64_t K, int32_t groups, const hgemm_fp8_config_t &c)
{
    const int64_t outs = form == HGEMM_FP8_FORWARD ? N : K;                   // columns of the result
    const int64_t bt = c.cta_group == 2 ? 256 : c.block_q, bo = c.cta_group == 2 ? 256 : 128;
    if (form == HGEMM_FP8_WEIGHT_GRAD) return std::max(groups, 1) * ceil_div(N, c.cta_group == 2 ? 256 : 128) * ceil_div(K, c.cta_group == 2 ? 256 : 128);
    if (groups == 0) return ceil_div(M, bt) * ceil_div(outs, bo);
    return (std::min<int64_t>(groups, M) + M / bt) * ceil_div(outs, bo);
}

// Estimated time of a configuration in microseconds: a start-up, then rounds of tiles over the SMs, each block of 128 of a tile's contraction
// and each tile's end at their measured cost (B200, operands in L2).  One block of a pair's 256 x 256 tile takes 0.46 us (0.56
// with a scale per column), of a single CTA's 128 x {16, 32, 64, 128} tile 0.16, 0.20, 0.27, 0.45 us
// (0.62 with most SMs busy: operands from L2); sharing a contraction costs about 1 us
// for two CTAs and 1.7 us for eight.  512 x 4096 x 4096: pairs 21.5 us, 128-row tiles 24.9 us; 256 x 4096 x 4096: 20.5 and 16.4 us
// (two CTAs a tile); 64 x 4096 x 4096: one CTA a tile 13.8 us, four 9.9 us.
double estimate_us(int32_t form, int64_t M, int64_t N, int64_t K, int32_t groups, int32_t num_sms, const hgemm_fp8_config_t &c)
{
    const bool wgrad = form == HGEMM_FP8_WEIGHT_GRAD, pair = c.cta_group == 2;
    const int64_t outs = form == HGEMM_FP8_FORWARD ? N : K;
    const double rows = groups > 0 ? double(M) / groups : double(M);           // rows of one group, on average
    double tiles, blocks;
    if (wgrad) {
        tiles = double(tiles_of(form, M, N, K, groups, c));
        blocks = std::ceil(rows / 128.0) + (groups > 0 && rows > 128.0 ? 0.5 : 0.0);
    } else {
        const int64_t bt = pair ? 256 : c.block_q, bo = pair ? 256 : 128;
        // groups are uneven: each ends in a partly filled tile
        const double of_rows = groups > 0 ? std::min<double>(groups, double(M)) * std::max(1.0, rows / double(bt) + 0.7) : double(ceil_div(M, bt));
        tiles = of_rows * double(ceil_div(outs, bo));
        blocks = double(ceil_div(form == HGEMM_FP8_FORWARD ? K : N, 128));
    }
    const double block_us = pair ? (wgrad ? 0.56 : 0.46) : c.block_q == 16 ? 0.16 : c.block_q == 32 ? 0.20 : c.block_q == 64 ? 0.27 : tiles * c.split_k > 0.6 * num_sms ? 0.62 : 0.45;
    const int units = std::max(1, num_sms / (pair ? 2 : c.split_k));
    const double rounds = std::ceil(tiles / units);
    const double shared_us = c.split_k == 1 ? 0.0 : c.split_k == 2 ? 1.0 : c.split_k == 4 ? 1.2 : 1.7;
    const double tile_us = (pair ? 1.6 : 1.0) + (c.split_k > 1 ? 2.0 : 0.0);   // CTAs that share a tile do not go on to another: each round starts anew
    return 4.5 + rounds * (std::ceil(blocks / c.split_k) * block_us) + std::max(0.0, rounds - 1.0) * tile_us + (pair ? 1.6 : 0.5) + shared_us;
}

hgemm_fp8_config_t choose(int32_t form, int64_t M, int64_t N, int64_t K, int32_t groups, int32_t num_sms)
{
    hgemm_fp8_config_t best;
    std::memset(&best, 0, sizeof(best));
    best.cta_group = 2;
    best.block_q = 256;
    best.split_k = 1;
    double least = estimate_us(form, M, N, K, groups, num_sms, best);
    for (int32_t bq = form == HGEMM_FP8_WEIGHT_GRAD ? 128 : 16; bq <= 128; bq *= 2) {
        for (int32_t split = 1; split <= 8; split *= 2) {
            hgemm_fp8_config_t c = best;
            c.cta_group = 1;
            c.block_q = bq;
            c.split_k = split;
            // CTAs beyond the tiles that exist are launched where groups share contractions: only for problems that fit one round
            if (split > 1 && tiles_of(form, M, N, K, groups, c) * split > (split == 8 ? num_sms / 2 : num_sms)) continue;     // (clusters of eight do not fill the GPU)
            const double t = estimate_us(form, M, N, K, groups, num_sms, c);
            if (t < least) {
                least = t;
                best = c;
            }
        }
    }
    return best;
}

int stages_of(int32_t form, const hgemm_fp8_config_t &c, int32_t groups, int *smem)
{
    const bool q_col = c.cta_group == 1 || form == HGEMM_FP8_WEIGHT_GRAD;
    const int bn = c.block_q, stage = hgemm_dev::kFp8PBytes + bn / c.cta_group * 128;
    const int fixed = 1024 + (c.cta_group == 2 ? 8 * hgemm_dev::kFp8StagingPerWarp : 0) + hgemm_dev::fp8_ring(c.cta_group) * hgemm_dev::kFp8Batch * hgemm_dev::fp8_slot_bytes(bn, q_col) + hgemm_dev::kFp8CtrlBytes +
                      (groups > 0 ? 8 * (groups + 1) : 8);
    const int stages = std::min((kSmemOptIn - fixed) / stage, hgemm_dev::kFp8MaxStages);
    *smem = kSmemOptIn;            // all of it: a second CTA on the SM could wait for this one's tensor memory
    return stages;
}

const void *kernel_of(int32_t form, const hgemm_fp8_config_t &c)
{
    using namespace hgemm_dev;
    if (c.cta_group == 2)
        return form == HGEMM_FP8_WEIGHT_GRAD ? reinterpret_cast<const void *>(fp8_product_kernel<2, 256, true, true>)
                                             : reinterpret_cast<const void *>(fp8_product_kernel<2, 256, true, false>);
    if (form == HGEMM_FP8_WEIGHT_GRAD) return reinterpret_cast<const void *>(fp8_product_kernel<1, 128, true, true>);
    switch (c.block_q) {
    case 16: return reinterpret_cast<const void *>(fp8_product_kernel<1, 16, false, true>);
    case 32: return reinterpret_cast<const void *>(fp8_product_kernel<1, 32, false, true>);
    case 64: return reinterpret_cast<const void *>(fp8_product_kernel<1, 64, false, true>);
    default: return reinterpret_cast<const void *>(fp8_product_kernel<1, 128, false, true>);
    }
}

// {inner, outer, matrices} elements with `ld` between rows; boxes of 128 bytes x box_outer rows of one matrix.
bool encode(hgemm_ctx_s *ctx, CUtensorMap *map, CUtensorMapDataType type, int bytes, const void *base, int64_t inner, int64_t outer, int64_t matrices, int64_t ld,
            uint32_t box_outer)
{
    cuuint64_t dims[3] = {cuuint64_t(inner), cuuint64_t(outer), cuuint64_t(matrices)};
    cuuint64_t strides[2] = {cuuint64_t(ld) * unsigned(bytes), cuuint64_t(ld) * unsigned(bytes) * cuuint64_t(outer)};
    cuuint32_t box[3] = {128u / unsigned(bytes), box_outer, 1};
    cuuint32_t estr[3] = {1, 1, 1};
    const CUresult r = ctx->encode(map, type, 3, const_cast<void *>(base), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
                                   CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    if (r != CUDA_SUCCESS) {
        ctx->last_cuda_error = int(r);
        return false;
    }
    return true;
}

template <class T, bool E5M2>
const void *quantize_kernel(int32_t blocks, bool many, bool dense)
{
    using namespace hgemm_dev;
    switch (blocks) {
    case HGEMM_FP8_ROWS:
        if (dense) return many ? reinterpret_cast<const void *>(fp8_quantize_rows_kernel<T, 4, true, E5M2>) : reinterpret_cast<const void *>(fp8_quantize_rows_kernel<T, 1, true, E5M2>);
        return many ? reinterpret_cast<const void *>(fp8_quantize_rows_kernel<T, 4, false, E5M2>) : reinterpret_cast<const void *>(fp8_quantize_rows_kernel<T, 1, false, E5M2>);
    case HGEMM_FP8_COLS: return reinterpret_cast<const void *>(fp8_quantize_tile_kernel<T, 2, E5M2>);
    case HGEMM_FP8_ROWS | HGEMM_FP8_COLS: return reinterpret_cast<const void *>(fp8_quantize_tile_kernel<T, 3, E5M2>);
    default: return reinterpret_cast<const void *>(fp8_quantize_tile_kernel<T, 4, E5M2>);
    }
}

template <class T>
const void *quantize_kernel(const hgemm_fp8_quantize_t &d, bool many, bool dense)
{
    return d.q_type == HGEMM_TYPE_E5M2 ? quantize_kernel<T, true>(d.blocks, many, dense) : quantize_kernel<T, false>(d.blocks, many, dense);
}

bool aligned16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }
bool aligned4(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 3u) == 0; }

hgemm_status_t launch(hgemm_ctx_s *ctx, const void *fn, dim3 grid, int threads, int smem, int cluster, void **args, void *stream)
{
    cudaLaunchConfig_t lc;
    std::memset(&lc, 0, sizeof(lc));
    lc.gridDim = grid;
    lc.blockDim = dim3(unsigned(threads), 1, 1);
    lc.dynamicSmemBytes = size_t(smem);
    lc.stream = static_cast<cudaStream_t>(stream);
    cudaLaunchAttribute attr[2];
    int n = 0;
    if (cluster > 1) {
        attr[n].id = cudaLaunchAttributeClusterDimension;
        attr[n].val.clusterDim.x = unsigned(cluster);
        attr[n].val.clusterDim.y = 1;
        attr[n].val.clusterDim.z = 1;
        ++n;
    }
    if (ctx->dependent_launch) {
        attr[n].id = cudaLaunchAttributeProgrammaticStreamSerialization;
        attr[n].val.programmaticStreamSerializationAllowed = 1;
        ++n;
    }
    lc.attrs = attr;
    lc.numAttrs = unsigned(n);
    const cudaError_t e = cudaLaunchKernelExC(&lc, fn, args);
    return e == cudaSuccess ? HGEMM_OK : cuda_fail(ctx, e);
}

} // namespace

namespace hgemm_host {

int status_slot_of(const hgemm_fp8_plan_s *plan) { return plan->status_slot; }

} // namespace hgemm_host

extern "C" {

int64_t hgemm_fp8_padded_rows(int64_t M, int32_t groups)
{
    if (M < 0 || M > kMaxDim || groups < 0 || groups > hgemm_dev::kFp8MaxGroups) return -1;
    return ceil_div(M + 127 * int64_t(groups), 128) * 128;
}

hgemm_status_t hgemm_fp8_quantize(hgemm_ctx_t *ctx, const hgemm_fp8_quantize_t *d, void *stream)
{
    if (!ctx || !d) return HGEMM_ERR_INVALID_ARG;
    const bool by_rows = (d->blocks & HGEMM_FP8_ROWS) != 0, by_cols = (d->blocks & HGEMM_FP8_COLS) != 0, tiles = d->blocks == HGEMM_FP8_TILES;
    if (!tiles && (d->blocks < 1 || d->blocks > 3)) return HGEMM_ERR_INVALID_ARG;
    if (!is_wide(d->x_type) || !is_fp8(d->q_type) || d->pow2 < 0 || d->pow2 > 1) return HGEMM_ERR_INVALID_ARG;
    if (d->rows < 0 || d->rows > kMaxDim || d->cols < 1 || d->cols > kMaxDim || d->ldx < d->cols || d->groups < 0 || d->groups > hgemm_dev::kQuantMaxGroups) return HGEMM_ERR_INVALID_ARG;
    if (tiles ? (d->row_index || d->offsets || d->groups < 1) : (d->offsets ? !by_cols || d->groups < 1 : d->groups != 0)) return HGEMM_ERR_INVALID_ARG;
    if (d->row_index && (d->x_rows < 0 || !aligned4(d->row_index))) return HGEMM_ERR_INVALID_ARG;
    if (d->offsets && !aligned4(d->offsets)) return HGEMM_ERR_INVALID_ARG;
    if (d->rows == 0) return HGEMM_OK;
    const int es = type_bytes(d->x_type);
    const bool no_source = d->row_index && d->x_rows == 0;   // rows of zeros: x is never read
    if ((!d->x && !no_source) || (reinterpret_cast<uintptr_t>(d->x) % unsigned(es)) != 0) return HGEMM_ERR_INVALID_ARG;
    if ((by_rows || tiles) && (!d->q || !d->scales || !aligned16(d->q) || !aligned4(d->scales) || d->ldq < d->cols || (d->ldq & 15) != 0)) return HGEMM_ERR_INVALID_ARG;
    if (by_cols && (!d->q_cols || !d->scales_cols || !aligned16(d->q_cols) || !aligned4(d->scales_cols) || d->ldq_cols < d->cols || (d->ldq_cols & 15) != 0)) return HGEMM_ERR_INVALID_ARG;
    hgemm_dev::QuantParams p;
    std::memset(&p, 0, sizeof(p));
    p.x = d->x;
    p.ldx = d->ldx;
    p.rows = d->rows;
    p.cols = d->cols;
    p.x_rows = d->x_rows;
    p.row_index = d->row_index;
    p.offsets = d->offsets;
    p.groups = d->groups;
    p.vec_ok = aligned16(d->x) && (d->ldx * es) % 16 == 0 ? 1 : 0;
    p.pow2 = d->pow2;
    p.q = static_cast<uint8_t *>(d->q);
    p.ldq = d->ldq;
    p.scales = d->scales;
    p.q_cols = static_cast<uint8_t *>(d->q_cols);
    p.ldq_cols = d->ldq_cols;
    p.scales_cols = d->scales_cols;
    const int64_t col_blocks = ceil_div(d->cols, 128);
    dim3 grid(1, 1, 1);
    p.fd_blocks = hgemm_dev::make_fast_div(uint32_t(col_blocks));
    // four blocks in flight per group of lanes once that still leaves every SM a full set of warps (128 blocks a CTA, eight CTAs)
    const int64_t row_work = d->rows * col_blocks;
    const bool many = row_work >= int64_t(ctx->num_sms) * 8 * 128;
    const bool dense = !d->row_index && d->cols % 128 == 0 && p.vec_ok && d->ldx == d->cols && d->ldq == d->cols;
    if (row_work >= (int64_t(1) << 31) - 65536) return HGEMM_ERR_UNSUPPORTED;
    if (d->blocks == HGEMM_FP8_ROWS) {
        grid.x = unsigned(std::min<int64_t>(ceil_div(row_work, many ? 128 : 32), int64_t(ctx->num_sms) * 64));
    } else {
        // per group: as many as the copy has room for; the row copies of rows of no group lie in two more runs of rows
        const int64_t row_blocks = d->offsets ? ceil_div(d->rows + 127 * int64_t(d->groups + (by_rows ? 2 : 0)), 128) : ceil_div(d->rows, 128);
        grid.x = unsigned(col_blocks);
        grid.y = unsigned(row_blocks);                         // at most 2^15 + 1025 with these sizes: within the limit of 65535
        grid.z = unsigned(tiles ? d->groups : 1);
    }
    const void *fn = d->x_type == HGEMM_TYPE_F32 ? quantize_kernel<float>(*d, many, dense) : d->x_type == HGEMM_TYPE_F16 ? quantize_kernel<__half>(*d, many, dense)
                                                                                                               : quantize_kernel<__nv_bfloat16>(*d, many, dense);
    void *args[1] = {&p};
    return launch(ctx, fn, grid, hgemm_dev::kQuantThreads, 0, 1, args, stream);
}

hgemm_status_t hgemm_fp8_planned_config(int32_t form, int64_t M, int64_t N, int64_t K, int32_t groups, int32_t num_sms, hgemm_fp8_config_t *out)
{
    if (!out || num_sms < 1) return HGEMM_ERR_INVALID_ARG;
    if (!legal_shape(form, M, N, K, groups)) return HGEMM_ERR_INVALID_ARG;
    *out = choose(form, M, N, K, groups, num_sms);
    return HGEMM_OK;
}

hgemm_status_t hgemm_fp8_plan(hgemm_ctx_t *ctx, int32_t form, int64_t M, int64_t N, int64_t K, int32_t groups, int32_t a_type, int32_t b_type, int32_t out_type,
                              hgemm_fp8_plan_t **out)
{
    if (!ctx || !out || !legal_shape(form, M, N, K, groups) || !is_fp8(a_type) || !is_fp8(b_type) || !is_wide(out_type)) return HGEMM_ERR_INVALID_ARG;
    if (ctx->free_status_slots.empty()) return HGEMM_ERR_ALLOC;
    const hgemm_fp8_config_t cfg = choose(form, M, N, K, groups, ctx->num_sms);
    // every kernel that the plan may be given takes all of the shared memory
    hgemm_fp8_config_t each[5];
    int n = 0;
    each[n++] = {2, 256, 1, 0};
    for (int bq = 128; bq >= (form == HGEMM_FP8_WEIGHT_GRAD ? 128 : 16); bq >>= 1) each[n++] = {1, bq, 1, 0};
    for (int i = 0; i < n; ++i) {
        const cudaError_t e = cudaFuncSetAttribute(kernel_of(form, each[i]), cudaFuncAttributeMaxDynamicSharedMemorySize, kSmemOptIn);
        if (e != cudaSuccess) return cuda_fail(ctx, e);
    }
    hgemm_fp8_plan_s *pl = new (std::nothrow) hgemm_fp8_plan_s;
    if (!pl) return HGEMM_ERR_ALLOC;
    pl->ctx = ctx;
    pl->form = form;
    pl->M = M;
    pl->N = N;
    pl->K = K;
    pl->groups = groups;
    pl->a_type = a_type;
    pl->b_type = b_type;
    pl->out_type = out_type;
    pl->cfg = cfg;
    try {
        ctx->fp8_plans.push_back(pl);
    } catch (const std::bad_alloc &) {
        delete pl;
        return HGEMM_ERR_ALLOC;
    }
    pl->status_slot = ctx->free_status_slots.back();
    ctx->free_status_slots.pop_back();
    *out = pl;
    return HGEMM_OK;
}

hgemm_status_t hgemm_fp8_plan_destroy(hgemm_fp8_plan_t *plan)
{
    if (!plan) return HGEMM_ERR_INVALID_ARG;
    hgemm_ctx_s *ctx = plan->ctx;
    auto it = std::find(ctx->fp8_plans.begin(), ctx->fp8_plans.end(), plan);
    if (it != ctx->fp8_plans.end()) ctx->fp8_plans.erase(it);
    ctx->free_status_slots.push_back(plan->status_slot);     // its capacity holds every slot: this cannot allocate
    delete plan;
    return HGEMM_OK;
}

hgemm_status_t hgemm_fp8_last_device_status(hgemm_fp8_plan_t *plan, uint32_t *code)
{
    if (!plan || !code) return HGEMM_ERR_INVALID_ARG;
    uint32_t v = 0;
    const hgemm_status_t st = hgemm_host::take_status_word(plan->ctx, plan->status_slot, &v);
    if (st != HGEMM_ERR_CUDA) *code = v;
    return st;
}

hgemm_status_t hgemm_fp8_debug_timeout_probe(hgemm_fp8_plan_t *plan, void *stream)
{
    return plan ? hgemm_host::launch_timeout_probe(plan->ctx, plan->status_slot, stream) : HGEMM_ERR_INVALID_ARG;
}

hgemm_status_t hgemm_fp8_plan_get_config(const hgemm_fp8_plan_t *plan, hgemm_fp8_config_t *out)
{
    if (!plan || !out) return HGEMM_ERR_INVALID_ARG;
    *out = plan->cfg;
    return HGEMM_OK;
}

hgemm_status_t hgemm_fp8_plan_set_config(hgemm_fp8_plan_t *plan, const hgemm_fp8_config_t *cfg)
{
    if (!plan || !cfg) return HGEMM_ERR_INVALID_ARG;
    if (!legal_config(plan->form, *cfg)) return HGEMM_ERR_UNSUPPORTED;
    plan->cfg = *cfg;
    return HGEMM_OK;
}

hgemm_status_t hgemm_fp8_run(hgemm_fp8_plan_t *plan, const void *A, int64_t lda, const float *a_scales, const void *B, int64_t ldb, const float *b_scales, void *C,
                             int64_t ldc, const int32_t *offsets, int32_t accumulate, void *stream)
{
    if (!plan) return HGEMM_ERR_INVALID_ARG;
    hgemm_ctx_s *ctx = plan->ctx;
    const int32_t form = plan->form, groups = plan->groups;
    const int64_t M = plan->M, N = plan->N, K = plan->K;
    const bool wgrad = form == HGEMM_FP8_WEIGHT_GRAD;
    const int64_t out_cols = form == HGEMM_FP8_FORWARD ? N : K, a_cols = form == HGEMM_FP8_FORWARD ? K : N;
    if ((groups > 0) != (offsets != nullptr) || accumulate < 0 || accumulate > 1 || (accumulate && plan->out_type != HGEMM_TYPE_F32)) return HGEMM_ERR_INVALID_ARG;
    if (lda < a_cols || ldb < K || ldc < out_cols || (lda & 15) != 0 || (ldb & 15) != 0) return HGEMM_ERR_INVALID_ARG;
    const int es = type_bytes(plan->out_type);
    if (M == 0 && !wgrad) return HGEMM_OK;
    if (!C || (reinterpret_cast<uintptr_t>(C) % unsigned(es)) != 0) return HGEMM_ERR_INVALID_ARG;
    if (M == 0) {
        if (accumulate) return HGEMM_OK;
        const cudaError_t e = cudaMemset2DAsync(C, size_t(ldc) * size_t(es), 0, size_t(K) * size_t(es), size_t(N) * size_t(std::max(groups, 1)), static_cast<cudaStream_t>(stream));
        return e == cudaSuccess ? HGEMM_OK : cuda_fail(ctx, e);
    }
    if (!A || !B || !a_scales || !b_scales || !aligned16(A) || !aligned16(B) || !aligned4(a_scales) || !aligned4(b_scales) || !aligned4(offsets)) return HGEMM_ERR_INVALID_ARG;

    const hgemm_fp8_config_t &c = plan->cfg;
    const bool swap = c.cta_group == 1;                      // the kernel's P operand is the caller's B
    Fp8Params p;
    std::memset(&p, 0, sizeof(p));
    int smem = 0;
    p.stages = stages_of(form, c, groups, &smem);
    if (p.stages < 2) return HGEMM_ERR_UNSUPPORTED;
    p.split = c.split_k;
    p.groups = groups;
    p.offsets = offsets;
    p.rows_ragged = int32_t(M);
    const int64_t a_rows = wgrad && groups > 0 ? hgemm_fp8_padded_rows(M, groups) : M;
    const int64_t matrices = std::max(groups, 1);
    const int64_t k_blk = ceil_div(K, 128), n_blk = ceil_div(N, 128);

    // one side of the product: rows, matrix extents, whether the contraction runs down the columns, scales
    struct Side {
        const void *base;
        int64_t rows, inner, outer, count, ld;
        bool mn;
        const float *s;
        int64_t s_row, s_kb, s_group;
        int32_t type;
    } a, b;
    if (form == HGEMM_FP8_FORWARD) {
        a = {A, M, K, M, 1, lda, false, a_scales, k_blk, 1, 0, plan->a_type};
        b = {B, N, K, N, matrices, ldb, false, b_scales, k_blk, 1, n_blk * k_blk, plan->b_type};
        p.kblocks = int32_t(k_blk);
    } else if (form == HGEMM_FP8_INPUT_GRAD) {
        a = {A, M, N, M, 1, lda, false, a_scales, n_blk, 1, 0, plan->a_type};
        b = {B, K, K, N, matrices, ldb, true, b_scales, 1, k_blk, n_blk * k_blk, plan->b_type};
        p.kblocks = int32_t(n_blk);
    } else {
        a = {A, N, N, a_rows, 1, lda, true, a_scales, 1, N, 0, plan->a_type};
        b = {B, K, K, a_rows, 1, ldb, true, b_scales, 1, K, 0, plan->b_type};
        p.kblocks = int32_t(ceil_div(M, 128));
        p.k_capacity = int32_t(a_rows / 128);
    }
    const Side &P = swap ? b : a, &Q = swap ? a : b;
    const int tp = 128 * c.cta_group, tq = c.block_q;
    p.rows_p = int32_t(P.rows);
    p.rows_q = int32_t(Q.rows);
    p.tiles_p = int32_t(ceil_div(P.rows, tp));
    p.tiles_q = int32_t(ceil_div(Q.rows, tq));
    p.ragged = groups == 0 ? hgemm_dev::kRaggedNone : wgrad ? hgemm_dev::kRaggedK : swap ? hgemm_dev::kRaggedQ : hgemm_dev::kRaggedP;
    const int64_t tiles = tiles_of(form, M, N, K, groups, c);
    if (tiles > (int64_t(1) << 30)) return HGEMM_ERR_UNSUPPORTED;
    p.total = int32_t(tiles);
    p.raster = std::min(8, p.tiles_p);
    {
        using hgemm_dev::make_fast_div;
        const int32_t last = p.tiles_p - (p.tiles_p - 1) / p.raster * p.raster;         // rows of tiles of the last sweep
        p.fd_other = make_fast_div(uint32_t(p.ragged == hgemm_dev::kRaggedP ? p.tiles_q : p.tiles_p));
        p.fd_group = make_fast_div(uint32_t(p.tiles_p) * uint32_t(p.tiles_q));
        p.fd_sweep = make_fast_div(uint32_t(p.raster) * uint32_t(p.tiles_q));
        p.fd_raster = make_fast_div(uint32_t(p.raster));
        p.fd_last = make_fast_div(uint32_t(last));
    }
    p.sp = P.s;
    p.sp_row = P.s_row;
    p.sp_kb = P.s_kb;
    p.sp_group = P.s_group;
    p.sq = Q.s;
    p.sq_row = Q.s_row;
    p.sq_kb = Q.s_kb;
    p.sq_group = Q.s_group;
    p.p_mn = P.mn ? 1 : 0;
    p.q_mn = Q.mn ? 1 : 0;
    p.out = C;
    p.ldc = ldc;
    p.c_group = wgrad ? N * ldc : 0;
    p.out_type = plan->out_type;
    p.accumulate = accumulate;
    p.vec_ok = aligned16(C) && (ldc * es) % 16 == 0 && (out_cols * es) % 16 == 0 ? 1 : 0;      // a tensor store clips at multiples of 16 bytes only
    // instruction descriptor: fp32 accumulators; formats 0 = e4m3, 1 = e5m2; bits 15 / 16: operand stored along its own rows
    p.idesc = (1u << 4) | (P.type == HGEMM_TYPE_E5M2 ? 1u << 7 : 0u) | (Q.type == HGEMM_TYPE_E5M2 ? 1u << 10 : 0u) | (P.mn ? 1u << 15 : 0u) | (Q.mn ? 1u << 16 : 0u) |
              (uint32_t((tq / c.cta_group) >> 3) << 17) | (uint32_t(tp >> 4) << 24);
    p.status = ctx->d_status + plan->status_slot;
    p.wait_budget = ctx->wait_budget;

    CUtensorMap map_p, map_q, map_c;
    if (!encode(ctx, &map_p, CU_TENSOR_MAP_DATA_TYPE_UINT8, 1, P.base, P.inner, P.outer, P.count, P.ld, 128)) return HGEMM_ERR_CUDA;
    if (!encode(ctx, &map_q, CU_TENSOR_MAP_DATA_TYPE_UINT8, 1, Q.base, Q.inner, Q.outer, Q.count, Q.ld, Q.mn ? 128u : uint32_t(tq / c.cta_group))) return HGEMM_ERR_CUDA;
    map_c = map_p;                                           // not used by the kernels that store through pointers
    if (c.cta_group == 2 && p.vec_ok && !accumulate) {
        const CUtensorMapDataType t = plan->out_type == HGEMM_TYPE_F32 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT32 : plan->out_type == HGEMM_TYPE_F16 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT16
                                                                                                                                        : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16;
        if (!encode(ctx, &map_c, t, es, C, out_cols, wgrad ? N : M, wgrad ? matrices : 1, ldc, 32)) return HGEMM_ERR_CUDA;
    }
    const int per_unit = c.cta_group == 2 ? 2 : c.split_k;
    // CTAs that share a tile through a cluster's shared memory take one tile each; the others walk the tiles
    const int64_t units = c.split_k > 1 ? tiles : std::min<int64_t>(tiles, std::max(1, ctx->num_sms / per_unit));
    if (units * per_unit > 0x7fffffff) return HGEMM_ERR_UNSUPPORTED;
    void *args[4] = {&map_p, &map_q, &map_c, &p};
    return launch(ctx, kernel_of(form, c), dim3(unsigned(units * per_unit), 1, 1), hgemm_dev::kFp8Threads, smem, per_unit, args, stream);
}

} // extern "C"
