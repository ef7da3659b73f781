// C ABI of the 4-bit products with block scales (see include/hgemm_fp4.h): quantisation, plans, launches.
#include <cuda.h>
#include <cuda_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstring>
#include <new>

#include "../../include/hgemm_fp4.h"
#include "fp4_product_kernel.cuh"
#include "fp4_quantize_kernel.cuh"
#include "hgemm_context.h"

using hgemm_dev::Fp4Params;

struct hgemm_fp4_plan_s {
    hgemm_ctx_s *ctx = nullptr;
    int32_t form = 0;
    int64_t M = 0, N = 0, K = 0;
    int32_t groups = 0, format = 0, out_type = 0;
    hgemm_fp4_config_t cfg{};
    int status_slot = 0;
};

namespace {

constexpr int64_t kMaxDim = int64_t(1) << 22;
constexpr int kSmemOptIn = 232448;
constexpr int kMaxMatrices = 1024;

int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

bool is_format(int32_t f) { return f == HGEMM_FP4_NV || f == HGEMM_FP4_MX; }
bool is_wide(int32_t t) { return t == HGEMM_TYPE_F32 || t == HGEMM_TYPE_F16 || t == HGEMM_TYPE_BF16; }
int type_bytes(int32_t t) { return t == HGEMM_TYPE_F32 ? 4 : 2; }
int64_t atoms_of(int64_t cols, int32_t format) { return ceil_div(cols, format == HGEMM_FP4_NV ? 64 : 128); }      // scale tiles across

bool legal_shape(int32_t form, int64_t M, int64_t N, int64_t K, int32_t groups)
{
    return form >= HGEMM_FP8_FORWARD && form <= HGEMM_FP8_WEIGHT_GRAD && M >= 0 && M <= kMaxDim && N >= 1 && N <= kMaxDim && K >= 1 && K <= kMaxDim &&
           groups >= 0 && groups <= hgemm_dev::kFp4MaxGroups;
}

bool legal_config(const hgemm_fp4_config_t &c)
{
    if (c.cta_group == 2) return (c.block_q == 256 || c.block_q == 128) && c.split_k == 1;
    if (c.cta_group != 1) return false;
    return (c.block_q == 128 || c.block_q == 64) && (c.split_k == 1 || c.split_k == 2 || c.split_k == 4 || c.split_k == 8);
}

// Tiles of a configuration, over all groups (for groups that follow offsets on the device: at most).
int64_t tiles_of(int32_t form, int64_t M, int64_t N, int64_t K, int32_t groups, const hgemm_fp4_config_t &c)
{
    const bool pair = c.cta_group == 2;
    const int64_t outs = form == HGEMM_FP8_FORWARD ? N : K;                   // columns of the result
    const int64_t tp = pair ? 256 : 128;
    if (form == HGEMM_FP8_WEIGHT_GRAD) return std::max(groups, 1) * (pair ? ceil_div(N, tp) * ceil_div(K, c.block_q) : ceil_div(K, tp) * ceil_div(N, c.block_q));
    const int64_t bt = pair ? 256 : c.block_q, bo = pair ? c.block_q : 128;
    if (groups == 0) return ceil_div(M, bt) * ceil_div(outs, bo);
    return (std::min<int64_t>(groups, M) + M / bt) * ceil_div(outs, bo);
}

// Estimated time of a configuration in microseconds: a start (launch, first loads, last stores), the first round's stages (256 of the contraction), then rounds of
// tiles over the SMs, whose stages share L2 with the other SMs' and whose ends cost what the epilogue does not hide.  Measured (B200, bf16 results, operands in
// L2): 256 x 4096 x 4096: pairs of 256 columns 9.6 us, of 128 columns 7.1, single CTAs of 64 rows 8.5, of 128 rows 10.7; 4096^3: 28.0, 29.6, 53.8, 44.1;
// 16 x 4096 x 4096: 64 rows by one, two, four CTAs a tile 7.1, 6.5, 6.7; 16 x 1024 x 4096: by four, eight 5.3, 5.1.
double estimate_us(int32_t form, int64_t M, int64_t N, int64_t K, int32_t groups, int32_t num_sms, int32_t out_bytes, const hgemm_fp4_config_t &c)
{
    const bool wgrad = form == HGEMM_FP8_WEIGHT_GRAD, pair = c.cta_group == 2;
    const int64_t outs = form == HGEMM_FP8_FORWARD ? N : K;
    const double rows = groups > 0 ? double(M) / groups : double(M);           // rows of one group, on average
    double tiles, stages;
    if (wgrad) {
        tiles = double(tiles_of(form, M, N, K, groups, c));
        stages = std::ceil(rows / 256.0) + (groups > 0 && rows > 256.0 ? 0.5 : 0.0);
    } else {
        const int64_t bt = pair ? 256 : c.block_q, bo = pair ? c.block_q : 128;
        // groups are uneven: each ends in a partly filled tile
        const double of_rows = groups > 0 ? std::min<double>(groups, double(M)) * std::max(1.0, rows / double(bt) + 0.7) : double(ceil_div(M, bt));
        tiles = of_rows * double(ceil_div(outs, bo));
        stages = double(ceil_div(form == HGEMM_FP8_FORWARD ? K : N, 256));
    }
    struct Cost {
        double start, first, stage, end;
    };
    const Cost t = pair ? (c.block_q == 256 ? Cost{5.2, 0.27, 0.37, 0.5} : Cost{4.6, 0.15, 0.21, 0.45}) : c.block_q == 64 ? Cost{4.9, 0.17, 0.17, 1.7} : Cost{7.0, 0.20, 0.20, 3.2};
    const double widen = out_bytes == 4 ? 1.6 : 1.0;                           // fp32 results: twice the bytes at a tile's end
    const int units = std::max(1, num_sms / (pair ? 2 : c.split_k));
    const double rounds = std::ceil(tiles / units), own = std::ceil(stages / c.split_k);
    const double shared = c.split_k == 1 ? 0.0 : c.split_k == 2 ? 0.5 : c.split_k == 4 ? 0.6 : 0.8;
    const double thin = pair && groups == 0 && !wgrad && M <= 32 ? 1.0 : 0.0;       // (1 x 8192 x 2048: pairs 7.8 us, 64 rows 6.1; with 128 rows 6.0 and 7.1)
    const double again = t.end * widen + (c.split_k > 1 ? 3.0 : 0.0);          // CTAs that share a tile do not go on to another: each round starts anew
    return t.start + thin + own * t.first + shared + (rounds - 1.0) * (own * t.stage + again);
}

hgemm_fp4_config_t choose(int32_t form, int64_t M, int64_t N, int64_t K, int32_t groups, int32_t num_sms, int32_t out_bytes)
{
    hgemm_fp4_config_t best{2, 256, 1, 0};
    double least = estimate_us(form, M, N, K, groups, num_sms, out_bytes, best);
    auto consider = [&](const hgemm_fp4_config_t &c) {
        const double t = estimate_us(form, M, N, K, groups, num_sms, out_bytes, c);
        if (t < least) {
            least = t;
            best = c;
        }
    };
    consider({2, 128, 1, 0});
    for (int32_t bq = 64; bq <= 128; bq *= 2) {
        for (int32_t split = 1; split <= 8; split *= 2) {
            const hgemm_fp4_config_t c{1, bq, split, 0};
            // CTAs beyond the tiles that exist are launched where groups share contractions: only for problems that fit one round
            if (split > 1 && tiles_of(form, M, N, K, groups, c) * split > (split == 8 ? num_sms / 2 : num_sms)) continue;     // (clusters of eight do not fill the GPU)
            consider(c);
        }
    }
    return best;
}

int stages_of(const hgemm_fp4_config_t &c, bool nv, int32_t groups, int smem)
{
    const int fixed = 1024 + (c.cta_group == 2 ? 8 * hgemm_dev::kFp4StagingPerWarp : 0) + hgemm_dev::kFp4CtrlBytes + 12 * (groups + 1);
    return std::min((smem - fixed) / hgemm_dev::fp4_stage_bytes(c.cta_group, c.block_q, nv), hgemm_dev::kFp4MaxStages);
}

template <bool NV>
const void *kernel_of(const hgemm_fp4_config_t &c)
{
    using namespace hgemm_dev;
    if (c.cta_group == 2) return c.block_q == 256 ? reinterpret_cast<const void *>(fp4_product_kernel<2, 256, NV>) : reinterpret_cast<const void *>(fp4_product_kernel<2, 128, NV>);
    return c.block_q == 128 ? reinterpret_cast<const void *>(fp4_product_kernel<1, 128, NV>) : reinterpret_cast<const void *>(fp4_product_kernel<1, 64, NV>);
}
const void *kernel_of(const hgemm_fp4_config_t &c, int32_t format) { return format == HGEMM_FP4_NV ? kernel_of<true>(c) : kernel_of<false>(c); }

bool encode3(hgemm_ctx_s *ctx, CUtensorMap *map, CUtensorMapDataType type, const void *base, const cuuint64_t (&dims)[3], const cuuint64_t (&strides)[2], const cuuint32_t (&box)[3],
             CUtensorMapSwizzle swizzle)
{
    const cuuint32_t estr[3] = {1, 1, 1};
    const CUresult r = ctx->encode(map, type, 3, const_cast<void *>(base), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE, swizzle, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                                   CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    if (r != CUDA_SUCCESS) {
        ctx->last_cuda_error = int(r);
        return false;
    }
    return true;
}

// Packed values: `matrices` matrices of rows x bytes, `ld` bytes between rows; boxes of 128 bytes x box_rows.
bool encode_values(hgemm_ctx_s *ctx, CUtensorMap *map, const void *base, int64_t bytes, int64_t rows, int64_t matrices, int64_t ld, uint32_t box_rows)
{
    return encode3(ctx, map, CU_TENSOR_MAP_DATA_TYPE_UINT8, base, {cuuint64_t(bytes), cuuint64_t(rows), cuuint64_t(matrices)}, {cuuint64_t(ld), cuuint64_t(ld) * cuuint64_t(rows)},
                   {128, box_rows, 1}, CU_TENSOR_MAP_SWIZZLE_128B);
}

// Scale tiles: `tiles` runs of `atoms` tiles of 512 bytes; boxes of a stage's tiles x box_tiles runs.
bool encode_scales(hgemm_ctx_s *ctx, CUtensorMap *map, const void *base, int64_t atoms, int64_t tiles, bool nv, uint32_t box_tiles)
{
    return encode3(ctx, map, CU_TENSOR_MAP_DATA_TYPE_UINT32, base, {128, cuuint64_t(atoms), cuuint64_t(tiles)}, {512, 512 * cuuint64_t(atoms)},
                   {128, cuuint32_t(hgemm_dev::fp4_atoms(nv)), box_tiles}, CU_TENSOR_MAP_SWIZZLE_NONE);
}

// Results: boxes of 128 bytes x 32 rows.
bool encode_results(hgemm_ctx_s *ctx, CUtensorMap *map, int32_t type, const void *base, int64_t cols, int64_t rows, int64_t matrices, int64_t ld)
{
    const unsigned es = unsigned(type_bytes(type));
    const CUtensorMapDataType t = type == HGEMM_TYPE_F32 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT32 : type == HGEMM_TYPE_F16 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT16 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16;
    return encode3(ctx, map, t, base, {cuuint64_t(cols), cuuint64_t(rows), cuuint64_t(matrices)}, {cuuint64_t(ld) * es, cuuint64_t(ld) * es * cuuint64_t(rows)}, {128u / es, 32, 1},
                   CU_TENSOR_MAP_SWIZZLE_128B);
}

template <class T, bool NV>
const void *quantize_kernel(int32_t blocks)
{
    using namespace hgemm_dev;
    return blocks == HGEMM_FP4_ROWS ? reinterpret_cast<const void *>(fp4_quantize_kernel<T, 1, NV>)
           : blocks == HGEMM_FP4_COLS ? reinterpret_cast<const void *>(fp4_quantize_kernel<T, 2, NV>) : reinterpret_cast<const void *>(fp4_quantize_kernel<T, 3, NV>);
}
template <class T>
const void *quantize_kernel(int32_t blocks, int32_t format) { return format == HGEMM_FP4_NV ? quantize_kernel<T, true>(blocks) : quantize_kernel<T, false>(blocks); }

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

constexpr int kDigits = hgemm_dev::kFp4Digits;

const void *digits_kernel_of(const hgemm_fp4_config_t &c, int32_t format)
{
    using namespace hgemm_dev;
    if (format == HGEMM_FP4_NV) return c.block_q == 128 ? reinterpret_cast<const void *>(fp4_product_kernel<1, 128, true, true>) : reinterpret_cast<const void *>(fp4_product_kernel<1, 64, true, true>);
    return c.block_q == 128 ? reinterpret_cast<const void *>(fp4_product_kernel<1, 128, false, true>) : reinterpret_cast<const void *>(fp4_product_kernel<1, 64, false, true>);
}

// At most as many tiles as `choices` rows of eight digits, over `groups` groups, can have.
int64_t digits_tiles(int64_t choices, int64_t N, int32_t groups, const hgemm_fp4_config_t &c)
{
    return (std::min<int64_t>(groups, choices) + choices * kDigits / c.block_q) * ceil_div(N, 128);
}

// Shared memory of a CTA; DIGITS: with room beside it for one that makes digits, so that the first weights are on their way before those end (16 tokens of 8 among
// 64 experts: 47.6 us; with all of it 53.0).
constexpr int product_smem(bool digits) { return digits ? kSmemOptIn - 8192 : kSmemOptIn; }

// The forward product of rows that are written as sums of eight 4-bit rows each (DIGITS: M counts those), or any product of a plan.
template <bool DIGITS>
hgemm_status_t run_product(const hgemm_fp4_plan_s &plan, const void *A, int64_t lda, const void *a_scales, const float *a_factor, const void *B, int64_t ldb, const void *b_scales,
                           const float *b_factor, void *C, int64_t ldc, const int32_t *offsets, int32_t accumulate, void *stream, const int32_t *indices = nullptr)
{
    hgemm_ctx_s *ctx = plan.ctx;
    const int32_t form = plan.form, groups = plan.groups;
    const int64_t M = plan.M, N = plan.N, K = plan.K;
    const bool wgrad = form == HGEMM_FP8_WEIGHT_GRAD, nv = plan.format == HGEMM_FP4_NV;
    const int64_t out_cols = form == HGEMM_FP8_FORWARD ? N : K;
    const int64_t depth = wgrad ? (groups > 0 ? hgemm_fp8_padded_rows(M, groups) : M) : form == HGEMM_FP8_FORWARD ? K : N;       // contracted elements of the copies
    if ((groups > 0) != ((DIGITS ? indices : offsets) != nullptr) || accumulate < 0 || accumulate > 1 || (accumulate && plan.out_type != HGEMM_TYPE_F32)) return HGEMM_ERR_INVALID_ARG;
    if (lda < ceil_div(depth, 2) || ldb < ceil_div(depth, 2) || ldc < out_cols || (lda & 15) != 0 || (ldb & 15) != 0) return HGEMM_ERR_INVALID_ARG;
    const int es = type_bytes(plan.out_type);
    if (M == 0 && !wgrad) return HGEMM_OK;
    if (!C || (reinterpret_cast<uintptr_t>(C) % unsigned(es)) != 0) return HGEMM_ERR_INVALID_ARG;
    if (M == 0) {
        if (accumulate) return HGEMM_OK;
        const cudaError_t e = cudaMemset2DAsync(C, size_t(ldc) * size_t(es), 0, size_t(K) * size_t(es), size_t(N) * size_t(std::max(groups, 1)), static_cast<cudaStream_t>(stream));
        return e == cudaSuccess ? HGEMM_OK : cuda_fail(ctx, e);
    }
    if (!A || !B || !a_scales || !b_scales || !aligned16(A) || !aligned16(B) || !aligned16(a_scales) || !aligned16(b_scales) || !aligned4(offsets)) return HGEMM_ERR_INVALID_ARG;
    if ((nv && !DIGITS) != (a_factor != nullptr) || nv != (b_factor != nullptr) || !aligned4(a_factor) || !aligned4(b_factor)) return HGEMM_ERR_INVALID_ARG;

    const hgemm_fp4_config_t &c = plan.cfg;
    const bool swap = c.cta_group == 1;                      // the kernel's P operand is the caller's B
    Fp4Params p;
    std::memset(&p, 0, sizeof(p));
    p.stages = stages_of(c, nv, groups, product_smem(DIGITS));
    if (p.stages < 2) return HGEMM_ERR_UNSUPPORTED;
    p.split = c.split_k;
    p.groups = groups;
    p.offsets = offsets;
    p.indices = indices;
    p.choices = DIGITS ? int32_t(M / kDigits) : 0;
    p.rows_ragged = int32_t(M);
    p.kblocks = int32_t(ceil_div(depth, 128));
    p.k_capacity = int32_t(ceil_div(depth, 128));
    const int64_t matrices = std::max(groups, 1);

    // one side of the product: values (rows x depth, `count` matrices), their scale tiles, their factors
    struct Side {
        const void *base;
        int64_t rows, count, ld;
        const void *scales;
        int64_t scale_tiles;
        const float *factor;
    } a, b;
    const int64_t a_rows = wgrad ? N : M, b_rows = form == HGEMM_FP8_FORWARD ? N : K;
    a = {A, a_rows, 1, lda, a_scales, !wgrad && groups > 0 ? hgemm_fp8_padded_rows(M, groups) / 128 : ceil_div(a_rows, 128), a_factor};
    b = {B, b_rows, wgrad ? 1 : matrices, ldb, b_scales, ceil_div(b_rows, 128) * (wgrad ? 1 : matrices), b_factor};
    const Side &P = swap ? b : a, &Q = swap ? a : b;
    const int tp = 128 * c.cta_group, tq = c.block_q;
    p.rows_p = int32_t(P.rows);
    p.rows_q = int32_t(Q.rows);
    p.tiles_p = int32_t(ceil_div(P.rows, tp));
    p.tiles_q = int32_t(ceil_div(Q.rows, tq));
    p.ragged = groups == 0 ? hgemm_dev::kRaggedNone : wgrad ? hgemm_dev::kRaggedK : swap ? hgemm_dev::kRaggedQ : hgemm_dev::kRaggedP;
    const int64_t tiles = DIGITS ? digits_tiles(M / kDigits, N, groups, c) : tiles_of(form, M, N, K, groups, c);
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
    p.sp_group = int32_t(ceil_div(P.rows, 128));
    p.sq_group = int32_t(ceil_div(Q.rows, 128));
    p.fp = P.factor;
    p.fq = Q.factor;
    p.fp_group = P.count > 1 ? 1 : 0;
    p.fq_group = Q.count > 1 ? 1 : 0;
    p.out = C;
    p.ldc = ldc;
    p.c_group = wgrad ? N * ldc : 0;
    p.out_type = plan.out_type;
    p.accumulate = accumulate;
    p.vec_ok = aligned16(C) && (ldc * es) % 16 == 0 && (out_cols * es) % 16 == 0 ? 1 : 0;      // a tensor store clips at multiples of 16 bytes only
    // instruction descriptor of the block-scaled kinds: e2m1 operands (1) along the contraction; bit 23: scales are powers of two; bits 4 and 29: the
    // scales' place in their word, set by the kernel
    p.idesc = (1u << 7) | (1u << 10) | (uint32_t(tq >> 3) << 17) | (nv ? 0u : 1u << 23) | (uint32_t(tp >> 4) << 24);
    p.status = ctx->d_status + plan.status_slot;
    p.wait_budget = ctx->wait_budget;

    CUtensorMap map_p, map_q, map_sp, map_sq, map_c;
    const int64_t bytes = ceil_div(depth, 2), atoms = atoms_of(depth, plan.format);
    if (!encode_values(ctx, &map_p, P.base, bytes, P.rows, P.count, P.ld, 128)) return HGEMM_ERR_CUDA;
    if (!encode_values(ctx, &map_q, Q.base, bytes, Q.rows, Q.count, Q.ld, uint32_t(tq / c.cta_group))) return HGEMM_ERR_CUDA;
    if (!encode_scales(ctx, &map_sp, P.scales, atoms, P.scale_tiles, nv, 1)) return HGEMM_ERR_CUDA;
    if (!encode_scales(ctx, &map_sq, Q.scales, atoms, Q.scale_tiles, nv, uint32_t(hgemm_dev::fp4_scale_tiles(tq)))) return HGEMM_ERR_CUDA;
    map_c = map_p;                                           // not used by the kernels that store through pointers
    if (c.cta_group == 2 && p.vec_ok && !accumulate) {
        if (!encode_results(ctx, &map_c, plan.out_type, C, out_cols, wgrad ? N : M, wgrad ? matrices : 1, ldc)) return HGEMM_ERR_CUDA;
    }
    const int per_unit = c.cta_group == 2 ? 2 : c.split_k;
    // CTAs that share a tile through a cluster's shared memory take one tile each; the others walk the tiles
    const int64_t units = c.split_k > 1 ? tiles : std::min<int64_t>(tiles, std::max(1, ctx->num_sms / per_unit));
    if (units * per_unit > 0x7fffffff) return HGEMM_ERR_UNSUPPORTED;
    void *args[6] = {&map_p, &map_q, &map_sp, &map_sq, &map_c, &p};
    return launch(ctx, DIGITS ? digits_kernel_of(c, plan.format) : kernel_of(c, plan.format), dim3(unsigned(units * per_unit), 1, 1), hgemm_dev::kFp4Threads, product_smem(DIGITS), per_unit, args, stream);
}

} // namespace

namespace hgemm_host {

int status_slot_of(const hgemm_fp4_plan_s *plan) { return plan->status_slot; }

hgemm_status_t fp4_digits_prepare(hgemm_ctx_s *ctx)
{
    for (const int32_t format : {HGEMM_FP4_NV, HGEMM_FP4_MX}) {
        for (const int32_t width : {64, 128}) {
            const cudaError_t e = cudaFuncSetAttribute(digits_kernel_of({1, width, 1, 0}, format), cudaFuncAttributeMaxDynamicSharedMemorySize, product_smem(true));
            if (e != cudaSuccess) return cuda_fail(ctx, e);
        }
    }
    return HGEMM_OK;
}

hgemm_status_t fp4_digits_product(hgemm_ctx_s *ctx, int32_t format, int64_t choices, int64_t N, int64_t K, int32_t groups, const void *digits, int64_t ld, const void *digit_scales, const void *B,
                                  int64_t ldb, const void *b_scales, const float *b_factor, float *C, int64_t ldc, const int32_t *indices, void *stream)
{
    hgemm_fp4_plan_s plan;
    plan.ctx = ctx;
    plan.form = HGEMM_FP8_FORWARD;
    plan.M = choices * kDigits;
    plan.N = N;
    plan.K = K;
    plan.groups = groups;
    plan.format = format;
    plan.out_type = HGEMM_TYPE_F32;
    // 8 choices a tile (64 columns), or 16 where experts have more than 6 on average (2048 -> 1024 -> 2048, SwiGLU, the whole layer: 8 choices of 64 experts 16.6 against
    // 18.4 us; 256: 52.3 and 55.3; 512: 62.8 and 60.7; 512 of 16 experts: 49.0 and 41.8).  CTAs that share a contraction only where tiles leave SMs without
    // work: each round of them starts anew (8 choices of 64 experts, tiles for every SM, shared by two: 32.9 us).
    plan.cfg = {1, choices > 8 && choices > 6 * groups ? 128 : 64, 1, 0};
    while (plan.cfg.split_k < 8 && digits_tiles(choices, N, groups, plan.cfg) * plan.cfg.split_k * 2 <= ctx->num_sms && ceil_div(K, 256) >= 2 * plan.cfg.split_k * 2) plan.cfg.split_k *= 2;
    return run_product<true>(plan, digits, ld, digit_scales, nullptr, B, ldb, b_scales, b_factor, C, ldc, nullptr, 0, stream, indices);
}

} // namespace hgemm_host

extern "C" {

int64_t hgemm_fp4_scale_bytes(int64_t rows, int64_t cols, int32_t format)
{
    // a column copy per group contracts over up to hgemm_fp8_padded_rows elements
    if (rows < 0 || rows > 2 * kMaxDim || cols < 0 || cols > 2 * kMaxDim || !is_format(format)) return -1;
    return ceil_div(rows, 128) * atoms_of(cols, format) * 512;
}

hgemm_status_t hgemm_fp4_tensor_factor(hgemm_ctx_t *ctx, int32_t x_type, int64_t matrices, int64_t rows, int64_t cols, const void *x, int64_t ldx, float *factor, void *stream)
{
    if (!ctx || !is_wide(x_type) || matrices < 1 || matrices > kMaxMatrices || rows < 0 || rows > kMaxDim || cols < 1 || cols > kMaxDim || ldx < cols) return HGEMM_ERR_INVALID_ARG;
    if (!factor || !aligned4(factor)) return HGEMM_ERR_INVALID_ARG;
    const int es = type_bytes(x_type);
    if (rows > 0 && (!x || (reinterpret_cast<uintptr_t>(x) % unsigned(es)) != 0)) return HGEMM_ERR_INVALID_ARG;
    int32_t vec = aligned16(x) && (ldx * es) % 16 == 0 ? 1 : 0;
    // Up to 2 MB a matrix: eight CTAs (a cluster) have all of it, and one launch does; beyond that the GPU is wider than a cluster, and the factors,
    // set to zero first, are raised to the maximum (bf16, 4096 columns: 24 rows 2.4 against 5.8 us, 256 rows 4.5 and 5.8, 512 rows 6.8 and 5.9).
    const bool cluster = rows * cols * es <= (int64_t(1) << 21);
    if (!cluster) {
        const cudaError_t e = cudaMemsetAsync(factor, 0, size_t(matrices) * 4, static_cast<cudaStream_t>(stream));
        if (e != cudaSuccess) return cuda_fail(ctx, e);
    }
    using namespace hgemm_dev;
    const void *fn = x_type == HGEMM_TYPE_F32   ? (cluster ? reinterpret_cast<const void *>(fp4_factor_kernel<float, true>) : reinterpret_cast<const void *>(fp4_factor_kernel<float, false>))
                     : x_type == HGEMM_TYPE_F16 ? (cluster ? reinterpret_cast<const void *>(fp4_factor_kernel<__half, true>) : reinterpret_cast<const void *>(fp4_factor_kernel<__half, false>))
                                                : (cluster ? reinterpret_cast<const void *>(fp4_factor_kernel<__nv_bfloat16, true>) : reinterpret_cast<const void *>(fp4_factor_kernel<__nv_bfloat16, false>));
    const int64_t runs = rows * ceil_div(cols, 16);
    const int64_t ctas = cluster ? kFp4FactorCluster : std::max<int64_t>(1, std::min<int64_t>(ceil_div(runs, kFp4FactorThreads * 4), ceil_div(int64_t(ctx->num_sms) * 4, matrices)));
    void *args[6] = {&x, &ldx, &rows, &cols, &vec, &factor};
    return launch(ctx, fn, dim3(unsigned(ctas), unsigned(matrices), 1), kFp4FactorThreads, 0, cluster ? kFp4FactorCluster : 1, args, stream);
}

hgemm_status_t hgemm_fp4_quantize(hgemm_ctx_t *ctx, const hgemm_fp4_quantize_t *d, void *stream)
{
    if (!ctx || !d) return HGEMM_ERR_INVALID_ARG;
    if (d->blocks < 1 || d->blocks > 3 || !is_wide(d->x_type) || !is_format(d->format)) return HGEMM_ERR_INVALID_ARG;
    const bool by_rows = (d->blocks & HGEMM_FP4_ROWS) != 0, by_cols = (d->blocks & HGEMM_FP4_COLS) != 0, nv = d->format == HGEMM_FP4_NV;
    if (d->rows < 0 || d->rows > kMaxDim || d->cols < 1 || d->cols > kMaxDim || d->ldx < d->cols || d->matrices < 1 || d->matrices > kMaxMatrices) return HGEMM_ERR_INVALID_ARG;
    if (d->matrices > 1 && (d->row_index || d->offsets)) return HGEMM_ERR_INVALID_ARG;
    if (d->offsets ? d->groups < 1 || d->groups > hgemm_dev::kFp4MaxGroups : d->groups != 0) return HGEMM_ERR_INVALID_ARG;
    if (d->row_index && (d->x_rows < 0 || !aligned4(d->row_index))) return HGEMM_ERR_INVALID_ARG;
    if ((d->offsets && !aligned4(d->offsets)) || nv != (d->factor != nullptr) || (d->factor && !aligned4(d->factor))) return HGEMM_ERR_INVALID_ARG;
    if (d->rows == 0) return HGEMM_OK;
    const int es = type_bytes(d->x_type);
    const bool no_source = d->row_index && d->x_rows == 0;   // rows of zeros: x is never read
    if ((!d->x && !no_source) || (reinterpret_cast<uintptr_t>(d->x) % unsigned(es)) != 0) return HGEMM_ERR_INVALID_ARG;
    const int64_t col_rows = d->offsets ? hgemm_fp8_padded_rows(d->rows, d->groups) : d->rows;
    if (by_rows && (!d->q || !d->scales || !aligned16(d->q) || !aligned16(d->scales) || d->ldq < ceil_div(d->cols, 2) || (d->ldq & 15) != 0)) return HGEMM_ERR_INVALID_ARG;
    if (by_cols && (!d->q_cols || !d->scales_cols || !aligned16(d->q_cols) || !aligned16(d->scales_cols) || d->ldq_cols < ceil_div(col_rows, 2) || (d->ldq_cols & 15) != 0)) return HGEMM_ERR_INVALID_ARG;
    hgemm_dev::Fp4QuantParams p;
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
    p.factor = d->factor;
    p.q = static_cast<uint8_t *>(d->q);
    p.ldq = d->ldq;
    p.scales = static_cast<uint8_t *>(d->scales);
    p.q_cols = static_cast<uint8_t *>(d->q_cols);
    p.ldq_cols = d->ldq_cols;
    p.scales_cols = static_cast<uint8_t *>(d->scales_cols);
    p.col_rows = col_rows;
    p.row_tiles = ceil_div(d->rows, 128);
    const int64_t col_tiles = ceil_div(d->cols, 128), row_tiles = ceil_div(col_rows, 128);      // (per group: as many as the copy has room for)
    // A CTA walks the offsets before its first tile.  Beyond 64 groups that is worth sharing: it takes several tiles of its 128 rows, eight CTAs an SM in all.  Up to there one CTA a tile,
    // whose rounds end more evenly (both copies in nvfp4, bf16; eight an SM against one a tile: 16384 x 2048, 32 groups 42.5 and 38.6 us, 64 47.5 and 44.0, 128 53.2 and 55.9,
    // 256 76 and 93, 1024 269 and 505; 8192 x 7168, 32 groups 78 and 72, 96 93 and 101; 2048 x 4096, 32 groups 21.8 and 17.9, 96 53 and 51, 256 127 and 150).
    const int64_t per_row = d->groups > 64 ? std::min(col_tiles, std::max<int64_t>(1, int64_t(ctx->num_sms) * 8 / row_tiles)) : col_tiles;
    const void *fn = d->x_type == HGEMM_TYPE_F32 ? quantize_kernel<float>(d->blocks, d->format) : d->x_type == HGEMM_TYPE_F16 ? quantize_kernel<__half>(d->blocks, d->format)
                                                                                                                             : quantize_kernel<__nv_bfloat16>(d->blocks, d->format);
    const int smem = hgemm_dev::fp4_quant_smem(es, nv, by_cols);
    if (smem > 48 * 1024) {
        const cudaError_t e = cudaFuncSetAttribute(fn, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
        if (e != cudaSuccess) return cuda_fail(ctx, e);
    }
    void *args[1] = {&p};
    return launch(ctx, fn, dim3(unsigned(per_row), unsigned(row_tiles), unsigned(d->matrices)), hgemm_dev::kFp4QuantThreads, smem, 1, args, stream);
}

hgemm_status_t hgemm_fp4_dequantize(hgemm_ctx_t *ctx, int32_t format, int32_t out_type, int64_t matrices, int64_t rows, int64_t cols, const void *q, int64_t ldq, const void *scales,
                                    const float *factor, const int32_t *offsets, int32_t groups, void *out, int64_t ldo, void *stream)
{
    if (!ctx || !is_format(format) || !is_wide(out_type) || matrices < 1 || matrices > kMaxMatrices || rows < 0 || rows > 2 * kMaxDim || cols < 1 || cols > 2 * kMaxDim) return HGEMM_ERR_INVALID_ARG;
    if (offsets ? groups < 1 || groups > hgemm_dev::kFp4MaxGroups || matrices != 1 || rows > kMaxDim || !aligned4(offsets) : groups != 0) return HGEMM_ERR_INVALID_ARG;
    if ((format == HGEMM_FP4_NV) != (factor != nullptr) || (factor && !aligned4(factor))) return HGEMM_ERR_INVALID_ARG;
    if (ldq < ceil_div(cols, 2) || (ldq & 15) != 0 || ldo < cols) return HGEMM_ERR_INVALID_ARG;
    if (rows == 0) return HGEMM_OK;
    const int es = type_bytes(out_type);
    if (!q || !scales || !out || !aligned16(q) || !aligned16(scales) || (reinterpret_cast<uintptr_t>(out) % unsigned(es)) != 0) return HGEMM_ERR_INVALID_ARG;
    const int64_t col_tiles = ceil_div(cols, 128), row_tiles = ceil_div(offsets ? hgemm_fp8_padded_rows(rows, groups) : rows, 128);
    // One tile a CTA; several of one row tile where it walks the offsets first, eight CTAs an SM in all (16384 x 2048, eight an SM against one a tile: 1 group 16.1 and 16.5 us, 16
    // 16.3 and 17.3, 32 17.7 and 17.6, 128 22 and 26, 256 26 and 43, 1024 60 and 230; 2048 x 4096, 32 groups 8.4 and 7.7, 64 10.7 and 12.3).
    const int64_t walkers = offsets ? std::min(col_tiles, std::max<int64_t>(1, int64_t(ctx->num_sms) * 8 / row_tiles)) : col_tiles;
    if (row_tiles * walkers > 0x7fffffff) return HGEMM_ERR_UNSUPPORTED;       // (a grid's limit)
    hgemm_dev::Fp4DequantParams p;
    std::memset(&p, 0, sizeof(p));
    p.q = static_cast<const uint8_t *>(q);
    p.ldq = ldq;
    p.scales = static_cast<const uint8_t *>(scales);
    p.factor = factor;
    p.rows = rows;
    p.cols = cols;
    p.row_tiles = row_tiles;
    p.walkers = int32_t(walkers);
    p.vec_ok = aligned16(out) && (ldo * es) % 16 == 0 ? 1 : 0;
    p.out = out;
    p.ldo = ldo;
    p.offsets = offsets;
    p.groups = groups;
    using namespace hgemm_dev;
    const bool nv = format == HGEMM_FP4_NV;
    const void *fn = out_type == HGEMM_TYPE_F32   ? (nv ? reinterpret_cast<const void *>(fp4_dequantize_kernel<float, true>) : reinterpret_cast<const void *>(fp4_dequantize_kernel<float, false>))
                     : out_type == HGEMM_TYPE_F16 ? (nv ? reinterpret_cast<const void *>(fp4_dequantize_kernel<__half, true>) : reinterpret_cast<const void *>(fp4_dequantize_kernel<__half, false>))
                                                  : (nv ? reinterpret_cast<const void *>(fp4_dequantize_kernel<__nv_bfloat16, true>) : reinterpret_cast<const void *>(fp4_dequantize_kernel<__nv_bfloat16, false>));
    void *args[1] = {&p};
    return launch(ctx, fn, dim3(unsigned(row_tiles * walkers), unsigned(matrices), 1), kFp4DequantThreads, 0, 1, args, stream);
}

hgemm_status_t hgemm_fp4_planned_config(int32_t form, int64_t M, int64_t N, int64_t K, int32_t groups, int32_t num_sms, hgemm_fp4_config_t *out)
{
    if (!out || num_sms < 1) return HGEMM_ERR_INVALID_ARG;
    if (!legal_shape(form, M, N, K, groups)) return HGEMM_ERR_INVALID_ARG;
    *out = choose(form, M, N, K, groups, num_sms, 2);
    return HGEMM_OK;
}

hgemm_status_t hgemm_fp4_plan(hgemm_ctx_t *ctx, int32_t form, int64_t M, int64_t N, int64_t K, int32_t groups, int32_t format, int32_t out_type, hgemm_fp4_plan_t **out)
{
    if (!ctx || !out || !legal_shape(form, M, N, K, groups) || !is_format(format) || !is_wide(out_type)) return HGEMM_ERR_INVALID_ARG;
    if (ctx->free_status_slots.empty()) return HGEMM_ERR_ALLOC;
    // every kernel that the plan may be given takes all of the shared memory
    const hgemm_fp4_config_t each[4] = {{2, 256, 1, 0}, {2, 128, 1, 0}, {1, 128, 1, 0}, {1, 64, 1, 0}};
    for (const hgemm_fp4_config_t &c : each) {
        const cudaError_t e = cudaFuncSetAttribute(kernel_of(c, format), cudaFuncAttributeMaxDynamicSharedMemorySize, kSmemOptIn);
        if (e != cudaSuccess) return cuda_fail(ctx, e);
    }
    hgemm_fp4_plan_s *pl = new (std::nothrow) hgemm_fp4_plan_s;
    if (!pl) return HGEMM_ERR_ALLOC;
    pl->ctx = ctx;
    pl->form = form;
    pl->M = M;
    pl->N = N;
    pl->K = K;
    pl->groups = groups;
    pl->format = format;
    pl->out_type = out_type;
    pl->cfg = choose(form, M, N, K, groups, ctx->num_sms, type_bytes(out_type));
    try {
        ctx->fp4_plans.push_back(pl);
    } catch (const std::bad_alloc &) {
        delete pl;
        return HGEMM_ERR_ALLOC;
    }
    pl->status_slot = ctx->free_status_slots.back();
    ctx->free_status_slots.pop_back();
    *out = pl;
    return HGEMM_OK;
}

hgemm_status_t hgemm_fp4_plan_destroy(hgemm_fp4_plan_t *plan)
{
    if (!plan) return HGEMM_ERR_INVALID_ARG;
    hgemm_ctx_s *ctx = plan->ctx;
    auto it = std::find(ctx->fp4_plans.begin(), ctx->fp4_plans.end(), plan);
    if (it != ctx->fp4_plans.end()) ctx->fp4_plans.erase(it);
    ctx->free_status_slots.push_back(plan->status_slot);     // its capacity holds every slot: this cannot allocate
    delete plan;
    return HGEMM_OK;
}

hgemm_status_t hgemm_fp4_last_device_status(hgemm_fp4_plan_t *plan, uint32_t *code)
{
    if (!plan || !code) return HGEMM_ERR_INVALID_ARG;
    uint32_t v = 0;
    const hgemm_status_t st = hgemm_host::take_status_word(plan->ctx, plan->status_slot, &v);
    if (st != HGEMM_ERR_CUDA) *code = v;
    return st;
}

hgemm_status_t hgemm_fp4_debug_timeout_probe(hgemm_fp4_plan_t *plan, void *stream)
{
    return plan ? hgemm_host::launch_timeout_probe(plan->ctx, plan->status_slot, stream) : HGEMM_ERR_INVALID_ARG;
}

hgemm_status_t hgemm_fp4_plan_get_config(const hgemm_fp4_plan_t *plan, hgemm_fp4_config_t *out)
{
    if (!plan || !out) return HGEMM_ERR_INVALID_ARG;
    *out = plan->cfg;
    return HGEMM_OK;
}

hgemm_status_t hgemm_fp4_plan_set_config(hgemm_fp4_plan_t *plan, const hgemm_fp4_config_t *cfg)
{
    if (!plan || !cfg) return HGEMM_ERR_INVALID_ARG;
    if (!legal_config(*cfg)) return HGEMM_ERR_UNSUPPORTED;
    plan->cfg = *cfg;
    return HGEMM_OK;
}

hgemm_status_t hgemm_fp4_run(hgemm_fp4_plan_t *plan, const void *A, int64_t lda, const void *a_scales, const float *a_factor, const void *B, int64_t ldb, const void *b_scales,
                             const float *b_factor, void *C, int64_t ldc, const int32_t *offsets, int32_t accumulate, void *stream)
{
    return plan ? run_product<false>(*plan, A, lda, a_scales, a_factor, B, ldb, b_scales, b_factor, C, ldc, offsets, accumulate, stream) : HGEMM_ERR_INVALID_ARG;
}

} // extern "C"
