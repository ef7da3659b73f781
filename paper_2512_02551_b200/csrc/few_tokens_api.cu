// C ABI of the layer of experts for a few tokens (see include/hgemm_few_tokens.h): checks, launches.
#include <cuda_runtime.h>

#include <algorithm>
#include <cstring>

#include "../../include/hgemm_few_tokens.h"
#include "few_tokens_kernel.cuh"
#include "hgemm_context.h"

using hgemm_dev::FewParams;
using hgemm_dev::FewWeights;

namespace {

constexpr int32_t kMaxWidth = 1 << 20;

int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }
bool aligned16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }
bool aligned4(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 3u) == 0; }
bool is4(const hgemm_few_tokens_t &d) { return d.weights == HGEMM_WEIGHTS_NVFP4 || d.weights == HGEMM_WEIGHTS_MXFP4; }
int32_t chunk_of(const hgemm_few_tokens_t &d) { return is4(d) ? 128 : 32; }

bool legal(const hgemm_few_tokens_t &d)
{
    if (d.hidden < 1 || d.hidden > kMaxWidth || d.inner < 1 || d.inner > kMaxWidth || d.experts < 1 || d.experts > 1024 || d.top_k < 1 || d.top_k > 32) return false;
    if (d.activation != HGEMM_ACT_SILU && d.activation != HGEMM_ACT_SWIGLU) return false;
    if (d.type != HGEMM_TYPE_F16 && d.type != HGEMM_TYPE_BF16) return false;
    if (d.weights == HGEMM_WEIGHTS_F16) return d.type == HGEMM_TYPE_F16;
    if (d.weights == HGEMM_WEIGHTS_BF16) return d.type == HGEMM_TYPE_BF16;
    return is4(d);
}

int64_t h_stride(const hgemm_few_tokens_t &d) { return ceil_div(d.inner, chunk_of(d)) * chunk_of(d); }

bool fill(FewWeights *w, const hgemm_few_tokens_t &d, const hgemm_expert_weights_t &m, int32_t rows, int32_t depth)
{
    const bool four = is4(d);
    if (!m.values || (d.weights == HGEMM_WEIGHTS_NVFP4) != (m.factor != nullptr) || four != (m.scales != nullptr) || !aligned4(m.factor)) return false;
    if (four ? m.ld < ceil_div(depth, 2) || (m.ld & 15) != 0 || !aligned16(m.values) || !aligned16(m.scales) : m.ld < depth || (reinterpret_cast<uintptr_t>(m.values) & 1u) != 0) return false;
    w->values = static_cast<const uint8_t *>(m.values);
    w->ld = four ? m.ld : m.ld * 2;
    w->matrix = w->ld * rows;
    w->scales = static_cast<const uint8_t *>(m.scales);
    w->atoms = int32_t(ceil_div(depth, d.weights == HGEMM_WEIGHTS_NVFP4 ? 64 : 128));
    w->scale_matrix = ceil_div(rows, 128) * w->atoms * 512;
    w->factor = m.factor;
    w->rows = rows;
    w->depth = depth;
    w->align = aligned16(m.values) && w->ld % 16 == 0 ? 16 : aligned4(m.values) && w->ld % 4 == 0 ? 4 : 2;
    return true;
}

const void *up_kernel(const hgemm_few_tokens_t &d)
{
    using namespace hgemm_dev;
    const bool x16 = d.type == HGEMM_TYPE_F16;
    switch (d.weights) {
    case HGEMM_WEIGHTS_F16: return reinterpret_cast<const void *>(few_up_kernel<kFewF16, true>);
    case HGEMM_WEIGHTS_BF16: return reinterpret_cast<const void *>(few_up_kernel<kFewBf16, false>);
    case HGEMM_WEIGHTS_NVFP4: return x16 ? reinterpret_cast<const void *>(few_up_kernel<kFewNv, true>) : reinterpret_cast<const void *>(few_up_kernel<kFewNv, false>);
    default: return x16 ? reinterpret_cast<const void *>(few_up_kernel<kFewMx, true>) : reinterpret_cast<const void *>(few_up_kernel<kFewMx, false>);
    }
}

const void *down_kernel(const hgemm_few_tokens_t &d)
{
    using namespace hgemm_dev;
    const bool y16 = d.type == HGEMM_TYPE_F16;
    switch (d.weights) {
    case HGEMM_WEIGHTS_F16: return reinterpret_cast<const void *>(few_down_kernel<kFewF16, __half>);
    case HGEMM_WEIGHTS_BF16: return reinterpret_cast<const void *>(few_down_kernel<kFewBf16, __nv_bfloat16>);
    case HGEMM_WEIGHTS_NVFP4: return y16 ? reinterpret_cast<const void *>(few_down_kernel<kFewNv, __half>) : reinterpret_cast<const void *>(few_down_kernel<kFewNv, __nv_bfloat16>);
    default: return y16 ? reinterpret_cast<const void *>(few_down_kernel<kFewMx, __half>) : reinterpret_cast<const void *>(few_down_kernel<kFewMx, __nv_bfloat16>);
    }
}

hgemm_status_t launch(hgemm_ctx_s *ctx, const void *fn, unsigned grid, int threads, int smem, FewParams *p, void *stream)
{
    if (smem > 48 * 1024) {
        const cudaError_t e = cudaFuncSetAttribute(fn, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
        if (e != cudaSuccess) return cuda_fail(ctx, e);
    }
    cudaLaunchConfig_t lc;
    std::memset(&lc, 0, sizeof(lc));
    lc.gridDim = dim3(grid, 1, 1);
    lc.blockDim = dim3(unsigned(threads), 1, 1);
    lc.dynamicSmemBytes = size_t(smem);
    lc.stream = static_cast<cudaStream_t>(stream);
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    lc.attrs = attr;
    lc.numAttrs = ctx->dependent_launch ? 1 : 0;
    void *args[1] = {p};
    const cudaError_t e = cudaLaunchKernelExC(&lc, fn, args);
    return e == cudaSuccess ? HGEMM_OK : cuda_fail(ctx, e);
}

// Warps that share a contraction of `chunks` chunks: as many as leave each the four chunks that it fetches together, so that rounds of work are short and the last one too.
int32_t slices_of(int64_t chunks, int64_t most)
{
    int32_t s = 1;
    while (s < 8 && s * 2 <= most && chunks >= int64_t(s) * 2 * 4) s *= 2;
    return s;
}

} // namespace

extern "C" {

int64_t hgemm_few_tokens_scratch(const hgemm_few_tokens_t *d, int64_t tokens)
{
    if (!d || !legal(*d) || tokens < 0 || tokens > HGEMM_FEW_TOKENS_MAX) return -1;
    return tokens * d->top_k * h_stride(*d) * 4;
}

hgemm_status_t hgemm_few_tokens(hgemm_ctx_t *ctx, const hgemm_few_tokens_t *d, int64_t tokens, const void *x, int64_t ldx, const hgemm_expert_weights_t *w1,
                                const hgemm_expert_weights_t *w2, const int32_t *indices, const float *weights, void *y, int64_t ldy, void *scratch, int64_t scratch_bytes, void *stream)
{
    if (!ctx || !d || !w1 || !w2 || !legal(*d) || tokens < 0 || tokens > HGEMM_FEW_TOKENS_MAX || ldx < d->hidden || ldy < d->hidden) return HGEMM_ERR_INVALID_ARG;
    if (tokens == 0) return HGEMM_OK;
    if (!x || !y || !indices || !weights || !scratch || (reinterpret_cast<uintptr_t>(x) & 1u) != 0 || (reinterpret_cast<uintptr_t>(y) & 1u) != 0) return HGEMM_ERR_INVALID_ARG;
    if (!aligned4(indices) || !aligned4(weights) || !aligned16(scratch) || scratch_bytes < hgemm_few_tokens_scratch(d, tokens)) return HGEMM_ERR_INVALID_ARG;
    FewParams p;
    std::memset(&p, 0, sizeof(p));
    p.gated = d->activation == HGEMM_ACT_SWIGLU ? 1 : 0;
    FewWeights up, down;
    std::memset(&up, 0, sizeof(up));
    std::memset(&down, 0, sizeof(down));
    if (!fill(&up, *d, *w1, d->inner * (p.gated ? 2 : 1), d->hidden) || !fill(&down, *d, *w2, d->hidden, d->inner)) return HGEMM_ERR_INVALID_ARG;
    p.x = x;
    p.ldx = ldx;
    p.x_vec = aligned16(x) && ldx % 8 == 0 ? 1 : 0;
    p.y = y;
    p.ldy = ldy;
    p.indices = indices;
    p.weights = weights;
    p.h = static_cast<__nv_bfloat16 *>(scratch);
    p.h_stride = h_stride(*d);
    p.inner = d->inner;
    p.experts = d->experts;
    p.top_k = d->top_k;
    p.tokens = int32_t(tokens);
    p.choices = int32_t(tokens * d->top_k);
    p.tiles = int32_t(ceil_div(d->inner, p.gated ? 8 : 16));
    const int lists = (hgemm_dev::few_list_bytes(p.experts, p.choices) + 15) & ~15;
    const int64_t entries = hgemm_dev::few_max_entries(p.experts, p.choices);

    p.w = up;
    const int64_t up_chunks = ceil_div(d->hidden, chunk_of(*d));
    p.slices = slices_of(up_chunks, 8);
    p.slice_chunks = int32_t(ceil_div(up_chunks, p.slices));
    const int64_t per_cta = hgemm_dev::kFewUpThreads / 32 / p.slices;
    const unsigned grid = unsigned(std::min<int64_t>(ceil_div(entries * p.tiles, per_cta), int64_t(ctx->num_sms) * 2));
    hgemm_status_t st = launch(ctx, up_kernel(*d), grid, hgemm_dev::kFewUpThreads, lists, &p, stream);
    if (st != HGEMM_OK) return st;

    p.w = down;
    const int64_t down_chunks = ceil_div(d->inner, chunk_of(*d));
    p.slices = slices_of(down_chunks, hgemm_dev::kFewMaxChoices / p.choices);
    p.slice_chunks = int32_t(ceil_div(down_chunks, p.slices));
    return launch(ctx, down_kernel(*d), unsigned(ceil_div(d->hidden, 16)), hgemm_dev::kFewDownThreads, lists + p.slices * p.choices * 64, &p, stream);
}

} // extern "C"
