// C ABI of the layer of experts for a few tokens (see include/hgemm_few_tokens.h): checks, launches.
#include <cuda_runtime.h>

#include <algorithm>
#include <cstring>

#include "../../include/hgemm_few_tokens.h"
#include "few_digits_kernel.cuh"
#include "few_tokens_kernel.cuh"
#include "hgemm_context.h"

using hgemm_dev::FewParams;
using hgemm_dev::FewWeights;

namespace {

constexpr int32_t kMaxWidth = 1 << 20;
constexpr int kMaxX = 64 * 1024;                 // shared memory of the 16-bit kernels' first launch for x: two CTAs share an SM
constexpr int kDigits = hgemm_dev::kDigits;

int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }
int64_t up_to(int64_t a, int64_t unit) { return ceil_div(a, unit) * unit; }
bool aligned16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }
bool aligned4(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 3u) == 0; }
bool is4(const hgemm_few_tokens_t &d) { return d.weights == HGEMM_WEIGHTS_NVFP4 || d.weights == HGEMM_WEIGHTS_MXFP4; }
int32_t format_of(const hgemm_few_tokens_t &d) { return d.weights == HGEMM_WEIGHTS_NVFP4 ? HGEMM_FP4_NV : HGEMM_FP4_MX; }
int32_t up_rows(const hgemm_few_tokens_t &d) { return d.activation == HGEMM_ACT_SWIGLU ? 2 * d.inner : d.inner; }

bool legal(const hgemm_few_tokens_t &d)
{
    if (d.hidden < 1 || d.hidden > kMaxWidth || d.inner < 1 || d.inner > kMaxWidth || d.experts < 1 || d.experts > 1024 || d.top_k < 1 || d.top_k > 32) return false;
    if (d.activation != HGEMM_ACT_SILU && d.activation != HGEMM_ACT_SWIGLU) return false;
    if (d.type != HGEMM_TYPE_F16 && d.type != HGEMM_TYPE_BF16) return false;
    if (d.weights == HGEMM_WEIGHTS_F16) return d.type == HGEMM_TYPE_F16;
    if (d.weights == HGEMM_WEIGHTS_BF16) return d.type == HGEMM_TYPE_BF16;
    return is4(d);
}

// ---- 16-bit weights ------------------------------------------------------------------------------------------------

// h of a choice in scratch memory: whole chunks, in two parts
int64_t h_stride(const hgemm_few_tokens_t &d) { return up_to(d.inner, hgemm_dev::kFewChunk); }

FewWeights weights16(const hgemm_expert_weights_t &m, int32_t rows, int32_t depth)
{
    FewWeights w;
    w.values = static_cast<const uint8_t *>(m.values);
    w.ld = m.ld * 2;
    w.matrix = w.ld * rows;
    w.rows = rows;
    w.depth = depth;
    w.align = aligned16(m.values) && w.ld % 16 == 0 ? 16 : aligned4(m.values) && w.ld % 4 == 0 ? 4 : 2;
    return w;
}

template <class T>
const void *up_kernel(int align)
{
    using namespace hgemm_dev;
    return align == 16 ? reinterpret_cast<const void *>(few_up_kernel<T, 16>) : align == 4 ? reinterpret_cast<const void *>(few_up_kernel<T, 4>) : reinterpret_cast<const void *>(few_up_kernel<T, 2>);
}

template <class T>
const void *down_kernel(int align)
{
    using namespace hgemm_dev;
    return align == 16 ? reinterpret_cast<const void *>(few_down_kernel<T, 16>) : align == 4 ? reinterpret_cast<const void *>(few_down_kernel<T, 4>) : reinterpret_cast<const void *>(few_down_kernel<T, 2>);
}

hgemm_status_t launch(hgemm_ctx_s *ctx, const void *fn, dim3 grid, int threads, int smem, void *params, void *stream, int cluster = 1)
{
    cudaLaunchConfig_t lc;
    std::memset(&lc, 0, sizeof(lc));
    lc.gridDim = grid;
    lc.blockDim = dim3(unsigned(threads), 1, 1);
    lc.dynamicSmemBytes = size_t(smem);
    lc.stream = static_cast<cudaStream_t>(stream);
    cudaLaunchAttribute attr[2];
    unsigned n = 0;
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
    lc.numAttrs = n;
    void *args[1] = {params};
    const cudaError_t e = cudaLaunchKernelExC(&lc, fn, args);
    return e == cudaSuccess ? HGEMM_OK : cuda_fail(ctx, e);
}

struct Call {
    int64_t tokens;
    const void *x;
    int64_t ldx;
    const int32_t *indices;
    const float *weights;
    void *y;
    int64_t ldy;
    uint8_t *scratch;
    void *stream;
};

// Shared memory of the second launch: lists, the choices' weights, slices of 16 sums a choice.
constexpr int down_smem(int experts, int choices, int slices) { return hgemm_dev::few_list_bytes(experts, choices) + 4 * ((choices + 3) & ~3) + slices * choices * 64; }

// Once a context and type: the shared memory that any call may ask for.  The limit is the kernel's, whoever launches it: it is never lowered, so that a call on another thread is not
// refused.  (What a kernel may have unasked, 48 KB, counts its static shared memory too.)
template <class T>
hgemm_status_t prepare16(hgemm_ctx_s *ctx)
{
    constexpr int kLists = hgemm_dev::few_list_bytes(1024, hgemm_dev::kFewMaxChoices), kDown = down_smem(1024, hgemm_dev::kFewMaxChoices, 1);
    static_assert(kLists + kMaxX <= 100 * 1024 && kDown <= 224 * 1024, "shared memory of a CTA");
    for (const int align : {16, 4, 2}) {
        cudaError_t e = cudaFuncSetAttribute(up_kernel<T>(align), cudaFuncAttributeMaxDynamicSharedMemorySize, kLists + kMaxX);
        if (e == cudaSuccess) e = cudaFuncSetAttribute(down_kernel<T>(align), cudaFuncAttributeMaxDynamicSharedMemorySize, kDown);
        if (e != cudaSuccess) return cuda_fail(ctx, e);
    }
    ctx->few16_ready[std::is_same<T, __half>::value ? 0 : 1] = true;
    return HGEMM_OK;
}

hgemm_status_t run16(hgemm_ctx_s *ctx, const hgemm_few_tokens_t &d, const Call &c, const hgemm_expert_weights_t &w1, const hgemm_expert_weights_t &w2)
{
    const bool half = d.type == HGEMM_TYPE_F16;
    if (!ctx->few16_ready[half ? 0 : 1]) {
        const hgemm_status_t st = half ? prepare16<__half>(ctx) : prepare16<__nv_bfloat16>(ctx);
        if (st != HGEMM_OK) return st;
    }
    FewParams p;
    std::memset(&p, 0, sizeof(p));
    p.gated = d.activation == HGEMM_ACT_SWIGLU ? 1 : 0;
    p.x = c.x;
    p.ldx = c.ldx;
    p.x_vec = aligned16(c.x) && c.ldx % 8 == 0 ? 1 : 0;
    p.y = c.y;
    p.ldy = c.ldy;
    p.indices = c.indices;
    p.weights = c.weights;
    p.h_stride = int32_t(h_stride(d));
    p.inner = d.inner;
    p.experts = d.experts;
    p.top_k = d.top_k;
    p.tokens = int32_t(c.tokens);
    p.choices = int32_t(c.tokens * d.top_k);
    p.h = reinterpret_cast<__nv_bfloat16 *>(c.scratch);
    // launch 1 writes whole chunks of h (zeros beyond inner), eight tiles of 8 (SWIGLU) or 16 rows together
    p.groups = int32_t(ceil_div(p.h_stride, p.gated ? 64 : 128));
    p.fd_groups = hgemm_dev::make_fast_div(uint32_t(p.groups));
    const int lists = hgemm_dev::few_list_bytes(p.experts, p.choices);
    const int64_t entries = hgemm_dev::few_max_entries(p.experts, p.choices);

    // x of 8 choices at once, or as many chunks of it as fit
    p.w = weights16(w1, up_rows(d), d.hidden);
    p.piece = int32_t(std::min<int64_t>(up_to(d.hidden, hgemm_dev::kFewAhead * hgemm_dev::kFewChunk) * 16, kMaxX));
    p.most_slices = 8;
    const unsigned grid = unsigned(std::min<int64_t>(entries * p.groups * 8, int64_t(ctx->num_sms) * 2));
    const hgemm_status_t st = launch(ctx, half ? up_kernel<__half>(p.w.align) : up_kernel<__nv_bfloat16>(p.w.align), dim3(grid), hgemm_dev::kFewUpThreads, lists + p.piece, &p, c.stream);
    if (st != HGEMM_OK) return st;

    p.w = weights16(w2, d.hidden, d.inner);
    p.most_slices = 1;
    while (p.most_slices < 8 && p.most_slices * 2 * p.choices <= hgemm_dev::kFewMaxChoices) p.most_slices *= 2;
    // Few outputs: up to eight CTAs (a cluster) share 16 of them, as many as there are SMs for, each with two choices at least (bf16, hidden 64, inner 2048, 32 tokens of 8
    // among 64 experts: 39 us, with one CTA 101; hidden 1024, inner 1024, 16 tokens: 60 and 71; hidden 256, inner 2048, 1 token: four 16.7, eight 21.5, one 18.7).
    const int64_t tiles = ceil_div(d.hidden, 16);
    p.ranks = 1;
    while (p.ranks < 8 && tiles * p.ranks * 2 <= ctx->num_sms && p.ranks * 4 <= p.choices) p.ranks *= 2;
    return launch(ctx, half ? down_kernel<__half>(p.w.align) : down_kernel<__nv_bfloat16>(p.w.align), dim3(unsigned(tiles * p.ranks)), hgemm_dev::kFewDownThreads,
                  down_smem(p.experts, p.choices, p.most_slices), &p, c.stream, p.ranks);
}

// ---- 4-bit weights -------------------------------------------------------------------------------------------------

// Scratch memory: where its parts begin (multiples of 256 bytes).  Both products' digits share a place, and so do both products' results: each is used up before
// the second's is written.
struct Layout {
    int64_t position, place, x_factor, h_factor, digits, scales, results, bytes;
    int64_t ld_x, ld_h;        // bytes between digit rows
    int64_t ld_u, ld_z;        // results' rows, in numbers
};

Layout layout_of(const hgemm_few_tokens_t &d, int64_t choices)
{
    Layout l;
    int64_t at = 0;
    auto part = [&](int64_t bytes) {
        const int64_t here = at;
        at = up_to(at + bytes, 256);
        return here;
    };
    l.ld_x = up_to(ceil_div(d.hidden, 2), 16);
    l.ld_h = up_to(ceil_div(d.inner, 2), 16);
    l.ld_u = up_to(up_rows(d), 4);
    l.ld_z = up_to(d.hidden, 4);
    const int64_t rows = hgemm_fp8_padded_rows(choices * kDigits, d.experts);
    l.position = part(4 * choices);
    l.place = part(4 * choices);
    l.x_factor = part(4 * choices);
    l.h_factor = part(4 * choices);
    l.digits = part(choices * kDigits * std::max(l.ld_x, l.ld_h));
    l.scales = part(std::max(hgemm_fp4_scale_bytes(rows, d.hidden, format_of(d)), hgemm_fp4_scale_bytes(rows, d.inner, format_of(d))));
    l.results = part(choices * 4 * std::max(l.ld_u, l.ld_z));
    l.bytes = at;
    return l;
}

// Once a context: an SM that makes digits can take a CTA of the product too, which needs nearly all of its shared memory.
hgemm_status_t prepare4(hgemm_ctx_s *ctx)
{
    using namespace hgemm_dev;
    const void *const kernels[4] = {reinterpret_cast<const void *>(few_digits_kernel<true, true>), reinterpret_cast<const void *>(few_digits_kernel<true, false>),
                                    reinterpret_cast<const void *>(few_digits_kernel<false, true>), reinterpret_cast<const void *>(few_digits_kernel<false, false>)};
    for (const void *fn : kernels) {
        const cudaError_t e = cudaFuncSetAttribute(fn, cudaFuncAttributePreferredSharedMemoryCarveout, cudaSharedmemCarveoutMaxShared);
        if (e != cudaSuccess) return cuda_fail(ctx, e);
    }
    const hgemm_status_t st = hgemm_host::fp4_digits_prepare(ctx);
    if (st == HGEMM_OK) ctx->few_ready = true;
    return st;
}

hgemm_status_t run4(hgemm_ctx_s *ctx, const hgemm_few_tokens_t &d, const Call &c, const hgemm_expert_weights_t &w1, const hgemm_expert_weights_t &w2)
{
    using namespace hgemm_dev;
    if (!ctx->few_ready) {
        const hgemm_status_t st = prepare4(ctx);
        if (st != HGEMM_OK) return st;
    }
    const int64_t choices = c.tokens * d.top_k;
    const Layout l = layout_of(d, choices);
    const bool nv = d.weights == HGEMM_WEIGHTS_NVFP4;
    const int32_t format = format_of(d), gated = d.activation == HGEMM_ACT_SWIGLU ? 1 : 0;
    float *results = reinterpret_cast<float *>(c.scratch + l.results);

    // x as digits
    DigitParams p;
    std::memset(&p, 0, sizeof(p));
    p.x = c.x;
    p.ldx = c.ldx;
    p.x_half = d.type == HGEMM_TYPE_F16 ? 1 : 0;
    p.x_vec = (reinterpret_cast<uintptr_t>(c.x) & 7u) == 0 && c.ldx % 4 == 0 ? 1 : 0;
    p.depth = d.hidden;
    p.top_k = d.top_k;
    p.experts = d.experts;
    p.choices = int32_t(choices);
    p.indices = c.indices;
    p.position = reinterpret_cast<int32_t *>(c.scratch + l.position);
    p.place = reinterpret_cast<int32_t *>(c.scratch + l.place);
    p.q = c.scratch + l.digits;
    p.ldq = l.ld_x;
    p.scales = c.scratch + l.scales;
    p.atoms = int32_t(ceil_div(d.hidden, nv ? 64 : 128));
    p.factor = reinterpret_cast<float *>(c.scratch + l.x_factor);
    const void *first = nv ? reinterpret_cast<const void *>(few_digits_kernel<true, true>) : reinterpret_cast<const void *>(few_digits_kernel<false, true>);
    const void *second = nv ? reinterpret_cast<const void *>(few_digits_kernel<true, false>) : reinterpret_cast<const void *>(few_digits_kernel<false, false>);
    hgemm_status_t st = launch(ctx, first, dim3(unsigned(choices)),
                               kDigitThreads, 4 * d.experts, &p, c.stream);
    if (st != HGEMM_OK) return st;
    st = hgemm_host::fp4_digits_product(ctx, format, choices, up_rows(d), d.hidden, d.experts, p.q, l.ld_x, p.scales, w1.values, w1.ld, w1.scales, w1.factor, results, l.ld_u, c.indices,
                                        c.stream);
    if (st != HGEMM_OK) return st;

    // h as digits
    p.x = nullptr;
    p.u = results;
    p.ldu = l.ld_u;
    p.gated = gated;
    p.u_vec = !gated || d.inner % 4 == 0 ? 1 : 0;
    p.u_factor = p.factor;
    p.depth = d.inner;
    p.ldq = l.ld_h;
    p.atoms = int32_t(ceil_div(d.inner, nv ? 64 : 128));
    p.factor = reinterpret_cast<float *>(c.scratch + l.h_factor);
    st = launch(ctx, second, dim3(unsigned(choices)),
                kDigitThreads, 0, &p, c.stream);
    if (st != HGEMM_OK) return st;
    st = hgemm_host::fp4_digits_product(ctx, format, choices, d.hidden, d.inner, d.experts, p.q, l.ld_h, p.scales, w2.values, w2.ld, w2.scales, w2.factor, results, l.ld_z, c.indices,
                                        c.stream);
    if (st != HGEMM_OK) return st;

    CombineParams q;
    std::memset(&q, 0, sizeof(q));
    q.z = results;
    q.ldz = l.ld_z;
    q.factor = p.factor;
    q.position = p.position;
    q.weights = c.weights;
    q.top_k = d.top_k;
    q.hidden = d.hidden;
    q.y = c.y;
    q.ldy = c.ldy;
    q.y_vec = (reinterpret_cast<uintptr_t>(c.y) & 7u) == 0 && c.ldy % 4 == 0 ? 1 : 0;
    return launch(ctx, d.type == HGEMM_TYPE_F16 ? reinterpret_cast<const void *>(few_combine_kernel<__half>) : reinterpret_cast<const void *>(few_combine_kernel<__nv_bfloat16>),
                  dim3(unsigned(ceil_div(d.hidden, 4 * kCombineThreads)), unsigned(c.tokens)), kCombineThreads, 0, &q, c.stream);
}

bool legal_weights(const hgemm_few_tokens_t &d, const hgemm_expert_weights_t &m, int32_t depth)
{
    const bool four = is4(d);
    if (!m.values || (d.weights == HGEMM_WEIGHTS_NVFP4) != (m.factor != nullptr) || four != (m.scales != nullptr) || !aligned4(m.factor)) return false;
    if (four) return m.ld >= ceil_div(depth, 2) && (m.ld & 15) == 0 && aligned16(m.values) && aligned16(m.scales);
    return m.ld >= depth && (reinterpret_cast<uintptr_t>(m.values) & 1u) == 0;
}

} // namespace

extern "C" {

int64_t hgemm_few_tokens_scratch(const hgemm_few_tokens_t *d, int64_t tokens)
{
    if (!d || !legal(*d) || tokens < 0 || tokens > HGEMM_FEW_TOKENS_MAX) return -1;
    const int64_t choices = tokens * d->top_k;
    if (choices == 0) return 0;
    return is4(*d) ? layout_of(*d, choices).bytes : choices * h_stride(*d) * 4;
}

hgemm_status_t hgemm_few_tokens(hgemm_ctx_t *ctx, const hgemm_few_tokens_t *d, int64_t tokens, const void *x, int64_t ldx, const hgemm_expert_weights_t *w1,
                                const hgemm_expert_weights_t *w2, const int32_t *indices, const float *weights, void *y, int64_t ldy, void *scratch, int64_t scratch_bytes, void *stream)
{
    if (!ctx || !d || !w1 || !w2 || !legal(*d) || tokens < 0 || tokens > HGEMM_FEW_TOKENS_MAX || ldx < d->hidden || ldy < d->hidden) return HGEMM_ERR_INVALID_ARG;
    if (tokens == 0) return HGEMM_OK;
    if (!x || !y || !indices || !weights || !scratch || (reinterpret_cast<uintptr_t>(x) & 1u) != 0 || (reinterpret_cast<uintptr_t>(y) & 1u) != 0) return HGEMM_ERR_INVALID_ARG;
    if (!aligned4(indices) || !aligned4(weights) || !aligned16(scratch) || scratch_bytes < hgemm_few_tokens_scratch(d, tokens)) return HGEMM_ERR_INVALID_ARG;
    if (!legal_weights(*d, *w1, d->hidden) || !legal_weights(*d, *w2, d->inner)) return HGEMM_ERR_INVALID_ARG;
    const Call c{tokens, x, ldx, indices, weights, y, ldy, static_cast<uint8_t *>(scratch), stream};
    return is4(*d) ? run4(ctx, *d, c, *w1, *w2) : run16(ctx, *d, c, *w1, *w2);
}

} // extern "C"
