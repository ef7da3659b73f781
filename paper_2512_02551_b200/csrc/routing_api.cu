// C ABI of the routing to experts (see include/hgemm_routing.h): argument checks and launches.
#include <cuda_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstring>

#include "../../include/hgemm_routing.h"
#include "hgemm_context.h"
#include "routing_kernel.cuh"

using hgemm_dev::RouteParams;

namespace {

constexpr int64_t kMaxTokens = int64_t(1) << 22, kMaxChoices = int64_t(1) << 26;

bool legal(const hgemm_routing_t &r)
{
    if (r.experts < 1 || r.experts > 512 || r.top_k < 1 || r.top_k > 32 || r.groups < 1 || r.groups > 32 || r.experts % r.groups != 0) return false;
    if (r.top_groups < 1 || r.top_groups > r.groups || r.top_k > r.top_groups * (r.experts / r.groups)) return false;
    if (r.score != HGEMM_SCORE_SOFTMAX && r.score != HGEMM_SCORE_SIGMOID) return false;
    if (r.group_score != HGEMM_GROUP_MAX && r.group_score != HGEMM_GROUP_TOP2) return false;
    if (r.groups > 1 && r.group_score == HGEMM_GROUP_TOP2 && r.experts / r.groups < 2) return false;
    return (r.renormalize == 0 || r.renormalize == 1) && std::isfinite(r.scale);
}

int type_bytes(int32_t t) { return t == HGEMM_TYPE_F32 ? 4 : t == HGEMM_TYPE_F16 || t == HGEMM_TYPE_BF16 ? 2 : 0; }

bool aligned(const void *p, int n) { return p != nullptr && (reinterpret_cast<uintptr_t>(p) % unsigned(n)) == 0; }

void fill(RouteParams *p, const hgemm_routing_t &r, int64_t tokens, const void *logits, int64_t ld, bool bias)
{
    std::memset(p, 0, sizeof(*p));
    p->logits = logits;
    p->tokens = tokens;
    p->ld = ld;
    p->experts = r.experts;
    p->top_k = r.top_k;
    p->sigmoid = r.score == HGEMM_SCORE_SIGMOID ? 1 : 0;
    p->groups = r.groups;
    p->top_groups = r.top_groups;
    p->group_size = r.experts / r.groups;
    p->inv_group = 1.0f / float(p->group_size);
    p->per_lane = (r.experts + 31) / 32;
    const int32_t lanes = p->group_size % p->per_lane == 0 ? p->group_size / p->per_lane : 0;
    p->group_lanes = (lanes & (lanes - 1)) == 0 ? lanes : 0;
    p->top2 = r.group_score == HGEMM_GROUP_TOP2 ? 1 : 0;
    p->renormalize = r.renormalize;
    p->by_logit = r.score == HGEMM_SCORE_SOFTMAX && !bias ? 1 : 0;
    p->scale = r.scale;
}

template <class T>
const void *route_fn(int32_t experts, bool backward)
{
    using namespace hgemm_dev;
#define HGEMM_ROUTE(N) (backward ? reinterpret_cast<const void *>(route_backward_kernel<T, N>) : reinterpret_cast<const void *>(route_kernel<T, N>))
    return experts <= 32 ? HGEMM_ROUTE(1) : experts <= 64 ? HGEMM_ROUTE(2) : experts <= 128 ? HGEMM_ROUTE(4) : experts <= 256 ? HGEMM_ROUTE(8) : HGEMM_ROUTE(16);
#undef HGEMM_ROUTE
}

const void *route_fn(int32_t type, int32_t experts, bool backward)
{
    return type == HGEMM_TYPE_F32 ? route_fn<float>(experts, backward) : type == HGEMM_TYPE_F16 ? route_fn<__half>(experts, backward) : route_fn<__nv_bfloat16>(experts, backward);
}

hgemm_status_t launch(hgemm_ctx_s *ctx, const void *fn, unsigned grid, int threads, size_t smem, unsigned cluster, void **args, void *stream)
{
    cudaLaunchConfig_t lc;
    std::memset(&lc, 0, sizeof(lc));
    lc.gridDim = dim3(grid, 1, 1);
    lc.blockDim = dim3(unsigned(threads), 1, 1);
    lc.dynamicSmemBytes = smem;
    lc.stream = static_cast<cudaStream_t>(stream);
    cudaLaunchAttribute attr[2];
    int n = 0;
    if (cluster > 0) {
        attr[n].id = cudaLaunchAttributeClusterDimension;
        attr[n].val.clusterDim.x = cluster;
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

unsigned route_grid(const hgemm_ctx_s *ctx, int64_t tokens)
{
    constexpr int64_t per = hgemm_dev::kRouteThreads / 32;
    return unsigned(std::min<int64_t>((tokens + per - 1) / per, int64_t(ctx->num_sms) * 64));
}

} // namespace

extern "C" {

hgemm_status_t hgemm_route(hgemm_ctx_t *ctx, const hgemm_routing_t *routing, int64_t tokens, const void *logits, int32_t type, int64_t ld, const float *bias,
                           float *weights, int32_t *indices, void *stream)
{
    if (!ctx || !routing || !legal(*routing) || tokens < 0 || tokens > kMaxTokens || type_bytes(type) == 0 || ld < routing->experts) return HGEMM_ERR_INVALID_ARG;
    if (routing->groups > 1 && routing->group_score == HGEMM_GROUP_TOP2 && routing->score == HGEMM_SCORE_SOFTMAX && !bias) return HGEMM_ERR_INVALID_ARG;
    if (tokens == 0) return HGEMM_OK;
    if (!aligned(logits, type_bytes(type)) || !aligned(weights, 4) || !aligned(indices, 4) || (bias && !aligned(bias, 4))) return HGEMM_ERR_INVALID_ARG;
    RouteParams p;
    fill(&p, *routing, tokens, logits, ld, bias != nullptr);
    p.bias = bias;
    // vectors of a lane's elements: 32 x 1, 2, 4, 8 or 16 experts (the kernel's slots, exactly filled), rows at multiples of 16 bytes
    const int32_t per = p.per_lane;
    p.vec_ok = routing->experts == 32 * per && (per & (per - 1)) == 0 && aligned(logits, 16) && (ld * type_bytes(type)) % 16 == 0 ? 1 : 0;
    p.weights = weights;
    p.indices = indices;
    void *args[1] = {&p};
    return launch(ctx, route_fn(type, routing->experts, false), route_grid(ctx, tokens), hgemm_dev::kRouteThreads, 0, 0, args, stream);
}

hgemm_status_t hgemm_route_backward(hgemm_ctx_t *ctx, const hgemm_routing_t *routing, int64_t tokens, const void *logits, int32_t type, int64_t ld, const int32_t *indices,
                                    const float *dweights, void *dlogits, int64_t ldd, void *stream)
{
    if (!ctx || !routing || !legal(*routing) || tokens < 0 || tokens > kMaxTokens || type_bytes(type) == 0 || ld < routing->experts || ldd < routing->experts) return HGEMM_ERR_INVALID_ARG;
    if (tokens == 0) return HGEMM_OK;
    if (!aligned(logits, type_bytes(type)) || !aligned(dlogits, type_bytes(type)) || !aligned(indices, 4) || !aligned(dweights, 4)) return HGEMM_ERR_INVALID_ARG;
    RouteParams p;
    fill(&p, *routing, tokens, logits, ld, false);
    p.chosen = indices;
    p.dweights = dweights;
    p.dlogits = dlogits;
    p.ldd = ldd;
    void *args[1] = {&p};
    return launch(ctx, route_fn(type, routing->experts, true), route_grid(ctx, tokens), hgemm_dev::kRouteThreads, 0, 0, args, stream);
}

hgemm_status_t hgemm_route_sort(hgemm_ctx_t *ctx, const int32_t *indices, int64_t count, int32_t experts, int32_t *offsets, int32_t *order, int32_t *position, void *stream)
{
    if (!ctx || count < 0 || count > kMaxChoices || experts < 1 || experts > 1024 || !aligned(offsets, 4)) return HGEMM_ERR_INVALID_ARG;
    if (count > 0 && (!aligned(indices, 4) || !aligned(order, 4) || !aligned(position, 4))) return HGEMM_ERR_INVALID_ARG;
    using namespace hgemm_dev;
    int ctas = 1;
    while (ctas < kSortMaxCtas && count > int64_t(ctas) * 4096) ctas *= 2;
    SortParams p;
    p.indices = indices;
    p.count = int32_t(count);
    p.experts = experts;
    p.bits = 1;
    while ((experts >> p.bits) != 0) ++p.bits;
    const int64_t warps = int64_t(ctas) * kSortWarps;
    p.run = int32_t(((count + warps - 1) / warps + 31) / 32 * 32);
    p.offsets = offsets;
    p.order = order;
    p.position = position;
    const size_t smem = size_t(kSortWarps * experts + 2 * experts + kSortWarps) * 4;
    cudaError_t e = cudaFuncSetAttribute(route_sort_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (kSortWarps * 1024 + 2 * 1024 + kSortWarps) * 4);
    if (e == cudaSuccess) e = cudaFuncSetAttribute(route_sort_kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
    if (e != cudaSuccess) return cuda_fail(ctx, e);
    void *args[1] = {&p};
    return launch(ctx, reinterpret_cast<const void *>(route_sort_kernel), unsigned(ctas), kSortThreads, smem, unsigned(ctas), args, stream);
}

} // extern "C"
