// Routing of tokens to experts (see include/hgemm_routing.h).
//
// hgemm_route: one warp per token, its experts in registers, consecutive ones in one lane.  A value becomes an unsigned key in the same
// order, so that a maximum over the warp is one redux instruction; the lowest lane that has it holds the lowest index.  Groups that
// are whole lanes, a power of two of them, find their best values all at once by shuffles among those lanes.  Bound by
// instruction issue (top_k rounds of redux, ballot and a scan of the lane's slots; an instruction in 76 % of the active cycles at
// 16384 x 128), not by the logits' bytes.  The gradient issues in 66 % of them and waits for its 2-byte loads.
//
// hgemm_route_sort: a stable counting sort in one launch.  The CTAs of one cluster divide the choices into consecutive runs, one per
// warp; per-warp histograms, prefix sums over warps, CTAs (through distributed shared memory) and experts give every run its
// first place for every expert, and each warp then places its run in order.  It has 16 SMs, which issue in 52 % of the active cycles.
//
// Measured (B200): 16384 tokens, 8 of 128 experts: choice 11.8 us, order 11.1 us, gradient 7.8 us; 256 experts in 8 groups, sigmoid: choice
// 23 us; 33 tokens: 4.2 and 3.8 us.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <stdint.h>

#include "hgemm_device.cuh"

namespace hgemm_dev {

constexpr int kRouteThreads = 128;
constexpr int kSortThreads = 1024;
constexpr int kSortWarps = kSortThreads / 32;
constexpr int kSortMaxCtas = 16;                   // one cluster
constexpr int kSortAhead = 4;                      // rounds of 32 choices whose indices a warp fetches together

struct RouteParams {
    const void *logits;
    int64_t tokens, ld, ldd;
    int32_t experts, top_k, sigmoid, groups, top_groups, group_size, top2, renormalize, by_logit;   // by_logit: v = l
    int32_t per_lane, group_lanes, vec_ok;   // experts of a lane; lanes of a group (0: groups do not consist of a power of two of lanes); rows may be read in vectors
    float scale, inv_group;
    const float *bias;
    float *weights;
    int32_t *indices;
    const int32_t *chosen;
    const float *dweights;
    void *dlogits;
};

// Unsigned keys in the order of the floats (-0 as +0, NaN as -infinity); 0 is below all of them.
__device__ __forceinline__ uint32_t order_key(float v)
{
    if (!(v == v)) v = __int_as_float(0xff800000);
    const uint32_t b = __float_as_uint(v + 0.0f);
    return b ^ ((b >> 31) ? 0xffffffffu : 0x80000000u);
}
__device__ __forceinline__ float key_value(uint32_t k) { return __uint_as_float(k ^ ((k >> 31) ? 0x80000000u : 0xffffffffu)); }
constexpr uint32_t kKeyLowest = 0x007fffffu;           // -infinity

__device__ __forceinline__ float route_load(const float *p) { return *p; }
__device__ __forceinline__ float route_load(const __half *p) { return __half2float(*p); }
__device__ __forceinline__ float route_load(const __nv_bfloat16 *p) { return __bfloat162float(*p); }
__device__ __forceinline__ void route_store(float *p, float v) { *p = v; }
__device__ __forceinline__ void route_store(__half *p, float v) { *p = __float2half_rn(v); }
__device__ __forceinline__ void route_store(__nv_bfloat16 *p, float v) { *p = __float2bfloat16_rn(v); }

__device__ __forceinline__ float warp_max(float v)
{
#pragma unroll
    for (int d = 16; d >= 1; d >>= 1) v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, d));
    return v;
}
__device__ __forceinline__ float warp_sum(float v)
{
#pragma unroll
    for (int d = 16; d >= 1; d >>= 1) v += __shfl_xor_sync(0xffffffffu, v, d);
    return v;
}

// Score of a logit; softmax: m the row's maximum, sum that of the exponentials.
__device__ __forceinline__ float route_score(float l, bool sigmoid, float m, float sum)
{
    if (sigmoid) return 1.0f / (1.0f + expf(-l));
    return m == __int_as_float(0xff800000) ? 0.0f : expf(l - m) / sum;
}

// NPL: slots per lane (experts <= 32 NPL).
template <class T, int NPL>
__global__ void __launch_bounds__(kRouteThreads)
route_kernel(const RouteParams p)
{
    grid_launch_dependents();
    grid_dependency_wait();
    const int32_t lane = static_cast<int32_t>(lane_id());
    const bool sigmoid = p.sigmoid != 0;
    for (int64_t t = blockIdx.x * static_cast<int64_t>(kRouteThreads / 32) + (threadIdx.x >> 5); t < p.tokens; t += gridDim.x * static_cast<int64_t>(kRouteThreads / 32)) {
        const T *row = static_cast<const T *>(p.logits) + t * p.ld;
        const int32_t e0 = lane * p.per_lane, mine_n = min(p.per_lane, p.experts - e0);        // this lane's experts: e0 .. e0 + mine_n - 1 (none: <= 0)
        float l[NPL];
        if (p.vec_ok) {                                 // rows of NPL elements per lane, aligned
            constexpr int kBytes = NPL * static_cast<int>(sizeof(T));
            __align__(16) T t[NPL];
            if constexpr (kBytes >= 16) {
#pragma unroll
                for (int i = 0; i < kBytes / 16; ++i) reinterpret_cast<uint4 *>(t)[i] = reinterpret_cast<const uint4 *>(row + e0)[i];
            } else if constexpr (kBytes == 8) {
                *reinterpret_cast<uint2 *>(t) = *reinterpret_cast<const uint2 *>(row + e0);
            } else {
#pragma unroll
                for (int i = 0; i < NPL; ++i) t[i] = row[e0 + i];
            }
#pragma unroll
            for (int i = 0; i < NPL; ++i) l[i] = route_load(t + i);
        } else {
#pragma unroll
            for (int i = 0; i < NPL; ++i) l[i] = i < mine_n ? route_load(row + e0 + i) : __int_as_float(0xff800000);
        }
        float m = 0.0f, sum = 1.0f;
        if (!sigmoid) {
            m = __int_as_float(0xff800000);
#pragma unroll
            for (int i = 0; i < NPL; ++i) m = fmaxf(m, l[i]);
            m = warp_max(m);
            sum = 0.0f;
#pragma unroll
            for (int i = 0; i < NPL; ++i)
                if (i < mine_n) sum += expf(l[i] - m);
            sum = warp_sum(sum);
        }
        uint32_t key[NPL];
#pragma unroll
        for (int i = 0; i < NPL; ++i) {
            float v = l[i];
            if (!p.by_logit) {
                v = route_score(l[i], sigmoid, m, sum);
                if (p.bias != nullptr && i < mine_n) v += p.bias[e0 + i];
            }
            key[i] = i < mine_n ? order_key(v) : 0u;
        }
        if (p.groups > 1) {
            uint32_t of_lane = 0, kept = 0;             // lane g: key of group g's value; bit g: the group stays
            if (p.group_lanes > 0) {
                uint32_t k1 = 0, k2 = 0;                // the two largest keys of this lane, then of its group's lanes
#pragma unroll
                for (int i = 0; i < NPL; ++i) {
                    k2 = max(k2, min(k1, key[i]));
                    k1 = max(k1, key[i]);
                }
                for (int d = 1; d < p.group_lanes; d <<= 1) {
                    const uint32_t o1 = __shfl_xor_sync(0xffffffffu, k1, d), o2 = __shfl_xor_sync(0xffffffffu, k2, d);
                    k2 = max(min(k1, o1), max(k2, o2));
                    k1 = max(k1, o1);
                }
                if (p.top2) k1 = order_key(key_value(k1) + key_value(max(k2, kKeyLowest)));
                of_lane = __shfl_sync(0xffffffffu, k1, (lane * p.group_lanes) & 31);
                if (lane >= p.groups) of_lane = 0;
            } else {
                for (int32_t g = 0; g < p.groups; ++g) {
                    uint32_t k1 = 0, k2 = 0;
#pragma unroll
                    for (int i = 0; i < NPL; ++i) {
                        const int32_t e = e0 + i;
                        const uint32_t k = e >= g * p.group_size && e < (g + 1) * p.group_size ? key[i] : 0u;
                        k2 = max(k2, min(k1, k));
                        k1 = max(k1, k);
                    }
                    uint32_t best = __reduce_max_sync(0xffffffffu, k1);
                    if (p.top2) {
                        const int owner = __ffs(__ballot_sync(0xffffffffu, k1 == best)) - 1;
                        const uint32_t second = __reduce_max_sync(0xffffffffu, lane == owner ? k2 : k1);
                        best = order_key(key_value(best) + key_value(max(second, kKeyLowest)));
                    }
                    if (lane == g) of_lane = best;
                }
            }
            for (int32_t j = 0; j < p.top_groups; ++j) {
                const uint32_t best = __reduce_max_sync(0xffffffffu, of_lane);
                const int g = __ffs(__ballot_sync(0xffffffffu, of_lane == best)) - 1;
                kept |= 1u << g;
                if (lane == g) of_lane = 0;
            }
#pragma unroll
            for (int i = 0; i < NPL; ++i) {
                const int32_t g = static_cast<int32_t>((static_cast<float>(e0 + i) + 0.5f) * p.inv_group);      // (e0 + i) / group_size: below 512, off by less than half
                if (i < mine_n && !((kept >> g) & 1u)) key[i] = kKeyLowest;
            }
        }
        int32_t mine = 0;                               // lane j: the j-th choice
        for (int32_t j = 0; j < p.top_k; ++j) {
            uint32_t k = key[0];
            int32_t slot = 0;
#pragma unroll
            for (int i = 1; i < NPL; ++i)
                if (key[i] > k) { k = key[i]; slot = i; }
            const uint32_t best = __reduce_max_sync(0xffffffffu, k);
            const int owner = __ffs(__ballot_sync(0xffffffffu, k == best)) - 1;
            const int32_t e = __shfl_sync(0xffffffffu, e0 + slot, owner);
            if (lane == j) mine = e;
#pragma unroll
            for (int i = 0; i < NPL; ++i)
                if (lane == owner && i == slot) key[i] = 0u;
        }
        float s = 0.0f;
        if (lane < p.top_k) s = route_score(route_load(row + mine), sigmoid, m, sum);
        if (p.renormalize) s = s / (warp_sum(s) + 1e-20f);
        if (lane < p.top_k) {
            p.weights[t * p.top_k + lane] = s * p.scale;
            p.indices[t * p.top_k + lane] = mine;
        }
    }
}

// dl from dw: with S = sum of the chosen scores + 1e-20 and w = s / S,  ds_j = scale (dw_j - sum_i dw_i w_i) / S  (renormalised)  or
// scale dw_j;  sigmoid: dl = ds s (1 - s);  softmax: dl = s (ds - sum_i s_i ds_i).  One warp per token; lane j holds choice j.
template <class T, int NPL>
__global__ void __launch_bounds__(kRouteThreads)
route_backward_kernel(const RouteParams p)
{
    grid_launch_dependents();
    grid_dependency_wait();
    const int32_t lane = static_cast<int32_t>(lane_id());
    const bool sigmoid = p.sigmoid != 0;
    for (int64_t t = blockIdx.x * static_cast<int64_t>(kRouteThreads / 32) + (threadIdx.x >> 5); t < p.tokens; t += gridDim.x * static_cast<int64_t>(kRouteThreads / 32)) {
        const T *row = static_cast<const T *>(p.logits) + t * p.ld;
        T *out = static_cast<T *>(p.dlogits) + t * p.ldd;
        int32_t e = -1;
        float dw = 0.0f;
        if (lane < p.top_k) {
            e = p.chosen[t * p.top_k + lane];
            dw = p.dweights[t * p.top_k + lane] * p.scale;
        }
        const bool has = e >= 0 && e < p.experts;
        float x[NPL];                                   // softmax: the scores
        float m = 0.0f, sum = 1.0f;
        if (!sigmoid) {
            m = __int_as_float(0xff800000);
#pragma unroll
            for (int i = 0; i < NPL; ++i) {
                x[i] = i * 32 + lane < p.experts ? route_load(row + i * 32 + lane) : __int_as_float(0xff800000);
                m = fmaxf(m, x[i]);
            }
            m = warp_max(m);
            sum = 0.0f;
#pragma unroll
            for (int i = 0; i < NPL; ++i) {
                x[i] = i * 32 + lane < p.experts && m != __int_as_float(0xff800000) ? expf(x[i] - m) : 0.0f;
                sum += x[i];
            }
            sum = warp_sum(sum);
        }
        const float s = has ? route_score(route_load(row + e), sigmoid, m, sum) : 0.0f;
        float d = has ? dw : 0.0f;
        if (p.renormalize) {
            // dw_j - sum_i dw_i w_i, taken from the first choice's dw: with r = dw_0 it is  (dw_j - r) - (sum_i s_i (dw_i - r) - r (S - sum s)) / S.
            // Equal dw (one choice above all) then leave exactly 0 where S = sum s in 32 bits, not the rounding of dw s / s, which the
            // division by S would blow up; and the two sums do not wait for one another.
            const float r = __shfl_sync(0xffffffffu, d, 0);
            const float sum_s = warp_sum(s), moved = warp_sum(s * (d - r)), total = sum_s + 1e-20f;
            d = has ? ((d - r) - (moved - r * (total - sum_s)) / total) / total : 0.0f;
        }
        if (sigmoid) {
#pragma unroll
            for (int i = 0; i < NPL; ++i)
                if (i * 32 + lane < p.experts) route_store(out + i * 32 + lane, 0.0f);
            __syncwarp();
            if (has) route_store(out + e, d * s * (1.0f - s));
        } else {
            const float dot = warp_sum(s * d), inv = sum > 0.0f ? 1.0f / sum : 0.0f;
#pragma unroll
            for (int i = 0; i < NPL; ++i)
                if (i * 32 + lane < p.experts) route_store(out + i * 32 + lane, -(x[i] * inv) * dot);
            __syncwarp();
            if (has) route_store(out + e, s * (d - dot));
        }
    }
}

struct SortParams {
    const int32_t *indices;
    int32_t count, experts, run;       // run: choices per warp, a multiple of 32
    int32_t bits;                      // of the numbers 0 .. experts
    int32_t *offsets, *order, *position;
};

// The lanes whose code is this lane's: one ballot per bit.  (The match instruction compares value by value: some 30 cycles of the SM for
// each warp, two thirds of the sort's time.)
__device__ __forceinline__ uint32_t same_code(uint32_t code, int32_t bits)
{
    uint32_t peers = 0xffffffffu;
    for (int32_t b = 0; b < bits; ++b) {
        const bool one = (code >> b) & 1u;
        const uint32_t ones = __ballot_sync(0xffffffffu, one);
        peers &= one ? ones : ~ones;
    }
    return peers;
}

__global__ void __launch_bounds__(kSortThreads)
route_sort_kernel(const SortParams p)
{
    extern __shared__ int32_t s_sort[];                 // [kSortWarps][experts] histograms, then [experts] totals of this CTA, [experts] first places, [33]
    int32_t *hist = s_sort, *total = s_sort + kSortWarps * p.experts, *first = total + p.experts, *partial = first + p.experts;
    grid_launch_dependents();
    grid_dependency_wait();
    const int32_t tid = static_cast<int32_t>(threadIdx.x), warp = tid >> 5, lane = tid & 31;
    const int32_t rank = static_cast<int32_t>(cluster_ctarank()), ctas = static_cast<int32_t>(gridDim.x);
    for (int32_t i = tid; i < kSortWarps * p.experts; i += kSortThreads) hist[i] = 0;
    __syncthreads();
    int32_t *mine = hist + warp * p.experts;
    const int64_t begin = (static_cast<int64_t>(rank) * kSortWarps + warp) * p.run, end = min(begin + p.run, static_cast<int64_t>(p.count));
    for (int64_t i = begin; i < end; i += 32 * kSortAhead) {
        int32_t e[kSortAhead];
#pragma unroll
        for (int u = 0; u < kSortAhead; ++u) e[u] = i + u * 32 + lane < end ? p.indices[i + u * 32 + lane] : -1;
#pragma unroll
        for (int u = 0; u < kSortAhead; ++u)
            if (e[u] >= 0 && e[u] < p.experts) atomicAdd(mine + e[u], 1);       // counts: the order of the additions does not show
    }
    __syncthreads();
    for (int32_t e = tid; e < p.experts; e += kSortThreads) {
        int32_t sum = 0;
        for (int32_t w = 0; w < kSortWarps; ++w) {
            const int32_t n = hist[w * p.experts + e];
            hist[w * p.experts + e] = sum;
            sum += n;
        }
        total[e] = sum;
    }
    cluster_arrive();
    cluster_wait();
    // thread e: expert e (experts <= threads); places before it: experts below, then the CTAs before this one
    int32_t all = 0, before = 0;
    if (tid < p.experts) {
        int32_t n[kSortMaxCtas];
#pragma unroll
        for (int r = 0; r < kSortMaxCtas; ++r)
            asm volatile("ld.shared::cluster.s32 %0, [%1];" : "=r"(n[r]) : "r"(mapa(smem_addr(total + tid), static_cast<uint32_t>(min(r, ctas - 1)))) : "memory");
#pragma unroll
        for (int r = 0; r < kSortMaxCtas; ++r) {
            if (r < ctas) all += n[r];
            if (r < rank) before += n[r];
        }
    }
    int32_t scan = all;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
        const int32_t x = __shfl_up_sync(0xffffffffu, scan, d);
        if (lane >= d) scan += x;
    }
    if (lane == 31) partial[warp] = scan;
    __syncthreads();
    if (warp == 0) {
        int32_t x = partial[lane];
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
            const int32_t y = __shfl_up_sync(0xffffffffu, x, d);
            if (lane >= d) x += y;
        }
        partial[lane] = x;
    }
    __syncthreads();
    const int32_t offset = scan - all + (warp > 0 ? partial[warp - 1] : 0);
    const int32_t placed = partial[kSortWarps - 1];
    if (tid < p.experts) {
        first[tid] = offset + before;
        if (rank == 0) {
            p.offsets[tid] = offset;
            if (tid == p.experts - 1) p.offsets[p.experts] = placed;
        }
    }
    __syncthreads();
    for (int64_t i = begin; i < end; i += 32 * kSortAhead) {
        int32_t es[kSortAhead];
#pragma unroll
        for (int u = 0; u < kSortAhead; ++u) es[u] = i + u * 32 + lane < end ? p.indices[i + u * 32 + lane] : -1;
#pragma unroll
        for (int u = 0; u < kSortAhead; ++u) {
            if (i + u * 32 >= end) break;               // (the same for the whole warp)
            const int64_t slot = i + u * 32 + lane;
            const bool valid = es[u] >= 0 && es[u] < p.experts;
            const int32_t e = valid ? es[u] : -1;
            const uint32_t peers = same_code(static_cast<uint32_t>(valid ? e : p.experts), p.bits);
            if (valid) {
                const int32_t place = first[e] + mine[e] + __popc(peers & ((1u << lane) - 1u));
                p.order[place] = static_cast<int32_t>(slot);
                p.position[slot] = place;
            } else if (slot < end) {
                p.position[slot] = -1;
            }
            __syncwarp();
            if (valid && lane == __ffs(peers) - 1) mine[e] += __popc(peers);
            __syncwarp();
        }
    }
    for (int64_t i = placed + static_cast<int64_t>(rank) * kSortThreads + tid; i < p.count; i += static_cast<int64_t>(ctas) * kSortThreads) p.order[i] = -1;
    cluster_arrive();                                   // no CTA leaves while another may still read its totals
    cluster_wait();
}

} // namespace hgemm_dev
