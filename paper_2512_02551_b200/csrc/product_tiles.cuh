// Tiles of the products with block scales: their numbering over a result, or over the results of groups whose extents live on the device, and the
// rounding of results.
//
// Params (of each kernel) has the members that product_tile and scan_groups read: rows_p, rows_q, kblocks, tiles_p, tiles_q, raster, groups, ragged,
// rows_ragged, k_capacity, offsets, and the divisors fd_other, fd_group, fd_sweep, fd_raster, fd_last.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <stdint.h>

#include "hgemm_device.cuh"

namespace hgemm_dev {

// which side of the tile grid follows the groups' offsets
enum : int32_t { kRaggedNone = 0, kRaggedP = 1, kRaggedQ = 2, kRaggedK = 3 };

struct ProductTile {
    int32_t group, p0, p_end, q0, q_end, kb0, kbn;
};

// The tile with number w; whole (converged) warp.  pre: prefix sums over the groups (tiles, or blocks for kRaggedK); off: clamped offsets.
template <int TP, int TQ, class Params>
__device__ __forceinline__ ProductTile product_tile(int32_t w, const Params &p, const int32_t *pre, const int32_t *off, uint32_t lane)
{
    ProductTile t;
    t.group = 0;
    t.kb0 = 0;
    t.kbn = p.kblocks;
    t.p_end = p.rows_p;
    t.q_end = p.rows_q;
    if (p.ragged == kRaggedP || p.ragged == kRaggedQ) {
        const int32_t other = p.ragged == kRaggedP ? p.tiles_q : p.tiles_p;
        const int32_t r = fast_div(w, p.fd_other), o = w - r * other;
        int32_t g = 0;                                   // groups whose tiles all come before r
        for (int32_t base = 0; base < p.groups; base += 32) {
            const int32_t e = base + static_cast<int32_t>(lane);
            const uint32_t before = __ballot_sync(0xffffffffu, e < p.groups && pre[e + 1] <= r);
            g += __popc(before);
            if (before != 0xffffffffu) break;
        }
        t.group = g;
        const int32_t i = r - pre[g];
        if (p.ragged == kRaggedP) {
            t.p0 = off[g] + i * TP;
            t.p_end = off[g + 1];
            t.q0 = o * TQ;
        } else {
            t.q0 = off[g] + i * TQ;
            t.q_end = off[g + 1];
            t.p0 = o * TP;
        }
        return t;
    }
    if (p.ragged == kRaggedK) {
        const int32_t per = p.tiles_p * p.tiles_q;
        t.group = fast_div(w, p.fd_group);
        w -= t.group * per;
        t.kb0 = pre[t.group];
        t.kbn = pre[t.group + 1] - t.kb0;
    }
    const int32_t sweep = p.raster * p.tiles_q;          // tiles of `raster` rows of tiles
    const int32_t rg = fast_div(w, p.fd_sweep), first = rg * p.raster, size = min(p.raster, p.tiles_p - first), rem = w - rg * sweep;
    const int32_t tq = fast_div(rem, size == p.raster ? p.fd_raster : p.fd_last);
    t.p0 = (first + rem - tq * size) * TP;
    t.q0 = tq * TQ;
    return t;
}

// Clamped offsets and the prefix sums product_tile reads; one whole warp.  The offsets are fetched first, so that their latencies are one; unit2, pre2 (or nullptr): the prefix
// sums of another unit.  FETCH = false: off has the offsets already.
template <bool FETCH = true, class Params>
__device__ __forceinline__ void scan_groups(const Params &p, int32_t *pre, int32_t *off, int32_t unit, uint32_t lane, int32_t *pre2 = nullptr, int32_t unit2 = 1)
{
    if constexpr (FETCH)
        for (int32_t e = static_cast<int32_t>(lane); e <= p.groups; e += 32) off[e] = min(max(p.offsets[e], 0), p.rows_ragged);
    __syncwarp();
    int32_t carry = 0, carry2 = 0, last = off[0];
    for (int32_t base = 0; base < p.groups; base += 32) {
        const int32_t e = base + static_cast<int32_t>(lane);
        int32_t nxt = off[min(e + 1, p.groups)];                 // where group e ends
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {                       // non-decreasing whatever the caller's values
            const int32_t x = __shfl_up_sync(0xffffffffu, nxt, d);
            if (static_cast<int32_t>(lane) >= d) nxt = max(nxt, x);
        }
        nxt = max(nxt, last);
        int32_t o = __shfl_up_sync(0xffffffffu, nxt, 1);
        if (lane == 0) o = last;
        last = __shfl_sync(0xffffffffu, nxt, 31);
        const int32_t rows = e < p.groups ? nxt - o : 0;
        int32_t n = (rows + unit - 1) / unit, n2 = (rows + unit2 - 1) / unit2;
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
            const int32_t x = __shfl_up_sync(0xffffffffu, n, d), y = __shfl_up_sync(0xffffffffu, n2, d);
            if (static_cast<int32_t>(lane) >= d) n += x, n2 += y;
        }
        if (e < p.groups) {
            off[e + 1] = nxt;
            pre[e + 1] = p.ragged == kRaggedK ? min(carry + n, p.k_capacity) : carry + n;
            if (pre2 != nullptr) pre2[e + 1] = carry2 + n2;
        }
        carry += __shfl_sync(0xffffffffu, n, 31);
        carry2 += __shfl_sync(0xffffffffu, n2, 31);
    }
    if (lane == 0) {
        pre[0] = 0;
        if (pre2 != nullptr) pre2[0] = 0;
    }
}

template <class T>
__device__ __forceinline__ T narrow_to(float v);
template <>
__device__ __forceinline__ float narrow_to<float>(float v) { return v; }
template <>
__device__ __forceinline__ __half narrow_to<__half>(float v) { return __float2half_rn(v); }
template <>
__device__ __forceinline__ __nv_bfloat16 narrow_to<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }

__device__ __forceinline__ uint32_t pack_pair(float a, float b, __half)
{
    const __half2 h = __floats2half2_rn(a, b);
    return *reinterpret_cast<const uint32_t *>(&h);
}
__device__ __forceinline__ uint32_t pack_pair(float a, float b, __nv_bfloat16)
{
    const __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<const uint32_t *>(&h);
}

} // namespace hgemm_dev
