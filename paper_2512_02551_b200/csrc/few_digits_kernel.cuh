// What a layer of experts with 4-bit weights needs around its two products (fp4_product_kernel.cuh) for a few tokens.
//
// The tensor cores multiply 4-bit weights with 4-bit operands at the speed at which memory delivers them; making 16-bit operands of the weights instead
// costs the other pipes more than that (measured: 3 to 4 times the time for 16 tokens).  So the ACTIVATIONS take the weights' form: each is a sum of eight 4-bit
// digits whose blocks' scales fall by powers of two, which costs nothing where the products wait for weights.
//
//     s_1 = the smallest power of two with max |v| <= 6 s_1 in the block;  digit d = e2m1(r_d / s_d);  r_{d+1} = r_d - digit * s_d
//     s_2 = s_1 / 4 (|r_2| <= s_1: half the step below 6),  s_{d+1} = s_d / 8 (|r| <= s_d / 2: half the step below 4)
//
// Every step is exact, so that what is missing is the last remainder: at most s_8 / 2 = s_1 2^-21 (MX), less than 2^-22 of the block's largest magnitude, which is above 3 s_1.  NV scales
// are e4m3, whose smallest is 2^-9, the last that a block's digits have: values are scaled by a power of two for each choice, so that its largest s_1 is 2^8 and its largest
// magnitude above 768; the remainder is at most 2^-10, less than 2^-19 of that.  (So a block far below the largest has fewer digits, the largest seven.)  Where numbers near
// fp32's smallest stop the scales (MX: 2^-126) or that power of two (NV: 2^-126), the remainder is at most 2^-127 and 2^-136.
//
// Choices are sorted by expert; choice number c lies at position[c], its digits in rows 8 position[c] .. + 7, their scales in tiles that begin anew for each
// expert.  One CTA per choice makes its digits: from x, or from the first product by way of the activation.  Latency bounds these kernels: a few thousand elements each.
// The products start beside them and fetch their first weights meanwhile.  Measured (2048 -> 1024 -> 2048, SwiGLU, nvfp4, 8 of 64 experts): 1 token 16.9 us in a graph, of which the digits
// of x take 3.6, the first product's rest 3.7, the digits of h 2.5, the second product's rest 3.4, the sum 1.1, and 1 passes between one's end and the next's reading; 16 tokens
// 48.2 us, 4.1 TB/s.  With all their runs of four elements unrolled the digits took 5.7 and 2.7 us: a launch fetches its instructions anew.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_fp4.h>
#include <stdint.h>

#include "fp4_quantize_kernel.cuh"
#include "hgemm_device.cuh"
#include "product_tiles.cuh"

namespace hgemm_dev {

constexpr int kDigitThreads = 512;
constexpr int kCombineThreads = 128;
constexpr int kDigits = 8;

struct DigitParams {
    const void *x;             // tokens x depth (fp16 or bf16), or nullptr: u
    int64_t ldx;
    int32_t x_half, x_vec;     // fp16; rows start at multiples of 8 bytes
    const float *u;            // the first product: [position][gated ? 2 * depth : depth], ldu apart
    int64_t ldu;
    int32_t u_vec, gated;      // rows (and their second halves) start at multiples of 16 bytes
    const float *u_factor;     // of a position: u counts times this
    int32_t depth, top_k, experts, choices;
    const int32_t *indices;
    // written by the kernel that reads x, read by the others
    int32_t *position;         // of a choice; -1: of no expert
    int32_t *place;            // row of the scale tiles of a choice's first digit
    // the digits
    uint8_t *q;
    int64_t ldq;
    uint8_t *scales;
    int32_t atoms;             // scale tiles across
    float *factor;             // of a position: digits count times this (MX: 1)
};

// The sums of three numbers over the CTA, in every thread; scratch: 3 words, zero on entry.
__device__ __forceinline__ void digit_sums(int32_t &a, int32_t &b, int32_t &c, int32_t *scratch)
{
    a = __reduce_add_sync(0xffffffffu, a);
    b = __reduce_add_sync(0xffffffffu, b);
    c = __reduce_add_sync(0xffffffffu, c);
    if ((threadIdx.x & 31u) == 0u) {
        atomicAdd(&scratch[0], a);
        atomicAdd(&scratch[1], b);
        atomicAdd(&scratch[2], c);
    }
    __syncthreads();
    a = scratch[0];
    b = scratch[1];
    c = scratch[2];
}

__device__ __forceinline__ float digit_silu(float u) { return u / (1.0f + __expf(-u)); }

// Elements k .. k + 3 (zeros beyond the depth).
__device__ __forceinline__ void digit_load(const DigitParams &p, const uint16_t *x, const float *u, float factor, int32_t k, float (&f)[4])
{
    if (x != nullptr) {
        uint32_t w[2];
        if (p.x_vec && k + 4 <= p.depth) {
            const uint2 a = *reinterpret_cast<const uint2 *>(x + k);
            w[0] = a.x, w[1] = a.y;
        } else {
#pragma unroll
            for (int i = 0; i < 2; ++i) w[i] = (k + 2 * i < p.depth ? x[k + 2 * i] : 0u) | (k + 2 * i + 1 < p.depth ? static_cast<uint32_t>(x[k + 2 * i + 1]) << 16 : 0u);
        }
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            if (p.x_half) two_floats(w[i], f[2 * i], f[2 * i + 1], __half());
            else two_floats(w[i], f[2 * i], f[2 * i + 1], __nv_bfloat16());
        }
        return;
    }
    float g[4] = {0.0f, 0.0f, 0.0f, 0.0f}, v[4] = {0.0f, 0.0f, 0.0f, 0.0f};
    if (p.u_vec && k + 4 <= p.depth) {
        const float4 a = *reinterpret_cast<const float4 *>(u + k);
        g[0] = a.x, g[1] = a.y, g[2] = a.z, g[3] = a.w;
        if (p.gated) {
            const float4 b = *reinterpret_cast<const float4 *>(u + p.depth + k);
            v[0] = b.x, v[1] = b.y, v[2] = b.z, v[3] = b.w;
        }
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if (k + i < p.depth) {
                g[i] = u[k + i];
                if (p.gated) v[i] = u[p.depth + k + i];
            }
        }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float h = digit_silu(g[i] * factor);
        f[i] = p.gated ? h * (v[i] * factor) : h;
    }
}

// The digits of a warp's runs of four elements (run r of this lane; beyond `runs`: nothing is written).  Whole warps.
template <bool NV>
__device__ __forceinline__ void digit_write(const DigitParams &p, float (&f)[4], float inverse, int32_t r, int32_t runs, uint8_t *q, uint8_t *scales)
{
    constexpr int32_t kLeast = NV ? 127 - 9 : 1;                  // the smallest scale's exponent, biased
    const int32_t bytes = (p.depth + 1) / 2;
    float amax = 0.0f;
    bool odd = false;                                             // a NaN or an infinity in the block
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        odd = odd || (__float_as_uint(f[i]) & 0x7fffffffu) >= 0x7f800000u;
        f[i] *= inverse;
        amax = fmaxf(amax, fabsf(f[i]));
    }
    // the block's four (NV) or eight lanes
    uint32_t top = odd ? 0x7f800000u : __float_as_uint(amax);
#pragma unroll
    for (int d = 1; d < (NV ? 4 : 8); d <<= 1) top = max(top, __shfl_xor_sync(0xffffffffu, top, d));
    odd = top >= 0x7f800000u;
    int32_t e = top != 0u && !odd ? max(power_above(__uint_as_float(top), 2, kMantissa6), kLeast) : 0;      // s_1's exponent; 0: no digit
    // the scales: lane d of an atom's lanes (16, or 32) makes digit d's, of four blocks a word
    constexpr int kAtomLanes = NV ? 16 : 32;
    {
        const int32_t lane = static_cast<int32_t>(lane_id()), d = lane & 7;
        uint32_t word = 0u;
#pragma unroll
        for (int b = 0; b < 4; ++b) {
            const int32_t first = __shfl_sync(0xffffffffu, odd ? -1 : e, (lane & ~(kAtomLanes - 1)) + b * (kAtomLanes / 4));
            // digit d's exponent: first, less 2 and then 3 a digit, down to the least, which is the last
            const int32_t ahead = d == 0 ? first : first - (d == 1 ? 0 : 3 * d - 4), here = d == 0 ? first : max(first - (3 * d - 1), kLeast);      // the digit before, this one
            const bool there = first > 0 && (d == 0 || ahead > kLeast);
            uint32_t byte = there ? static_cast<uint32_t>(min(here, 253)) : 0u;
            if constexpr (NV) {
                const int32_t n = here - 127;                     // 2^8 .. 2^-9 as e4m3
                byte = !there ? 0u : n >= -6 ? static_cast<uint32_t>(n + 7) << 3 : 1u << (n + 9);
            }
            if (first < 0 && d == 0) byte = NV ? 0x7fu : 0xffu;
            word |= byte << (8 * b);
        }
        if ((lane & (kAtomLanes - 1)) < kDigits && (r & ~(kAtomLanes - 1)) < runs) *reinterpret_cast<uint32_t *>(scales + static_cast<int64_t>(r / kAtomLanes) * 512 + d * 16) = word;
    }
    uint8_t *dst = q + r * 2;
#pragma unroll 1                                                  // (see few_digits_kernel: short code)
    for (int32_t d = 0; d < kDigits; ++d, dst += p.ldq) {
        const bool some = e > 0;
        const float step = some ? __uint_as_float(static_cast<uint32_t>(min(e, 253)) << 23) : 0.0f, back = some ? __uint_as_float(static_cast<uint32_t>(254 - min(e, 253)) << 23) : 0.0f;
        uint32_t w = 0u;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const uint32_t b = __nv_cvt_float2_to_fp4x2(make_float2(f[2 * i] * back, f[2 * i + 1] * back), __NV_E2M1, cudaRoundNearest);
            w |= b << (8 * i);
            const float2 v = __half22float2(__half2(__nv_cvt_fp4x2_to_halfraw2(static_cast<__nv_fp4x2_storage_t>(b), __NV_E2M1)));
            f[2 * i] = fmaf(-v.x, step, f[2 * i]);
            f[2 * i + 1] = fmaf(-v.y, step, f[2 * i + 1]);
        }
        if (odd) w = 0u;                                          // the scale says it
        if (r * 2 + 2 <= bytes) *reinterpret_cast<uint16_t *>(dst) = static_cast<uint16_t>(w);
        else if (r * 2 < bytes) *dst = static_cast<uint8_t>(w);
        e = e <= kLeast ? 0 : max(e - (d == 0 ? 2 : 3), kLeast);  // after the smallest scale, no more digits
    }
}

// One CTA per choice.  The code is short rather than unrolled: a launch of a few microseconds fetches its instructions anew.  FIRST: the kernel that reads x; it finds the choices' places (dynamic shared memory: a word for each expert).  (Fetching the next product's weights to L2 meanwhile was tried: the launch then ends with the last of them, 1 token 25 -> 31 us.)
template <bool NV, bool FIRST>
__global__ void __launch_bounds__(kDigitThreads)
few_digits_kernel(const DigitParams p)
{
    constexpr int kBlock = NV ? 16 : 32, kAtom = 4 * kBlock;
    extern __shared__ int32_t s_count[];
    __shared__ int32_t s_sums[3];
    __shared__ uint32_t s_top;
    const int32_t c = static_cast<int32_t>(blockIdx.x), me = static_cast<int32_t>(threadIdx.x);
    int32_t position = 0, place = 0;
    float u_factor = 1.0f;
    if constexpr (!FIRST) {                                       // the first kernel's, which the product has waited for
        position = ld_older(p.position + c);
        place = ld_older(p.place + c);
        if (position >= 0) u_factor = ld_older(p.u_factor + position);
    }
    grid_dependency_wait();
    grid_launch_dependents();                                     // from here on the product may read the call's inputs (fp4_digits_product)
    const int32_t runs = p.atoms * (kAtom / 4);                   // of four elements, those that fill the last scale tile among them
    const uint16_t *x = FIRST ? static_cast<const uint16_t *>(p.x) + static_cast<int64_t>(c / p.top_k) * p.ldx : nullptr;
    float f[4];                                                   // the first run, kept between the two looks at it
    if constexpr (FIRST) digit_load(p, x, nullptr, 1.0f, min(me, runs) * 4, f);                      // (run number `runs`: beyond the depth)
    if (me == 0) {
        s_sums[0] = s_sums[1] = s_sums[2] = 0;
        s_top = 0u;
    }
    if constexpr (FIRST) {
        for (int32_t e = me; e < p.experts; e += kDigitThreads) s_count[e] = 0;
        __syncthreads();
        const int32_t mine = p.indices[c];
        int32_t ahead = 0;                                        // choices of the same expert ahead of this one
        for (int32_t i = me; i < p.choices; i += kDigitThreads) {
            const int32_t e = p.indices[i];
            if (e >= 0 && e < p.experts) {
                atomicAdd(&s_count[e], 1);
                ahead += e == mine && i < c ? 1 : 0;
            }
        }
        __syncthreads();
        if (mine < 0 || mine >= p.experts) {
            if (me == 0) p.position[c] = -1;
            return;
        }
        int32_t before = 0, tiles = 0;                            // positions and scale tiles of the experts ahead
        for (int32_t e = me; e < mine; e += kDigitThreads) {
            before += s_count[e];
            tiles += (s_count[e] * kDigits + 127) / 128;
        }
        digit_sums(before, tiles, ahead, s_sums);
        position = before + ahead;
        place = tiles * 128 + ahead * kDigits;
        if (me == 0) {
            p.position[c] = position;
            p.place[c] = place;
        }
    } else {
        if (position < 0) return;
        __syncthreads();
    }
    const float *u = FIRST ? nullptr : p.u + position * p.ldu;
    if constexpr (!FIRST) digit_load(p, nullptr, u, u_factor, min(me, runs) * 4, f);
    float inverse = 1.0f;
    if constexpr (NV) {
        uint32_t top = 0u;
        auto look = [&](const float (&v)[4]) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const uint32_t b = __float_as_uint(v[i]) & 0x7fffffffu;
                if (b < 0x7f800000u) top = max(top, b);
            }
        };
        look(f);
#pragma unroll 1
        for (int32_t r = me + kDigitThreads; r < runs; r += kDigitThreads) {
            float v[4];
            digit_load(p, x, u, u_factor, r * 4, v);
            look(v);
        }
        top = __reduce_max_sync(0xffffffffu, top);
        if ((me & 31) == 0) atomicMax(&s_top, top);
        __syncthreads();
        // the smallest power of two that is at least the largest magnitude / 1536 (6 * 2^8), inside fp32's normal numbers
        const int32_t e = min(max(power_above(__uint_as_float(s_top), 10, 0x400000u), 1), 253);
        inverse = __uint_as_float(static_cast<uint32_t>(254 - e) << 23);
        if (me == 0) p.factor[position] = s_top == 0u ? 1.0f : __uint_as_float(static_cast<uint32_t>(e) << 23);
    } else {
        if (me == 0) p.factor[position] = 1.0f;
    }
    uint8_t *q = p.q + static_cast<int64_t>(position) * kDigits * p.ldq;
    uint8_t *scales = p.scales + static_cast<int64_t>(place >> 7) * p.atoms * 512 + (place & 31) * 16 + ((place >> 5) & 3) * 4;      // a choice's rows never cross 32
    const int32_t base = me & ~31, lane = me & 31;
#pragma unroll 1
    for (int32_t r0 = base; r0 < runs; r0 += kDigitThreads) {
        if (r0 != base) digit_load(p, x, u, u_factor, min(r0 + lane, runs) * 4, f);
        digit_write<NV>(p, f, inverse, r0 + lane, runs, q, scales);
    }
}

struct CombineParams {
    const float *z;            // [position][hidden], ldz apart (a multiple of 4)
    int64_t ldz;
    const float *factor;       // of a position
    const int32_t *position;   // of a choice
    const float *weights;
    int32_t top_k, hidden;
    void *y;
    int64_t ldy;
    int32_t y_vec;             // rows of y start at multiples of 8 bytes
};

// y = sum over a token's choices, in their order.  grid: x = runs of 512 outputs, y = tokens.
template <class Y>
__global__ void __launch_bounds__(kCombineThreads)
few_combine_kernel(const CombineParams p)
{
    grid_launch_dependents();
    const int32_t n = (static_cast<int32_t>(blockIdx.x) * kCombineThreads + static_cast<int32_t>(threadIdx.x)) * 4, t = static_cast<int32_t>(blockIdx.y);
    // lane j has choice j's row and factor: the digits' kernels', which the product has waited for
    const int32_t lane = static_cast<int32_t>(threadIdx.x & 31u);
    int32_t mine = -1;
    float w = 0.0f;
    if (lane < p.top_k) {
        mine = ld_older(p.position + t * p.top_k + lane);
        w = ld_older(p.weights + t * p.top_k + lane);
    }
    const float s = mine >= 0 ? ld_older(p.factor + mine) : 0.0f;
    grid_dependency_wait();
    float sum[4] = {0.0f, 0.0f, 0.0f, 0.0f};
    for (int32_t j0 = 0; j0 < p.top_k; j0 += 8) {
        float4 z[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const int32_t at = __shfl_sync(0xffffffffu, mine, (j0 + j) & 31);
            z[j] = j0 + j < p.top_k && at >= 0 && n < p.hidden ? *reinterpret_cast<const float4 *>(p.z + at * p.ldz + n) : make_float4(0.0f, 0.0f, 0.0f, 0.0f);      // (beyond hidden: the row's padding, not stored)
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const bool there = j0 + j < p.top_k && __shfl_sync(0xffffffffu, mine, (j0 + j) & 31) >= 0;
            const float wj = __shfl_sync(0xffffffffu, w, (j0 + j) & 31), sj = __shfl_sync(0xffffffffu, s, (j0 + j) & 31);
            if (there) {
                sum[0] = fmaf(wj, z[j].x * sj, sum[0]);
                sum[1] = fmaf(wj, z[j].y * sj, sum[1]);
                sum[2] = fmaf(wj, z[j].z * sj, sum[2]);
                sum[3] = fmaf(wj, z[j].w * sj, sum[3]);
            }
        }
    }
    if (n >= p.hidden) return;
    Y *y = static_cast<Y *>(p.y) + t * p.ldy + n;
    if (p.y_vec && n + 4 <= p.hidden) {
        *reinterpret_cast<uint2 *>(y) = make_uint2(pack_pair(sum[0], sum[1], Y()), pack_pair(sum[2], sum[3], Y()));
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (n + i < p.hidden) y[i] = narrow_to<Y>(sum[i]);
    }
}

} // namespace hgemm_dev
