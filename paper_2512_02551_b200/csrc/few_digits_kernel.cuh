// What a layer of experts with 4-bit weights needs around its two products (fp4_product_kernel.cuh) for a few tokens.
//
// The tensor cores multiply 4-bit weights with 4-bit operands at the speed at which memory delivers them; making 16-bit operands of the weights instead
// costs the other pipes more than that (measured: 3 to 4 times the time for 16 tokens).  So the ACTIVATIONS take the weights' form: each is a sum of eight 4-bit
// digits whose blocks' scales fall by powers of two, which costs nothing where the products wait for weights.
//
//     s_1 = the smallest power of two with max |v| <= 6 s_1 in the block;  digit d = e2m1(r_d / s_d);  r_{d+1} = r_d - digit * s_d
//     s_2 = s_1 / 4 (|r_2| <= s_1: half the step below 6),  s_{d+1} = s_d / 8 (|r| <= s_d / 2: half the step below 4)
//
// Every step is exact, so that what is missing is the last remainder: at most s_8 / 2 = s_1 2^-21 (MX).  NV scales are e4m3, whose smallest is 2^-9, the last that a
// block's digits have: values are scaled by a power of two for each choice, so that its largest s_1 is at most 2^8 and its largest magnitude above
// 768; the remainder is at most 2^-10, less than 2^-19 of that.
//
// Choices are sorted by expert; choice number c lies at position[c], its digits in rows 8 position[c] .. + 7, their scales in tiles that begin anew for each
// expert.  One CTA per choice makes its digits: from x, or from the first product by way of the activation.  Latency bounds these kernels: a few thousand elements each.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_fp4.h>
#include <stdint.h>

#include "fp4_quantize_kernel.cuh"
#include "hgemm_device.cuh"
#include "product_tiles.cuh"

namespace hgemm_dev {

constexpr int kDigitThreads = 256;
constexpr int kDigits = 8;

struct DigitParams {
    const void *x;             // tokens x depth (fp16 or bf16), or nullptr: u
    int64_t ldx;
    int32_t x_half, x_vec;     // fp16; rows start at multiples of 16 bytes
    const float *u;            // the first product: [position][gated ? 2 * depth : depth], ldu apart
    int64_t ldu;
    int32_t u_vec, gated;      // rows (and their second halves) start at multiples of 16 bytes
    const float *u_factor;     // of a position: u counts times this
    int32_t depth, top_k, experts, choices;
    const int32_t *indices;
    // written by the kernel that reads x, read by the others
    int32_t *offsets;          // 8 times the experts' first positions, experts + 1
    int32_t *position;         // of a choice; -1: of no expert
    int32_t *place;            // row of the scale tiles of a choice's first digit
    float *one;                // 1
    // the digits
    uint8_t *q;
    int64_t ldq;
    uint8_t *scales;
    int32_t atoms;             // scale tiles across
    float *factor;             // of a position: digits count times this (MX: 1)
};

// The sum of two numbers over the CTA, in every thread; scratch: 2 words, zero on entry.
__device__ __forceinline__ void digit_sums(int32_t &a, int32_t &b, int32_t *scratch)
{
    a = __reduce_add_sync(0xffffffffu, a);
    b = __reduce_add_sync(0xffffffffu, b);
    if ((threadIdx.x & 31u) == 0u) {
        atomicAdd(&scratch[0], a);
        atomicAdd(&scratch[1], b);
    }
    __syncthreads();
    a = scratch[0];
    b = scratch[1];
}

__device__ __forceinline__ float digit_silu(float u) { return u / (1.0f + __expf(-u)); }

// Elements k .. k + 15 (zeros beyond the depth).
__device__ __forceinline__ void digit_load(const DigitParams &p, const uint16_t *x, const float *u, float factor, int32_t k, float (&f)[16])
{
    if (x != nullptr) {
        if (p.x_vec && k + 16 <= p.depth) {
            const uint4 a = reinterpret_cast<const uint4 *>(x + k)[0], b = reinterpret_cast<const uint4 *>(x + k)[1];
            const uint32_t w[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                if (p.x_half) two_floats(w[i], f[2 * i], f[2 * i + 1], __half());
                else two_floats(w[i], f[2 * i], f[2 * i + 1], __nv_bfloat16());
            }
        } else {
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const uint32_t w = k + i < p.depth ? x[k + i] : 0u;
                f[i] = p.x_half ? __half2float(__ushort_as_half(static_cast<unsigned short>(w))) : __uint_as_float(w << 16);
            }
        }
        return;
    }
    float g[16], v[16];
    if (p.u_vec && k + 16 <= p.depth) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float4 a = reinterpret_cast<const float4 *>(u + k)[i];
            g[4 * i] = a.x, g[4 * i + 1] = a.y, g[4 * i + 2] = a.z, g[4 * i + 3] = a.w;
            if (p.gated) {
                const float4 b = reinterpret_cast<const float4 *>(u + p.depth + k)[i];
                v[4 * i] = b.x, v[4 * i + 1] = b.y, v[4 * i + 2] = b.z, v[4 * i + 3] = b.w;
            }
        }
    } else {
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            g[i] = k + i < p.depth ? u[k + i] : 0.0f;
            v[i] = k + i < p.depth && p.gated ? u[p.depth + k + i] : 0.0f;
        }
    }
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        const float h = digit_silu(g[i] * factor);
        f[i] = p.gated ? h * (v[i] * factor) : h;
    }
}

// One CTA per choice.  FIRST: the kernel that reads x; it finds the choices' places (dynamic shared memory: a word for each expert), and its last CTA
// writes the experts' offsets.
template <bool NV, bool FIRST>
__global__ void __launch_bounds__(kDigitThreads)
few_digits_kernel(const DigitParams p)
{
    constexpr int kBlock = NV ? 16 : 32, kAtom = 4 * kBlock;
    extern __shared__ int32_t s_count[];
    __shared__ int32_t s_sums[2];
    __shared__ uint32_t s_top;
    grid_launch_dependents();
    grid_dependency_wait();
    const int32_t c = static_cast<int32_t>(blockIdx.x), me = static_cast<int32_t>(threadIdx.x);
    int32_t position, place;
    if (me == 0) {
        s_sums[0] = s_sums[1] = 0;
        s_top = 0u;
    }
    if constexpr (FIRST) {
        for (int32_t e = me; e < p.experts; e += kDigitThreads) s_count[e] = 0;
        __syncthreads();
        const int32_t mine = c < p.choices ? p.indices[c] : -1;
        int32_t ahead = 0;                                        // choices of the same expert ahead of this one
        for (int32_t i = me; i < p.choices; i += kDigitThreads) {
            const int32_t e = p.indices[i];
            if (e >= 0 && e < p.experts) {
                atomicAdd(&s_count[e], 1);
                ahead += e == mine && i < c ? 1 : 0;
            }
        }
        __syncthreads();
        if (c == p.choices) {                                     // the offsets
            if (me < 32) {
                int32_t carry = 0;
                for (int32_t base = 0; base < p.experts; base += 32) {
                    const int32_t e = base + me;
                    int32_t sum = e < p.experts ? s_count[e] : 0;
#pragma unroll
                    for (int d = 1; d < 32; d <<= 1) {
                        const int32_t v = __shfl_up_sync(0xffffffffu, sum, d);
                        if (me >= d) sum += v;
                    }
                    if (e < p.experts) p.offsets[e + 1] = kDigits * (carry + sum);
                    carry += __shfl_sync(0xffffffffu, sum, 31);
                }
                if (me == 0) {
                    p.offsets[0] = 0;
                    *p.one = 1.0f;
                }
            }
            return;
        }
        if (mine < 0 || mine >= p.experts) {
            if (me == 0) p.position[c] = -1;
            return;
        }
        int32_t before = ahead, tiles = 0;                        // positions ahead; scale tiles of the experts ahead
        for (int32_t e = me; e < mine; e += kDigitThreads) {
            before += s_count[e];
            tiles += (s_count[e] * kDigits + 127) / 128;
        }
        // `ahead` counts towards both this expert's place and all positions
        int32_t own = ahead, none = 0;
        digit_sums(before, tiles, s_sums);
        __syncthreads();
        if (me == 0) s_sums[0] = s_sums[1] = 0;
        __syncthreads();
        digit_sums(own, none, s_sums);
        position = before;
        place = tiles * 128 + own * kDigits;
        if (me == 0) {
            p.position[c] = position;
            p.place[c] = place;
        }
    } else {
        position = p.position[c];
        if (position < 0) return;
        place = p.place[c];
        __syncthreads();
    }
    const uint16_t *x = FIRST ? static_cast<const uint16_t *>(p.x) + static_cast<int64_t>(c / p.top_k) * p.ldx : nullptr;
    const float *u = FIRST ? nullptr : p.u + position * p.ldu;
    const float u_factor = FIRST ? 1.0f : p.u_factor[position];
    const int32_t runs = p.atoms * (kAtom / 16);                  // of 16 elements, those that fill the last scale tile among them
    float f[16];
    float inverse = 1.0f;
    if constexpr (NV) {
        uint32_t top = 0u;
        for (int32_t r = me; r < runs; r += kDigitThreads) {
            digit_load(p, x, u, u_factor, r * 16, f);
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const uint32_t b = __float_as_uint(f[i]) & 0x7fffffffu;
                if (b < 0x7f800000u) top = max(top, b);
            }
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
    const int32_t bytes = (p.depth + 1) / 2;
    for (int32_t r0 = me & ~31; r0 < runs; r0 += kDigitThreads) {   // whole warps; runs is a multiple of 4
        const int32_t r = r0 + (me & 31);
        float amax = 0.0f;
        bool odd = false;
        if (r < runs) {
            digit_load(p, x, u, u_factor, r * 16, f);
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                odd = odd || (__float_as_uint(f[i]) & 0x7fffffffu) >= 0x7f800000u;
                f[i] *= inverse;
                amax = fmaxf(amax, fabsf(f[i]));
            }
        }
        if constexpr (!NV) {
            amax = fmaxf(amax, __shfl_xor_sync(0xffffffffu, amax, 1));
            odd = odd || __shfl_xor_sync(0xffffffffu, static_cast<int>(odd), 1) != 0;
        }
        constexpr int32_t kLeast = NV ? 127 - 9 : 1;              // the smallest scale's exponent, biased
        int32_t e = power_above(amax, 2, kMantissa6);             // s_1's
        e = amax > 0.0f && !odd ? max(e, kLeast) : 0;             // (0: no digit)
#pragma unroll 1
        for (int32_t d = 0; d < kDigits; ++d) {
            const bool some = e > 0;
            const float step = some ? __uint_as_float(static_cast<uint32_t>(min(e, 253)) << 23) : 0.0f, back = some ? __uint_as_float(static_cast<uint32_t>(254 - min(e, 253)) << 23) : 0.0f;
            uint32_t w[2] = {0u, 0u};
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const uint32_t b = __nv_cvt_float2_to_fp4x2(make_float2(f[2 * i] * back, f[2 * i + 1] * back), __NV_E2M1, cudaRoundNearest);
                w[i / 4] |= b << (8 * (i & 3));
                const float2 v = __half22float2(__half2(__nv_cvt_fp4x2_to_halfraw2(static_cast<__nv_fp4x2_storage_t>(b), __NV_E2M1)));
                f[2 * i] = fmaf(-v.x, step, f[2 * i]);
                f[2 * i + 1] = fmaf(-v.y, step, f[2 * i + 1]);
            }
            if (odd) w[0] = w[1] = 0u;                            // the scale says it
            uint32_t byte;
            if constexpr (NV) {
                const int32_t n = e - 127;                        // 2^8 .. 2^-9 as e4m3
                byte = odd ? (d == 0 ? 0x7fu : 0u) : !some ? 0u : n >= -6 ? static_cast<uint32_t>(n + 7) << 3 : 1u << (n + 9);
                byte <<= 8 * (r & 3);
            } else {
                byte = odd ? (d == 0 ? 0xffu : 0u) : static_cast<uint32_t>(min(e, 253));
                byte <<= 8 * ((r >> 1) & 3);
            }
            // the scales of four blocks make a word
            byte |= __shfl_xor_sync(0xffffffffu, byte, NV ? 1 : 2);
            byte |= __shfl_xor_sync(0xffffffffu, byte, NV ? 2 : 4);
            if (r < runs) {
                if ((r & (NV ? 3 : 7)) == 0) *reinterpret_cast<uint32_t *>(scales + static_cast<int64_t>(r / (NV ? 4 : 8)) * 512 + d * 16) = byte;
                uint8_t *dst = q + d * p.ldq + r * 8;
                if (r * 8 + 8 <= bytes) {
                    *reinterpret_cast<uint2 *>(dst) = make_uint2(w[0], w[1]);
                } else {
#pragma unroll
                    for (int j = 0; j < 8; ++j)
                        if (r * 8 + j < bytes) dst[j] = static_cast<uint8_t>(w[j / 4] >> (8 * (j & 3)));
                }
            }
            e = e <= kLeast ? 0 : max(e - (d == 0 ? 2 : 3), kLeast);      // after the smallest scale, no more digits
        }
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

// y = sum over a token's choices, in their order.  grid: x = runs of 1024 outputs, y = tokens.
template <class Y>
__global__ void __launch_bounds__(kDigitThreads)
few_combine_kernel(const CombineParams p)
{
    grid_launch_dependents();
    grid_dependency_wait();
    const int32_t n = (static_cast<int32_t>(blockIdx.x) * kDigitThreads + static_cast<int32_t>(threadIdx.x)) * 4, t = static_cast<int32_t>(blockIdx.y);
    if (n >= p.hidden) return;
    float sum[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll 8
    for (int32_t j = 0; j < p.top_k; ++j) {
        const int32_t at = p.position[t * p.top_k + j];
        if (at < 0) continue;
        const float w = p.weights[t * p.top_k + j], s = p.factor[at];
        const float4 z = *reinterpret_cast<const float4 *>(p.z + at * p.ldz + n);      // (beyond hidden: the row's padding, not stored)
        sum[0] = fmaf(w, z.x * s, sum[0]);
        sum[1] = fmaf(w, z.y * s, sum[1]);
        sum[2] = fmaf(w, z.z * s, sum[2]);
        sum[3] = fmaf(w, z.w * s, sum[3]);
    }
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
