// 4-bit quantisation with one scale per block of 16 (e4m3, and a factor for the tensor) or 32 (a power of two) along rows, along columns, or both
// in one pass; the tensor's factor; and the way back.
//
// Bytes: 2 or 4 read and a half (both copies: one) written per element.  Ten instructions per quantised element, and too few warps to issue them at every cycle: three CTAs of 77 registers
// an SM keep 34 % of its warps, and 61 % of the issue slots are used (8191 x 4096 bf16, both copies: 35 us, 3.0 TB/s; 2048 tiles are 4.6 rounds; four CTAs an SM spilled).  The
// factor before it takes 14 us, 4.8 TB/s, waiting for loads; back to bf16 17 us along rows, 5.1 TB/s, and 25 us along columns,
// whose rows of 8191 start at every second byte.  256 threads own a tile of 128 x 128 elements.  As it is
// loaded, 8 lanes hold a row's 128 elements, 16 each: a block, or half of one, whose maximum needs at most one shuffle.  For the column copy
// the tile goes to shared memory as it came; there a thread takes 32 rows of two columns (16-bit types) or of one (fp32, twice), so that
// blocks lie in registers again, and the packed columns and their scale tiles leave through shared memory in runs of 64 and 1024 bytes.
//
// A value is the nearest 4-bit value of the correctly rounded quotient x / step (step = scale * factor): q = x * r, then one residual step with two
// multiply-adds (r = 1 / step is correctly rounded, which makes that quotient so), two values an instruction.  A plain product with the reciprocal would be off by an ulp where x lies
// halfway between two values, which inputs of few bits often do.  Maxima are taken on the bit patterns: a NaN or an infinity is larger than every number.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_fp4.h>
#include <cuda_fp8.h>
#include <stdint.h>

#include "hgemm_device.cuh"
#include "product_tiles.cuh"

namespace hgemm_dev {

constexpr int kFp4QuantThreads = 256;
constexpr int kFp4OutPitch = 80;                  // bytes between packed columns in shared memory
__host__ __device__ constexpr int fp4_raw_pitch(int size) { return 128 * size + 16; }      // bytes between a tile's rows in shared memory
__host__ __device__ constexpr int fp4_quant_smem(int size, bool nv, bool columns) { return columns ? 128 * (fp4_raw_pitch(size) + kFp4OutPitch) + (nv ? 1024 : 512) : 0; }

struct Fp4QuantParams {
    const void *x;
    int64_t ldx, rows, cols, x_rows;
    const int32_t *row_index;
    const int32_t *offsets;
    int32_t groups;
    int32_t vec_ok;            // rows of x start at multiples of 16 bytes
    const float *factor;
    uint8_t *q;
    int64_t ldq;
    uint8_t *scales;
    uint8_t *q_cols;
    int64_t ldq_cols;
    uint8_t *scales_cols;
    int64_t col_rows;          // contracted elements of the column copy
    int64_t row_tiles;         // scale tiles along the rows of one matrix
};

// 16 consecutive elements as they came.
template <class T>
struct Raw16 {
    uint32_t w[4 * sizeof(T)];
};

template <class T>
__device__ __forceinline__ Raw16<T> load16(const T *row, int64_t col, int64_t cols, int32_t vec_ok)
{
    Raw16<T> r;
    constexpr int kVec = static_cast<int>(sizeof(T));            // 16-byte pieces
    if (row != nullptr && vec_ok && col + 16 <= cols) {
#pragma unroll
        for (int i = 0; i < kVec; ++i) {
            const uint4 v = reinterpret_cast<const uint4 *>(row + col)[i];
            r.w[4 * i] = v.x, r.w[4 * i + 1] = v.y, r.w[4 * i + 2] = v.z, r.w[4 * i + 3] = v.w;
        }
    } else {
#pragma unroll
        for (int i = 0; i < 4 * kVec; ++i) {
            if constexpr (sizeof(T) == 4) {
                r.w[i] = row != nullptr && col + i < cols ? __float_as_uint(row[col + i]) : 0u;
            } else {
                const unsigned short *s = reinterpret_cast<const unsigned short *>(row);
                const uint32_t a = row != nullptr && col + 2 * i < cols ? s[col + 2 * i] : 0u, b = row != nullptr && col + 2 * i + 1 < cols ? s[col + 2 * i + 1] : 0u;
                r.w[i] = a | (b << 16);
            }
        }
    }
    return r;
}

// Bit patterns of magnitudes; for the 16-bit types two at a time.
template <class T>
__device__ __forceinline__ uint32_t magnitude_max(uint32_t m, uint32_t w)
{
    if constexpr (sizeof(T) == 4) return max(m, w & 0x7fffffffu);
    else return __vmaxu2(m, w & 0x7fff7fffu);
}
// The largest magnitudes of N registers of pairs (an even number).  Numbers without sign find the largest of the negative ones (their sign bits are the highest), numbers with
// sign that of the others; three at a time.
template <int N>
__device__ __forceinline__ uint32_t pair_magnitudes(const uint32_t *w)
{
    uint32_t below = 0u, above = 0u;
#pragma unroll
    for (int j = 0; j < N; j += 2) {
        below = __vimax3_u16x2(below, w[j], w[j + 1]);
        above = __vimax3_s16x2(above, w[j], w[j + 1]);
    }
    return __vmaxu2(below & 0x7fff7fffu, above);
}
// The larger of a register's two 16-bit magnitudes, as the type's bit pattern.
__device__ __forceinline__ uint32_t larger16(uint32_t m) { return max(m & 0xffffu, m >> 16); }

// A magnitude's bit pattern as fp32; NaN for a NaN or an infinity.
__device__ __forceinline__ float magnitude_of(uint32_t m, float) { return m >= 0x7f800000u ? __int_as_float(0x7fffffff) : __uint_as_float(m); }
__device__ __forceinline__ float magnitude_of(uint32_t m, __half) { return m >= 0x7c00u ? __int_as_float(0x7fffffff) : __half2float(__ushort_as_half(static_cast<unsigned short>(m))); }
__device__ __forceinline__ float magnitude_of(uint32_t m, __nv_bfloat16) { return m >= 0x7f80u ? __int_as_float(0x7fffffff) : __uint_as_float(m << 16); }

__device__ __forceinline__ void two_floats(uint32_t w, float &a, float &b, __half)
{
    const float2 f = __half22float2(*reinterpret_cast<const __half2 *>(&w));
    a = f.x, b = f.y;
}
__device__ __forceinline__ void two_floats(uint32_t w, float &a, float &b, __nv_bfloat16) { a = __uint_as_float(w << 16), b = __uint_as_float(w & 0xffff0000u); }

// The exponent byte of the smallest power of two s with a <= top * s; top = (1 + top_mantissa / 2^23) * 2^top_exponent.
__device__ __forceinline__ int32_t power_above(float a, int32_t top_exponent, uint32_t top_mantissa)
{
    const uint32_t b = __float_as_uint(a);
    return static_cast<int32_t>(b >> 23) - top_exponent + ((b & 0x7fffffu) > top_mantissa ? 1 : 0);
}
constexpr uint32_t kMantissa6 = 0x400000u, kMantissa2688 = 0x280000u;        // 6 = 1.5 * 2^2, 2688 = 1.3125 * 2^11

struct BlockStep {
    uint32_t byte;             // the scale
    float step, inverse;       // what values are divided by, and its reciprocal (0 where values are 0)
    bool far;                  // the block's largest quotient is beyond fp32 (NV: a factor much smaller than the block's values ask for)
};

// amax: NaN for a block with a NaN or an infinity.  g = 1 / factor (NV).
template <bool NV>
__device__ __forceinline__ BlockStep block_step(float amax, float factor, float g)
{
    BlockStep s;
    if constexpr (NV) {
        const float u = amax * g * (1.0f / 6.0f);
        s.byte = __nv_cvt_float_to_fp8(u, __NV_SATFINITE, __NV_E4M3);
        const float step = __half2float(__half(__nv_cvt_fp8_to_halfraw(static_cast<__nv_fp8_storage_t>(s.byte), __NV_E4M3))) * factor;
        s.step = step > 0.0f ? step : 0.0f;                      // (a NaN: the block's zeros stay zeros)
        s.inverse = step > 0.0f ? __frcp_rn(step) : 0.0f;
        s.far = amax * s.inverse > 3.402823466e38f;
    } else {
        const int32_t e = min(max(power_above(amax, 2, kMantissa6), 0), 254);
        s.byte = amax != amax ? 255u : static_cast<uint32_t>(e);
        s.step = 0.0f;
        s.inverse = __uint_as_float(static_cast<uint32_t>(254 - e) << 23);   // 2^(127 - e), exactly (e = 254: below the smallest normal number; no finite block has it)
        s.far = false;
    }
    return s;
}

// 16 elements of a block that has quotients beyond fp32: those would be infinities, of which the residual step makes NaN, whose sign is lost.  What lies beyond 8 steps has
// the value of 8 steps: the largest, with its sign.
template <bool NV>
__device__ __forceinline__ void bring_near(float (&f)[16], const BlockStep &s)
{
    if constexpr (NV) {
        if (s.far) {
            const float most = 8.0f * s.step;
#pragma unroll
            for (int i = 0; i < 16; ++i) f[i] = fminf(fmaxf(f[i], -most), most);
        }
    }
}

// Eight quotients as 4-bit values in a word.
template <bool NV>
__device__ __forceinline__ uint32_t quantize8(const float *f, const BlockStep &s)
{
    const uint64_t r = pack_f32x2(__float_as_uint(s.inverse), __float_as_uint(s.inverse)), step = pack_f32x2(__float_as_uint(-s.step), __float_as_uint(-s.step));
    float x[8];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint64_t v = pack_f32x2(__float_as_uint(f[2 * i]), __float_as_uint(f[2 * i + 1]));
        uint64_t q = mul_f32x2(v, r);
        if constexpr (NV) q = fma_f32x2(fma_f32x2(q, step, v), r, q);
        unpack_f32x2(q, x[2 * i], x[2 * i + 1]);
    }
    return pack_e2m1(x[0], x[1], x[2], x[3], x[4], x[5], x[6], x[7]);
}

// The group that holds block rb (of 128 rows) of the copy laid out per group, and the block's rows: first .. end - 1 of the input (end: the group's).  The offsets are
// clamped as the products clamp them.  One whole warp; false beyond the last group's.
__device__ __forceinline__ bool block_of_group(const int32_t *offsets, int32_t groups, int32_t limit, int32_t rb, uint32_t lane, int32_t &first, int32_t &end)
{
    int32_t carry = 0, last = 0;
    for (int32_t base = 0; base < groups; base += 32) {
        const int32_t e = base + static_cast<int32_t>(lane);
        int32_t a = min(max(offsets[min(e, groups)], 0), limit);
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
            const int32_t x = __shfl_up_sync(0xffffffffu, a, d);
            if (static_cast<int32_t>(lane) >= d) a = max(a, x);
        }
        a = max(a, last);
        int32_t z = __shfl_down_sync(0xffffffffu, a, 1);
        if (lane == 31) z = max(a, min(max(offsets[min(e + 1, groups)], 0), limit));
        last = __shfl_sync(0xffffffffu, z, 31);
        const int32_t n = e < groups ? (z - a + 127) / 128 : 0;
        int32_t sum = n;
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
            const int32_t x = __shfl_up_sync(0xffffffffu, sum, d);
            if (static_cast<int32_t>(lane) >= d) sum += x;
        }
        const uint32_t hit = __ballot_sync(0xffffffffu, n > 0 && carry + sum > rb);
        if (hit) {
            const int src = __ffs(hit) - 1;
            first = __shfl_sync(0xffffffffu, a + (rb - (carry + sum - n)) * 128, src);
            end = __shfl_sync(0xffffffffu, z, src);
            return true;
        }
        carry += __shfl_sync(0xffffffffu, sum, 31);
    }
    return false;
}

// MODE: HGEMM_FP4_ROWS (1), COLS (2) or both (3).  grid: x = column tiles (each CTA walks on by gridDim.x), y = row tiles (as many as the padded copy has), z = matrices.
template <class T, int MODE, bool NV>
__global__ void __launch_bounds__(kFp4QuantThreads, sizeof(T) == 4 ? 2 : NV ? 3 : 4)
fp4_quantize_kernel(const Fp4QuantParams p)
{
    constexpr int kBlock = NV ? 16 : 32, kAtom = 4 * kBlock;     // elements of a block; of a scale tile's four
    constexpr int kPitch = fp4_raw_pitch(sizeof(T)), kOutPitch = kFp4OutPitch;
    extern __shared__ __align__(16) uint8_t s_raw[];              // the tile as it came, packed columns, their scales (not with MODE 1)
    uint8_t *s_out = s_raw + 128 * kPitch, *s_scale = s_out + 128 * kOutPitch;
    __shared__ int32_t s_place[3];
    grid_launch_dependents();
    grid_dependency_wait();
    const int32_t rb = static_cast<int32_t>(blockIdx.y);
    int64_t row0 = rb * 128ll, row_end = p.rows;                  // rows row0 .. row_end - 1 of the input
    if (p.offsets != nullptr) {
        if (threadIdx.x < 32) {
            int32_t first = 0, end = 0;
            const bool found = block_of_group(p.offsets, p.groups, static_cast<int32_t>(p.rows), rb, threadIdx.x, first, end);
            if (threadIdx.x == 0) { s_place[0] = found; s_place[1] = first; s_place[2] = end; }
        }
        __syncthreads();
        if (!s_place[0]) return;                                  // beyond the last group (block-uniform)
        row0 = s_place[1];
        row_end = s_place[2];
    }
    const int64_t matrix = blockIdx.z;
    const float factor = NV ? p.factor[matrix] : 0.0f, g = factor >= 7.888609052210118e-31f ? __frcp_rn(factor) : 0.0f;        // 2^-100
    const T *x = static_cast<const T *>(p.x) + matrix * p.rows * p.ldx;
    uint8_t *q = p.q + matrix * p.rows * p.ldq, *q_cols = p.q_cols + matrix * p.cols * p.ldq_cols;
    const int64_t atoms = (p.cols + kAtom - 1) / kAtom, col_atoms = (p.col_rows + kAtom - 1) / kAtom, col_tiles = (p.cols + 127) / 128;
    uint8_t *scales = p.scales + (matrix * p.row_tiles + rb) * atoms * 512, *scales_cols = p.scales_cols + matrix * col_tiles * col_atoms * 512;
    const uint32_t sub = threadIdx.x & 7u;
    for (int64_t ct = blockIdx.x; ct < col_tiles; ct += gridDim.x) {
        const int64_t col = ct * 128 + sub * 16;
        Raw16<T> raw[4];
        // a whole tile of a plain matrix takes its loads and stores without a test per row
        const bool whole = p.vec_ok && p.row_index == nullptr && row0 + 128 <= row_end && ct * 128 + 128 <= p.cols;
        const int64_t my_row = row0 + (threadIdx.x >> 3);
        if (whole) {
            const T *src = x + my_row * p.ldx + col;
#pragma unroll
            for (int i = 0; i < 4; ++i) raw[i] = load16<T>(src + i * 32 * p.ldx, 0, 16, 1);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if (whole) break;
            const int64_t r = my_row + 32 * i;
            const T *src = nullptr;
            if (r < row_end) {
                if (p.row_index == nullptr) {
                    src = x + r * p.ldx;
                } else {
                    const int64_t k = p.row_index[r];
                    if (k >= 0 && k < p.x_rows) src = x + k * p.ldx;
                }
            }
            raw[i] = load16<T>(src, col, p.cols, p.vec_ok);
        }
        if constexpr (MODE != 1) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                uint8_t *dst = s_raw + ((threadIdx.x >> 3) + 32 * i) * kPitch + sub * 16 * sizeof(T);
                constexpr int kVec = static_cast<int>(sizeof(T));
#pragma unroll
                for (int j = 0; j < kVec; ++j) {
                    // lanes 4 to 7 start at another piece: the eight lanes of a row then reach all banks
                    const uint32_t k = sizeof(T) == 2 ? (static_cast<uint32_t>(j) ^ (sub >> 2)) : (static_cast<uint32_t>(j) + (sub >> 1)) & 3u;
                    uint4 v;
                    if constexpr (kVec == 2) {
                        v = k ? make_uint4(raw[i].w[4], raw[i].w[5], raw[i].w[6], raw[i].w[7]) : make_uint4(raw[i].w[0], raw[i].w[1], raw[i].w[2], raw[i].w[3]);
                    } else {
                        const uint4 a = k & 1u ? make_uint4(raw[i].w[4], raw[i].w[5], raw[i].w[6], raw[i].w[7]) : make_uint4(raw[i].w[0], raw[i].w[1], raw[i].w[2], raw[i].w[3]);
                        const uint4 b = k & 1u ? make_uint4(raw[i].w[12], raw[i].w[13], raw[i].w[14], raw[i].w[15]) : make_uint4(raw[i].w[8], raw[i].w[9], raw[i].w[10], raw[i].w[11]);
                        v = k & 2u ? b : a;
                    }
                    reinterpret_cast<uint4 *>(dst)[k] = v;
                }
            }
        }
        if constexpr (MODE != 2) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                uint32_t m = 0u;
                if constexpr (sizeof(T) == 2) {
                    m = larger16(pair_magnitudes<8>(raw[i].w));
                } else {
#pragma unroll
                    for (int j = 0; j < 16; ++j) m = magnitude_max<T>(m, raw[i].w[j]);
                }
                if constexpr (!NV) m = max(m, __shfl_xor_sync(0xffffffffu, m, 1));
                const BlockStep s = block_step<NV>(magnitude_of(m, T()), factor, g);
                // the scales of four blocks make a word
                uint32_t word = NV ? s.byte << (8u * (sub & 3u)) : s.byte << (8u * (sub >> 1));
                word |= __shfl_xor_sync(0xffffffffu, word, NV ? 1 : 2);
                word |= __shfl_xor_sync(0xffffffffu, word, NV ? 2 : 4);
                const uint32_t k = (threadIdx.x >> 3) + 32u * i;
                const int64_t atom = ct * (128 / kAtom) + (NV ? sub >> 2 : 0u);
                if ((NV ? sub & 3u : sub) == 0u && atom < atoms) *reinterpret_cast<uint32_t *>(scales + atom * 512 + (k & 31u) * 16u + (k >> 5) * 4u) = word;
                float f[16];
                if constexpr (sizeof(T) == 4) {
#pragma unroll
                    for (int j = 0; j < 16; ++j) f[j] = __uint_as_float(raw[i].w[j]);
                } else {
#pragma unroll
                    for (int j = 0; j < 8; ++j) two_floats(raw[i].w[j], f[2 * j], f[2 * j + 1], T());
                }
                bring_near<NV>(f, s);
                const uint2 v = make_uint2(quantize8<NV>(f, s), quantize8<NV>(f + 8, s));
                const int64_t r = row0 + k;
                if (whole) {
                    *reinterpret_cast<uint2 *>(q + my_row * p.ldq + i * 32 * p.ldq + col / 2) = v;
                } else if (r < row_end) {
                    uint8_t *dst = q + r * p.ldq + col / 2;
                    if (col + 16 <= p.cols) {
                        *reinterpret_cast<uint2 *>(dst) = v;
                    } else {
#pragma unroll
                        for (int j = 0; j < 8; ++j)
                            if (col + 2 * j < p.cols) dst[j] = static_cast<uint8_t>((j < 4 ? v.x >> (8 * j) : v.y >> (8 * (j - 4))) & 0xffu);
                    }
                }
            }
        }
        if constexpr (MODE != 1) {
            __syncthreads();
            // 32 rows (part of the tile's four) of a column, or of two: blocks, values, scales.  A part of a block, 16 rows, at a time
            auto put = [&](const uint2 (&v)[2], uint32_t c, uint32_t part, uint32_t b0, uint32_t b1) {
                *reinterpret_cast<uint4 *>(s_out + c * kOutPitch + part * 16u) = make_uint4(v[0].x, v[0].y, v[1].x, v[1].y);
                if constexpr (NV) *reinterpret_cast<unsigned short *>(s_scale + (part >> 1) * 512u + (c & 31u) * 16u + (c >> 5) * 4u + (part & 1u) * 2u) = static_cast<unsigned short>(b0 | (b1 << 8));
                else s_scale[(c & 31u) * 16u + (c >> 5) * 4u + part] = static_cast<uint8_t>(b0);
            };
            if constexpr (sizeof(T) == 2) {
                const uint32_t pair = threadIdx.x & 63u, part = threadIdx.x >> 6;
                const uint8_t *src = s_raw + part * 32u * kPitch + pair * 4u;
                uint32_t w[32];
                uint2 lo[2], hi[2];
                uint32_t byte_lo[2], byte_hi[2];
                BlockStep s_lo, s_hi;
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    if (NV || k == 0) {
#pragma unroll
                        for (int j = 0; j < (NV ? 16 : 32); ++j) w[16 * k + j] = *reinterpret_cast<const uint32_t *>(src + (16 * k + j) * kPitch);
                        const uint32_t m = pair_magnitudes<NV ? 16 : 32>(w + 16 * k);
                        s_lo = block_step<NV>(magnitude_of(m & 0xffffu, T()), factor, g);
                        s_hi = block_step<NV>(magnitude_of(m >> 16, T()), factor, g);
                    }
                    float f[16], h[16];
#pragma unroll
                    for (int j = 0; j < 16; ++j) two_floats(w[16 * k + j], f[j], h[j], T());
                    bring_near<NV>(f, s_lo);
                    bring_near<NV>(h, s_hi);
                    lo[k] = make_uint2(quantize8<NV>(f, s_lo), quantize8<NV>(f + 8, s_lo));
                    hi[k] = make_uint2(quantize8<NV>(h, s_hi), quantize8<NV>(h + 8, s_hi));
                    byte_lo[k] = s_lo.byte;
                    byte_hi[k] = s_hi.byte;
                }
                put(lo, 2u * pair, part, byte_lo[0], byte_lo[1]);
                put(hi, 2u * pair + 1u, part, byte_hi[0], byte_hi[1]);
            } else {
#pragma unroll 1
                for (uint32_t i = 0; i < 2; ++i) {
                    const uint32_t c = threadIdx.x & 127u, part = (threadIdx.x >> 7) + 2u * i;
                    float f[2][16];
                    uint32_t m[2] = {0u, 0u};
#pragma unroll
                    for (int j = 0; j < 32; ++j) {
                        const uint32_t w = *reinterpret_cast<const uint32_t *>(s_raw + (part * 32u + j) * kPitch + c * 4u);
                        m[j / 16] = magnitude_max<T>(m[j / 16], w);
                        f[j / 16][j % 16] = __uint_as_float(w);
                    }
                    if constexpr (!NV) m[0] = m[1] = max(m[0], m[1]);
                    uint2 v[2];
                    uint32_t byte[2];
#pragma unroll
                    for (int k = 0; k < 2; ++k) {
                        const BlockStep s = block_step<NV>(magnitude_of(m[k], T()), factor, g);
                        bring_near<NV>(f[k], s);
                        v[k] = make_uint2(quantize8<NV>(f[k], s), quantize8<NV>(f[k] + 8, s));
                        byte[k] = s.byte;
                    }
                    put(v, c, part, byte[0], byte[1]);
                }
            }
            __syncthreads();
            const int64_t at = rb * 64ll, width = (p.col_rows + 1) / 2;           // the tile's bytes of a column; the column's
#pragma unroll
            for (uint32_t i = 0; i < 2; ++i) {
                const uint32_t c = (threadIdx.x >> 2) + 64u * i, k = threadIdx.x & 3u;
                if (ct * 128 + c < p.cols) {
                    uint8_t *dst = q_cols + (ct * 128 + c) * p.ldq_cols + at + k * 16u;
                    const uint4 v = *reinterpret_cast<const uint4 *>(s_out + c * kOutPitch + k * 16u);
                    const int64_t room = width - at - k * 16;
                    if (room >= 16) {
                        *reinterpret_cast<uint4 *>(dst) = v;
                    } else {
                        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
                        for (int j = 0; j < 16; ++j)
                            if (j < room) dst[j] = static_cast<uint8_t>((w[j / 4] >> (8 * (j & 3))) & 0xffu);
                    }
                }
            }
            if (threadIdx.x < (128 / kAtom) * 32u) {
                const int64_t atom = rb * (128 / kAtom) + (threadIdx.x >> 5);
                if (atom < col_atoms)
                    *reinterpret_cast<uint4 *>(scales_cols + (ct * col_atoms + atom) * 512 + (threadIdx.x & 31u) * 16u) = *reinterpret_cast<const uint4 *>(s_scale + threadIdx.x * 16u);
            }
            if (ct + gridDim.x < col_tiles) __syncthreads();      // the next tile's staging
        }
    }
}

// ---- the tensor's factor -------------------------------------------------------------------------------------------

constexpr int kFp4FactorThreads = 512;
constexpr int kFp4FactorCluster = 8;

// max |x| over the finite elements of a matrix, as the factor's bit pattern (monotone in the maximum, so that factors meet by their maximum).  CLUSTER: the CTAs of one
// cluster have the whole matrix (grid.y: matrices) and write the factor; else every CTA raises it by an atomic maximum (whose order does not matter).
template <class T, bool CLUSTER>
__global__ void __launch_bounds__(kFp4FactorThreads)
fp4_factor_kernel(const T *x0, int64_t ldx, int64_t rows, int64_t cols, int32_t vec_ok, float *factor)
{
    __shared__ uint32_t s_max[kFp4FactorThreads / 32];
    __shared__ uint32_t s_all;
    grid_launch_dependents();
    grid_dependency_wait();
    const T *x = x0 + blockIdx.y * rows * ldx;
    constexpr uint32_t kInf = sizeof(T) == 4 ? 0x7f800000u : 0u;
    uint32_t m = 0u;
    const int64_t chunks = (cols + 15) / 16, all = rows * chunks;
    const bool flat = ldx == cols && cols % 16 == 0;               // one run of elements
    auto take = [&](const Raw16<T> &r) {
        uint32_t k = 0u;
#pragma unroll
        for (int j = 0; j < static_cast<int>(4 * sizeof(T)); ++j) k = magnitude_max<T>(k, r.w[j]);
        bool odd;                                                  // a NaN or an infinity among them: element by element
        if constexpr (sizeof(T) == 4) odd = k >= kInf;
        else odd = magnitude_of(larger16(k), T()) != magnitude_of(larger16(k), T());
        if (odd) {
            k = 0u;
#pragma unroll
            for (int j = 0; j < static_cast<int>(4 * sizeof(T)); ++j) {
                if constexpr (sizeof(T) == 4) {
                    const uint32_t a = r.w[j] & 0x7fffffffu;
                    if (a < kInf) k = max(k, a);
                } else {
                    const uint32_t a = r.w[j] & 0x7fffu, b = (r.w[j] >> 16) & 0x7fffu;
                    if (magnitude_of(a, T()) == magnitude_of(a, T())) k = max(k, a);
                    if (magnitude_of(b, T()) == magnitude_of(b, T())) k = max(k, b);
                }
            }
        } else if constexpr (sizeof(T) == 2) {
            k = larger16(k);
        }
        m = max(m, k);
    };
    const int64_t step = static_cast<int64_t>(gridDim.x) * kFp4FactorThreads;
    int64_t i = static_cast<int64_t>(blockIdx.x) * kFp4FactorThreads + threadIdx.x;
    if (flat && vec_ok) {
        for (; i + 3 * step < all; i += 4 * step) {
            Raw16<T> r[4];
#pragma unroll
            for (int u = 0; u < 4; ++u) r[u] = load16<T>(x, (i + u * step) * 16, INT64_MAX, 1);
#pragma unroll
            for (int u = 0; u < 4; ++u) take(r[u]);
        }
        for (; i < all; i += step) take(load16<T>(x, i * 16, INT64_MAX, 1));
    } else {
        for (; i < all; i += step) {
            const int64_t r = i / chunks;
            take(load16<T>(x + r * ldx, (i - r * chunks) * 16, cols, vec_ok));
        }
    }
    m = __reduce_max_sync(0xffffffffu, m);
    if ((threadIdx.x & 31u) == 0u) s_max[threadIdx.x >> 5] = m;
    __syncthreads();
    if (threadIdx.x < 32) {
        m = threadIdx.x < kFp4FactorThreads / 32 ? s_max[threadIdx.x] : 0u;
        m = __reduce_max_sync(0xffffffffu, m);
        if (threadIdx.x == 0) s_all = m;
    }
    if constexpr (CLUSTER) {
        __syncthreads();
        cluster_arrive();
        cluster_wait();
        if (cluster_ctarank() == 0 && threadIdx.x < 32) {
            m = 0u;
            if (threadIdx.x < kFp4FactorCluster) {
                const uint32_t from = mapa(smem_addr(&s_all), threadIdx.x);
                asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(m) : "r"(from) : "memory");
            }
            m = __reduce_max_sync(0xffffffffu, m);
        }
        cluster_arrive();
        cluster_wait();                                            // no CTA leaves while its maximum is read
    }
    if (threadIdx.x == 0 && (!CLUSTER || cluster_ctarank() == 0)) {
        const float a = magnitude_of(m, T());
        // exponents stay inside fp32's: 2^-127 and below become 0, which the quantiser takes for a tensor of zeros
        const int32_t e = a > 0.0f ? max(power_above(a, 11, kMantissa2688), 0) : 0;
        const uint32_t bits = static_cast<uint32_t>(e) << 23;
        if constexpr (CLUSTER) factor[blockIdx.y] = __uint_as_float(bits);
        else atomicMax(reinterpret_cast<uint32_t *>(factor) + blockIdx.y, bits);
    }
}

// ---- back to wide values -------------------------------------------------------------------------------------------

// The values of eight e2m1 codes as pairs of fp16: by CUDA's own conversion, which takes the byte in the lowest place of its register.  (Taking a word, or its halves, apart into 8-bit
// registers in an asm block saves the shifts -- both copies' values of 8191 x 4096 bf16 and the copies themselves 87.9 instead of 90.1 us -- but the compiler loses such a byte's place
// where it knows, or shifts, other parts of the word: zeros after a 16-bit load, wrong values of the fourth byte.)
__device__ __forceinline__ void unpack_e2m1(uint32_t w, uint32_t (&d)[4])
{
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const __half2_raw h = __nv_cvt_fp4x2_to_halfraw2(static_cast<__nv_fp4x2_storage_t>((w >> (8 * i)) & 0xffu), __NV_E2M1);
        d[i] = h.x | static_cast<uint32_t>(h.y) << 16;
    }
}

struct Fp4DequantParams {
    const uint8_t *q;
    const uint8_t *scales;
    const float *factor;
    int64_t rows, cols, ldq, ldo;
    int64_t row_tiles;         // of 128 rows (per group: as many as the padded copy has)
    int32_t walkers;           // CTAs that share a row tile's column tiles
    int32_t vec_ok;            // rows of out start at multiples of 16 bytes
    void *out;
    const int32_t *offsets;
    int32_t groups;
};

constexpr int kFp4DequantThreads = 256;

// A row of a tile, whose pieces 8 lanes hold (v; the lanes of four rows a warp), to a place `to` that starts anywhere: each lane stores the 16 bytes from the next multiple
// of 16 bytes on, its own piece's end and the next piece's start; what the first piece has before that and the last behind it, a piece together, leave by the
// element.  n: elements of the row (0: none); edge: room for a piece.  Whole warps.
template <class T, int PIECES>
__device__ __forceinline__ void store_anywhere(const uint32_t (&v)[PIECES][4], T *to, int32_t n, T *edge)
{
    constexpr int32_t kPiece = 16 / static_cast<int32_t>(sizeof(T));
    const int32_t sub = static_cast<int32_t>(lane_id() & 7u), s = static_cast<int32_t>((0u - static_cast<uint32_t>(reinterpret_cast<uintptr_t>(to))) & 15u) / static_cast<int32_t>(sizeof(T));      // elements up to the first such place
    const int32_t words = s * static_cast<int32_t>(sizeof(T)) / 4;
    const uint32_t pick = sizeof(T) == 2 && (s & 1) ? 0x5432u : 0x3210u;
    const int src = static_cast<int>((lane_id() & 24u) | ((lane_id() + 1u) & 7u));
    uint32_t after[PIECES][4];
#pragma unroll
    for (int u = 0; u < PIECES; ++u)
#pragma unroll
        for (int k = 0; k < 4; ++k) after[u][k] = __shfl_sync(0xffffffffu, v[u][k], src);
    __syncwarp();                                                 // (the edges of the call before)
#pragma unroll
    for (int u = 0; u < PIECES; ++u) {
        uint32_t x[8], y[5], z[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            x[k] = v[u][k];
            x[4 + k] = sub == 7 ? after[(u + 1) % PIECES][k] : after[u][k];      // (the last piece's next is the first)
        }
#pragma unroll
        for (int k = 0; k < 6; ++k) x[k] = words & 2 ? x[k + 2] : x[k];
#pragma unroll
        for (int k = 0; k < 5; ++k) y[k] = words & 1 ? x[k + 1] : x[k];
#pragma unroll
        for (int k = 0; k < 4; ++k) z[k] = __byte_perm(y[k], y[k + 1], pick);
        const uint4 out = make_uint4(z[0], z[1], z[2], z[3]);
        const int32_t e = (u * 8 + sub) * kPiece + s;
        if (u == PIECES - 1 && sub == 7) {
            *reinterpret_cast<uint4 *>(edge) = out;
        } else if (e + kPiece <= n) {
            *reinterpret_cast<uint4 *>(to + e) = out;
        } else if (e < n) {
#pragma unroll
            for (int j = 0; j < kPiece; ++j) {
                if (e + j >= n) continue;
                if constexpr (sizeof(T) == 4) reinterpret_cast<uint32_t *>(to)[e + j] = z[j];
                else reinterpret_cast<unsigned short *>(to)[e + j] = static_cast<unsigned short>(z[j / 2] >> (16 * (j & 1)));
            }
        }
    }
    __syncwarp();
    const int32_t at = sub < kPiece - s ? 128 - kPiece + s + sub : sub - (kPiece - s);
    if (sub < kPiece && at < n) to[at] = edge[sub];
}

// A tile of 128 x 128 elements, as the quantiser's: 8 lanes hold a row's 16-byte pieces of the result, so that their stores fill whole sectors, and a
// thread's four rows (32 apart) have their scales in the same 16 bytes of a scale tile.  (One run of 16 elements per thread, its scale fetched by the byte
// and its result stored in two halves or through shared memory: 8191 x 4096 bf16 21 us along rows, 28 along columns.)
template <class T, bool NV>
__global__ void __launch_bounds__(kFp4DequantThreads)
fp4_dequantize_kernel(const Fp4DequantParams p)
{
    constexpr int kAtom = NV ? 64 : 128, kAtoms = 128 / kAtom;
    constexpr int kPiece = 16 / static_cast<int>(sizeof(T)), kPieces = 16 / kPiece;      // elements of a lane's piece; its pieces of a row
    __shared__ int32_t s_place[3];
    __shared__ __align__(16) T s_edge[kFp4DequantThreads / 8][kPiece];
    grid_launch_dependents();
    grid_dependency_wait();
    const int64_t rb = static_cast<int64_t>(blockIdx.x) / p.walkers;
    int64_t row0 = rb * 128, row_end = p.rows;
    if (p.offsets != nullptr) {
        if (threadIdx.x < 32) {
            int32_t first = 0, end = 0;
            const bool found = block_of_group(p.offsets, p.groups, static_cast<int32_t>(p.rows), static_cast<int32_t>(rb), threadIdx.x, first, end);
            if (threadIdx.x == 0) { s_place[0] = found; s_place[1] = first; s_place[2] = end; }
        }
        __syncthreads();
        if (!s_place[0]) return;                                  // beyond the last group (block-uniform)
        row0 = s_place[1];
        row_end = s_place[2];
    }
    const int64_t matrix = blockIdx.y, atoms = (p.cols + kAtom - 1) / kAtom, col_tiles = (p.cols + 127) / 128;
    const uint8_t *q = p.q + matrix * p.rows * p.ldq, *scales = p.scales + (matrix * p.row_tiles + rb) * atoms * 512;
    T *out = static_cast<T *>(p.out) + matrix * p.rows * p.ldo;
    const float factor = NV ? p.factor[matrix] : 1.0f;
    const uint32_t sub = threadIdx.x & 7u, line = threadIdx.x >> 3;
    const int64_t my_row = row0 + line;
    const int32_t rows = static_cast<int32_t>(min(row_end - row0, static_cast<int64_t>(128)));       // of this tile
    for (int64_t ct = static_cast<int64_t>(blockIdx.x) % p.walkers; ct < col_tiles; ct += p.walkers) {
        const int64_t col0 = ct * 128;
        const int32_t cols = static_cast<int32_t>(min(p.cols - col0, static_cast<int64_t>(128)));
        const bool whole = rows == 128 && cols == 128;            // its loads and stores need no test of their own
        uint32_t sc[kAtoms][4];
#pragma unroll
        for (int a = 0; a < kAtoms; ++a) {
            uint4 v = make_uint4(0u, 0u, 0u, 0u);
            if (a == 0 || ct * kAtoms + a < atoms) v = *reinterpret_cast<const uint4 *>(scales + (ct * kAtoms + a) * 512 + line * 16);
            sc[a][0] = v.x, sc[a][1] = v.y, sc[a][2] = v.z, sc[a][3] = v.w;
        }
        uint32_t w[4][2];                                         // 8 elements each: a piece, or two
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint8_t *src = q + my_row * p.ldq + col0 / 2 + i * 32 * p.ldq;
#pragma unroll
            for (int u = 0; u < kPieces; ++u) {
                const uint32_t at = u * 4 * kPiece + sub * (kPiece / 2);                  // bytes of the tile's row
                uint32_t v = 0u;
                if (whole || (static_cast<int32_t>(line) + 32 * i < rows && static_cast<int32_t>(2 * at) + kPiece <= cols)) {
                    if constexpr (kPiece == 8) v = *reinterpret_cast<const uint32_t *>(src + at);
                    else v = *reinterpret_cast<const unsigned short *>(src + at);
                } else if (static_cast<int32_t>(line) + 32 * i < rows) {
#pragma unroll
                    for (int j = 0; j < kPiece / 2; ++j)
                        if (static_cast<int32_t>(2 * (at + j)) < cols) v |= static_cast<uint32_t>(src[at + j]) << (8 * j);
                }
                if (kPiece == 8 || u % 2 == 0) w[i][u * kPiece / 8] = v;
                else w[i][u / 2] |= v << 16;
            }
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if (32 * i >= rows) break;
            T *dst = out + my_row * p.ldo + col0 + i * 32 * p.ldo;
            uint32_t h[4], v[kPieces][4];
#pragma unroll
            for (int u = 0; u < kPieces; ++u) {
                if (kPiece == 8 || u % 2 == 0) unpack_e2m1(w[i][u * kPiece / 8], h);
                const uint32_t e0 = u * 8 * kPiece + sub * kPiece, b = NV ? (e0 & 63u) >> 4 : e0 >> 5;
                const uint32_t byte = (sc[NV ? u * 8 * kPiece / 64 : 0][i] >> (8u * b)) & 0xffu;
                float s;
                if constexpr (NV) s = __half2float(__half(__nv_cvt_fp8_to_halfraw(static_cast<__nv_fp8_storage_t>(byte), __NV_E4M3))) * factor;
                else s = byte == 0u ? 5.877471754111438e-39f : byte == 255u ? __int_as_float(0x7fffffff) : __uint_as_float(byte << 23);
                float f[kPiece];
#pragma unroll
                for (int j = 0; j < kPiece / 2; ++j) {
                    float lo, hi;
                    two_floats(h[(u * kPiece / 2 + j) & 3], lo, hi, __half());
                    unpack_f32x2(mul_f32x2(pack_f32x2(__float_as_uint(lo), __float_as_uint(hi)), pack_f32x2(__float_as_uint(s), __float_as_uint(s))), f[2 * j], f[2 * j + 1]);
                }
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    if constexpr (sizeof(T) == 4) v[u][k] = __float_as_uint(f[k]);
                    else v[u][k] = pack_pair(f[2 * k], f[2 * k + 1], T());
                }
            }
            if (p.vec_ok && cols == 128) {
                if (static_cast<int32_t>(line) + 32 * i >= rows) continue;
#pragma unroll
                for (int u = 0; u < kPieces; ++u) *reinterpret_cast<uint4 *>(dst + (u * 8 + sub) * kPiece) = make_uint4(v[u][0], v[u][1], v[u][2], v[u][3]);
            } else {
                store_anywhere<T>(v, dst, static_cast<int32_t>(line) + 32 * i < rows ? cols : 0, s_edge[line]);
            }
        }
    }
}

} // namespace hgemm_dev
