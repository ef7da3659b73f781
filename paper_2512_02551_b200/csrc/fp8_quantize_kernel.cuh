// 8-bit quantisation with one scale per block of 128 (1 x 128, 128 x 1, or 128 x 128 elements).
//
// Bound by memory: 2 or 4 bytes read and 1 (rows and columns together: 2) written per element.  Every element is read once and
// stays in registers between the block's maximum and the rounding.
//
//   by rows      16 lanes own a 1 x 128 block, 8 elements each (16 bytes of a 16-bit input); the maximum is four shuffles.
//   otherwise    256 threads own a 128 x 128 tile, thread t the 8 columns 8 (t % 16) of the rows t / 16 + 16 i, i = 0 .. 7; column
//                maxima meet in shared memory.  The same tile gives the row blocks, so both forms cost one read.
//
// Values are x * (m / a) with the quotient rounded once per block; a division per element would bound the kernel by
// arithmetic.  NaN and infinities are left out of the maximum and come out as NaN: x - x is added to the product (0 for every finite x).
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_fp8.h>
#include <stdint.h>

#include "hgemm_device.cuh"

namespace hgemm_dev {

constexpr int kQuantThreads = 256;
constexpr int kQuantMaxGroups = 1024;

struct QuantParams {
    const void *x;
    int64_t ldx, rows, cols, x_rows;
    const int32_t *row_index;
    const int32_t *offsets;
    int32_t groups;
    int32_t vec_ok;            // rows of x start at multiples of 16 bytes
    int32_t e5m2, pow2;
    uint8_t *q;
    int64_t ldq;
    float *scales;
    uint8_t *q_cols;
    int64_t ldq_cols;
    float *scales_cols;
};

struct BlockScale {
    float scale, factor;
};

__device__ __forceinline__ BlockScale block_scale(float amax, int32_t e5m2, int32_t pow2)
{
    const float top = e5m2 ? 57344.0f : 448.0f;
    BlockScale s;
    if (!(amax >= 7.888609052210118e-31f)) {            // 2^-100
        s.scale = 1.0f;
        s.factor = 0.0f;
        return s;
    }
    s.scale = amax / top;
    if (pow2) {
        const uint32_t bits = __float_as_uint(s.scale), e = (bits >> 23) + ((bits & 0x7fffffu) != 0u ? 1u : 0u);
        s.scale = __uint_as_float(e << 23);
        s.factor = __uint_as_float((254u - e) << 23);
    } else {
        s.factor = top / amax;
    }
    return s;
}

__device__ __forceinline__ float finite_or_zero(float a) { return a < __int_as_float(0x7f800000) ? a : 0.0f; }   // a >= 0 or NaN

// Largest magnitude of eight elements, infinities and NaN left out.
__device__ __forceinline__ float amax8(const float (&v)[8])
{
    float m = 0.0f;
#pragma unroll
    for (int i = 0; i < 8; ++i) m = fmaxf(m, finite_or_zero(fabsf(v[i])));
    return m;
}

// Eight elements, quantised.
__device__ __forceinline__ uint2 quantize8(const float (&v)[8], float factor, int32_t e5m2)
{
    uint32_t h[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        float2 f;
        f.x = fmaf(v[2 * i], factor, v[2 * i] - v[2 * i]);
        f.y = fmaf(v[2 * i + 1], factor, v[2 * i + 1] - v[2 * i + 1]);
        h[i] = e5m2 ? __nv_cvt_float2_to_fp8x2(f, __NV_SATFINITE, __NV_E5M2) : __nv_cvt_float2_to_fp8x2(f, __NV_SATFINITE, __NV_E4M3);
    }
    return make_uint2(h[0] | (h[1] << 16), h[2] | (h[3] << 16));
}

__device__ __forceinline__ float to_float(float v) { return v; }
__device__ __forceinline__ float to_float(__half v) { return __half2float(v); }
__device__ __forceinline__ float to_float(__nv_bfloat16 v) { return __bfloat162float(v); }

// Elements col .. col + 7 of a row of x (zeros beyond the matrix; row == nullptr: a row of zeros).
template <class T>
__device__ __forceinline__ void load8(float (&v)[8], const T *row, int64_t col, int64_t cols, int32_t vec_ok)
{
    if (row != nullptr && vec_ok && col + 8 <= cols) {
        __align__(16) T t[8];
        const uint4 *src = reinterpret_cast<const uint4 *>(row + col);
        *reinterpret_cast<uint4 *>(t) = src[0];
        if constexpr (sizeof(T) == 4) *reinterpret_cast<uint4 *>(t + 4) = src[1];
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = to_float(t[i]);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = row != nullptr && col + i < cols ? to_float(row[col + i]) : 0.0f;
    }
}

__device__ __forceinline__ void store8(uint8_t *row, int64_t col, int64_t cols, uint2 v)
{
    if (col + 8 <= cols) {
        *reinterpret_cast<uint2 *>(row + col) = v;             // rows start at multiples of 16 bytes, col is a multiple of 8
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (col + i < cols) row[col + i] = static_cast<uint8_t>((i < 4 ? v.x >> (8 * i) : v.y >> (8 * (i - 4))) & 0xffu);
    }
}

template <class T>
__device__ __forceinline__ const T *source_row(const QuantParams &p, int64_t r)
{
    const T *x = static_cast<const T *>(p.x);
    if (p.row_index == nullptr) return x + r * p.ldx;
    const int64_t i = p.row_index[r];
    return i >= 0 && i < p.x_rows ? x + i * p.ldx : nullptr;
}

template <class T>
__global__ void __launch_bounds__(kQuantThreads)
fp8_quantize_rows_kernel(const QuantParams p)
{
    grid_launch_dependents();
    grid_dependency_wait();
    const int64_t blocks = (p.cols + 127) / 128, total = p.rows * blocks;
    const uint32_t sub = threadIdx.x & 15u;
    // whole warps stay in the loop together: the bound is the warp's first block
    for (int64_t b0 = (blockIdx.x * static_cast<int64_t>(kQuantThreads) + (threadIdx.x & ~31u)) / 16; b0 < total; b0 += gridDim.x * static_cast<int64_t>(kQuantThreads / 16)) {
        const int64_t b = b0 + ((threadIdx.x >> 4) & 1u);
        const bool mine = b < total;
        const int64_t r = mine ? b / blocks : 0, kb = mine ? b - r * blocks : 0, col = kb * 128 + sub * 8;
        float v[8];
        load8<T>(v, mine ? source_row<T>(p, r) : nullptr, col, p.cols, p.vec_ok);
        float m = amax8(v);
#pragma unroll
        for (int d = 8; d >= 1; d >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, d));
        const BlockScale s = block_scale(m, p.e5m2, p.pow2);
        if (mine) {
            store8(p.q + r * p.ldq, col, p.cols, quantize8(v, s.factor, p.e5m2));
            if (sub == 0) p.scales[r * blocks + kb] = s.scale;
        }
    }
}

// MODE: HGEMM_FP8_COLS (2), ROWS | COLS (3) or TILES (4).  grid: x = column blocks of 128, y = row blocks (of the padded copy), z = matrices (TILES).
template <class T, int MODE>
__global__ void __launch_bounds__(kQuantThreads)
fp8_quantize_tile_kernel(const QuantParams p)
{
    __shared__ float s_max[8][128];
    __shared__ int32_t s_place[3];
    grid_launch_dependents();
    grid_dependency_wait();
    const uint32_t warp = threadIdx.x >> 5, lane = threadIdx.x & 31u;
    const int64_t blocks = (p.cols + 127) / 128;
    for (int64_t rb = blockIdx.y;; rb += gridDim.y) {
        int64_t row0 = rb * 128, row_end = p.rows, out0 = row0;        // rows row0 .. row_end - 1 of the input, out0: first row of the copy
        if (MODE == 2 || MODE == 3) {
            if (p.offsets != nullptr) {
                // the group that holds block rb of the padded copy
                __syncthreads();
                if (warp == 0) {
                    int64_t carry = 0;
                    int32_t found = 0, limit = static_cast<int32_t>(p.rows), first = 0, end = 0;
                    for (int32_t base = 0; base < p.groups && !found; base += 32) {
                        const int32_t e = base + static_cast<int32_t>(lane);
                        const int32_t a = min(max(p.offsets[min(e, p.groups)], 0), limit), z = min(max(p.offsets[min(e + 1, p.groups)], 0), limit);
                        int32_t n = e < p.groups && z > a ? (z - a + 127) / 128 : 0, sum = n;
#pragma unroll
                        for (int d = 1; d < 32; d <<= 1) {
                            const int32_t x = __shfl_up_sync(0xffffffffu, sum, d);
                            if (static_cast<int32_t>(lane) >= d) sum += x;
                        }
                        const uint32_t hit = __ballot_sync(0xffffffffu, n > 0 && carry + sum > rb);
                        if (hit) {
                            const int src = __ffs(hit) - 1;
                            const int32_t before = static_cast<int32_t>(carry) + sum - n;
                            first = __shfl_sync(0xffffffffu, a + (static_cast<int32_t>(rb) - before) * 128, src);
                            end = __shfl_sync(0xffffffffu, z, src);
                            found = 1;
                        }
                        carry += __shfl_sync(0xffffffffu, sum, 31);
                    }
                    if (lane == 0) { s_place[0] = found; s_place[1] = first; s_place[2] = end; }
                }
                __syncthreads();
                if (!s_place[0]) return;                               // beyond the last group's rows (block-uniform)
                row0 = s_place[1];
                row_end = s_place[2];
            } else if (row0 >= p.rows) {
                return;
            }
        } else if (row0 >= p.rows) {
            return;
        }
        const int64_t matrix = MODE == 4 ? blockIdx.z : 0;
        const int64_t col = blockIdx.x * 128ll + (threadIdx.x & 15u) * 8;
        float v[8][8];
        float row_max[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int64_t r = row0 + (threadIdx.x >> 4) + 16 * i;
            const T *src = nullptr;
            if (r < row_end) src = MODE == 4 ? static_cast<const T *>(p.x) + (matrix * p.rows + r) * p.ldx : source_row<T>(p, r);
            load8<T>(v[i], src, col, p.cols, p.vec_ok);
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            row_max[i] = amax8(v[i]);
            if (MODE == 3) {
#pragma unroll
                for (int d = 8; d >= 1; d >>= 1) row_max[i] = fmaxf(row_max[i], __shfl_xor_sync(0xffffffffu, row_max[i], d));
            }
        }
        if (MODE == 3) {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int64_t r = row0 + (threadIdx.x >> 4) + 16 * i;
                if (r < row_end) {
                    const BlockScale s = block_scale(row_max[i], p.e5m2, p.pow2);
                    store8(p.q + r * p.ldq, col, p.cols, quantize8(v[i], s.factor, p.e5m2));
                    if ((threadIdx.x & 15u) == 0) p.scales[r * blocks + blockIdx.x] = s.scale;
                }
            }
        }
        if (MODE == 4) {
            float m = 0.0f;
#pragma unroll
            for (int i = 0; i < 8; ++i) m = fmaxf(m, row_max[i]);
#pragma unroll
            for (int d = 16; d >= 1; d >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, d));
            __syncthreads();
            if (lane == 0) s_max[0][warp] = m;
            __syncthreads();
#pragma unroll
            for (int i = 0; i < 8; ++i) m = fmaxf(m, s_max[0][i]);
            const BlockScale s = block_scale(m, p.e5m2, p.pow2);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int64_t r = row0 + (threadIdx.x >> 4) + 16 * i;
                if (r < row_end) store8(p.q + (matrix * p.rows + r) * p.ldq, col, p.cols, quantize8(v[i], s.factor, p.e5m2));
            }
            if (threadIdx.x == 0) p.scales[(matrix * ((p.rows + 127) / 128) + rb) * blocks + blockIdx.x] = s.scale;
        } else {
            float cm[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                cm[j] = 0.0f;
#pragma unroll
                for (int i = 0; i < 8; ++i) cm[j] = fmaxf(cm[j], finite_or_zero(fabsf(v[i][j])));
                cm[j] = fmaxf(cm[j], __shfl_xor_sync(0xffffffffu, cm[j], 16));
            }
            __syncthreads();                                            // the previous turn's readers are done
            if (lane < 16) {
#pragma unroll
                for (int j = 0; j < 8; ++j) s_max[warp][lane * 8 + j] = cm[j];
            }
            __syncthreads();
            BlockScale s[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                float m = 0.0f;
#pragma unroll
                for (int w = 0; w < 8; ++w) m = fmaxf(m, s_max[w][(threadIdx.x & 15u) * 8 + j]);
                s[j] = block_scale(m, p.e5m2, p.pow2);
            }
            const bool padded = p.offsets != nullptr;                   // rows up to the next multiple of 128 are written (zeros)
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int64_t k = (threadIdx.x >> 4) + 16 * i;
                if (row0 + k < row_end || padded) {
                    uint32_t h[4];
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        float2 f;
                        f.x = fmaf(v[i][2 * j], s[2 * j].factor, v[i][2 * j] - v[i][2 * j]);
                        f.y = fmaf(v[i][2 * j + 1], s[2 * j + 1].factor, v[i][2 * j + 1] - v[i][2 * j + 1]);
                        h[j] = p.e5m2 ? __nv_cvt_float2_to_fp8x2(f, __NV_SATFINITE, __NV_E5M2) : __nv_cvt_float2_to_fp8x2(f, __NV_SATFINITE, __NV_E4M3);
                    }
                    store8(p.q_cols + (out0 + k) * p.ldq_cols, col, p.cols, make_uint2(h[0] | (h[1] << 16), h[2] | (h[3] << 16)));
                }
            }
            if (threadIdx.x < 16) {
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    if (col + j < p.cols) p.scales_cols[rb * p.cols + col + j] = s[j].scale;
            }
        }
    }
}

} // namespace hgemm_dev
