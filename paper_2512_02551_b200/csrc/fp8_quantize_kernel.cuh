// 8-bit quantisation with one scale per block of 128 (1 x 128, 128 x 1, or 128 x 128 elements).
//
// Bound by memory: 2 or 4 bytes read and 1 (rows and columns together: 2) written per element.  Every element is read once and
// stays in registers, as it came, between the block's maximum and the rounding.
//
//   by rows      8 lanes own a 1 x 128 block, 16 elements each (16-byte stores); the maximum is three shuffles.  Four blocks in
//                flight per lane once there are enough of them to fill the GPU.
//   otherwise    256 threads own a 128 x 128 tile, thread t the 8 columns 8 (t % 16) of the rows t / 16 + 16 i, i = 0 .. 7; column
//                maxima meet in shared memory.  The same tile gives the row blocks, so both forms cost one read.
//
// Values are x * (m / a) with the quotient rounded once per block; a division per element would bound the kernel by arithmetic, and
// so would every lane dividing for every row or column it holds: one lane per block does.  NaN passes through maximum (which skips
// it) and product by itself; a block whose maximum is infinite has its infinities made NaN first.
//
// Measured (B200): 8192 x 8192 bf16 by rows 30 us (6.6 TB/s, the copy rate), rows and columns 53 us (5.1 TB/s), tiles 35 us (5.7 TB/s); fp32
// rows and columns 72 us (5.6 TB/s).  The 16-bit forms that make columns are bound by instructions (17 an element).  Laid out per group, a
// warp of every CTA walks the offsets first, 32 groups a step: 32768 x 2048 bf16, rows and columns, 51 us without groups, 62 us with 32 of
// them, 124 us with 256, 528 us with 1024; gathered from 8192 rows on the way 89 us with 32.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_fp8.h>
#include <stdint.h>

#include <type_traits>

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
    int32_t pow2;
    FastDiv fd_blocks;         // blocks of a row
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

__device__ __forceinline__ float quant_inf() { return __int_as_float(0x7f800000); }

// Eight consecutive elements as they came.
template <class T>
struct Raw8 {
    uint4 v[sizeof(T) / 2];
};

template <class T>
__device__ __forceinline__ Raw8<T> load8_whole(const T *src)
{
    Raw8<T> r;
    r.v[0] = reinterpret_cast<const uint4 *>(src)[0];
    if constexpr (sizeof(T) == 4) r.v[1] = reinterpret_cast<const uint4 *>(src)[1];
    return r;
}

// Elements col .. col + 7 of a row of x (zeros beyond the matrix; row == nullptr: a row of zeros).
template <class T>
__device__ __forceinline__ Raw8<T> load8(const T *row, int64_t col, int64_t cols, int32_t vec_ok)
{
    Raw8<T> r;
    if (row != nullptr && vec_ok && col + 8 <= cols) {
        r = load8_whole<T>(row + col);
    } else {
        __align__(16) T t[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) t[i] = row != nullptr && col + i < cols ? row[col + i] : T(0.0f);
        r.v[0] = *reinterpret_cast<const uint4 *>(t);
        if constexpr (sizeof(T) == 4) r.v[1] = *reinterpret_cast<const uint4 *>(t + 4);
    }
    return r;
}

__device__ __forceinline__ void floats_of(const Raw8<float> &r, float (&f)[8])
{
    const uint32_t w[8] = {r.v[0].x, r.v[0].y, r.v[0].z, r.v[0].w, r.v[1].x, r.v[1].y, r.v[1].z, r.v[1].w};
#pragma unroll
    for (int i = 0; i < 8; ++i) f[i] = __uint_as_float(w[i]);
}
__device__ __forceinline__ float2 pair_of(uint32_t w, __half) { return __half22float2(*reinterpret_cast<const __half2 *>(&w)); }
__device__ __forceinline__ float2 pair_of(uint32_t w, __nv_bfloat16) { return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u)); }
template <class T>
__device__ __forceinline__ void floats_of(const Raw8<T> &r, float (&f)[8])
{
    const uint32_t w[4] = {r.v[0].x, r.v[0].y, r.v[0].z, r.v[0].w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float2 p = pair_of(w[i], T());
        f[2 * i] = p.x;
        f[2 * i + 1] = p.y;
    }
}

// Infinities become NaN.
__device__ __forceinline__ uint32_t no_infinity(uint32_t w, float) { return (w & 0x7fffffffu) == 0x7f800000u ? 0x7fffffffu : w; }
template <class T>
__device__ __forceinline__ uint32_t no_infinity(uint32_t w, T)
{
    constexpr uint32_t inf = std::is_same<T, __half>::value ? 0x7c00u : 0x7f80u;
    if ((w & 0x7fffu) == inf) w |= 0x7fffu;
    if (((w >> 16) & 0x7fffu) == inf) w |= 0x7fff0000u;
    return w;
}
template <class T>
__device__ __forceinline__ void no_infinities(Raw8<T> &r)
{
#pragma unroll
    for (int i = 0; i < static_cast<int>(sizeof(T) / 2); ++i)
        r.v[i] = make_uint4(no_infinity(r.v[i].x, T()), no_infinity(r.v[i].y, T()), no_infinity(r.v[i].z, T()), no_infinity(r.v[i].w, T()));
}

// Two magnitudes of a 16-bit type in one register, compared two at a time; NaN loses against a number.
__device__ __forceinline__ uint32_t abs_max2(uint32_t m, uint32_t w, __half)
{
    const __half2 r = __hmax2(*reinterpret_cast<const __half2 *>(&m), __habs2(*reinterpret_cast<const __half2 *>(&w)));
    return *reinterpret_cast<const uint32_t *>(&r);
}
__device__ __forceinline__ uint32_t abs_max2(uint32_t m, uint32_t w, __nv_bfloat16)
{
    const __nv_bfloat162 r = __hmax2(*reinterpret_cast<const __nv_bfloat162 *>(&m), __habs2(*reinterpret_cast<const __nv_bfloat162 *>(&w)));
    return *reinterpret_cast<const uint32_t *>(&r);
}
template <class T>
__device__ __forceinline__ float larger_half(uint32_t m)
{
    const float2 f = pair_of(m, T());
    return fmaxf(f.x, f.y);
}

// Largest magnitude of eight elements, NaN left out.
__device__ __forceinline__ float amax8(const Raw8<float> &r)
{
    float f[8], m = 0.0f;
    floats_of(r, f);
#pragma unroll
    for (int i = 0; i < 8; ++i) m = fmaxf(m, fabsf(f[i]));
    return m;
}
template <class T>
__device__ __forceinline__ float amax8(const Raw8<T> &r)
{
    uint32_t m = abs_max2(0u, r.v[0].x, T());
    m = abs_max2(m, r.v[0].y, T());
    m = abs_max2(m, r.v[0].z, T());
    return larger_half<T>(abs_max2(m, r.v[0].w, T()));
}
// Keeps the compiler from holding converted copies of `r` in registers from here on.
template <class T>
__device__ __forceinline__ void forget_conversions(Raw8<T> &r)
{
    asm volatile("" : "+r"(r.v[0].x), "+r"(r.v[0].y), "+r"(r.v[0].z), "+r"(r.v[0].w));
}

__device__ __forceinline__ uint32_t to_fp8x2(float a, float b, int32_t e5m2)
{
    const float2 f = make_float2(a, b);
    return e5m2 ? __nv_cvt_float2_to_fp8x2(f, __NV_SATFINITE, __NV_E5M2) : __nv_cvt_float2_to_fp8x2(f, __NV_SATFINITE, __NV_E4M3);
}

__device__ __forceinline__ uint2 quantize8(const float (&v)[8], float factor, int32_t e5m2)
{
    uint32_t h[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) h[i] = to_fp8x2(v[2 * i] * factor, v[2 * i + 1] * factor, e5m2);
    return make_uint2(h[0] | (h[1] << 16), h[2] | (h[3] << 16));
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

// UNROLL: blocks in flight per group of 8 lanes.  DENSE: x and the copy are one run of whole blocks (no gather, rows of whole blocks
// that follow one another), so that a block's place is its number.
template <class T, int UNROLL, bool DENSE, bool E5M2>
__global__ void __launch_bounds__(kQuantThreads, UNROLL == 1 ? 4 : sizeof(T) == 4 ? 2 : 3)
fp8_quantize_rows_kernel(const QuantParams p)
{
    grid_launch_dependents();
    grid_dependency_wait();
    const int32_t blocks = static_cast<int32_t>(p.fd_blocks.d);
    const int32_t total = static_cast<int32_t>(p.rows) * blocks;          // below 2^31: checked by the host
    const int32_t sub = static_cast<int32_t>(threadIdx.x & 7u), lane_block = static_cast<int32_t>((threadIdx.x >> 3) & 3u);
    const int32_t warps = static_cast<int32_t>(gridDim.x) * (kQuantThreads / 32);
    const int32_t warp = static_cast<int32_t>(blockIdx.x) * (kQuantThreads / 32) + static_cast<int32_t>(threadIdx.x >> 5);
    // a warp takes 4 UNROLL consecutive blocks at a time; whole warps stay in the loop together
    for (int64_t b0 = static_cast<int64_t>(warp) * (4 * UNROLL); b0 < total; b0 += static_cast<int64_t>(warps) * (4 * UNROLL)) {
        Raw8<T> raw[UNROLL][2];
        int64_t q_at[UNROLL];                                             // where a lane's values go (-1: no block)
        int32_t room[UNROLL];                                             // elements up to the row's end
        const int32_t r0 = DENSE ? 0 : fast_div(static_cast<int32_t>(b0), p.fd_blocks), k0 = static_cast<int32_t>(b0) - r0 * blocks;
        if (DENSE || k0 + 4 * UNROLL <= blocks) {
            // the warp's blocks lie in one row
            const T *src = DENSE ? static_cast<const T *>(p.x) : source_row<T>(p, r0);
#pragma unroll
            for (int u = 0; u < UNROLL; ++u) {
                const int64_t k = (DENSE ? b0 : static_cast<int64_t>(k0)) + u * 4 + lane_block;
                const bool mine = !DENSE || k < total;
                const int64_t col = k * 128 + sub * 16;
                q_at[u] = mine ? (DENSE ? col : r0 * p.ldq + col) : -1;
                room[u] = DENSE ? 128 : static_cast<int32_t>(p.cols - col);
                if (DENSE || (src != nullptr && p.vec_ok && room[u] >= 16)) {
                    raw[u][0] = load8_whole<T>(src + (mine ? col : 0));
                    raw[u][1] = load8_whole<T>(src + (mine ? col + 8 : 8));
                } else {
                    raw[u][0] = load8<T>(src, col, p.cols, 0);
                    raw[u][1] = load8<T>(src, col + 8, p.cols, 0);
                }
            }
        } else {
#pragma unroll
            for (int u = 0; u < UNROLL; ++u) {
                const int64_t b = b0 + u * 4 + lane_block;
                const bool mine = b < total;
                const int32_t r = mine ? fast_div(static_cast<int32_t>(b), p.fd_blocks) : 0;
                const int64_t col = (static_cast<int32_t>(b) - r * blocks) * 128ll + sub * 16;
                const T *src = mine ? source_row<T>(p, r) : nullptr;
                q_at[u] = mine ? r * p.ldq + col : -1;
                room[u] = static_cast<int32_t>(p.cols - col);
                raw[u][0] = load8<T>(src, col, p.cols, p.vec_ok);
                raw[u][1] = load8<T>(src, col + 8, p.cols, p.vec_ok);
            }
        }
        float m[UNROLL], top = 0.0f;
#pragma unroll
        for (int u = 0; u < UNROLL; ++u) {
            m[u] = fmaxf(amax8(raw[u][0]), amax8(raw[u][1]));
            top = fmaxf(top, m[u]);
        }
        if (__any_sync(0xffffffffu, top == quant_inf())) {
#pragma unroll
            for (int u = 0; u < UNROLL; ++u) {
                no_infinities(raw[u][0]);
                no_infinities(raw[u][1]);
                m[u] = fmaxf(amax8(raw[u][0]), amax8(raw[u][1]));
            }
        }
        float own = 0.0f;                                                 // lane u of a group of 8 makes the scale of its block u
#pragma unroll
        for (int u = 0; u < UNROLL; ++u) {
#pragma unroll
            for (int d = 4; d >= 1; d >>= 1) m[u] = fmaxf(m[u], __shfl_xor_sync(0xffffffffu, m[u], d));
            if (sub == u) own = m[u];
        }
        const BlockScale s = block_scale(own, E5M2, p.pow2);
        const int64_t own_block = b0 + sub * 4 + lane_block;
        if (sub < UNROLL && own_block < total) p.scales[own_block] = s.scale;
#pragma unroll
        for (int u = 0; u < UNROLL; ++u) {
            const float factor = __shfl_sync(0xffffffffu, s.factor, u, 8);
            if (q_at[u] >= 0) {
                float f[8], g[8];
                floats_of(raw[u][0], f);
                floats_of(raw[u][1], g);
                const uint2 lo = quantize8(f, factor, E5M2), hi = quantize8(g, factor, E5M2);
                uint8_t *dst = p.q + q_at[u];
                if (DENSE || room[u] >= 16) {
                    *reinterpret_cast<uint4 *>(dst) = make_uint4(lo.x, lo.y, hi.x, hi.y);
                } else {
                    store8(dst, 0, room[u], lo);
                    store8(dst, 8, room[u], hi);
                }
            }
        }
    }
}

// MODE: HGEMM_FP8_COLS (2), ROWS | COLS (3) or TILES (4).  grid: x = column blocks of 128, y = row blocks (as many as the padded copy has; ROWS | COLS: and those of rows of no group), z = matrices (TILES).
template <class T, int MODE, bool E5M2>
__global__ void __launch_bounds__(kQuantThreads, sizeof(T) == 4 ? 2 : 3)
fp8_quantize_tile_kernel(const QuantParams p)
{
    __shared__ float s_max[8][128];
    __shared__ __align__(16) float s_factor[128];
    __shared__ int32_t s_place[3];
    grid_launch_dependents();
    grid_dependency_wait();
    const uint32_t warp = threadIdx.x >> 5, lane = threadIdx.x & 31u;
    const int64_t blocks = (p.cols + 127) / 128;
    const int64_t rb = blockIdx.y;
    int64_t row0 = rb * 128, row_end = p.rows;                         // rows row0 .. row_end - 1 of the input
    const int64_t out0 = row0;                                         // first row of the copy
    bool rows_only = false;                                            // rows of no group: they have a row copy alone
    if (MODE != 4 && p.offsets != nullptr) {
        // The group that holds block rb of the padded copy.  The offsets are clamped as the products clamp them: to [0, rows], each at
        // least as large as those before it.  Then the groups' blocks fit the copy, whatever the caller's values.  Blocks behind those of the
        // groups take the rows of no group, those ahead of the first group's and then those from the last offset on.
        if (warp == 0) {
            int32_t carry = 0, found = 0, first = 0, end = 0, last = 0;
            const int32_t limit = static_cast<int32_t>(p.rows);
            for (int32_t base = 0; base < p.groups && !found; base += 32) {
                const int32_t e = base + static_cast<int32_t>(lane);
                int32_t a = min(max(p.offsets[min(e, p.groups)], 0), limit);
#pragma unroll
                for (int d = 1; d < 32; d <<= 1) {
                    const int32_t x = __shfl_up_sync(0xffffffffu, a, d);
                    if (static_cast<int32_t>(lane) >= d) a = max(a, x);
                }
                a = max(a, last);
                int32_t z = __shfl_down_sync(0xffffffffu, a, 1);
                if (lane == 31) z = max(a, min(max(p.offsets[min(e + 1, p.groups)], 0), limit));
                last = __shfl_sync(0xffffffffu, z, 31);
                const int32_t n = e < p.groups ? (z - a + 127) / 128 : 0;
                int32_t sum = n;
#pragma unroll
                for (int d = 1; d < 32; d <<= 1) {
                    const int32_t x = __shfl_up_sync(0xffffffffu, sum, d);
                    if (static_cast<int32_t>(lane) >= d) sum += x;
                }
                const uint32_t hit = __ballot_sync(0xffffffffu, n > 0 && carry + sum > rb);
                if (hit) {
                    const int src = __ffs(hit) - 1;
                    const int32_t before = carry + sum - n;
                    first = __shfl_sync(0xffffffffu, a + (static_cast<int32_t>(rb) - before) * 128, src);
                    end = __shfl_sync(0xffffffffu, z, src);
                    found = 1;
                }
                carry += __shfl_sync(0xffffffffu, sum, 31);
            }
            if (MODE == 3 && !found) {
                const int32_t ahead = min(max(p.offsets[0], 0), limit), n = (ahead + 127) / 128, i = static_cast<int32_t>(rb) - carry;
                first = i < n ? i * 128 : last + (i - n) * 128;
                end = i < n ? ahead : limit;
                found = first < end ? 2 : 0;
            }
            if (lane == 0) { s_place[0] = found; s_place[1] = first; s_place[2] = end; }
        }
        __syncthreads();
        if (!s_place[0]) return;                                       // beyond the last rows (block-uniform)
        rows_only = s_place[0] == 2;
        row0 = s_place[1];
        row_end = s_place[2];
    }
    const int64_t matrix = MODE == 4 ? blockIdx.z : 0;
    const int64_t col = blockIdx.x * 128ll + (threadIdx.x & 15u) * 8;
    const int64_t my_row = row0 + (threadIdx.x >> 4);              // and every 16th after it
    Raw8<T> raw[8];
    // a whole tile of a plain matrix takes its loads and stores without a test per row
    const bool whole = p.vec_ok && p.row_index == nullptr && row0 + 128 <= row_end && blockIdx.x * 128ll + 128 <= p.cols;
    if (whole) {
        const T *src = static_cast<const T *>(p.x) + (matrix * p.rows + my_row) * p.ldx + col;
#pragma unroll
        for (int i = 0; i < 8; ++i) raw[i] = load8_whole<T>(src + 16 * i * p.ldx);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int64_t r = my_row + 16 * i;
            const T *src = nullptr;
            if (r < row_end) src = MODE == 4 ? static_cast<const T *>(p.x) + (matrix * p.rows + r) * p.ldx : source_row<T>(p, r);
            raw[i] = load8<T>(src, col, p.cols, p.vec_ok);
        }
    }
    // Maxima; once more, with the infinities made NaN, if the tile has any.
    float row_max[8], col_max[8];
    auto maxima = [&]() {
        if constexpr (sizeof(T) == 4) {
#pragma unroll
            for (int j = 0; j < 8; ++j) col_max[j] = 0.0f;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                float f[8];
                floats_of(raw[i], f);
                row_max[i] = amax8(raw[i]);
                if (MODE != 4) {
#pragma unroll
                    for (int j = 0; j < 8; ++j) col_max[j] = fmaxf(col_max[j], fabsf(f[j]));
                }
            }
        } else {
            uint32_t c[4] = {0u, 0u, 0u, 0u};
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                row_max[i] = amax8(raw[i]);
                if (MODE != 4) {
                    c[0] = abs_max2(c[0], raw[i].v[0].x, T());
                    c[1] = abs_max2(c[1], raw[i].v[0].y, T());
                    c[2] = abs_max2(c[2], raw[i].v[0].z, T());
                    c[3] = abs_max2(c[3], raw[i].v[0].w, T());
                }
            }
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const float2 f = pair_of(c[j], T());
                col_max[2 * j] = f.x;
                col_max[2 * j + 1] = f.y;
            }
        }
        float top = 0.0f;
#pragma unroll
        for (int i = 0; i < 8; ++i) top = fmaxf(top, row_max[i]);
        return top;
    };
    if (__syncthreads_or(maxima() == quant_inf())) {
#pragma unroll
        for (int i = 0; i < 8; ++i) no_infinities(raw[i]);
        (void)maxima();
    }
    if constexpr (sizeof(T) == 2) {
#pragma unroll
        for (int i = 0; i < 8; ++i) forget_conversions(raw[i]);
    }
    if (MODE == 3) {
        // Rows: 16 lanes hold 8 rows.  Each exchange halves the rows a lane keeps, so that after three of them (and a last
        // plain one) a lane has the maximum of one row, whose scale it makes; the factors go back by shuffles.
        float m4[4], m2[2], m1;
        const bool h8 = (lane & 8u) != 0u, h4 = (lane & 4u) != 0u, h2 = (lane & 2u) != 0u;
#pragma unroll
        for (int i = 0; i < 4; ++i) m4[i] = fmaxf(h8 ? row_max[i + 4] : row_max[i], __shfl_xor_sync(0xffffffffu, h8 ? row_max[i] : row_max[i + 4], 8));
#pragma unroll
        for (int i = 0; i < 2; ++i) m2[i] = fmaxf(h4 ? m4[i + 2] : m4[i], __shfl_xor_sync(0xffffffffu, h4 ? m4[i] : m4[i + 2], 4));
        m1 = fmaxf(h2 ? m2[1] : m2[0], __shfl_xor_sync(0xffffffffu, h2 ? m2[0] : m2[1], 2));
        m1 = fmaxf(m1, __shfl_xor_sync(0xffffffffu, m1, 1));
        const BlockScale s = block_scale(m1, E5M2, p.pow2);
        const int64_t own = my_row + 16 * ((h8 ? 4 : 0) + (h4 ? 2 : 0) + (h2 ? 1 : 0));
        if ((lane & 1u) == 0u && own < row_end) p.scales[own * blocks + blockIdx.x] = s.scale;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float factor = __shfl_sync(0xffffffffu, s.factor, (i & 4) * 2 + (i & 2) * 2 + (i & 1) * 2, 16);
            const int64_t r = my_row + 16 * i;
            float f[8];
            floats_of(raw[i], f);
            const uint2 v = quantize8(f, factor, E5M2);
            if (whole) *reinterpret_cast<uint2 *>(p.q + r * p.ldq + col) = v;
            else if (r < row_end) store8(p.q + r * p.ldq, col, p.cols, v);
            if constexpr (sizeof(T) == 2) forget_conversions(raw[i]);
        }
    }
    if (MODE == 3 && rows_only) return;
    if (MODE == 4) {
        float m = 0.0f;
#pragma unroll
        for (int i = 0; i < 8; ++i) m = fmaxf(m, row_max[i]);
#pragma unroll
        for (int d = 16; d >= 1; d >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, d));
        if (lane == 0) s_max[0][warp] = m;
        __syncthreads();
#pragma unroll
        for (int i = 0; i < 8; ++i) m = fmaxf(m, s_max[0][i]);
        const BlockScale s = block_scale(m, E5M2, p.pow2);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int64_t r = my_row + 16 * i;
            float f[8];
            floats_of(raw[i], f);
            const uint2 v = quantize8(f, s.factor, E5M2);
            uint8_t *dst = p.q + (matrix * p.rows + r) * p.ldq;
            if (whole) *reinterpret_cast<uint2 *>(dst + col) = v;
            else if (r < row_end) store8(dst, col, p.cols, v);
        }
        if (threadIdx.x == 0) p.scales[(matrix * ((p.rows + 127) / 128) + rb) * blocks + blockIdx.x] = s.scale;
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) col_max[j] = fmaxf(col_max[j], __shfl_xor_sync(0xffffffffu, col_max[j], 16));
        if (lane < 16) {
            float4 *dst = reinterpret_cast<float4 *>(&s_max[warp][lane * 8]);
            dst[0] = make_float4(col_max[0], col_max[1], col_max[2], col_max[3]);
            dst[1] = make_float4(col_max[4], col_max[5], col_max[6], col_max[7]);
        }
        __syncthreads();
        if (threadIdx.x < 128) {                                    // thread c makes the scale of column c
            float m = 0.0f;
#pragma unroll
            for (int w = 0; w < 8; ++w) m = fmaxf(m, s_max[w][threadIdx.x]);
            const BlockScale s = block_scale(m, E5M2, p.pow2);
            s_factor[threadIdx.x] = s.factor;
            const int64_t c = blockIdx.x * 128ll + threadIdx.x;
            if (c < p.cols) p.scales_cols[rb * p.cols + c] = s.scale;
        }
        __syncthreads();
        const float4 fa = *reinterpret_cast<const float4 *>(&s_factor[(threadIdx.x & 15u) * 8]), fb = *reinterpret_cast<const float4 *>(&s_factor[(threadIdx.x & 15u) * 8 + 4]);
        const bool padded = p.offsets != nullptr;                   // rows up to the next multiple of 128 are written (zeros)
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int64_t k = (threadIdx.x >> 4) + 16 * i;
            {
                float f[8];
                floats_of(raw[i], f);
                const uint32_t h0 = to_fp8x2(f[0] * fa.x, f[1] * fa.y, E5M2), h1 = to_fp8x2(f[2] * fa.z, f[3] * fa.w, E5M2);
                const uint32_t h2 = to_fp8x2(f[4] * fb.x, f[5] * fb.y, E5M2), h3 = to_fp8x2(f[6] * fb.z, f[7] * fb.w, E5M2);
                const uint2 v = make_uint2(h0 | (h1 << 16), h2 | (h3 << 16));
                uint8_t *dst = p.q_cols + (out0 + k) * p.ldq_cols;
                if (whole) *reinterpret_cast<uint2 *>(dst + col) = v;
                else if (row0 + k < row_end || padded) store8(dst, col, p.cols, v);
            }
        }
    }
}

} // namespace hgemm_dev
