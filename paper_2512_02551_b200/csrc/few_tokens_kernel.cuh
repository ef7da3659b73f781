// A layer of experts for a few tokens: W1 and the activation in one launch, W2 and the weighted sum over a token's choices in another.
//
// Bound by the chosen experts' weights, read once from memory: 0.5 to 2 bytes a weight for a handful of multiply-adds.  The weights go from memory to
// registers (16 bytes a lane, eight or sixteen of them in flight) and from there to mma.sync: a warp's 16 rows of a weight matrix are the operand that
// fills the instruction's rows, up to 16 choices of the expert are its columns.  (Tensor memory and a ring of shared-memory stages would only lengthen the
// way: the tensor pipe is idle nearly all the time, and 4-bit weights have to become 16-bit ones on the way, which tcgen05 cannot do.)
//
// Which k a lane holds is free as long as both operands agree.  A lane takes 16 consecutive bytes of its row, four lanes 64: 32 weights of 16 bits,
// or 128 of 4 bits.  4-bit weights: the four bits s e e m become a bf16 by moving s and eem to their places, which is the value times 2^-126;
// one packed product with the block's scale (times 2^118) makes it the weight times 2^-8, exactly.  Moved this way, a word's codes come out as pairs 4 apart, so
// the other operand is permuted alike.  Instructions bound the 4-bit kernels (24 a warp for 256 weights) as much as memory does.
//
// The products are bf16 with fp32 sums wherever an operand's range asks for it: 4-bit weights with powers of two, and h, which is held as the sum of
// two bf16 (16 bits of mantissa).  fp16 weights and x meet as fp16; against h an fp16 weight is the sum of two bf16 too, and of the four products that of both
// second parts, 2^-16 of the whole, is left out.  fp16 x against powers of two is the sum of two bf16 (exactly).
//
// Work: launch 1 has a tile of 16 rows (SWIGLU: 8 rows of each half, whose products meet in one lane) of one expert per warp, its contraction shared by up to eight
// warps of the CTA; launch 2 has one CTA for 16 outputs of all tokens, whose warps take the chosen experts in turn, so that every sum over a token's
// choices stays in a CTA and has a fixed order.  Every CTA makes the list of the experts' choices for itself; launch 2 does so, and fetches its
// first weights, before launch 1 ends (both are inputs of the call, which launch 1 has waited for).
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_fp8.h>
#include <stdint.h>

#include "hgemm_device.cuh"
#include "product_tiles.cuh"

namespace hgemm_dev {

enum : int { kFewBf16 = 0, kFewF16 = 1, kFewNv = 2, kFewMx = 3 };
constexpr int kFewUpThreads = 256, kFewDownThreads = 512;
constexpr int kFewMaxChoices = 2048;              // 64 tokens of 32
constexpr int kFewEntry = 16;                     // choices of an expert that share a pass over its weights
constexpr uint32_t kFewNone = 0xffffu;

struct FewWeights {
    const uint8_t *values;
    int64_t ld, matrix;        // bytes between rows, between experts
    const uint8_t *scales;
    int64_t scale_matrix;
    const float *factor;
    int32_t rows, depth;       // of one expert
    int32_t atoms;             // scale tiles across
    int32_t align;             // 16-bit weights: what rows' addresses are multiples of: 16, 4 or 2
};

struct FewParams {
    FewWeights w;
    const void *x;             // launch 1
    int64_t ldx;
    int32_t x_vec;             // rows of x start at multiples of 16 bytes
    void *y;                   // launch 2
    int64_t ldy;
    const int32_t *indices;
    const float *weights;
    __nv_bfloat16 *h;          // [2 parts][choices][h_stride]
    int64_t h_stride;
    int32_t inner, experts, top_k, tokens, choices, gated;
    int32_t tiles;             // launch 1: tiles of an expert
    int32_t slices;            // warps that share a contraction
    int32_t slice_chunks;      // chunks of a slice
};

__host__ __device__ constexpr int few_chunk(int w) { return w >= kFewNv ? 128 : 32; }          // k of a chunk: 64 bytes of a row
__host__ __device__ constexpr bool few_is4(int w) { return w >= kFewNv; }

// Shared memory of the lists: words for the experts' counts, the entries (expert | first << 16), 16-bit places and lists of the choices.
__host__ __device__ constexpr int few_max_entries(int experts, int choices) { return (experts < choices ? experts : choices) + choices / kFewEntry; }
__host__ __device__ constexpr int few_list_bytes(int experts, int choices)
{
    return 16 + 4 * experts + 8 * few_max_entries(experts, choices) + 2 * 2 * ((choices + 7) & ~7);
}

struct FewLists {
    int32_t *total;            // entries
    uint32_t *count;           // of an expert, later where its list begins
    uint32_t *entry;           // [2 i]: expert; [2 i + 1]: first | number << 16
    uint16_t *rank, *list;     // place of a choice among its expert's (kFewNone: of no expert); choices by expert
};

__device__ __forceinline__ FewLists few_lists(uint8_t *smem, const FewParams &p)
{
    FewLists l;
    l.total = reinterpret_cast<int32_t *>(smem);
    l.count = reinterpret_cast<uint32_t *>(smem + 16);
    l.entry = l.count + p.experts;
    l.rank = reinterpret_cast<uint16_t *>(l.entry + 2 * few_max_entries(p.experts, p.choices));
    l.list = l.rank + ((p.choices + 7) & ~7);
    return l;
}

// The whole CTA.  An expert's choices keep their order.
__device__ __forceinline__ void few_make_lists(const FewParams &p, const FewLists &l)
{
    for (int32_t e = static_cast<int32_t>(threadIdx.x); e < p.experts; e += static_cast<int32_t>(blockDim.x)) l.count[e] = 0u;
    __syncthreads();
    if (threadIdx.x < 32) {
        const uint32_t lane = threadIdx.x;
        for (int32_t base = 0; base < p.choices; base += 32) {
            const int32_t c = base + static_cast<int32_t>(lane);
            int32_t e = c < p.choices ? p.indices[c] : -1;
            if (e < 0 || e >= p.experts) e = -1;
            const uint32_t peers = __match_any_sync(0xffffffffu, e);
            const uint32_t before = __popc(peers & ((1u << lane) - 1u)), start = e >= 0 ? l.count[e] : 0u;
            __syncwarp();
            if (e >= 0 && before == 0u) l.count[e] = start + __popc(peers);
            __syncwarp();
            if (c < p.choices) l.rank[c] = static_cast<uint16_t>(e >= 0 ? start + before : kFewNone);
        }
        uint32_t places = 0u, entries = 0u;
        for (int32_t base = 0; base < p.experts; base += 32) {
            const int32_t e = base + static_cast<int32_t>(lane);
            const uint32_t n = e < p.experts ? l.count[e] : 0u, m = (n + kFewEntry - 1) / kFewEntry;
            uint32_t sum = n | (m << 16);                      // both sums at once: below 2^12 each
#pragma unroll
            for (int d = 1; d < 32; d <<= 1) {
                const uint32_t v = __shfl_up_sync(0xffffffffu, sum, d);
                if (static_cast<int32_t>(lane) >= d) sum += v;
            }
            const uint32_t first = places + (sum & 0xffffu) - n, at = entries + (sum >> 16) - m;
            if (e < p.experts) l.count[e] = first;
            for (uint32_t i = 0; i < m; ++i) {
                l.entry[2 * (at + i)] = static_cast<uint32_t>(e);
                l.entry[2 * (at + i) + 1] = (first + i * kFewEntry) | (min(n - i * kFewEntry, static_cast<uint32_t>(kFewEntry)) << 16);
            }
            const uint32_t all = __shfl_sync(0xffffffffu, sum, 31);
            places += all & 0xffffu;
            entries += all >> 16;
        }
        if (lane == 0) *l.total = static_cast<int32_t>(entries);
    }
    __syncthreads();
    for (int32_t c = static_cast<int32_t>(threadIdx.x); c < p.choices; c += static_cast<int32_t>(blockDim.x))
        if (l.rank[c] != kFewNone) l.list[l.count[p.indices[c]] + l.rank[c]] = static_cast<uint16_t>(c);
    __syncthreads();
}

// ---- operands -----------------------------------------------------------------------------------------------------

__device__ __forceinline__ void few_mma(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1, __nv_bfloat16)
{
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                 : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void few_mma(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1, __half)
{
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                 : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// 16 bytes of a row of 4-bit weights, or of 16-bit ones (whose addresses are multiples of `align`); zeros beyond the row's `bytes`.
template <int W>
__device__ __forceinline__ uint4 few_load(const uint8_t *row, int32_t at, int32_t bytes, int32_t align)
{
    uint4 v = make_uint4(0u, 0u, 0u, 0u);
    if (row == nullptr || at >= bytes) return v;
    if ((few_is4(W) || align == 16) && at + 16 <= bytes) {
        asm volatile("ld.global.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(row + at));
        return v;
    }
    uint32_t w[4] = {0u, 0u, 0u, 0u};
    if constexpr (few_is4(W)) {
#pragma unroll
        for (int i = 0; i < 16; ++i)
            if (at + i < bytes) w[i / 4] |= static_cast<uint32_t>(row[at + i]) << (8 * (i & 3));
    } else if (align >= 4) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if (at + 4 * i + 4 <= bytes) w[i] = *reinterpret_cast<const uint32_t *>(row + at + 4 * i);
            else if (at + 4 * i < bytes) w[i] = *reinterpret_cast<const uint16_t *>(row + at + 4 * i);
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (at + 2 * i < bytes) w[i / 2] |= static_cast<uint32_t>(*reinterpret_cast<const uint16_t *>(row + at + 2 * i)) << (16 * (i & 1));
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
}

// Two rows' 16 bytes of a chunk, and the scale bytes of a lane's blocks.
struct FewRaw {
    uint4 v[2];
    uint32_t s[2];
};

// What a lane needs to know about its two rows.
struct FewRows {
    const uint8_t *row[2];     // nullptr: no such row
    const uint8_t *scale[2];   // scale tiles of the row's 128, at the row's place
};

template <int W>
__device__ __forceinline__ FewRows few_rows(const FewWeights &w, int32_t expert, int32_t r0, int32_t r1, bool has0, bool has1)
{
    FewRows f;
    const int32_t r[2] = {r0, r1};
    const bool has[2] = {has0, has1};
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        f.row[i] = has[i] ? w.values + expert * w.matrix + r[i] * w.ld : nullptr;
        f.scale[i] = nullptr;
        if constexpr (few_is4(W)) {
            if (has[i]) f.scale[i] = w.scales + expert * w.scale_matrix + static_cast<int64_t>(r[i] >> 7) * w.atoms * 512 + (r[i] & 31) * 16 + ((r[i] >> 5) & 3) * 4;
        }
    }
    return f;
}

template <int W>
__device__ __forceinline__ void few_fetch(FewRaw &raw, const FewWeights &w, const FewRows &f, int32_t chunk, int32_t end, uint32_t q)
{
    const int32_t bytes = few_is4(W) ? (w.depth + 1) / 2 : w.depth * 2;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        raw.v[i] = few_load<W>(chunk < end ? f.row[i] : nullptr, chunk * 64 + static_cast<int32_t>(q) * 16, bytes, w.align);
        raw.s[i] = 0u;
        if constexpr (W == kFewNv) {
            const int32_t atom = chunk * 2 + static_cast<int32_t>(q >> 1);
            if (f.row[i] != nullptr && chunk < end && atom < w.atoms) raw.s[i] = *reinterpret_cast<const uint16_t *>(f.scale[i] + static_cast<int64_t>(atom) * 512 + (q & 1u) * 2u);
        } else if constexpr (W == kFewMx) {
            if (f.row[i] != nullptr && chunk < end) raw.s[i] = f.scale[i][static_cast<int64_t>(chunk) * 512 + q];
        }
    }
}

__device__ __forceinline__ uint32_t few_mul2(uint32_t a, uint32_t b, __nv_bfloat16)
{
    uint32_t d;
    asm("mul.rn.bf16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
    return d;
}
__device__ __forceinline__ uint32_t few_mul2(uint32_t a, uint32_t b, __half)
{
    uint32_t d;
    asm("mul.rn.f16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
    return d;
}

// Eight codes as four pairs (0, 4), (1, 5), (2, 6), (3, 7): bf16 times 2^-126, or fp16 times 2^-14.
template <class T>
__device__ __forceinline__ void few_spread(uint32_t w, uint32_t (&d)[4])
{
    constexpr bool kHalf = sizeof(T) == 2 && std::is_same<T, __half>::value;
    constexpr int kUp = kHalf ? 9 : 6;
    constexpr uint32_t kMag = kHalf ? 0x0e000e00u : 0x01c001c0u, kSign = 0x80008000u;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int m = kUp - 4 * i, s = 12 - 4 * i;
        const uint32_t mag = m >= 0 ? w << m : w >> -m, sign = s >= 0 ? w << s : w >> -s;
        d[i] = (mag & kMag) | (sign & kSign);
    }
}

// The scales of a lane's run of 32 weights as pairs to multiply by (one for 16 of them each), and what the sums are then too small by.
template <int W, class T>
__device__ __forceinline__ void few_scales(uint32_t s, uint32_t (&d)[2])
{
    constexpr bool kHalf = std::is_same<T, __half>::value;
    if constexpr (W == kFewNv) {
        const __half2 h = __half2(__nv_cvt_fp8x2_to_halfraw2(static_cast<__nv_fp8x2_storage_t>(s), __NV_E4M3));
        if constexpr (kHalf) {
            const __half2 v = __hmul2(h, __floats2half2_rn(128.0f, 128.0f));             // at most 57344
            const uint32_t b = *reinterpret_cast<const uint32_t *>(&v);
            d[0] = __byte_perm(b, 0u, 0x1010);
            d[1] = __byte_perm(b, 0u, 0x3232);
        } else {
            const float2 f = __half22float2(h);
            d[0] = __byte_perm(__float_as_uint(f.x * 0x1p118f), 0u, 0x3232);
            d[1] = __byte_perm(__float_as_uint(f.y * 0x1p118f), 0u, 0x3232);
        }
    } else {
        // 2^(s - 127), a bf16 (the smallest is subnormal; 255: NaN)
        const uint32_t b = s == 0u ? 0x40u : s == 255u ? 0x7fffu : s << 7;
        d[0] = d[1] = b | (b << 16);
    }
}
template <int W, class T>
__device__ __forceinline__ float few_missing(const FewWeights &w, int32_t expert)
{
    if constexpr (W == kFewNv) return w.factor[expert] * (std::is_same<T, __half>::value ? 128.0f : 256.0f);
    else if constexpr (W == kFewMx) return 64.0f;
    else return 1.0f;
}

// Word i of a run of 4-bit weights as the instruction's operand.
template <int W, class T>
__device__ __forceinline__ void few_weights4(uint32_t word, const uint32_t (&s)[2], int i, uint32_t (&d)[4])
{
    few_spread<T>(word, d);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        if constexpr (W == kFewMx) d[j] = few_mul2(d[j], 0x7b807b80u, T());              // 2^120 first: 2^-126 times 2^(120 + ...) may not have a scale of its own
        d[j] = few_mul2(d[j], s[i / 2], T());
    }
}

// The sum of two bf16 that a number is, or is nearest to; pairs of numbers.
__device__ __forceinline__ void few_two_parts(float a, float b, uint32_t &hi, uint32_t &lo)
{
    const __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
    hi = *reinterpret_cast<const uint32_t *>(&h);
    const float ah = __uint_as_float(hi << 16), bh = __uint_as_float(hi & 0xffff0000u);
    // infinities and NaN are their first part alone
    lo = pack_pair(fabsf(ah) < __int_as_float(0x7f800000) ? a - ah : 0.0f, fabsf(bh) < __int_as_float(0x7f800000) ? b - bh : 0.0f, __nv_bfloat16());
}
__device__ __forceinline__ void few_two_parts(uint32_t f16x2, uint32_t &hi, uint32_t &lo)
{
    const float2 f = __half22float2(*reinterpret_cast<const __half2 *>(&f16x2));
    few_two_parts(f.x, f.y, hi, lo);
}

// The order in which a run of 8 consecutive k meets 8 codes.
__device__ __forceinline__ uint4 few_like_codes(uint4 v)
{
    return make_uint4(__byte_perm(v.x, v.z, 0x5410), __byte_perm(v.x, v.z, 0x7632), __byte_perm(v.y, v.w, 0x5410), __byte_perm(v.y, v.w, 0x7632));
}

// Where element k of h lies in its choice's row.
template <int W>
__device__ __forceinline__ int64_t few_h_place(int32_t k)
{
    if constexpr (few_is4(W)) {
        const int32_t run = k >> 3, e = k & 7;                   // run (c * 4 + q) * 4 + i lies at (c * 4 + i) * 4 + q
        return ((run & ~15) + (run & 3) * 4 + ((run >> 2) & 3)) * 8 + (e & 3) * 2 + (e >> 2);
    } else {
        return k;
    }
}

// ---- launch 1: h = act(W1 x) ------------------------------------------------------------------------------------------

// 8 consecutive elements of x, zeros beyond its end.
__device__ __forceinline__ uint4 few_load_x(const uint16_t *row, int32_t k, int32_t depth, int32_t vec)
{
    uint4 v = make_uint4(0u, 0u, 0u, 0u);
    if (row == nullptr || k >= depth) return v;
    if (vec && k + 8 <= depth) return *reinterpret_cast<const uint4 *>(row + k);
    uint32_t w[4] = {0u, 0u, 0u, 0u};
#pragma unroll
    for (int i = 0; i < 8; ++i)
        if (k + i < depth) w[i / 2] |= static_cast<uint32_t>(row[k + i]) << (16 * (i & 1));
    return make_uint4(w[0], w[1], w[2], w[3]);
}

// One chunk of a tile's contraction for NT runs of 8 choices.  T: the products' type; X16: x is fp16.
template <int W, class T, bool X16, int NT>
__device__ __forceinline__ void few_up_chunk(float (&acc)[2][4], const FewRaw &raw, const uint16_t *const (&x)[2], int32_t chunk, int32_t depth, int32_t vec, uint32_t q)
{
    constexpr bool kTwo = X16 && !std::is_same<T, __half>::value;      // x in two parts
    auto products = [&](int n, const uint32_t (&a)[4], const uint32_t (&b)[4], const uint4 &v) {
        few_mma(acc[n], a[0], b[0], a[1], b[1], v.x, v.y, T());
        few_mma(acc[n], a[2], b[2], a[3], b[3], v.z, v.w, T());
    };
    auto with_x = [&](const uint32_t (&a)[4], const uint32_t (&b)[4], int32_t k) {
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            uint4 v = few_load_x(x[n], k, depth, vec);
            if constexpr (few_is4(W)) v = few_like_codes(v);
            if constexpr (kTwo) {
                uint4 hi, lo;
                few_two_parts(v.x, hi.x, lo.x);
                few_two_parts(v.y, hi.y, lo.y);
                few_two_parts(v.z, hi.z, lo.z);
                few_two_parts(v.w, hi.w, lo.w);
                products(n, a, b, hi);
                products(n, a, b, lo);
            } else {
                products(n, a, b, v);
            }
        }
    };
    if constexpr (few_is4(W)) {
        uint32_t s0[2], s1[2];
        few_scales<W, T>(raw.s[0], s0);
        few_scales<W, T>(raw.s[1], s1);
        const uint32_t w0[4] = {raw.v[0].x, raw.v[0].y, raw.v[0].z, raw.v[0].w}, w1[4] = {raw.v[1].x, raw.v[1].y, raw.v[1].z, raw.v[1].w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            uint32_t a[4], b[4];
            few_weights4<W, T>(w0[i], s0, i, a);
            few_weights4<W, T>(w1[i], s1, i, b);
            with_x(a, b, chunk * 128 + static_cast<int32_t>(q) * 32 + i * 8);
        }
    } else {
        const uint32_t a[4] = {raw.v[0].x, raw.v[0].y, raw.v[0].z, raw.v[0].w}, b[4] = {raw.v[1].x, raw.v[1].y, raw.v[1].z, raw.v[1].w};
        with_x(a, b, chunk * 32 + static_cast<int32_t>(q) * 8);
    }
}

__device__ __forceinline__ float few_silu(float u) { return u / (1.0f + __expf(-u)); }

template <int W, bool X16>
__global__ void __launch_bounds__(kFewUpThreads, 2)
few_up_kernel(const FewParams p)
{
    using T = std::conditional_t<X16 && W != kFewMx, __half, __nv_bfloat16>;
    constexpr int kWarps = kFewUpThreads / 32, kAhead = 4;        // chunks fetched together
    extern __shared__ __align__(16) uint8_t smem[];
    __shared__ float s_part[kWarps][32][8];
    const FewLists l = few_lists(smem, p);
    grid_dependency_wait();
    grid_launch_dependents();                                     // launch 2 may read the call's inputs from here on
    few_make_lists(p, l);
    const uint32_t warp = threadIdx.x >> 5, lane = threadIdx.x & 31u, q = lane & 3u, m = lane >> 2;
    const int32_t slice = static_cast<int32_t>(warp) % p.slices, per_cta = kWarps / p.slices;
    const int64_t items = static_cast<int64_t>(*l.total) * p.tiles;
    const int32_t begin = slice * p.slice_chunks, depth_chunks = (p.w.depth + few_chunk(W) - 1) / few_chunk(W), end = min(begin + p.slice_chunks, depth_chunks);
    const int32_t groups = max(0, (end - begin + kAhead - 1) / kAhead);

    struct Item {
        int32_t expert, first, count, row0, row1;
        bool has0, has1;
    };
    auto item_of = [&](int64_t i) {
        Item t;
        const int32_t e = static_cast<int32_t>(i / p.tiles), tile = static_cast<int32_t>(i - static_cast<int64_t>(e) * p.tiles);
        t.expert = static_cast<int32_t>(l.entry[2 * e]);
        t.first = static_cast<int32_t>(l.entry[2 * e + 1] & 0xffffu);
        t.count = static_cast<int32_t>(l.entry[2 * e + 1] >> 16);
        t.row0 = tile * (p.gated ? 8 : 16) + static_cast<int32_t>(m);
        t.row1 = p.gated ? t.row0 + p.inner : t.row0 + 8;
        t.has0 = t.row0 < p.inner;
        t.has1 = p.gated ? t.has0 : t.row1 < p.inner;
        return t;
    };
    FewRaw next[kAhead];
    auto fetch = [&](const FewRows &f, int32_t chunk) {
#pragma unroll
        for (int u = 0; u < kAhead; ++u) few_fetch<W>(next[u], p.w, f, chunk + u, end, q);
    };
    const int64_t stride = static_cast<int64_t>(gridDim.x) * per_cta;
    int64_t i = static_cast<int64_t>(blockIdx.x) * per_cta + warp / p.slices;
    if (i < items && groups > 0) {
        const Item t = item_of(i);
        fetch(few_rows<W>(p.w, t.expert, t.row0, t.row1, t.has0, t.has1), begin);
    }
    // CTA-uniform rounds: a round's slices meet in shared memory
    for (int64_t round = static_cast<int64_t>(blockIdx.x) * per_cta; round < items; round += stride, i += stride) {
        const bool mine = i < items;
        Item t{};
        float acc[2][4] = {};
        if (mine) {
            t = item_of(i);
            const FewRows f = few_rows<W>(p.w, t.expert, t.row0, t.row1, t.has0, t.has1);
            const uint16_t *x[2];
#pragma unroll
            for (int n = 0; n < 2; ++n) {
                const int32_t at = n * 8 + static_cast<int32_t>(m);
                x[n] = at < t.count ? static_cast<const uint16_t *>(p.x) + static_cast<int64_t>(l.list[t.first + at] / p.top_k) * p.ldx : nullptr;
            }
            for (int32_t g = 0; g < groups; ++g) {
                FewRaw now[kAhead];
#pragma unroll
                for (int u = 0; u < kAhead; ++u) now[u] = next[u];
                if (g + 1 < groups) {
                    fetch(f, begin + (g + 1) * kAhead);
                } else if (i + stride < items) {
                    const Item o = item_of(i + stride);
                    fetch(few_rows<W>(p.w, o.expert, o.row0, o.row1, o.has0, o.has1), begin);
                }
#pragma unroll
                for (int u = 0; u < kAhead; ++u) {
                    const int32_t chunk = begin + g * kAhead + u;
                    if (chunk < end) {
                        if (t.count <= 8) few_up_chunk<W, T, X16, 1>(acc, now[u], x, chunk, p.w.depth, p.x_vec, q);
                        else few_up_chunk<W, T, X16, 2>(acc, now[u], x, chunk, p.w.depth, p.x_vec, q);
                    }
                }
            }
        }
        if (p.slices > 1) {
            if (slice > 0) {
                *reinterpret_cast<float4 *>(&s_part[warp][lane][0]) = make_float4(acc[0][0], acc[0][1], acc[0][2], acc[0][3]);
                *reinterpret_cast<float4 *>(&s_part[warp][lane][4]) = make_float4(acc[1][0], acc[1][1], acc[1][2], acc[1][3]);
            }
            __syncthreads();
            if (slice == 0) {
                for (int32_t s = 1; s < p.slices; ++s) {
#pragma unroll
                    for (int j = 0; j < 8; ++j) acc[j / 4][j & 3] += s_part[warp + s][lane][j];
                }
            }
            __syncthreads();
        }
        if (mine && slice == 0) {
            const float missing = few_missing<W, T>(p.w, t.expert);
#pragma unroll
            for (int n = 0; n < 2; ++n) {
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    const int32_t at = n * 8 + static_cast<int32_t>(q) * 2 + j;
                    if (at >= t.count) continue;
                    const int64_t c = l.list[t.first + at];
                    const float u0 = acc[n][j] * missing, u1 = acc[n][2 + j] * missing;
                    // runs of 8 are written whole: zeros beyond inner
                    const int32_t room = (p.inner + 7) & ~7;
                    auto put = [&](int32_t k, float v) {
                        if (k >= room) return;
                        uint32_t hi, lo;
                        few_two_parts(v, 0.0f, hi, lo);
                        __nv_bfloat16 *dst = p.h + c * p.h_stride + few_h_place<W>(k);
                        *reinterpret_cast<uint16_t *>(dst) = static_cast<uint16_t>(hi);
                        *reinterpret_cast<uint16_t *>(dst + p.choices * p.h_stride) = static_cast<uint16_t>(lo);
                    };
                    if (p.gated) {
                        put(t.row0, t.has0 ? few_silu(u0) * u1 : 0.0f);
                    } else {
                        put(t.row0, t.has0 ? few_silu(u0) : 0.0f);
                        put(t.row1, t.has1 ? few_silu(u1) : 0.0f);
                    }
                }
            }
        }
    }
}

// ---- launch 2: y = sum of weight * (W2 h) ------------------------------------------------------------------------------

template <int W, int NT>
__device__ __forceinline__ void few_down_chunk(float (&acc)[2][4], const FewRaw &raw, const uint8_t *const (&h)[2], int64_t part, int32_t chunk, int32_t runs, uint32_t q)
{
    using B = __nv_bfloat16;
    auto with_h = [&](const uint32_t (&a)[4], const uint32_t (&b)[4], const uint32_t (&a2)[4], const uint32_t (&b2)[4], int32_t run, int32_t at) {
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            uint4 hi = make_uint4(0u, 0u, 0u, 0u), lo = hi;
            if (h[n] != nullptr && run < runs) {
                hi = *reinterpret_cast<const uint4 *>(h[n] + at * 16);
                lo = *reinterpret_cast<const uint4 *>(h[n] + part + at * 16);
            }
            few_mma(acc[n], a[0], b[0], a[1], b[1], hi.x, hi.y, B());
            few_mma(acc[n], a[2], b[2], a[3], b[3], hi.z, hi.w, B());
            few_mma(acc[n], a[0], b[0], a[1], b[1], lo.x, lo.y, B());
            few_mma(acc[n], a[2], b[2], a[3], b[3], lo.z, lo.w, B());
            if constexpr (W == kFewF16) {
                few_mma(acc[n], a2[0], b2[0], a2[1], b2[1], hi.x, hi.y, B());
                few_mma(acc[n], a2[2], b2[2], a2[3], b2[3], hi.z, hi.w, B());
            }
        }
    };
    if constexpr (few_is4(W)) {
        uint32_t s0[2], s1[2];
        few_scales<W, B>(raw.s[0], s0);
        few_scales<W, B>(raw.s[1], s1);
        const uint32_t w0[4] = {raw.v[0].x, raw.v[0].y, raw.v[0].z, raw.v[0].w}, w1[4] = {raw.v[1].x, raw.v[1].y, raw.v[1].z, raw.v[1].w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            uint32_t a[4], b[4];
            few_weights4<W, B>(w0[i], s0, i, a);
            few_weights4<W, B>(w1[i], s1, i, b);
            with_h(a, b, a, b, (chunk * 4 + static_cast<int32_t>(q)) * 4 + i, (chunk * 4 + i) * 4 + static_cast<int32_t>(q));
        }
    } else {
        uint32_t a[4] = {raw.v[0].x, raw.v[0].y, raw.v[0].z, raw.v[0].w}, b[4] = {raw.v[1].x, raw.v[1].y, raw.v[1].z, raw.v[1].w}, a2[4], b2[4];
        if constexpr (W == kFewF16) {
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const uint32_t wa = j == 0 ? raw.v[0].x : j == 1 ? raw.v[0].y : j == 2 ? raw.v[0].z : raw.v[0].w;
                const uint32_t wb = j == 0 ? raw.v[1].x : j == 1 ? raw.v[1].y : j == 2 ? raw.v[1].z : raw.v[1].w;
                few_two_parts(wa, a[j], a2[j]);
                few_two_parts(wb, b[j], b2[j]);
            }
        }
        const int32_t run = chunk * 4 + static_cast<int32_t>(q);
        with_h(a, b, a2, b2, run, run);
    }
}

// grid: 16 rows of W2 (outputs) a CTA.  Dynamic shared memory: the lists, then slices x choices x 16 sums.
template <int W, class Y>
__global__ void __launch_bounds__(kFewDownThreads, 1)
few_down_kernel(const FewParams p)
{
    constexpr int kWarps = kFewDownThreads / 32, kAhead = 4;
    extern __shared__ __align__(16) uint8_t smem[];
    const FewLists l = few_lists(smem, p);
    float *part = reinterpret_cast<float *>(smem + ((few_list_bytes(p.experts, p.choices) + 15) & ~15));
    grid_launch_dependents();
    few_make_lists(p, l);                                         // an input of the call: launch 1 has waited for it
    const uint32_t warp = threadIdx.x >> 5, lane = threadIdx.x & 31u, q = lane & 3u, m = lane >> 2;
    const int32_t items = *l.total * p.slices, row0 = static_cast<int32_t>(blockIdx.x) * 16 + static_cast<int32_t>(m);
    const int32_t depth_chunks = (p.w.depth + few_chunk(W) - 1) / few_chunk(W), runs = (p.w.depth + 7) / 8;
    const bool has0 = row0 < p.w.rows, has1 = row0 + 8 < p.w.rows;
    FewRaw next[kAhead];
    struct Span {
        int32_t begin, end;
    };
    auto span_of = [&](int32_t i) {
        const int32_t b = (i % p.slices) * p.slice_chunks;
        return Span{b, min(b + p.slice_chunks, depth_chunks)};
    };
    auto fetch = [&](int32_t i, int32_t g) {
        const Span s = span_of(i);
        const FewRows f = few_rows<W>(p.w, static_cast<int32_t>(l.entry[2 * (i / p.slices)]), row0, row0 + 8, has0, has1);
#pragma unroll
        for (int u = 0; u < kAhead; ++u) few_fetch<W>(next[u], p.w, f, s.begin + g * kAhead + u, s.end, q);
    };
    int32_t i = static_cast<int32_t>(warp);
    if (i < items) fetch(i, 0);
    grid_dependency_wait();                                       // h
    const int32_t groups = (p.slice_chunks + kAhead - 1) / kAhead;
    for (; i < items; i += kWarps) {
        const uint32_t expert = l.entry[2 * (i / p.slices)], where = l.entry[2 * (i / p.slices) + 1];
        const int32_t first = static_cast<int32_t>(where & 0xffffu), count = static_cast<int32_t>(where >> 16);
        const Span s = span_of(i);
        const uint8_t *h[2];
#pragma unroll
        for (int n = 0; n < 2; ++n) {
            const int32_t at = n * 8 + static_cast<int32_t>(m);
            h[n] = at < count ? reinterpret_cast<const uint8_t *>(p.h + l.list[first + at] * p.h_stride) : nullptr;
        }
        const int64_t second = p.choices * p.h_stride * 2;
        float acc[2][4] = {};
        for (int32_t g = 0; g < groups; ++g) {
            FewRaw now[kAhead];
#pragma unroll
            for (int u = 0; u < kAhead; ++u) now[u] = next[u];
            if (g + 1 < groups) fetch(i, g + 1);
            else if (i + kWarps < items) fetch(i + kWarps, 0);
#pragma unroll
            for (int u = 0; u < kAhead; ++u) {
                const int32_t chunk = s.begin + g * kAhead + u;
                if (chunk < s.end) {
                    if (count <= 8) few_down_chunk<W, 1>(acc, now[u], h, second, chunk, runs, q);
                    else few_down_chunk<W, 2>(acc, now[u], h, second, chunk, runs, q);
                }
            }
        }
        const float missing = few_missing<W, __nv_bfloat16>(p.w, static_cast<int32_t>(expert));
#pragma unroll
        for (int n = 0; n < 2; ++n) {
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const int32_t at = n * 8 + static_cast<int32_t>(q) * 2 + j;
                if (at >= count) continue;
                float *dst = part + (static_cast<int64_t>(i % p.slices) * p.choices + l.list[first + at]) * 16;
                dst[m] = acc[n][j] * missing;
                dst[m + 8] = acc[n][2 + j] * missing;
            }
        }
    }
    __syncthreads();
    for (int32_t o = static_cast<int32_t>(threadIdx.x); o < p.tokens * 16; o += kFewDownThreads) {
        const int32_t t = o >> 4, r = o & 15, row = static_cast<int32_t>(blockIdx.x) * 16 + r;
        if (row >= p.w.rows) continue;
        float sum = 0.0f;
        for (int32_t j = 0; j < p.top_k; ++j) {
            const int32_t c = t * p.top_k + j;
            if (l.rank[c] == kFewNone) continue;
            float v = 0.0f;
            for (int32_t s = 0; s < p.slices; ++s) v += part[(static_cast<int64_t>(s) * p.choices + c) * 16 + r];
            sum = fmaf(p.weights[c], v, sum);
        }
        static_cast<Y *>(p.y)[t * p.ldy + row] = narrow_to<Y>(sum);
    }
}

} // namespace hgemm_dev
