// A layer of experts with 16-bit weights for a few tokens: W1 and the activation in one launch, W2 and the weighted sum over a token's choices in another.
// (4-bit weights: few_digits_kernel.cuh.)
//
// Bound by the chosen experts' weights, read once from memory for a handful of multiply-adds (5 tokens, 4 of 32 experts, 2048 -> 1000 -> 2048, bf16: 34.4 us in a graph, 3.7 TB/s, 35-38 a call; a
// launch's start, its list of choices and its last tiles take some 6 us each).  They go from memory to registers (16 bytes a lane, four
// chunks of two rows in flight at any time) and from there to mma.sync: a warp's 16 rows of a weight matrix are the operand that fills the instruction's
// rows, up to 8 choices of the expert are its columns.  A lane takes 16 consecutive bytes of its row, four lanes 64 (a chunk): which k a lane holds is free as
// long as both operands agree.  (Tensor memory and a ring of shared-memory stages would lengthen the way of rows that start anywhere: tensor copies
// need rows at multiples of 16 bytes.)
//
// h is the sum of two bf16 (16 bits of mantissa, in bf16's range: fp16 would not hold every h, one bf16 would round it as coarsely as y).  What that loses, 2^-16 of each h, is small beside
// y's own rounding (2^-8 or 2^-11), and a third part would be half as much again to write, read and multiply.  Against h an fp16 weight is the sum of two bf16 too, and of the
// four products that of both second parts, 2^-16 of the whole, is left out for the same reason.
//
// Work.  Launch 1: a warp has a tile of 16 rows (SWIGLU: 8 rows of each half, whose products meet in one lane), a CTA eight tiles of one expert, whose
// tokens it lays out in shared memory as the instruction wants them.  As many rounds as give every CTA the same; the groups of tiles that are left over are
// shared by up to eight CTAs each, whose warps split the contraction.  Launch 2: one CTA, or a cluster, for 16 outputs of all tokens; its warps take the chosen
// experts in turn (those left over by several warps each), so that every sum over a token's choices stays in a cluster and has a fixed order.  Every CTA makes
// the list of the experts' choices for itself; launch 2 does so, and fetches its first weights, before launch 1 ends (both are inputs of the call,
// which launch 1 has waited for).  A column of the instruction that has no choice computes with whatever is there; its sums are not used.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <stdint.h>

#include <type_traits>

#include "hgemm_device.cuh"
#include "product_tiles.cuh"

namespace hgemm_dev {

constexpr int kFewUpThreads = 256, kFewDownThreads = 512;
constexpr int kFewMaxChoices = 2048;              // 64 tokens of 32
constexpr int kFewEntry = 8;                      // choices of an expert that share a pass over its weights
constexpr int kFewAhead = 4;                      // chunks in flight
constexpr uint32_t kFewNone = 0xffffu;

struct FewWeights {
    const uint8_t *values;
    int64_t ld, matrix;        // bytes between rows, between experts
    int32_t rows, depth;       // of one expert
    int32_t align;             // what rows' addresses are multiples of: 16, 4 or 2
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
    __nv_bfloat16 *h;          // two parts of choices x h_stride (whole chunks)
    int32_t h_stride;
    int32_t inner, experts, top_k, tokens, choices, gated;
    int32_t groups;            // launch 1: groups of eight tiles of an expert
    FastDiv fd_groups;
    int32_t piece;             // launch 1: bytes of shared memory for x
    int32_t most_slices;       // warps that may share a contraction
    int32_t ranks;             // launch 2: CTAs (a cluster) that share 16 outputs
};

constexpr int kFewChunk = 32;                     // k of a chunk: 64 bytes of a row

// ---- lists --------------------------------------------------------------------------------------------------------

// Shared memory of the lists: words for the experts' counts and the entries, 16-bit experts, places and lists of the choices.
__host__ __device__ constexpr int few_max_entries(int experts, int choices) { return (experts < choices ? experts : choices) + choices / kFewEntry; }
__host__ __device__ constexpr int few_list_bytes(int experts, int choices)
{
    return ((16 + 4 * experts + 8 * few_max_entries(experts, choices) + 15) & ~15) + ((3 * 2 * ((choices + 7) & ~7) + 15) & ~15);
}

struct FewLists {
    int32_t *total;            // entries
    uint32_t *count;           // of an expert, later where its list begins
    uint32_t *entry;           // [2 i]: expert; [2 i + 1]: first | number << 16
    uint16_t *expert;          // of a choice (kFewNone: none)
    uint16_t *rank, *list;     // place of a choice among its expert's; choices by expert
};

__device__ __forceinline__ FewLists few_lists(uint8_t *smem, const FewParams &p)
{
    FewLists l;
    l.total = reinterpret_cast<int32_t *>(smem);
    l.count = reinterpret_cast<uint32_t *>(smem + 16);
    l.entry = l.count + p.experts;
    l.expert = reinterpret_cast<uint16_t *>(smem + ((16 + 4 * p.experts + 8 * few_max_entries(p.experts, p.choices) + 15) & ~15));
    l.rank = l.expert + ((p.choices + 7) & ~7);
    l.list = l.rank + ((p.choices + 7) & ~7);
    return l;
}

// The whole CTA.  An expert's choices keep their order.
__device__ __forceinline__ void few_make_lists(const FewParams &p, const FewLists &l)
{
    const int32_t threads = static_cast<int32_t>(blockDim.x), me = static_cast<int32_t>(threadIdx.x);
    for (int32_t e = me; e < p.experts; e += threads) l.count[e] = 0u;
    for (int32_t c = me; c < ((p.choices + 7) & ~7); c += threads) {
        const int32_t e = c < p.choices ? ld_older(p.indices + c) : -1;
        l.expert[c] = static_cast<uint16_t>(e >= 0 && e < p.experts ? e : kFewNone);
    }
    __syncthreads();
    if (p.choices <= 128) {
        // a choice's place is the number of choices of its expert ahead of it: all of them compared at once
        if (me < p.choices) {
            const uint32_t e = l.expert[me], ee = e | (e << 16);
            uint32_t before = 0u;
            for (int32_t c = 0; c < me; c += 8) {
                const uint4 v = *reinterpret_cast<const uint4 *>(l.expert + c);
                const uint32_t w[4] = {v.x ^ ee, v.y ^ ee, v.z ^ ee, v.w ^ ee};
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    before += (w[i] & 0xffffu) == 0u && c + 2 * i < me;
                    before += (w[i] >> 16) == 0u && c + 2 * i + 1 < me;
                }
            }
            l.rank[me] = static_cast<uint16_t>(before);
            if (e != kFewNone) atomicAdd(&l.count[e], 1u);
        }
    } else if (me < 32) {
        for (int32_t base = 0; base < p.choices; base += 32) {
            const int32_t c = base + me;
            const uint32_t e = c < p.choices ? l.expert[c] : kFewNone;
            const uint32_t peers = __match_any_sync(0xffffffffu, e);
            const uint32_t before = __popc(peers & ((1u << me) - 1u)), start = e != kFewNone ? l.count[e] : 0u;
            __syncwarp();
            if (e != kFewNone && before == 0u) l.count[e] = start + __popc(peers);
            __syncwarp();
            if (c < p.choices) l.rank[c] = static_cast<uint16_t>(start + before);
        }
    }
    __syncthreads();
    if (me < 32) {
        uint32_t places = 0u, entries = 0u;
        for (int32_t base = 0; base < p.experts; base += 32) {
            const int32_t e = base + me;
            const uint32_t n = e < p.experts ? l.count[e] : 0u, m = (n + kFewEntry - 1) / kFewEntry;
            uint32_t sum = n | (m << 16);                      // both sums at once: below 2^12 each
#pragma unroll
            for (int d = 1; d < 32; d <<= 1) {
                const uint32_t v = __shfl_up_sync(0xffffffffu, sum, d);
                if (me >= d) sum += v;
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
        if (me == 0) *l.total = static_cast<int32_t>(entries);
    }
    __syncthreads();
    for (int32_t c = me; c < p.choices; c += threads)
        if (l.expert[c] != kFewNone) l.list[l.count[l.expert[c]] + l.rank[c]] = static_cast<uint16_t>(c);
    __syncthreads();
}

// ---- weights ------------------------------------------------------------------------------------------------------

// Two rows' 16 bytes of a chunk (N = 2), and the other operand's two parts (N = 4: launch 2, where they come from memory too).
template <int N>
struct FewRaw {
    uint4 v[N];
};

// Part of a contraction: chunks of a lane's two rows.  Rows that are not there (a matrix's last tile) stand for the expert's first: they are loaded like the
// others, and their sums are not used.
template <int N>
struct FewSpan {
    const uint8_t *row[N];     // at the lane's bytes of the first chunk
    int32_t first, n;          // chunks; those of them that rows have whole
    bool tail;                 // a last chunk follows, of which rows have a part
};

template <int N>
__device__ __forceinline__ FewSpan<N> few_span(const FewWeights &w, int32_t expert, int32_t r0, int32_t r1, int32_t first, int32_t n, uint32_t q)
{
    FewSpan<N> f;
    f.row[0] = w.values + expert * w.matrix + r0 * w.ld + first * 64 + q * 16;
    f.row[1] = w.values + expert * w.matrix + r1 * w.ld + first * 64 + q * 16;
    f.first = first;
    f.n = max(0, min(first + n, w.depth / kFewChunk) - first);
    f.tail = f.n < n;
    return f;
}

// 16 bytes at a multiple of ALIGN.
template <int ALIGN>
__device__ __forceinline__ uint4 few_load16(const uint8_t *p)
{
    uint4 v;
    if constexpr (ALIGN == 16) {
        asm volatile("ld.global.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p));
    } else if constexpr (ALIGN == 4) {
        asm volatile("ld.global.u32 %0, [%4];\n\tld.global.u32 %1, [%4 + 4];\n\tld.global.u32 %2, [%4 + 8];\n\tld.global.u32 %3, [%4 + 12];"
                     : "=&r"(v.x), "=&r"(v.y), "=&r"(v.z), "=&r"(v.w) : "l"(p));
    } else {
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i)
            asm volatile("{\n\t.reg .b16 a, b;\n\tld.global.u16 a, [%1];\n\tld.global.u16 b, [%1 + 2];\n\tmov.b32 %0, {a, b};\n\t}" : "=r"(w[i]) : "l"(p + 4 * i));
        v = make_uint4(w[0], w[1], w[2], w[3]);
    }
    return v;
}

// The same ahead of the kernel's own wait (see ld_older).
template <int ALIGN>
__device__ __forceinline__ uint4 few_load16_older(const uint8_t *p)
{
    uint4 v;
    if constexpr (ALIGN == 16) {
        asm volatile("ld.relaxed.gpu.global.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p) : "memory");
    } else if constexpr (ALIGN == 4) {
        const uint32_t *w = reinterpret_cast<const uint32_t *>(p);
        v = make_uint4(ld_older(w), ld_older(w + 1), ld_older(w + 2), ld_older(w + 3));
    } else {
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i)
            asm volatile("{\n\t.reg .b16 a, b;\n\tld.relaxed.gpu.global.u16 a, [%1];\n\tld.relaxed.gpu.global.u16 b, [%1 + 2];\n\tmov.b32 %0, {a, b};\n\t}" : "=r"(w[i]) : "l"(p + 4 * i) : "memory");
        v = make_uint4(w[0], w[1], w[2], w[3]);
    }
    return v;
}

// Chunk i behind a span's pointers (loads without a condition around them: they stay in flight).
template <int ALIGN, int N>
__device__ __forceinline__ void few_fetch(FewRaw<N> &raw, const uint8_t *const (&row)[N], int i)
{
#pragma unroll
    for (int j = 0; j < N; ++j) raw.v[j] = j < 2 ? few_load16<ALIGN>(row[j] + i * 64) : few_load16<16>(row[j] + i * 64);
}

// The chunk behind the whole ones; zeros beyond the rows' ends.
template <int N>
__device__ __forceinline__ void few_fetch_tail(FewRaw<N> &raw, const FewWeights &w, const FewSpan<N> &f, uint32_t q)
{
    const int32_t room = w.depth * 2 - (f.first + f.n) * 64 - static_cast<int32_t>(q) * 16;
#pragma unroll
    for (int j = 0; j < 2; ++j) {
        const uint8_t *p = f.row[j] + static_cast<int64_t>(f.n) * 64;
        uint32_t v[4] = {0u, 0u, 0u, 0u};
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (2 * i < room) v[i / 2] |= static_cast<uint32_t>(*reinterpret_cast<const uint16_t *>(p + 2 * i)) << (16 * (i & 1));
        raw.v[j] = make_uint4(v[0], v[1], v[2], v[3]);
    }
#pragma unroll
    for (int j = 2; j < N; ++j) raw.v[j] = few_load16<16>(f.row[j] + static_cast<int64_t>(f.n) * 64);      // (h has whole chunks)
}

// The chunks of a span, one after the other: chunk(raw, i).  The first four are on their way on entry (few_begin), those of `next` when it returns,
// if there are as many.  The last four of a number that is no multiple of four overlap those before them; fewer than four, and a chunk that is there in
// part, are fetched on their own.
template <int ALIGN, int N, class Chunk>
__device__ __forceinline__ void few_walk(FewRaw<N> (&raw)[kFewAhead], const FewWeights &w, const FewSpan<N> &f, const FewSpan<N> &next, uint32_t q, Chunk &&chunk)
{
    const int32_t n = f.n;
    if (n >= kFewAhead) {
        const uint8_t *row[N];
#pragma unroll
        for (int i = 0; i < N; ++i) row[i] = f.row[i];
#pragma unroll 1
        for (int32_t j = 0; j < n; j += kFewAhead) {
            const int32_t from = min(j, n - kFewAhead), step = min(j + kFewAhead, n - kFewAhead) - from;
            const bool other = j + kFewAhead >= n && next.n >= kFewAhead;       // (with none to come, the last ones again, to no use)
#pragma unroll
            for (int i = 0; i < N; ++i) row[i] = other ? next.row[i] : row[i] + step * 64;
#pragma unroll
            for (int u = 0; u < kFewAhead; ++u) {
                if (from + u >= j) chunk(raw[u], from + u);
                few_fetch<ALIGN, N>(raw[u], row, u);
            }
        }
    }
#pragma unroll 1
    for (int32_t i = n >= kFewAhead ? n : 0; i < n + (f.tail ? 1 : 0); ++i) {
        FewRaw<N> r;
        if (i < n) {
            few_fetch<ALIGN, N>(r, f.row, i);
        } else {
            few_fetch_tail(r, w, f, q);
        }
        chunk(r, i);
    }
}
template <int ALIGN, int N>
__device__ __forceinline__ void few_begin(FewRaw<N> (&raw)[kFewAhead], const FewSpan<N> &f)
{
    if (f.n >= kFewAhead) {
#pragma unroll
        for (int u = 0; u < kFewAhead; ++u) few_fetch<ALIGN, N>(raw[u], f.row, u);
    }
}

// ---- operands -----------------------------------------------------------------------------------------------------

__device__ __forceinline__ void few_mma(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1, __nv_bfloat16)
{
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                 : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void few_mma(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1, __half)
{
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                 : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// Two rows' eight k of each lane (a, b) against those of eight choices (v).
template <class T>
__device__ __forceinline__ void few_products(float (&acc)[4], const uint4 &a, const uint4 &b, const uint4 &v)
{
    few_mma(acc, a.x, b.x, a.y, b.y, v.x, v.y, T());
    few_mma(acc, a.z, b.z, a.w, b.w, v.z, v.w, T());
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
__device__ __forceinline__ void few_two_parts(const uint4 &f16, uint4 &hi, uint4 &lo)
{
    const uint32_t w[4] = {f16.x, f16.y, f16.z, f16.w};
    uint32_t h[4], l[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float2 f = __half22float2(*reinterpret_cast<const __half2 *>(&w[i]));
        few_two_parts(f.x, f.y, h[i], l[i]);
    }
    hi = make_uint4(h[0], h[1], h[2], h[3]);
    lo = make_uint4(l[0], l[1], l[2], l[3]);
}

// The chunks of slice s of S: whole runs of four but for the last slice's.
__device__ __forceinline__ void few_slice(int32_t chunks, int32_t s, int32_t slices, int32_t &first, int32_t &n)
{
    const int32_t runs = (chunks + kFewAhead - 1) / kFewAhead;
    first = min(chunks, runs * s / slices * kFewAhead);
    n = min(chunks, runs * (s + 1) / slices * kFewAhead) - first;
}

// ---- launch 1: h = act(W1 x) ------------------------------------------------------------------------------------------

// 8 consecutive elements of x, zeros beyond its end.
__device__ __forceinline__ uint4 few_load_x(const uint16_t *row, int32_t k, int32_t depth, int32_t vec)
{
    if (k >= depth) return make_uint4(0u, 0u, 0u, 0u);
    if (vec && k + 8 <= depth) return *reinterpret_cast<const uint4 *>(row + k);
    uint32_t w[4] = {0u, 0u, 0u, 0u};
#pragma unroll
    for (int i = 0; i < 8; ++i)
        if (k + i < depth) w[i / 2] |= static_cast<uint32_t>(row[k + i]) << (16 * (i & 1));
    return make_uint4(w[0], w[1], w[2], w[3]);
}

__device__ __forceinline__ float few_silu(float u) { return u / (1.0f + __expf(-u)); }

// T: the type of x and of the weights.  Dynamic shared memory: the lists, then x.
template <class T, int ALIGN>
__global__ void __launch_bounds__(kFewUpThreads, 2)
few_up_kernel(const FewParams p)
{
    constexpr int kWarps = kFewUpThreads / 32;
    extern __shared__ __align__(16) uint8_t smem[];
    __shared__ float4 s_part[kWarps][32];
    __shared__ const uint16_t *s_row[kFewEntry];                  // the entry's tokens
    const FewLists l = few_lists(smem, p);
    uint4 *s_x = reinterpret_cast<uint4 *>(smem + few_list_bytes(p.experts, p.choices));      // [chunk][8 choices][4 lanes]
    grid_dependency_wait();
    grid_launch_dependents();                                     // launch 2 may read the call's inputs from here on
    few_make_lists(p, l);
    const int32_t warp = static_cast<int32_t>(threadIdx.x >> 5);
    const uint32_t lane = threadIdx.x & 31u, q = lane & 3u, m = lane >> 2;
    const int32_t chunks = (p.w.depth + kFewChunk - 1) / kFewChunk;

    // Every CTA has as many whole groups, one after the other; those left over are shared by `rest_slices` CTAs each.
    const int32_t units = *l.total * p.groups, ctas = static_cast<int32_t>(gridDim.x), cta = static_cast<int32_t>(blockIdx.x);
    const int32_t rounds = units / ctas, rest = units - rounds * ctas;
    int32_t rest_slices = 1;
    while (rest_slices * 2 <= p.most_slices && rest * rest_slices * 2 <= ctas) rest_slices *= 2;
    const int32_t my_rounds = rounds + (cta < rest * rest_slices ? 1 : 0);

    struct Work {
        int32_t entry, expert, first, count, row0, row1, slices, slice;
        bool has0, has1;
    };
    auto work_of = [&](int32_t round) {
        Work t;
        const bool whole = round < rounds;
        t.slices = whole ? 1 : rest_slices;
        const int32_t unit = whole ? cta * rounds + round : rounds * ctas + cta / rest_slices;
        t.entry = fast_div(unit, p.fd_groups);
        const int32_t group = unit - t.entry * p.groups;
        // a CTA's share of the group's eight tiles, and of each tile's contraction
        const int32_t tile = group * kWarps + (whole ? warp : (cta % rest_slices) * (kWarps / rest_slices) + warp / rest_slices);
        t.slice = whole ? 0 : warp % rest_slices;
        t.expert = static_cast<int32_t>(l.entry[2 * t.entry]);
        t.first = static_cast<int32_t>(l.entry[2 * t.entry + 1] & 0xffffu);
        t.count = static_cast<int32_t>(l.entry[2 * t.entry + 1] >> 16);
        const int32_t r0 = tile * (p.gated ? 8 : 16) + static_cast<int32_t>(m), r1 = p.gated ? r0 : r0 + 8;
        t.has0 = r0 < p.inner;
        t.has1 = r1 < p.inner;
        t.row0 = t.has0 ? r0 : 0;
        t.row1 = !t.has1 ? 0 : p.gated ? r1 + p.inner : r1;
        return t;
    };
    // x in pieces: the chunks (whole runs of four) whose tokens fit the shared memory
    const int32_t piece = min(chunks, p.piece / 512 & ~(kFewAhead - 1));
    auto span_of = [&](const Work &t, int32_t begin) {
        int32_t first, n;
        few_slice(min(piece, chunks - begin), t.slice, t.slices, first, n);
        return few_span<2>(p.w, t.expert, t.row0, t.row1, begin + first, __any_sync(0xffffffffu, t.has0) ? n : 0, q);
    };

    FewRaw<2> raw[kFewAhead];
    FewSpan<2> span{};
    if (my_rounds > 0) {
        span = span_of(work_of(0), 0);
        few_begin<ALIGN>(raw, span);
    }
    int32_t staged_entry = -1, staged_begin = -1;
    for (int32_t round = 0; round < my_rounds; ++round) {
        const Work now = work_of(round);
        float acc[4] = {};
        for (int32_t begin = 0; begin < chunks; begin += piece) {
            if (now.entry != staged_entry || begin != staged_begin) {
                // the entry's tokens, as the products read them
                __syncthreads();
                if (now.entry != staged_entry) {
                    if (threadIdx.x < now.count)
                        s_row[threadIdx.x] = static_cast<const uint16_t *>(p.x) + static_cast<int64_t>(l.list[now.first + threadIdx.x] / p.top_k) * p.ldx;
                    __syncthreads();
                }
                // 16-byte pieces in their places: chunk, eight choices, four lanes.  Four on their way at a time.
                const int32_t pieces = min(piece, chunks - begin) * 4;      // of a choice
                for (int32_t n = 0; n < now.count; ++n) {
                    const uint16_t *row = s_row[n];
                    for (int32_t u0 = static_cast<int32_t>(threadIdx.x); u0 < pieces; u0 += 4 * kFewUpThreads) {
                        uint4 v[4];
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const int32_t u = u0 + i * kFewUpThreads;
                            v[i] = u < pieces ? few_load_x(row, begin * kFewChunk + u * 8, p.w.depth, p.x_vec) : make_uint4(0u, 0u, 0u, 0u);
                        }
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const int32_t u = u0 + i * kFewUpThreads;
                            if (u < pieces) s_x[(u >> 2) * 32 + n * 4 + (u & 3)] = v[i];
                        }
                    }
                }
                __syncthreads();
                staged_entry = now.entry;
                staged_begin = begin;
            }
            const FewSpan<2> here = span;
            span.n = 0;
            if (begin + piece < chunks) span = span_of(now, begin + piece);
            else if (round + 1 < my_rounds) span = span_of(work_of(round + 1), 0);
            const uint4 *x = s_x + (here.first - begin) * 32 + lane;
            few_walk<ALIGN>(raw, p.w, here, span, q, [&](const FewRaw<2> &r, int32_t i) { few_products<T>(acc, r.v[0], r.v[1], x[i * 32]); });
            if (here.n < kFewAhead) few_begin<ALIGN>(raw, span);      // nothing was fetched on the way
        }
        if (now.slices > 1) {
            if (now.slice > 0) s_part[warp][lane] = make_float4(acc[0], acc[1], acc[2], acc[3]);
            __syncthreads();
            if (now.slice == 0) {
                for (int32_t s = 1; s < now.slices; ++s) {
                    const float4 v = s_part[warp + s][lane];
                    acc[0] += v.x, acc[1] += v.y, acc[2] += v.z, acc[3] += v.w;
                }
            }
        }
        if (now.slice == 0) {
            // this lane's row of h (without a gate: its two rows); whole chunks are written, zeros beyond inner
            const int32_t unit = round < rounds ? cta * rounds + round : rounds * ctas + cta / rest_slices;
            const int32_t tile = (unit - now.entry * p.groups) * kWarps + (round < rounds ? warp : (cta % rest_slices) * (kWarps / rest_slices) + warp / rest_slices);
            const int32_t k0 = tile * (p.gated ? 8 : 16) + static_cast<int32_t>(m);
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const int32_t at = static_cast<int32_t>(q) * 2 + j;
                const bool used = at < now.count;
                const int64_t c = used ? l.list[now.first + at] : 0;
                const float u0 = acc[j], u1 = acc[2 + j];
                const float v[2] = {now.has0 ? (p.gated ? few_silu(u0) * u1 : few_silu(u0)) : 0.0f, now.has1 && !p.gated ? few_silu(u1) : 0.0f};
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    if (i == 1 && p.gated) break;
                    const int32_t k = k0 + 8 * i;
                    if (!used || k >= p.h_stride) continue;
                    uint32_t hi, lo;
                    few_two_parts(v[i], 0.0f, hi, lo);
                    uint16_t *dst = reinterpret_cast<uint16_t *>(p.h + c * p.h_stride + k);
                    dst[0] = static_cast<uint16_t>(hi);
                    dst[static_cast<int64_t>(p.choices) * p.h_stride] = static_cast<uint16_t>(lo);
                }
            }
        }
    }
}

// ---- launch 2: y = sum of weight * (W2 h) ------------------------------------------------------------------------------

// grid: 16 rows of W2 (outputs) a cluster of `ranks` CTAs, which take the entries in turn (entry i: CTA i % ranks).  Dynamic shared memory: the lists, the choices' weights, most_slices x choices x 16 sums.
template <class T, int ALIGN>
__global__ void __launch_bounds__(kFewDownThreads, 1)
few_down_kernel(const FewParams p)
{
    constexpr int kWarps = kFewDownThreads / 32;
    extern __shared__ __align__(16) uint8_t smem[];
    const FewLists l = few_lists(smem, p);
    float *s_weight = reinterpret_cast<float *>(smem + few_list_bytes(p.experts, p.choices)), *part = s_weight + ((p.choices + 3) & ~3);
    grid_launch_dependents();
    for (int32_t c = static_cast<int32_t>(threadIdx.x); c < p.choices; c += kFewDownThreads) s_weight[c] = ld_older(p.weights + c);      // inputs of the call: launch 1 has waited for them
    few_make_lists(p, l);
    const int32_t warp = static_cast<int32_t>(threadIdx.x >> 5);
    const uint32_t lane = threadIdx.x & 31u, q = lane & 3u, m = lane >> 2;
    const int32_t rank = p.ranks > 1 ? static_cast<int32_t>(cluster_ctarank()) : 0, out0 = static_cast<int32_t>(blockIdx.x) / p.ranks * 16;
    const int32_t r0 = out0 + static_cast<int32_t>(m), chunks = (p.w.depth + kFewChunk - 1) / kFewChunk;
    const int32_t row0 = r0 < p.w.rows ? r0 : 0, row1 = r0 + 8 < p.w.rows ? r0 + 8 : 0;
    // rounds of an entry per warp; those left over are shared by several warps
    const int32_t entries = *l.total, all = kWarps * p.ranks, rounds = entries / all, rest = entries - rounds * all;
    int32_t rest_slices = 1;
    while (rest_slices * 2 <= p.most_slices && (rest + p.ranks - 1) / p.ranks * rest_slices * 2 <= kWarps) rest_slices *= 2;
    const int32_t my_rounds = rounds + (warp / rest_slices * p.ranks + rank < rest ? 1 : 0);
    struct Work {
        int32_t expert, first, count, slice;
    };
    auto work_of = [&](int32_t round) {
        Work t;
        const bool whole = round < rounds;
        const int32_t entry = (whole ? round * all + warp * p.ranks : rounds * all + warp / rest_slices * p.ranks) + rank;
        t.slice = whole ? 0 : warp % rest_slices;
        t.expert = static_cast<int32_t>(l.entry[2 * entry]);
        t.first = static_cast<int32_t>(l.entry[2 * entry + 1] & 0xffffu);
        t.count = static_cast<int32_t>(l.entry[2 * entry + 1] >> 16);
        return t;
    };
    auto span_of = [&](int32_t round) {
        const Work t = work_of(round);
        int32_t first, n;
        few_slice(chunks, t.slice, round < rounds ? 1 : rest_slices, first, n);
        FewSpan<4> f = few_span<4>(p.w, t.expert, row0, row1, first, n, q);
        const int64_t c = l.list[t.first + min(static_cast<int32_t>(m), t.count - 1)];
        f.row[2] = reinterpret_cast<const uint8_t *>(p.h + c * p.h_stride) + first * 64 + q * 16;
        f.row[3] = f.row[2] + static_cast<int64_t>(p.choices) * p.h_stride * 2;
        return f;
    };
    FewRaw<4> raw[kFewAhead];
    FewSpan<4> span{};
    if (my_rounds > 0) {
        span = span_of(0);
        if (span.n >= kFewAhead) {                                // the weights' first chunks: those of h are not there yet
#pragma unroll
            for (int u = 0; u < kFewAhead; ++u) {
                raw[u].v[0] = few_load16_older<ALIGN>(span.row[0] + u * 64);
                raw[u].v[1] = few_load16_older<ALIGN>(span.row[1] + u * 64);
            }
        }
    }
    grid_dependency_wait();                                       // h
    if (my_rounds > 0 && span.n >= kFewAhead) {
#pragma unroll
        for (int u = 0; u < kFewAhead; ++u) {
            raw[u].v[2] = few_load16<16>(span.row[2] + u * 64);
            raw[u].v[3] = few_load16<16>(span.row[3] + u * 64);
        }
    }
    for (int32_t round = 0; round < my_rounds; ++round) {
        const Work now = work_of(round);
        float acc[4] = {};
        const FewSpan<4> here = span;
        span.n = 0;
        if (round + 1 < my_rounds) span = span_of(round + 1);
        few_walk<ALIGN>(raw, p.w, here, span, q, [&](const FewRaw<4> &r, int32_t) {
            using B = __nv_bfloat16;
            if constexpr (std::is_same<T, B>::value) {
                few_products<B>(acc, r.v[0], r.v[1], r.v[2]);
                few_products<B>(acc, r.v[0], r.v[1], r.v[3]);
            } else {
                uint4 a[2], b[2];
                few_two_parts(r.v[0], a[0], a[1]);
                few_two_parts(r.v[1], b[0], b[1]);
                few_products<B>(acc, a[0], b[0], r.v[2]);
                few_products<B>(acc, a[0], b[0], r.v[3]);
                few_products<B>(acc, a[1], b[1], r.v[2]);
            }
        });
        if (here.n < kFewAhead) few_begin<ALIGN>(raw, span);      // nothing was fetched on the way
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const int32_t at = static_cast<int32_t>(q) * 2 + j;
            if (at >= now.count) continue;
            float *dst = part + (now.slice * p.choices + l.list[now.first + at]) * 16;
            dst[m] = acc[j];
            dst[m + 8] = acc[2 + j];
        }
        // an entry that one warp had alone has one sum for each choice: the other slices' are zeros
        if (round < rounds) {
            for (int32_t s = 1; s < rest_slices; ++s) {
                for (int32_t i = static_cast<int32_t>(lane); i < now.count * 16; i += 32) part[(s * p.choices + l.list[now.first + (i >> 4)]) * 16 + (i & 15)] = 0.0f;
            }
        }
    }
    // places are not needed any more: whose sums a choice has
    for (int32_t i = static_cast<int32_t>(threadIdx.x); i < entries; i += kFewDownThreads) {
        const uint32_t e = l.entry[2 * i + 1];
        for (uint32_t k = 0; k < e >> 16; ++k) l.rank[l.list[(e & 0xffffu) + k]] = static_cast<uint16_t>(i % p.ranks);
    }
    __syncthreads();
    if (rest_slices > 1) {                                        // the slices of this CTA's own
        for (int32_t i = static_cast<int32_t>(threadIdx.x); i < p.choices * 16; i += kFewDownThreads) {
            if (l.expert[i >> 4] == kFewNone || l.rank[i >> 4] != rank) continue;
            float v = part[i];
            for (int32_t s = 1; s < rest_slices; ++s) v += part[s * p.choices * 16 + i];
            part[i] = v;
        }
        __syncthreads();
    }
    if (p.ranks > 1) {
        cluster_arrive();
        cluster_wait();
    }
    for (int32_t o = rank * kFewDownThreads + static_cast<int32_t>(threadIdx.x); o < p.tokens * 16; o += p.ranks * kFewDownThreads) {
        const int32_t t = o >> 4, r = o & 15, row = out0 + r;
        if (row >= p.w.rows) continue;
        float sum = 0.0f;
        for (int32_t j0 = 0; j0 < p.top_k; j0 += 4) {
            float v[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int32_t c = t * p.top_k + min(j0 + j, p.top_k - 1);
                const bool there = j0 + j < p.top_k && l.expert[c] != kFewNone;
                v[j] = 0.0f;
                if (there && p.ranks > 1) asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v[j]) : "r"(mapa(smem_addr(part + c * 16 + r), l.rank[c])) : "memory");
                else if (there) v[j] = part[c * 16 + r];
            }
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int32_t c = t * p.top_k + min(j0 + j, p.top_k - 1);
                if (j0 + j < p.top_k && l.expert[c] != kFewNone) sum = fmaf(s_weight[c], v[j], sum);
            }
        }
        static_cast<T *>(p.y)[t * p.ldy + row] = narrow_to<T>(sum);
    }
    __syncwarp();
    if (p.ranks > 1) {                                            // no CTA leaves while another reads its sums
        cluster_arrive();
        cluster_wait();
    }
}

} // namespace hgemm_dev
