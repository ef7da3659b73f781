// The 8-bit product with block scales: D = sum_b sP[., b] sQ[., b] (P_b Q_b^T), b = blocks of 128 of the contraction.
//
// fp32 scales rule out letting the tensor cores sum the whole contraction (their own block scales are powers of two), so each
// block of 128 is a product of its own: four tcgen05.mma (kind::f8f6f4, K = 32) into a fresh tensor-memory accumulator, which
// eight warps then read, multiply by the block's scales and add to running sums in REGISTERS ("promotion").  One accumulator is
// read while the next is computed, so the tensor pipe and the promotion overlap; the budget per block and SM of a 256 x 256
// pair tile is 512 cycles of MMA against 256 cycles of tensor-memory reads and 256 (one scale per row and 128-column block: a
// multiply-add per element) or 512 (a scale per column: a product besides) cycles of fp32 arithmetic per scheduler.  The packed
// form of two elements an instruction issues at half rate: it saves instructions, not pipe time.
//
// Roles (384 threads): warp 0 fills a ring of shared-memory stages by TMA (one stage = one block of 128: 128 bytes of every
// row, or 128 rows of 128 columns where an operand is stored along its own dimension); warp 1 issues the MMAs; warp 2 fetches
// the blocks' scales into a ring of their own with 4-byte asynchronous copies; warps 4..11 promote and store.
//
// Two shapes: CTA pairs with 256 x 256 tiles, results stored by rows through a small staging buffer (large problems); single
// CTAs with 128 x BN tiles, BN = 16 .. 128, for which P is the WEIGHT (its rows fill the 128 lanes of an accumulator
// however few tokens there are) and the tile is stored transposed; there the CTAs of a cluster may share one tile's
// contraction and add their parts through distributed shared memory in rank order.
//
// Products over experts: the tiles of all groups are numbered through with prefix sums of the groups' tile counts, which
// every CTA computes for itself from the offsets.  A tile never crosses a group; the rows it computes beyond its group's end
// are not stored.  Weight gradients contract over a group's rows, which the column-quantised copy pads with zeros to whole blocks.
//
// Measured (B200, bf16 results unless said), bursts of launches on the same operands: 4096^3 forward 69 us (2000 TFLOP/s), 8192^3
// 501 us (2190; 408 us without the promotion), 8192 x 4096 x 4096 weight gradient in fp32 178 us (1540); 1000 x 4096 x 4096 21.5 us;
// 7 x 8192 x 4096 9.9 us (3.4 TB/s).  As passes whose operands change from one to the next: 8192^3 555 us (1980), the weight gradient
// 201 us (1370), 1000 x 4096 x 4096 22.8 us, 7 x 8192 x 4096 11.6 us, 64 experts x 4 rows with 2048 x 2048 weights 43 us (6.3 TB/s).
// In loops of seconds the power cap adds to that (8192^3 584 us at 1.36 GHz).  What bounds the large ones is the promoting warps
// (multiply-adds, barrier round trips and, on the MMA warp's scheduler, its instructions), 720-770 cycles a block of 512 cycles of MMA.
//
// Every mbarrier wait is bounded (see hgemm_device.cuh): a wait that runs out raises the status word and the CTA's abort flag, and
// every role falls through to the common teardown.
#pragma once

#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <stdint.h>

#include <type_traits>

#include "hgemm_device.cuh"

namespace hgemm_dev {

constexpr int kFp8Threads = 384;
constexpr int kFp8Block = 128;                    // the scales' block, and one stage's share of the contraction
constexpr int kFp8PBytes = 128 * 128;             // P part of a stage: 128 rows of 128 bytes
constexpr int kFp8MaxStages = 12;
constexpr int kFp8MaxGroups = 1024;
constexpr int kFp8CtrlBytes = 512;
constexpr int kFp8StagingPerWarp = 8192;          // results on their way out: two boxes of 32 rows x 128 bytes
constexpr uint32_t kRoleFp8Load = 8, kRoleFp8Mma = 9, kRoleFp8Scale = 10, kRoleFp8Promote = 11;
constexpr uint32_t kFp8PartPitch = 132;            // words between the columns of a slice's part
constexpr int kFp8Batch = 4;                      // scales travel in batches of four blocks (one barrier round per batch)
__host__ __device__ constexpr int fp8_ring(int cta_group) { return cta_group == 2 ? 2 : 4; }     // batches in flight: single CTAs go through theirs faster than two arrive
__host__ __device__ constexpr int fp8_slot_bytes(int bn, bool q_col) { return (128 + (q_col ? bn : 4)) * 4; }     // one block's scales

// which side of the tile grid follows the groups' offsets
enum : int32_t { kRaggedNone = 0, kRaggedP = 1, kRaggedQ = 2, kRaggedK = 3 };

struct Fp8Params {
    int32_t rows_p, rows_q;        // rows of P and Q (per group, or all of them on the side that follows the offsets)
    int32_t kblocks;               // blocks of the contraction (not with kRaggedK)
    int32_t tiles_p, tiles_q;      // tiles per group (unused for the side that follows the offsets)
    int32_t total;                 // tiles, where the host knows them (kRaggedNone, kRaggedK)
    int32_t raster;                // tiles of P visited together
    FastDiv fd_other, fd_group, fd_sweep, fd_raster, fd_last;   // divisors of the tile numbering: see fp8_tile
    int32_t groups, ragged, rows_ragged, k_capacity;   // rows_ragged: clamp of the offsets; k_capacity: blocks the padded copy has
    const int32_t *offsets;
    const float *sp, *sq;          // scale of row r (or of block r / 128), block b: s[r * _row + b * _kb + group * _group]
    int64_t sp_row, sp_kb, sp_group, sq_row, sq_kb, sq_group;
    void *out;
    int64_t ldc, c_group;
    int32_t out_type, accumulate, vec_ok;   // out_type: 0 fp32, 1 fp16, 2 bf16; vec_ok: rows of C start and end at multiples of 16 bytes
    int32_t split, stages;
    int32_t p_mn, q_mn;            // operand stored along its own rows' dimension (contraction down the columns)
    uint32_t idesc;
    uint32_t *status;
    long long wait_budget;
};

struct Fp8Tile {
    int32_t group, p0, p_end, q0, q_end, kb0, kbn;
};

// The tile with number w; whole (converged) warp.  pre: prefix sums over the groups (tiles, or blocks for kRaggedK); off: clamped offsets.
template <int TP, int TQ>
__device__ __forceinline__ Fp8Tile fp8_tile(int32_t w, const Fp8Params &p, const int32_t *pre, const int32_t *off, uint32_t lane)
{
    Fp8Tile t;
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

// Clamped offsets and the prefix sums fp8_tile reads; one whole warp.
__device__ __forceinline__ void fp8_scan_groups(const Fp8Params &p, int32_t *pre, int32_t *off, int32_t unit, uint32_t lane)
{
    int32_t carry = 0, last = 0;
    for (int32_t base = 0; base < p.groups; base += 32) {
        const int32_t e = base + static_cast<int32_t>(lane);
        int32_t o = p.offsets[min(e, p.groups)];
        o = min(max(o, 0), p.rows_ragged);
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {               // non-decreasing whatever the caller's values
            const int32_t x = __shfl_up_sync(0xffffffffu, o, d);
            if (static_cast<int32_t>(lane) >= d) o = max(o, x);
        }
        o = max(o, last);
        int32_t nxt = __shfl_down_sync(0xffffffffu, o, 1);
        if (lane == 31) nxt = max(o, min(max(p.offsets[min(e + 1, p.groups)], 0), p.rows_ragged));
        last = __shfl_sync(0xffffffffu, nxt, 31);
        int32_t n = e < p.groups ? (nxt - o + unit - 1) / unit : 0;
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
            const int32_t x = __shfl_up_sync(0xffffffffu, n, d);
            if (static_cast<int32_t>(lane) >= d) n += x;
        }
        if (e < p.groups) {
            off[e] = o;
            off[e + 1] = nxt;
            pre[e + 1] = p.ragged == kRaggedK ? min(carry + n, p.k_capacity) : carry + n;
        }
        carry += __shfl_sync(0xffffffffu, n, 31);
    }
    if (lane == 0) pre[0] = 0;
}

template <class T>
__device__ __forceinline__ T fp8_to(float v);
template <>
__device__ __forceinline__ float fp8_to<float>(float v) { return v; }
template <>
__device__ __forceinline__ __half fp8_to<__half>(float v) { return __float2half_rn(v); }
template <>
__device__ __forceinline__ __nv_bfloat16 fp8_to<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }

__device__ __forceinline__ uint32_t fp8_pack2(float a, float b, __half)
{
    const __half2 h = __floats2half2_rn(a, b);
    return *reinterpret_cast<const uint32_t *>(&h);
}
__device__ __forceinline__ uint32_t fp8_pack2(float a, float b, __nv_bfloat16)
{
    const __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<const uint32_t *>(&h);
}

// Where the column-scaled promotion keeps its sums: chunks of 16 rows x 32 columns, rows 0..15 before 16..31, each chunk by eights of
// columns, each of those as the lane's column pair of row t / 4, then of row t / 4 + 8.  f: eight of columns, hi: eight of rows (0..3).
template <int REPS = 4>
__host__ __device__ constexpr int fp8_frag_index(int f, int hi) { return (((f / REPS) * 2 + hi / 2) * REPS + f % REPS) * 2 + hi % 2; }

// One warp's 32 rows x 128 columns of running sums (64 columns from col0, 64 from col0 + 128) to C, by rows.  Each lane packs its
// row into boxes of 32 rows x 128 bytes in shared memory (16-byte pieces swizzled as TMA reads them: conflict-free), which leave as
// tensor stores while the warp goes on with the next tile; stores by the warp itself kept it for 3500 cycles a tile.  A warp whose
// rows end inside its 32 (a group's end) stores 16 bytes a lane; rows of C that are not multiples of 16 bytes, and C +=, take
// ordinary stores of 4 bytes a lane.
// FRAG: the sums lie as the fragments of 16 x 8 that the column-scaled promotion reads (see there), else a lane holds its row.
template <class T, bool FRAG>
__device__ __forceinline__ void fp8_store_rows(const uint64_t (&acc)[64], uint32_t staging, const Fp8Params &p, const CUtensorMap *tmap_c, const Fp8Tile &t,
                                               int32_t row0, int32_t col0, uint32_t lane)
{
    constexpr int kSize = static_cast<int>(sizeof(T));
    constexpr int kBox = 128 / kSize;                             // columns of a box
    constexpr int kPass = 2 * kBox;                               // columns of one pass: two boxes
    const bool whole = p.vec_ok && !p.accumulate && (row0 + 32 <= t.p_end || t.p_end == p.rows_p);   // the map clips at the matrix's own end
#pragma unroll
    for (int c = 0; c < 128; c += kPass) {
        bulk_wait_group_read<0>();                                // earlier stores have read the boxes
        __syncwarp();
        if constexpr (FRAG) {
            const uint32_t fr = lane >> 2, fc = lane & 3u;        // row and column pair of this lane in a fragment
#pragma unroll
            for (int n = 0; n < kPass / 8; ++n) {                 // fragments across the pass
                const int f = c / 8 + n;                          // eight columns 8 f .. 8 f + 7
                const uint32_t box = staging + static_cast<uint32_t>(n * 8 / kBox) * 4096u;
#pragma unroll
                for (int hi = 0; hi < 4; ++hi) {                  // rows 8 hi + fr
                    const uint64_t v = acc[fp8_frag_index(f, hi)];
                    const uint32_t at = box + (8u * hi + fr) * 128u;
                    if constexpr (kSize == 4) {
                        st_shared_u64(at + (((static_cast<uint32_t>(2 * n) & 7u) + (fc >> 1)) ^ fr) * 16u + (fc & 1u) * 8u, v);
                    } else {
                        float x, y;
                        unpack_f32x2(v, x, y);
                        st_shared_u32(at + ((static_cast<uint32_t>(n) & 7u) ^ fr) * 16u + fc * 4u, fp8_pack2(x, y, T()));
                    }
                }
            }
        } else {
            const uint32_t mine = staging + lane * 128u, swz = lane & 7u;
#pragma unroll
            for (int j = 0; j < 16; ++j) {
                uint32_t v[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    float lo, hi;
                    if constexpr (kSize == 4) {
                        unpack_f32x2(acc[(c + j * 4 + i) / 2], lo, hi);
                        v[i] = __float_as_uint((i & 1) ? hi : lo);
                    } else {
                        unpack_f32x2(acc[j * 4 + i], lo, hi);
                        v[i] = fp8_pack2(lo, hi, T());
                    }
                }
                st_shared_v4(mine + (j / 8) * 4096u + (((j & 7u) ^ swz) * 16u), v[0], v[1], v[2], v[3]);
            }
        }
        if (whole) {
            fence_proxy_async_smem();
            __syncwarp();
#pragma unroll
            for (int r = 0; r < 2; ++r) {
                const int at = c + r * kBox, col = col0 + at + (at & 64);
                if (row0 < t.p_end && col < t.q_end) tma_store_3d_elect(tmap_c, col, row0, p.ragged == kRaggedK ? t.group : 0, staging + r * 4096u);
            }
        } else if (p.vec_ok && !p.accumulate) {
            // a group's end inside the 32 rows: 16 bytes a lane, two rows at a time
            __syncwarp();
            T *out = static_cast<T *>(p.out) + t.group * p.c_group;
            const uint32_t k = lane & 7u, box = (lane >> 3) & 1u;
            const int32_t at = c + static_cast<int32_t>(box) * kBox + static_cast<int32_t>(k) * (16 / kSize), col = col0 + at + (at & 64);
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const uint32_t r = 2u * i + (lane >> 4);
                const float4 v = ld_shared_v4(staging + box * 4096u + r * 128u + ((k ^ (r & 7u)) * 16u));
                if (row0 + static_cast<int32_t>(r) < t.p_end && col < t.q_end)         // rows of C are multiples of 16 bytes: a piece is inside or outside
                    *reinterpret_cast<float4 *>(out + static_cast<int64_t>(row0 + static_cast<int32_t>(r)) * p.ldc + col) = v;
            }
        } else if constexpr (kSize == 2) {
            // rows at any even address: two elements a lane where the pair starts at a multiple of 4 bytes.  In a run of 64 that does not,
            // lane 0 takes its first and its last element.
            __syncwarp();
            T *out = static_cast<T *>(p.out) + t.group * p.c_group;
#pragma unroll 1
            for (int32_t i0 = 0; i0 < 32; i0 += 8) {                     // the loads of eight rows before their stores
                uint32_t h[8][2];
#pragma unroll
                for (int j = 0; j < 8; ++j) {
#pragma unroll
                    for (int r = 0; r < 2; ++r) {
                        const int32_t i = i0 + j;
                        const int32_t e = 2 * static_cast<int32_t>(lane) - (static_cast<int32_t>(reinterpret_cast<uintptr_t>(out + static_cast<int64_t>(row0 + i) * p.ldc + col0) >> 1) & 1);
                        const int32_t ea = e < 0 ? 0 : e, eb = e < 0 ? 63 : e + 1;
                        const uint32_t from = staging + r * 4096u + i * 128u;
                        h[j][r] = ld_shared_u16(from + (((ea >> 3) ^ j) * 16u) + (ea & 7) * 2u) | static_cast<uint32_t>(ld_shared_u16(from + (((eb >> 3) ^ j) * 16u) + (eb & 7) * 2u)) << 16;
                    }
                }
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    if (row0 + i0 + j >= t.p_end) break;
                    T *row = out + static_cast<int64_t>(row0 + i0 + j) * p.ldc + col0;
                    const int32_t e = 2 * static_cast<int32_t>(lane) - (static_cast<int32_t>(reinterpret_cast<uintptr_t>(row) >> 1) & 1);
#pragma unroll
                    for (int r = 0; r < 2; ++r) {
                        const int32_t left = t.q_end - col0 - 128 * r;             // columns of the run
                        unsigned short *d = reinterpret_cast<unsigned short *>(row + 128 * r);
                        if (e >= 0 && e + 1 < left) {
                            *reinterpret_cast<uint32_t *>(d + e) = h[j][r];
                        } else {
                            if (max(e, 0) < left) d[max(e, 0)] = static_cast<unsigned short>(h[j][r]);
                            if (e < 0 && 63 < left) d[63] = static_cast<unsigned short>(h[j][r] >> 16);
                        }
                    }
                }
            }
        } else {
            __syncwarp();
            float *out = static_cast<float *>(p.out) + t.group * p.c_group;
#pragma unroll 1
            for (int32_t i0 = 0; i0 < 32; i0 += 8) {
                float v[8][2];
#pragma unroll
                for (int j = 0; j < 8; ++j) {
#pragma unroll
                    for (int x = 0; x < 2; ++x) v[j][x] = ld_shared_f32(staging + x * 4096u + (i0 + j) * 128u + (((lane >> 2) ^ j) * 16u) + (lane & 3u) * 4u);
                }
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    if (row0 + i0 + j >= t.p_end) break;
#pragma unroll
                    for (int x = 0; x < 2; ++x) {
                        const int32_t at = c + x * 32 + static_cast<int32_t>(lane), col = col0 + at + (at & 64);
                        float *dst = out + static_cast<int64_t>(row0 + i0 + j) * p.ldc + col;
                        if (col < t.q_end) *dst = p.accumulate ? *dst + v[j][x] : v[j][x];
                    }
                }
            }
        }
    }
}

template <class T>
__device__ __forceinline__ void fp8_store_one(T *dst, float v, int32_t accumulate)
{
    if constexpr (sizeof(T) == 4) *dst = accumulate ? *dst + v : v;
    else *dst = fp8_to<T>(v);
}

// CG: CTAs per tile.  BN: rows of Q per tile.  P_ROW: P has a scale per row (else one per 128 rows).  Q_COL: Q has a scale per row
// (else one per 128).  CG == 2 stores by rows, CG == 1 transposed.
template <int CG, int BN, bool P_ROW, bool Q_COL>
__global__ void __launch_bounds__(kFp8Threads, 1)
fp8_product_kernel(const __grid_constant__ CUtensorMap tmap_p, const __grid_constant__ CUtensorMap tmap_q, const __grid_constant__ CUtensorMap tmap_c, const Fp8Params p)
{
    constexpr int TP = 128 * CG, TQ = BN;
    constexpr int kCols = BN / 2;                                 // columns of the tile a promoting warp holds
    constexpr int kParts = CG;                                    // accumulators of a block: a pair's columns come in two parts, promoted by four warps each
    constexpr int kDepth = CG == 2 ? 2 : 4;                       // blocks in tensor memory
    constexpr uint32_t kTmemCols = kDepth * BN;
    constexpr uint32_t kStageBytes = kFp8PBytes + (BN / CG) * 128;
    constexpr uint32_t kSlotBytes = fp8_slot_bytes(BN, Q_COL);
    constexpr int kRing = fp8_ring(CG);
    static_assert(kTmemCols >= 32 && (kTmemCols & (kTmemCols - 1)) == 0 && kTmemCols <= 512, "tensor memory is allocated in powers of two");

    extern __shared__ uint8_t smem_raw[];
    const uint32_t smem_base = (smem_addr(smem_raw) + 1023u) & ~1023u;
    uint8_t *smem_gen = smem_raw + (smem_base - smem_addr(smem_raw));
    const uint32_t staging_base = smem_base + static_cast<uint32_t>(p.stages) * kStageBytes;
    const uint32_t ring_base = staging_base + (CG == 2 ? 8u * kFp8StagingPerWarp : 0u);
    const uint32_t ctrl_base = ring_base + kRing * kFp8Batch * kSlotBytes;
    uint8_t *ctrl_gen = smem_gen + (ctrl_base - smem_base);
    const uint32_t bar_full = ctrl_base, bar_empty = bar_full + 8 * kFp8MaxStages, bar_tfull = bar_empty + 8 * kFp8MaxStages, bar_tempty = bar_tfull + 32;
    const uint32_t bar_sfull = bar_tempty + 32, bar_sempty = bar_sfull + 8 * kRing;          // ends at 320
    volatile uint32_t *tmem_slot = reinterpret_cast<volatile uint32_t *>(ctrl_gen + 320);
    volatile uint32_t *abort_flag = reinterpret_cast<volatile uint32_t *>(ctrl_gen + 324);
    int32_t *pre = reinterpret_cast<int32_t *>(ctrl_gen + kFp8CtrlBytes);             // groups + 1 each
    int32_t *off = pre + (p.groups + 1);

    const uint32_t warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0);
    const uint32_t lane = lane_id();
    const bool in_cluster = CG == 2 || p.split > 1;
    const uint32_t rank = in_cluster ? cluster_ctarank() : 0u;    // place in the pair, or slice of the contraction
    const bool is_leader = CG == 1 || rank == 0;
    const int32_t per_unit = CG == 2 ? 2 : p.split;
    const int32_t unit = static_cast<int32_t>(blockIdx.x) / per_unit, units = static_cast<int32_t>(gridDim.x) / per_unit;
    WaitCtl ctl{abort_flag, p.status, p.wait_budget};

    grid_launch_dependents();
    if (threadIdx.x == 0) {
        *abort_flag = 0u;
        for (int s = 0; s < p.stages; ++s) {
            mbar_init(bar_full + 8 * s, CG);
            mbar_init(bar_empty + 8 * s, 1);
        }
        for (int b = 0; b < kDepth * kParts; ++b) {
            mbar_init(bar_tfull + 8 * b, 1);
            mbar_init(bar_tempty + 8 * b, 8);      // a pair: four warps of each CTA; one CTA: its eight
        }
        for (int s = 0; s < kRing; ++s) {
            mbar_init(bar_sfull + 8 * s, 32);
            mbar_init(bar_sempty + 8 * s, 8);
        }
        fence_mbar_init();
        prefetch_tensormap(&tmap_p);
        prefetch_tensormap(&tmap_q);
    }
    if (warp == 1) tmem_alloc<CG>(smem_addr(const_cast<uint32_t *>(tmem_slot)), kTmemCols);
    // No thread reads or writes global memory before the kernels ahead in the stream are complete.
    grid_dependency_wait();
    if (warp == 2 && p.groups > 0) fp8_scan_groups(p, pre, off, p.ragged == kRaggedK ? kFp8Block : p.ragged == kRaggedP ? TP : TQ, lane);
    tc_fence_before_sync();
    __syncthreads();
    if (in_cluster) {
        cluster_arrive();
        cluster_wait();
    }
    tc_fence_after_sync();
    const uint32_t tmem_base = __shfl_sync(0xffffffffu, *tmem_slot, 0);
    const int32_t total = p.ragged == kRaggedP ? pre[p.groups] * p.tiles_q : p.ragged == kRaggedQ ? pre[p.groups] * p.tiles_p : p.total;

    auto tile_of = [&](int32_t w) {
        Fp8Tile t = fp8_tile<TP, TQ>(w, p, pre, off, lane);
        if (CG == 1 && p.split > 1) {                              // this CTA's share of the contraction
            const int32_t b = t.kbn * static_cast<int32_t>(rank) / p.split, e = t.kbn * (static_cast<int32_t>(rank) + 1) / p.split;
            t.kb0 += b;
            t.kbn = e - b;
        }
        return t;
    };

    if (warp == 0) {
        // ===== operands =====
        if constexpr (CG == 2) regs_lower<56>();
        int s = 0;
        uint32_t ph = 0;
        const uint32_t full_leader = CG == 2 ? mapa(bar_full, 0) : bar_full;
        bool ok = true;
        for (int32_t w = unit; ok && w < total; w += units) {
            const Fp8Tile t = tile_of(w);
            const int32_t prow = t.p0 + static_cast<int32_t>(CG == 2 ? rank : 0u) * 128, qrow = t.q0 + static_cast<int32_t>(CG == 2 ? rank : 0u) * (BN / CG);
            const int32_t pz = p.ragged == kRaggedQ ? t.group : 0, qz = p.ragged == kRaggedP ? t.group : 0;      // the operand with one matrix per group
            for (int32_t kb = 0; kb < t.kbn; ++kb) {
                ok = mbar_wait_warp(bar_empty + 8 * s, ph ^ 1u, ctl, status_code(kRoleFp8Load, 0, s));
                if (!ok) break;
                const uint32_t p_dst = smem_base + static_cast<uint32_t>(s) * kStageBytes, q_dst = p_dst + kFp8PBytes;
                const int32_t k0 = (t.kb0 + kb) * kFp8Block;
                const uint32_t fb = full_leader + 8 * s;
                if constexpr (CG == 1) {
                    mbar_arrive_expect_tx_elect(bar_full + 8 * s, kStageBytes);
                    tma_load_3d_elect(p_dst, &tmap_p, p.p_mn ? prow : k0, p.p_mn ? k0 : prow, pz, fb);
                    tma_load_3d_elect(q_dst, &tmap_q, p.q_mn ? qrow : k0, p.q_mn ? k0 : qrow, qz, fb);
                } else {
                    if (is_leader) mbar_arrive_expect_tx_elect(bar_full + 8 * s, kStageBytes);
                    else mbar_arrive_expect_tx_cluster_relaxed_elect(fb, kStageBytes);
                    tma_load_3d_pair_elect(p_dst, &tmap_p, p.p_mn ? prow : k0, p.p_mn ? k0 : prow, pz, fb);
                    tma_load_3d_pair_elect(q_dst, &tmap_q, p.q_mn ? qrow : k0, p.q_mn ? k0 : qrow, qz, fb);
                }
                if (++s == p.stages) { s = 0; ph ^= 1u; }
            }
        }
        // Every commit that signals this CTA's stage barriers (the pair's leader signals both CTAs') arrives before the CTA may leave:
        // the promoting warps wait for the accumulators' barriers only.
        for (int i = 0; ok && i < p.stages; ++i) {
            ok = mbar_wait_warp(bar_empty + 8 * s, ph ^ 1u, ctl, status_code(kRoleFp8Load, 1, s));
            if (++s == p.stages) { s = 0; ph ^= 1u; }
        }
    } else if (warp == 1) {
        // ===== MMA issuer =====
        if constexpr (CG == 2) regs_lower<56>();
        if (is_leader) {
            int s = 0;
            uint32_t ph = 0, par = 0;                             // par: bit d = phase of accumulator d's barriers
            const uint64_t desc_p0 = p.p_mn ? make_smem_desc_sw128_mn_major(smem_base, kFp8PBytes) : make_smem_desc_sw128(smem_base);
            const uint64_t desc_q0 = p.q_mn ? make_smem_desc_sw128_mn_major(smem_base + kFp8PBytes, kFp8PBytes) : make_smem_desc_sw128(smem_base + kFp8PBytes);
            // 32 further along the contraction: 32 bytes inside a swizzled row, or 32 rows of 128 bytes
            const uint32_t p_step = p.p_mn ? (32u * 128u) >> 4 : 2u, q_step = p.q_mn ? (32u * 128u) >> 4 : 2u;
            const uint32_t q_part = p.q_mn ? 64u >> 4 : (64u * 128u) >> 4;        // a pair's second part: the next 64 of this CTA's 128 rows of Q
            uint64_t dp = desc_p0, dq = desc_q0;
            uint32_t full = bar_full;
            // Each barrier is asked ahead of its use (the answer of a completed one takes some 100 cycles); only a "not yet" waits.
            bool full_ready = false, acc_ready[kParts] = {};
            bool ok = true;
            auto block = [&](auto dc) {                            // one block into accumulator dc
                constexpr uint32_t d = decltype(dc)::value;
                const uint32_t want = ((par >> d) & 1u) ^ 1u;
                par ^= 1u << d;
                if (!__all_sync(0xffffffffu, full_ready)) ok = mbar_wait_warp(full, ph, ctl, status_code(kRoleFp8Mma, 0, s));
#pragma unroll
                for (uint32_t h = 0; h < kParts; ++h) {
                    constexpr uint32_t acc0 = d * kParts;
                    if (h + 1 < kParts) acc_ready[h + 1] = mbar_test_wait(bar_tempty + 8 * (acc0 + h + 1), want);
                    if (ok && !__all_sync(0xffffffffu, acc_ready[h])) ok = mbar_wait_warp(bar_tempty + 8 * (acc0 + h), want, ctl, status_code(kRoleFp8Mma, 1, acc0 + h));
                    if (!ok) return;
                    tc_fence_after_sync();
#pragma unroll
                    for (uint32_t k = 0; k < 4; ++k) umma_f8_elect<CG>(tmem_base + d * BN + h * (BN / kParts), dp + k * p_step, dq + h * q_part + k * q_step, p.idesc, k);
                    if constexpr (CG == 2) {
                        umma_commit_both_elect(bar_tfull + 8 * (acc0 + h));
                        if (h + 1 == kParts) umma_commit_both_elect(full + 8 * kFp8MaxStages);
                    } else {
                        umma_commit_elect<1>(bar_tfull + 8 * (acc0 + h), 0);
                        umma_commit_elect<1>(full + 8 * kFp8MaxStages, 0);
                    }
                }
                dp += kStageBytes >> 4;
                dq += kStageBytes >> 4;
                full += 8;
                if (++s == p.stages) { s = 0; ph ^= 1u; dp = desc_p0; dq = desc_q0; full = bar_full; }
                full_ready = mbar_test_wait(full, ph);
                constexpr uint32_t nd = (d + 1) % kDepth;
                acc_ready[0] = mbar_test_wait(bar_tempty + 8 * nd * kParts, ((par >> nd) & 1u) ^ 1u);
            };
            for (int32_t w = unit; ok && w < total; w += units) {
                const int32_t kbn = __shfl_sync(0xffffffffu, tile_of(w).kbn, 0);
                acc_ready[0] = false;                              // every tile begins with accumulator 0
                for (int32_t kb = 0; ok && kb < kbn; kb += kDepth) {
                    block(std::integral_constant<uint32_t, 0>());
                    if (ok && kb + 1 < kbn) block(std::integral_constant<uint32_t, 1>());
                    if constexpr (kDepth == 4) {
                        if (ok && kb + 2 < kbn) block(std::integral_constant<uint32_t, 2>());
                        if (ok && kb + 3 < kbn) block(std::integral_constant<uint32_t, 3>());
                    }
                }
            }
        }
    } else if (warp == 2) {
        // ===== scales =====
        if constexpr (CG == 2) regs_lower<56>();
        uint32_t it = 0;
        bool ok = true;
        for (int32_t w = unit; ok && w < total; w += units) {
            const Fp8Tile t = tile_of(w);
            const int32_t prow = t.p0 + static_cast<int32_t>(CG == 2 ? rank : 0u) * 128;
            const float *sp = p.sp + t.group * p.sp_group + t.kb0 * p.sp_kb, *sq = p.sq + t.group * p.sq_group + t.kb0 * p.sq_kb;
            for (int32_t kb = 0; kb < t.kbn; ++kb, ++it, sp += p.sp_kb, sq += p.sq_kb) {
                const uint32_t batch = it / kFp8Batch, s = batch % kRing, slot = ring_base + (it % (kRing * kFp8Batch)) * kSlotBytes;
                if (it % kFp8Batch == 0) ok = mbar_wait_warp(bar_sempty + 8 * s, ((batch / kRing) & 1u) ^ 1u, ctl, status_code(kRoleFp8Scale, 0, s));
                if (!ok) break;
                if constexpr (P_ROW) {
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const int32_t r = prow + i * 32 + static_cast<int32_t>(lane);
                        cp_async_4(slot + (i * 32 + lane) * 4u, r < t.p_end ? sp + r * p.sp_row : sp, r < t.p_end ? 4u : 0u);
                    }
                } else {
                    if (lane == 0) cp_async_4(slot, sp + (prow >> 7) * p.sp_row, 4u);
                }
                if constexpr (Q_COL) {
#pragma unroll
                    for (int i = 0; i < (BN + 31) / 32; ++i) {
                        const int32_t c = i * 32 + static_cast<int32_t>(lane), r = t.q0 + c;
                        if (BN >= 32 || c < BN) cp_async_4(slot + 512u + c * 4u, r < t.q_end ? sq + r * p.sq_row : sq, r < t.q_end ? 4u : 0u);
                    }
                } else {
                    const int32_t r = t.q0 + static_cast<int32_t>(lane) * 128;
                    if (lane < BN / 128) cp_async_4(slot + 512u + lane * 4u, r < t.q_end ? sq + (r >> 7) * p.sq_row : sq, r < t.q_end ? 4u : 0u);
                }
                if (it % kFp8Batch == kFp8Batch - 1) cp_async_mbar_arrive(bar_sfull + 8 * s);
            }
        }
        if (it % kFp8Batch != 0) cp_async_mbar_arrive(bar_sfull + 8 * ((it / kFp8Batch) % kRing));      // the last, partly filled batch
        cp_async_wait_all();
    } else if (warp == 3) {
        if constexpr (CG == 2) regs_lower<56>();
    } else {
        // ===== promotion (warps 4..11) =====
        if constexpr (CG == 2) regs_raise<224>();
        const uint32_t ew = warp - 4u, quarter = warp & 3u, half = ew >> 2;         // half: which BN / 2 accumulator columns
        const uint32_t taddr = tmem_base + ((quarter * 32u) << 16) + half * kCols;
        const uint32_t row_in_tile = quarter * 32u + lane;
        const uint32_t tempty = CG == 2 ? mapa(bar_tempty, 0) + half * 8u : bar_tempty, tfull = bar_tfull + (CG == 2 ? half * 8u : 0u);
        const uint32_t ring_end = ring_base + kRing * kFp8Batch * kSlotBytes;
        uint32_t it = 0;                                          // blocks so far (scales)
        uint32_t slot = ring_base;                                // the next block's scales
        uint32_t par = 0;                                         // bit d = phase of accumulator d's barriers
        bool ok = true;
        for (int32_t w = unit; ok && w < total; w += units) {
            const int32_t kbn = __shfl_sync(0xffffffffu, tile_of(w).kbn, 0);
            uint64_t acc[kCols / 2];
#pragma unroll
            for (int i = 0; i < kCols / 2; ++i) acc[i] = 0ull;
            // A block's scales -- the row's, and those of the first and the last 64 of a pair's columns -- are read one block
            // ahead, and its accumulator's barrier is asked ahead too, so that neither round trip lies between two accumulators.
            float row_s[Q_COL && P_ROW ? 4 : 1] = {}, col_s0 = 1.0f, col_s1 = 1.0f;
            uint32_t sq_next = 0;                                 // Q_COL: where this lane's column scales of the block that was read last begin
            bool ready = false;
            auto read_scales = [&](bool first) {
                const uint32_t batch = it / kFp8Batch;
                if (it % kFp8Batch == 0 || first) ok = mbar_wait_warp(bar_sfull + 8 * (batch % kRing), (batch / kRing) & 1u, ctl, status_code(kRoleFp8Promote, 0, 0));
                if constexpr (Q_COL) {
                    if constexpr (P_ROW) {
#pragma unroll
                        for (int i = 0; i < 4; ++i) row_s[i] = ld_shared_f32(slot + (quarter * 32u + 8u * i + (lane >> 2)) * 4u);
                    } else {
                        row_s[0] = ld_shared_f32(slot);
                    }
                    sq_next = slot + 512u + ((CG == 2 ? half * 64u : half * kCols) + (lane & 3u) * 2u) * 4u;
                } else {
                    row_s[0] = ld_shared_f32(slot + (P_ROW ? row_in_tile * 4u : 0u));
                    col_s0 = ld_shared_f32(slot + 512u);
                    col_s1 = ld_shared_f32(slot + 516u);
                }
                slot += kSlotBytes;
                if (slot == ring_end) slot = ring_base;
            };
            if (kbn > 0) read_scales(true);
            auto block = [&](auto dc, bool last) {                 // one block from accumulator dc
                constexpr uint32_t d = decltype(dc)::value, nd = (d + 1) % kDepth;
                [[maybe_unused]] const uint32_t sq = sq_next;
                // factors of this lane's values: of each row's (FRAG), or of the first and the last 64 columns
                uint64_t rows2[Q_COL ? (P_ROW ? 4 : 1) : 2];
                if constexpr (Q_COL) {
#pragma unroll
                    for (int i = 0; i < (P_ROW ? 4 : 1); ++i) rows2[i] = pack_f32x2(__float_as_uint(row_s[i]), __float_as_uint(row_s[i]));
                } else {
                    const float sc0 = row_s[0] * col_s0, sc1 = row_s[0] * col_s1;
                    rows2[0] = pack_f32x2(__float_as_uint(sc0), __float_as_uint(sc0));
                    rows2[1] = pack_f32x2(__float_as_uint(sc1), __float_as_uint(sc1));
                }
                const uint32_t batch_bar = bar_sempty + 8 * ((it / kFp8Batch) % kRing);
                const bool batch_end = it % kFp8Batch == kFp8Batch - 1;
                if (!Q_COL && batch_end) mbar_arrive_elect(batch_bar);        // the batch's last scales are in registers
                if (!__all_sync(0xffffffffu, ready)) ok = mbar_wait_warp(tfull + 8 * kParts * d, (par >> d) & 1u, ctl, status_code(kRoleFp8Promote, 1, d));
                if (!ok) return;
                par ^= 1u << d;
                ++it;
                tc_fence_after_sync();
                // Chunks of 16 registers, the next one in flight while one is added up.  One scale per row: a lane reads 16 columns of its
                // own row.  A scale per column: fragments of 16 rows x 8 columns, of which a lane holds two columns each; with
                // whole rows every lane would need every column's scale, and fetching those from shared memory (512 bytes a lane
                // and block) took twice the MMA's time.
                constexpr int kReps = kCols >= 32 ? 4 : kCols / 8;         // Q_COL: eights of columns of a chunk
                constexpr int kChunk = Q_COL ? 4 * kReps : 16, kChunks = 32 * kCols / (32 * kChunk);
                uint32_t v[2][kChunk];
                auto load = [&](int c) {
                    if constexpr (Q_COL) tmem_ld_16x256b(taddr + d * BN + (c / 2) * (8 * kReps) + ((c & 1) ? 16u << 16 : 0u), v[c & 1]);
                    else tmem_ld_32x32b_x16(taddr + d * BN + c * 16, v[c & 1]);
                };
                [[maybe_unused]] uint64_t qs[2][kReps];            // the column scales of a chunk's eights, one pair of chunks ahead
                auto load_q = [&](int g) {
                    if constexpr (Q_COL) {
#pragma unroll
                        for (int j = 0; j < kReps; ++j) {
                            const int col = (g * kReps + j) * 8;
                            qs[g & 1][j] = ld_shared_u64(sq + static_cast<uint32_t>(CG == 2 && col >= 64 ? col + 64 : col) * 4u);
                        }
                    }
                };
                load_q(0);
                load(0);
#pragma unroll
                for (int c = 0; c < kChunks; ++c) {
                    tmem_ld_wait_for(v[c & 1]);
                    if (c + 1 < kChunks) {
                        load(c + 1);
                        if (Q_COL && (c & 1) == 0 && c + 2 < kChunks) load_q(c / 2 + 1);
                    } else {
                        tc_fence_before_sync();                    // the accumulator is in registers: a later block may have it
                        if constexpr (CG == 2) mbar_arrive_cluster_elect(tempty + 8 * kParts * d);
                        else mbar_arrive_elect(tempty + 8 * kParts * d);
                        ready = false;
                        if (!last) {
                            read_scales(false);
                            ready = mbar_test_wait(tfull + 8 * kParts * nd, (par >> nd) & 1u);
                        }
                    }
                    const uint32_t *x = v[c & 1];
                    if constexpr (Q_COL) {
#pragma unroll
                        for (int j = 0; j < kReps; ++j) {
                            const uint64_t q = qs[(c / 2) & 1][j];
#pragma unroll
                            for (int i = 0; i < 2; ++i) {
                                uint64_t &a = acc[(c * kReps + j) * 2 + i];
                                a = fma_f32x2(pack_f32x2(x[4 * j + 2 * i], x[4 * j + 2 * i + 1]), mul_f32x2(q, rows2[P_ROW ? 2 * (c & 1) + i : 0]), a);
                            }
                        }
                    } else {
#pragma unroll
                        for (int i = 0; i < 16; i += 2) {
                            uint64_t &a = acc[(c * 16 + i) / 2];
                            a = fma_f32x2(pack_f32x2(x[i], x[i + 1]), rows2[c * 16 >= 64 ? 1 : 0], a);
                        }
                    }
                }
                if constexpr (Q_COL) {
                    __syncwarp();                                  // every lane has read this block's scales
                    if (batch_end) mbar_arrive_elect(batch_bar);
                }
            };
#pragma unroll 1
            for (int32_t kb = 0; ok && kb < kbn; kb += kDepth) {
                block(std::integral_constant<uint32_t, 0>(), kb + 1 == kbn);
                if (ok && kb + 1 < kbn) block(std::integral_constant<uint32_t, 1>(), kb + 2 == kbn);
                if constexpr (kDepth == 4) {
                    if (ok && kb + 2 < kbn) block(std::integral_constant<uint32_t, 2>(), kb + 3 == kbn);
                    if (ok && kb + 3 < kbn) block(std::integral_constant<uint32_t, 3>(), kb + 4 == kbn);
                }
            }
            const Fp8Tile t = tile_of(w);
            if (!ok) break;
            if constexpr (CG == 2) {
                const int32_t row0 = t.p0 + static_cast<int32_t>(rank * 128u + quarter * 32u), col0 = t.q0 + static_cast<int32_t>(half) * 64;
                const uint32_t staging = staging_base + ew * kFp8StagingPerWarp;
                if (p.out_type == 0) fp8_store_rows<float, Q_COL>(acc, staging, p, &tmap_c, t, row0, col0, lane);
                else if (p.out_type == 1) fp8_store_rows<__half, Q_COL>(acc, staging, p, &tmap_c, t, row0, col0, lane);
                else fp8_store_rows<__nv_bfloat16, Q_COL>(acc, staging, p, &tmap_c, t, row0, col0, lane);
            } else {
                constexpr int kReps = kCols >= 32 ? 4 : kCols / 8;
                if (p.split > 1) {
                    // this slice's part where the operand stages were (every MMA that read them is complete): columns of 128 rows,
                    // 132 words apart (conflict-free for fragments)
#pragma unroll
                    for (int f = 0; f < kCols / 8; ++f) {
#pragma unroll
                        for (int hi = 0; hi < 4; ++hi) {
                            float x, y;
                            unpack_f32x2(acc[fp8_frag_index<kReps>(f, hi)], x, y);
                            const uint32_t at = smem_base + ((half * kCols + 8u * f + (lane & 3u) * 2u) * kFp8PartPitch + quarter * 32u + 8u * hi + (lane >> 2)) * 4u;
                            st_shared_f32(at, x);
                            st_shared_f32(at + kFp8PartPitch * 4u, y);
                        }
                    }
                } else {
                    const int64_t base = t.group * p.c_group;
#pragma unroll
                    for (int f = 0; f < kCols / 8; ++f) {
#pragma unroll
                        for (int hi = 0; hi < 4; ++hi) {
                            float x, y;
                            unpack_f32x2(acc[fp8_frag_index<kReps>(f, hi)], x, y);
                            const int32_t row = t.p0 + static_cast<int32_t>(quarter * 32u + 8u * hi + (lane >> 2)), col = t.q0 + static_cast<int32_t>(half * kCols + 8u * f + (lane & 3u) * 2u);
                            if (row < t.p_end) {
#pragma unroll
                                for (int i = 0; i < 2; ++i) {
                                    if (col + i >= t.q_end) break;
                                    const int64_t at = base + static_cast<int64_t>(col + i) * p.ldc + row;
                                    const float v = i ? y : x;
                                    if (p.out_type == 0) fp8_store_one(static_cast<float *>(p.out) + at, v, p.accumulate);
                                    else if (p.out_type == 1) fp8_store_one(static_cast<__half *>(p.out) + at, v, 0);
                                    else fp8_store_one(static_cast<__nv_bfloat16 *>(p.out) + at, v, 0);
                                }
                            }
                        }
                    }
                }
            }
        }
    }

    if constexpr (CG == 2) bulk_wait_group<0>();              // the results are in memory
    // ---- sum over the slices of a tile (one tile per cluster: gridDim.x = split * tiles) --------------------------
    __syncwarp();
    if (CG == 1 && p.split > 1) {
        cluster_arrive();
        cluster_wait();
        if (unit < total && !*abort_flag) {
            const Fp8Tile t = fp8_tile<TP, TQ>(unit, p, pre, off, lane);
            const int32_t share = BN / p.split, row = t.p0 + static_cast<int32_t>(lane) * 4;
            for (int32_t c = static_cast<int32_t>(rank) * share + static_cast<int32_t>(warp); c < (static_cast<int32_t>(rank) + 1) * share; c += kFp8Threads / 32) {
                const int32_t col = t.q0 + c;
                if (col >= t.q_end) break;
                float v[4] = {0.0f, 0.0f, 0.0f, 0.0f};
                for (int32_t r = 0; r < p.split; ++r) {
                    const float4 x = ld_shared_cluster_v4(mapa(smem_base + (static_cast<uint32_t>(c) * kFp8PartPitch + lane * 4u) * 4u, static_cast<uint32_t>(r)));
                    v[0] += x.x; v[1] += x.y; v[2] += x.z; v[3] += x.w;
                }
                const int64_t at = t.group * p.c_group + static_cast<int64_t>(col) * p.ldc + row;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    if (row + i < t.p_end) {
                        if (p.out_type == 0) fp8_store_one(static_cast<float *>(p.out) + at + i, v[i], p.accumulate);
                        else if (p.out_type == 1) fp8_store_one(static_cast<__half *>(p.out) + at + i, v[i], 0);
                        else fp8_store_one(static_cast<__nv_bfloat16 *>(p.out) + at + i, v[i], 0);
                    }
                }
            }
        }
    }

    // ---- teardown (every thread, also after an abort) -----------------------------------------------------------------
    tc_fence_before_sync();
    __syncthreads();
    if (in_cluster) {                            // no CTA leaves while another may still signal it or read its shared memory
        cluster_arrive();
        cluster_wait();
    }
    if (warp == 1) {
        if (*abort_flag)
            for (int i = 0; i < 200; ++i) __nanosleep(1000);      // loads and MMAs in flight when a wait ran out
        tc_fence_after_sync();
        tmem_dealloc<CG>(tmem_base, kTmemCols);
    }
}

} // namespace hgemm_dev
