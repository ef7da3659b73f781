// The 4-bit product with block scales: D = f * sum_b sP[., b] sQ[., b] (P_b Q_b^T), b = blocks of 16 or 32 of the contraction.
//
// The tensor cores apply the block scales themselves (tcgen05.mma kind::mxf4nvf4 / mxf4, K = 64), so a tile's whole contraction stays in one
// tensor-memory accumulator; what is left for the epilogue is the operands' tensor factors, the rounding and the store.  At this rate (four
// times the 16-bit one) a 256 x 256 pair tile takes 512 cycles of MMA per 256 of the contraction, in which each SM fetches 38 KB from L2.
//
// Both operands are K-major: two values to a byte along the contraction.  A stage of the ring is 256 elements: 128 bytes of every row (128-byte swizzle), and
// the scale tiles of those rows: 512 bytes for 128 rows x 4 scales, laid out in memory as tensor memory wants them, so that a
// tile goes there by one TMA box and one tcgen05.cp.  The copies and the MMAs are issued by one thread, which orders them.
//
// Roles (320 threads): warp 0 fills the ring by TMA; warp 1 copies the scales and issues the MMAs; warps 2..9 drain accumulators and store.
//
// Two shapes.  CTA pairs with 256 x 256 (or 256 x 128) tiles, stored by rows through a staging buffer: large problems.  Two accumulators of 256
// columns would leave no tensor memory for the scales, so the two share 128 columns: the epilogue drains those first, and the next tile's
// first MMA waits for that alone.  Single CTAs with 128 x {64, 128} tiles, for which P is the WEIGHT (its rows fill the 128 lanes however few
// tokens there are) and the tile is stored transposed; there the CTAs of a cluster may share one tile's contraction and add their parts
// through distributed shared memory in rank order.
//
// Products over groups: see product_tiles.cuh.  A group's scale tiles start at a tile boundary wherever its rows start.  Weight gradients contract
// over a group's rows, which the column copy pads with zeros to multiples of 128; a stage's second half is left out where the group ends.
//
// What it reaches (B200, bf16 results, nvfp4): 8192^3 225 us in calls one after the other, 4.9 PFLOP/s, and 192 in bursts of 24 launches, before the power cap takes hold;
// 1000 x 4096 x 4096 (mxfp4) 10.3 us, one round of 64 tiles, of which 5 are start and end; a gradient of 4096 x 2000 weights over 8000 rows 37-42 us (128 tiles on 74 pairs: two
// rounds for 1.7 rounds' work); 7 x 8192 x 4096 7.3 us and 512 rows over 64 experts (2048 x 2048 each) 28.5-30 us, 5.1-5.4 TB/s of weights.  At 8192^3 the tensor pipe is
// active 80 % of the time at 1.5 GHz; small calls are bound by their start and end, about 5 us; short contractions by the ends of their tiles (a gradient of 2048 x 2048 weights over
// 1024 rows for each of 32 experts, bf16: 83 us, 3 a tile of four stages, for which the tensor pipe needs 1.1).
//
// Every mbarrier wait is bounded (see hgemm_device.cuh): a wait that runs out raises the status word and the CTA's abort flag, and
// every role falls through to the common teardown.
#pragma once

#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <stdint.h>

#include "hgemm_device.cuh"
#include "product_tiles.cuh"

namespace hgemm_dev {

constexpr int kFp4Threads = 320;
constexpr int kFp4Stage = 256;                    // elements of the contraction in a stage
constexpr int kFp4Unit = 128;                     // the contraction is counted in these: a group's part is a multiple
constexpr int kFp4MaxStages = 10;
constexpr int kFp4MaxGroups = 1024;
constexpr int kFp4CtrlBytes = 512;
constexpr int kFp4Digits = 8;                     // rows of Q that stand for one (DIGITS)
constexpr int kFp4StagingPerWarp = 4096;          // results on their way out: a box of 32 rows x 128 bytes
constexpr uint32_t kRoleFp4Load = 12, kRoleFp4Mma = 13, kRoleFp4Store = 14;
constexpr uint32_t kFp4PartPitch = 132;           // words between the columns of a slice's part
constexpr uint32_t kFp4Overlap = 128;             // columns that the two accumulators of a 256-wide tile share

// Scale tiles of a stage for 128 rows, and shared memory of one stage.
__host__ __device__ constexpr int fp4_atoms(bool nv) { return nv ? 4 : 2; }
__host__ __device__ constexpr int fp4_scale_tiles(int bn) { return bn > 128 ? 2 : 1; }
__host__ __device__ constexpr int fp4_stage_bytes(int cta_group, int bn, bool nv)
{
    return 128 * 128 + bn / cta_group * 128 + fp4_atoms(nv) * 512 * (1 + fp4_scale_tiles(bn));
}

struct Fp4Params {
    int32_t rows_p, rows_q;        // rows of P and Q (per group, or all of them on the side that follows the offsets)
    int32_t kblocks;               // units of 128 of the contraction (not with kRaggedK)
    int32_t tiles_p, tiles_q;      // tiles per group (unused for the side that follows the offsets)
    int32_t total;                 // tiles, where the host knows them (kRaggedNone, kRaggedK)
    int32_t raster;                // tiles of P visited together
    FastDiv fd_other, fd_group, fd_sweep, fd_raster, fd_last;   // divisors of the tile numbering: see product_tile
    int32_t groups, ragged, rows_ragged, k_capacity;   // rows_ragged: clamp of the offsets; k_capacity: units the padded copy has
    const int32_t *offsets;
    const int32_t *indices;        // DIGITS: the group of each of `choices` rows of the caller's, instead of offsets
    int32_t choices;
    int32_t sp_group, sq_group;    // scale tiles (along the rows) between the matrices of an operand with one per group
    const float *fp, *fq;          // tensor factors (nullptr: 1), one, or one per group where f*_group is 1
    int32_t fp_group, fq_group;
    void *out;
    int64_t ldc, c_group;
    int32_t out_type, accumulate, vec_ok;   // out_type: 0 fp32, 1 fp16, 2 bf16; vec_ok: rows of C start and end at multiples of 16 bytes
    int32_t split, stages;
    uint32_t idesc;
    uint32_t *status;
    long long wait_budget;
};

// 32 rows x 128 bytes of results (columns col .. of C's rows row0 ..; v: this lane's row, fp32) to C.  Each lane packs its row into the staging box (16-byte pieces
// swizzled as TMA reads them: conflict-free), which leaves as a tensor store while the warp goes on.  A warp whose rows end inside its 32
// (a group's end) stores 16 bytes a lane; rows of C that are not multiples of 16 bytes, and C +=, take ordinary stores of 4 bytes a lane.
template <class T>
__device__ __forceinline__ void fp4_store_box(const uint32_t *v, float2 alpha, uint32_t staging, const Fp4Params &p, const CUtensorMap *tmap_c, const ProductTile &t, int32_t row0,
                                              int32_t col, uint32_t lane)
{
    constexpr int kSize = static_cast<int>(sizeof(T));
    const bool whole = p.vec_ok && !p.accumulate && (row0 + 32 <= t.p_end || t.p_end == p.rows_p);   // the map clips at the matrix's own end
    bulk_wait_group_read<0>();                                    // the earlier store has read the box
    __syncwarp();
    const uint32_t mine = staging + lane * 128u, swz = lane & 7u;
#pragma unroll
    for (uint32_t j = 0; j < 8; ++j) {
        uint32_t h[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if constexpr (kSize == 4) h[i] = __float_as_uint(__uint_as_float(v[4 * j + i]) * alpha.x * alpha.y);
            else h[i] = pack_pair(__uint_as_float(v[8 * j + 2 * i]) * alpha.x * alpha.y, __uint_as_float(v[8 * j + 2 * i + 1]) * alpha.x * alpha.y, T());
        }
        st_shared_v4(mine + ((j ^ swz) * 16u), h[0], h[1], h[2], h[3]);
    }
    if (whole) {
        fence_proxy_async_smem();
        __syncwarp();
        if (row0 < t.p_end && col < t.q_end) tma_store_3d_elect(tmap_c, col, row0, p.ragged == kRaggedK ? t.group : 0, staging);
        return;
    }
    __syncwarp();
    T *out = static_cast<T *>(p.out) + t.group * p.c_group;
    if (p.vec_ok && !p.accumulate) {
        const uint32_t k = lane & 7u;
        const int32_t at = col + static_cast<int32_t>(k) * (16 / kSize);
#pragma unroll
        for (uint32_t i = 0; i < 8; ++i) {
            const uint32_t r = 4u * i + (lane >> 3);
            const float4 x = ld_shared_v4(staging + r * 128u + ((k ^ (r & 7u)) * 16u));
            if (row0 + static_cast<int32_t>(r) < t.p_end && at < t.q_end)             // rows of C are multiples of 16 bytes: a piece is inside or outside
                *reinterpret_cast<float4 *>(out + static_cast<int64_t>(row0 + static_cast<int32_t>(r)) * p.ldc + at) = x;
        }
    } else if constexpr (kSize == 2) {
        // rows at any even address: two elements a lane where the pair starts at a multiple of 4 bytes.  In a run of 64 that does not, lane 0
        // takes its first and its last element.
        const int32_t left = t.q_end - col;                       // columns of the run
#pragma unroll 1
        for (int32_t i0 = 0; i0 < 32; i0 += 8) {                  // the loads of eight rows before their stores
            uint32_t h[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const int32_t i = i0 + j;
                const int32_t e = 2 * static_cast<int32_t>(lane) - (static_cast<int32_t>(reinterpret_cast<uintptr_t>(out + static_cast<int64_t>(row0 + i) * p.ldc + col) >> 1) & 1);
                const int32_t ea = e < 0 ? 0 : e, eb = e < 0 ? 63 : e + 1;
                const uint32_t from = staging + i * 128u;
                h[j] = ld_shared_u16(from + (((ea >> 3) ^ j) * 16u) + (ea & 7) * 2u) | static_cast<uint32_t>(ld_shared_u16(from + (((eb >> 3) ^ j) * 16u) + (eb & 7) * 2u)) << 16;
            }
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                if (row0 + i0 + j >= t.p_end) break;
                unsigned short *d = reinterpret_cast<unsigned short *>(out + static_cast<int64_t>(row0 + i0 + j) * p.ldc + col);
                const int32_t e = 2 * static_cast<int32_t>(lane) - (static_cast<int32_t>(reinterpret_cast<uintptr_t>(d) >> 1) & 1);
                if (e >= 0 && e + 1 < left) {
                    *reinterpret_cast<uint32_t *>(d + e) = h[j];
                } else {
                    if (max(e, 0) < left) d[max(e, 0)] = static_cast<unsigned short>(h[j]);
                    if (e < 0 && 63 < left) d[63] = static_cast<unsigned short>(h[j] >> 16);
                }
            }
        }
    } else {
#pragma unroll 1
        for (int32_t i0 = 0; i0 < 32; i0 += 8) {
            float x[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) x[j] = ld_shared_f32(staging + (i0 + j) * 128u + (((lane >> 2) ^ j) * 16u) + (lane & 3u) * 4u);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                if (row0 + i0 + j >= t.p_end) break;
                float *dst = reinterpret_cast<float *>(out) + static_cast<int64_t>(row0 + i0 + j) * p.ldc + col + static_cast<int32_t>(lane);
                if (col + static_cast<int32_t>(lane) < t.q_end) *dst = p.accumulate ? *dst + x[j] : x[j];
            }
        }
    }
}

// The operands' factors: 1 and their product, or, where that is no normal number of fp32 (the result may be one all the same: sums reach from 2^-20 to 2^43), the larger one
// and the smaller.  Sums are multiplied by one after the other.
__device__ __forceinline__ float2 fp4_factors(const Fp4Params &p, int32_t group)
{
    const float a = p.fp ? ld_older(p.fp + (p.fp_group ? group : 0)) : 1.0f, b = p.fq ? ld_older(p.fq + (p.fq_group ? group : 0)) : 1.0f, both = a * b;
    if (fabsf(both) >= 1.17549435e-38f && fabsf(both) <= 3.402823466e38f) return make_float2(1.0f, both);
    return fabsf(a) > fabsf(b) ? make_float2(a, b) : make_float2(b, a);
}

// One element of a result of type out_type.
__device__ __forceinline__ void fp4_store_one(const Fp4Params &p, int64_t at, float v)
{
    if (p.out_type == 0) {
        float *d = static_cast<float *>(p.out) + at;
        *d = p.accumulate ? *d + v : v;
    } else if (p.out_type == 1) {
        static_cast<__half *>(p.out)[at] = __float2half_rn(v);
    } else {
        static_cast<__nv_bfloat16 *>(p.out)[at] = __float2bfloat16_rn(v);
    }
}

// CG: CTAs per tile.  BN: rows of Q per tile.  NV: e4m3 scales of 16 elements, else powers of two of 32.  CG == 2 stores by rows, CG == 1 transposed.
// DIGITS (CG == 1): each eight rows of Q are one row of the caller's, written as a sum of eight; the result has their sums.  The kernel ahead in the stream makes those
// rows; P, its scales and factors and the rows' groups are older (that kernel starts this one when all before it is complete), and the first tile's P is fetched meanwhile.
template <int CG, int BN, bool NV, bool DIGITS = false>
__global__ void __launch_bounds__(kFp4Threads, 1)
fp4_product_kernel(const __grid_constant__ CUtensorMap tmap_p, const __grid_constant__ CUtensorMap tmap_q, const __grid_constant__ CUtensorMap tmap_sp,
                   const __grid_constant__ CUtensorMap tmap_sq, const __grid_constant__ CUtensorMap tmap_c, const Fp4Params p)
{
    constexpr int TP = 128 * CG, TQ = BN;
    constexpr int kDigits = DIGITS ? kFp4Digits : 1;
    constexpr bool kShared = 2 * BN > 384;                        // the accumulators share columns
    constexpr uint32_t kAccStep = kShared ? BN - kFp4Overlap : BN;
    constexpr uint32_t kScaleCol = 384;                           // tensor memory of the scales: two stages' worth
    constexpr int kAtoms = fp4_atoms(NV), kQTiles = fp4_scale_tiles(BN);
    constexpr uint32_t kScaleCols = 4 * kAtoms * (1 + kQTiles);   // of one stage
    constexpr uint32_t kPBytes = 128 * 128, kQBytes = BN / CG * 128, kSpBytes = kAtoms * 512, kSqBytes = kSpBytes * kQTiles;
    constexpr uint32_t kStageBytes = kPBytes + kQBytes + kSpBytes + kSqBytes;
    static_assert(kStageBytes == fp4_stage_bytes(CG, BN, NV), "the host counts the same bytes");
    static_assert(kScaleCol + 2 * kScaleCols <= 512 && kAccStep + BN <= kScaleCol, "tensor memory");
    // operands first, stage after stage (each a multiple of 1024 bytes: the swizzle), then the scales
    constexpr uint32_t kOperandBytes = kPBytes + kQBytes;

    extern __shared__ uint8_t smem_raw[];
    const uint32_t smem_base = (smem_addr(smem_raw) + 1023u) & ~1023u;
    uint8_t *smem_gen = smem_raw + (smem_base - smem_addr(smem_raw));
    const uint32_t scale_base = smem_base + static_cast<uint32_t>(p.stages) * kOperandBytes;
    const uint32_t staging_base = scale_base + static_cast<uint32_t>(p.stages) * (kSpBytes + kSqBytes);
    const uint32_t ctrl_base = staging_base + (CG == 2 ? 8u * kFp4StagingPerWarp : 0u);
    uint8_t *ctrl_gen = smem_gen + (ctrl_base - smem_base);
    const uint32_t bar_full = ctrl_base, bar_empty = bar_full + 8 * kFp4MaxStages, bar_tfull = bar_empty + 8 * kFp4MaxStages, bar_tempty = bar_tfull + 16;
    const uint32_t bar_early = bar_tempty + 16;                   // ends at 208
    volatile uint32_t *tmem_slot = reinterpret_cast<volatile uint32_t *>(ctrl_gen + 320);
    volatile uint32_t *abort_flag = reinterpret_cast<volatile uint32_t *>(ctrl_gen + 324);
    int32_t *pre = reinterpret_cast<int32_t *>(ctrl_gen + kFp4CtrlBytes);             // groups + 1 each
    int32_t *off = pre + (p.groups + 1), *scale_pre = off + (p.groups + 1);

    const uint32_t warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0);
    const uint32_t lane = lane_id();
    const bool in_cluster = CG == 2 || p.split > 1;
    const uint32_t rank = in_cluster ? cluster_ctarank() : 0u;    // place in the pair, or slice of the contraction
    const bool is_leader = CG == 1 || rank == 0;
    const int32_t per_unit = CG == 2 ? 2 : p.split;
    const int32_t unit = static_cast<int32_t>(blockIdx.x) / per_unit, units = static_cast<int32_t>(gridDim.x) / per_unit;
    WaitCtl ctl{abort_flag, p.status, p.wait_budget};

    int32_t mine = -1;                                            // a choice's group, on its way during the set-up
    if constexpr (DIGITS) {
        if (static_cast<int32_t>(threadIdx.x) < p.choices) mine = ld_older(p.indices + threadIdx.x);
    } else {
        grid_launch_dependents();
    }
    if (threadIdx.x == 0) {
        *abort_flag = 0u;
        for (int s = 0; s < p.stages; ++s) {
            mbar_init(bar_full + 8 * s, CG);
            mbar_init(bar_empty + 8 * s, 1);
        }
        for (int b = 0; b < 2; ++b) {
            mbar_init(bar_tfull + 8 * b, 1);
            mbar_init(bar_tempty + 8 * b, 8 * CG);
            mbar_init(bar_early + 8 * b, 8 * CG);
        }
        fence_mbar_init();
        prefetch_tensormap(&tmap_p);
        prefetch_tensormap(&tmap_q);
        prefetch_tensormap(&tmap_sp);
        prefetch_tensormap(&tmap_sq);
    }
    if (warp == 1) tmem_alloc<CG>(smem_addr(const_cast<uint32_t *>(tmem_slot)), 512);
    if constexpr (DIGITS) {
        // the groups' rows from the choices, then their places as below
        for (int32_t e = static_cast<int32_t>(threadIdx.x); e <= p.groups; e += kFp4Threads) off[e] = 0;
        __syncthreads();
        for (int32_t c = static_cast<int32_t>(threadIdx.x); c < p.choices; c += kFp4Threads) {
            const int32_t e = c < kFp4Threads ? mine : ld_older(p.indices + c);
            if (e >= 0 && e < p.groups) atomicAdd(&off[e + 1], kDigits);
        }
        __syncthreads();
        if (warp == 2) {
            int32_t carry = 0;
            for (int32_t base = 1; base <= p.groups; base += 32) {
                const int32_t e = base + static_cast<int32_t>(lane);
                int32_t n = e <= p.groups ? off[e] : 0;
#pragma unroll
                for (int d = 1; d < 32; d <<= 1) {
                    const int32_t x = __shfl_up_sync(0xffffffffu, n, d);
                    if (static_cast<int32_t>(lane) >= d) n += x;
                }
                n += carry;
                if (e <= p.groups) off[e] = n;
                carry = __shfl_sync(0xffffffffu, n, 31);
            }
            scan_groups<false>(p, pre, off, TQ, lane, scale_pre, 128);
        }
    } else {
        // No thread reads or writes global memory before the kernels ahead in the stream are complete.
        grid_dependency_wait();
        if (warp == 2 && p.groups > 0) {
            // the groups' places among the result's tiles, and among the scale tiles
            scan_groups(p, pre, off, p.ragged == kRaggedK ? kFp4Unit : p.ragged == kRaggedP ? TP : TQ, lane, scale_pre, 128);
        }
    }
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
        ProductTile t = product_tile<TP, TQ>(w, p, pre, off, lane);
        if (CG == 1 && p.split > 1) {                              // this CTA's share of the contraction
            const int32_t b = t.kbn * static_cast<int32_t>(rank) / p.split, e = t.kbn * (static_cast<int32_t>(rank) + 1) / p.split;
            t.kb0 += b;
            t.kbn = e - b;
        }
        return t;
    };
    // where a tile's rows of Q begin, counted from the first row of a scale tile
    auto q_from = [&](const ProductTile &t) { return p.ragged == kRaggedQ ? t.q0 - off[t.group] : t.q0; };

    if (warp == 0) {
        // ===== operands and their scales =====
        int s = 0;
        uint32_t ph = 0;
        const uint32_t full_leader = CG == 2 ? mapa(bar_full, 0) : bar_full;
        bool ok = true;
        int32_t ahead = 0;                                        // contracted elements of the first tile whose P is on its way, in units
        if constexpr (DIGITS) {
            if (unit < total) {
                const ProductTile t = tile_of(unit);
                ahead = min(t.kbn, 2 * p.stages);
                fence_proxy_async_all();
                for (int32_t kb = 0; kb < ahead; kb += 2) {
                    const uint32_t fb = bar_full + 4 * kb, p_dst = smem_base + static_cast<uint32_t>(kb / 2) * kOperandBytes, sp_dst = scale_base + static_cast<uint32_t>(kb / 2) * (kSpBytes + kSqBytes);
                    mbar_arrive_expect_tx_elect(fb, kStageBytes);
                    tma_load_3d_elect(p_dst, &tmap_p, (t.kb0 + kb) * (kFp4Unit / 2), t.p0, t.group, fb);
                    tma_load_3d_elect(sp_dst, &tmap_sp, 0, (t.kb0 + kb) * (kAtoms / 2), t.group * p.sp_group + (t.p0 >> 7), fb);
                }
            }
            grid_dependency_wait();                               // in every CTA, with a tile or without: this kernel's end says that the one ahead has ended
            grid_launch_dependents();                             // and its results may be read by the next from here on
        }
        for (int32_t w = unit; ok && w < total; w += units) {
            const ProductTile t = tile_of(w);
            const int32_t prow = t.p0 + static_cast<int32_t>(CG == 2 ? rank : 0u) * 128, qrow = t.q0 + static_cast<int32_t>(CG == 2 ? rank : 0u) * (BN / CG);
            const int32_t pz = p.ragged == kRaggedQ ? t.group : 0, qz = p.ragged == kRaggedP ? t.group : 0;      // the operand with one matrix per group
            const int32_t sp = p.ragged == kRaggedP ? scale_pre[t.group] + ((prow - off[t.group]) >> 7) : pz * p.sp_group + (prow >> 7);
            const int32_t sq = (p.ragged == kRaggedQ ? scale_pre[t.group] : qz * p.sq_group) + (q_from(t) >> 7);
            for (int32_t kb = 0; kb < t.kbn; kb += 2) {
                ok = mbar_wait_warp(bar_empty + 8 * s, ph ^ 1u, ctl, status_code(kRoleFp4Load, 0, s));
                if (!ok) break;
                const uint32_t p_dst = smem_base + static_cast<uint32_t>(s) * kOperandBytes, q_dst = p_dst + kPBytes;
                const uint32_t sp_dst = scale_base + static_cast<uint32_t>(s) * (kSpBytes + kSqBytes), sq_dst = sp_dst + kSpBytes;
                const int32_t k0 = (t.kb0 + kb) * (kFp4Unit / 2), a0 = (t.kb0 + kb) * (kAtoms / 2);
                const uint32_t fb = full_leader + 8 * s;
                if constexpr (CG == 1) {
                    if (!DIGITS || w != unit || kb >= ahead) {
                        mbar_arrive_expect_tx_elect(bar_full + 8 * s, kStageBytes);
                        tma_load_3d_elect(p_dst, &tmap_p, k0, prow, pz, fb);
                        tma_load_3d_elect(sp_dst, &tmap_sp, 0, a0, sp, fb);
                    }
                    tma_load_3d_elect(q_dst, &tmap_q, k0, qrow, qz, fb);
                    tma_load_3d_elect(sq_dst, &tmap_sq, 0, a0, sq, fb);
                } else {
                    if (is_leader) mbar_arrive_expect_tx_elect(bar_full + 8 * s, kStageBytes);
                    else mbar_arrive_expect_tx_cluster_relaxed_elect(fb, kStageBytes);
                    tma_load_3d_pair_elect(p_dst, &tmap_p, k0, prow, pz, fb);
                    tma_load_3d_pair_elect(q_dst, &tmap_q, k0, qrow, qz, fb);
                    tma_load_3d_pair_elect(sp_dst, &tmap_sp, 0, a0, sp, fb);
                    tma_load_3d_pair_elect(sq_dst, &tmap_sq, 0, a0, sq, fb);          // each CTA's tensor memory has the scales of all of Q's rows
                }
                if (++s == p.stages) { s = 0; ph ^= 1u; }
            }
        }
        // Every commit that signals this CTA's stage barriers (the pair's leader signals both CTAs') arrives before the CTA may leave:
        // the storing warps wait for the accumulators' barriers only.
        for (int i = 0; ok && i < p.stages; ++i) {
            ok = mbar_wait_warp(bar_empty + 8 * s, ph ^ 1u, ctl, status_code(kRoleFp4Load, 1, s));
            if (++s == p.stages) { s = 0; ph ^= 1u; }
        }
    } else if (warp == 1) {
        // ===== scales to tensor memory, MMAs =====
        if (is_leader) {
            int s = 0;
            uint32_t ph = 0, n = 0;                               // n: tiles so far (those with a contraction)
            bool ok = true;
            uint32_t parity = 0;                                  // which half of the scales' columns the stage takes
            const uint64_t desc_p0 = make_smem_desc_sw128(smem_base), desc_q0 = make_smem_desc_sw128(smem_base + kPBytes), desc_s0 = make_smem_desc_rows16(scale_base);
            for (int32_t w = unit; ok && w < total; w += units) {
                const ProductTile t = tile_of(w);
                const int32_t kbn = __shfl_sync(0xffffffffu, t.kbn, 0);
                if (kbn == 0) continue;
                const uint32_t shift = kQTiles == 1 ? __shfl_sync(0xffffffffu, static_cast<uint32_t>(q_from(t) & 127) >> 5, 0) : 0u;
                const uint32_t d = n & 1u, use = n >> 1;
                ok = mbar_wait_warp(bar_tempty + 8 * d, (use & 1u) ^ 1u, ctl, status_code(kRoleFp4Mma, 1, d));
                if (kShared && ok && n > 0) ok = mbar_wait_warp(bar_early + 8 * (d ^ 1u), ((n - 1) >> 1) & 1u, ctl, status_code(kRoleFp4Mma, 2, d));
                const uint32_t acc = tmem_base + d * kAccStep;
                for (int32_t kb = 0; ok && kb < kbn; kb += 2) {
                    ok = mbar_wait_warp(bar_full + 8 * s, ph, ctl, status_code(kRoleFp4Mma, 0, s));
                    if (!ok) break;
                    tc_fence_after_sync();
                    const uint64_t dp = desc_p0 + static_cast<uint64_t>((static_cast<uint32_t>(s) * kOperandBytes) >> 4), dq = desc_q0 + static_cast<uint64_t>((static_cast<uint32_t>(s) * kOperandBytes) >> 4);
                    const uint64_t ds = desc_s0 + static_cast<uint64_t>((static_cast<uint32_t>(s) * (kSpBytes + kSqBytes)) >> 4);
                    const uint32_t sa = tmem_base + kScaleCol + parity * kScaleCols, sb = sa + 4 * kAtoms;
#pragma unroll
                    for (uint32_t j = 0; j < kAtoms; ++j) {
                        tmem_copy_scales_elect<CG>(sa + 4 * j, ds + j * 32);
#pragma unroll
                        for (uint32_t q = 0; q < kQTiles; ++q) tmem_copy_scales_elect<CG>(sb + 4 * (j * kQTiles + q), ds + (kSpBytes >> 4) + (q * kAtoms + j) * 32);
                    }
                    const bool both = kb + 1 < kbn;               // the stage's second half is part of the contraction
#pragma unroll
                    for (uint32_t k = 0; k < 4; ++k) {
                        if (k < 2 || both) {
                            const uint32_t a = NV ? k : k / 2, id = NV ? 0u : (k & 1u) * 2u;
                            umma_f4_elect<CG, NV>(acc, dp + k * 2, dq + k * 2, p.idesc | (id << 4) | (id << 29), sa + 4 * a, sb + 4 * kQTiles * a + shift, kb > 0 || k > 0);
                        }
                    }
                    parity ^= 1u;
                    if constexpr (CG == 2) umma_commit_both_elect(bar_empty + 8 * s);
                    else umma_commit_elect<1>(bar_empty + 8 * s, 0);
                    if (++s == p.stages) { s = 0; ph ^= 1u; }
                }
                if (!ok) break;
                if constexpr (CG == 2) umma_commit_both_elect(bar_tfull + 8 * d);
                else umma_commit_elect<1>(bar_tfull + 8 * d, 0);
                ++n;
            }
        }
    } else {
        // ===== results (warps 2..9) =====
        const uint32_t ew = warp - 2u, quarter = warp & 3u, half = ew >> 2;
        const uint32_t tempty = CG == 2 ? mapa(bar_tempty, 0) : bar_tempty, early = CG == 2 ? mapa(bar_early, 0) : bar_early;
        const uint32_t staging = staging_base + ew * kFp4StagingPerWarp;
        uint32_t n = 0;
        for (int32_t w = unit; w < total; w += units) {
            const ProductTile t = tile_of(w);
            const int32_t kbn = __shfl_sync(0xffffffffu, t.kbn, 0);
            const float2 alpha = fp4_factors(p, t.group);
            const uint32_t d = n & 1u;
            if (kbn > 0) {
                if (!mbar_wait_warp(bar_tfull + 8 * d, (n >> 1) & 1u, ctl, status_code(kRoleFp4Store, 0, d))) break;
                tc_fence_after_sync();
                if (DIGITS && n == 0) grid_dependency_wait();     // before the first store; the kernel ahead is complete (it made what this tile was computed from)
                ++n;
            }
            const uint32_t taddr = tmem_base + ((quarter * 32u) << 16) + d * kAccStep;
            if constexpr (CG == 2) {
                const int32_t row0 = t.p0 + static_cast<int32_t>(rank * 128u + quarter * 32u);
                constexpr int kMine = BN / 128;                   // chunks of 64 columns of this warp; those that the accumulators share come first
#pragma unroll
                for (int i = 0; i < kMine; ++i) {
                    const uint32_t chunk = (kMine == 2 ? (d ? i : 1 - i) * 2 : 0) + half;
                    uint32_t v[64];
                    if (kbn > 0) {
#pragma unroll
                        for (int j = 0; j < 4; ++j) tmem_ld_32x32b_x16(taddr + chunk * 64 + j * 16, v + 16 * j);
#pragma unroll
                        for (int j = 0; j < 4; ++j) tmem_ld_wait_for(*reinterpret_cast<uint32_t(*)[16]>(v + 16 * j));
                        tc_fence_before_sync();
                        if (kShared && i == 0) mbar_arrive_cluster_elect(early + 8 * d);
                        if (i == kMine - 1) mbar_arrive_cluster_elect(tempty + 8 * d);
                    } else {
#pragma unroll
                        for (int j = 0; j < 64; ++j) v[j] = 0u;
                    }
                    const int32_t col = t.q0 + static_cast<int32_t>(chunk) * 64;
                    if (p.out_type == 0) {
                        fp4_store_box<float>(v, alpha, staging, p, &tmap_c, t, row0, col, lane);
                        fp4_store_box<float>(v + 32, alpha, staging, p, &tmap_c, t, row0, col + 32, lane);
                    } else if (p.out_type == 1) {
                        fp4_store_box<__half>(v, alpha, staging, p, &tmap_c, t, row0, col, lane);
                    } else {
                        fp4_store_box<__nv_bfloat16>(v, alpha, staging, p, &tmap_c, t, row0, col, lane);
                    }
                }
            } else {
                constexpr int kCols = BN / 2, kOut = kCols / kDigits;
                uint32_t v[kCols];
                if (kbn > 0) {
#pragma unroll
                    for (int j = 0; j < kCols / 16; ++j) tmem_ld_32x32b_x16(taddr + half * kCols + j * 16, v + 16 * j);
#pragma unroll
                    for (int j = 0; j < kCols / 16; ++j) tmem_ld_wait_for(*reinterpret_cast<uint32_t(*)[16]>(v + 16 * j));
                    tc_fence_before_sync();
                    mbar_arrive_elect(tempty + 8 * d);
                } else {
#pragma unroll
                    for (int j = 0; j < kCols; ++j) v[j] = 0u;
                }
                float o[kOut];
#pragma unroll
                for (int j = 0; j < kOut; ++j) {
                    o[j] = __uint_as_float(v[j * kDigits]);
#pragma unroll
                    for (int i = 1; i < kDigits; ++i) o[j] += __uint_as_float(v[j * kDigits + i]);
                    o[j] = o[j] * alpha.x * alpha.y;
                }
                if (p.split > 1) {
                    // this slice's part where the operand stages were (every MMA that read them is complete): columns of 128 rows, 132 words apart
#pragma unroll
                    for (int j = 0; j < kOut; ++j) st_shared_f32(smem_base + ((half * kOut + j) * kFp4PartPitch + quarter * 32u + lane) * 4u, o[j]);
                } else {
                    const int32_t row = t.p0 + static_cast<int32_t>(quarter * 32u + lane);
                    const int64_t base = t.group * p.c_group + row;
                    if (row < t.p_end) {
#pragma unroll
                        for (int j = 0; j < kOut; ++j) {
                            const int32_t col = t.q0 / kDigits + static_cast<int32_t>(half * kOut) + j;
                            if (col < t.q_end / kDigits) fp4_store_one(p, base + static_cast<int64_t>(col) * p.ldc, o[j]);
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
        if constexpr (DIGITS) grid_dependency_wait();             // (as above)
        cluster_arrive();
        cluster_wait();
        if (unit < total && !*abort_flag) {
            const ProductTile t = product_tile<TP, TQ>(unit, p, pre, off, lane);
            const int32_t share = BN / kDigits / p.split, row = t.p0 + static_cast<int32_t>(lane) * 4;
            for (int32_t c = static_cast<int32_t>(rank) * share + static_cast<int32_t>(warp); c < (static_cast<int32_t>(rank) + 1) * share; c += kFp4Threads / 32) {
                const int32_t col = t.q0 / kDigits + c;
                if (col >= t.q_end / kDigits) break;
                float v[4] = {0.0f, 0.0f, 0.0f, 0.0f};
                for (int32_t r = 0; r < p.split; ++r) {
                    const float4 x = ld_shared_cluster_v4(mapa(smem_base + (static_cast<uint32_t>(c) * kFp4PartPitch + lane * 4u) * 4u, static_cast<uint32_t>(r)));
                    v[0] += x.x; v[1] += x.y; v[2] += x.z; v[3] += x.w;
                }
                const int64_t at = t.group * p.c_group + static_cast<int64_t>(col) * p.ldc + row;
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (row + i < t.p_end) fp4_store_one(p, at + i, v[i]);
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
        tmem_dealloc<CG>(tmem_base, 512);
    }
}

} // namespace hgemm_dev
