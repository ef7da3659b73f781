// Device code that the kernels share: division by run-time constants, bounded waits on mbarriers with a status word, and the shared-memory matrix
// descriptors of tiles that TMA lays out with the 128-byte swizzle.
#pragma once

#include <stdint.h>

#include "ptx_sm100.cuh"

namespace hgemm_dev {

using namespace hgemm_ptx;

// x / d for x < 2^31 without a division instruction: q = umulhi(x, mul) >> shr (d == 1: q = x).
// mul = ceil(2^(31 + ceil(log2 d)) / d), shr = ceil(log2 d) - 1.
struct FastDiv {
    uint32_t mul, shr, d;
};

__host__ __device__ inline FastDiv make_fast_div(uint32_t d)
{
    FastDiv f;
    f.d = d < 1u ? 1u : d;
    f.mul = 0u;
    f.shr = 0u;
    if (f.d > 1u) {
        uint32_t lg = 0;
        while ((1ull << lg) < f.d) ++lg;                                 // ceil(log2 d) >= 1
        const unsigned long long pw = 1ull << (31u + lg);
        f.mul = static_cast<uint32_t>((pw + f.d - 1u) / f.d);
        f.shr = lg - 1u;
    }
    return f;
}

__host__ __device__ __forceinline__ int32_t fast_div(int32_t x, const FastDiv &f)
{
#ifdef __CUDA_ARCH__
    return f.d == 1u ? x : static_cast<int32_t>(__umulhi(static_cast<uint32_t>(x), f.mul) >> f.shr);
#else
    return static_cast<int32_t>(static_cast<uint32_t>(x) / f.d);      // the host's copy (layout computations, tests)
#endif
}

// -------------------------------------------------------------------------------------
// bounded wait

struct WaitCtl {
    volatile uint32_t *abort_flag;  // shared memory
    uint32_t *status;               // global memory
    long long budget;
};

static __device__ __noinline__ bool mbar_wait_slow(uint32_t bar, uint32_t parity, const WaitCtl &ctl, uint32_t code)
{
    const long long t0 = clock64();
#pragma unroll 1
    while (true) {
        if (mbar_try_wait(bar, parity)) return true;
        if (*ctl.abort_flag) return false;
        if (clock64() - t0 > ctl.budget) {
            *ctl.abort_flag = 1u;
            atomicCAS(ctl.status, 0u, code);
            return false;
        }
    }
}

__device__ __forceinline__ bool mbar_wait(uint32_t bar, uint32_t parity, const WaitCtl &ctl, uint32_t code)
{
    if (mbar_test_wait(bar, parity)) return true;      // already complete: the cheap query answers
#pragma unroll 1
    for (int i = 0; i < 16; ++i)
        if (mbar_try_wait(bar, parity)) return true;
    return mbar_wait_slow(bar, parity, ctl, code);
}

constexpr uint32_t kWaitSuspendNs = 20000;     // a suspended warp leaves its scheduler to the others; the budget is looked at this often

// The same wait for a converged warp, without a call (for code that keeps most of its registers live across it); the result is
// the same in every lane.
__device__ __forceinline__ bool mbar_wait_warp(uint32_t bar, uint32_t parity, const WaitCtl &ctl, uint32_t code)
{
    if (__all_sync(0xffffffffu, mbar_try_wait_for(bar, parity, kWaitSuspendNs))) return true;
    const long long t0 = clock64();
#pragma unroll 1
    while (!__all_sync(0xffffffffu, mbar_try_wait_for(bar, parity, kWaitSuspendNs))) {
        const bool late = clock64() - t0 > ctl.budget;
        if (__any_sync(0xffffffffu, late || *ctl.abort_flag != 0u)) {
            if (late && *ctl.abort_flag == 0u) {
                *ctl.abort_flag = 1u;
                atomicCAS(ctl.status, 0u, code);
            }
            __syncwarp();
            return false;
        }
    }
    return true;
}

__device__ __forceinline__ uint32_t status_code(uint32_t role, uint32_t barrier_index, uint32_t stage)
{
    return (role << 24) | ((barrier_index & 0xffffu) << 8) | (stage & 0xffu);
}

// -------------------------------------------------------------------------------------
// descriptors

// Shared-memory matrix descriptor of a K-major tile whose rows are 64 fp16 = 128 bytes,
// laid out by TMA with the 128-byte swizzle: 8-row groups are 1024 bytes apart.
__device__ __forceinline__ uint64_t make_smem_desc_sw128(uint32_t smem_byte_addr)
{
    uint64_t d = 0;
    d |= static_cast<uint64_t>((smem_byte_addr & 0x3ffffu) >> 4);        // [0,14)  start address >> 4
    d |= static_cast<uint64_t>(1) << 16;                                 // [16,30) leading byte offset (unused here)
    d |= static_cast<uint64_t>(1024 >> 4) << 32;                         // [32,46) stride byte offset: 8 rows * 128 B
    d |= static_cast<uint64_t>(1) << 46;                                 // [46,48) descriptor version (sm_100)
    d |= static_cast<uint64_t>(2) << 61;                                 // [61,64) 128-byte swizzle
    return d;
}

// The same for a tile that is contiguous along its M/N dimension (a row-major K x N operand): the tile
// is stored as blocks of 64 columns, each block 64 k-rows of 128 bytes under the 128-byte swizzle.
// Leading byte offset = distance between 64-column blocks, stride byte offset = distance between
// groups of 8 k-rows (1024 bytes); one UMMA (K = 16) spans two such groups.
__device__ __forceinline__ uint64_t make_smem_desc_sw128_mn_major(uint32_t smem_byte_addr, uint32_t block_bytes)
{
    uint64_t d = 0;
    d |= static_cast<uint64_t>((smem_byte_addr & 0x3ffffu) >> 4);
    d |= static_cast<uint64_t>((block_bytes >> 4) & 0x3fffu) << 16;
    d |= static_cast<uint64_t>(1024 >> 4) << 32;
    d |= static_cast<uint64_t>(1) << 46;
    d |= static_cast<uint64_t>(2) << 61;
    return d;
}

// Shared-memory matrix descriptor of 32 rows of 16 bytes that follow one another (no swizzle): groups of 8 rows are 128 bytes apart.
__device__ __forceinline__ uint64_t make_smem_desc_rows16(uint32_t smem_byte_addr)
{
    uint64_t d = 0;
    d |= static_cast<uint64_t>((smem_byte_addr & 0x3ffffu) >> 4);
    d |= static_cast<uint64_t>(128 >> 4) << 16;
    d |= static_cast<uint64_t>(128 >> 4) << 32;
    d |= static_cast<uint64_t>(1) << 46;
    return d;
}

} // namespace hgemm_dev
