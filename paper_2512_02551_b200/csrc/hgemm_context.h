// The library's context object, shared by the translation units that implement the C ABI.
#pragma once

#include <atomic>
#include <cuda.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include <vector>

#include "../../include/hgemm.h"

struct hgemm_fp8_plan_s;
struct hgemm_fp4_plan_s;

typedef CUresult (*encode_tiled_fn)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *,
                                    const cuuint64_t *, const cuuint32_t *, const cuuint32_t *, CUtensorMapInterleave,
                                    CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

// Device status words: one array per context.  Slot 0 belongs to the context itself (the timeout probe), every
// plan owns one of the others, so that a wait that ran out names the plan whose launch it was.
constexpr int kStatusSlots = 4096;

struct hgemm_ctx_s {
    int device = 0;
    int num_sms = 0;
    uint32_t *d_status = nullptr;          // kStatusSlots words
    std::vector<int> free_status_slots;    // slots no plan owns (never holds 0)
    int pass_allocs = 0, fail_allocs = 0;  // test hook: after pass_allocs more device allocations, fail_allocs of them report failure
    long long wait_budget = 2000000000LL;
    encode_tiled_fn encode = nullptr;
    int last_cuda_error = 0;
    bool dependent_launch = true;
    std::atomic<bool> few_ready{false};            // the few-token kernels' attributes are set: 4-bit weights
    std::atomic<bool> few16_ready[2] = {};         // fp16, bf16 weights
    bool tma_3d = true;
    std::vector<hgemm_plan_s *> plans;
    std::vector<hgemm_fp8_plan_s *> fp8_plans;
    std::vector<hgemm_fp4_plan_s *> fp4_plans;
    // hgemm_run_host: the operand copies and the result copy run on streams of their own (created by its first call), so that
    // one call's copies overlap the compute and the opposite-direction copy of the calls around it
    cudaStream_t copy_in = nullptr, copy_out = nullptr;
};

namespace hgemm_host {
int status_slot_of(const hgemm_fp8_plan_s *plan);   // the plan's word in the context's status array
int status_slot_of(const hgemm_fp4_plan_s *plan);
// What fp4_digits_product's kernels need once on a context's device.
hgemm_status_t fp4_digits_prepare(hgemm_ctx_s *ctx);
// C[i][n] (fp32) = sum of the products of the eight digit rows 8 i .. 8 i + 7 with row n of their group's matrix of B, i = the place of a choice among all, sorted by
// group; indices: the choices' groups (outside [0, groups): no row).  The kernel ahead in the stream makes the digits; everything else that is read is older: it is read
// before that kernel ends, so that one lets this one start only when all before it is complete.  Reports to the context's own status word.
hgemm_status_t fp4_digits_product(hgemm_ctx_s *ctx, int32_t format, int64_t choices, int64_t N, int64_t K, int32_t groups, const void *digits, int64_t ld, const void *digit_scales, const void *B,
                                  int64_t ldb, const void *b_scales, const float *b_factor, float *C, int64_t ldc, const int32_t *indices, void *stream);
// Synchronises the device, reads a status word and clears it: HGEMM_OK, or what the word stands for.
hgemm_status_t take_status_word(hgemm_ctx_s *ctx, int slot, uint32_t *code);
// One small kernel whose only wait is on a barrier that nothing signals; it reports to the slot.
hgemm_status_t launch_timeout_probe(hgemm_ctx_s *ctx, int slot, void *stream);
}

inline hgemm_status_t cuda_fail(hgemm_ctx_s *ctx, cudaError_t e)
{
    if (ctx) ctx->last_cuda_error = int(e);
    (void)cudaGetLastError();
    return HGEMM_ERR_CUDA;
}

// Every device allocation of the library goes through here (hgemm_debug_fail_allocs can make it fail).
inline cudaError_t ctx_malloc(hgemm_ctx_s *ctx, void **out, size_t bytes)
{
    if (ctx && ctx->fail_allocs > 0) {
        if (ctx->pass_allocs > 0) {
            --ctx->pass_allocs;
        } else {
            --ctx->fail_allocs;
            *out = nullptr;
            return cudaErrorMemoryAllocation;
        }
    }
    return cudaMalloc(out, bytes);
}
