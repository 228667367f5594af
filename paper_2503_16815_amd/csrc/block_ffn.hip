// The feed-forward block's scratch memory, and its calls by type (each type's kernels are a file of their own).
#include "block_epilogue.h"
#include "ends_shapes.h"

namespace deft {
namespace {

// The largest finite magnitude of the pieces of eight that a workgroup has.
__global__ void __launch_bounds__(256) largest_kernel(LargestArgs a)
{
    __shared__ float of_wave[4];
    float top = 0.0f;
    for (unsigned block = blockIdx.x;; block += kFactorParts) {
        if (block >= a.by.blocks()) break;
        int row, piece;
        if (!a.by.own(block, &row, &piece)) continue;
        const int at = piece * kEight;
        const Eight<f16>::type x = load_eight<false>(a.x + row * a.x_stride + at, at, a.cols);
#pragma unroll
        for (int r = 0; r < kEight; ++r) top = fmaxf(top, is_finite((float)x[r]) ? fabsf((float)x[r]) : 0.0f);
    }
    top = wave_max(top);
    if ((threadIdx.x & 63) == 0) of_wave[threadIdx.x >> 6] = top;
    __syncthreads();
    if (threadIdx.x == 0) a.largest[blockIdx.x] = fmaxf(fmaxf(of_wave[0], of_wave[1]), fmaxf(of_wave[2], of_wave[3]));
}

}  // namespace

hipError_t ffn_largest_launch(const LargestArgs &a, hipStream_t st)
{
    largest_kernel<<<kFactorParts, 256, 0, st>>>(a);
    return hipGetLastError();
}

#define DEFT_FFN_TYPE(NAME)                                                             \
    hipError_t ffn_prepare_##NAME();                                                    \
    hipError_t ffn_##NAME(const FfnPlan &, const deft_ffn_t &, void *, int, hipStream_t); \
    hipError_t ffn_grad_##NAME(const FfnPlan &, const deft_ffn_grad_t &, void *, int, hipStream_t);
DEFT_FFN_TYPE(bf16)
DEFT_FFN_TYPE(f16)
DEFT_FFN_TYPE(f32)

void ffn_plan(int dtype, int max_rows, int max_hidden, int max_inner, bool grad, int compute_units, FfnPlan *plan)
{
    const int64_t n = up(max_rows, kTile), hidden = up(max_hidden, kTile), inner = up(max_inner, kTile);
    int64_t at = 0;
    const auto take = [&](int64_t bytes) {
        const int64_t here = at;
        at += up(bytes, 256);
        return here;
    };
    const int64_t element = dtype == DEFT_F32 ? 6 : 2, own = dtype == DEFT_F32 ? 4 : 2;   // of an operand (three 16-bit arrays), of the type
    if (!grad && max_rows <= few_rows(dtype == DEFT_F32, (int64_t)max_hidden * max_inner, true)) {   // (the kernels for few alone: two arrays of h)
        plan->h = take(2 * kFew * up(max_inner, 8) * own);
        plan->scratch_bytes = at;
        return;
    }
    plan->largest = take(kFactorParts * 4);
    // (whether a call's rows can be read in place is known when it is made)
    plan->x = take(n * up(max_hidden, kStep) * element);
    plan->w_gate = take(inner * up(max_hidden, kStep) * element);
    plan->w_up = take(inner * up(max_hidden, kStep) * element);
    plan->w_down = take(hidden * up(max_inner, kStep) * element);
    plan->h = take(n * inner * element);
    int64_t most = n * (2 * inner > hidden ? 2 * inner : hidden);   // sums of one part
    if (grad) {
        plan->grad_y = take(n * up(max_hidden, kStep) * element);
        plan->d = take(2 * n * inner * element);
        const int64_t kept = n * up(max_inner, kStep) * own + n * (up(max_inner, kStep) / kGroup) * 2;   // and scales
        plan->gate = take(kept);
        plan->up = take(kept);
        most = most > 2 * inner * hidden ? most : 2 * inner * hidden;
    }
    // parts of sums: parts * tiles stays within twice the compute units
    const int64_t tiles = 2 * (int64_t)compute_units * kTile * kTile;
    plan->sums = take((tiles < most * kMaxSplits ? tiles : most * kMaxSplits) * 4);
    plan->scratch_bytes = at;
}

hipError_t ffn_prepare()
{
    hipError_t e = ffn_prepare_bf16();
    if (e == hipSuccess) e = ffn_prepare_f16();
    if (e == hipSuccess) e = ffn_prepare_f32();
    return e;
}

hipError_t ffn_launch(const FfnPlan &plan, int dtype, const deft_ffn_t &a, void *scratch, int compute_units, hipStream_t st)
{
    if (dtype == DEFT_F32) return ffn_f32(plan, a, scratch, compute_units, st);
    if (dtype == DEFT_F16) return ffn_f16(plan, a, scratch, compute_units, st);
    return ffn_bf16(plan, a, scratch, compute_units, st);
}

hipError_t ffn_grad_launch(const FfnPlan &plan, int dtype, const deft_ffn_grad_t &a, void *scratch, int compute_units, hipStream_t st)
{
    if (dtype == DEFT_F32) return ffn_grad_f32(plan, a, scratch, compute_units, st);
    if (dtype == DEFT_F16) return ffn_grad_f16(plan, a, scratch, compute_units, st);
    return ffn_grad_bf16(plan, a, scratch, compute_units, st);
}

}  // namespace deft
