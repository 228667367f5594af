// The feed-forward block in f32.
#include "block_ffn.h"

namespace deft {

hipError_t ffn_prepare_f32() { return Ffn<float, bf16, 3>::prepare(); }

hipError_t ffn_f32(const FfnPlan &plan, const deft_ffn_t &a, void *scratch, int compute_units, hipStream_t st)
{
    return Ffn<float, bf16, 3>::forward(a, FfnScratch(plan, scratch), compute_units, st);
}

hipError_t ffn_grad_f32(const FfnPlan &plan, const deft_ffn_grad_t &a, void *scratch, int compute_units, hipStream_t st)
{
    return Ffn<float, bf16, 3>::backward(a, FfnScratch(plan, scratch), compute_units, st);
}

}  // namespace deft
