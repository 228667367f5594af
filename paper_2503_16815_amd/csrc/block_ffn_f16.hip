// The feed-forward block in f16.
#include "block_ffn.h"

namespace deft {

hipError_t ffn_prepare_f16() { return Ffn<f16, f16, 1>::prepare(); }

hipError_t ffn_f16(const FfnPlan &plan, const deft_ffn_t &a, void *scratch, int compute_units, hipStream_t st)
{
    return Ffn<f16, f16, 1>::forward(a, FfnScratch(plan, scratch), compute_units, st);
}

hipError_t ffn_grad_f16(const FfnPlan &plan, const deft_ffn_grad_t &a, void *scratch, int compute_units, hipStream_t st)
{
    return Ffn<f16, f16, 1>::backward(a, FfnScratch(plan, scratch), compute_units, st);
}

}  // namespace deft
