// The head in 32-bit floats, operands held as three bf16 arrays each.
#include "ends_head.h"

namespace deft {

hipError_t head_prepare_f32() { return allow_all<bf16, float, true>(); }

hipError_t head_loss_f32(const HeadPlan &plan, const deft_head_loss_t &a, void *scratch, int compute_units, hipStream_t st)
{
    return Head<float, bf16, 3>::loss(plan, a, Scratch(plan, scratch), compute_units, st);
}

hipError_t head_grad_f32(const HeadPlan &plan, const deft_head_grad_t &a, void *scratch, int compute_units, hipStream_t st)
{
    return Head<float, bf16, 3>::gradient(plan, a, Scratch(plan, scratch), compute_units, st);
}

}  // namespace deft
