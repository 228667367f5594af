// The head in bf16.
#include "ends_head.h"

namespace deft {

hipError_t head_prepare_bf16() { return allow_all<bf16, bf16, false>(); }

hipError_t head_loss_bf16(const HeadPlan &plan, const deft_head_loss_t &a, void *scratch, int compute_units, hipStream_t st)
{
    return Head<bf16, bf16, 1>::loss(plan, a, Scratch(plan, scratch), compute_units, st);
}

hipError_t head_grad_bf16(const HeadPlan &plan, const deft_head_grad_t &a, void *scratch, int compute_units, hipStream_t st)
{
    return Head<bf16, bf16, 1>::gradient(plan, a, Scratch(plan, scratch), compute_units, st);
}

}  // namespace deft
