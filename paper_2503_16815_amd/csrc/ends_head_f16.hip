// The head in 16-bit floats.
#include "ends_head.h"

namespace deft {

hipError_t head_prepare_f16() { return allow_all<f16, f16, false>(); }

hipError_t head_loss_f16(const HeadPlan &plan, const deft_head_loss_t &a, void *scratch, int compute_units, hipStream_t st)
{
    return Head<f16, f16, 1>::loss(plan, a, Scratch(plan, scratch), compute_units, st);
}

hipError_t head_grad_f16(const HeadPlan &plan, const deft_head_grad_t &a, void *scratch, int compute_units, hipStream_t st)
{
    return Head<f16, f16, 1>::gradient(plan, a, Scratch(plan, scratch), compute_units, st);
}

}  // namespace deft
