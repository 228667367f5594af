// The head's scratch memory, and its calls by type (each type's kernels are a file of their own).
#include "ends_shapes.h"

namespace deft {

#define DEFT_HEAD_TYPE(NAME)                                                                                                   \
    hipError_t head_prepare_##NAME();                                                                                          \
    hipError_t head_loss_##NAME(const HeadPlan &, const deft_head_loss_t &, void *, int, hipStream_t);                         \
    hipError_t head_grad_##NAME(const HeadPlan &, const deft_head_grad_t &, void *, int, hipStream_t);
DEFT_HEAD_TYPE(bf16)
DEFT_HEAD_TYPE(f16)
DEFT_HEAD_TYPE(f32)

void head_plan(int dtype, int max_rows, int max_vocab, int max_hidden, bool grad, int compute_units, HeadPlan *plan)
{
    const int64_t n = up(max_rows, kTile), k = up(max_hidden, kStep);
    plan->max_rows = max_rows;
    plan->max_vocab = max_vocab;
    plan->max_hidden = max_hidden;
    plan->grad = grad;
    plan->planes = dtype == DEFT_F32 ? 3 : 1;
    int64_t piece = kWeightBytes / (2 * plan->planes * k);
    if (grad) {
        const int64_t by_d = kPieceBytes / (2 * plan->planes * n);
        piece = piece < by_d ? piece : by_d;
    }
    piece = piece / kTile * kTile;
    if (piece < 4 * kTile) piece = 4 * kTile;
    if (piece > up(max_vocab, kTile)) piece = up(max_vocab, kTile);
    if (grad) {   // of the sizes that fit, the one whose products leave the fewest compute units idle over all pieces
        const int64_t products = plan->planes == 3 ? 6 : 1, most = piece;
        double least = 1e300;
        for (int64_t p = most; p >= kTile && p * 8 >= most; p -= kTile) {
            double t = 0.0;
            const int64_t whole = max_vocab / p, rest = max_vocab % p;
            for (int last = 0; last < 2; ++last) {
                const int64_t rows = last ? rest : p, times = last ? 1 : whole;
                if (rows == 0 || times == 0) continue;
                const int64_t steps = up(rows, kStep) / kStep * products;
                t += (double)times * (12.0 + least_cost(rows, max_rows, k / kStep * products, 1, compute_units) +
                                      least_cost(max_hidden, rows, up(max_rows, kStep) / kStep * products, 1, compute_units) +
                                      least_cost(max_hidden, max_rows, steps, splits_of(max_hidden, max_rows, steps, compute_units), compute_units));
            }
            if (t < least) {
                least = t;
                piece = p;
            }
        }
    }
    plan->piece = (int)piece;
    int64_t at = 0;
    const auto take = [&](int64_t bytes) {
        const int64_t here = at;
        at += up(bytes, 256);
        return here;
    };
    plan->ints = take((64 + 3 * n) * 4);
    plan->floats = take((64 + 5 * n) * 4);
    plan->hidden = take(plan->planes * n * k * 2);
    plan->weight = take(plan->planes * piece * k * 2);
    plan->parts = take(n * ((max_vocab + 127) / 128) * 8);
    if (grad) {
        plan->hidden_t = take(plan->planes * n * k * 2);
        plan->d = take(plan->planes * (n < 2 * kTile ? 2 * kTile : n) * piece * 2);   // (room for a second array of few positions)
        // one array of sums, or several where splits * tiles stays within twice the compute units
        const int64_t one = n * up(max_hidden, 4), split = 2 * (int64_t)compute_units * kTile * kTile;
        plan->sums = take((one > split ? one : split) * 4);
    }
    plan->scratch_bytes = at;
}

hipError_t head_prepare()
{
    hipError_t e = head_prepare_bf16();
    if (e == hipSuccess) e = head_prepare_f16();
    if (e == hipSuccess) e = head_prepare_f32();
    return e;
}

hipError_t head_loss_launch(const HeadPlan &plan, int dtype, const deft_head_loss_t &a, void *scratch, int compute_units,
                            hipStream_t st)
{
    if (dtype == DEFT_F32) return head_loss_f32(plan, a, scratch, compute_units, st);
    if (dtype == DEFT_F16) return head_loss_f16(plan, a, scratch, compute_units, st);
    return head_loss_bf16(plan, a, scratch, compute_units, st);
}

hipError_t head_grad_launch(const HeadPlan &plan, int dtype, const deft_head_grad_t &a, void *scratch, int compute_units,
                            hipStream_t st)
{
    if (dtype == DEFT_F32) return head_grad_f32(plan, a, scratch, compute_units, st);
    if (dtype == DEFT_F16) return head_grad_f16(plan, a, scratch, compute_units, st);
    return head_grad_bf16(plan, a, scratch, compute_units, st);
}

}  // namespace deft
