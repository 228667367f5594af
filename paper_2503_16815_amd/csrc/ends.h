// What the operators at a language model's ends share: types and their conversions, small device
// helpers, and the launch interface between the C ABI (ends_api.hip) and the kernels.
#pragma once
#include <hip/hip_runtime.h>

#include <cstdint>

#include "../../include/deft_ends.h"

namespace deft {

typedef _Float16 f16;
typedef __bf16 bf16;
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef int i32x4 __attribute__((ext_vector_type(4)));

// ---- device helpers -------------------------------------------------------------------------

constexpr int kWave = 64;

__device__ __forceinline__ float wave_max(float x)
{
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) x = fmaxf(x, __shfl_xor(x, d));
    return x;
}

__device__ __forceinline__ float wave_sum(float x)
{
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) x += __shfl_xor(x, d);
    return x;
}

// 16 bytes of a row, at any address that its elements may have
template <typename T> struct Vec;
template <> struct Vec<float> {
    typedef float type __attribute__((ext_vector_type(4), aligned(4)));
    static constexpr int n = 4;
};
template <> struct Vec<f16> {
    typedef f16 type __attribute__((ext_vector_type(8), aligned(2)));
    static constexpr int n = 8;
};
template <> struct Vec<bf16> {
    typedef bf16 type __attribute__((ext_vector_type(8), aligned(2)));
    static constexpr int n = 8;
};

// What stands for the largest of values that are all -infinity, or of none: -infinity less this gives an exponential of 0,
// and no finite value is below it.
constexpr float kLowest = -3.402823466e38f;

// A running softmax sum: the largest value so far and the sum of exp(value - largest).  -infinity
// adds nothing to it; a NaN or +infinity makes the sum NaN, as the definition does.
struct SoftSum {
    float top, sum;
};

__device__ __forceinline__ SoftSum soft_join(SoftSum a, SoftSum b)
{
    const float top = fmaxf(a.top, b.top);   // (fmaxf drops NaN: it stays in the sums)
    SoftSum r;
    r.top = top;
    r.sum = (a.top == top ? a.sum : a.sum * __expf(a.top - top)) + (b.top == top ? b.sum : b.sum * __expf(b.top - top));
    return r;
}

// ---- launches (each returns hipGetLastError() of its launches) ------------------------------

struct EmbedPlan {
    int64_t scratch_bytes = 0;
    int max_rows = 0, max_vocab = 0, max_hidden = 0;
};
void embed_grad_plan(int max_rows, int max_vocab, int max_hidden, EmbedPlan *plan);
hipError_t embed_launch(int dtype, const deft_embed_t &e, hipStream_t st);
hipError_t embed_grad_launch(const EmbedPlan &plan, int dtype, const deft_embed_grad_t &e, void *scratch, int compute_units,
                             hipStream_t st);

struct HeadPlan {
    int64_t scratch_bytes = 0;
    int max_rows = 0, max_vocab = 0, max_hidden = 0;
    int planes = 1;      // 16-bit arrays that an operand is held in: 1, or 3 for 32-bit types
    int piece = 0;       // rows of the vocabulary at a time
    bool grad = false;
    // offsets into the scratch memory
    int64_t ints, floats, hidden, weight, parts, hidden_t, d, sums;
};
void head_plan(int dtype, int max_rows, int max_vocab, int max_hidden, bool grad, int compute_units, HeadPlan *plan);
hipError_t head_prepare();   // kernel attributes, on the current device
hipError_t head_loss_launch(const HeadPlan &plan, int dtype, const deft_head_loss_t &a, void *scratch, int compute_units,
                            hipStream_t st);
hipError_t head_grad_launch(const HeadPlan &plan, int dtype, const deft_head_grad_t &a, void *scratch, int compute_units,
                            hipStream_t st);

hipError_t distill_launch(int dtype, const deft_distill_t &a, int compute_units, hipStream_t st);

}  // namespace deft
