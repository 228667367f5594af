// Distillation from a teacher's top logits.
//
//   p = softmax(t / T) over the entries that the teacher kept,  q = softmax(z / T) over the vocabulary
//   loss = T^2 sum_k p_k (log p_k - log q_{i_k}),   dz = g T (q - p scattered to its indices)
//
// A workgroup owns a row.  Bound by the row's bytes: one read for the loss, one more write for the gradient.
#include "ends.h"

namespace deft {
namespace {

constexpr int kThreads = 512, kWaves = kThreads / kWave;

template <typename T> struct Vec;   // 16 bytes of a row, at any address that its elements may have
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

// Sum over the workgroup; every thread gets it.  `room` is read until the next barrier.
__device__ __forceinline__ float block_sum(float x, float *room)
{
    x = wave_sum(x);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) room[threadIdx.x >> 6] = x;
    __syncthreads();
    float s = 0.0f;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) s += room[w];
    return s;
}

__device__ __forceinline__ float block_max(float x, float *room)
{
    x = wave_max(x);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) room[threadIdx.x >> 6] = x;
    __syncthreads();
    float m = room[0];
#pragma unroll
    for (int w = 1; w < kWaves; ++w) m = fmaxf(m, room[w]);
    return m;
}

template <typename T>
__global__ void __launch_bounds__(kThreads) distill_kernel(deft_distill_t a)
{
    extern __shared__ __align__(16) char lds[];
    int32_t *index = reinterpret_cast<int32_t *>(lds);
    float *prob = reinterpret_cast<float *>(lds) + a.top_k;
    __shared__ float room[kWaves];
    constexpr int n = Vec<T>::n;
    const int tid = threadIdx.x;
    const int64_t row = blockIdx.x;
    const T *z = static_cast<const T *>(a.logits) + row * a.logits_stride;
    T *grad = a.grad_logits ? static_cast<T *>(a.grad_logits) + row * a.grad_stride : nullptr;
    const float inv_t = 1.0f / a.temperature;

    // the teacher's entries
    int kept = 0, bad = 0;
    float top = -INFINITY;
    for (int k = tid; k < a.top_k; k += kThreads) {
        const int v = a.teacher_index[row * a.top_k + k];
        const bool in = v >= 0 && v < a.vocab;
        const float u = in ? a.teacher_logit[row * a.top_k + k] * inv_t : -INFINITY;
        index[k] = in ? v : -1;
        prob[k] = u;
        kept |= v != -1;
        bad |= !in && v != -1;
        top = fmaxf(top, u);
    }
    kept = __syncthreads_or(kept);
    bad = __syncthreads_or(bad);
    top = block_max(top, room);
    float part = 0.0f;
    for (int k = tid; k < a.top_k; k += kThreads)
        if (index[k] >= 0) part += __expf(prob[k] - top);
    const float total = block_sum(part, room);
    bad |= kept && top == -INFINITY && total != total;

    // the student's softmax
    SoftSum s = {-INFINITY, 0.0f};
    if (kept && !bad) {
        const int whole = a.vocab / n * n;
        for (int at = tid * n; at < whole; at += kThreads * n) {
            const typename Vec<T>::type x = *reinterpret_cast<const typename Vec<T>::type *>(z + at);
            SoftSum b = {-INFINITY, 0.0f};
#pragma unroll
            for (int i = 0; i < n; ++i) b.top = fmaxf(b.top, (float)x[i] * inv_t);
            if (b.top == -INFINITY) b.top = -3.0e38f;   // (exp(-inf - that) is 0, and NaN stays NaN)
#pragma unroll
            for (int i = 0; i < n; ++i) b.sum += __expf((float)x[i] * inv_t - b.top);
            s = soft_join(s, b);
        }
        for (int at = whole + tid; at < a.vocab; at += kThreads) {
            const float x = (float)z[at] * inv_t;
            const SoftSum b = {x == -INFINITY ? -3.0e38f : x, x == -INFINITY ? 0.0f : __expf(x - x)};
            s = soft_join(s, b);
        }
    }
    const float most = block_max(s.top, room);
    const float sum = block_sum(s.sum == 0.0f ? 0.0f : s.sum * __expf(s.top - most), room);
    bad |= kept && sum == 0.0f;
    const bool ok = kept && !bad;
    const float lse = most + __logf(sum);
    if (tid == 0 && a.status) a.status[row] = bad ? DEFT_ERR_INVALID_ARG : DEFT_OK;

    // loss; prob becomes the teacher's probabilities
    float by = 0.0f;
    if (ok) {
        const float log_total = __logf(total);
        for (int k = tid; k < a.top_k; k += kThreads) {
            const float u = prob[k] - top;
            const float p = index[k] >= 0 ? __expf(u) / total : 0.0f;
            if (p > 0.0f || p != p) by += p * (u - log_total - ((float)z[index[k]] * inv_t - lse));
            prob[k] = p;
        }
    }
    by = block_sum(by, room);
    if (tid == 0) a.loss[row] = ok ? by * a.temperature * a.temperature : 0.0f;
    if (!grad) return;

    const float g = ok ? a.row_grad[row] * a.temperature : 0.0f;
    // what the indices' elements become, before the logits may be overwritten
    float fixed[2] = {};
    for (int k = tid, j = 0; k < a.top_k && ok; k += kThreads, ++j) {
        if (index[k] < 0) continue;
        float p = 0.0f;
        for (int o = 0; o < a.top_k; ++o) p += index[o] == index[k] ? prob[o] : 0.0f;
        fixed[j & 1] = g * (__expf((float)z[index[k]] * inv_t - lse) - p);
    }
    __syncthreads();
    const int whole = a.vocab / n * n;
    for (int at = tid * n; at < whole; at += kThreads * n) {
        typename Vec<T>::type x = {};
        if (ok) {
            x = *reinterpret_cast<const typename Vec<T>::type *>(z + at);
#pragma unroll
            for (int i = 0; i < n; ++i) x[i] = (T)(g * __expf((float)x[i] * inv_t - lse));
        }
        *reinterpret_cast<typename Vec<T>::type *>(grad + at) = x;
    }
    for (int at = whole + tid; at < a.vocab; at += kThreads)
        grad[at] = ok ? (T)(g * __expf((float)z[at] * inv_t - lse)) : (T)0.0f;
    __syncthreads();
    for (int k = tid, j = 0; k < a.top_k && ok; k += kThreads, ++j)
        if (index[k] >= 0) grad[index[k]] = (T)fixed[j & 1];
}

}  // namespace

hipError_t distill_launch(int dtype, const deft_distill_t &a, int, hipStream_t st)
{
    const size_t lds = (size_t)a.top_k * 8;
    if (dtype == DEFT_F32) distill_kernel<float><<<a.n_rows, kThreads, lds, st>>>(a);
    else if (dtype == DEFT_F16) distill_kernel<f16><<<a.n_rows, kThreads, lds, st>>>(a);
    else distill_kernel<bf16><<<a.n_rows, kThreads, lds, st>>>(a);
    return hipGetLastError();
}

}  // namespace deft
