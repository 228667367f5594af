// Distillation from a teacher's top logits.
//
//   p = softmax(t / T) over the entries that the teacher kept,  q = softmax(z / T) over the vocabulary
//   loss = T^2 sum_k p_k (log p_k - log q_{i_k}),   dz = g T (q - p scattered to its indices)
//
// Bound by the row's bytes: one read for the loss, one more write for the gradient.  A row of up to 256 KB
// stays in the registers of one workgroup of 1024 lanes from its one read to the gradient's write
// (131072 16-bit logits take 64 registers a lane).  The workgroup goes on from row to row, and each
// 16 bytes of the next row are asked for as soon as the gradient of the present row's has been stored,
// so memory is idle only during the row's two reductions.  Rows that are longer are read once more.
// With the gradient, 64 entries of the teacher a row: 4096 x 50257 bf16 177 us, 4.7 TB/s read and written (a large copy 5.1);
// 8192 x 131071 f16 978 us, 4.4 TB/s; rows too long for registers, 1024 x 200000 f32: 497 us, 4.9 TB/s with the second read.
#include "ends.h"

namespace deft {
namespace {

constexpr int kThreads = 512, kWaves = kThreads / kWave;

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
        if (prob[k] != -INFINITY) part += __expf(prob[k] - top);   // (a NaN, which is no maximum, makes the sum one)
    const float total = block_sum(part, room);
    bad |= kept && total == 0.0f;                                  // all of them -infinity

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

// ---- rows that stay in registers -------------------------------------------------------------

constexpr int kMarkBits = 1 << 17;   // of the map that shows whether an index occurs twice
constexpr float kLog2e = 1.44269504088896340736f, kLn2 = 0.69314718055994530942f;

__device__ __forceinline__ float exp2_of(float x) { return __builtin_amdgcn_exp2f(x); }

__device__ __forceinline__ SoftSum soft_join2(SoftSum a, SoftSum b)   // with powers of two
{
    const float top = fmaxf(a.top, b.top);
    return {top, (a.top == top ? a.sum : a.sum * exp2_of(a.top - top)) + (b.top == top ? b.sum : b.sum * exp2_of(b.top - top))};
}

__device__ __forceinline__ SoftSum wave_join2(SoftSum s, int from)
{
    for (int d = from; d > 0; d >>= 1) s = soft_join2(s, SoftSum{__shfl_xor(s.top, d), __shfl_xor(s.sum, d)});
    return s;
}

// 16 bytes of logits as floats
__device__ __forceinline__ void widen(i32x4 v, float (&x)[4], float)
{
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = __int_as_float(v[i]);
}
__device__ __forceinline__ void widen(i32x4 v, float (&x)[8], bf16)
{
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        x[2 * i] = __int_as_float(v[i] << 16);
        x[2 * i + 1] = __int_as_float(v[i] & (int)0xffff0000);
    }
}
__device__ __forceinline__ void widen(i32x4 v, float (&x)[8], f16)
{
    typedef f16 f16x8 __attribute__((ext_vector_type(8)));
    const f16x8 h = __builtin_bit_cast(f16x8, v);
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = (float)h[i];
}

// Each lane holds NV vectors of the row, kRowThreads vectors apart, from the row's first 16-byte boundary on (a wave's
// vectors that straddle such boundaries cost a tenth of the time), and one of the elements before and behind them;
// the k-th lane the teacher's k-th entry.  Logits are scaled by log2(e) / T as they are used.
template <typename T, int kRowThreads, int NV, bool GRAD>
__global__ void __launch_bounds__(kRowThreads, 4) distill_row_kernel(deft_distill_t a)
{
    constexpr int kRowWaves = kRowThreads / kWave;
    typedef typename Vec<T>::type V;
    constexpr int n = Vec<T>::n;
    __shared__ unsigned mark[kMarkBits / 32];
    __shared__ SoftSum student[kRowWaves], teacher[kRowWaves];
    __shared__ int flags[kRowWaves], twice[2];
    __shared__ float part[kRowWaves];
    __shared__ int same_index[kRowThreads];
    __shared__ float same_prob[kRowThreads];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const float c = kLog2e / a.temperature;
    const T *const logits = static_cast<const T *>(a.logits);
    for (int i = tid; i < kMarkBits / 32; i += kRowThreads) mark[i] = 0;
    if (tid < 2) twice[tid] = 0;

    // where a row's vectors begin, how many elements they have, and this lane's single element (or -1)
    const auto before = [&](int64_t row) {
        const int at = (int)((uintptr_t)(logits + row * a.logits_stride) & 15);
        return min(at ? (16 - at) / (int)sizeof(T) : 0, a.vocab);
    };
    const auto inside = [&](int head) { return (a.vocab - head) / n * n; };
    const auto single = [&](int head, int whole) {
        const int at = tid < head ? tid : tid + whole;
        return at < a.vocab && tid < 2 * n ? at : -1;
    };
    i32x4 x[NV];
    T last = (T)0.0f;
    const auto load = [&](int64_t row, int head, int whole, int j) {
        const int at = (j * kRowThreads + tid) * n;
        if (at < whole) x[j] = __builtin_bit_cast(i32x4, *reinterpret_cast<const V *>(logits + row * a.logits_stride + head + at));
    };
    const auto entry = [&](int64_t row, int &index, float &u) {
        index = -1;
        u = -INFINITY;
        if (row < a.n_rows && tid < a.top_k) {
            index = a.teacher_index[row * a.top_k + tid];
            u = a.teacher_logit[row * a.top_k + tid];
        }
    };
    int index, next_index;
    float u, next_u;
    entry(blockIdx.x, index, u);
    bool kept = __syncthreads_or(index != -1);
    int head = before(blockIdx.x), whole = inside(head);
    if (kept) {
#pragma unroll
        for (int j = 0; j < NV; ++j) load(blockIdx.x, head, whole, j);
        if (single(head, whole) >= 0) last = logits[(int64_t)blockIdx.x * a.logits_stride + single(head, whole)];
    }

    int odd = 0;
    for (int64_t row = blockIdx.x; row < a.n_rows; row += gridDim.x, odd ^= 1) {
        const int64_t next = row + gridDim.x;
        const int at_last = single(head, whole);
        const bool in = index >= 0 && index < a.vocab;
        float z_at = 0.0f;   // the logit at this lane's entry
        if (in) z_at = (float)logits[row * a.logits_stride + index] * c;
        entry(next, next_index, next_u);
        if (in) {
            const unsigned bit = 1u << (index & 31);
            if (atomicOr(&mark[(index % kMarkBits) >> 5], bit) & bit) twice[odd] = 1;
        }
        SoftSum s = {-INFINITY, 0.0f}, t = {in ? u * c : -INFINITY, 0.0f};
        if (kept) {
            // -3e38 in the place of -infinity: exp2(-infinity - that) is 0, and a NaN stays one
            float top = at_last >= 0 ? (float)last : -3.0e38f;
#pragma unroll
            for (int j = 0; j < NV; ++j) {
                if ((j * kRowThreads + tid) * n < whole) {
                    float w[n];
                    widen(x[j], w, T());
#pragma unroll
                    for (int i = 0; i < n; i += 2) top = fmaxf(top, fmaxf(w[i], w[i + 1]));
                }
                asm volatile("" : "+v"(x[j]));   // (widened again for the sum: kept as floats the row would not fit)
            }
            top = fmaxf(top * c, -3.0e38f);
            float sum[2] = {at_last >= 0 ? exp2_of(__builtin_fmaf((float)last, c, -top)) : 0.0f, 0.0f};
#pragma unroll
            for (int j = 0; j < NV; ++j) {
                if ((j * kRowThreads + tid) * n < whole) {
                    float w[n];
                    widen(x[j], w, T());
#pragma unroll
                    for (int i = 0; i < n; ++i) sum[i & 1] += exp2_of(__builtin_fmaf(w[i], c, -top));
                }
                asm volatile("" : "+v"(x[j]));
            }
            s = wave_join2(SoftSum{top, sum[0] + sum[1]}, 32);
            if (in) t.sum = t.top == -INFINITY ? 0.0f : exp2_of(t.top - t.top);   // (1, or the NaN that the entry is)
            t = wave_join2(t, 32);
        }
        const int flag = (__any(index != -1 && !in) ? 1 : 0) | (__any(next_index != -1) ? 2 : 0);
        if (lane == 0) {
            student[wave] = s;
            teacher[wave] = t;
            flags[wave] = flag;
        }
        __syncthreads();
        s = wave_join2(student[lane & (kRowWaves - 1)], kRowWaves / 2);
        t = wave_join2(teacher[lane & (kRowWaves - 1)], kRowWaves / 2);
        const int all = flags[lane & (kRowWaves - 1)];
        const bool outside = __any(all & 1), next_kept = __any(all & 2);
        const bool bad = kept && (outside || s.sum == 0.0f || t.sum == 0.0f), ok = kept && !bad;
        const float lse = s.top + __log2f(s.sum);
        float p = 0.0f, by = 0.0f;
        if (in && ok) {
            const float v = u * c - t.top;
            p = exp2_of(v) / t.sum;
            if (p > 0.0f || p != p) by = p * (v - __log2f(t.sum) - (z_at - lse)) * kLn2;
        }
        by = wave_sum(by);
        if (lane == 0) part[wave] = by;
        float g = 0.0f, fixed = 0.0f;
        if (GRAD && ok) {
            g = a.row_grad[row] * a.temperature;
            if (twice[odd]) {   // an index that occurs twice counts with the sum of its entries
                same_index[tid] = in ? index : -1;
                same_prob[tid] = p;
                __syncthreads();
                p = 0.0f;
                for (int k = 0; k < a.top_k; ++k) p += same_index[k] == index ? same_prob[k] : 0.0f;
            }
            fixed = g * (exp2_of(z_at - lse) - p);
        }
        if (in) mark[(index % kMarkBits) >> 5] = 0;
        if (tid == 0) twice[odd ^ 1] = 0;

        T *grad = GRAD ? static_cast<T *>(a.grad_logits) + row * a.grad_stride : nullptr;
        if (GRAD && at_last >= 0) grad[at_last] = ok ? (T)(g * exp2_of(__builtin_fmaf((float)last, c, -lse))) : (T)0.0f;
        const int next_head = before(next), next_whole = inside(next_head);
        if (next_kept && single(next_head, next_whole) >= 0) last = logits[next * a.logits_stride + single(next_head, next_whole)];
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const int at = (j * kRowThreads + tid) * n;
            if (GRAD && at < whole) {
                V y = {};
                if (ok) {
                    float w[n];
                    widen(x[j], w, T());
#pragma unroll
                    for (int i = 0; i < n; ++i) y[i] = (T)(g * exp2_of(__builtin_fmaf(w[i], c, -lse)));
                }
                *reinterpret_cast<V *>(grad + head + at) = y;
            }
            if (next_kept) load(next, next_head, next_whole, j);
        }
        if (GRAD) asm volatile("s_waitcnt vmcnt(0)" ::: "memory");   // the stores above come before those below
        __syncthreads();
        if (GRAD && in && ok) grad[index] = (T)fixed;
        if (tid == 0) {
            float loss = 0.0f;
#pragma unroll
            for (int w = 0; w < kRowWaves; ++w) loss += part[w];
            a.loss[row] = ok ? loss * a.temperature * a.temperature : 0.0f;
            if (a.status) a.status[row] = bad ? DEFT_ERR_INVALID_ARG : DEFT_OK;
        }
        index = next_index;
        u = next_u;
        kept = next_kept;
        head = next_head;
        whole = next_whole;
    }
}

// PER_UNIT: workgroups that a compute unit holds at once, by their registers.
template <typename T, int THREADS, int NV, int PER_UNIT>
hipError_t row_launch(const deft_distill_t &a, int compute_units, hipStream_t st)
{
    const int most = compute_units * PER_UNIT, blocks = a.n_rows < most ? a.n_rows : most;
    if (a.grad_logits) distill_row_kernel<T, THREADS, NV, true><<<blocks, THREADS, 0, st>>>(a);
    else distill_row_kernel<T, THREADS, NV, false><<<blocks, THREADS, 0, st>>>(a);
    return hipGetLastError();
}

// By the row's bytes alone (and by top_k, an entry a lane): as few lanes as hold it, so that more workgroups
// share a compute unit and one's reductions fall into the others' reads and writes.  (4096 rows of 16-bit logits with
// 64 entries each, the time for 1024 lanes behind it: 8000 logits 46 us, 138; 12000: 66, 129; 30000: 129, 170;
// 50257: 190, 224.  200 rows: 8000 logits 18, 21; 30000: 21, 23; 50257: 25, 26.)
template <typename T>
hipError_t any_launch(const deft_distill_t &a, int compute_units, hipStream_t st)
{
    const int vectors = a.vocab / Vec<T>::n;
    if (a.top_k <= 256 && vectors <= 256 * 4) return row_launch<T, 256, 4, 7>(a, compute_units, st);
    if (a.top_k <= 512 && vectors <= 512 * 4) return row_launch<T, 512, 4, 3>(a, compute_units, st);
    if (a.top_k <= 512 && vectors <= 512 * 8) return row_launch<T, 512, 8, 2>(a, compute_units, st);
    if (a.top_k <= 512 && vectors <= 512 * 16) return row_launch<T, 512, 16, 2>(a, compute_units, st);
    if (vectors <= 1024 * 16) return row_launch<T, 1024, 16, 1>(a, compute_units, st);
    distill_kernel<T><<<a.n_rows, kThreads, (size_t)a.top_k * 8, st>>>(a);
    return hipGetLastError();
}

}  // namespace

hipError_t distill_launch(int dtype, const deft_distill_t &a, int compute_units, hipStream_t st)
{
    if (dtype == DEFT_F32) return any_launch<float>(a, compute_units, st);
    if (dtype == DEFT_F16) return any_launch<f16>(a, compute_units, st);
    return any_launch<bf16>(a, compute_units, st);
}

}  // namespace deft
