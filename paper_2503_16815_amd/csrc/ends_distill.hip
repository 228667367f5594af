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
// 8192 x 131071 f16 966 us, 4.4 TB/s; rows too long for registers, 1024 x 200000 f32: 492 us, 5.0 TB/s with the second read.
// The loss alone: 4096 x 50257 bf16 91 us, 4.5 TB/s; 8192 x 131071 f16 449 us, 4.8 TB/s.
#include "ends.h"

namespace deft {
namespace {

constexpr int kThreads = 512, kWaves = kThreads / kWave;
constexpr float kLog2e = 1.44269504088896340736f, kLn2 = 0.69314718055994530942f;

// Exponentials are powers of two of (z - largest) log2(e) / T: the difference first, so that neither what a row's
// logits have in common nor a logit at the end of the type's range costs any bits.
__device__ __forceinline__ float exp2_of(float x) { return __builtin_amdgcn_exp2f(x); }

// of running sums whose largest values are logits as they are, kLowest or more (NaN is in the sums alone); c = log2(e) / T
__device__ __forceinline__ SoftSum soft_join2(SoftSum a, SoftSum b, float c)
{
    const float less = exp2_of(-fabsf((a.top - b.top) * c));
    const bool first = a.top >= b.top;
    return {first ? a.top : b.top, __builtin_fmaf(first ? b.sum : a.sum, less, first ? a.sum : b.sum)};
}

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
    const float c = kLog2e / a.temperature;

    // the teacher's entries
    int kept = 0, bad = 0;
    float top = -INFINITY;
    for (int k = tid; k < a.top_k; k += kThreads) {
        const int v = a.teacher_index[row * a.top_k + k];
        const bool in = v >= 0 && v < a.vocab;
        const float u = in ? a.teacher_logit[row * a.top_k + k] : -INFINITY;
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
        if (prob[k] != -INFINITY) part += exp2_of((prob[k] - top) * c);   // (a NaN, which is no maximum, makes the sum one)
    const float total = block_sum(part, room);
    bad |= kept && total == 0.0f;                                         // all of them -infinity

    // the student's softmax
    SoftSum s = {kLowest, 0.0f};
    if (kept && !bad) {
        const int whole = a.vocab / n * n;
        for (int at = tid * n; at < whole; at += kThreads * n) {
            const typename Vec<T>::type x = *reinterpret_cast<const typename Vec<T>::type *>(z + at);
            SoftSum b = {kLowest, 0.0f};
#pragma unroll
            for (int i = 0; i < n; ++i) b.top = fmaxf(b.top, (float)x[i]);
#pragma unroll
            for (int i = 0; i < n; ++i) b.sum += exp2_of(((float)x[i] - b.top) * c);
            s = soft_join2(s, b, c);
        }
        for (int at = whole + tid; at < a.vocab; at += kThreads) {
            const float x = (float)z[at], at_least = fmaxf(x, kLowest);
            s = soft_join2(s, SoftSum{at_least, exp2_of((x - at_least) * c)}, c);
        }
    }
    const float most = block_max(s.top, room);
    const float sum = block_sum(s.sum == 0.0f ? 0.0f : s.sum * exp2_of((s.top - most) * c), room);
    bad |= kept && sum == 0.0f;
    const bool ok = kept && !bad;
    const float log_sum = __log2f(sum);
    if (tid == 0 && a.status) a.status[row] = bad ? DEFT_ERR_INVALID_ARG : DEFT_OK;

    // loss; prob becomes the teacher's probabilities
    float by = 0.0f;
    if (ok) {
        const float logs = (__log2f(total) - log_sum) * kLn2;
        for (int k = tid; k < a.top_k; k += kThreads) {
            const float u = prob[k] - top;
            const float p = index[k] >= 0 ? exp2_of(u * c) / total : 0.0f;
            if (p > 0.0f || p != p) by += p * (u / a.temperature - ((float)z[index[k]] - most) / a.temperature - logs);
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
        fixed[j & 1] = g * (exp2_of(__builtin_fmaf((float)z[index[k]] - most, c, -log_sum)) - p);
    }
    __syncthreads();
    const int whole = a.vocab / n * n;
    for (int at = tid * n; at < whole; at += kThreads * n) {
        typename Vec<T>::type x = {};
        if (ok) {
            x = *reinterpret_cast<const typename Vec<T>::type *>(z + at);
#pragma unroll
            for (int i = 0; i < n; ++i) x[i] = (T)(g * exp2_of(__builtin_fmaf((float)x[i] - most, c, -log_sum)));
        }
        *reinterpret_cast<typename Vec<T>::type *>(grad + at) = x;
    }
    for (int at = whole + tid; at < a.vocab; at += kThreads)
        grad[at] = ok ? (T)(g * exp2_of(__builtin_fmaf((float)z[at] - most, c, -log_sum))) : (T)0.0f;
    __syncthreads();
    for (int k = tid, j = 0; k < a.top_k && ok; k += kThreads, ++j)
        if (index[k] >= 0) grad[index[k]] = (T)fixed[j & 1];
}

// ---- rows that stay in registers -------------------------------------------------------------

constexpr int kMarkBits = 1 << 17;   // of the map that shows whether an index occurs twice

// (w - top) c as one instruction, fma(w, c, -product), which leaves the product's rounding in every power alike:
// they are 2^rounding times as large.  Not where that could be far from 1, nor where the product is not finite.  (The
// difference first is an instruction more, for 16-bit floats, whose widening the fma takes with it, two.  Loss alone of 8192 x 131071
// f16: 449 us so, 489 with the difference; with the gradient 966 and 990; 4096 x 8000 bf16 28.3 and 28.9.)
struct Scaled {
    float product, rounding;
    bool far;
    __device__ __forceinline__ Scaled(float top, float c) : product(top * c)
    {
        far = !(fabsf(product) < 0x1p20f);
        rounding = __builtin_fmaf(top, c, -product);
    }
    __device__ __forceinline__ float shrink() const { return exp2_of(-rounding); }
};

__device__ __forceinline__ SoftSum wave_join2(SoftSum s, int from, float c)
{
    for (int d = from; d > 0; d >>= 1) s = soft_join2(s, SoftSum{__shfl_xor(s.top, d), __shfl_xor(s.sum, d)}, c);
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

template <typename T, int N>
__device__ __forceinline__ void narrow(const float (&x)[N], i32x4 &v, T)
{
    typedef T V __attribute__((ext_vector_type(N)));
    V y;
#pragma unroll
    for (int i = 0; i < N; ++i) y[i] = (T)x[i];
    v = __builtin_bit_cast(i32x4, y);
}

// Each lane holds NV vectors of the row, kRowThreads vectors apart, from the row's first 16-byte boundary on (a wave's
// vectors that straddle such boundaries cost a tenth of the time), and one of the elements before and behind them;
// the k-th lane the teacher's k-th entry.
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
    const float c = kLog2e / a.temperature, inv_t = 1.0f / a.temperature;
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
        if (in) z_at = (float)logits[row * a.logits_stride + index];
        entry(next, next_index, next_u);
        if (in) {
            const unsigned bit = 1u << (index & 31);
            if (atomicOr(&mark[(index % kMarkBits) >> 5], bit) & bit) twice[odd] = 1;
        }
        // Everything asked for is there, whether the row is kept or not: otherwise the compiler lets each of the next row's
        // loads wait for the one before it (8192 x 131071 f16, loss alone: 474 us, 600 so).
        __builtin_amdgcn_s_waitcnt(0x0f70);   // (vmcnt 0)
        SoftSum s = {kLowest, 0.0f}, t = {in ? fmaxf(u, kLowest) : kLowest, 0.0f};
        if (kept) {
            float top = at_last >= 0 ? fmaxf((float)last, kLowest) : kLowest;
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
            const bool some = at_last >= 0 || tid * n < whole;
            const Scaled scaled(top, c);
            float sum[2] = {at_last >= 0 ? exp2_of(__builtin_fmaf((float)last, c, -scaled.product)) : 0.0f, 0.0f};
#pragma unroll
            for (int j = 0; j < NV; ++j) {
                if ((j * kRowThreads + tid) * n < whole) {
                    float w[n];
                    widen(x[j], w, T());
#pragma unroll
                    for (int i = 0; i < n; ++i) sum[i & 1] += exp2_of(__builtin_fmaf(w[i], c, -scaled.product));
                }
                asm volatile("" : "+v"(x[j]));
            }
            s = {top, some ? (sum[0] + sum[1]) * scaled.shrink() : 0.0f};
            if (__any(some && scaled.far)) {
                s.sum = at_last >= 0 ? exp2_of(((float)last - top) * c) : 0.0f;
#pragma unroll
                for (int j = 0; j < NV; ++j) {
                    if ((j * kRowThreads + tid) * n >= whole) continue;
                    i32x4 copy = x[j];
                    asm volatile("" : "+v"(copy));   // (or it would be widened for both sums at once)
                    float w[n];
                    widen(copy, w, T());
#pragma unroll
                    for (int i = 0; i < n; ++i) s.sum += exp2_of((w[i] - top) * c);
                }
            }
            s = wave_join2(s, 32, c);
            if (in) t.sum = exp2_of((u - t.top) * c);   // (1, 0 of -infinity, or the NaN that the entry is)
            t = wave_join2(t, 32, c);
        }
        const int flag = (__any(index != -1 && !in) ? 1 : 0) | (__any(next_index != -1) ? 2 : 0);
        if (lane == 0) {
            student[wave] = s;
            teacher[wave] = t;
            flags[wave] = flag;
        }
        __syncthreads();
        s = wave_join2(student[lane & (kRowWaves - 1)], kRowWaves / 2, c);
        t = wave_join2(teacher[lane & (kRowWaves - 1)], kRowWaves / 2, c);
        const int all = flags[lane & (kRowWaves - 1)];
        const bool outside = __any(all & 1), next_kept = __any(all & 2);
        const bool bad = kept && (outside || s.sum == 0.0f || t.sum == 0.0f), ok = kept && !bad;
        const float log_sum = __log2f(s.sum);
        float p = 0.0f, by = 0.0f;
        if (in && ok) {
            p = exp2_of((u - t.top) * c) * __builtin_amdgcn_rcpf(t.sum);
            if (p > 0.0f || p != p) by = p * ((u - t.top) * inv_t - (z_at - s.top) * inv_t - (__log2f(t.sum) - log_sum) * kLn2);
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
            fixed = g * (exp2_of(__builtin_fmaf(z_at - s.top, c, -log_sum)) - p);
        }
        if (in) mark[(index % kMarkBits) >> 5] = 0;
        if (tid == 0) twice[odd ^ 1] = 0;

        T *grad = GRAD ? static_cast<T *>(a.grad_logits) + row * a.grad_stride : nullptr;
        if (GRAD && at_last >= 0) grad[at_last] = ok ? (T)(g * exp2_of(__builtin_fmaf((float)last - s.top, c, -log_sum))) : (T)0.0f;
        Scaled scaled(s.top, c);
        const float over_sum = g * __builtin_amdgcn_rcpf(s.sum);
        float part_of_sum = over_sum * scaled.shrink();
        if (GRAD && ok && __any(scaled.far)) {   // (the same in every lane)
            // The difference in the row's own type: 16-bit logits this large are equal to the largest or so far
            // below it that nothing is left of their exponential, whatever the difference's rounding.
#pragma unroll
            for (int j = 0; j < NV; ++j) {
                float w[n];
                widen(x[j], w, T());
#pragma unroll
                for (int i = 0; i < n; ++i) w[i] -= s.top;
                narrow(w, x[j], T());
            }
            scaled.product = 0.0f;
            part_of_sum = over_sum;
        }
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
                    for (int i = 0; i < n; ++i) y[i] = (T)(part_of_sum * exp2_of(__builtin_fmaf(w[i], c, -scaled.product)));
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
// 64 entries each, the time for 1024 lanes behind it: 8000 logits 28 us, 89; 12000: 45, 93; 30000: 112, 146;
// 50257: 177, 207.  200 rows of 30000: 13.6, 13.5.)
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
