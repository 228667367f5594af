// Token embedding and its gradient.
//
//   out[n] = scale * table[token_n];   grad_table[v] = scale * sum over {n: token_n = v} of grad_out[n]
//
// Nothing here computes: both are bound by the rows that they move.  The lookup gives each row to a
// wavefront.  The gradient sorts the token numbers (a stable radix sort, so that the rows of a
// token are summed in their own order, whatever the order in which wavefronts run), cuts the sorted list into
// chunks of equal length and sums each chunk's rows token by token.  A token whose rows
// lie in one chunk is written at once; one that spans chunks leaves 32-bit partial sums, which are
// joined in the chunks' order.  So a token that takes half the batch costs no more than others.
#include "ends.h"

namespace deft {
namespace {

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

// The elements at `at` .. `at` + n - 1 of a row of `width`, as floats; beyond the row they are 0.
template <typename T>
__device__ __forceinline__ void load_part(const T *row, int at, int width, float (&x)[Vec<T>::n])
{
    constexpr int n = Vec<T>::n;
    if (at + n <= width) {
        const typename Vec<T>::type v = *reinterpret_cast<const typename Vec<T>::type *>(row + at);
#pragma unroll
        for (int i = 0; i < n; ++i) x[i] = (float)v[i];
    } else {
#pragma unroll
        for (int i = 0; i < n; ++i) x[i] = at + i < width ? (float)row[at + i] : 0.0f;
    }
}

template <typename T>
__device__ __forceinline__ void store_part(T *row, int at, int width, const float (&x)[Vec<T>::n])
{
    constexpr int n = Vec<T>::n;
    if (at + n <= width) {
        typename Vec<T>::type v;
#pragma unroll
        for (int i = 0; i < n; ++i) v[i] = (T)x[i];
        *reinterpret_cast<typename Vec<T>::type *>(row + at) = v;
    } else {
#pragma unroll
        for (int i = 0; i < n; ++i)
            if (at + i < width) row[at + i] = (T)x[i];
    }
}

template <typename T>
__global__ void __launch_bounds__(256) embed_kernel(deft_embed_t e)
{
    const int row = blockIdx.x * 4 + (threadIdx.x >> 6), lane = threadIdx.x & 63;
    if (row >= e.n_rows) return;
    constexpr int n = Vec<T>::n;
    const int token = e.tokens[row];
    const bool in = token >= 0 && token < e.vocab;
    if (lane == 0 && e.status) e.status[row] = in || token == -1 ? DEFT_OK : DEFT_ERR_INVALID_ARG;
    T *out = static_cast<T *>(e.out) + (int64_t)row * e.out_stride;
    const T *from = static_cast<const T *>(e.table) + (int64_t)(in ? token : 0) * e.table_stride;
    for (int at = lane * n; at < e.hidden; at += kWave * n) {
        float x[n] = {};
        if (in) {
            load_part<T>(from, at, e.hidden, x);
#pragma unroll
            for (int i = 0; i < n; ++i) x[i] *= e.scale;
        }
        store_part<T>(out, at, e.hidden, x);
    }
}

// ---- stable radix sort of (token, row) ------------------------------------------------------

constexpr int kSortThreads = 256, kSortItems = 16, kSortBlock = kSortThreads * kSortItems, kDigits = 256;

struct SortArgs {
    int n, vocab, shift;
    const int32_t *tokens;               // the first pass reads these (rows are 0 .. n-1) ...
    const int32_t *keys_in, *rows_in;    // ... the others what the pass before wrote
    int32_t *keys_out, *rows_out;
    int32_t *hist;                       // [kDigits][blocks]
    int blocks;
};

__device__ __forceinline__ int sort_key(const SortArgs &a, int i)
{
    if (!a.tokens) return a.keys_in[i];
    const int t = a.tokens[i];
    return t >= 0 && t < a.vocab ? t : a.vocab;   // tokens that add nothing come last
}

__global__ void __launch_bounds__(kSortThreads) sort_count_kernel(SortArgs a)
{
    __shared__ int count[kDigits];
    count[threadIdx.x] = 0;
    __syncthreads();
    const int base = blockIdx.x * kSortBlock;
    for (int r = 0; r < kSortItems; ++r) {
        const int i = base + r * kSortThreads + threadIdx.x;
        if (i < a.n) atomicAdd(&count[(sort_key(a, i) >> a.shift) & (kDigits - 1)], 1);
    }
    __syncthreads();
    a.hist[threadIdx.x * a.blocks + blockIdx.x] = count[threadIdx.x];
}

// exclusive prefix sums over all digits and blocks, in place
__global__ void __launch_bounds__(1024) sort_scan_kernel(int32_t *hist, int n)
{
    __shared__ int wave_total[16];
    int carry = 0;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    for (int base = 0; base < n; base += 1024) {
        const int i = base + threadIdx.x;
        const int own = i < n ? hist[i] : 0;
        int x = own;
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
            const int y = __shfl_up(x, d);
            if (lane >= d) x += y;
        }
        if (lane == 63) wave_total[wave] = x;
        __syncthreads();
        int before = 0, all = 0;
#pragma unroll
        for (int w = 0; w < 16; ++w) {
            if (w < wave) before += wave_total[w];
            all += wave_total[w];
        }
        __syncthreads();
        if (i < n) hist[i] = carry + before + x - own;
        carry += all;
    }
}

// the lanes whose digit is this lane's
__device__ __forceinline__ uint64_t same_digit(int digit, bool valid)
{
    uint64_t m = __ballot(valid);
#pragma unroll
    for (int b = 0; b < 8; ++b) {
        const uint64_t v = __ballot((digit >> b) & 1);
        m &= ((digit >> b) & 1) ? v : ~v;
    }
    return m;
}

__global__ void __launch_bounds__(kSortThreads) sort_place_kernel(SortArgs a)
{
    __shared__ int next[kDigits];              // where the block's next item of a digit goes
    __shared__ int in_wave[4][kDigits];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    next[tid] = a.hist[tid * a.blocks + blockIdx.x];
    const int base = blockIdx.x * kSortBlock;
    for (int r = 0; r < kSortItems && base + r * kSortThreads < a.n; ++r) {
#pragma unroll
        for (int w = 0; w < 4; ++w) in_wave[w][tid] = 0;
        __syncthreads();
        const int i = base + r * kSortThreads + tid;
        const bool valid = i < a.n;
        const int key = valid ? sort_key(a, i) : 0;
        const int row = valid ? (a.tokens ? i : a.rows_in[i]) : 0;
        const int digit = (key >> a.shift) & (kDigits - 1);
        const uint64_t same = same_digit(digit, valid);
        const int rank = __popcll(same & ((1ull << lane) - 1));
        if (valid && rank == 0) in_wave[wave][digit] = __popcll(same);
        __syncthreads();
        if (valid) {
            int at = next[digit] + rank;
            for (int w = 0; w < wave; ++w) at += in_wave[w][digit];
            a.keys_out[at] = key;
            a.rows_out[at] = row;
        }
        __syncthreads();
        next[tid] += in_wave[0][tid] + in_wave[1][tid] + in_wave[2][tid] + in_wave[3][tid];
        __syncthreads();
    }
}

// ---- sums over the sorted rows --------------------------------------------------------------

constexpr int kChunk = 32, kBatch = 8;

struct SumArgs {
    int n, vocab, hidden, accumulate, chunks;
    int lanes;            // threads that share a chunk: a power of two, 16 bytes of the row each
    float scale;
    const int32_t *keys, *rows;
    const void *grad_out;
    int64_t grad_out_stride;
    void *grad_table;
    int64_t grad_table_stride;
    float *partial;       // [chunks][2][hidden]: of the run that a chunk begins in, of the one it ends in
};

template <typename T>
__device__ __forceinline__ void write_sum(const SumArgs &a, int token, int at, const float (&acc)[Vec<T>::n])
{
    constexpr int n = Vec<T>::n;
    T *row = static_cast<T *>(a.grad_table) + (int64_t)token * a.grad_table_stride;
    float x[n];
    if (a.accumulate) {
        load_part<T>(row, at, a.hidden, x);
#pragma unroll
        for (int i = 0; i < n; ++i) x[i] += a.scale * acc[i];
    } else {
#pragma unroll
        for (int i = 0; i < n; ++i) x[i] = a.scale * acc[i];
    }
    store_part<T>(row, at, a.hidden, x);
}

template <typename T>
__device__ __forceinline__ void write_partial(const SumArgs &a, int chunk, int which, int at, const float (&acc)[Vec<T>::n])
{
    float *p = a.partial + ((int64_t)chunk * 2 + which) * a.hidden;
#pragma unroll
    for (int i = 0; i < Vec<T>::n; ++i)
        if (at + i < a.hidden) p[at + i] = acc[i];
}

template <typename T>
__global__ void __launch_bounds__(256) embed_sum_kernel(SumArgs a)
{
    constexpr int n = Vec<T>::n;
    const int per_block = 256 / a.lanes;
    const int chunk = blockIdx.x * per_block + threadIdx.x / a.lanes;
    const int at = (blockIdx.y * a.lanes + threadIdx.x % a.lanes) * n;
    if (chunk >= a.chunks || at >= a.hidden) return;
    const int first = chunk * kChunk, last = min(first + kChunk, a.n);
    int token = a.keys[first];
    bool from_left = first > 0 && a.keys[first - 1] == token;
    float acc[n] = {};
    for (int p = first; p < last; p += kBatch) {
        int key[kBatch];
        float x[kBatch][n];
#pragma unroll
        for (int j = 0; j < kBatch; ++j) {   // a batch's rows are on their way together
            key[j] = p + j < last ? a.keys[p + j] : a.vocab;
#pragma unroll
            for (int i = 0; i < n; ++i) x[j][i] = 0.0f;
            if (key[j] < a.vocab)
                load_part<T>(static_cast<const T *>(a.grad_out) + (int64_t)a.rows[p + j] * a.grad_out_stride, at, a.hidden, x[j]);
        }
#pragma unroll
        for (int j = 0; j < kBatch; ++j) {
            if (p + j >= last) break;
            if (key[j] != token) {
                if (token < a.vocab) {
                    if (from_left) write_partial<T>(a, chunk, 0, at, acc);
                    else write_sum<T>(a, token, at, acc);
                }
                token = key[j];
                from_left = false;
#pragma unroll
                for (int i = 0; i < n; ++i) acc[i] = 0.0f;
            }
#pragma unroll
            for (int i = 0; i < n; ++i) acc[i] += x[j][i];
        }
    }
    if (token >= a.vocab) return;
    const bool to_right = last < a.n && a.keys[last] == token;
    if (from_left) write_partial<T>(a, chunk, 0, at, acc);
    else if (to_right) write_partial<T>(a, chunk, 1, at, acc);
    else write_sum<T>(a, token, at, acc);
}

// the runs that begin in a chunk and go on in the next ones
template <typename T>
__global__ void __launch_bounds__(256) embed_join_kernel(SumArgs a)
{
    constexpr int n = Vec<T>::n;
    const int per_block = 256 / a.lanes;
    const int chunk = blockIdx.x * per_block + threadIdx.x / a.lanes;
    const int at = (blockIdx.y * a.lanes + threadIdx.x % a.lanes) * n;
    if (chunk >= a.chunks || at >= a.hidden) return;
    const int first = chunk * kChunk, end = first + kChunk;
    if (end >= a.n) return;
    const int token = a.keys[end - 1];
    if (token >= a.vocab || a.keys[end] != token) return;               // nothing goes on
    if (a.keys[first] == token && first > 0 && a.keys[first - 1] == token) return;   // it began further left
    float acc[n];
    load_part<float>(a.partial + ((int64_t)chunk * 2 + 1) * a.hidden, at, a.hidden, reinterpret_cast<float(&)[4]>(acc[0]));
    if (n == 8) load_part<float>(a.partial + ((int64_t)chunk * 2 + 1) * a.hidden, at + 4, a.hidden, reinterpret_cast<float(&)[4]>(acc[n - 4]));
    for (int c = chunk + 1; c < a.chunks && a.keys[c * kChunk] == token; ++c) {
        const float *p = a.partial + (int64_t)c * 2 * a.hidden;
#pragma unroll
        for (int k = 0; k < n; k += 4) {
            float x[4];
            load_part<float>(p, at + k, a.hidden, x);
#pragma unroll
            for (int i = 0; i < 4; ++i) acc[k + i] += x[i];
        }
    }
    write_sum<T>(a, token, at, acc);
}

template <typename T>
__global__ void __launch_bounds__(256) zero_rows_kernel(T *table, int64_t stride, int vocab, int hidden)
{
    constexpr int n = Vec<T>::n;
    const float zero[n] = {};
    for (int row = blockIdx.x * 4 + (threadIdx.x >> 6); row < vocab; row += gridDim.x * 4)
        for (int at = (threadIdx.x & 63) * n; at < hidden; at += kWave * n)
            store_part<T>(table + (int64_t)row * stride, at, hidden, zero);
}

int bits_of(int x)
{
    int b = 0;
    while (x >> b) ++b;
    return b;
}

struct Layout {
    int64_t keys_a, rows_a, keys_b, rows_b, hist, partial, bytes;
};

Layout layout(int64_t rows, int64_t hidden)
{
    Layout l;
    int64_t at = 0;
    const auto take = [&](int64_t bytes) {
        const int64_t here = at;
        at += (bytes + 255) / 256 * 256;
        return here;
    };
    l.keys_a = take(rows * 4);
    l.rows_a = take(rows * 4);
    l.keys_b = take(rows * 4);
    l.rows_b = take(rows * 4);
    l.hist = take((rows + kSortBlock - 1) / kSortBlock * kDigits * 4);
    l.partial = take((rows + kChunk - 1) / kChunk * 2 * hidden * 4);
    l.bytes = at;
    return l;
}

template <typename T>
hipError_t grad_launch(const EmbedPlan &plan, const deft_embed_grad_t &e, char *scratch, hipStream_t st)
{
    T *table = static_cast<T *>(e.grad_table);
    if (!e.accumulate) {
        const int blocks = (e.vocab + 3) / 4;
        zero_rows_kernel<T><<<blocks < 4096 ? blocks : 4096, 256, 0, st>>>(table, e.grad_table_stride, e.vocab, e.hidden);
    }
    if (e.n_rows == 0) return hipGetLastError();
    const Layout l = layout(plan.max_rows, plan.max_hidden);
    int32_t *keys[2] = {reinterpret_cast<int32_t *>(scratch + l.keys_a), reinterpret_cast<int32_t *>(scratch + l.keys_b)};
    int32_t *rows[2] = {reinterpret_cast<int32_t *>(scratch + l.rows_a), reinterpret_cast<int32_t *>(scratch + l.rows_b)};
    SortArgs s{};
    s.n = e.n_rows;
    s.vocab = e.vocab;
    s.hist = reinterpret_cast<int32_t *>(scratch + l.hist);
    s.blocks = (e.n_rows + kSortBlock - 1) / kSortBlock;
    const int bits = bits_of(e.vocab);
    int out = 0;
    for (int shift = 0; shift < bits; shift += 8, out ^= 1) {
        s.shift = shift;
        s.tokens = shift == 0 ? e.tokens : nullptr;
        s.keys_in = keys[out ^ 1];
        s.rows_in = rows[out ^ 1];
        s.keys_out = keys[out];
        s.rows_out = rows[out];
        sort_count_kernel<<<s.blocks, kSortThreads, 0, st>>>(s);
        sort_scan_kernel<<<1, 1024, 0, st>>>(s.hist, s.blocks * kDigits);
        sort_place_kernel<<<s.blocks, kSortThreads, 0, st>>>(s);
    }
    out ^= 1;
    SumArgs a{};
    a.n = e.n_rows;
    a.vocab = e.vocab;
    a.hidden = e.hidden;
    a.accumulate = e.accumulate;
    a.scale = e.scale;
    a.keys = keys[out];
    a.rows = rows[out];
    a.grad_out = e.grad_out;
    a.grad_out_stride = e.grad_out_stride;
    a.grad_table = e.grad_table;
    a.grad_table_stride = e.grad_table_stride;
    a.partial = reinterpret_cast<float *>(scratch + l.partial);
    a.chunks = (e.n_rows + kChunk - 1) / kChunk;
    const int parts = (e.hidden + Vec<T>::n - 1) / Vec<T>::n;
    a.lanes = 8;
    while (a.lanes < parts && a.lanes < 256) a.lanes *= 2;
    const int per_block = 256 / a.lanes;
    const dim3 grid((a.chunks + per_block - 1) / per_block, (parts + a.lanes - 1) / a.lanes);
    embed_sum_kernel<T><<<grid, 256, 0, st>>>(a);
    if (a.chunks > 1) embed_join_kernel<T><<<grid, 256, 0, st>>>(a);
    return hipGetLastError();
}

}  // namespace

void embed_grad_plan(int max_rows, int max_vocab, int max_hidden, EmbedPlan *plan)
{
    plan->max_rows = max_rows;
    plan->max_vocab = max_vocab;
    plan->max_hidden = max_hidden;
    plan->scratch_bytes = layout(max_rows, max_hidden).bytes;
}

hipError_t embed_launch(int dtype, const deft_embed_t &e, hipStream_t st)
{
    const int blocks = (e.n_rows + 3) / 4;
    if (dtype == DEFT_F32) embed_kernel<float><<<blocks, 256, 0, st>>>(e);
    else if (dtype == DEFT_F16) embed_kernel<f16><<<blocks, 256, 0, st>>>(e);
    else embed_kernel<bf16><<<blocks, 256, 0, st>>>(e);
    return hipGetLastError();
}

hipError_t embed_grad_launch(const EmbedPlan &plan, int dtype, const deft_embed_grad_t &e, void *scratch, int, hipStream_t st)
{
    char *s = static_cast<char *>(scratch);
    if (dtype == DEFT_F32) return grad_launch<float>(plan, e, s, st);
    if (dtype == DEFT_F16) return grad_launch<f16>(plan, e, s, st);
    return grad_launch<bf16>(plan, e, s, st);
}

}  // namespace deft
