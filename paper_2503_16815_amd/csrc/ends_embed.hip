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
// 16384 rows of 1600 bf16, vocabulary 50257: lookup 18 us (5.7 TB/s read and written), gradient 58 us: sorting beside the
// table's zeros (161 MB) 29 us, sums 18, joins 11; 65536 rows: lookup 61 us, zeros 21, sort by radix 57, sums 77, joins 9.
#include "ends.h"

namespace deft {
namespace {

// The 16 bytes from element `at` of a row of `width` on; beyond the row they are 0.
template <typename T>
__device__ __forceinline__ typename Vec<T>::type load_part(const T *row, int at, int width)
{
    constexpr int n = Vec<T>::n;
    if (at + n <= width) return *reinterpret_cast<const typename Vec<T>::type *>(row + at);
    typename Vec<T>::type v = {};
#pragma unroll
    for (int i = 0; i < n; ++i)
        if (at + i < width) v[i] = row[at + i];
    return v;
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
    constexpr int kAhead = 4;   // vectors of a lane that are on their way together
    for (int first = lane * n; first < e.hidden; first += kWave * n * kAhead) {
        typename Vec<T>::type v[kAhead];
#pragma unroll
        for (int j = 0; j < kAhead; ++j) {
            const int at = first + j * kWave * n;
            v[j] = typename Vec<T>::type{};
            if (in && at < e.hidden) v[j] = load_part<T>(from, at, e.hidden);
        }
#pragma unroll
        for (int j = 0; j < kAhead; ++j) {
            const int at = first + j * kWave * n;
            float x[n];
#pragma unroll
            for (int i = 0; i < n; ++i) x[i] = in ? e.scale * (float)v[j][i] : 0.0f;
            if (at < e.hidden) store_part<T>(out, at, e.hidden, x);
        }
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

// ---- up to 16384 rows: two launches ---------------------------------------------------------

// A token number and its row fit one word (18 and 14 bits); no two words are the same, so any sort of them is the stable
// one.  The first launch sorts lists of 1024 words, a workgroup each.  The second finds each word's place: its
// place in its own list plus, by bisection, the words of every other list below it.  The other workgroups of
// both launches clear half of the table each; the rows that have tokens are written again by the sums, which costs
// less than finding out which these are.  (Measured on 16384 tokens of a vocabulary of 50257: radix sort in memory,
// six launches, 50 us; radix sort by one workgroup in registers and LDS 32 us, bound by the instructions of a
// single compute unit; this 18 us.)
constexpr int kListBits = 10, kList = 1 << kListBits, kSmallThreads = 1024, kSmallWaves = kSmallThreads / kWave;
constexpr int kRowBits = 14, kSmall = 1 << kRowBits, kSmallVocab = 1 << (32 - kRowBits);
constexpr int kRanked = 256, kShare = kSmallThreads / kRanked;   // words that a workgroup places, lanes to a word

struct SmallArgs {
    int n, vocab, hidden, lists;
    int workers;               // workgroups that sort; the others clear
    int clear_from, clear_to;  // rows of the table
    const int32_t *tokens;
    unsigned *words;
    int32_t *keys, *rows;
    void *table;
    int64_t stride;
};

// This workgroup's share of the rows; rows that follow one another are one stretch (measured on 41348 rows of 1944 32-bit
// elements: 5.7 TB/s, row by row 5.4).
template <typename T>
__device__ __forceinline__ void clear_rows(const SmallArgs &a)
{
    const int share = blockIdx.x - a.workers, shares = gridDim.x - a.workers, rows = a.clear_to - a.clear_from;
    const int from = a.clear_from + (int)((int64_t)rows * share / shares);
    const int to = a.clear_from + (int)((int64_t)rows * (share + 1) / shares);
    constexpr int n = Vec<T>::n;
    const float zero[n] = {};
    T *const first = static_cast<T *>(a.table) + (int64_t)from * a.stride;
    if (a.stride == a.hidden) {
        const int64_t length = (int64_t)(to - from) * a.hidden;
        int64_t head = (int64_t)(-(uintptr_t)first & 127) / (int64_t)sizeof(T);   // to a cache line's boundary
        if (head > length) head = length;
        const int64_t whole = (length - head) / n * n, rest = length - whole;
        for (int64_t i = threadIdx.x; i < rest; i += kSmallThreads) first[i < head ? i : whole + i] = (T)0.0f;
        for (int64_t at = head + (int64_t)threadIdx.x * n; at < head + whole; at += (int64_t)kSmallThreads * n)
            *reinterpret_cast<typename Vec<T>::type *>(first + at) = typename Vec<T>::type{};
        return;
    }
    for (int row = from + (int)(threadIdx.x >> 6); row < to; row += kSmallWaves) {
        T *to_row = first + (int64_t)(row - from) * a.stride;
        for (int at = (threadIdx.x & 63) * n; at < a.hidden; at += kWave * n) store_part<T>(to_row, at, a.hidden, zero);
    }
}

__device__ __forceinline__ void write_place(const SmallArgs &a, int at, unsigned word)
{
    a.keys[at] = (int32_t)(word >> kRowBits);
    a.rows[at] = (int32_t)(word & (kSmall - 1));
}

template <typename T>
__global__ void __launch_bounds__(kSmallThreads) sort_lists_kernel(SmallArgs a)
{
    __shared__ unsigned other[kList];
    if ((int)blockIdx.x >= a.workers) {
        clear_rows<T>(a);
        return;
    }
    const int tid = threadIdx.x, i = blockIdx.x * kList + tid;
    unsigned word = ~0u;   // beyond the list: after all others
    if (i < a.n) {
        const int t = a.tokens[i];
        word = (unsigned)(t >= 0 && t < a.vocab ? t : a.vocab) << kRowBits | (unsigned)i;   // tokens that add nothing come last
    }
    for (int size = 2; size <= kList; size <<= 1)          // bitonic: runs of `size` become sorted
        for (int d = size >> 1; d > 0; d >>= 1) {
            unsigned with;
            if (d >= kWave) {
                __syncthreads();
                other[tid] = word;
                __syncthreads();
                with = other[tid ^ d];
            } else {
                with = __shfl_xor(word, d);
            }
            const bool up = (tid & size) == 0, first = (tid & d) == 0;
            word = up == first ? min(word, with) : max(word, with);
        }
    if (i >= a.n) return;                                  // (as many words as tokens come before the fill)
    if (a.lists == 1) write_place(a, i, word);
    else a.words[i] = word;
}

template <typename T>
__global__ void __launch_bounds__(kSmallThreads) place_words_kernel(SmallArgs a)
{
    __shared__ unsigned words[kSmall];
    if ((int)blockIdx.x >= a.workers) {
        clear_rows<T>(a);
        return;
    }
    const int tid = threadIdx.x;
    for (int i = tid; i < a.lists * kList; i += kSmallThreads) words[i] = i < a.n ? a.words[i] : ~0u;
    __syncthreads();
    const int i = blockIdx.x * kRanked + tid / kShare, own = i >> kListBits;
    const unsigned word = i < a.n ? words[i] : 0;
    int below = 0;
    for (int list = tid % kShare; list < a.lists; list += kShare) {
        const unsigned *w = words + list * kList;
        int at = 0;
#pragma unroll
        for (int d = kList / 2; d > 0; d >>= 1) at += w[at + d - 1] < word ? d : 0;
        at += w[at] < word ? 1 : 0;
        below += list == own ? i & (kList - 1) : at;
    }
    below += __shfl_xor(below, 1);
    below += __shfl_xor(below, 2);
    if (i < a.n && tid % kShare == 0) write_place(a, below, word);
}

// ---- sums over the sorted rows --------------------------------------------------------------

constexpr int kBatch = 8, kJoin = 16;

struct SumArgs {
    int n, vocab, hidden, accumulate, chunk, chunks;
    int lanes;            // threads that share a chunk: a power of two, 16 bytes of the row each
    float scale;
    const int32_t *keys, *rows;
    const void *grad_out;
    int64_t grad_out_stride;
    void *grad_table;
    int64_t grad_table_stride;
    float *partial;       // [chunks][2][width]: of the run that a chunk begins in, of the one it ends in
    int width;            // of a partial sum's row: hidden, rounded up to a lane's part
};

// Chunks of 16 rows keep 16384 tokens' rows on four workgroups per compute unit; longer lists have longer chunks, so
// that a token with many rows leaves no more than a few thousand partial sums.
int chunk_of(int n)
{
    const int c = (n + 1023) / 1024;
    return c <= 16 ? 16 : c >= 256 ? 256 : (c + 7) / 8 * 8;
}

template <typename T>
__device__ __forceinline__ void write_sum(const SumArgs &a, int token, int at, const float (&acc)[Vec<T>::n])
{
    constexpr int n = Vec<T>::n;
    T *row = static_cast<T *>(a.grad_table) + (int64_t)token * a.grad_table_stride;
    float x[n];
#pragma unroll
    for (int i = 0; i < n; ++i) x[i] = a.scale * acc[i];
    if (a.accumulate) {
        const typename Vec<T>::type v = load_part<T>(row, at, a.hidden);
#pragma unroll
        for (int i = 0; i < n; ++i) x[i] += (float)v[i];
    }
    store_part<T>(row, at, a.hidden, x);
}

template <int N>
__device__ __forceinline__ void write_partial(const SumArgs &a, int chunk, int which, int at, const float (&acc)[N])
{
    float *p = a.partial + ((int64_t)chunk * 2 + which) * a.width + at;
#pragma unroll
    for (int i = 0; i < N; i += 4) *reinterpret_cast<f32x4 *>(p + i) = f32x4{acc[i], acc[i + 1], acc[i + 2], acc[i + 3]};
}

template <typename T>
__global__ void __launch_bounds__(256) embed_sum_kernel(SumArgs a)
{
    constexpr int n = Vec<T>::n;
    const int per_block = 256 / a.lanes;
    const int chunk = blockIdx.x * per_block + threadIdx.x / a.lanes;
    const int at = (blockIdx.y * a.lanes + threadIdx.x % a.lanes) * n;
    if (chunk >= a.chunks || at >= a.hidden) return;
    const int first = chunk * a.chunk, last = min(first + a.chunk, a.n);
    int token = a.keys[first];
    bool from_left = first > 0 && a.keys[first - 1] == token;
    float acc[n] = {};
    for (int p = first; p < last; p += kBatch) {
        int key[kBatch], row[kBatch];
        typename Vec<T>::type x[kBatch];
#pragma unroll
        for (int j = 0; j < kBatch; ++j) {
            const int i = min(p + j, last - 1);
            key[j] = a.keys[i];
            row[j] = a.rows[i];
        }
#pragma unroll
        for (int j = 0; j < kBatch; ++j) {   // a batch's rows are on their way together
            x[j] = typename Vec<T>::type{};
            if (key[j] < a.vocab)
                x[j] = load_part<T>(static_cast<const T *>(a.grad_out) + (int64_t)row[j] * a.grad_out_stride, at, a.hidden);
        }
#pragma unroll
        for (int j = 0; j < kBatch; ++j) {
            if (p + j >= last) break;
            if (key[j] != token) {
                if (token < a.vocab) {
                    if (from_left) write_partial(a, chunk, 0, at, acc);
                    else write_sum<T>(a, token, at, acc);
                }
                token = key[j];
                from_left = false;
#pragma unroll
                for (int i = 0; i < n; ++i) acc[i] = 0.0f;
            }
#pragma unroll
            for (int i = 0; i < n; ++i) acc[i] += (float)x[j][i];
        }
    }
    if (token >= a.vocab) return;
    const bool to_right = last < a.n && a.keys[last] == token;
    if (from_left) write_partial(a, chunk, 0, at, acc);
    else if (to_right) write_partial(a, chunk, 1, at, acc);
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
    const int first = chunk * a.chunk, end = first + a.chunk;
    if (end >= a.n) return;
    const int token = a.keys[end - 1];
    if (token >= a.vocab || a.keys[end] != token) return;               // nothing goes on
    if (a.keys[first] == token && first > 0 && a.keys[first - 1] == token) return;   // it began further left
    float acc[n];
    const float *p = a.partial + ((int64_t)chunk * 2 + 1) * a.width + at;
#pragma unroll
    for (int i = 0; i < n; ++i) acc[i] = p[i];
    p = a.partial + at;
    bool on = true;
    for (int c = chunk + 1; on && c < a.chunks; c += kJoin) {   // several chunks' sums are on their way together
        int key[kJoin];
        f32x4 x[kJoin][n / 4];
#pragma unroll
        for (int j = 0; j < kJoin; ++j) {
            const int from = min(c + j, a.chunks - 1);
            key[j] = c + j < a.chunks ? a.keys[from * a.chunk] : -1;
#pragma unroll
            for (int k = 0; k < n / 4; ++k)
                x[j][k] = *reinterpret_cast<const f32x4 *>(p + (int64_t)from * 2 * a.width + k * 4);
        }
#pragma unroll
        for (int j = 0; j < kJoin; ++j) {
            on = on && key[j] == token;
            if (on) {
#pragma unroll
                for (int i = 0; i < n; ++i) acc[i] += x[j][i / 4][i % 4];
            }
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
    const int64_t by_16 = (rows + 15) / 16, by_256 = (rows + 255) / 256;
    const int64_t chunks = by_16 < 1024 ? by_16 : by_256 > 1024 ? by_256 : 1024;   // the most of any shorter list
    l.partial = take(chunks * 2 * ((hidden + 7) / 8 * 8) * 4);
    l.bytes = at;
    return l;
}

template <typename T>
hipError_t grad_launch(const EmbedPlan &plan, const deft_embed_grad_t &e, char *scratch, int compute_units, hipStream_t st)
{
    T *table = static_cast<T *>(e.grad_table);
    const Layout l = layout(plan.max_rows, plan.max_hidden);
    int32_t *keys[2] = {reinterpret_cast<int32_t *>(scratch + l.keys_a), reinterpret_cast<int32_t *>(scratch + l.keys_b)};
    int32_t *rows[2] = {reinterpret_cast<int32_t *>(scratch + l.rows_a), reinterpret_cast<int32_t *>(scratch + l.rows_b)};
    const int bits = bits_of(e.vocab);
    int out = 0;
    if (e.n_rows > 0 && e.n_rows <= kSmall && e.vocab < kSmallVocab) {
        SmallArgs s{};
        s.n = e.n_rows;
        s.vocab = e.vocab;
        s.hidden = e.hidden;
        s.lists = (e.n_rows + kList - 1) / kList;
        s.tokens = e.tokens;
        s.words = reinterpret_cast<unsigned *>(scratch + l.keys_b);
        s.keys = keys[0];
        s.rows = rows[0];
        s.table = table;
        s.stride = e.grad_table_stride;
        const auto clearers = [&](int rows_to_clear, int workers) {
            const int most = 2 * compute_units > workers ? 2 * compute_units - workers : 1;
            return e.accumulate ? 0 : rows_to_clear < most ? rows_to_clear : most;
        };
        s.workers = s.lists;
        s.clear_to = s.lists == 1 ? e.vocab : e.vocab / 2;
        sort_lists_kernel<T><<<s.workers + clearers(s.clear_to, s.workers), kSmallThreads, 0, st>>>(s);
        if (s.lists > 1) {
            s.workers = (e.n_rows + kRanked - 1) / kRanked;
            s.clear_from = s.clear_to;
            s.clear_to = e.vocab;
            place_words_kernel<T><<<s.workers + clearers(s.clear_to - s.clear_from, s.workers), kSmallThreads, 0, st>>>(s);
        }
    } else {
        if (!e.accumulate) {
            const int blocks = (e.vocab + 3) / 4;
            zero_rows_kernel<T><<<blocks < 4096 ? blocks : 4096, 256, 0, st>>>(table, e.grad_table_stride, e.vocab, e.hidden);
        }
        if (e.n_rows == 0) return hipGetLastError();
        SortArgs s{};
        s.n = e.n_rows;
        s.vocab = e.vocab;
        s.hist = reinterpret_cast<int32_t *>(scratch + l.hist);
        s.blocks = (e.n_rows + kSortBlock - 1) / kSortBlock;
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
    }
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
    a.width = (e.hidden + 7) / 8 * 8;
    a.chunk = chunk_of(e.n_rows);
    a.chunks = (e.n_rows + a.chunk - 1) / a.chunk;
    const int parts = (e.hidden + Vec<T>::n - 1) / Vec<T>::n;
    a.lanes = 8;
    while (a.lanes < parts && a.lanes < 256) a.lanes *= 2;
    const int per_block = 256 / a.lanes;
    const dim3 grid((a.chunks + per_block - 1) / per_block, (parts + a.lanes - 1) / a.lanes);
    embed_sum_kernel<T><<<grid, 256, 0, st>>>(a);
    if (a.chunks > 1) {   // a long run's sums are spread over several compute units by their columns
        a.lanes = a.lanes < 32 ? a.lanes : 32;
        const int joined = 256 / a.lanes;
        embed_join_kernel<T><<<dim3((a.chunks + joined - 1) / joined, (parts + a.lanes - 1) / a.lanes), 256, 0, st>>>(a);
    }
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

hipError_t embed_grad_launch(const EmbedPlan &plan, int dtype, const deft_embed_grad_t &e, void *scratch, int compute_units,
                             hipStream_t st)
{
    char *s = static_cast<char *>(scratch);
    if (dtype == DEFT_F32) return grad_launch<float>(plan, e, s, compute_units, st);
    if (dtype == DEFT_F16) return grad_launch<f16>(plan, e, s, compute_units, st);
    return grad_launch<bf16>(plan, e, s, compute_units, st);
}

}  // namespace deft
