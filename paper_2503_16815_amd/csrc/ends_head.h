// The head of a language model with its softmax cross entropy, the logits never kept.
//
//   z = s h w^T;  lse = log sum_v exp z_v;  loss = lse - z_label
//   d = g (exp(z - lse) - [v == label]);  dh = s d w;  dw = s d^T h
//
// Each row's g is taken apart, g = f 2^e with 1 <= f < 2.  d is rounded to the type with f alone (in 16-bit floats times
// 2^14, so that softmax values down to 1e-9 keep their bits); the powers of two come back in
// dh by the row, in dw with the transposed hidden states relative to the largest: exactly, but for what a 16-bit float cannot hold.
// There a power 2^-r of the largest is divided: four octaves to the hidden states, the next twelve to d, whose row in dh
// gets them back exactly too, the rest to the hidden states.  (All of it in the hidden states, r = 20, an element of 0.0137 was 0.)
// All f are divided by that of the largest
// g, and both sums multiplied by it: where all g are one number, a mean's, the labels' entries, the largest of
// d, so lie just below a power of two, where rounding takes least of them (up to half of what it takes just above).  What the rounding takes from the
// label's entry, mostly the largest of its row, is added to dh afterwards in 32 bits.  Up to 64 positions, where dw is
// bound by writing it, what the rounding takes from every entry is kept in a second array and multiplied too.
//
// Positions without a label are left out first: the others are packed together, so that they cost nothing.
// The loss is one product whose tiles leave each position's softmax sum (largest logit, sum of
// exponentials) behind, joined afterwards.  The gradient takes the vocabulary in pieces: the product
// again, its tiles turned into d as they come out of the matrix units, then dw of the piece, final at
// once, and the piece's part of dh, summed in 32 bits over the pieces.  Four products of 2 n V D operations: bound by the matrix
// units where positions are many, and by reading w where they are few.
//
// Loss and gradient: 8192 x 50257 x 1600 bf16 4.6 ms (1150 TFLOP/s over four products; a library's single product of that size
// 1100), 8192 x 131072 x 4096 bf16 25.5 ms (1380; 1530), 1024 x 8209 x 640 f32 0.30 ms.  Loss alone of one position of 50257 x
// 1600 35 us, of 13 of 131072 x 4096 176 us (6.1 TB/s).
#pragma once
#include "ends_operands.h"
#include "ends_shapes.h"

namespace deft {
namespace {

// ---- positions that count -------------------------------------------------------------------

struct RowsArgs {
    int n, vocab;
    const int32_t *labels;
    int32_t *status;
    float *loss, *lse_out;          // the loss call: zeros for the others
    const float *lse, *row_grad;    // the gradient call: packed too
    int32_t *count, *row_of, *at_of, *label;   // [1], [n] each
    float *lse_packed, *grad_packed, *power;   // [n]: f times d_scale and 2^e (divided: f d_scale 2^-s and 2^(e + s))
    float *most;                    // [4]: of the largest g, with f or, where d is kept in 32 bits, 1: 2^e, 1 / f, f 2^e, f
    float d_scale;
    int whole;                      // d is kept in 32 bits
    int divided;                    // d and the hidden states are 16-bit floats
};

__global__ void __launch_bounds__(1024) rows_kernel(RowsArgs a)
{
    __shared__ int wave_count[16];
    __shared__ float wave_top[16], wave_low[16];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    int base = 0;
    float top = 0.0f, low = INFINITY;
    for (int first = 0; first < a.n; first += 1024) {
        const int i = first + tid;
        const int label = i < a.n ? a.labels[i] : -1;
        const bool in = label >= 0 && label < a.vocab;
        const uint64_t mask = __ballot(in);
        if (lane == 0) wave_count[wave] = __popcll(mask);
        __syncthreads();
        int at = base, all = 0;
#pragma unroll
        for (int w = 0; w < 16; ++w) {
            if (w < wave) at += wave_count[w];
            all += wave_count[w];
        }
        at += __popcll(mask & ((1ull << lane) - 1));
        if (i < a.n) {
            if (a.status) a.status[i] = in || label == -1 ? DEFT_OK : DEFT_ERR_INVALID_ARG;
            a.at_of[i] = in ? at : -1;
            if (in) {
                a.row_of[at] = i;
                a.label[at] = label;
                if (a.row_grad) {
                    const float g = a.row_grad[i], size = fabsf(g);
                    // (Zero, infinity and NaN stay as they are, the smallest numbers have f < 1.  A zero's power is the least that
                    // there is, so that its hidden states are never scaled up, past their type's range; that of infinity and NaN is
                    // above all others: their hidden states stay as they are.)
                    const bool taken = size > 0.0f && size < INFINITY;
                    const int e = taken ? max(ilogbf(size), -100) : size == 0.0f ? -100 : 127;
                    a.lse_packed[at] = a.lse[i];
                    a.grad_packed[at] = (taken ? ldexpf(g, -e) : g) * a.d_scale;
                    a.power[at] = ldexpf(1.0f, e);
                    if (taken) top = fmaxf(top, size), low = fminf(low, size);
                }
            } else if (a.loss) {
                a.loss[i] = 0.0f;
                a.lse_out[i] = 0.0f;
            }
        }
        base += all;
        __syncthreads();
    }
    top = wave_max(top);
    low = -wave_max(-low);
    if (lane == 0) {
        wave_top[wave] = top;
        wave_low[wave] = low;
    }
    __syncthreads();
#pragma unroll
    for (int w = 0; w < 16; ++w) {
        top = fmaxf(top, wave_top[w]);
        low = fminf(low, wave_low[w]);
    }
    const int e = top > 0.0f ? max(ilogbf(top), -100) : 0;
    if (tid == 0) {
        *a.count = base;
        if (a.most) {
            const float f = ldexpf(top, -e), by = a.whole || f < 1.0f ? 1.0f : f, power = ldexpf(1.0f, e);
            a.most[0] = power;
            a.most[1] = 1.0f / by;
            a.most[2] = power * by;
            a.most[3] = by;
        }
    }
    if (!a.divided || low >= ldexpf(1.0f, e - 4)) return;
    for (int at = tid; at < base; at += 1024) {
        const int own = ilogbf(a.power[at]), s = min(max(e - own - 4, 0), 12);
        a.grad_packed[at] = ldexpf(a.grad_packed[at], -s);
        a.power[at] = ldexpf(1.0f, own + s);
    }
}

// ---- operands with a transposed copy ------------------------------------------------------------

template <typename S, typename T, int P>
__global__ void __launch_bounds__(256) pack_kernel(PackArgs a)
{
    typedef S S8 __attribute__((ext_vector_type(8), aligned(sizeof(S))));
    typedef T T8 __attribute__((ext_vector_type(8)));
    constexpr int kPitch = 66;
    __shared__ T tile[P][64][kPitch];
    const int col0 = blockIdx.x * 64, row0 = blockIdx.y * 64, tid = threadIdx.x;
    const int rows = a.rows_dev ? *a.rows_dev : a.rows;
    if (row0 >= (rows + kTile - 1) / kTile * kTile) return;
#pragma unroll
    for (int half = 0; half < 2; ++half) {
        const int r = half * 32 + (tid >> 3), c = (tid & 7) * 8, row = row0 + r, col = col0 + c;
        S x[8] = {};
        if (row < rows) {
            const S *from = static_cast<const S *>(a.src) + (int64_t)(a.row_of ? a.row_of[row] : row) * a.src_stride;
            if (col + 8 <= a.cols) {
                const S8 v = *reinterpret_cast<const S8 *>(from + col);
#pragma unroll
                for (int i = 0; i < 8; ++i) x[i] = v[i];
            } else {
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    if (col + i < a.cols) x[i] = from[col + i];
            }
        }
        T8 y[P];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            if constexpr (P == 3) {
                bf16 s[3];
                split3(x[i], s);
#pragma unroll
                for (int p = 0; p < 3; ++p) y[p][i] = s[p];
            } else {
                y[0][i] = x[i];
            }
        }
#pragma unroll
        for (int p = 0; p < P; ++p)
            *reinterpret_cast<T8 *>(static_cast<T *>(a.out) + p * a.out_plane + (int64_t)row * a.out_ld + col) = y[p];
        const float scale = a.power && row < rows ? fminf(a.power[row] / *a.most, 1.0f) : 1.0f;   // (a power of two)
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            if constexpr (P == 3) {
                bf16 s[3];
                split3(x[i] * scale, s);
#pragma unroll
                for (int p = 0; p < 3; ++p) tile[p][r][c + i] = s[p];
            } else {
                tile[0][r][c + i] = (T)((float)x[i] * scale);
            }
        }
    }
    __syncthreads();
#pragma unroll
    for (int half = 0; half < 2; ++half) {
        const int c = half * 32 + (tid >> 3), r = (tid & 7) * 8;
        if (col0 + c >= a.cols) continue;
#pragma unroll
        for (int p = 0; p < P; ++p) {
            T8 y;
#pragma unroll
            for (int i = 0; i < 8; ++i) y[i] = tile[p][r + i][c];
            *reinterpret_cast<T8 *>(static_cast<T *>(a.out_t) + p * a.t_plane + (int64_t)(col0 + c) * a.t_ld + row0 + r) = y;
        }
    }
}

// ---- joins ----------------------------------------------------------------------------------

struct JoinArgs {
    int tiles, parts_ld;
    const int *count, *row_of;
    const float2 *parts;
    const float *z_label;
    float *loss, *lse;
};

__global__ void __launch_bounds__(256) join_loss_kernel(JoinArgs a)
{
    const int at = blockIdx.x * 4 + (threadIdx.x >> 6), lane = threadIdx.x & 63;
    if (at >= *a.count) return;
    SoftSum s = {-INFINITY, 0.0f};
    for (int t = lane; t < a.tiles; t += kWave) {
        const float2 x = a.parts[(int64_t)at * a.parts_ld + t];
        s = soft_join(s, SoftSum{x.x, x.y});
    }
    const float top = wave_max(s.top);
    const float sum = wave_sum(s.sum == 0.0f ? 0.0f : s.sum * __expf(s.top - top));
    if (lane == 0) {
        const float lse = top + __logf(sum);
        a.lse[a.row_of[at]] = lse;
        a.loss[a.row_of[at]] = lse - a.z_label[at];
    }
}

// Up to 64 positions are not packed together: those without a label are left out here.
struct FewArgs {
    int n, vocab, tiles;
    const int32_t *labels;
    const float2 *parts;
    const float *z_label;
    float *loss, *lse;
    int32_t *status;
};

__global__ void __launch_bounds__(256) join_few_kernel(FewArgs a)
{
    __shared__ SoftSum of_wave[4];
    const int row = blockIdx.x, tid = threadIdx.x;
    const int label = a.labels[row];
    SoftSum s = {-INFINITY, 0.0f};
    for (int t = tid; t < a.tiles; t += 256) {
        const float2 x = a.parts[(int64_t)row * a.tiles + t];
        s = soft_join(s, SoftSum{x.x, x.y});
    }
    const float top = wave_max(s.top);
    s.sum = wave_sum(s.sum == 0.0f ? 0.0f : s.sum * __expf(s.top - top));
    if ((tid & 63) == 0) of_wave[tid >> 6] = SoftSum{top, s.sum};
    __syncthreads();
    if (tid != 0) return;
    s = of_wave[0];
#pragma unroll
    for (int w = 1; w < 4; ++w) s = soft_join(s, of_wave[w]);
    const bool in = label >= 0 && label < a.vocab;
    const float lse = s.top + __logf(s.sum);
    a.lse[row] = in ? lse : 0.0f;
    a.loss[row] = in ? lse - a.z_label[row] : 0.0f;
    if (a.status) a.status[row] = in || label == -1 ? DEFT_OK : DEFT_ERR_INVALID_ARG;
}

// Logits of up to 64 positions in 32 bits, by 32-bit matrix instructions on the rows as they are: bound by reading the
// weights once (one position of 50257 x 1600: 63 us, 5.1 TB/s; 60 positions 189 us, by reading the positions from the
// caches; packed into three 16-bit arrays and multiplied as those, calls of 370 and 388 us for 68 and 186).  A wavefront takes 32 rows of the vocabulary and all positions; a lane loads four
// neighbouring elements of a row, so instruction j of four multiplies elements j, 4 + j, 8 + j, 12 + j of sixteen.
struct FewLogitsArgs {
    int n, vocab, hidden, tiles;
    const float *states, *weight;
    int64_t states_stride, weight_stride;
    float scale;
    const int32_t *labels;
    float2 *parts;                  // [n][tiles]
    float *z_label;
};
constexpr int kFewRows = 128, kFewTiles = kFewRows / 4 / 16;   // rows of a workgroup, tiles of a wavefront

template <int NT>
__global__ void __launch_bounds__(256) few_logits_kernel(FewLogitsArgs a)
{
    typedef float f32x4u __attribute__((ext_vector_type(4), aligned(4)));
    __shared__ float2 joined[4][NT * 16];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, row16 = lane & 15, part = lane >> 4;
    const int m0 = blockIdx.x * kFewRows + wave * (kFewTiles * 16);
    const float *w[kFewTiles], *h[NT];   // (rows past the last one read that one)
#pragma unroll
    for (int i = 0; i < kFewTiles; ++i) w[i] = a.weight + (int64_t)min(m0 + i * 16 + row16, a.vocab - 1) * a.weight_stride;
#pragma unroll
    for (int j = 0; j < NT; ++j) h[j] = a.states + (int64_t)min(j * 16 + row16, a.n - 1) * a.states_stride;
    f32x4 acc[kFewTiles][NT] = {};
    const auto multiply = [&](const f32x4 (&x)[kFewTiles], const f32x4 (&y)[NT]) {
#pragma unroll
        for (int k = 0; k < 4; ++k)
#pragma unroll
            for (int i = 0; i < kFewTiles; ++i)
#pragma unroll
                for (int j = 0; j < NT; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x4f32(x[i][k], y[j][k], acc[i][j], 0, 0, 0);
    };
    constexpr int kAhead = 4;   // steps of 16 that are on their way together
    int k0 = 0;
    for (; k0 + 16 * kAhead <= a.hidden; k0 += 16 * kAhead) {
        f32x4 x[kAhead][kFewTiles], y[kAhead][NT];
#pragma unroll
        for (int s = 0; s < kAhead; ++s) {
            const int k = k0 + s * 16 + part * 4;
#pragma unroll
            for (int i = 0; i < kFewTiles; ++i) x[s][i] = *reinterpret_cast<const f32x4u *>(w[i] + k);
#pragma unroll
            for (int j = 0; j < NT; ++j) y[s][j] = *reinterpret_cast<const f32x4u *>(h[j] + k);
        }
#pragma unroll
        for (int s = 0; s < kAhead; ++s) multiply(x[s], y[s]);
    }
    for (; k0 < a.hidden; k0 += 16) {
        f32x4 x[kFewTiles] = {}, y[NT] = {};
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const int k = k0 + part * 4 + r;
            if (k >= a.hidden) break;
#pragma unroll
            for (int i = 0; i < kFewTiles; ++i) x[i][r] = w[i][k];
#pragma unroll
            for (int j = 0; j < NT; ++j) y[j][r] = h[j][k];
        }
        multiply(x, y);
    }
    // acc[i][j][r] is the logit of row m0 + i * 16 + part * 4 + r and position j * 16 + row16
#pragma unroll
    for (int j = 0; j < NT; ++j) {
        const int n = j * 16 + row16;
        const int label = n < a.n ? a.labels[n] : -1;
        float top = -INFINITY, sum = 0.0f;
#pragma unroll
        for (int i = 0; i < kFewTiles; ++i)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int m = m0 + i * 16 + part * 4 + r;
                acc[i][j][r] *= a.scale;
                if (m < a.vocab) {
                    top = fmaxf(top, acc[i][j][r]);
                    if (m == label) a.z_label[n] = acc[i][j][r];
                }
            }
        top = fmaxf(top, __shfl_xor(top, 16));
        top = fmaxf(top, __shfl_xor(top, 32));
        if (top == -INFINITY) top = kLowest;   // (no row of the vocabulary here, or all -infinity)
#pragma unroll
        for (int i = 0; i < kFewTiles; ++i)
#pragma unroll
            for (int r = 0; r < 4; ++r)
                if (m0 + i * 16 + part * 4 + r < a.vocab) sum += __expf(acc[i][j][r] - top);
        sum += __shfl_xor(sum, 16);
        sum += __shfl_xor(sum, 32);
        if (part == 0) joined[wave][n] = make_float2(top, sum);
    }
    __syncthreads();
    if (tid >= NT * 16 || tid >= a.n) return;
    SoftSum s = {joined[0][tid].x, joined[0][tid].y};
#pragma unroll
    for (int v = 1; v < 4; ++v) s = soft_join(s, SoftSum{joined[v][tid].x, joined[v][tid].y});
    a.parts[(int64_t)tid * a.tiles + blockIdx.x] = make_float2(s.top, s.sum);
}

struct HiddenArgs {
    int n, hidden, splits;
    const int *at_of;
    const float *sums, *power, *factor;
    const float *residual;          // times the label's row of the weights
    const int *label;
    const void *weight;
    int64_t weight_stride;
    int64_t sums_ld, sums_split;
    float scale;
    void *out;
    int64_t out_stride;
};

// A wavefront takes a row, or a part of one where rows are fewer than the card holds wavefronts (1003 rows of 1021 elements
// in 8 parts of a sum: 15.9 us a row each, 8.0 a quarter each; 8192 rows of 1600: 21 and 26).
constexpr int kJoinWaves = 8192;

template <typename O>
__global__ void __launch_bounds__(256) join_hidden_kernel(HiddenArgs a)
{
    const int row = blockIdx.x * 4 + (threadIdx.x >> 6), lane = threadIdx.x & 63;
    if (row >= a.n) return;
    const int at = a.at_of[row];
    O *out = static_cast<O *>(a.out) + (int64_t)row * a.out_stride;
    const float alpha = at >= 0 ? a.power[at] * a.scale * *a.factor : 0.0f;
    for (int c = (blockIdx.y * kWave + lane) * 4; c < a.hidden; c += gridDim.y * kWave * 4) {
        f32x4 x = {0.0f, 0.0f, 0.0f, 0.0f};
        if (at >= 0) {
            const float *sums = a.sums + (int64_t)at * a.sums_ld + c;
            int s = 0;
            for (; s + 8 <= a.splits; s += 8) {   // (eight loads under way)
                f32x4 y[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) y[i] = *reinterpret_cast<const f32x4 *>(sums + (s + i) * a.sums_split);
#pragma unroll
                for (int i = 0; i < 8; ++i) x += y[i];
            }
            for (; s < a.splits; ++s) x += *reinterpret_cast<const f32x4 *>(sums + s * a.sums_split);
            if (a.residual) {
                const O *w = static_cast<const O *>(a.weight) + (int64_t)a.label[at] * a.weight_stride + c;
                const float residual = a.residual[at];
                typedef O O4 __attribute__((ext_vector_type(4), aligned(sizeof(O))));
                if (c + 4 <= a.hidden) {
                    const O4 v = *reinterpret_cast<const O4 *>(w);
#pragma unroll
                    for (int i = 0; i < 4; ++i) x[i] += residual * (float)v[i];
                } else {
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        if (c + i < a.hidden) x[i] += residual * (float)w[i];
                }
            }
            x *= alpha;
        }
        if (c + 4 <= a.hidden) {
            typedef O O4 __attribute__((ext_vector_type(4), aligned(sizeof(O))));
            *reinterpret_cast<O4 *>(out + c) = O4{(O)x[0], (O)x[1], (O)x[2], (O)x[3]};
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (c + i < a.hidden) out[c + i] = (O)x[i];
        }
    }
}

// ---- launches -------------------------------------------------------------------------------

template <typename T, typename O, int E, bool SPLIT>
hipError_t product(const ProductArgs &p, Shape shape, hipStream_t st)
{
    switch (shape) {
    case kMiddle: return product_shape<T, O, E, 2, 4, 6, 4, SPLIT>(p, st);
    case kLow: return product_shape<T, O, E, 2, 4, 5, 4, SPLIT>(p, st);
    case kHalf: return product_shape<T, O, E, 4, 2, 4, 4, SPLIT>(p, st);
    case kSmall: return product_shape<T, O, E, 2, 2, 4, 4, SPLIT>(p, st);
    case kNarrow:
        if constexpr (!SPLIT || E != kSoftmax) return product_shape<T, O, E, 4, 2, 4, 2, SPLIT>(p, st);
        return hipErrorInvalidValue;   // (few_logits_kernel)
    default: return product_shape<T, O, E, 2, 4, 8, 4, SPLIT>(p, st);
    }
}

template <typename T, typename O, int E, bool SPLIT>
hipError_t allow_lds()
{
    hipError_t e = allow_shape<T, O, E, 2, 4, 8, 4, SPLIT>();
    if (e == hipSuccess) e = allow_shape<T, O, E, 2, 4, 6, 4, SPLIT>();
    if (e == hipSuccess) e = allow_shape<T, O, E, 2, 4, 5, 4, SPLIT>();
    if (e == hipSuccess) e = allow_shape<T, O, E, 4, 2, 4, 4, SPLIT>();
    if (e == hipSuccess) e = allow_shape<T, O, E, 2, 2, 4, 4, SPLIT>();
    if constexpr (!SPLIT || E != kSoftmax)
        if (e == hipSuccess) e = allow_shape<T, O, E, 4, 2, 4, 2, SPLIT>();
    return e;
}

template <typename T, typename O, bool SPLIT>
hipError_t allow_all()
{
    hipError_t e = allow_lds<T, O, kSoftmax, SPLIT>();
    if (e == hipSuccess) e = allow_lds<T, O, kDerivative, SPLIT>();
    if (e == hipSuccess) e = allow_lds<T, O, kSums, SPLIT>();
    if (e == hipSuccess) e = allow_lds<T, O, kGradient, SPLIT>();
    return e;
}

// One call's view of the scratch memory.
struct Scratch {
    int32_t *count, *row_of, *at_of, *label;
    float *lse, *grad, *z_label, *power, *most, *residual;
    float2 *parts;
    char *hidden, *weight, *hidden_t, *d;
    float *sums;
    Scratch(const HeadPlan &plan, void *scratch)
    {
        char *s = static_cast<char *>(scratch);
        const int64_t n = up(plan.max_rows, kTile);
        count = reinterpret_cast<int32_t *>(s + plan.ints);
        row_of = count + 64;
        at_of = row_of + n;
        label = at_of + n;
        most = reinterpret_cast<float *>(s + plan.floats);
        lse = most + 64;
        grad = lse + n;
        z_label = grad + n;
        power = z_label + n;
        residual = power + n;
        parts = reinterpret_cast<float2 *>(s + plan.parts);
        hidden = s + plan.hidden;
        weight = s + plan.weight;
        hidden_t = s + plan.hidden_t;
        d = s + plan.d;
        sums = reinterpret_cast<float *>(s + plan.sums);
    }
};

template <typename S, typename T, int P>
struct Head {
    static constexpr bool kSplit = P == 3;
    static constexpr bool kHalf = __is_same(T, f16);

    static hipError_t pack(const PackArgs &a, int rows_to, hipStream_t st)
    {
        if (a.out_t) {
            const dim3 grid((unsigned)(up(a.cols, kStep) / 64), (unsigned)(rows_to / 64));
            pack_kernel<S, T, P><<<grid, 256, 0, st>>>(a);
        } else {
            pack_rows_kernel<S, T, P><<<(unsigned)(up((int64_t)rows_to * (a.out_ld >> 3), 1024) / 1024), 256, 0, st>>>(a);
        }
        return hipGetLastError();
    }

    // hidden states (and, for the gradient, their transpose): of the positions that count, packed together, or of all
    static hipError_t positions(const Scratch &s, const void *hidden_states, int64_t stride, int n, int hidden, bool counted,
                                bool transposed, hipStream_t st)
    {
        const int64_t n_up = up(n, kTile), k = up(hidden, kStep);
        PackArgs h{};
        h.src = hidden_states;
        h.src_stride = stride;
        h.rows = n;
        h.cols = hidden;
        if (counted) {
            h.row_of = s.row_of;
            h.rows_dev = s.count;
        }
        h.out = s.hidden;
        h.out_ld = k;
        h.out_plane = n_up * k;
        if (transposed) {
            h.out_t = s.hidden_t;
            h.t_ld = n_up;
            h.t_plane = n_up * k;
            h.power = s.power;
            h.most = s.most;
        }
        return pack(h, (int)n_up, st);
    }

    // the operands of the logits of the vocabulary's rows `first` .. `first` + `rows` - 1
    static hipError_t logits(const HeadPlan &plan, const Scratch &s, const void *weight, int64_t stride, int first, int rows, int n,
                             int hidden, float scale, ProductArgs *p, hipStream_t st)
    {
        const int64_t k = up(hidden, kStep);
        const S *from = static_cast<const S *>(weight) + (int64_t)first * stride;
        const bool direct = !kSplit && in_place(weight, stride, hidden);
        if (!direct) {
            PackArgs w{};
            w.src = from;
            w.src_stride = stride;
            w.rows = rows;
            w.cols = hidden;
            w.out = s.weight;
            w.out_ld = k;
            w.out_plane = (int64_t)plan.piece * k;
            const hipError_t e = pack(w, (int)up(rows, kTile), st);
            if (e != hipSuccess) return e;
        }
        *p = ProductArgs{};
        p->a = direct ? static_cast<const void *>(from) : s.weight;
        p->a_ld = direct ? stride : k;
        p->a_plane = (int64_t)plan.piece * k;
        p->b = s.hidden;
        p->b_ld = k;
        p->b_plane = up(n, kTile) * k;
        p->m = rows;
        p->n = n;
        p->n_dev = s.count;
        p->k = (int)k;
        p->splits = 1;
        p->scale = scale;
        p->m_first = first;
        p->label = s.label;
        return hipSuccess;
    }

    // up to 64 positions: what their tiles left behind
    static hipError_t join_few(const deft_head_loss_t &a, const Scratch &s, int tiles, hipStream_t st)
    {
        FewArgs f{};
        f.n = a.n_rows;
        f.vocab = a.vocab;
        f.tiles = tiles;
        f.labels = a.labels;
        f.parts = s.parts;
        f.z_label = s.z_label;
        f.loss = a.loss;
        f.lse = a.lse;
        f.status = a.status;
        join_few_kernel<<<a.n_rows, 256, 0, st>>>(f);
        return hipGetLastError();
    }

    static hipError_t few_logits(const deft_head_loss_t &a, const Scratch &s, hipStream_t st)
    {
        FewLogitsArgs f{};
        f.n = a.n_rows;
        f.vocab = a.vocab;
        f.hidden = a.hidden;
        f.tiles = (a.vocab + kFewRows - 1) / kFewRows;
        f.states = static_cast<const float *>(a.hidden_states);
        f.weight = static_cast<const float *>(a.weight);
        f.states_stride = a.hidden_stride;
        f.weight_stride = a.weight_stride;
        f.scale = a.logit_scale;
        f.labels = a.labels;
        f.parts = s.parts;
        f.z_label = s.z_label;
        if (f.n <= 16) few_logits_kernel<1><<<f.tiles, 256, 0, st>>>(f);
        else if (f.n <= 32) few_logits_kernel<2><<<f.tiles, 256, 0, st>>>(f);
        else few_logits_kernel<4><<<f.tiles, 256, 0, st>>>(f);
        const hipError_t e = hipGetLastError();
        return e == hipSuccess ? join_few(a, s, f.tiles, st) : e;
    }

    static hipError_t loss(const HeadPlan &plan, const deft_head_loss_t &a, const Scratch &s, int compute_units, hipStream_t st)
    {
        const int n = a.n_rows;
        const bool few = n <= kFew;
        if constexpr (kSplit)
            if (few) return few_logits(a, s, st);
        const bool from_caller = few && !kSplit && in_place(a.hidden_states, a.hidden_stride, a.hidden);
        hipError_t e = hipSuccess;
        if (!few) {
            RowsArgs r{};
            r.n = n;
            r.vocab = a.vocab;
            r.labels = a.labels;
            r.status = a.status;
            r.loss = a.loss;
            r.lse_out = a.lse;
            r.count = s.count;
            r.row_of = s.row_of;
            r.at_of = s.at_of;
            r.label = s.label;
            rows_kernel<<<1, 1024, 0, st>>>(r);
        }
        if (!from_caller) e = positions(s, a.hidden_states, a.hidden_stride, n, a.hidden, !few, false, st);
        const bool whole = !kSplit && in_place(a.weight, a.weight_stride, a.hidden);   // nothing to pack: no pieces
        const int piece = whole || a.vocab < plan.piece ? a.vocab : plan.piece;
        const int64_t steps = up(a.hidden, kStep) / kStep * (kSplit ? 6 : 1);
        const Shape shape = shape_of(piece, n, steps, 1, compute_units);
        const int tm = kCosts[shape].tm;
        int tiles = 0;
        for (int first = 0; first < a.vocab; first += piece) tiles += ((a.vocab - first < piece ? a.vocab - first : piece) + tm - 1) / tm;
        int parts_first = 0;
        for (int first = 0; first < a.vocab && e == hipSuccess; first += piece) {
            const int rows = a.vocab - first < piece ? a.vocab - first : piece;
            ProductArgs p;
            e = logits(plan, s, a.weight, a.weight_stride, first, rows, n, a.hidden, a.logit_scale, &p, st);
            p.parts = s.parts;
            p.parts_ld = tiles;
            p.parts_first = parts_first;
            parts_first += (rows + tm - 1) / tm;
            p.z_label = s.z_label;
            if (few) {
                p.n_dev = nullptr;
                p.label = a.labels;
            }
            if (from_caller) {
                p.b = a.hidden_states;
                p.b_ld = a.hidden_stride;
            }
            if (e == hipSuccess) e = product<T, S, kSoftmax, kSplit>(p, shape, st);
        }
        if (e != hipSuccess) return e;
        if (few) return join_few(a, s, tiles, st);
        JoinArgs j{};
        j.tiles = tiles;
        j.parts_ld = tiles;
        j.count = s.count;
        j.row_of = s.row_of;
        j.parts = s.parts;
        j.z_label = s.z_label;
        j.loss = a.loss;
        j.lse = a.lse;
        join_loss_kernel<<<(n + 3) / 4, 256, 0, st>>>(j);
        return hipGetLastError();
    }

    static hipError_t gradient(const HeadPlan &plan, const deft_head_grad_t &a, const Scratch &s, int compute_units, hipStream_t st)
    {
        const int n = a.n_rows;
        const int64_t n_up = up(n, kTile), k = up(a.hidden, kStep), sums_ld = up(a.hidden, 4);
        const float d_scale = kHalf ? 16384.0f : 1.0f;   // |softmax - one| f < 2 fills the range of a 16-bit float
        RowsArgs r{};
        r.n = n;
        r.vocab = a.vocab;
        r.labels = a.labels;
        r.lse = a.lse;
        r.row_grad = a.row_grad;
        r.count = s.count;
        r.row_of = s.row_of;
        r.at_of = s.at_of;
        r.label = s.label;
        r.lse_packed = s.lse;
        r.grad_packed = s.grad;
        r.power = s.power;
        r.most = s.most;
        r.d_scale = d_scale;
        r.whole = kSplit;
        r.divided = kHalf;
        rows_kernel<<<1, 1024, 0, st>>>(r);
        hipError_t e = hipGetLastError();
        if (e == hipSuccess && n > 0) e = positions(s, a.hidden_states, a.hidden_stride, n, a.hidden, true, a.grad_weight != nullptr, st);

        const int products = kSplit ? 6 : 1;   // of the arrays that an operand is held in
        const int64_t logit_steps = k / kStep * products, weight_steps = up(n, kStep) / kStep * products;
        const int splits = splits_of(a.hidden, n, up(plan.piece < a.vocab ? plan.piece : a.vocab, kStep) / kStep * products, compute_units);
        const int arrays = n <= kFew && !kSplit ? 2 : 1;
        int piece_number = 0;
        for (int first = 0; first < a.vocab && e == hipSuccess; first += plan.piece, ++piece_number) {
            const int rows = a.vocab - first < plan.piece ? a.vocab - first : plan.piece;
            ProductArgs p{};
            if (n > 0) {
                e = logits(plan, s, a.weight, a.weight_stride, first, rows, n, a.hidden, a.logit_scale, &p, st);
                p.lse = s.lse;
                p.row_grad = s.grad;
                p.row_factor = s.most + 1;
                p.d = s.d;
                p.residual = a.grad_hidden && !kSplit ? s.residual : nullptr;
                p.d_cols = plan.piece;
                p.d_panel = n_up * 256;
                p.d_plane = n_up * plan.piece;
                p.d_arrays = arrays;
                if (e == hipSuccess) e = product<T, S, kDerivative, kSplit>(p, shape_of(rows, n, logit_steps, 1, compute_units), st);
            }
            if (e == hipSuccess && a.grad_weight) {
                ProductArgs q{};
                q.a = s.hidden_t;
                q.a_ld = n_up;
                q.a_plane = n_up * k;
                q.b = s.d;
                q.b_ld = 256;
                q.b_plane = n_up * plan.piece;
                q.d_panel = n_up * 256;
                q.m = a.hidden;
                q.n = rows;
                q.k_dev = s.count;
                q.splits = 1;
                q.scale = a.logit_scale / d_scale;
                q.out_scale = s.most + 2;
                q.d_plane = n_up * plan.piece;
                q.d_arrays = arrays;
                q.add = a.accumulate;
                q.out = static_cast<S *>(a.grad_weight) + (int64_t)first * a.grad_weight_stride;
                q.out_ld = a.grad_weight_stride;
                e = product<T, S, kGradient, kSplit>(q, shape_of(a.hidden, rows, weight_steps, 1, compute_units), st);
            }
            if (e == hipSuccess && piece_number < a.n_piece_events)
                e = hipEventRecord(static_cast<hipEvent_t>(a.piece_events[piece_number]), st);
            if (e == hipSuccess && a.grad_hidden && n > 0) {
                ProductArgs q{};
                q.a = p.a;   // (as the logits' product read it)
                q.a_ld = p.a_ld;
                q.a_plane = p.a_plane;
                q.a_rows = rows;
                q.b = s.d;
                q.b_ld = 256;
                q.b_plane = n_up * plan.piece;
                q.d_panel = n_up * 256;
                q.m = a.hidden;
                q.n = n;
                q.n_dev = s.count;
                q.k = (int)up(rows, kStep);
                q.splits = splits;
                q.sums = s.sums;
                q.sums_ld = sums_ld;
                q.sums_split = n_up * sums_ld;
                q.add = first > 0;
                e = product<T, S, kSums, kSplit>(q, shape_of(a.hidden, n, q.k / kStep * products, splits, compute_units), st);
            }
        }
        for (; e == hipSuccess && piece_number < a.n_piece_events; ++piece_number)   // (bounds past the vocabulary's end)
            e = hipEventRecord(static_cast<hipEvent_t>(a.piece_events[piece_number]), st);
        if (e != hipSuccess || !a.grad_hidden || n == 0) return e;
        HiddenArgs j{};
        j.n = n;
        j.hidden = a.hidden;
        j.splits = splits;
        j.at_of = s.at_of;
        j.sums = s.sums;
        j.power = s.power;
        j.factor = s.most + 3;
        if (!kSplit) {
            j.residual = s.residual;
            j.label = s.label;
            j.weight = a.weight;
            j.weight_stride = a.weight_stride;
        }
        j.sums_ld = sums_ld;
        j.sums_split = n_up * sums_ld;
        j.scale = a.logit_scale / d_scale;
        j.out = a.grad_hidden;
        j.out_stride = a.grad_hidden_stride;
        const int64_t parts = up(a.hidden, 4 * kWave) / (4 * kWave), fill = (kJoinWaves + n - 1) / n;
        join_hidden_kernel<S><<<dim3((n + 3) / 4, (unsigned)(parts < fill ? parts : fill)), 256, 0, st>>>(j);
        return hipGetLastError();
    }
};

}  // namespace
}  // namespace deft
