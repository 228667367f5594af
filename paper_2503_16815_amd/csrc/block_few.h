// The feed-forward block of up to 64 tokens, as a program that generates them calls it.
//
// Bound by reading the three matrices once (13 tokens of 4096 x 12288 bf16 61 us in both launches, 5.0 TB/s; one of 1600 x 6400 18, of which
// a third is latency).  Nothing is packed: a wavefront takes sixteen rows of a matrix at a time, 16 bytes a
// lane from memory to the matrix instructions, and eight or sixteen wavefronts share a workgroup's rows along their length (an
// inner product's terms may come in any order, as long as both operands' do in the same; a tile of 32-bit operands takes
// four instructions, one for each element of a lane's 16 bytes).  The wavefronts' sums meet in LDS.
//
// Of up to 8 tokens the hidden activations go from the first launch to the second as two numbers of the type, the rounded one and
// what the rounding took, which are the two halves of a tile's sixteen rows: so y is rounded once.  Of more they are a second
// tile: of 9 to 16 that costs more than it is worth (16 tokens of 1600 x 6400 bf16 30 us for 24), of 17 to 32 it is done where asked.
#pragma once
#include "block_epilogue.h"
#include "ends_shapes.h"

namespace deft {
namespace {

constexpr int kGateWaves = 8, kOutWaves = 16;   // that share a workgroup's rows

template <typename S> struct FewTile;   // how a wavefront multiplies sixteen rows by sixteen
template <> struct FewTile<bf16> {
    typedef bf16 operand __attribute__((ext_vector_type(8)));
    static constexpr int kVec = 8;
    static __device__ __forceinline__ f32x4 run(operand a, operand b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
};
template <> struct FewTile<f16> {
    typedef f16 operand __attribute__((ext_vector_type(8)));
    static constexpr int kVec = 8;
    static __device__ __forceinline__ f32x4 run(operand a, operand b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }
};
template <> struct FewTile<float> {
    typedef float operand __attribute__((ext_vector_type(4)));
    static constexpr int kVec = 4;
    static __device__ __forceinline__ f32x4 run(operand a, operand b, f32x4 c)
    {
#pragma unroll
        for (int i = 0; i < 4; ++i) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a[i], b[i], c, 0, 0, 0);
        return c;
    }
};

// Sums of MT tiles of rows with NT tiles of rows over this wavefront's part of k.  All of a few steps' loads are on
// their way before the first is multiplied (in the order that the compiler would choose, few are).
template <typename S, int WAVES, int MT, int NT>
__device__ __forceinline__ void few_sums(const S *const (&rows_a)[MT], const S *const (&rows_b)[NT], int k_all, int wave, int lane,
                                         f32x4 (&acc)[MT][NT])
{
    typedef typename FewTile<S>::operand Operand;
    typedef S Loaded __attribute__((ext_vector_type(FewTile<S>::kVec), aligned(sizeof(S))));
    constexpr int kVec = FewTile<S>::kVec, kFewStep = 8 * kVec;   // a lane has two pieces of 16 bytes: a row's are 128
    constexpr int kEach = MT + NT, kAhead = kEach > 7 ? 2 : 16 / kEach / 2 * 2;   // pieces at a time, about 64 registers of them
    struct Batch {
        Operand x[kAhead][MT], y[kAhead][NT];
    };
    const int steps = (k_all + kFewStep - 1) / kFewStep, last = steps * (wave + 1) / WAVES;
    const int part = (lane >> 4) * 2 * kVec;
    int step = steps * wave / WAVES;
    const S *a[MT], *b[NT];
#pragma unroll
    for (int i = 0; i < MT; ++i) a[i] = rows_a[i] + step * kFewStep + part;
#pragma unroll
    for (int j = 0; j < NT; ++j) b[j] = rows_b[j] + step * kFewStep + part;
    const auto load = [&](Batch &w) __attribute__((always_inline)) {
#pragma unroll
        for (int q = 0; q < kAhead; ++q) {
#pragma unroll
            for (int i = 0; i < MT; ++i) w.x[q][i] = *reinterpret_cast<const Loaded *>(a[i] + (q >> 1) * kFewStep + (q & 1) * kVec);
#pragma unroll
            for (int j = 0; j < NT; ++j) w.y[q][j] = *reinterpret_cast<const Loaded *>(b[j] + (q >> 1) * kFewStep + (q & 1) * kVec);
        }
#pragma unroll
        for (int i = 0; i < MT; ++i) a[i] += kAhead / 2 * kFewStep;
#pragma unroll
        for (int j = 0; j < NT; ++j) b[j] += kAhead / 2 * kFewStep;
        __builtin_amdgcn_sched_barrier(0);
    };
    const auto multiply = [&](const Batch &w) __attribute__((always_inline)) {
#pragma unroll
        for (int q = 0; q < kAhead; ++q)
#pragma unroll
            for (int i = 0; i < MT; ++i)
#pragma unroll
                for (int j = 0; j < NT; ++j) acc[i][j] = FewTile<S>::run(w.x[q][i], w.y[q][j], acc[i][j]);
        __builtin_amdgcn_sched_barrier(0);
    };
    const int whole = min(last, k_all / kFewStep);   // steps that end within the rows
    const int batches = whole > step ? (whole - step) / (kAhead / 2) : 0;
    step += batches * (kAhead / 2);
    for (int n = 0; n < batches; ++n) {
        Batch now;
        load(now);
        multiply(now);
    }
    // what is left, at most kAhead / 2 steps, one of which may end beyond the rows: zeros there
    if (step >= last) return;
    Batch rest = {};
#pragma unroll
    for (int q = 0; q < kAhead; ++q) {
        if (step + (q >> 1) >= last) break;
        const int left = k_all - (step + (q >> 1)) * kFewStep - part - (q & 1) * kVec;   // elements that the row has here
        if (left >= kVec) {
#pragma unroll
            for (int i = 0; i < MT; ++i) rest.x[q][i] = *reinterpret_cast<const Loaded *>(a[i] + (q >> 1) * kFewStep + (q & 1) * kVec);
#pragma unroll
            for (int j = 0; j < NT; ++j) rest.y[q][j] = *reinterpret_cast<const Loaded *>(b[j] + (q >> 1) * kFewStep + (q & 1) * kVec);
        } else {
#pragma unroll
            for (int r = 0; r < kVec; ++r) {
                if (r >= left) break;
#pragma unroll
                for (int i = 0; i < MT; ++i) rest.x[q][i][r] = a[i][(q >> 1) * kFewStep + (q & 1) * kVec + r];
#pragma unroll
                for (int j = 0; j < NT; ++j) rest.y[q][j][r] = b[j][(q >> 1) * kFewStep + (q & 1) * kVec + r];
            }
        }
    }
    multiply(rest);
}

struct FewArgs {
    int n, hidden, inner, activation;
    const void *x, *w_gate, *w_up, *w_down;
    int64_t x_stride, w_gate_stride, w_up_stride, w_down_stride;
    void *h;             // [arrays][n][h_stride]
    int64_t h_stride, h_array;
    int h_arrays;
    deft_saved_t saved;
    void *y;
    int64_t y_stride;
};

// The sums of all wavefronts for sixteen tokens, [token][row] behind one another.
template <int MT>
__device__ __forceinline__ void few_meet(const f32x4 (&acc)[MT], float *lds, int wave, int lane)
{
    constexpr int kPitch = MT * 16 + 4;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < MT; ++i)
        *reinterpret_cast<f32x4 *>(lds + (wave * 16 + (lane & 15)) * kPitch + i * 16 + (lane >> 4) * 4) = acc[i];
    __syncthreads();
}

template <int WAVES, int MT>
__device__ __forceinline__ float few_sum(const float *lds, int token, int row)
{
    constexpr int kPitch = MT * 16 + 4;
    float x = 0.0f;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) x += lds[(w * 16 + token) * kPitch + row];
    return x;
}

// A sum as its part of a checkpoint's group, which 32 neighbouring lanes hold.  `least`: of positive sums' codes.
template <typename C>
__device__ __forceinline__ void few_code(deft_checkpoint_t to, int n, int at, bool in, float x, float least)
{
    constexpr float kLargest = sizeof(C) == 1 ? kCodes8 : kCodes16;
    unsigned top = in ? __float_as_uint(x) & 0x7fffffffu : 0u;
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) top = max(top, (unsigned)__shfl_xor((int)top, d));
    const float s = checkpoint_scale(__uint_as_float(top), kLargest, 1.0f / kLargest);
    if (!in) return;
    static_cast<C *>(to.codes)[n * to.codes_stride + at] = (C)(int)__builtin_rintf(fminf(fmaxf(x / s, x > 0.0f ? least : -kLargest), kLargest));
    if (at % kGroup == 0)
        static_cast<unsigned short *>(to.scales)[n * to.scales_stride + at / kGroup] = top < 0x7f800000u ? __float_as_uint(s) >> 16 : 0x7fc0;
}

template <typename S>
__device__ __forceinline__ void few_save(int kind, deft_checkpoint_t to, int n, int at, bool in, float x, float least = 0.0f)
{
    if (kind == DEFT_SAVE_PACKED) {
        few_code<int8_t>(to, n, at, in, x, 0.0f);
    } else if constexpr (sizeof(S) == 4) {
        if (in) static_cast<float *>(to.codes)[n * to.codes_stride + at] = x;
    } else {
        few_code<int16_t>(to, n, at, in, x, least);
    }
}

// Workgroup b: columns 16 TILES b .. of both projections (32: a checkpoint's group).
template <typename S, int TILES, int NT>
__global__ void __launch_bounds__(kGateWaves *kWave, 4) few_gate_kernel(FewArgs a)
{
    constexpr int MT = 2 * TILES, kCols = 16 * TILES;
    __shared__ __align__(16) float lds[kGateWaves * 16 * (MT * 16 + 4)];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, row16 = lane & 15, first = blockIdx.x * kCols;
    const S *w[MT], *x[NT];   // (rows past the last one read that one)
#pragma unroll
    for (int i = 0; i < TILES; ++i) {
        const int row = min(first + i * 16 + row16, a.inner - 1);
        w[i] = static_cast<const S *>(a.w_gate) + row * a.w_gate_stride;
        w[TILES + i] = static_cast<const S *>(a.w_up) + row * a.w_up_stride;
    }
#pragma unroll
    for (int j = 0; j < NT; ++j) x[j] = static_cast<const S *>(a.x) + min(j * 16 + row16, a.n - 1) * a.x_stride;
    f32x4 acc[MT][NT] = {};
    few_sums<S, kGateWaves, MT, NT>(w, x, a.hidden, wave, lane, acc);
    const int token = tid / kCols, col = tid % kCols, at = first + col;
#pragma unroll
    for (int j = 0; j < NT; ++j) {
        f32x4 own[MT];
#pragma unroll
        for (int i = 0; i < MT; ++i) own[i] = acc[i][j];
        few_meet<MT>(own, lds, wave, lane);
        if (token >= 16) continue;   // (whole wavefronts)
        const int n = j * 16 + token;
        const float gate = few_sum<kGateWaves, MT>(lds, token, col), up = few_sum<kGateWaves, MT>(lds, token, kCols + col);
        const bool in = n < a.n && at < a.inner;
        if (TILES == 2 && a.saved.kind != DEFT_SAVE_NONE) {
            few_save<S>(a.saved.kind, a.saved.gate, n, at, in, gate, a.activation == DEFT_RELU ? 1.0f : 0.0f);
            few_save<S>(a.saved.kind, a.saved.up, n, at, in, up);
        }
        if (!in) continue;
        float y, slope;
        constexpr bool kExact = sizeof(S) == 4;
        if (a.activation == DEFT_SILU) act_of<DEFT_SILU, kExact>(gate, y, slope);
        else if (a.activation == DEFT_GELU) act_of<DEFT_GELU, kExact>(gate, y, slope);
        else if (a.activation == DEFT_GELU_TANH) act_of<DEFT_GELU_TANH, kExact>(gate, y, slope);
        else act_of<DEFT_RELU, kExact>(gate, y, slope);
        S *h = static_cast<S *>(a.h) + n * a.h_stride + at;
        const float of_both = y * up;
        *h = (S)of_both;
        if (a.h_arrays == 2) h[a.h_array] = (S)taken(of_both, (S)of_both);
    }
}

// Workgroup b: columns MT * 16 b .. of y.  FOLD: up to 8 tokens, whose two arrays are one tile's sixteen rows.  TWO: the second array
// is as many tiles again, whose sums are added before the wavefronts' meet.
template <typename S, int MT, int NT, bool FOLD, bool TWO = false>
__global__ void __launch_bounds__(kOutWaves *kWave) few_out_kernel(FewArgs a)
{
    __shared__ __align__(16) float lds[kOutWaves * 16 * (MT * 16 + 4)];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, row16 = lane & 15, first = blockIdx.x * MT * 16;
    constexpr int kTiles = TWO ? 2 * NT : NT;
    const S *w[MT], *h[kTiles];
#pragma unroll
    for (int i = 0; i < MT; ++i) w[i] = static_cast<const S *>(a.w_down) + min(first + i * 16 + row16, a.hidden - 1) * a.w_down_stride;
#pragma unroll
    for (int j = 0; j < kTiles; ++j)
        h[j] = static_cast<const S *>(a.h) + (FOLD ? (row16 >> 3) * a.h_array : j / NT * a.h_array) +
               min(FOLD ? row16 & 7 : j % NT * 16 + row16, a.n - 1) * a.h_stride;
    f32x4 acc[MT][kTiles] = {};
    few_sums<S, kOutWaves, MT, kTiles>(w, h, a.inner, wave, lane, acc);
#pragma unroll
    for (int j = 0; j < NT; ++j) {
        f32x4 own[MT];
#pragma unroll
        for (int i = 0; i < MT; ++i) own[i] = TWO ? acc[i][j] + acc[i][kTiles - NT + j] : acc[i][j];
        few_meet<MT>(own, lds, wave, lane);
        for (int at = tid; at < (FOLD ? 8 : 16) * MT * 16; at += kOutWaves * kWave) {
            const int token = at / (MT * 16), row = at % (MT * 16), n = j * 16 + token;
            if (n >= a.n || first + row >= a.hidden) continue;
            float y = few_sum<kOutWaves, MT>(lds, token, row);
            if (FOLD) y += few_sum<kOutWaves, MT>(lds, token + 8, row);
            static_cast<S *>(a.y)[n * a.y_stride + first + row] = (S)y;
        }
    }
}

template <typename S, int NT>
hipError_t few_tokens(const FewArgs &a, int compute_units, hipStream_t st)
{
    if (a.saved.kind == DEFT_SAVE_NONE) few_gate_kernel<S, 1, NT><<<(a.inner + 15) / 16, kGateWaves * kWave, 0, st>>>(a);
    else few_gate_kernel<S, 2, NT><<<(a.inner + 31) / 32, kGateWaves * kWave, 0, st>>>(a);
    const unsigned ones = (unsigned)(a.hidden + 15) / 16, twos = (unsigned)(a.hidden + 31) / 32;
    if constexpr (NT == 1 && sizeof(S) == 2)
        if (a.h_arrays == 2) {
            few_out_kernel<S, 1, 1, true><<<ones, kOutWaves * kWave, 0, st>>>(a);
            return hipGetLastError();
        }
    if constexpr (NT == 2 && sizeof(S) == 2)
        if (a.h_arrays == 2) {
            few_out_kernel<S, 1, NT, false, true><<<ones, kOutWaves * kWave, 0, st>>>(a);
            return hipGetLastError();
        }
    // (rows two tiles at a time read the activations half as often)
    if (a.hidden < 32 * compute_units) few_out_kernel<S, 1, NT, false><<<ones, kOutWaves * kWave, 0, st>>>(a);
    else few_out_kernel<S, 2, NT, false><<<twos, kOutWaves * kWave, 0, st>>>(a);
    return hipGetLastError();
}

}  // namespace
}  // namespace deft
