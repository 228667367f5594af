// What the feed-forward block's products do with their sums: act(gate) * up as they leave the matrix units, the
// derivatives by both projections, and the rounded outputs.
//
// All pass their sums through LDS, sixteen rows of a wavefront's tile at a time, so that a lane has eight
// neighbouring columns of one row, what it loads and stores is 16 bytes, a row's lanes are next to each other, and a
// checkpoint's group of 32 is four lanes'.
#pragma once
#include "block.h"

namespace deft {

constexpr int kEight = 8;   // columns of a lane

// What eight elements do: act(a), or act(a) and its derivative.  kExact: 32-bit outputs; otherwise exponentials and
// reciprocals are the hardware's (off by 1 or 2 units of the last 24 bits, and |a| of them in the exponential), far below the
// rounding to 16 bits that follows.
template <bool kExact, bool kSlope>
__device__ __forceinline__ void act_of(const float (&a)[kEight], int kind, float (&y)[kEight], float (&slope)[kEight])
{
    const auto exp_of = [](float x) { return kExact ? expf(x) : __expf(x); };
    const auto inverse = [](float x) { return kExact ? 1.0f / x : __builtin_amdgcn_rcpf(x); };
    if (kind == DEFT_SILU) {
#pragma unroll
        for (int i = 0; i < kEight; ++i) {
            const float p = inverse(1.0f + exp_of(-a[i]));
            y[i] = a[i] * p;
            if (kSlope) slope[i] = p * (1.0f + a[i] * (1.0f - p));
        }
    } else if (kind == DEFT_GELU) {
#pragma unroll
        for (int i = 0; i < kEight; ++i) {
            const float p = 0.5f * erfcf(-0.707106781f * a[i]);
            y[i] = a[i] * p;
            if (kSlope) slope[i] = p + a[i] * (0.398942280f * exp_of(-0.5f * a[i] * a[i]));
        }
    } else if (kind == DEFT_GELU_TANH) {   // (1 + tanh(u / 2)) / 2 = 1 / (1 + exp(-u))
#pragma unroll
        for (int i = 0; i < kEight; ++i) {
            const float square = a[i] * a[i], u = 1.595769122f * a[i] * (1.0f + 0.044715f * square), p = inverse(1.0f + exp_of(-u));
            const float rest = p * (1.0f - p);   // (0 where the square may be infinite)
            y[i] = a[i] * p;
            if (kSlope) slope[i] = p + (rest == 0.0f ? 0.0f : rest * 1.595769122f * a[i] * (1.0f + 0.134145f * square));
        }
    } else {
#pragma unroll
        for (int i = 0; i < kEight; ++i) {   // (NaN stays)
            y[i] = a[i] < 0.0f ? 0.0f : a[i];
            if (kSlope) slope[i] = a[i] > 0.0f ? 1.0f : 0.0f;
        }
    }
}

// Eight elements of a row from column `at` on, where `cols` is the first that the row does not have (0: none of it is there).
template <typename O>
__device__ __forceinline__ void store_eight(O *row, int at, int cols, const float (&x)[kEight])
{
    typedef O O8 __attribute__((ext_vector_type(8), aligned(sizeof(O))));
    if (at + kEight <= cols) {
        O8 y;
#pragma unroll
        for (int r = 0; r < kEight; ++r) y[r] = (O)x[r];
        *reinterpret_cast<O8 *>(row + at) = y;
    } else {
#pragma unroll
        for (int r = 0; r < kEight; ++r)
            if (at + r < cols) row[at + r] = (O)x[r];
    }
}

template <typename O>
__device__ __forceinline__ void load_eight(const O *row, int at, int cols, float (&x)[kEight])
{
    typedef O O8 __attribute__((ext_vector_type(8), aligned(sizeof(O))));
    if (at + kEight <= cols) {
        const O8 y = *reinterpret_cast<const O8 *>(row + at);
#pragma unroll
        for (int r = 0; r < kEight; ++r) x[r] = (float)y[r];
    } else {
#pragma unroll
        for (int r = 0; r < kEight; ++r) x[r] = at + r < cols ? (float)row[at + r] : 0.0f;
    }
}

// The same as codes C of a checkpoint, whose group this and three neighbouring lanes hold.
template <typename C>
__device__ __forceinline__ void store_codes(const deft_checkpoint_t &to, int n, int at, int cols, const float (&x)[kEight])
{
    typedef C C8 __attribute__((ext_vector_type(8), aligned(sizeof(C))));
    constexpr float kMost = sizeof(C) == 1 ? kCodes8 : kCodes16;
    float top = 0.0f;
#pragma unroll
    for (int r = 0; r < kEight; ++r) top = fmaxf(top, at + r < cols && is_finite(x[r]) ? fabsf(x[r]) : 0.0f);
    top = fmaxf(top, __shfl_xor(top, 1));
    top = fmaxf(top, __shfl_xor(top, 2));
    const float s = checkpoint_scale(top, kMost), inverse = 1.0f / s;
    C8 y;
#pragma unroll
    for (int r = 0; r < kEight; ++r) y[r] = (C)checkpoint_code_of_sum(x[r], inverse, kMost);
    C *row = static_cast<C *>(to.codes) + n * to.codes_stride;
    if (at + kEight <= cols) {
        *reinterpret_cast<C8 *>(row + at) = y;
    } else {
#pragma unroll
        for (int r = 0; r < kEight; ++r)
            if (at + r < cols) row[at + r] = y[r];
    }
    if (at % kGroup == 0 && at < cols) static_cast<bf16 *>(to.scales)[n * to.scales_stride + at / kGroup] = (bf16)s;   // (exactly)
}

template <typename C>
__device__ __forceinline__ void load_codes(const deft_checkpoint_t &from, int n, int at, int cols, float (&x)[kEight])
{
    typedef C C8 __attribute__((ext_vector_type(8), aligned(sizeof(C))));
    const C *row = static_cast<const C *>(from.codes) + n * from.codes_stride;
    C8 y = {};
    if (at + kEight <= cols) {
        y = *reinterpret_cast<const C8 *>(row + at);
    } else {
#pragma unroll
        for (int r = 0; r < kEight; ++r)
            if (at + r < cols) y[r] = row[at + r];
    }
    const float s = at < cols ? (float)static_cast<const bf16 *>(from.scales)[n * from.scales_stride + at / kGroup] : 0.0f;
#pragma unroll
    for (int r = 0; r < kEight; ++r) x[r] = checkpoint_value(y[r], s, sizeof(C) == 1 ? -128 : -32768, 3.402823466e38f);
}

// The same of a projection as it is kept: in 8 bits, or in as many as O has.
template <typename O>
__device__ __forceinline__ void store_saved(int kind, const deft_checkpoint_t &to, int n, int at, int cols, const float (&x)[kEight])
{
    if (kind == DEFT_SAVE_PACKED) store_codes<int8_t>(to, n, at, cols, x);
    else if constexpr (sizeof(O) == 4) store_eight(static_cast<float *>(to.codes) + n * to.codes_stride, at, cols, x);
    else store_codes<int16_t>(to, n, at, cols, x);
}

template <typename O>
__device__ __forceinline__ void load_saved(int kind, const deft_checkpoint_t &from, int n, int at, int cols, float (&x)[kEight])
{
    if (kind == DEFT_SAVE_PACKED) load_codes<int8_t>(from, n, at, cols, x);
    else if constexpr (sizeof(O) == 4) load_eight(static_cast<const float *>(from.codes) + n * from.codes_stride, at, cols, x);
    else load_codes<int16_t>(from, n, at, cols, x);
}

// Eight elements of an operand in panels: one array of T, or three of bf16 whose sum they are.
template <typename T, bool SPLIT>
__device__ __forceinline__ void store_operand(void *panels, int64_t panel, int64_t plane, int n, int at, int cols_up, const float (&x)[kEight])
{
    typedef T T8 __attribute__((ext_vector_type(8)));
    if (at >= cols_up) return;
    T *to = static_cast<T *>(panels) + (at >> 8) * panel + (int64_t)n * 256 + (at & 255);
    if constexpr (SPLIT) {
        T8 y[3];
#pragma unroll
        for (int r = 0; r < kEight; ++r) {
            bf16 p[3];
            split3(x[r], p);
#pragma unroll
            for (int s = 0; s < 3; ++s) y[s][r] = p[s];
        }
#pragma unroll
        for (int s = 0; s < 3; ++s) *reinterpret_cast<T8 *>(to + s * plane) = y[s];
    } else {
        T8 y;
#pragma unroll
        for (int r = 0; r < kEight; ++r) y[r] = (T)x[r];
        *reinterpret_cast<T8 *>(to) = y;
    }
}

constexpr __host__ __device__ int epilogue_pitch(int mt) { return mt * 16 + 4; }   // of a row of sums in LDS
constexpr __host__ __device__ int epilogue_floats(int mt) { return 16 * epilogue_pitch(mt); }   // of a wavefront

// Goes through a wavefront's tile sixteen rows at a time: its sums go to `lds` (the wavefront's own part), and `use` is called with a
// row's number in the tile and where its sums lie, for every lane and kLanes lanes a row; kEach columns of sums belong to a
// lane's eight elements.  acc[i][j][r] is row row16 + 16 j, column part * 4 + 16 i + r.
template <int MT, int NT, int kEach, typename F>
__device__ __forceinline__ void by_rows(const f32x4 (&acc)[MT][NT], float *lds, int lane, F use)
{
    constexpr int kPitch = epilogue_pitch(MT), kLanes = MT * 16 / kEach;
    const int row16 = lane & 15, part = lane >> 4;
#pragma clang loop unroll(disable)
    for (int j = 0; j < NT; ++j) {
#pragma unroll
        for (int which = 0; which < NT; ++which)
            if (j == which) {
#pragma unroll
                for (int i = 0; i < MT; ++i) *reinterpret_cast<f32x4 *>(lds + row16 * kPitch + i * 16 + part * 4) = acc[i][which];
            }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");   // (a wavefront's LDS accesses are done in order)
        __builtin_amdgcn_wave_barrier();
#pragma clang loop unroll(disable)
        for (int at = lane; at < 16 * kLanes; at += kWave) {
            const int row = at / kLanes;
            use(j * 16 + row, (at - row * kLanes) * 8, lds + row * kPitch);
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
    }
}

__device__ __forceinline__ void read_eight(const float *from, float (&x)[kEight])
{
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const f32x4 v = *reinterpret_cast<const f32x4 *>(from + h * 4);
#pragma unroll
        for (int r = 0; r < 4; ++r) x[h * 4 + r] = v[r];
    }
}

// Sixteens of columns are gate and up in turn.  The wavefront's tile begins at row n_wave and, of either, column m_wave.  Rows
// behind the last one and columns behind `cols` are zeros in h.
template <typename T, typename O, int MT, int NT, bool SPLIT>
__device__ __forceinline__ void gate_epilogue(const FfnArgs &f, const f32x4 (&acc)[MT][NT], float *lds, int lane, int m_wave, int n_wave, int n_rows, int cols)
{
    static_assert(MT % 4 == 0);   // whole groups of 32
    by_rows<MT, NT, 16>(acc, lds, lane, [&](int row, int col, const float *sums) {
        const int n = n_wave + row, at = m_wave + col, own_cols = n < n_rows ? cols : 0;
        float gate[kEight], up[kEight], h[kEight], none[kEight];
        read_eight(sums + (col >> 4) * 32 + (col & 15), gate);
        read_eight(sums + (col >> 4) * 32 + 16 + (col & 15), up);
        if (f.saved.kind != DEFT_SAVE_NONE) {
            store_saved<O>(f.saved.kind, f.saved.gate, n, at, own_cols, gate);
            store_saved<O>(f.saved.kind, f.saved.up, n, at, own_cols, up);
        }
        if (!f.h) return;
        act_of<SPLIT, false>(gate, f.activation, h, none);
#pragma unroll
        for (int r = 0; r < kEight; ++r) h[r] = at + r < own_cols ? h[r] * up[r] : 0.0f;
        store_operand<T, SPLIT>(f.h, f.panel, f.h_plane, n, at, f.cols_up, h);
    });
}

// The sums are the derivative by h.
template <typename T, typename O, int MT, int NT, bool SPLIT>
__device__ __forceinline__ void gate_grad_epilogue(const FfnArgs &f, const f32x4 (&acc)[MT][NT], float *lds, int lane, int m_wave, int n_wave, int n_rows,
                                                   int cols)
{
    static_assert(MT % 2 == 0);   // whole groups of 32
    const float factor = f.factor ? f.factor[0] : 1.0f;
    const int64_t behind = (int64_t)(f.cols_up >> 8) * f.panel;   // up's derivatives
    by_rows<MT, NT, 8>(acc, lds, lane, [&](int row, int col, const float *sums) {
        const int n = n_wave + row, at = m_wave + col, own_cols = n < n_rows ? cols : 0;
        float gate[kEight], up[kEight], by_h[kEight], y[kEight], slope[kEight];
        load_saved<O>(f.saved.kind, f.saved.gate, n, at, own_cols, gate);
        load_saved<O>(f.saved.kind, f.saved.up, n, at, own_cols, up);
        read_eight(sums + col, by_h);
        act_of<SPLIT, true>(gate, f.activation, y, slope);
        float h[kEight];
#pragma unroll
        for (int r = 0; r < kEight; ++r) {
            const bool here = at + r < own_cols;
            const float d = by_h[r] * factor;
            h[r] = here ? y[r] * up[r] : 0.0f;
            slope[r] = here ? d * up[r] * slope[r] : 0.0f;
            y[r] = here ? d * y[r] : 0.0f;
        }
        if (f.h) store_operand<T, SPLIT>(f.h, f.panel, f.h_plane, n, at, f.cols_up, h);
        if (f.d) {
            store_operand<T, SPLIT>(f.d, f.panel, f.d_plane, n, at, f.cols_up, slope);
            store_operand<T, SPLIT>(static_cast<T *>(f.d) + behind, f.panel, f.d_plane, n, at, f.cols_up, y);
        }
    });
}

// Where row n of a product's result goes, or NULL.
template <typename O>
__device__ __forceinline__ O *out_row(const FfnArgs &f, int n)
{
    const int which = n >= f.half ? 1 : 0, row = n - (which ? f.half : 0);
    O *out = static_cast<O *>(which ? f.out[1] : f.out[0]);
    return out && row < f.rows ? out + row * (which ? f.out_ld[1] : f.out_ld[0]) : nullptr;
}

// A lane's columns of a row: out = x / factor, or that and what is there, rounded once.
template <typename O>
__device__ __forceinline__ void store_out(O *row, int at, int cols, const float (&x)[kEight], float alpha, int add)
{
    float y[kEight] = {};
    if (add) load_eight(row, at, cols, y);
#pragma unroll
    for (int r = 0; r < kEight; ++r) y[r] += alpha * x[r];
    store_eight(row, at, cols, y);
}

// The sums are the result, or a part of it (`sums`: rows of sums_ld elements, a multiple of 8).
template <typename O, int MT, int NT>
__device__ __forceinline__ void out_epilogue(const FfnArgs &f, const f32x4 (&acc)[MT][NT], float *lds, int lane, int m_wave, int n_wave, int n_rows, int cols,
                                             int add, float *sums, int64_t sums_ld)
{
    const float alpha = f.factor ? f.factor[1] : 1.0f;
    by_rows<MT, NT, 8>(acc, lds, lane, [&](int row, int col, const float *from) {
        const int n = n_wave + row, at = m_wave + col;
        if (n >= n_rows || at >= cols) return;
        float x[kEight];
        read_eight(from + col, x);
        if (sums) {
            store_eight(sums + n * sums_ld, at, INT32_MAX, x);
        } else if (O *to = out_row<O>(f, n)) {
            store_out(to, at, cols, x, alpha, add);
        }
    });
}

}  // namespace deft
