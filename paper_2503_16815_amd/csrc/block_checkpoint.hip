// Activation checkpoints in 8 bits.
//
//   s = the smallest number of 8 significant bits, at least 2^-126, with 127 s >= max |x| over 32 elements of a row;
//   code = the whole number nearest to x / s;  x comes back as code * s, off by at most s / 2.
//
// One scale for 32 elements: an element that is many times as large as its neighbours costs 31 others their bits.  Scales of
// 8 significant bits: powers of two alone (half a byte less for 32 elements) would make the step larger by 1.47 in the
// root mean square.  Bound by memory, read and written once: four neighbouring lanes hold a group, 8 elements each.
#include "block.h"

namespace deft {
namespace {

struct StoreArgs {
    int rows, width;
    const void *x;
    int64_t x_stride;
    deft_checkpoint_t out;
};

typedef int8_t codes8 __attribute__((ext_vector_type(8), aligned(1)));

template <typename S>
__global__ void __launch_bounds__(256) store_kernel(StoreArgs a)
{
    typedef S S8 __attribute__((ext_vector_type(8), aligned(sizeof(S))));
    const unsigned pieces = (unsigned)((a.width + kGroup - 1) / kGroup) * 4;   // of 8 elements, of a row's groups
    const int64_t at = (int64_t)blockIdx.x * 256 + threadIdx.x;
    const int64_t row = at / pieces;
    const int piece = (int)(at - row * pieces), col = piece * 8;
    if (row >= a.rows) return;   // (whole groups of four lanes)
    const S *from = static_cast<const S *>(a.x) + row * a.x_stride + col;
    float x[8] = {};
    const bool whole = col + 8 <= a.width;
    if (whole) {
        const S8 v = *reinterpret_cast<const S8 *>(from);
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = (float)v[i];
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (col + i < a.width) x[i] = (float)from[i];
    }
    float top = 0.0f;
#pragma unroll
    for (int i = 0; i < 8; ++i) top = fmaxf(top, is_finite(x[i]) ? fabsf(x[i]) : 0.0f);
    top = fmaxf(top, __shfl_xor(top, 1));
    top = fmaxf(top, __shfl_xor(top, 2));
    const float s = checkpoint_scale(top, kCodes8), inverse = 1.0f / s;
    int8_t *to = static_cast<int8_t *>(a.out.codes) + row * a.out.codes_stride + col;
    codes8 y;
#pragma unroll
    for (int i = 0; i < 8; ++i) y[i] = (int8_t)checkpoint_code(x[i], s, inverse);
    if (whole) {
        *reinterpret_cast<codes8 *>(to) = y;
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (col + i < a.width) to[i] = y[i];
    }
    if ((piece & 3) == 0) static_cast<bf16 *>(a.out.scales)[row * a.out.scales_stride + (piece >> 2)] = (bf16)s;   // (exactly)
}

template <typename S> constexpr float kMost = 3.402823466e38f;
template <> constexpr float kMost<f16> = 65504.0f;
template <> constexpr float kMost<bf16> = 3.38953139e38f;

// T, P: the operand that it becomes (one array of S itself, or three of bf16).
template <typename S, typename T, int P>
__global__ void __launch_bounds__(256) restore_kernel(RestoreArgs a)
{
    typedef T T8 __attribute__((ext_vector_type(8), aligned(sizeof(T))));
    const unsigned pieces = (unsigned)((a.cols_to + 7) >> 3);
    const int64_t at = (int64_t)blockIdx.x * 256 + threadIdx.x;
    const int64_t row = at / pieces;
    const int col = (int)(at - row * pieces) * 8;
    if (row >= a.rows_to) return;
    float x[8] = {};
    if (row < a.rows && col < a.cols) {
        const int8_t *from = static_cast<const int8_t *>(a.from.codes) + row * a.from.codes_stride + col;
        const float s = (float)static_cast<const bf16 *>(a.from.scales)[row * a.from.scales_stride + col / kGroup];
        if (col + 8 <= a.cols) {
            const codes8 v = *reinterpret_cast<const codes8 *>(from);
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i] = checkpoint_value(v[i], s, -128, kMost<S>);
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (col + i < a.cols) x[i] = checkpoint_value(from[i], s, -128, kMost<S>);
        }
    }
    T8 y[P];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        if constexpr (P == 3) {
            bf16 p[3];
            split3((float)(S)x[i], p);
#pragma unroll
            for (int k = 0; k < 3; ++k) y[k][i] = p[k];
        } else {
            y[0][i] = (T)x[i];
        }
    }
#pragma unroll
    for (int k = 0; k < P; ++k) {
        T *to = static_cast<T *>(a.out) + k * a.out_plane + row * a.out_ld + col;
        if (col + 8 <= a.cols_to) {
            *reinterpret_cast<T8 *>(to) = y[k];
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (col + i < a.cols_to) to[i] = y[k][i];
        }
    }
}

unsigned blocks_of(int64_t rows, int64_t pieces) { return (unsigned)((rows * pieces + 255) / 256); }

template <typename S, typename T, int P>
hipError_t restore(const RestoreArgs &a, hipStream_t st)
{
    restore_kernel<S, T, P><<<blocks_of(a.rows_to, (a.cols_to + 7) >> 3), 256, 0, st>>>(a);
    return hipGetLastError();
}

}  // namespace

hipError_t checkpoint_launch(int dtype, const deft_checkpoint_call_t &c, hipStream_t st)
{
    const StoreArgs a = {c.n_rows, c.width, c.x, c.x_stride, c.out};
    const unsigned blocks = blocks_of(a.rows, (int64_t)(a.width + kGroup - 1) / kGroup * 4);
    if (dtype == DEFT_F32) store_kernel<float><<<blocks, 256, 0, st>>>(a);
    else if (dtype == DEFT_F16) store_kernel<f16><<<blocks, 256, 0, st>>>(a);
    else store_kernel<bf16><<<blocks, 256, 0, st>>>(a);
    return hipGetLastError();
}

hipError_t restore_launch(int dtype, const deft_restore_call_t &c, hipStream_t st)
{
    const RestoreArgs a = {c.n_rows, c.width, c.n_rows, c.width, c.from, c.out, c.out_stride, 0};
    if (dtype == DEFT_F32) return restore<float, float, 1>(a, st);
    if (dtype == DEFT_F16) return restore<f16, f16, 1>(a, st);
    return restore<bf16, bf16, 1>(a, st);
}

hipError_t restore_operand_launch(int dtype, const RestoreArgs &a, hipStream_t st)
{
    if (dtype == DEFT_F32) return restore<float, bf16, 3>(a, st);
    if (dtype == DEFT_F16) return restore<f16, f16, 1>(a, st);
    return restore<bf16, bf16, 1>(a, st);
}

}  // namespace deft
