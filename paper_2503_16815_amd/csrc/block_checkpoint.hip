// Activation checkpoints in 8 bits.
//
//   s = the smallest number of 8 significant bits, at least 2^-126, with 127 s >= max |x| over 32 elements of a row;
//   code = the whole number nearest to x / s;  x comes back as code * s, off by at most s / 2.
//
// One scale for 32 elements: an element that is many times as large as its neighbours costs 31 others their bits.  Scales of
// 8 significant bits: powers of two alone (half a byte less for 32 elements) would make the step larger by 1.47 in the
// root mean square.  Bound by memory, read and written once (16384 x 4096 bf16: 42 us, 4.9 TB/s; back
// 33, 6.2): four neighbouring lanes hold a group, 8 elements each.
#include "block_epilogue.h"

namespace deft {
namespace {

struct StoreArgs {
    int rows, width;
    const void *x;
    int64_t x_stride;
    deft_checkpoint_t out;
    RowPieces by;
};

template <typename S>
__global__ void __launch_bounds__(256) store_kernel(StoreArgs a)
{
    // (whole groups of four lanes)
    int n, piece;
    if (!a.by.own(blockIdx.x, &n, &piece)) return;
    const int64_t row = n;
    const int at = piece * kEight;
    const typename Eight<S>::type v = load_eight<false>(static_cast<const S *>(a.x) + row * a.x_stride + at, at, a.width);
    float x[kEight];
    unsigned own = 0;   // (as whole numbers infinity is above all finite magnitudes and NaN above infinity)
#pragma unroll
    for (int r = 0; r < kEight; ++r) {
        x[r] = (float)v[r];
        own = max(own, __float_as_uint(x[r]) & 0x7fffffffu);
    }
    unsigned top = quad_max(own);
    const bool all_finite = top < 0x7f800000u;
    if (!all_finite) {   // the others' largest
        own = 0;
#pragma unroll
        for (int r = 0; r < kEight; ++r) own = max(own, is_finite(x[r]) ? __float_as_uint(x[r]) & 0x7fffffffu : 0u);
        top = quad_max(own);
    }
    const float s = checkpoint_scale(__uint_as_float(top), kCodes8, 1.0f / kCodes8), inverse = __builtin_amdgcn_rcpf(s), half = 0.5f * s;
    // x / s rounded by way of 1 / s; what is left of x, which is exact, tells whether that ended on a half or beyond
    unsigned code[kEight];
    float left[kEight], most = 0.0f;
#pragma unroll
    for (int r = 0; r < kEight; ++r) {
        const float shifted = fmaf(x[r], inverse, kShift);
        left[r] = fmaf(kShift - shifted, s, x[r]);
        code[r] = __float_as_uint(shifted);
        most = fmaxf(most, fabsf(left[r]));
    }
    if (most >= half) {
#pragma unroll
        for (int r = 0; r < kEight; ++r) {
            const bool wrong = fabsf(left[r]) > half || ((code[r] & 1) && fabsf(left[r]) == half);
            code[r] += wrong ? (left[r] > 0.0f ? 1u : ~0u) : 0u;
        }
    }
    if (!all_finite) {
#pragma unroll
        for (int r = 0; r < kEight; ++r) code[r] = is_finite(x[r]) ? code[r] : 0x80u;
    }
    const uint2 all = make_uint2(pack_bytes(code[0], code[1], code[2], code[3]), pack_bytes(code[4], code[5], code[6], code[7]));
    store_eight<false>(static_cast<int8_t *>(a.out.codes) + row * a.out.codes_stride + at, at, a.width,
                       __builtin_bit_cast(Eight<int8_t>::type, all));
    if ((at & (kGroup - 1)) == 0) static_cast<unsigned short *>(a.out.scales)[row * a.out.scales_stride + at / kGroup] = __float_as_uint(s) >> 16;
}

// A checkpoint's rows from `first` on.
deft_checkpoint_t rows_from(const deft_checkpoint_t &c, int64_t first)
{
    return {static_cast<int8_t *>(c.codes) + first * c.codes_stride, c.codes_stride,
            static_cast<unsigned short *>(c.scales) + first * c.scales_stride, c.scales_stride};
}

template <typename S> constexpr float kMost = 3.402823466e38f;
template <> constexpr float kMost<f16> = 65504.0f;
template <> constexpr float kMost<bf16> = 3.38953139e38f;

// T, P: the operand that it becomes (one array of S itself, or three of bf16).
template <typename S, typename T, int P>
__global__ void __launch_bounds__(256) restore_kernel(RestoreArgs a)
{
    int n, piece;
    if (!a.by.own(blockIdx.x, &n, &piece)) return;
    const int64_t row = n;
    const int at = piece * kEight;
    float x[kEight] = {};
    if (row < a.rows && at < a.cols) {
        const float s = (float)static_cast<const bf16 *>(a.from.scales)[row * a.from.scales_stride + at / kGroup];
        const Eight<int8_t>::type v = load_eight<false>(static_cast<const int8_t *>(a.from.codes) + row * a.from.codes_stride + at, at, a.cols);
#pragma unroll
        for (int r = 0; r < kEight; ++r) x[r] = checkpoint_value(v[r], s, kMost<S>);
    }
    typename Eight<T>::type y[P];
#pragma unroll
    for (int r = 0; r < kEight; ++r) {
        if constexpr (P == 3) {
            bf16 p[3];
            split3(x[r], p);
#pragma unroll
            for (int k = 0; k < 3; ++k) y[k][r] = p[k];
        } else {
            y[0][r] = (T)x[r];
        }
    }
#pragma unroll
    for (int k = 0; k < P; ++k) store_eight<false>(static_cast<T *>(a.out) + k * a.out_plane + row * a.out_ld + at, at, a.cols_to, y[k]);
}

template <typename S>
hipError_t store(const deft_checkpoint_call_t &c, hipStream_t st)
{
    return by_launches(c.n_rows, ((int64_t)c.width + kGroup - 1) / kGroup * kGroup, [&](int64_t first, const RowPieces &by) {
        const StoreArgs a = {by.rows, c.width, static_cast<const S *>(c.x) + first * c.x_stride, c.x_stride, rows_from(c.out, first), by};
        store_kernel<S><<<by.blocks(), 256, 0, st>>>(a);
        return hipGetLastError();
    });
}

template <typename S, typename T, int P>
hipError_t restore(const RestoreArgs &c, hipStream_t st)
{
    return by_launches(c.rows_to, c.cols_to, [&](int64_t first, const RowPieces &by) {
        RestoreArgs a = c;
        a.rows = (int)(c.rows - first);   // (fewer than none where all of them are zeros)
        a.rows_to = by.rows;
        a.from = rows_from(c.from, first);
        a.out = static_cast<T *>(c.out) + first * c.out_ld;
        a.by = by;
        restore_kernel<S, T, P><<<by.blocks(), 256, 0, st>>>(a);
        return hipGetLastError();
    });
}

}  // namespace

hipError_t checkpoint_launch(int dtype, const deft_checkpoint_call_t &c, hipStream_t st)
{
    if (dtype == DEFT_F32) return store<float>(c, st);
    if (dtype == DEFT_F16) return store<f16>(c, st);
    return store<bf16>(c, st);
}

hipError_t restore_launch(int dtype, const deft_restore_call_t &c, hipStream_t st)
{
    const RestoreArgs a = {c.n_rows, c.width, c.n_rows, c.width, c.from, c.out, c.out_stride, 0, {}};
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
