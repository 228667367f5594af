// What the operators of a layer's feed-forward block share: the arguments of its products' epilogues, checkpoints in
// device code, and the launch interface between the C ABI (block_api.hip) and the kernels.
#pragma once
#include "../../include/deft_block.h"
#include "ends_shapes.h"

namespace deft {

// Beside the operands (ends_product.h).  Panels have 256 columns: [columns / 256][rows][256].
struct FfnArgs {
    const void *a2;                  // kGate: the other projection's rows; kInput: those that the second half of b multiplies
    int64_t a2_ld, a2_plane;
    int64_t a_panel;                 // kOuter: elements between a's panels (256: rows as they are)
    int64_t d_half;                  // kInput: elements between b's halves
    int arrays;                      // 16-bit types: 1, or 2 where h and d have a second array, what rounding took of the first
    int64_t b_array;                 // kOut, kInput: elements between the two of b
    int64_t a_step, b_step;          // kOuter: elements from a step's rows to the next one's (0: the second array's step takes the same)
    // kGate, kGateGrad
    int activation;
    int cols_up;                     // columns of the panels of h, and of each half of d's
    void *h, *d;                     // panels: hidden activations; derivatives by gate, and behind them by up; or NULL
    int64_t panel, h_plane, d_plane; // elements between panels, between arrays
    deft_saved_t saved;              // the projections
    const float *largest;            // 16-bit floats: [kFactorParts], which tell the power of two that d is held times; or NULL
    // kOut, kInput, kOuter: rows n < half go to the first, the others, less `half`, to the second
    void *out[2];                    // or NULL
    int64_t out_ld[2];
    int half, rows;                  // rows that each has
};

constexpr int kGroup = DEFT_CHECKPOINT_GROUP;
constexpr int kFactorParts = 256;

// How workgroups of 256 threads go through rows' pieces of eight elements, a piece each: as many whole rows as a workgroup has
// threads for, or a part of one.  (Worked out on the host: divisions by a thread would be half of a checkpoint's instructions.)
struct RowPieces {
    int rows, pieces, rows_each, parts;    // pieces and parts of a row
    float one_by;
    RowPieces() = default;
    RowPieces(int64_t n, int64_t cols)
        : rows((int)n), pieces((int)((cols + 7) / 8)), rows_each(pieces < 256 ? 256 / pieces : 1), parts((pieces + 255) / 256), one_by(1.0f / (float)pieces)
    {
    }
    __host__ __device__ unsigned blocks() const { return (unsigned)(((int64_t)rows + rows_each - 1) / rows_each) * (unsigned)parts; }
    // Rows that a launch can have, whose threads have to be fewer than 2^32.
    int64_t most_rows() const { return (int64_t)(((1 << 24) - 1) / parts) * rows_each; }

    // The row and piece of this thread, or false.
    __device__ bool own(unsigned block, int *row, int *piece) const
    {
        const int i = threadIdx.x;
        if (parts == 1) {   // (a whole number less than 256 and a half, divided: never within the error of a whole number)
            const int in_block = (int)(((float)i + 0.5f) * one_by);
            *row = (int)block * rows_each + in_block;
            *piece = i - in_block * pieces;
            return in_block < rows_each && *row < rows;
        }
        const unsigned of = block / (unsigned)parts;
        *row = (int)of;
        *piece = (int)(block - of * (unsigned)parts) * 256 + i;
        return *piece < pieces;
    }
};

// As many launches as n rows of `cols` take (one, but of about a million rows of more than 30720 columns): launch(its first row,
// RowPieces of its rows).
template <typename F>
hipError_t by_launches(int64_t n, int64_t cols, F launch)
{
    const int64_t most = RowPieces(n, cols).most_rows();
    hipError_t e = hipSuccess;
    for (int64_t first = 0; first < n && e == hipSuccess; first += most) e = launch(first, RowPieces(n - first < most ? n - first : most, cols));
    return e;
}

constexpr float kCodes8 = 127.0f, kCodes16 = 32767.0f;   // the largest codes
constexpr float kShift = 12582912.0f;   // 3 2^22: a sum with it is a whole number, in the low bits

// The scale of a group: the smallest number of 8 significant bits, at least 2^-126, `most` times which reaches `top`.
// (`one_by`: 1 / most.  The product's rounding, and the divisor's, may end a step of 8 bits beside it: both neighbours are tried.)
__device__ __forceinline__ float checkpoint_scale(float top, float most, float one_by)
{
    constexpr float kLeast = 1.17549435e-38f;
    const unsigned up8 = (__float_as_uint(fmaxf(top * one_by, kLeast)) + 0xffffu) & 0xffff0000u;
    const float s = __uint_as_float(up8), below = __uint_as_float(up8 - 0x10000u), above = __uint_as_float(up8 + 0x10000u);
    if (fmaf(s, most, -top) < 0.0f) return above;
    return below >= kLeast && fmaf(below, most, -top) >= 0.0f ? below : s;
}

__device__ __forceinline__ bool is_finite(float x) { return (__float_as_uint(x) & 0x7f800000u) != 0x7f800000u; }

// What a code stands for, up to `most`, the largest number of its type: the nearest multiple of s may lie beyond.  (A projection's group
// with a sum that is not finite has NaN as its scale, whatever its codes are: the limits alone would make a number of it.)
__device__ __forceinline__ float checkpoint_value(int code, float s, float most)
{
    return code == -128 || s != s ? __builtin_nanf("") : fminf(fmaxf((float)code * s, -most), most);
}

// ---- launches (each returns hipGetLastError() of its launches) ------------------------------

// `x`: its checkpoint as an operand of P arrays of T (ends_operands.h): rows up to a tile, zeros beyond the source.
struct RestoreArgs {
    int rows, cols;                  // of the checkpoint
    int rows_to, cols_to;            // that are written, zeros beyond
    deft_checkpoint_t from;
    void *out;
    int64_t out_ld, out_plane;
    RowPieces by;
};
hipError_t checkpoint_launch(int dtype, const deft_checkpoint_call_t &a, hipStream_t st);
hipError_t restore_launch(int dtype, const deft_restore_call_t &a, hipStream_t st);
hipError_t restore_operand_launch(int dtype, const RestoreArgs &a, hipStream_t st);

// 16-bit floats: the largest finite magnitudes of the rows' parts.
struct LargestArgs {
    int rows, cols;
    const f16 *x;
    int64_t x_stride;
    float *largest;    // [kFactorParts]
    RowPieces by;
};
hipError_t ffn_largest_launch(const LargestArgs &a, hipStream_t st);

struct FfnPlan {
    int64_t scratch_bytes = 0;
    // offsets into the scratch memory
    int64_t largest, x, grad_y, w_gate, w_up, w_down, h, d, gate, up, sums;
};
void ffn_plan(int dtype, int max_rows, int max_hidden, int max_inner, bool grad, int compute_units, FfnPlan *plan);
// Rows up to which the forward pass goes to the kernels for few (block_ffn.h has the reasons), of matrices of `size` elements; `whole`: all
// that it reads can be read in place.  The fewest are those of the largest matrices, read in place.
inline int few_rows(bool f32, int64_t size, bool whole)
{
    return f32 ? kFew : size <= 2 << 20 ? (whole ? 32 : kFew) : size <= 6 << 20 && !whole ? 32 : 16;
}
hipError_t ffn_prepare();            // kernel attributes, on the current device
hipError_t ffn_launch(const FfnPlan &plan, int dtype, const deft_ffn_t &a, void *scratch, int compute_units, hipStream_t st);
hipError_t ffn_grad_launch(const FfnPlan &plan, int dtype, const deft_ffn_grad_t &a, void *scratch, int compute_units, hipStream_t st);

}  // namespace deft
