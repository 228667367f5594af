// Operands as the products read them, and a product's launch: what the head and the feed-forward block share.
#pragma once
#include "ends_product.h"

namespace deft {
namespace {

// ---- operands as the products read them ------------------------------------------------------

struct PackArgs {
    const void *src;
    int64_t src_stride;
    int rows, cols;
    const int *row_of, *rows_dev;   // packed positions, or NULL
    void *out;                      // [rows up to a tile][out_ld], zeros beyond the source
    int64_t out_ld, out_plane;
    void *out_t;                    // [cols][t_ld]; or NULL
    int64_t t_ld, t_plane;
    const float *power, *most;      // out_t's columns are scaled by power[row] / most; or NULL
};

// 16 bytes a thread, four at a time, one row's after the other.  Bound by memory (30011
// rows of 1021 16-bit elements, 1026 apart: 24.5 us, 5.0 TB/s read and written; in tiles of 64 x 64 33 us).
template <typename S, typename T, int P>
__device__ __forceinline__ void pack_rows(const PackArgs &a, unsigned block)
{
    typedef S S8 __attribute__((ext_vector_type(8), aligned(sizeof(S))));
    typedef T T8 __attribute__((ext_vector_type(8)));
    const unsigned pieces = (unsigned)(a.out_ld >> 3), first = block * 1024 + threadIdx.x;
    const int rows = a.rows_dev ? *a.rows_dev : a.rows, rows_up = (rows + kTile - 1) / kTile * kTile;
    S x[4][8] = {};
    unsigned row[4], col[4];
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        row[q] = (first + q * 256) / pieces;
        col[q] = ((first + q * 256) - row[q] * pieces) * 8;
        if (row[q] >= (unsigned)rows) continue;
        const S *from = static_cast<const S *>(a.src) + (int64_t)(a.row_of ? a.row_of[row[q]] : (int)row[q]) * a.src_stride + col[q];
        if ((int)col[q] + 8 <= a.cols) {
            const S8 v = *reinterpret_cast<const S8 *>(from);
#pragma unroll
            for (int i = 0; i < 8; ++i) x[q][i] = v[i];
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if ((int)col[q] + i < a.cols) x[q][i] = from[i];
        }
    }
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        if (row[q] >= (unsigned)rows_up) continue;
        T8 y[P];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            if constexpr (P == 3) {
                bf16 s[3];
                split3(x[q][i], s);
#pragma unroll
                for (int p = 0; p < 3; ++p) y[p][i] = s[p];
            } else {
                y[0][i] = x[q][i];
            }
        }
#pragma unroll
        for (int p = 0; p < P; ++p)
            *reinterpret_cast<T8 *>(static_cast<T *>(a.out) + p * a.out_plane + (int64_t)row[q] * a.out_ld + col[q]) = y[p];
    }
}

template <typename S, typename T, int P>
__global__ void __launch_bounds__(256) pack_rows_kernel(PackArgs a) { pack_rows<S, T, P>(a, blockIdx.x); }

// Several matrices' rows in one launch (a launch alone is 5 us, as long as a small matrix takes).
constexpr int kPackMost = 5;
struct PackMany {
    PackArgs of[kPackMost];
    unsigned blocks[kPackMost];   // that each takes, none behind the last one
};

template <typename S, typename T, int P>
__global__ void __launch_bounds__(256) pack_many_kernel(PackMany a)
{
    unsigned block = blockIdx.x;
#pragma unroll
    for (int i = 0; i < kPackMost; ++i) {
        if (block < a.blocks[i]) return pack_rows<S, T, P>(a.of[i], block);
        block -= a.blocks[i];
    }
}

inline unsigned pack_blocks(int64_t rows, int64_t out_ld) { return (unsigned)(up(rows * (out_ld >> 3), 1024) / 1024); }

// Whether a product can read rows where they are: whole steps where their elements are its k (the next row's elements, or
// what lies between rows, must not come in), 16-byte pieces, offsets within 32 bits.
inline bool in_place(const void *p, int64_t stride, int cols, int whole = kStep)
{
    return cols % whole == 0 && stride % 8 == 0 && ((uintptr_t)p & 15) == 0 && stride <= (1 << 22);
}

// ---- launches -------------------------------------------------------------------------------

template <typename T, typename O, int E, int WM, int WN, int MT, int NT, bool SPLIT>
hipError_t product_shape(const ProductArgs &p, hipStream_t st)
{
    constexpr int TM = WM * MT * 16, TN = WN * NT * 16, kLds = product_lds(TM, TN, WM * WN * kWave);
    constexpr int kColumns = E == kGate ? TM / 2 : TM;
    const int grid = ((p.m + kColumns - 1) / kColumns) * ((p.n + TN - 1) / TN) * p.splits;
    product_kernel<T, O, E, WM, WN, MT, NT, SPLIT><<<grid, WM * WN * kWave, kLds, st>>>(p);
    return hipGetLastError();
}

template <typename T, typename O, int E, int WM, int WN, int MT, int NT, bool SPLIT>
hipError_t allow_shape()
{
    return hipFuncSetAttribute(reinterpret_cast<const void *>(&product_kernel<T, O, E, WM, WN, MT, NT, SPLIT>),
                               hipFuncAttributeMaxDynamicSharedMemorySize, product_lds(WM * MT * 16, WN * NT * 16, WM * WN * kWave));
}

}  // namespace
}  // namespace deft
