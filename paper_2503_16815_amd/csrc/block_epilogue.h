// What the feed-forward block's products do with their sums: act(gate) * up as they leave the matrix units, the
// derivatives by both projections, and the rounded outputs.
//
// All pass their sums through LDS, sixteen rows of a wavefront's tile at a time, so that a lane has eight
// neighbouring columns of one row, what it loads and stores is 16 bytes, a row's lanes are next to each other, and a
// checkpoint's group of 32 is four lanes'.  What the derivatives' epilogue reads of the rows ahead is on its way meanwhile.
//
// Bound by memory, which is idle while the sums are made: the derivatives by both projections of 8192 x 6400 bf16 read 216 MB and write
// 315 after a product of 140 us, 270 to 280 in all (without the writes 175, without the reads 226; with tiles two to a compute unit, one's
// epilogue beside the other's sums, the same).
#pragma once
#include <type_traits>

#include "block.h"

namespace deft {

constexpr int kEight = 8;   // columns of a lane

// An activation of the gate and its derivative.  kExact: 32-bit outputs; otherwise exponentials and reciprocals are the
// hardware's as they come (off by 1 or 2 units of the last 24 bits, and |a| of them in the exponential), far below the rounding
// to 16 bits that follows.
template <int KIND, bool kExact>
__device__ __forceinline__ void act_of(float a, float &y, float &slope)
{
    constexpr float kLog2e = 1.44269504f, kLog2eRest = 1.92596303e-8f;
    const auto exp_of = [](float x) {
        if constexpr (!kExact) return __builtin_amdgcn_exp2f(x * kLog2e);
        // (what x log2 e loses by its rounding, times ln 2; limits beyond which 1 + exp x is 1 or the gate's share of it 0)
        const float within = fminf(fmaxf(x, -104.0f), 88.0f), power = within * kLog2e;
        const float rest = fmaf(within, kLog2e, -power) + within * kLog2eRest, y = __builtin_amdgcn_exp2f(power);
        return x == x ? fmaf(y, 0.693147181f * rest, y) : x;   // (the limits would make a number of NaN)
    };
    const auto inverse = [](float x) {
        const float y = __builtin_amdgcn_rcpf(x);
        return kExact ? fmaf(fmaf(-x, y, 1.0f), y, y) : y;
    };
    if constexpr (KIND == DEFT_SILU) {
        const float p = inverse(1.0f + exp_of(-a));
        y = a * p;
        slope = fmaf(y, 1.0f - p, p);
    } else if constexpr (KIND == DEFT_GELU) {
        const float e = exp_of(-0.5f * a * a);
        float p;   // the normal distribution's share below a
        if constexpr (kExact) {
            p = 0.5f * erfcf(-0.707106781f * a);
        } else {
            // Of the share beyond |a|: exp(-a^2 / 2) times a polynomial in 1 / (1 + 0.3 |a|), fitted to erfcx(|a| / sqrt 2) / 2 for
            // |a| <= 14 (where 16-bit outputs are 0 beyond) with the least relative error, 8.5e-6 in 32 bits.
            const float t = inverse(fmaf(0.3f, fabsf(a), 1.0f));
            float q = -0.0770978130f;
            q = fmaf(q, t, 0.216038091f);
            q = fmaf(q, t, -0.0169490538f);
            q = fmaf(q, t, 0.144196782f);
            q = fmaf(q, t, 0.113741861f);
            q = fmaf(q, t, 0.120074235f) * t * e;
            p = a < 0.0f ? q : 1.0f - q;
        }
        y = a * p;
        slope = fmaf(a, 0.398942280f * e, p);
    } else if constexpr (KIND == DEFT_GELU_TANH) {   // (1 + tanh(u / 2)) / 2 = 1 / (1 + exp(-u))
        const float square = a * a, u = 1.595769122f * a * fmaf(0.044715f, square, 1.0f), p = inverse(1.0f + exp_of(-u));
        const float rest = p - p * p;   // (0 where the square may be infinite)
        y = a * p;
        slope = p + (rest == 0.0f ? 0.0f : rest * 1.595769122f * a * fmaf(0.134145f, square, 1.0f));
    } else {   // (NaN stays, in both)
        y = a < 0.0f ? 0.0f : a;
        slope = a > 0.0f ? 1.0f : a == a ? 0.0f : a;
    }
}

template <typename O> struct Eight {
    typedef O type __attribute__((ext_vector_type(8), aligned(sizeof(O))));
};

// Eight elements of a row from column `at` on, where `cols` is the first that the row does not have (0: none of it is there).
// kInside: it has them all.
template <bool kInside, typename O>
__device__ __forceinline__ void store_eight(O *to, int at, int cols, const typename Eight<O>::type &y)
{
    if (kInside || at + kEight <= cols) {
        *reinterpret_cast<typename Eight<O>::type *>(to) = y;
    } else {
#pragma unroll
        for (int r = 0; r < kEight; ++r)
            if (at + r < cols) to[r] = y[r];
    }
}

template <bool kInside, typename O>
__device__ __forceinline__ typename Eight<O>::type load_eight(const O *from, int at, int cols)
{
    typename Eight<O>::type y = {};
    if (kInside || at + kEight <= cols) {
        y = *reinterpret_cast<const typename Eight<O>::type *>(from);
    } else {
#pragma unroll
        for (int r = 0; r < kEight; ++r)
            if (at + r < cols) y[r] = from[r];
    }
    return y;
}

template <typename O>
__device__ __forceinline__ typename Eight<O>::type rounded(const float (&x)[kEight])
{
    typename Eight<O>::type y;
#pragma unroll
    for (int r = 0; r < kEight; ++r) y[r] = (O)x[r];
    return y;
}

// The largest of four neighbouring lanes.
__device__ __forceinline__ unsigned quad_max(unsigned x)
{
    x = max(x, (unsigned)__builtin_amdgcn_update_dpp(0, (int)x, 0xb1, 0xf, 0xf, true));
    return max(x, (unsigned)__builtin_amdgcn_update_dpp(0, (int)x, 0x4e, 0xf, 0xf, true));
}

// The low bytes of four numbers.
__device__ __forceinline__ unsigned pack_bytes(unsigned a, unsigned b, unsigned c, unsigned d)
{
    return __builtin_amdgcn_perm(__builtin_amdgcn_perm(d, c, 0x0c0c0400), __builtin_amdgcn_perm(b, a, 0x0c0c0400), 0x05040100);
}

// Sums as codes C of a checkpoint, whose group this and three neighbouring lanes hold.  A group with a sum that is not finite
// gets NaN as its scale.  Codes are the low bits of x / s + 3 2^22, rounded once (a sum in 32 bits is itself unsure of a half).
// kStaySigned: of 16 bits, positive sums get codes of at least `least`, 0 or 1 (relu's derivative is 1 down to 0: with a code of 0 for what
// is below half a step 2e-5 of a gate's elements lose theirs, 5e-3 of the derivative's norm, 25 times what 16-bit floats round).
template <bool kInside, typename C, bool kStaySigned>
__device__ __forceinline__ void store_codes(deft_checkpoint_t to, int n, int at, int cols, const float (&x)[kEight], float least = 0.0f)
{
    constexpr bool k8 = sizeof(C) == 1;
    constexpr float kLargest = k8 ? kCodes8 : kCodes16;
    unsigned top = 0;   // (as whole numbers infinity is above all finite magnitudes and NaN above infinity)
#pragma unroll
    for (int r = 0; r < kEight; ++r) top = max(top, kInside || at + r < cols ? __float_as_uint(x[r]) & 0x7fffffffu : 0u);
    top = quad_max(top);
    const float s = checkpoint_scale(__uint_as_float(top), kLargest, 1.0f / kLargest);
    const float inverse = __builtin_amdgcn_rcpf(s);
    unsigned c[kEight];
#pragma unroll
    for (int r = 0; r < kEight; ++r) {
        const float code = fmaf(x[r], inverse, kShift);
        c[r] = __float_as_uint(kStaySigned && !k8 && x[r] > 0.0f ? fmaxf(code, kShift + least) : code);
    }
    typename Eight<C>::type y;
    if constexpr (k8) {
        uint2 all;
        all.x = pack_bytes(c[0], c[1], c[2], c[3]);
        all.y = pack_bytes(c[4], c[5], c[6], c[7]);
        y = __builtin_bit_cast(typename Eight<C>::type, all);
    } else {
        uint4 all;
        all.x = __builtin_amdgcn_perm(c[1], c[0], 0x05040100);
        all.y = __builtin_amdgcn_perm(c[3], c[2], 0x05040100);
        all.z = __builtin_amdgcn_perm(c[5], c[4], 0x05040100);
        all.w = __builtin_amdgcn_perm(c[7], c[6], 0x05040100);
        y = __builtin_bit_cast(typename Eight<C>::type, all);
    }
    store_eight<kInside>(static_cast<C *>(to.codes) + n * to.codes_stride + at, at, cols, y);
    if ((at & (kGroup - 1)) == 0 && (kInside || at < cols))
        static_cast<unsigned short *>(to.scales)[n * to.scales_stride + at / kGroup] = top < 0x7f800000u ? __float_as_uint(s) >> 16 : 0x7fc0;
}

// A projection as it is kept: in 8 bits, or in as many as O has.
template <bool kInside, typename O, bool kStaySigned>
__device__ __forceinline__ void store_saved(int kind, deft_checkpoint_t to, int n, int at, int cols, const float (&x)[kEight], float least = 0.0f)
{
    if (kind == DEFT_SAVE_PACKED) store_codes<kInside, int8_t, false>(to, n, at, cols, x);
    else if constexpr (sizeof(O) == 4) store_eight<kInside>(static_cast<float *>(to.codes) + n * to.codes_stride + at, at, cols, rounded<float>(x));
    else store_codes<kInside, int16_t, kStaySigned>(to, n, at, cols, x, least);
}

// Eight elements of it as they come from memory: codes of 8 bits in the first two words, of 16 in four, or floats.
template <typename O> struct Kept {
    static constexpr bool kFloats = sizeof(O) == 4;
    i32x4 words, more;
    unsigned scale;
};

template <bool kInside, typename O>
__device__ __forceinline__ void load_saved(int kind, deft_checkpoint_t from, int n, int at, int cols, Kept<O> &k)
{
    k.words = k.more = i32x4{0, 0, 0, 0};
    k.scale = 0;
    if (kind == DEFT_SAVE_PACKED) {
        const uint2 y = __builtin_bit_cast(uint2, load_eight<kInside>(static_cast<const int8_t *>(from.codes) + n * from.codes_stride + at, at, cols));
        k.words[0] = (int)y.x;
        k.words[1] = (int)y.y;
    } else if constexpr (Kept<O>::kFloats) {
        const Eight<float>::type y = load_eight<kInside>(static_cast<const float *>(from.codes) + n * from.codes_stride + at, at, cols);
        k.words = __builtin_bit_cast(i32x4, __builtin_shufflevector(y, y, 0, 1, 2, 3));
        k.more = __builtin_bit_cast(i32x4, __builtin_shufflevector(y, y, 4, 5, 6, 7));
        return;
    } else {
        k.words = __builtin_bit_cast(i32x4, load_eight<kInside>(static_cast<const int16_t *>(from.codes) + n * from.codes_stride + at, at, cols));
    }
    if (kInside || at < cols) k.scale = static_cast<const unsigned short *>(from.scales)[n * from.scales_stride + at / kGroup];
}

template <typename O>
__device__ __forceinline__ void use_saved(int kind, const Kept<O> &k, float (&x)[kEight])
{
    const float s = __uint_as_float(k.scale << 16);
    if (kind == DEFT_SAVE_PACKED) {
#pragma unroll
        for (int r = 0; r < kEight; ++r) x[r] = (float)(int8_t)(k.words[r / 4] >> (8 * (r % 4))) * s;
    } else if constexpr (Kept<O>::kFloats) {
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            x[r] = __int_as_float(k.words[r]);
            x[r + 4] = __int_as_float(k.more[r]);
        }
    } else {
#pragma unroll
        for (int r = 0; r < kEight; ++r) x[r] = (float)(int16_t)(k.words[r / 2] >> (16 * (r % 2))) * s;
    }
}

// What rounding x to y took; of one that the rounding made infinite nothing (x less infinity would be the opposite one, and both
// arrays' products NaN together).
template <typename T>
__device__ __forceinline__ float taken(float x, T y) { return is_finite((float)y) ? x - (float)y : 0.0f; }

// Eight elements of an operand in panels: one array of T, two where the second has what rounding took of the first, or three of bf16
// whose sum they are.
template <typename T, bool SPLIT>
__device__ __forceinline__ void store_operand(T *to, int64_t plane, int arrays, const float (&x)[kEight])
{
    typedef T T8 __attribute__((ext_vector_type(8)));
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
        if (arrays == 2) {
#pragma unroll
            for (int r = 0; r < kEight; ++r) y[r] = (T)taken(x[r], y[r]);
            *reinterpret_cast<T8 *>(to + plane) = y;
        }
    }
}

constexpr __host__ __device__ int epilogue_pitch(int mt) { return mt * 16 + 4; }   // of a row of sums in LDS
constexpr __host__ __device__ int epilogue_floats(int mt) { return 16 * epilogue_pitch(mt); }   // of a wavefront

template <int MT, int NT>
__device__ __forceinline__ void to_lds(const f32x4 (&acc)[MT][NT], int j, float *to)
{
#pragma unroll
    for (int i = 0; i < MT; ++i) *reinterpret_cast<f32x4 *>(to + i * 16) = acc[i][j];
}

// Goes through a wavefront's tile sixteen rows at a time: its sums go to `lds` (the wavefront's own part), and `use(row, sums, ahead)` is
// called with a row's number in the tile, where its sums lie, and what `fetch(row, ahead)` brought; the next sixteen rows' are fetched
// meanwhile.  kLanes lanes have a row, each the same columns of all its rows.  acc[i][j][r] is row row16 + 16 j, column
// part * 4 + 16 i + r.
// kUnroll: the code of all rows that j has, sixteen rows ahead fetched; otherwise one row's, and the next one fetched.
template <typename Ahead, int kLanes, bool kUnroll, int MT, int NT, typename Fetch, typename Use>
__device__ __forceinline__ void by_rows(const f32x4 (&acc)[MT][NT], float *lds, int lane, Fetch fetch, Use use)
{
    static_assert(kLanes <= 16 && kWave % kLanes == 0);
    constexpr int kPitch = epilogue_pitch(MT), kRows = kWave / kLanes, kTimes = 16 / kRows, kDepth = kUnroll ? kTimes : 1;
    const int row16 = lane & 15, part = lane >> 4, own = lane / kLanes;
    Ahead ahead[kDepth];
#pragma unroll
    for (int t = 0; t < kDepth; ++t) fetch(t * kRows + own, ahead[t]);
#pragma clang loop unroll(disable)
    for (int j = 0; j < NT; ++j) {
#pragma unroll
        for (int which = 0; which < NT; ++which)
            if (j == which) {
                to_lds(acc, which, lds + row16 * kPitch + part * 4);
                asm volatile("; sixteen rows, number %0" ::"s"(which));   // (alike, the branches would become one that indexes registers in memory)
            }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");   // (a wavefront's LDS accesses are done in order)
        __builtin_amdgcn_wave_barrier();
        const auto rows = [&](int t, Ahead &a) __attribute__((always_inline)) {
            const int row = t * kRows + own;
            const Ahead now = a;
            if (kDepth < kTimes ? j * kTimes + t + 1 < NT * kTimes : j + 1 < NT) fetch(j * 16 + row + kDepth * kRows, a);
            use(j * 16 + row, lds + row * kPitch, now);
            __builtin_amdgcn_sched_barrier(0);   // (several rows' work at once would not fit the registers)
        };
        if constexpr (kUnroll) {
#pragma unroll
            for (int t = 0; t < kTimes; ++t) rows(t, ahead[t]);
        } else {
#pragma clang loop unroll(disable)
            for (int t = 0; t < kTimes; ++t) rows(t, ahead[0]);
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
    }
}

// The same piece by piece of eight columns, rows of any number of pieces (a tile of 192 columns has 24), nothing fetched.
template <int MT, int NT, typename Use>
__device__ __forceinline__ void by_pieces(const f32x4 (&acc)[MT][NT], float *lds, int lane, Use use)
{
    constexpr int kPitch = epilogue_pitch(MT), kLanes = MT * 2;
    const int row16 = lane & 15, part = lane >> 4;
#pragma clang loop unroll(disable)
    for (int j = 0; j < NT; ++j) {
#pragma unroll
        for (int which = 0; which < NT; ++which)
            if (j == which) {
                to_lds(acc, which, lds + row16 * kPitch + part * 4);
                asm volatile("; sixteen rows, number %0" ::"s"(which));   // (alike, the branches would become one that indexes registers in memory)
            }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
#pragma clang loop unroll(disable)
        for (int at = lane; at < 16 * kLanes; at += kWave) {
            const int row = at / kLanes;
            use(j * 16 + row, (at - row * kLanes) * kEight, lds + row * kPitch);
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

struct Nothing {};

// The power of two that brings the largest of kFactorParts magnitudes to 1 .. 2, and its reciprocal.
__device__ __forceinline__ float2 factor_of(const float *largest, int lane)
{
    const f32x4 x = *reinterpret_cast<const f32x4 *>(largest + lane * 4);
    const float top = wave_max(fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3])));
    const unsigned power = __float_as_uint(top) & 0x7f800000u;   // (a 16-bit float's: none is below 2^-24)
    return power ? make_float2(__uint_as_float(0x7f000000u - power), __uint_as_float(power)) : make_float2(1.0f, 1.0f);
}

template <int KIND, bool kExact>
__device__ __forceinline__ void act_of(const float (&a)[kEight], float (&y)[kEight], float (&slope)[kEight])
{
#pragma unroll
    for (int r = 0; r < kEight; ++r) act_of<KIND, kExact>(a[r], y[r], slope[r]);
}

// Whatever the activation is.
template <bool kExact>
__device__ __forceinline__ void act_of(int kind, const float (&a)[kEight], float (&y)[kEight], float (&slope)[kEight])
{
    if (kind == DEFT_SILU) act_of<DEFT_SILU, kExact>(a, y, slope);
    else if (kind == DEFT_GELU) act_of<DEFT_GELU, kExact>(a, y, slope);
    else if (kind == DEFT_GELU_TANH) act_of<DEFT_GELU_TANH, kExact>(a, y, slope);
    else act_of<DEFT_RELU, kExact>(a, y, slope);
}

// What a wavefront's tile is to the epilogues below.
struct Tile {
    float *lds;
    int lane, m, n;      // its first column (of either projection) and row
    int n_rows, cols;    // that the matrix has
};

// Eight elements of both projections, of row n and from column `at` on; own_cols: the columns that the row has (0: no such row, zeros
// in h).  h_at: where h has the column.  kInside: the row and the group's columns are there, and operands are one array (or three).
template <bool kInside, typename T, typename O, bool SPLIT, typename Act>
__device__ __forceinline__ void use_gate(const FfnArgs &f, int n, int at, int own_cols, const float (&gate)[kEight], const float (&up)[kEight], T *h_at, Act act)
{
    float y[kEight], slope[kEight];
    if (f.saved.kind != DEFT_SAVE_NONE) {
        store_saved<kInside, O, true>(f.saved.kind, f.saved.gate, n, at, own_cols, gate, f.activation == DEFT_RELU ? 1.0f : 0.0f);
        store_saved<kInside, O, false>(f.saved.kind, f.saved.up, n, at, own_cols, up);
    }
    if (!f.h || (!kInside && at >= f.cols_up)) return;
    act(gate, y, slope);
#pragma unroll
    for (int r = 0; r < kEight; ++r) y[r] = kInside || at + r < own_cols ? y[r] * up[r] : 0.0f;
    store_operand<T, SPLIT>(h_at + (int64_t)n * 256, f.h_plane, kInside ? 1 : f.arrays, y);
}

template <typename O> struct Ahead {
    Kept<O> gate, up;
};

// And of the derivative by h.
template <bool kInside, typename T, typename O, bool SPLIT, typename Act>
__device__ __forceinline__ void use_gate_grad(const FfnArgs &f, int n, int at, int own_cols, const float (&by_h)[kEight], const Ahead<O> &a, float factor,
                                              T *h_at, T *d_at, Act act)
{
    if (!kInside && at >= f.cols_up) return;
    float gate[kEight], up[kEight], y[kEight], slope[kEight], h[kEight];
    use_saved(f.saved.kind, a.gate, gate);
    use_saved(f.saved.kind, a.up, up);
    act(gate, y, slope);
#pragma unroll
    for (int r = 0; r < kEight; ++r) {
        const bool here = kInside || at + r < own_cols;
        const float d = __is_same(T, f16) ? by_h[r] * factor : by_h[r];
        h[r] = here ? y[r] * up[r] : 0.0f;
        gate[r] = here ? d * up[r] * slope[r] : 0.0f;
        up[r] = here ? d * y[r] : 0.0f;
    }
    const int64_t from = (int64_t)n * 256;
    if (f.h) store_operand<T, SPLIT>(h_at + from, f.h_plane, kInside ? 1 : f.arrays, h);
    if (f.d) {
        store_operand<T, SPLIT>(d_at + from, f.d_plane, kInside ? 1 : f.arrays, gate);
        store_operand<T, SPLIT>(d_at + (f.cols_up >> 8) * f.panel + from, f.d_plane, kInside ? 1 : f.arrays, up);
    }
}

template <bool kInside, typename O>
__device__ __forceinline__ void load_ahead(const FfnArgs &f, int n, int at, int own_cols, Ahead<O> &a)
{
    load_saved<kInside>(f.saved.kind, f.saved.gate, n, at, own_cols, a.gate);
    load_saved<kInside>(f.saved.kind, f.saved.up, n, at, own_cols, a.up);
}

// KIND: the activation; or -1, whichever the call has.
template <bool kGrad, int KIND, bool kInside, typename T, typename O, int MT, int NT, bool SPLIT>
__device__ __forceinline__ void act_rows(const FfnArgs &f, const f32x4 (&acc)[MT][NT], const Tile &t)
{
    constexpr int kLanes = kGrad ? MT * 2 : MT;
    const int col = (t.lane % kLanes) * kEight, at = t.m + col;
    const int64_t place = (at >> 8) * f.panel + (at & 255);
    T *const h_at = static_cast<T *>(f.h) + place;
    const auto act = [&](const float (&a)[kEight], float (&y)[kEight], float (&slope)[kEight]) __attribute__((always_inline)) {
        if constexpr (KIND >= 0) act_of<KIND, SPLIT>(a, y, slope);
        else act_of<SPLIT>(f.activation, a, y, slope);
    };
    const auto cols_of = [&](int n) __attribute__((always_inline)) { return kInside || n < t.n_rows ? t.cols : 0; };
    if constexpr (kGrad) {
        T *const d_at = static_cast<T *>(f.d) + place;
        const float factor = __is_same(T, f16) && f.largest ? factor_of(f.largest, t.lane).x : 1.0f;
        const auto use = [&](int row, const float *sums, const Ahead<O> &a) __attribute__((always_inline)) {
            float by_h[kEight];
            read_eight(sums + col, by_h);
            use_gate_grad<kInside, T, O, SPLIT>(f, t.n + row, at, cols_of(t.n + row), by_h, a, factor, h_at, d_at, act);
        };
        const auto fetch = [&](int row, Ahead<O> &a) __attribute__((always_inline)) { load_ahead<kInside>(f, t.n + row, at, cols_of(t.n + row), a); };
        if constexpr (SPLIT) {   // (nothing ahead: 16 more registers would push sums out of theirs)
            by_rows<Nothing, kLanes, false>(acc, t.lds, t.lane, [](int, Nothing &) {},
                                            [&](int row, const float *sums, const Nothing &) __attribute__((always_inline)) {
                                                Ahead<O> a;
                                                fetch(row, a);
                                                use(row, sums, a);
                                            });
        } else {
            by_rows<Ahead<O>, kLanes, (KIND >= 0)>(acc, t.lds, t.lane, fetch, use);
        }
    } else {
        by_rows<Nothing, kLanes, (KIND >= 0)>(
            acc, t.lds, t.lane, [](int, Nothing &) {},
            [&](int row, const float *sums, const Nothing &) __attribute__((always_inline)) {
                float gate[kEight], up[kEight];
                read_eight(sums + (col >> 4) * 32 + (col & 15), gate);   // (sixteens of columns are gate and up in turn)
                read_eight(sums + (col >> 4) * 32 + 16 + (col & 15), up);
                use_gate<kInside, T, O, SPLIT>(f, t.n + row, at, cols_of(t.n + row), gate, up, h_at, act);
            });
    }
}

template <bool kGrad, typename T, typename O, int MT, int NT, bool SPLIT>
__device__ __forceinline__ void act_epilogue(const FfnArgs &f, const f32x4 (&acc)[MT][NT], const Tile &t)
{
    static_assert(MT % 4 == 0);   // whole groups of 32
    const bool inside = f.arrays == 1 && t.n + NT * 16 <= t.n_rows && t.m + MT * (kGrad ? 16 : 8) <= t.cols;
    if (!inside) return act_rows<kGrad, -1, false, T, O, MT, NT, SPLIT>(f, acc, t);
    if constexpr (SPLIT) {   // (32-bit operands are multiplied six times over: less of the whole, and twice the registers)
        act_rows<kGrad, -1, true, T, O, MT, NT, SPLIT>(f, acc, t);
    } else {
        if (f.activation == DEFT_SILU) act_rows<kGrad, DEFT_SILU, true, T, O, MT, NT, SPLIT>(f, acc, t);
        else if (f.activation == DEFT_GELU) act_rows<kGrad, DEFT_GELU, true, T, O, MT, NT, SPLIT>(f, acc, t);
        else if (f.activation == DEFT_GELU_TANH) act_rows<kGrad, DEFT_GELU_TANH, true, T, O, MT, NT, SPLIT>(f, acc, t);
        else act_rows<kGrad, DEFT_RELU, true, T, O, MT, NT, SPLIT>(f, acc, t);
    }
}

// Where row n of a product's result goes, or NULL.
template <typename O>
__device__ __forceinline__ O *out_row(const FfnArgs &f, int n)
{
    const int which = n >= f.half ? 1 : 0, row = n - (which ? f.half : 0);
    O *out = static_cast<O *>(which ? f.out[1] : f.out[0]);
    return out && row < f.rows ? out + row * (which ? f.out_ld[1] : f.out_ld[0]) : nullptr;
}

// A lane's columns of a row: out = alpha x, or that and what is there, rounded once.
template <bool kInside, typename O>
__device__ __forceinline__ void store_out(O *row, int at, int cols, const float (&x)[kEight], float alpha, int add)
{
    float y[kEight] = {};
    if (add) {
        const auto there = load_eight<kInside>(row + at, at, cols);
#pragma unroll
        for (int r = 0; r < kEight; ++r) y[r] = (float)there[r];
    }
#pragma unroll
    for (int r = 0; r < kEight; ++r) y[r] += alpha * x[r];
    store_eight<kInside>(row + at, at, cols, rounded<O>(y));
}

// A part of the sums: rows of `ld` elements, a multiple of 8.
template <int MT, int NT>
__device__ __forceinline__ void sums_epilogue(float *sums, int64_t ld, const f32x4 (&acc)[MT][NT], const Tile &t)
{
    by_pieces(acc, t.lds, t.lane, [&](int row, int col, const float *from) __attribute__((always_inline)) {
        const int n = t.n + row, at = t.m + col;
        if (n >= t.n_rows || at >= t.cols) return;
        float x[kEight];
        read_eight(from + col, x);
        store_eight<true>(sums + n * ld + at, at, t.cols, rounded<float>(x));
    });
}

// The sums are the result.
template <typename O, int MT, int NT>
__device__ __forceinline__ void out_epilogue(const FfnArgs &f, const f32x4 (&acc)[MT][NT], const Tile &t, int add)
{
    const float alpha = __is_same(O, f16) && f.largest ? factor_of(f.largest, t.lane).y : 1.0f;
    by_pieces(acc, t.lds, t.lane, [&](int row, int col, const float *from) __attribute__((always_inline)) {
        const int n = t.n + row, at = t.m + col;
        if (n >= t.n_rows || at >= t.cols) return;
        float x[kEight];
        read_eight(from + col, x);
        if (O *to = out_row<O>(f, n)) store_out<false>(to, at, t.cols, x, alpha, add);
    });
}

}  // namespace deft
