// The gated feed-forward block and its gradient.
//
//   gate = x Wg^T;  up = x Wu^T;  h = act(gate) * up;  y = h Wd^T
//   d = dy Wd;  d_gate = d * up * act'(gate);  d_up = d * act(gate)
//   dWd = dy^T h;  dWg = d_gate^T x;  dWu = d_up^T x;  dx = d_gate Wg + d_up Wu
//
// Both projections are one product (rows of the two matrices alternate in a tile), which leaves h behind, and gate and up
// as the caller keeps them; y is the second.  The backward pass takes four: the derivative by h, whose epilogue reads gate and
// up and leaves d_gate, d_up and h behind; dWd; dWg and dWu together; dx, which sums over both.  Where nothing was kept
// the first product comes again.  9 products of 2 n H I operations (11): bound by the matrix units where rows are many.
//
// h, d_gate and d_up are written once, in panels of 256 columns, and read as they are by both products that need them, by
// one of them through transposing LDS reads; so are the matrices and x.  Where tiles would leave most of the card idle a sum is cut into
// parts, which are joined in one order, also before the activation.
//
// 16-bit floats hold d_gate and d_up times a power of two that brings the largest of dy to 1 .. 2: the gradient of a mean over many
// tokens is far below 1, and so out of their range's reach of 2^-14.
//
// Forward 8192 x 1600 x 6400 bf16 0.42 ms (1200 TFLOP/s in both products; a library's products of those sizes 1000 and 1230), with gradient 1.42 to 1.47 ms
// (1030 to 1060 over all nine; the derivative by h, bound by the 530 MB around its sums, 0.28 of it), 16384 x 4096 x 12288 kept in 8 bits 10.9 to 11.2 ms
// (1320 to 1370; 1550 to 1580), 1024 x 640 x 1728 f32 0.242 to 0.248 ms.
#pragma once
#include "block_few.h"
#include "ends_operands.h"

namespace deft {
namespace {

constexpr unsigned kNoAct = 1u << kMiddle | 1u << kLow, kNoOther = 1u << kLow;   // shapes without a kernel

struct JoinArgs {
    FfnArgs ffn;
    int m, n, splits, add;
    const float *sums;               // [splits][n][sums_ld]
    int64_t sums_ld, sums_split;
    RowPieces by;
};

// The sums of all parts, eight columns from `from` on.
__device__ __forceinline__ void joined(const JoinArgs &a, const float *from, float (&x)[kEight])
{
#pragma unroll
    for (int r = 0; r < kEight; ++r) x[r] = 0.0f;
    int s = 0;
    for (; s + 4 <= a.splits; s += 4) {   // (eight loads under way)
        Eight<float>::type y[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) y[k] = load_eight<true>(from + (s + k) * a.sums_split, 0, kEight);
#pragma unroll
        for (int k = 0; k < 4; ++k)
#pragma unroll
            for (int r = 0; r < kEight; ++r) x[r] += y[k][r];
    }
    for (; s < a.splits; ++s) {
        const Eight<float>::type y = load_eight<true>(from + s * a.sums_split, 0, kEight);
#pragma unroll
        for (int r = 0; r < kEight; ++r) x[r] += y[r];
    }
}

template <typename O>
__global__ void __launch_bounds__(256) join_out_kernel(JoinArgs a)
{
    const float alpha = __is_same(O, f16) && a.ffn.largest ? factor_of(a.ffn.largest, threadIdx.x & 63).y : 1.0f;
    int n, piece;
    if (!a.by.own(blockIdx.x, &n, &piece)) return;
    O *row = out_row<O>(a.ffn, n);
    if (!row) return;
    const int m = piece * kEight;
    float x[kEight];
    joined(a, a.sums + n * a.sums_ld + m, x);
    store_out<false>(row, m, a.m, x, alpha, a.add);
}

// What the products of the projections and of the derivative by h do with their sums, of sums that were cut into parts: m columns
// of n rows, zeros in what the next products read beyond (four neighbouring lanes have a checkpoint's group).
template <bool kGrad, typename T, typename O, bool SPLIT>
__global__ void __launch_bounds__(256) join_act_kernel(JoinArgs a)
{
    const FfnArgs &f = a.ffn;
    const float factor = kGrad && __is_same(T, f16) && f.largest ? factor_of(f.largest, threadIdx.x & 63).x : 1.0f;
    const auto act = [&](const float (&x)[kEight], float (&y)[kEight], float (&slope)[kEight])
        __attribute__((always_inline)) { act_of<SPLIT>(f.activation, x, y, slope); };
    const auto eight = [&](auto inside, int n, int at) __attribute__((always_inline)) {
        constexpr bool kInside = decltype(inside)::value;
        const int own_cols = kInside || n < a.n ? a.m : 0;
        const float *sums = a.sums + n * a.sums_ld;
        const int64_t place = (at >> 8) * f.panel + (at & 255);
        T *const h_at = static_cast<T *>(f.h) + place;
        float x[kEight] = {}, up[kEight] = {};
        if constexpr (kGrad) {
            Ahead<O> ahead = {};
            load_ahead<kInside>(f, n, at, own_cols, ahead);
            if (kInside || at < own_cols) joined(a, sums + at, x);
            use_gate_grad<kInside, T, O, SPLIT>(f, n, at, own_cols, x, ahead, factor, h_at, static_cast<T *>(f.d) + place, act);
        } else {
            if (kInside || at < own_cols) {
                joined(a, sums + (at >> 4) * 32 + (at & 15), x);
                joined(a, sums + (at >> 4) * 32 + 16 + (at & 15), up);
            }
            use_gate<kInside, T, O, SPLIT>(f, n, at, own_cols, x, up, h_at, act);
        }
    };
    int n, piece;
    if (!a.by.own(blockIdx.x, &n, &piece)) return;
    const int at = piece * kEight;
    if (f.arrays == 1 && n < a.n && (at & -kGroup) + kGroup <= a.m) eight(std::true_type{}, n, at);   // (a group's four lanes go the same way)
    else eight(std::false_type{}, n, at);
}

// One call's view of the scratch memory.
struct FfnScratch {
    float *largest, *sums;
    char *x, *grad_y, *w_gate, *w_up, *w_down, *h, *d, *gate, *up;
    FfnScratch(const FfnPlan &plan, void *scratch)
    {
        char *s = static_cast<char *>(scratch);
        largest = reinterpret_cast<float *>(s + plan.largest);
        x = s + plan.x;
        grad_y = s + plan.grad_y;
        w_gate = s + plan.w_gate;
        w_up = s + plan.w_up;
        w_down = s + plan.w_down;
        h = s + plan.h;
        d = s + plan.d;
        gate = s + plan.gate;
        up = s + plan.up;
        sums = reinterpret_cast<float *>(s + plan.sums);
    }
};

struct Operand {
    const void *p;
    int64_t ld, plane;
};

template <typename S, typename T, int P>
struct Ffn {
    static constexpr bool kSplit = P == 3, kHalf16 = __is_same(T, f16);
    static constexpr double kAlone = kSplit ? 1.6 : 1.0;   // (128 x 128 tiles 0.72 us a step for 0.46, 128 x 64 ones 0.45 for 0.28)

    template <int E>
    static hipError_t product(const ProductArgs &p, Shape shape, hipStream_t st)
    {
        switch (shape) {
        case kMiddle:
            if constexpr (E != kGate && E != kGateGrad) return product_shape<T, S, E, 2, 4, 6, 4, kSplit>(p, st);
            return hipErrorInvalidValue;
        case kHalf: return product_shape<T, S, E, 4, 2, 4, 4, kSplit>(p, st);
        case kSmall: return product_shape<T, S, E, 2, 2, 4, 4, kSplit>(p, st);
        case kNarrow: return product_shape<T, S, E, 4, 2, 4, 2, kSplit>(p, st);
        case kTiny: return product_shape<T, S, E, 2, 2, 4, 2, kSplit>(p, st);
        case kLarge: return product_shape<T, S, E, 2, 4, 8, 4, kSplit>(p, st);
        default: return hipErrorInvalidValue;
        }
    }

    template <int E>
    static hipError_t allow()
    {
        hipError_t e = allow_shape<T, S, E, 2, 4, 8, 4, kSplit>();
        if constexpr (E != kGate && E != kGateGrad)
            if (e == hipSuccess) e = allow_shape<T, S, E, 2, 4, 6, 4, kSplit>();
        if (e == hipSuccess) e = allow_shape<T, S, E, 4, 2, 4, 4, kSplit>();
        if (e == hipSuccess) e = allow_shape<T, S, E, 2, 2, 4, 4, kSplit>();
        if (e == hipSuccess) e = allow_shape<T, S, E, 4, 2, 4, 2, kSplit>();
        if (e == hipSuccess) e = allow_shape<T, S, E, 2, 2, 4, 2, kSplit>();
        return e;
    }

    static hipError_t prepare()
    {
        hipError_t e = allow<kGate>();
        if (e == hipSuccess) e = allow<kGateGrad>();
        if (e == hipSuccess) e = allow<kOut>();
        if (e == hipSuccess) e = allow<kInput>();
        if (e == hipSuccess) e = allow<kOuter>();
        return e;
    }

    // Rows as the products read them: where they are, or packed, by one launch for all that a call needs so.  `along`: a product
    // has their elements as its k, beside those that have them as m or n (whole pieces of 16 bytes are enough for these).
    struct Packing {
        PackMany many{};
        int count = 0;
        unsigned blocks = 0;

        static bool as_is(const void *p, int64_t stride, int cols, bool along) { return !kSplit && in_place(p, stride, cols, along ? kStep : 8); }

        Operand operand(const void *p, int64_t stride, int rows, int cols, bool along, void *packed)
        {
            if (as_is(p, stride, cols, along)) return {p, stride, 0};
            PackArgs &a = many.of[count];
            a.src = p;
            a.src_stride = stride;
            a.rows = rows;
            a.cols = cols;
            a.out = packed;
            a.out_ld = up(cols, kStep);
            a.out_plane = up(rows, kTile) * a.out_ld;
            blocks += many.blocks[count++] = pack_blocks(up(rows, kTile), a.out_ld);
            return {packed, a.out_ld, a.out_plane};
        }

        hipError_t launch(hipStream_t st) const
        {
            if (blocks == 0) return hipSuccess;
            pack_many_kernel<S, T, P><<<blocks, 256, 0, st>>>(many);
            return hipGetLastError();
        }
    };

    static hipError_t restored(const deft_checkpoint_t &from, int rows, int cols, int dtype, void *packed, Operand *out, hipStream_t st)
    {
        RestoreArgs a{};
        a.rows = rows;
        a.cols = cols;
        a.rows_to = (int)up(rows, kTile);
        a.cols_to = (int)up(cols, kStep);
        a.from = from;
        a.out = packed;
        a.out_ld = a.cols_to;
        a.out_plane = (int64_t)a.rows_to * a.cols_to;
        *out = {packed, a.out_ld, a.out_plane};
        return restore_operand_launch(dtype, a, st);
    }

    static FfnArgs panels(const FfnScratch &s, int n, int inner, int activation)
    {
        FfnArgs f{};
        f.activation = activation;
        f.cols_up = (int)up(inner, 256);
        // Up to 64 rows the products are bound by reading and writing the matrices: what is rounded in between keeps what that took, in
        // 64 more rows of each panel.
        f.arrays = !kSplit && n <= kFew ? 2 : 1;
        f.panel = up(n, n <= kFew ? kFew * f.arrays : kTile) * 256;
        f.h_plane = f.arrays == 2 ? kFew * 256 : f.cols_up / 256 * f.panel;
        f.d_plane = f.arrays == 2 ? kFew * 256 : 2 * f.h_plane;
        f.h = s.h;
        f.half = f.rows = INT32_MAX;
        f.a_panel = 256;
        return f;
    }

    // Parts of a sum, as splits_of has them, with the time that it takes to write and join them: a launch and 8 bytes an element
    // at 5 TB/s, in the time of a large tile's step.  (`steps` counts a 32-bit step's six products one by one, which the kernel does not
    // part: there may be more parts than steps, as 4 of 3.  Those without a step have sums of zero.)
    static int parts_of(int64_t m, int64_t n, int64_t steps, int64_t units, unsigned without)
    {
        const int64_t tiles = up(m, kTile) / kTile * (n <= kFew ? 1 : up(n, kTile) / kTile);
        int best = 1;
        double least = 1e300;
        for (int s = 1; s <= kMaxSplits && (s == 1 || (tiles * s <= 2 * units && steps >= s * 4)); s *= 2) {
            const double t = least_cost(m, n, steps, s, units, without, kAlone) + (s > 1 ? 2.0 + 1e-6 * (double)(m * n) * s : 0.0);
            if (t < least) {
                least = t;
                best = s;
            }
        }
        return best;
    }

    // A product of `rows` by `cols` sums, cut into parts where that is quicker.
    template <int E>
    static hipError_t parts(ProductArgs &p, int cols, const FfnScratch &s, int compute_units, hipStream_t st)
    {
        constexpr unsigned kWithout = E == kGate || E == kGateGrad ? kNoAct : kNoOther;
        const int64_t steps = (int64_t)(p.k / kStep) * (kSplit ? 6 : 1) * (E == kInput ? 2 : 1) * (E == kOut || E == kInput ? p.ffn.arrays : 1);
        p.splits = parts_of(cols, p.n, steps, compute_units, kWithout);
        p.sums = s.sums;
        p.sums_ld = up(cols, kEight);
        p.sums_split = p.n * p.sums_ld;
        return product<E>(p, shape_of(cols, p.n, steps, p.splits, compute_units, kWithout, kAlone), st);
    }

    static JoinArgs join(const ProductArgs &p, const RowPieces &by)
    {
        JoinArgs j{};
        j.by = by;
        j.ffn = p.ffn;
        j.m = p.m;
        j.n = p.n;
        j.splits = p.splits;
        j.add = p.add;
        j.sums = p.sums;
        j.sums_ld = p.sums_ld;
        j.sums_split = p.sums_split;
        return j;
    }

    // One whose sums go through the activation: both projections, or the derivative by h.
    template <int E>
    static hipError_t activated(ProductArgs &p, const FfnScratch &s, int compute_units, hipStream_t st)
    {
        const hipError_t e = parts<E>(p, E == kGate ? (int)up(p.m, 16) * 2 : p.m, s, compute_units, st);
        if (e != hipSuccess || p.splits == 1) return e;
        const JoinArgs j = join(p, RowPieces(up(p.n, kStep), up(p.m, kStep)));
        join_act_kernel<E == kGateGrad, T, S, kSplit><<<j.by.blocks(), 256, 0, st>>>(j);
        return hipGetLastError();
    }

    static hipError_t gate(const FfnArgs &f, const Operand &x, const Operand &w_gate, const Operand &w_up, int n, int hidden, int inner, const FfnScratch &s,
                           int compute_units, hipStream_t st)
    {
        ProductArgs p{};
        p.a = w_gate.p;
        p.a_ld = w_gate.ld;
        p.a_plane = w_gate.plane;
        p.b = x.p;
        p.b_ld = x.ld;
        p.b_plane = x.plane;
        p.m = inner;
        p.n = n;
        p.k = (int)up(hidden, kStep);
        p.ffn = f;
        p.ffn.a2 = w_up.p;
        p.ffn.a2_ld = w_up.ld;
        p.ffn.a2_plane = w_up.plane;
        return activated<kGate>(p, s, compute_units, st);
    }

    // One whose sums are the result.
    template <int E>
    static hipError_t summed(ProductArgs &p, const FfnScratch &s, int compute_units, hipStream_t st)
    {
        const hipError_t e = parts<E>(p, p.m, s, compute_units, st);
        if (e != hipSuccess || p.splits == 1) return e;
        const JoinArgs j = join(p, RowPieces(p.n, p.m));
        join_out_kernel<S><<<j.by.blocks(), 256, 0, st>>>(j);
        return hipGetLastError();
    }

    static hipError_t few(const deft_ffn_t &a, const FfnScratch &s, int h_arrays, int compute_units, hipStream_t st)
    {
        FewArgs f{};
        f.n = a.n_rows;
        f.hidden = a.hidden;
        f.inner = a.inner;
        f.activation = a.activation;
        f.x = a.x;
        f.x_stride = a.x_stride;
        f.w_gate = a.w_gate;
        f.w_gate_stride = a.w_gate_stride;
        f.w_up = a.w_up;
        f.w_up_stride = a.w_up_stride;
        f.w_down = a.w_down;
        f.w_down_stride = a.w_down_stride;
        f.h = s.h;
        f.h_stride = up(a.inner, 8);
        f.h_array = kFew * f.h_stride;   // (within the room for a tile's rows)
        f.h_arrays = h_arrays;
        f.saved = a.save;
        f.y = a.y;
        f.y_stride = a.y_stride;
        if (f.n <= 16) return few_tokens<S, 1>(f, compute_units, st);
        if (f.n <= 32) return few_tokens<S, 2>(f, compute_units, st);
        return few_tokens<S, 4>(f, compute_units, st);
    }

    static hipError_t forward(const deft_ffn_t &a, const FfnScratch &s, int compute_units, hipStream_t st)
    {
        // A few tokens go to kernels that read the matrices once as they lie.  32-bit types: up to 64 (64 of 1024 x 4096 62 us for 74 by
        // the products below, 32 of 4096 x 12288 189 for 532).  16-bit types: up to 16 (of 4096 x 12288 67 us for 80, of 1600 x 6400 24 for
        // 29), and where operands would have to be packed, as many as that is worth, by the matrices' size (64 of 515 x 1030 18 for 24; 32
        // of 1021 x 2731 24 for 29, 64 of it 35 for 32; 32 of 2047 x 8191 97 for 79).  Beyond 8 these kernels round what is between the
        // products once more, which the products below do not: so where nothing is packed 17 to 32 take them with what that takes beside it,
        // as a second array, which pays for small matrices only (32 of 768 x 2048 17 us for 20.6, without the array 13.5; 24 of 1024 x
        // 4096 24.0 for 23.4), and more do not, though 48 of 768 x 2048 would be quicker without (18 for 21).
        const bool whole = Packing::as_is(a.x, a.x_stride, a.hidden, true) && Packing::as_is(a.w_gate, a.w_gate_stride, a.hidden, true) &&
                           Packing::as_is(a.w_up, a.w_up_stride, a.hidden, true) && Packing::as_is(a.w_down, a.w_down_stride, a.inner, true);
        const bool two = !kSplit && (a.n_rows <= 8 || (a.n_rows > 16 && whole));
        if (a.n_rows <= few_rows(kSplit, (int64_t)a.hidden * a.inner, whole)) return few(a, s, two ? 2 : 1, compute_units, st);
        Packing pack;
        const Operand x = pack.operand(a.x, a.x_stride, a.n_rows, a.hidden, true, s.x);
        const Operand w_gate = pack.operand(a.w_gate, a.w_gate_stride, a.inner, a.hidden, true, s.w_gate);
        const Operand w_up = pack.operand(a.w_up, a.w_up_stride, a.inner, a.hidden, true, s.w_up);
        const Operand w_down = pack.operand(a.w_down, a.w_down_stride, a.hidden, a.inner, true, s.w_down);
        hipError_t e = pack.launch(st);
        if (e != hipSuccess) return e;
        FfnArgs f = panels(s, a.n_rows, a.inner, a.activation);
        f.saved = a.save;
        e = gate(f, x, w_gate, w_up, a.n_rows, a.hidden, a.inner, s, compute_units, st);
        if (e != hipSuccess) return e;
        ProductArgs p{};
        p.a = w_down.p;
        p.a_ld = w_down.ld;
        p.a_plane = w_down.plane;
        p.b = s.h;
        p.b_ld = 256;
        p.b_plane = f.h_plane;
        p.d_panel = f.panel;
        p.m = a.hidden;
        p.n = a.n_rows;
        p.k = (int)up(a.inner, kStep);
        p.ffn = f;
        p.ffn.b_array = f.h_plane;
        p.ffn.out[0] = a.y;
        p.ffn.out_ld[0] = a.y_stride;
        return summed<kOut>(p, s, compute_units, st);
    }

    static hipError_t backward(const deft_ffn_grad_t &a, const FfnScratch &s, int compute_units, hipStream_t st)
    {
        const int n = a.n_rows;
        const bool of_gate = a.grad_gate || a.grad_up, by_projections = of_gate || a.grad_x;
        Operand x{}, grad_y{}, w_gate{}, w_up{}, w_down{};
        FfnArgs f = panels(s, n, a.inner, a.activation);
        hipError_t e = hipSuccess;
        if (n > 0) {
            const bool again = a.saved.kind == DEFT_SAVE_NONE;
            Packing pack;
            grad_y = pack.operand(a.grad_y, a.grad_y_stride, n, a.hidden, true, s.grad_y);
            if ((again || of_gate) && a.x) x = pack.operand(a.x, a.x_stride, n, a.hidden, again, s.x);
            if (again || a.grad_x) {
                w_gate = pack.operand(a.w_gate, a.w_gate_stride, a.inner, a.hidden, again, s.w_gate);
                w_up = pack.operand(a.w_up, a.w_up_stride, a.inner, a.hidden, again, s.w_up);
            }
            if (by_projections) w_down = pack.operand(a.w_down, a.w_down_stride, a.hidden, a.inner, false, s.w_down);
            e = pack.launch(st);
            if (e == hipSuccess && (again || of_gate) && !a.x)
                e = restored(a.packed_x, n, a.hidden, kSplit ? DEFT_F32 : kHalf16 ? DEFT_F16 : DEFT_BF16, s.x, &x, st);
            if (e != hipSuccess) return e;
            if (again) {
                const int64_t ld = up(a.inner, kStep);
                f.saved.kind = DEFT_SAVE_FULL;
                f.saved.gate = {s.gate, ld, s.gate + up(n, kTile) * ld * (int64_t)sizeof(S), ld / kGroup};
                f.saved.up = {s.up, ld, s.up + up(n, kTile) * ld * (int64_t)sizeof(S), ld / kGroup};
                FfnArgs g = f;
                g.h = nullptr;
                e = gate(g, x, w_gate, w_up, n, a.hidden, a.inner, s, compute_units, st);
            } else {
                f.saved = a.saved;
            }
            if constexpr (kHalf16) {
                if (e == hipSuccess && by_projections) {
                    e = ffn_largest_launch({n, a.hidden, static_cast<const f16 *>(a.grad_y), a.grad_y_stride, s.largest, RowPieces(n, a.hidden)}, st);
                    f.largest = s.largest;
                }
            }
            if (e == hipSuccess) {   // (without the derivatives by the projections: h alone)
                ProductArgs p{};
                p.a = w_down.p;
                p.a_ld = w_down.ld;
                p.a_plane = w_down.plane;
                p.a_rows = a.hidden;
                p.b = grad_y.p;
                p.b_ld = grad_y.ld;
                p.b_plane = grad_y.plane;
                p.m = a.inner;
                p.n = n;
                p.k = by_projections ? (int)up(a.hidden, kStep) : 0;
                p.ffn = f;
                p.ffn.h = a.grad_down ? s.h : nullptr;
                p.ffn.d = by_projections ? s.d : nullptr;
                e = activated<kGateGrad>(p, s, compute_units, st);
            }
        }
        const bool weights = n > 0 || !a.accumulate;
        ProductArgs q{};   // of the matrices' gradients
        q.k = (int)up(n, kStep) * f.arrays;
        q.add = a.accumulate;
        q.ffn = f;
        if (e == hipSuccess && a.grad_down && weights) {
            ProductArgs p = q;
            p.a = s.h;
            p.a_ld = 256;
            p.a_plane = f.h_plane;
            p.a_rows = p.k;
            p.ffn.a_panel = f.panel;
            p.ffn.a_step = kStep * 256;
            p.ffn.b_step = f.arrays == 2 ? 0 : kStep * grad_y.ld;
            p.b = grad_y.p;
            p.b_ld = grad_y.ld;
            p.b_plane = grad_y.plane;
            p.b_rows = n;
            p.d_panel = 256;
            p.m = a.inner;
            p.n = a.hidden;
            p.ffn.out[0] = a.grad_down;
            p.ffn.out_ld[0] = a.grad_down_stride;
            p.ffn.largest = nullptr;
            e = summed<kOuter>(p, s, compute_units, st);
        }
        if (e == hipSuccess && a.events) e = hipEventRecord(static_cast<hipEvent_t>(a.events[0]), st);
        if (e == hipSuccess && of_gate && weights) {
            ProductArgs p = q;
            p.a = x.p;
            p.a_ld = x.ld;
            p.a_plane = x.plane;
            p.a_rows = n;
            p.b = s.d;
            p.b_ld = 256;
            p.b_plane = f.d_plane;
            p.b_rows = p.k;
            p.d_panel = f.panel;
            p.ffn.a_step = f.arrays == 2 ? 0 : kStep * x.ld;
            p.ffn.b_step = kStep * 256;
            p.m = a.hidden;
            p.n = 2 * f.cols_up;
            p.ffn.out[0] = a.grad_gate;
            p.ffn.out_ld[0] = a.grad_gate_stride;
            p.ffn.out[1] = a.grad_up;
            p.ffn.out_ld[1] = a.grad_up_stride;
            p.ffn.half = f.cols_up;
            p.ffn.rows = a.inner;
            e = summed<kOuter>(p, s, compute_units, st);
        }
        if (e == hipSuccess && a.events) e = hipEventRecord(static_cast<hipEvent_t>(a.events[1]), st);
        if (e == hipSuccess && a.grad_x && n > 0) {
            ProductArgs p{};
            p.a = w_gate.p;
            p.a_ld = w_gate.ld;
            p.a_plane = w_gate.plane;
            p.a_rows = a.inner;
            p.b = s.d;
            p.b_ld = 256;
            p.b_plane = f.d_plane;
            p.d_panel = f.panel;
            p.m = a.hidden;
            p.n = n;
            p.k = (int)up(a.inner, kStep);
            p.ffn = f;
            p.ffn.a2 = w_up.p;
            p.ffn.a2_ld = w_up.ld;
            p.ffn.a2_plane = w_up.plane;
            p.ffn.d_half = f.cols_up / 256 * f.panel;
            p.ffn.b_array = f.d_plane;
            p.ffn.out[0] = a.grad_x;
            p.ffn.out_ld[0] = a.grad_x_stride;
            e = summed<kInput>(p, s, compute_units, st);
        }
        return e;
    }
};

}  // namespace
}  // namespace deft
