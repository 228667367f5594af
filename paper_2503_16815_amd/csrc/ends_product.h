// The matrix product that the head's operators are made of:  C[m][n] = sum_k A[m][k] B[n][k], 16-bit
// elements, 32-bit sums.  Both operands have their k elements next to each other, or B its n
// elements (kGradient, which so reads the derivative as it was written) or A its m elements (kSums, which so reads
// the weights as they are).  What happens to C is the epilogue's business (it is never stored as it is): softmax statistics, the loss's derivative,
// or a sum into a gradient.
//
// A workgroup of eight wavefronts owns a tile of C.  Both operands' tiles go from memory to LDS without
// passing registers, 64 elements of k at a time.  LDS holds three of A's and two of B's (160 KB at 256 x 256):
// A's tile of the step after next is asked for in a step's first half, B's in its second, each spread
// over the half's matrix instructions, so that neither waits for the other (measured at 8192^3 in bf16: all of it at
// the step's beginning 1130 TFLOP/s, spread 1230; addresses in 64-bit registers instead of a buffer's 1180).  The fragments
// of a half are read from LDS during the half before.  The matrix instructions are written out, so that
// sums stay in accumulation registers and everything else comes between them in this order, and so are the loads to
// LDS, which have no register to wait for: the compiler would let every transposing LDS read wait for all of them.
//
// The 16-byte pieces of a row are permuted by the row's number, so that the sixteen rows that a wavefront
// reads together lie in different banks (no bank conflicts counted).  An A or B with its m or n elements
// next to each other lies in LDS as it came, a row of TM or TN elements to each k; the transposing LDS read gives every
// lane four k of its column, from four rows whose 32-byte pieces are permuted by the row's number too.
//
// The derivative lies in panels of 256 columns, so that a step of either product that reads it finds it in one
// stretch of memory.
//
// Tiles are dealt out so that the workgroups of an XCD work on neighbouring ones, four wide: 12 rows of tiles
// come into its L2 for 32 workgroups instead of 33 (131072 x 8192 x 4096: 890 to 1110 TFLOP/s by itself).  Where k is
// split, an XCD has all tiles of a part before the next part's: what they read is theirs alone (hidden states' gradient of
// 1024 positions, 8209 rows of 640 in 32 bits, 16 parts: 65 us; with each part's tiles on all XCDs 87, 272 MB fetched).
//
// Bound by the matrix units at the clock that the card keeps under them.  8192 positions, 50257 rows of 1600 elements, bf16, all
// pieces: logits with softmax sums 1165 us (1130 TFLOP/s), derivative 1290 (1020: 824 MB are written), weights' gradient and
// hidden states' gradient 1200 each (1100).
//
// 32-bit operands come as three 16-bit arrays whose sum they are (8 bits of the significand in
// each); the six products of those arrays that matter at 24 bits are summed one after the other, step by step (loss
// and gradients of 2 x 91134 x 305 334 us, 40 x 30000 x 512 176; all steps of one product before the next 357 and 191).
//
// The feed-forward block's products are the same kernel with epilogues of their own (block_epilogue.h).  kGate has two
// operands A, whose rows alternate sixteen at a time, so that a lane holds both projections of an element; kInput adds two
// products, one's steps behind the other's; kOuter has the elements of both operands' m and n next to each other.
#pragma once
#include "block_epilogue.h"
#include "ends_shapes.h"

namespace deft {

constexpr int kStepBytes = kStep * 2;

// kGate: both projections and the hidden activations; kGateGrad: the derivatives by both projections; kOut: y; kInput: x's
// gradient; kOuter: a matrix's gradient
enum Epilogue { kSoftmax = 0, kDerivative = 1, kSums = 2, kGradient = 3, kGate = 4, kGateGrad = 5, kOut = 6, kInput = 7, kOuter = 8 };

struct ProductArgs {
    const void *a, *b;               // kSums, kGradient: b is the derivative, as below
    int64_t a_ld, b_ld;              // elements between rows
    int64_t a_plane, b_plane;        // elements between the three arrays of a 32-bit operand
    int m, n;                        // rows of a and of b
    const int *n_dev;                // rows of b that count, where the device knows it, or NULL
    int k;                           // a multiple of kStep
    int a_rows, b_rows;              // the k that a has rows of where its m elements are next to each other; kOuter: that b has
    const int *k_dev;                // or the rows of another operand, rounded up to kStep
    int splits;                      // of k
    float scale;
    // kSoftmax, kDerivative: m counts rows of the vocabulary from m_first on, n packed positions
    int m_first;
    const int *label;                // [n]
    float2 *parts;                   // [n][parts_ld]: each tile's softmax sum of the position
    int parts_ld, parts_first;       // the number of the first tile's part
    float *z_label;                  // [n]
    const float *lse;                // [n]
    const float *row_grad, *row_factor;   // [n] and [1]: their product is scaled into d's range
    float *residual;                 // [n]: what rounding took from the label's derivative; or NULL
    void *d;                         // panels of 256 columns: [d_cols / 256][rows][256]
    int64_t d_panel, d_plane;        // elements between panels, between arrays
    int d_arrays;                    // 16-bit types: 1, or 2 where a second array holds what rounding took (kGradient reads both)
    int d_cols;
    // kSums: sums[split][n][m]; kGradient: out[n][m]
    float *sums;
    int64_t sums_ld, sums_split;
    int add;
    const float *out_scale;          // beside `scale`
    void *out;
    int64_t out_ld;
    FfnArgs ffn;                     // the feed-forward block's
};

template <typename T> struct Mfma;
template <> struct Mfma<f16> {
    typedef f16 operand __attribute__((ext_vector_type(8)));
    static __device__ __forceinline__ void run(operand a, operand b, f32x4 &c)
    {
        asm volatile("v_mfma_f32_16x16x32_f16 %0, %1, %2, %0" : "+a"(c) : "v"(a), "v"(b));
    }
};
template <> struct Mfma<bf16> {
    typedef bf16 operand __attribute__((ext_vector_type(8)));
    static __device__ __forceinline__ void run(operand a, operand b, f32x4 &c)
    {
        asm volatile("v_mfma_f32_16x16x32_bf16 %0, %1, %2, %0" : "+a"(c) : "v"(a), "v"(b));
    }
};

constexpr int kStagesA = 3, kStagesB = 2;
// The rows that a tile's loads bring: every thread loads 16 bytes, an eighth of a row, at a time.
constexpr int product_rows(int rows, int threads) { return (rows * 8 + threads - 1) / threads * threads / 8; }
constexpr int product_lds(int tm, int tn, int threads)
{
    return (kStagesA * product_rows(tm, threads) + kStagesB * product_rows(tn, threads)) * kStepBytes;
}

// All of this wavefront's LDS reads are done, and all but `N` of its loads; then the others' are too.
template <int N>
__device__ __forceinline__ void step_barrier()
{
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(N) : "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
}

// 16 bytes a lane from `from` + offset + at to LDS, a wavefront's lanes one after the other from to_lds on.
__device__ __forceinline__ void load_to_lds(i32x4 from, unsigned offset, int at, unsigned to_lds)
{
    asm volatile("s_mov_b32 m0, %3\n"
                 "s_nop 0\n"
                 "buffer_load_dwordx4 %1, %0, %2 offen lds"
                 :
                 : "s"(from), "v"(offset), "s"(at), "s"(to_lds)
                 : "memory", "m0");
}

// What the 32-byte pieces of row k are permuted by (an exclusive or with their number) in a tile of `wide` elements
// to a row: rows 0 .. 3 and 8 .. 11 of any sixteen, which a transposing read visits at a time, so fill all 64 banks.
constexpr __host__ __device__ int turn_of(int wide, int k)
{
    const int low = k & 3, high = (k >> 3) & 3;
    return wide == 160 ? high & 1 : wide == 192 ? low ^ (high & 1) : (low + high * 4) & ((wide / 16 < 16 ? wide / 16 : 16) - 1);
}

template <int H> struct HalfOf {
    static constexpr int value = H;
};

// T: element type of the operands.  O: type of the gradient that kGradient writes.  WM x WN wavefronts of MT x NT
// tiles of 16 x 16.  SPLIT: operands are three arrays each.
template <typename T, typename O, int E, int WM, int WN, int MT, int NT, bool SPLIT>
__global__ void __launch_bounds__(WM *WN *kWave, 2) product_kernel(ProductArgs p)
{
#ifdef __HIP_DEVICE_COMPILE__   // (the host has no such registers)
    constexpr int kThreads = WM * WN * kWave, TM = WM * MT * 16, TN = WN * NT * 16;
    constexpr int kARows = product_rows(TM, kThreads), kBRows = product_rows(TN, kThreads);   // that whole loads bring
    constexpr int kABytes = kARows * kStepBytes, kBBytes = kBRows * kStepBytes, kBAt = kStagesA * kABytes;
    constexpr int kALoads = kARows * 8 / kThreads, kBLoads = kBRows * 8 / kThreads;
    constexpr int kFetches = MT + NT, kProducts = MT * NT;
    constexpr bool kTurned = E == kGradient || E == kOuter;   // B's n elements are next to each other
    constexpr bool kTurnedA = E == kSums || E == kGateGrad || E == kInput || E == kOuter;   // A's m elements are
    constexpr bool kPanels = E == kSums || E == kGradient || E == kOut || E == kInput;
    constexpr bool kAimed = kPanels || kTurned || kTurnedA;   // a step's place is not the last one's and 64 elements more
    constexpr bool kTwo = !SPLIT && (E == kOut || E == kInput) && WM == 4 && TN == 64;   // b may have a second array (up to 64 rows)
    constexpr int kPanelSteps = 256 / kStep;
    constexpr int kColumns = E == kGate ? TM / 2 : TM;   // of C that a tile has
    constexpr int kPieces = TN / 8, kPiecesA = TM / 8;   // 16-byte pieces of a row of TN, of TM
    static_assert(!kTurned || kBRows == TN, "whole rows of k");
    typedef typename Mfma<T>::operand Operand;
    static_assert(E < kGate || WM * WN * epilogue_floats(MT) * 4 <= product_lds(TM, TN, kThreads));
    extern __shared__ __align__(16) char lds[];

    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), wm = wave / WN, wn = wave % WN;
    const int n_rows = p.n_dev ? *p.n_dev : p.n;
    const int tiles_m = (p.m + kColumns - 1) / kColumns, tiles_n = (n_rows + TN - 1) / TN;
    // workgroup b runs on XCD b % 8; each XCD has an equal share of the parts' tiles, in groups four wide
    const int tiles = tiles_m * tiles_n, items = tiles * p.splits, xcd = blockIdx.x & 7, share = items >> 3, more = items & 7;
    if ((int)(blockIdx.x >> 3) >= share + (xcd < more ? 1 : 0)) return;
    const int item = (int)(blockIdx.x >> 3) + xcd * share + (xcd < more ? xcd : more);
    const int split = item / tiles, tile = item - split * tiles;
    const int group = tile / (tiles_m * 4), in_group = tile - group * tiles_m * 4;
    const int wide = min(tiles_n - group * 4, 4);
    const int tm = in_group / wide, tn = group * 4 + in_group - tm * wide;
    const int m0 = tm * kColumns, n0 = tn * TN;

    const int steps_one = (p.k_dev ? *p.k_dev + kStep - 1 : p.k) / kStep, steps_all = E == kInput ? 2 * steps_one : steps_one;
    const int from = (int)((int64_t)steps_all * split / p.splits), to = (int)((int64_t)steps_all * (split + 1) / p.splits);
    const int steps = to - from, total = SPLIT ? steps * 6 : E == kGradient ? steps * p.d_arrays : kTwo ? steps * p.ffn.arrays : steps;

    // where this thread's 16-byte pieces come from (rows past the operand's last one read that one)
    const bool second = E == kGate && ((wave >> 1) & 1);   // this wavefront loads rows of the other projection
    const int64_t a_ld = second ? p.ffn.a2_ld : p.a_ld, a_plane = second ? p.ffn.a2_plane : p.a_plane;
    const char *a_base = static_cast<const char *>(second ? p.ffn.a2 : p.a);
    if (E == kOuter) a_base += ((m0 >> 8) * p.ffn.a_panel + (m0 & 255)) * 2;
    else a_base += (kTurnedA ? (int64_t)m0 : (int64_t)m0 * a_ld + (int64_t)from * kStep) * 2;
    const char *b_base = static_cast<const char *>(p.b);
    if (kTurned) b_base += ((n0 >> 8) * p.d_panel + (n0 & 255)) * 2;
    else if (kPanels) b_base += (int64_t)n0 * p.b_ld * 2;
    else b_base += ((int64_t)n0 * p.b_ld + (int64_t)from * kStep) * 2;
    unsigned a_off[kALoads], b_off[kBLoads];
    int at_step = 0, at_product = 0;   // the next tiles to load
    const auto turned_a = [&](int rows) {   // of a step that a has `rows` rows for; and columns past its last piece read that one
#pragma unroll
        for (int i = 0; i < kALoads; ++i) {
            const int c = tid + i * kThreads, row = c / kPiecesA, piece = c % kPiecesA;
            const int at = (piece >> 1 ^ turn_of(TM, row)) * 2 + (piece & 1);
            if constexpr (E == kOuter) {   // (a tile of 192 or 160 columns may lie in two panels)
                const int col = (m0 & 255) + min(at, ((p.m + 7) >> 3) - 1 - (m0 >> 3)) * 8;
                a_off[i] = (unsigned)min(row, rows - 1) * (unsigned)(p.a_ld * 2) +
                           ((unsigned)(col >> 8) * (unsigned)p.ffn.a_panel + (col & 255) - (m0 & 255)) * 2;
            } else {
                const int64_t ld = E == kInput && from + at_step >= steps_one ? p.ffn.a2_ld : p.a_ld;
                a_off[i] = (unsigned)min(row, rows - 1) * (unsigned)(ld * 2) + (min(at, ((p.m + 7) >> 3) - 1 - (m0 >> 3)) << 4);
            }
        }
    };
    const auto turned_b = [&](int rows) {   // the same of a b whose rows end where they end (kOuter)
#pragma unroll
        for (int i = 0; i < kBLoads; ++i) {
            const int c = tid + i * kThreads, row = c / kPieces, piece = c % kPieces;
            const int at = (piece >> 1 ^ turn_of(TN, row)) * 2 + (piece & 1);
            b_off[i] = (unsigned)min(row, rows - 1) * (unsigned)(p.b_ld * 2) + (min(at, ((p.n + 7) >> 3) - 1 - (n0 >> 3)) << 4);
        }
    };
#pragma unroll
    for (int i = 0; i < kALoads; ++i) {
        const int c = tid + i * kThreads, row = c >> 3;
        const int in_a = E == kGate ? (row >> 5) * 16 + (row & 15) : row;
        if (!kTurnedA) a_off[i] = (unsigned)min(in_a, p.m - 1 - m0) * (unsigned)(a_ld * 2) + (((c & 7) ^ ((row >> 1) & 7)) << 4);
    }
#pragma unroll
    for (int i = 0; i < kBLoads; ++i) {
        const int c = tid + i * kThreads;
        if constexpr (E == kOuter) {
            b_off[i] = 0;
        } else if constexpr (kTurned) {   // (a panel has whole tiles of 64 rows)
            const int row = c / kPieces, piece = c % kPieces, turn = turn_of(TN, row);
            b_off[i] = (unsigned)row * (unsigned)(p.b_ld * 2) + (((piece >> 1 ^ turn) * 2 + (piece & 1)) << 4);
        } else {
            const int row = c >> 3;
            b_off[i] = (unsigned)min(row, p.n - 1 - n0) * (unsigned)(p.b_ld * 2) + (((c & 7) ^ ((row >> 1) & 7)) << 4);
        }
    }
    // Where operands are three arrays: the six products of them that are kept, the smallest first.
    i32x4 a_from, b_from;   // buffer descriptors
    const auto descriptor = [](const char *base) {
        const uint64_t at = (uint64_t)base;
        return i32x4{__builtin_amdgcn_readfirstlane((int)(uint32_t)at),
                     __builtin_amdgcn_readfirstlane((int)(uint32_t)(at >> 32) & 0xffff), -1, 0x00020000};
    };
    const int64_t a_to_a2 = E == kInput ? (int64_t)((uintptr_t)p.ffn.a2 - (uintptr_t)p.a) : 0;
    const auto aim = [&]() {
        int64_t a_at = 0, b_at = 0;
        if (E == kOuter) b_at = (from + at_step) * p.ffn.b_step * 2;
        else if (kTurned) b_at = (int64_t)(from + at_step) * kStep * 512;
        else if (kPanels) b_at = ((from + at_step) / kPanelSteps * p.d_panel + (from + at_step) % kPanelSteps * kStep) * 2;
        if constexpr (E == kInput) {   // (steps of the second product: its own weights, and the other half of b)
            const int step = from + at_step, step_of = step >= steps_one ? step - steps_one : step, k = step_of * kStep;
            b_at = (step_of / kPanelSteps * p.d_panel + step_of % kPanelSteps * kStep) * 2;
            if (step >= steps_one) {
                a_at = (int64_t)k * p.ffn.a2_ld * 2 + a_to_a2;
                b_at += p.ffn.d_half * 2;
            } else {
                a_at = (int64_t)k * p.a_ld * 2;
            }
            if ((at_step == 0 || step_of == 0 || k + kStep > p.a_rows) && at_product == 0) turned_a(min(p.a_rows - k, kStep));
        } else if (kTurnedA) {
            const int k = E == kOuter && p.ffn.a_step == 0 ? 0 : (from + at_step) * kStep;
            a_at = E == kOuter ? (from + at_step) * p.ffn.a_step * 2 : (int64_t)k * p.a_ld * 2;
            if (E == kOuter) {
                const int k_b = p.ffn.b_step == 0 ? 0 : (from + at_step) * kStep;
                if ((at_step == 0 && at_product == 0) || k_b + kStep > p.b_rows) turned_b(min(p.b_rows - k_b, kStep));
            }
            if ((at_step == 0 && at_product == 0) || k + kStep > p.a_rows) turned_a(min(p.a_rows - k, kStep));
        }
        if (SPLIT) {
            a_at += ((0x021010 >> (4 * (5 - at_product))) & 15) *
                    (E == kInput && from + at_step >= steps_one ? p.ffn.a2_plane : a_plane) * 2;
            b_at += ((0x201100 >> (4 * (5 - at_product))) & 15) * p.b_plane * 2;
        } else if (E == kGradient) {
            b_at += at_product * p.d_plane * 2;
        } else if (kTwo) {
            b_at += at_product * p.ffn.b_array * 2;
        }
        a_from = descriptor(a_base + a_at);
        b_from = descriptor(b_base + b_at);
    };
    const auto next_step = [&]() {
        if (SPLIT) {   // (a step's products one after the other: its tiles are in the XCD's L2 then)
            if (++at_product == 6) {
                at_product = 0;
                ++at_step;
            }
            aim();
            return;
        }
        if (kTwo && ++at_product < p.ffn.arrays) return aim();   // (a step's second array)
        if (kTwo) at_product = 0;
        ++at_step;
        if (E == kGradient && at_step == steps) {
            at_step = 0;
            ++at_product;
            aim();
        } else if (kAimed) {   // (beyond an offset's 32 bits)
            aim();
        }
    };
    const unsigned lds_at = (unsigned)(uintptr_t)(__attribute__((address_space(3))) char *)lds + wave * (kWave * 16);
    const auto load_a = [&](int stage, int i) {
        load_to_lds(a_from, a_off[i], kTurnedA ? 0 : at_step * kStepBytes, lds_at + stage + i * kThreads * 16);
    };
    const auto load_b = [&](int stage, int i) {
        load_to_lds(b_from, b_off[i], kPanels || kTurned ? 0 : at_step * kStepBytes, lds_at + kBAt + stage + i * kThreads * 16);
    };

    f32x4 acc[MT][NT];
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int j = 0; j < NT; ++j) {
            acc[i][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
            asm volatile("" : "+a"(acc[i][j]));
        }
    asm volatile("s_nop 7" ::: "memory");

    const int row16 = lane & 15, part = lane >> 4, turn = (row16 >> 1) & 7;
    Operand fa[2][MT], fb[2][NT];   // of each half
    const char *a_read = lds + (wm * MT * 16 + row16) * kStepBytes, *b_read = lds + kBAt + (wn * NT * 16 + row16) * kStepBytes;
    const int piece[2] = {(part ^ turn) << 4, ((4 + part) ^ turn) << 4};
    // turned: rows part * 8 + 0 .. 7 of the half; lane i of sixteen asks for 4 columns of row i / 4 and gets column i of 4 rows
    const int t_row = part * 8 + (row16 >> 2), t_turn = turn_of(TN, t_row), t_turn_a = turn_of(TM, t_row);
    const char *t_read = lds + kBAt + t_row * (TN * 2) + (row16 & 3) * 8, *t_read_a = lds + t_row * (TM * 2) + (row16 & 3) * 8;
    const auto turned = [](const char *at, int row_bytes) {
        typedef short s16x4 __attribute__((ext_vector_type(4)));
        typedef __attribute__((address_space(3))) s16x4 lds16x4;
        const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds16x4 *)at);
        const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds16x4 *)(at + 4 * row_bytes));
        return __builtin_bit_cast(Operand, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
    };
    const auto fetch = [&](int a_stage, int b_stage, int half, int which) {
        if (which < NT) {
            if constexpr (kTurned)
                fb[half][which] = turned(t_read + b_stage + half * 32 * (TN * 2) + ((wn * NT + which) ^ t_turn) * 32, TN * 2);
            else
                fb[half][which] = *reinterpret_cast<const Operand *>(b_read + b_stage + piece[half] + which * 16 * kStepBytes);
        } else {
            const int i = which - NT;
            if constexpr (kTurnedA)
                fa[half][i] = turned(t_read_a + a_stage + half * 32 * (TM * 2) + ((wm * MT + i) ^ t_turn_a) * 32, TM * 2);
            else
                fa[half][i] = *reinterpret_cast<const Operand *>(a_read + a_stage + piece[half] + i * 16 * kStepBytes);
        }
    };
    // Multiplies a half; meanwhile fetches the other half's fragments from the stages given and, in the first half,
    // loads A's next tile to `to_stage`, in the second B's.
    const auto half = [&](auto which_half, bool fetching, int a_stage, int b_stage, bool loading, int to_stage) {
        constexpr int h = decltype(which_half)::value, kLoads = h == 0 ? kALoads : kBLoads;
        constexpr int kSpan = h == 0 ? kProducts : (kProducts + 1) / 2;   // B's have less time until they are needed
#pragma unroll
        for (int q = 0; q < kProducts; ++q) {
#pragma unroll
            for (int i = 0; i < kLoads; ++i)
                if (loading && i * kSpan / kLoads == q) {
                    if (h == 0) load_a(to_stage, i);
                    else load_b(to_stage, i);
                }
#pragma unroll
            for (int f = 0; f < kFetches; ++f)
                if (fetching && f * kProducts / kFetches == q) fetch(a_stage, b_stage, h ^ 1, f);
            Mfma<T>::run(fa[h][q / NT], fb[h][q % NT], acc[q / NT][q % NT]);
        }
    };

    if (total > 0) {
        aim();
#pragma unroll
        for (int s = 0; s < 2; ++s)
            if (s < total) {
#pragma unroll
                for (int i = 0; i < kALoads; ++i) load_a(s * kABytes, i);
#pragma unroll
                for (int i = 0; i < kBLoads; ++i) load_b(s * kBBytes, i);
                next_step();
            }
        step_barrier<0>();
#pragma unroll
        for (int f = 0; f < kFetches; ++f) fetch(0, 0, 0, f);
        int a0 = 0, a1 = kABytes, a2 = 2 * kABytes, b0 = 0, b1 = kBBytes, step = 0;
        const auto turn_stages = [&]() {
            const int a = a0, b = b0;
            a0 = a1;
            a1 = a2;
            a2 = a;
            b0 = b1;
            b1 = b;
        };
        for (; step + 2 < total; ++step) {
            half(HalfOf<0>{}, true, a0, b0, true, a2);
            step_barrier<kALoads>();   // the next step's tiles are there, and nobody reads b0 any more
            half(HalfOf<1>{}, true, a1, b1, true, b0);
            next_step();
            turn_stages();
        }
        for (; step < total; ++step) {
            half(HalfOf<0>{}, true, a0, b0, false, 0);
            step_barrier<0>();
            half(HalfOf<1>{}, step + 1 < total, a1, b1, false, 0);
            turn_stages();
        }
    }
    asm volatile("s_nop 15\n s_nop 15" ::: "memory");   // the last product's sums are written before they are read
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int j = 0; j < NT; ++j) asm volatile("" : "+a"(acc[i][j]));

    // acc[i][j][r] is C[m][n] at m = m_lane + i * 16 + r, n = n_lane + j * 16
    const int m_lane = m0 + wm * MT * 16 + part * 4, n_lane = n0 + wn * NT * 16 + row16;

    if constexpr (E == kSoftmax) {
        __syncthreads();
        float2 *joined = reinterpret_cast<float2 *>(lds);   // [WM][TN]
#pragma unroll
        for (int j = 0; j < NT; ++j) {
            const int n = n_lane + j * 16;
            const int label = n < n_rows ? p.label[n] - p.m_first - m_lane : -1;
            SoftSum s = {-INFINITY, 0.0f};
            float z[MT][4];
#pragma unroll
            for (int i = 0; i < MT; ++i)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    z[i][r] = acc[i][j][r] * p.scale;
                    if (m_lane + i * 16 + r < p.m) s.top = fmaxf(s.top, z[i][r]);
                    if (label == i * 16 + r) p.z_label[n] = z[i][r];
                }
            s.top = fmaxf(s.top, __shfl_xor(s.top, 16));
            s.top = fmaxf(s.top, __shfl_xor(s.top, 32));
            const float top = s.top == -INFINITY ? kLowest : s.top;   // (no row of the vocabulary here, or all -infinity)
#pragma unroll
            for (int i = 0; i < MT; ++i)
#pragma unroll
                for (int r = 0; r < 4; ++r)
                    if (m_lane + i * 16 + r < p.m) s.sum += __expf(z[i][r] - top);
            s.sum += __shfl_xor(s.sum, 16);
            s.sum += __shfl_xor(s.sum, 32);
            if (part == 0) joined[wm * TN + wn * NT * 16 + j * 16 + row16] = make_float2(top, s.sum);
        }
        __syncthreads();
        for (int i = tid; i < TN && n0 + i < n_rows; i += kThreads) {
            SoftSum s = {joined[i].x, joined[i].y};
#pragma unroll
            for (int w = 1; w < WM; ++w) s = soft_join(s, SoftSum{joined[w * TN + i].x, joined[w * TN + i].y});
            p.parts[(int64_t)(n0 + i) * p.parts_ld + p.parts_first + tm] = make_float2(s.top, s.sum);
        }
    } else if constexpr (E == kDerivative) {
#pragma unroll
        for (int j = 0; j < NT; ++j) {
            const int n = n_lane + j * 16;
            const bool in = n < n_rows;
            const int label = in ? p.label[n] - p.m_first - m_lane : -1;
            const float lse = in ? p.lse[n] : 0.0f, g = in ? p.row_grad[n] * *p.row_factor : 0.0f;
            float of_label = 0.0f;
#pragma unroll
            for (int i = 0; i < MT; i += 2) {
                constexpr int kBoth = SPLIT ? 3 : TN == 64 ? 2 : 1;   // arrays (16-bit types: two of up to 64 positions)
                uint2 x[2][kBoth] = {};
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    if (i + h == MT) break;
                    float d[4];
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        const int at = (i + h) * 16 + r;
                        const float q = __expf(acc[i + h][j][r] * p.scale - lse) - (label == at ? 1.0f : 0.0f);
                        d[r] = in && m_lane + at < p.m ? q * g : 0.0f;
                        if (!SPLIT) of_label = label == at ? d[r] : of_label;
                    }
                    if constexpr (SPLIT) {
                        bf16 y[4][3];
#pragma unroll
                        for (int r = 0; r < 4; ++r) split3(d[r], y[r]);
#pragma unroll
                        for (int s = 0; s < 3; ++s) x[h][s] = make_uint2(pack2(y[0][s], y[1][s]), pack2(y[2][s], y[3][s]));
                    } else {
                        T y[4];
#pragma unroll
                        for (int s = 0; s < kBoth; ++s) {   // (the second: what rounding took)
#pragma unroll
                            for (int r = 0; r < 4; ++r) {
                                y[r] = (T)d[r];
                                d[r] -= (float)y[r];
                            }
                            x[h][s] = make_uint2(pack2(y[0], y[1]), pack2(y[2], y[3]));
                        }
                    }
                }
                // Neighbouring sixteens of lanes exchange a part, so that each has eight elements of one tile of 16 rows to
                // store (of the last of an odd number of such tiles: four).  Four each: 75 us for 70 (1003 x 30011 x 1021 f16).
                const bool whole = i + 1 < MT;
                const int m = m_lane + i * 16 + (whole ? (part & 1) * 16 + (part >> 1) * 8 - part * 4 : 0);
                if (whole) {
#pragma unroll
                    for (int s = 0; s < kBoth; ++s) {
                        const auto first = __builtin_amdgcn_permlane16_swap(x[0][s].x, x[1][s].x, false, false);
                        const auto second = __builtin_amdgcn_permlane16_swap(x[0][s].y, x[1][s].y, false, false);
                        x[0][s] = make_uint2(first[0], second[0]);
                        x[1][s] = make_uint2(first[1], second[1]);
                    }
                }
                if (m >= p.d_cols) continue;   // (tiles of 192 and 160 rows may pass the last panel)
                T *to_d = static_cast<T *>(p.d) + (m >> 8) * p.d_panel + (int64_t)n * 256 + (m & 255);
#pragma unroll
                for (int s = 0; s < kBoth; ++s) {
                    if (whole) *reinterpret_cast<uint4 *>(to_d + s * p.d_plane) = make_uint4(x[0][s].x, x[0][s].y, x[1][s].x, x[1][s].y);
                    else *reinterpret_cast<uint2 *>(to_d + s * p.d_plane) = x[0][s];
                }
            }
            if (!SPLIT && p.residual && label >= 0 && label < MT * 16 && (label & 15) < 4 && m_lane + label < p.m)
                p.residual[n] = of_label - (float)(T)of_label;
        }
        // the next product reads whole steps of 64: what tiles of 160 rows leave of the last one is zero
        if (TM % kStep != 0 && tm == tiles_m - 1) {
            const int first = tiles_m * TM, end = (p.m + kStep - 1) / kStep * kStep;
            for (int i = tid; i < TN * kStep; i += kThreads) {
                const int m = first + i % kStep;
                if (m < end)
                    for (int s = 0; s < (SPLIT ? 3 : p.d_arrays); ++s)
                        static_cast<T *>(p.d)[s * p.d_plane + (m >> 8) * p.d_panel + (int64_t)(n0 + i / kStep) * 256 + (m & 255)] = (T)0.0f;
            }
        }
    } else if constexpr (E == kSums) {
        float *sums = p.sums + split * p.sums_split;
#pragma unroll
        for (int j = 0; j < NT; ++j) {
            const int n = n_lane + j * 16;
            if (n >= n_rows) continue;
#pragma unroll
            for (int i = 0; i < MT; ++i) {
                const int m = m_lane + i * 16;   // (sums_ld is a multiple of 4, so m < p.m leaves room for four)
                if (m >= p.m) continue;
                f32x4 *to_sum = reinterpret_cast<f32x4 *>(sums + (int64_t)n * p.sums_ld + m);
                *to_sum = p.add ? *to_sum + acc[i][j] : acc[i][j];
            }
        }
    } else if constexpr (E >= kGate) {
        __syncthreads();
        Tile t = {reinterpret_cast<float *>(lds) + wave * epilogue_floats(MT), lane, m0 + wm * MT * (E == kGate ? 8 : 16), n0 + wn * NT * 16, n_rows, p.m};
        if (p.splits > 1) {
            if (E == kGate) {   // (both projections as they lie in the tiles)
                t.m = tm * TM + wm * MT * 16;
                t.cols = (p.m + 15) / 16 * 32;
            }
            sums_epilogue(p.sums + split * p.sums_split, p.sums_ld, acc, t);
        } else if constexpr (E == kGate || E == kGateGrad) {
            act_epilogue<E == kGateGrad, T, O, MT, NT, SPLIT>(p.ffn, acc, t);
        } else {
            out_epilogue<O, MT, NT>(p.ffn, acc, t, p.add);
        }
    } else {
        const float alpha = p.scale * *p.out_scale;
        typedef O O4 __attribute__((ext_vector_type(4), aligned(sizeof(O))));
#pragma unroll
        for (int j = 0; j < NT; ++j) {
            const int n = n_lane + j * 16;
            if (n >= n_rows) continue;
            O *row = static_cast<O *>(p.out) + (int64_t)n * p.out_ld;
#pragma unroll
            for (int i = 0; i < MT; ++i) {
                const int m = m_lane + i * 16;
                if (m + 4 <= p.m) {
                    O4 x = {};
                    if (p.add) x = *reinterpret_cast<const O4 *>(row + m);
#pragma unroll
                    for (int r = 0; r < 4; ++r) x[r] = (O)((p.add ? (float)x[r] : 0.0f) + alpha * acc[i][j][r]);
                    *reinterpret_cast<O4 *>(row + m) = x;
                } else {
#pragma unroll
                    for (int r = 0; r < 4; ++r)
                        if (m + r < p.m) row[m + r] = (O)((p.add ? (float)row[m + r] : 0.0f) + alpha * acc[i][j][r]);
                }
            }
        }
    }
#else
    (void)p;
#endif
}

}  // namespace deft
