// How the head's products are cut: pieces of the vocabulary, tiles, parts of a long sum.
#pragma once
#include "ends.h"

namespace deft {

constexpr int kStep = 64;            // elements of k per step of a product
constexpr int kTile = 256;
constexpr int64_t kPieceBytes = (int64_t)3 << 27;    // of d
constexpr int64_t kWeightBytes = (int64_t)1 << 28;   // of a piece's rows, packed
constexpr int kMaxSplits = 128;
constexpr int kFew = 64;                             // positions that a tile of 64 holds

inline int64_t up(int64_t x, int64_t to) { return (x + to - 1) / to * to; }

// The shape of a product's tiles.  Up to 64 rows of b: 256 x 64, bound by reading a.  Otherwise the one whose rounds over
// the compute units take least: 256 x 256 is the quickest by element, the others leave fewer units idle at the end.  The
// 128 x 128 ones and the feed-forward block's 128 x 64 ones run two workgroups on a compute unit (80 and 64 KB of LDS each).
enum Shape { kLarge, kMiddle, kLow, kHalf, kSmall, kNarrow, kTiny, kShapes };

struct ShapeCost {
    int tm, tn;
    double step, fixed;   // of a round, in the time of a 256 x 256 tile's step (1.58 us)
};
// Measured in bf16 on 256 tiles (512 of the last) of 25 and 128 steps, TFLOP/s: 256 x 256 1092 and 1294, 192 x 256 1042
// and 1287, 160 x 256 996 and 1245, 256 x 128 951 and 1212, 128 x 128 906 and 1120 (256 tiles, one to a unit: 684, 1025).
constexpr ShapeCost kCosts[kShapes] = {{256, 256, 1.0, 6.0}, {192, 256, 0.745, 5.7}, {160, 256, 0.64, 5.3},
                                       {256, 128, 0.522, 4.7}, {128, 128, 0.571, 4.4}, {256, 64, 0.4, 4.5}, {128, 64, 0.33, 4.0}};
constexpr double kAloneStep = 0.29, kAloneFixed = 5.0;   // of a 128 x 128 tile that has a compute unit to itself
constexpr double kTinyStep = 0.18, kTinyFixed = 4.0;     // of a 128 x 64 one

// `alone`: by what a step of a tile that has a compute unit to itself takes longer than in bf16 (which waits for memory, and where
// operands are three arrays the card's caches give half as much again).
inline double cost_of(Shape shape, int64_t m, int64_t n, int64_t steps, int64_t splits, int64_t units, double alone = 1.0)
{
    const ShapeCost &c = kCosts[shape];
    const int64_t tiles = up(m, c.tm) / c.tm * (up(n, c.tn) / c.tn) * splits;
    const double each = (double)steps / (double)splits;
    if (shape != kSmall && shape != kTiny) return (double)(up(tiles, units) / units) * (c.step * each + c.fixed);
    const int64_t pairs = tiles / (2 * units), rest = tiles % (2 * units);
    return (double)(pairs + (rest > units ? 1 : 0)) * (c.step * each + c.fixed) +
           (rest > 0 && rest <= units ? (shape == kTiny ? kTinyStep * alone * each + kTinyFixed : kAloneStep * alone * each + kAloneFixed) : 0.0);
}

constexpr unsigned kHeadWithout = 1u << kTiny;

// `without`: shapes (their bits) that a product has no kernel for.
inline Shape shape_of(int64_t m, int64_t n, int64_t steps, int64_t splits, int64_t units, unsigned without = kHeadWithout, double alone = 1.0)
{
    if (n <= kFew) return kNarrow;
    Shape best = kLarge;
    for (int s = 1; s < kShapes; ++s)
        if (s != kNarrow && !(without >> s & 1) &&
            cost_of((Shape)s, m, n, steps, splits, units, alone) < cost_of(best, m, n, steps, splits, units, alone))
            best = (Shape)s;
    return best;
}

inline double least_cost(int64_t m, int64_t n, int64_t steps, int64_t splits, int64_t units, unsigned without = kHeadWithout, double alone = 1.0)
{
    return cost_of(shape_of(m, n, steps, splits, units, without, alone), m, n, steps, splits, units, alone);
}

// Parts that a sum over k is cut into, where its tiles leave compute units idle: each part's sums go to memory and are
// joined later, so there are no more of them than shorten the whole by a twentieth.
inline int splits_of(int64_t m, int64_t n, int64_t steps, int64_t units, unsigned without = kHeadWithout)
{
    const int64_t tiles = up(m, 256) / 256 * (n <= kFew ? 1 : up(n, 256) / 256);
    int best = 1;
    double least = 1e30;
    for (int s = 1; s <= kMaxSplits && (s == 1 || (tiles * s <= 2 * units && steps >= s * 8)); s *= 2) {
        const double t = least_cost(m, n, steps, s, units, without);
        if (t < 0.95 * least) {
            least = t;
            best = s;
        }
    }
    return best;
}

}  // namespace deft
