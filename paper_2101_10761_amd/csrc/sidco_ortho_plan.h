// How the steps of a Newton-Schulz call X <- P X, P = aI + bG + cG^2, G = X X^T, are taken: in which precision, and how many on
// one reading of X.  Host code without HIP.
#ifndef SIDCO_ORTHO_PLAN_H
#define SIDCO_ORTHO_PLAN_H

#include <math.h>
#include <stdint.h>

namespace sidco {

// The most that a step multiplies a direction by: |a + bx + cx^2| over the squares x of singular values up to 1.5.
inline float ortho_growth(float a, float b, float c)
{
    float top = fmaxf(fabsf(a), fabsf(a + 2.25f * b + 5.0625f * c));
    if (c != 0.0f && -b / (2 * c) > 0.0f && -b / (2 * c) < 2.25f) top = fmaxf(top, fabsf(a - b * b / (4 * c)));
    return top;
}

// Steps, from the first on, whose operands have 22 bits where the result's type decides.  The last one can do with 11 before a
// result of 8 bits (bf16): what it rounds is multiplied once, by 3.4445 of the usual coefficients to at most the result's own
// rounding, 1.4e-3 and 1.7e-3 of the result.  A growth of 4 keeps it there.
inline int ortho_paired(int steps, float a, float b, float c, bool eight_bits)
{
    return eight_bits && ortho_growth(a, b, c) <= 4.0f ? steps - 1 : steps;
}

// How many steps share a pass over X.  Steps after the first of a group know their G without X: P and G commute, so that
// (PX)(PX)^T = P G P, and the group's X is Q X with Q the product of its P.  In products of m x m x m operations, symmetric ones
// counting half, and with n = r m, a step of its own costs 3r + 1 and one that joins a group 4.  What rounding leaves in G where
// it should be small grows by a^2 with every step of a group, as the error of X itself does by a; with a = 3.4445, errors of
// groups of 2 in halves are those of single steps (1e-3 to 3e-3 for spectra from flat to 1/k; of 3 up to 6e-3), of 3 with 22 bits
// too (3e-7 to 5e-6 with exact sums), of 4 with 22 bits 3e-7 to 1.2e-5, and of 5 without bound.  A launch counts 4 us against 6e14 operations a
// second.
inline int ortho_group(int batch, int64_t m, int64_t n, int steps, bool pairs, int most)
{
    const double r = (double)n / (double)m, unit = (double)batch * (double)m * (double)m * (double)m * (pairs ? 3.0 : 1.0) / 6e8;
    int best = 1;
    double least = 0.0;
    for (int g = 1; g <= most && g <= steps; ++g) {
        const int groups = (steps + g - 1) / g, joined = steps - groups;
        const double t = (groups * (3 * r + 1) + joined * 4) * unit + (groups * 3 + joined * 4) * 4.0;
        if (g == 1 || t < least) least = t, best = g;
    }
    return best;
}

// Whether one block takes a matrix through all its steps, in LDS: 160 KB less 16 KB for G hold 576 rows of 64 pairs of halves;
// of halves alone the registers have room for 768.  Offsets within the matrix have 32 bits there.
constexpr int kOneSide = 64, kOnePairs = 576, kOneHalves = 768;
inline bool ortho_one_block(int64_t rows, int64_t cols, int64_t ldx, bool pairs)
{
    const int64_t m = rows < cols ? rows : cols, n = rows < cols ? cols : rows;
    return m <= kOneSide && n <= (pairs ? kOnePairs : kOneHalves) && ldx <= (1 << 20);
}

struct OrthoGroups {
    int paired, halves;  // steps in a group of either kind; 0 where there is none
};

// With halves behind them, the steps in pairs need not be better than those: up to 4 go together, always, for then the other X
// of the workspace has no low halves.  For small matrices that is a launch more than single steps.
inline OrthoGroups ortho_groups(int batch, int64_t m, int64_t n, int steps, int paired)
{
    const int halves = steps - paired;
    OrthoGroups g = {0, 0};
    if (paired > 0) g.paired = halves > 0 ? (paired < 4 ? paired : 4) : ortho_group(batch, m, n, paired, true, 3);
    if (halves > 0) g.halves = ortho_group(batch, m, n, halves, false, 2);
    return g;
}

}  // namespace sidco
#endif
