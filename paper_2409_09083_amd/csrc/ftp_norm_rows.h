// Which form of the row kernels of the layer norm a row takes, shared by their launchers and the host check of tests/host_checks (plain integer arithmetic).
#pragma once
#include <algorithm>

namespace ftp {

inline int ceil_pow2(int v) { int p = 1; while (p < v) p <<= 1; return p; }

// Vectors of a lane at most: 8, and 32 values.
constexpr int row_most(int vec) { return 32 / vec < 8 ? 32 / vec : 8; }

// Lanes of a row and vectors of a lane: a row in one wavefront where its vectors fit, else a workgroup.  NV 0: too long for registers.
struct RowForm { int lanes, nv; bool wide; };
inline RowForm row_form(int C, int vec)
{
    const int vecs = (C - 1) / vec + 1, most = row_most(vec);
    if (vecs <= 64 * most) {
        const int lanes = std::min(64, ceil_pow2(vecs));
        return {lanes, ceil_pow2((vecs + lanes - 1) / lanes), false};
    }
    if (vecs <= 256 * most) return {256, ceil_pow2((vecs + 255) / 256), true};
    return {256, 0, true};
}

// The forms that rows take: a workgroup's lanes hold more than a quarter of what a wavefront's could.
constexpr bool row_built(int vec, int nv, bool wide) { return nv <= row_most(vec) && (!wide || 4 * nv > row_most(vec)); }

}  // namespace ftp
