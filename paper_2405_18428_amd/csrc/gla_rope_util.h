// A token's position on an axis and the sine and cosine of a pair's angle (gfx950 device code).
#pragma once
#include "gla_ops.h"

namespace gla {
namespace {

__device__ inline int position(const RopeParams &p, long long token, int n, int axis) {
    if (p.positions != nullptr) return p.positions[token * p.axes + axis];
    if (p.axes == 1) return n;
    const int cell = p.grid_h * p.grid_w, f = n / cell, r = n - f * cell;
    const int which = p.axes == 2 ? axis + 1 : axis;
    return which == 0 ? f : which == 1 ? r / p.grid_w : r % p.grid_w;
}

// of a pair at a position
__device__ __forceinline__ void turn(const RopeParams &p, int pair, double pos, float *cs, float *sn) {
    const double whole = pos * p.turns[pair];                        // exact
    const double turns = __builtin_fma(pos, p.rest[pair], whole - __builtin_rint(whole));
    const float f = (float)(turns - __builtin_rint(turns));          // -1/2 .. 1/2
    sincospif(2.f * f, sn, cs);
}

}  // namespace
}  // namespace gla
