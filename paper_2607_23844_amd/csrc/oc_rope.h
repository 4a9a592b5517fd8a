// Turning pairs of channels by a position (k_rope.hip, k_short.hip).
#pragma once
#include "oc_device.h"
#include "oc_ops.h"

namespace oc {

struct Turn { float c, s; };

// A position times turns per position in 64 bits, less the whole turns: the
// fp32 fraction is at most a half (positions of 2^20 would lose 2^-4 of a turn
// in 32 bits).
__device__ __forceinline__ float rope_fraction(int at, double origin, double turn) {
    const double t = ((double)at + origin) * turn;
    return (float)(t - rint(t));
}
__device__ __forceinline__ Turn rope_turn(float x) { return Turn{cospif(2.f * x), sinpif(2.f * x)}; }
// For values of 16 bits: the hardware's sine and cosine of a fraction of a turn,
// one instruction each, off by at most 2^-22.9 there (measured over 2^22
// fractions in [-1/2, 1/2]).
__device__ __forceinline__ Turn rope_turn16(float x) {
    return Turn{__builtin_amdgcn_cosf(x), __builtin_amdgcn_sinf(x)};
}

__device__ __forceinline__ int rope_axis(const RopeGeom &g, int p) { return p < g.axis1 ? 0 : p < g.axis2 ? 1 : 2; }

// channels of pair p in its head
__device__ __forceinline__ void rope_channels(const RopeGeom &g, int p, int &lo, int &hi) {
    lo = 2 * p;
    hi = lo + 1;
    if (g.pairs) return;
#pragma unroll
    for (int m = 0; m < 4; ++m)
        if (p >= g.sect[m] && p < g.sect[m + 1]) {
            lo = g.sect[m] + p;
            hi = lo + g.sect[m + 1] - g.sect[m];
        }
}

__device__ __forceinline__ void turn_pair(float &x, float &y, const Turn &t) {
    const float x0 = x, y0 = y;
    x = fmaf(x0, t.c, -(y0 * t.s));
    y = fmaf(x0, t.s, y0 * t.c);
}

}  // namespace oc
