// Turning pairs of channels by a position (k_rope.hip, and where k_short.hip and
// k_proj.hip have staged Q and K).
#pragma once
#include "oc_device.h"
#include "oc_internal.h"
#include "oc_mfma_tile.h"
#include "oc_ops.h"
#include <type_traits>

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

// A turned value in its tensor's type; fp16 saturates as the projections do: a pair
// inside its range can be turned out of it, up to sqrt(2) 65504.
template <typename T>
__device__ __forceinline__ T turned(float v) {
    if constexpr (std::is_same<T, _Float16>::value) return __builtin_bit_cast(_Float16, f2h_bits(v));
    else return (T)v;
}

// V pairs of a head, from pair p0 on (all of them turned), staged in LDS in fp16:
// a run of 2 V channels, or two of V.  V = 1, or 4 where it divides the sections
// (vec).
template <bool PAIRS, int V>
struct RopeUnit {
    static constexpr int W = PAIRS ? 2 * V : V;
    typedef _Float16 Run __attribute__((ext_vector_type(W)));
    struct Vals { Run a, b; };
    int lo, hi;                  // first channels
    int on_x[V], on_y[V], on_z[V];   // masks of a pair's axis (selects became branches)
    double turn[V], origin[V];
    __device__ __forceinline__ RopeUnit(const RopeGeom &g, int p0) {
        rope_channels(g, p0, lo, hi);
#pragma unroll
        for (int j = 0; j < V; ++j) {
            const int axis = rope_axis(g, p0 + j);
            on_x[j] = -(axis == 0);
            on_y[j] = -(axis == 1);
            on_z[j] = -(axis == 2);
            turn[j] = g.turn[p0 + j];
            origin[j] = g.origin[axis];
        }
    }
    __device__ __forceinline__ Vals load(const _Float16 *head) const {
        Vals v;
        v.a = *reinterpret_cast<const Run *>(head + lo);
        if constexpr (!PAIRS) v.b = *reinterpret_cast<const Run *>(head + hi);
        return v;
    }
    __device__ __forceinline__ void store(_Float16 *head, const Vals &v) const {
        *reinterpret_cast<Run *>(head + lo) = v.a;
        if constexpr (!PAIRS) *reinterpret_cast<Run *>(head + hi) = v.b;
    }
    // pair j's angle at frame w.x, row w.y, column w.z
    __device__ __forceinline__ Turn at(const int4 &w, int j) const {
        return rope_turn16(rope_fraction((w.x & on_x[j]) | (w.y & on_y[j]) | (w.z & on_z[j]), origin[j], turn[j]));
    }
    __device__ __forceinline__ static void apply(Vals &v, int j, const Turn &t) {
        float x = (float)v.a[PAIRS ? 2 * j : j], y = PAIRS ? (float)v.a[PAIRS ? 2 * j + 1 : 0] : (float)v.b[j];
        turn_pair(x, y, t);
        v.a[PAIRS ? 2 * j : j] = turned<_Float16>(x);
        (PAIRS ? v.a : v.b)[PAIRS ? 2 * j + 1 : j] = turned<_Float16>(y);
    }
};

// Where token t of the grid lies (w = 0: it has no place)
__device__ __forceinline__ int4 rope_place(const RopeGeom &g, long t) {
    int4 w = {0, 0, 0, t >= 0 && t < g.FN};
    if (w.w) {   // (fewer than 2^30 tokens)
        const int n = (int)t % g.N;
        w.x = (int)t / g.N;
        w.y = n / g.W;
        w.z = n % g.W;
    }
    return w;
}

// Last argument of a kernel that stages Q and K: no rotation, or this one and its
// row -> token table (NULL: as the rows are read).
struct NoRope {};
struct StagedRope {
    RopeGeom g;
    const int32_t *idx;
};
template <typename ROPE> constexpr bool ROTATES = std::is_same<ROPE, StagedRope>::value;
inline StagedRope staged_rope(const AttnArgs &a) {
    return StagedRope{*a.rope, a.rope_idx != nullptr ? a.rope_idx : a.row_idx};
}

}  // namespace oc
