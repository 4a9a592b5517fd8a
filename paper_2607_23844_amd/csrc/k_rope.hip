// Rotary positions of q and k rows with up to three axes.
//
// A thread owns one unit of a head's channels, the same for all heads of its
// row: 8 neighbouring channels (pairs side by side), or V channels and their V
// partners half a section further.  The cosines and sines of its pairs are
// computed once and used for every head of q and k.  Angles: a position times
// turns per position in 64 bits, less the whole turns, then cospi and sinpi of
// a fp32 fraction of at most a half (positions of 2^20 would lose 2^-4 of a
// turn in 32 bits).
#include "oc_attn_common.h"
#include "oc_device.h"
#include "oc_launch.h"
#include "oc_ops.h"
#include <cmath>
#include <cstring>

namespace oc {

namespace {

template <typename T, int V> struct Chunk { typedef T type __attribute__((ext_vector_type(V))); };
template <typename T> struct Chunk<T, 1> { typedef T type; };

template <typename T, int V>
__device__ __forceinline__ void get(const T *p, float (&v)[V]) {
    typedef typename Chunk<T, V>::type C;
    const C c = *reinterpret_cast<const C *>(p);
    if constexpr (V == 1) v[0] = (float)c;
    else {
#pragma unroll
        for (int i = 0; i < V; ++i) v[i] = (float)c[i];
    }
}
template <typename T, int V>
__device__ __forceinline__ void put(T *p, const float (&v)[V]) {
    typedef typename Chunk<T, V>::type C;
    C c;
    if constexpr (V == 1) c = (T)v[0];
    else {
#pragma unroll
        for (int i = 0; i < V; ++i) c[i] = (T)v[i];
    }
    *reinterpret_cast<C *>(p) = c;
}

// PAIRS: unit u is channels 8u..8u+7 (V = 4 pairs); else channels lo.. and hi.. of V pairs
template <typename T, bool PAIRS, int V>
__global__ __launch_bounds__(256) void k_rope(RopeGeom g, RopeArgs a) {
    const int units = g.dh / 2 / V;
    const long id = (long)folded_block() * 256 + threadIdx.x, row = id / units;
    const int u = (int)(id - row * units), p0 = u * V;
    if (row >= a.rows) return;
    double at[3];
    if (a.pos != nullptr) {
#pragma unroll
        for (int i = 0; i < 3; ++i) at[i] = a.pos[row * 3 + i];
    } else {
        const long t = batch_token((int)row, a.idx, a.tF, a.tN);
        if (t < 0 || t >= g.FN) return;
        const int f = (int)(t / g.N), n = (int)(t - (long)f * g.N);
        at[0] = f;
        at[1] = n / g.W;
        at[2] = n % g.W;
    }
    float co[V], si[V];
    bool on[V];
#pragma unroll
    for (int j = 0; j < V; ++j) {
        const int p = p0 + j;
        on[j] = p < g.P;
        const int axis = p < g.axis1 ? 0 : p < g.axis2 ? 1 : 2;
        const double pos = axis == 0 ? at[0] + g.origin[0] : axis == 1 ? at[1] + g.origin[1] : at[2] + g.origin[2];
        const double t = on[j] ? pos * g.turn[p] : 0.0;
        const float x = 2.f * (float)(t - rint(t));
        co[j] = cospif(x);
        si[j] = a.inverse ? -sinpif(x) : sinpif(x);
    }
    int lo = 2 * p0, hi = 0;
    if constexpr (!PAIRS) {
        int s0 = 0, s1 = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (p0 >= g.sect[i] && p0 < g.sect[i + 1]) {
                s0 = g.sect[i];
                s1 = g.sect[i + 1];
            }
        lo = s0 + p0;
        hi = lo + (s1 - s0);
    }
    auto turn = [&](const T *src, T *dst) {
        if constexpr (PAIRS) {
            float v[8];
            get<T, 8>(src + lo, v);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                if (!on[j]) continue;
                const float x = v[2 * j], y = v[2 * j + 1];
                v[2 * j] = fmaf(x, co[j], -(y * si[j]));
                v[2 * j + 1] = fmaf(x, si[j], y * co[j]);
            }
            put<T, 8>(dst + lo, v);
        } else {
            float v[V], w[V];
            get<T, V>(src + lo, v);
            get<T, V>(src + hi, w);
#pragma unroll
            for (int j = 0; j < V; ++j) {
                if (!on[j]) continue;
                const float x = v[j], y = w[j];
                v[j] = fmaf(x, co[j], -(y * si[j]));
                w[j] = fmaf(x, si[j], y * co[j]);
            }
            put<T, V>(dst + lo, v);
            put<T, V>(dst + hi, w);
        }
    };
    if (a.q != nullptr)
        for (int h = 0; h < a.heads; ++h)
            turn((const T *)a.q + row * a.ld_q + h * g.dh, (T *)a.qo + row * a.ld_qo + h * g.dh);
    if (a.k != nullptr)
        for (int h = 0; h < a.k_heads; ++h)
            turn((const T *)a.k + row * a.ld_k + h * g.dh, (T *)a.ko + row * a.ld_ko + h * g.dh);
}

template <typename T, bool PAIRS, int V>
hipError_t go_rope(const RopeGeom &g, const RopeArgs &a, hipStream_t st) {
    const long threads = (long)a.rows * (g.dh / 2 / V);
    launch_k(k_rope<T, PAIRS, V>, folded_grid((threads + 255) / 256, 256), 256, 0, st, g, a);
    return hipGetLastError();
}

template <typename T>
hipError_t type_rope(const RopeGeom &g, const RopeArgs &a, hipStream_t st) {
    if (g.pairs) return go_rope<T, true, 4>(g, a, st);
    switch (g.vec) {
        case 8: return go_rope<T, false, 8>(g, a, st);
        case 4: return go_rope<T, false, 4>(g, a, st);
        case 2: return go_rope<T, false, 2>(g, a, st);
        default: return go_rope<T, false, 1>(g, a, st);
    }
}

}  // namespace

void rope_geom(const int *dim, int layout, int shared, const int *origin, double theta, const double *scale, int F,
               int H, int W, int head_dim, RopeGeom &g) {
    std::memset(&g, 0, sizeof(g));
    g.axis1 = dim[0] / 2;
    g.axis2 = g.axis1 + dim[1] / 2;
    g.P = g.axis2 + dim[2] / 2;
    g.dh = head_dim;
    g.N = H * W;
    g.W = W;
    g.FN = (long)F * g.N;
    g.pairs = layout == 0;
    const bool halves = layout == 1;
    const int sect[5] = {0, halves ? g.axis1 : g.P, halves ? g.axis2 : g.P, g.P, head_dim / 2};
    std::memcpy(g.sect, sect, sizeof(sect));
    g.vec = 8;
    for (int s : sect)
        while (s % g.vec) g.vec /= 2;
    int p = 0;
    for (int i = 0; i < 3; ++i) {
        g.origin[i] = origin[i];
        for (int j = 0; j < dim[i] / 2; ++j, ++p) {
            const double e = shared ? (double)p / g.P : 2.0 * j / dim[i];
            g.turn[p] = scale[i] * std::pow(theta, -e) / (2.0 * 3.14159265358979323846);
        }
    }
}

hipError_t launch_rope(const RopeGeom &g, const RopeArgs &a, RopeType type, hipStream_t st) {
    if (a.rows == 0 || (a.q == nullptr && a.k == nullptr)) return hipSuccess;
    StageScope _stage(st, "rope");
    switch (type) {
        case ROPE_BF16: return type_rope<__bf16>(g, a, st);
        case ROPE_F16: return type_rope<_Float16>(g, a, st);
        default: return type_rope<float>(g, a, st);
    }
}

}  // namespace oc
