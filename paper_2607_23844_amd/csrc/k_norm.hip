// Norms before and after a sublayer, fused with its gate, its modulation and
// the residual, and their gradients.
//   z = post(y), h = rs x + g z, n = pre(h)(1 + s) + t
// With u the normalised h (rstd r), a = u w + b its weighted form, v and r_y
// the same of y, the gradients are
//   ds = sum dn a, dt = sum dn, da = dn (1 + s), dw = sum da u, db = sum da,
//   H  = dh + r (da w - m1 - u m2), m2 = mean(da w u), m1 = mean(da w) (layer; 0 for rms),
//   dx = rs H, dg = sum H z, dz = g H, dw_post = sum dz v, db_post = sum dz,
//   dy = r_y (dz w_post - k1 - v k2), k1 and k2 the same means over dz w_post
// (sums over the rows that share the vector, means over the channels).
#include "oc_device.h"
#include "oc_launch.h"
#include "oc_norm_plan.h"
#include "oc_ops.h"
#include "oc_attn_common.h"
#include <algorithm>
#include <type_traits>

namespace oc {

namespace {

constexpr int NORM_RMS = 1, NORM_LAYER = 2;   // oc_norm_kind

// Eight consecutive elements as fp32, and back (rounded to nearest even; a NaN
// stays one).
__device__ __forceinline__ void load8(const uint16_t *p, float (&v)[8]) {
    const uint4 w = *reinterpret_cast<const uint4 *>(p);
    const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        v[2 * i] = __uint_as_float(u[i] << 16);
        v[2 * i + 1] = __uint_as_float(u[i] & 0xFFFF0000u);
    }
}
__device__ __forceinline__ void load8(const float *p, float (&v)[8]) {
    *reinterpret_cast<f32x4 *>(v) = *reinterpret_cast<const f32x4 *>(p);
    *reinterpret_cast<f32x4 *>(v + 4) = *reinterpret_cast<const f32x4 *>(p + 4);
}
__device__ __forceinline__ void store8(uint16_t *p, const float (&v)[8]) {
    bf16x8 o;
#pragma unroll
    for (int i = 0; i < 8; ++i) o[i] = (__bf16)v[i];
    *reinterpret_cast<bf16x8 *>(p) = o;
}
__device__ __forceinline__ void store8(float *p, const float (&v)[8]) {
    *reinterpret_cast<f32x4 *>(p) = *reinterpret_cast<const f32x4 *>(v);
    *reinterpret_cast<f32x4 *>(p + 4) = *reinterpret_cast<const f32x4 *>(v + 4);
}
template <typename T>
__device__ __forceinline__ void load8_or(const T *p, long at, float other, float (&v)[8]) {
    if (p != nullptr) {
        load8(p + at, v);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = other;
    }
}

// the same of four or eight elements
template <int N, typename T>
__device__ __forceinline__ void load_or(const T *p, long at, float other, float (&v)[N]) {
    static_assert(N == 4 || N == 8, "chunks of four or eight");
    if constexpr (N == 8) {
        load8_or(p, at, other, v);
    } else if (p == nullptr) {
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = other;
    } else if constexpr (sizeof(T) == 2) {
        const u16x4 w = *reinterpret_cast<const u16x4 *>(p + at);
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = bf2f(w[i]);
    } else {
        *reinterpret_cast<f32x4 *>(v) = *reinterpret_cast<const f32x4 *>(p + at);
    }
}

// Sum over the block's 256 threads, the same order for every thread.
__device__ __forceinline__ float block_sum(float v, float *red) {
    v = wave_sum(v);
    __syncthreads();   // red may still be read
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
    __syncthreads();
    return (red[0] + red[1]) + (red[2] + red[3]);
}

// ---------------------------------------------------------------------------
// Rows that stay in registers.  A team (16, 32 or 64 lanes, or the block of 256)
// holds a row in CH chunks of 8 channels per thread, so x, y, dh and dn are
// read once, whatever the number of means over them.
// ---------------------------------------------------------------------------
template <int TPR>
struct Team {
    static constexpr int PER_BLOCK = 256 / TPR;
    static __device__ __forceinline__ int lane() { return threadIdx.x % TPR; }
    static __device__ __forceinline__ int id() { return threadIdx.x / TPR; }
    // sums over the team, in every thread (red: 8 floats, for the block)
    static __device__ __forceinline__ void sum2(float &a, float &b, float *red) {
        a = lanes_sum<(TPR < 64 ? TPR : 64)>(a);
        b = lanes_sum<(TPR < 64 ? TPR : 64)>(b);
        if constexpr (TPR > 64) {
            __syncthreads();   // red may still be read
            if ((threadIdx.x & 63) == 0) {
                red[threadIdx.x >> 6] = a;
                red[4 + (threadIdx.x >> 6)] = b;
            }
            __syncthreads();
            a = (red[0] + red[1]) + (red[2] + red[3]);
            b = (red[4] + red[5]) + (red[6] + red[7]);
        }
    }
    static __device__ __forceinline__ float sum(float a, float *red) {
        float b = 0.f;
        if constexpr (TPR > 64) sum2(a, b, red);
        else a = lanes_sum<TPR>(a);
        return a;
    }
};

// A row of 8 elements per chunk, kept as it was read.
template <typename T> struct Raw8 { uint4 v[sizeof(T) / 2]; };
__device__ __forceinline__ void widen(const Raw8<uint16_t> &r, float (&v)[8]) {
    const uint32_t w[4] = {r.v[0].x, r.v[0].y, r.v[0].z, r.v[0].w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        v[2 * i] = __uint_as_float(w[i] << 16);
        v[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
    }
}
__device__ __forceinline__ void widen(const Raw8<float> &r, float (&v)[8]) {
    const uint32_t w[8] = {r.v[0].x, r.v[0].y, r.v[0].z, r.v[0].w, r.v[1].x, r.v[1].y, r.v[1].z, r.v[1].w};
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = __uint_as_float(w[i]);
}

template <typename T, int TPR, int CH>
struct RegRow {
    typedef float Vals[CH][8];
    int C, c0;   // channels, this thread's first
    __device__ __forceinline__ explicit RegRow(int channels) : C(channels), c0(Team<TPR>::lane() * 8) {}
    __device__ __forceinline__ int at(int i) const { return c0 + i * TPR * 8; }
    __device__ __forceinline__ bool in(int i) const { return at(i) < C; }
    // as it is read (widened where it is used; channels past C: 0)
    typedef Raw8<T> Raws[CH];
    __device__ __forceinline__ void fetch(const T *p, Raws &raw) const {
#pragma unroll
        for (int i = 0; i < CH; ++i) {
            raw[i] = Raw8<T>{};
            if (p != nullptr && in(i)) {
#pragma unroll
                for (int k = 0; k < (int)sizeof(T) / 2; ++k)
                    raw[i].v[k] = reinterpret_cast<const uint4 *>(p + at(i))[k];
            }
        }
    }
    // channels past C: other
    __device__ __forceinline__ void load(const T *p, Vals &v, float other) const {
#pragma unroll
        for (int i = 0; i < CH; ++i) {
            if (p != nullptr && in(i)) {
                load8(p + at(i), v[i]);
            } else {
#pragma unroll
                for (int e = 0; e < 8; ++e) v[i][e] = other;
            }
        }
    }
    __device__ __forceinline__ void store(T *p, const Vals &v) const {
#pragma unroll
        for (int i = 0; i < CH; ++i)
            if (in(i)) store8(p + at(i), v[i]);
    }
    // v -> (v - mean) rstd; values past C stay 0
    __device__ __forceinline__ float normalise(int kind, float eps, Vals &v, float *red) const {
        if (kind == 0) return 1.f;
        float mean = 0.f, s = 0.f;
        if (kind == NORM_LAYER) {
#pragma unroll
            for (int i = 0; i < CH; ++i)
#pragma unroll
                for (int e = 0; e < 8; ++e) s += v[i][e];
            mean = Team<TPR>::sum(s, red) / (float)C;
            s = 0.f;
        }
#pragma unroll
        for (int i = 0; i < CH; ++i)
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                if (kind == NORM_LAYER) v[i][e] = in(i) ? v[i][e] - mean : 0.f;
                s = fmaf(v[i][e], v[i][e], s);
            }
        const float rstd = 1.f / sqrtf(Team<TPR>::sum(s, red) / (float)C + eps);
#pragma unroll
        for (int i = 0; i < CH; ++i)
#pragma unroll
            for (int e = 0; e < 8; ++e) v[i][e] *= rstd;
        return rstd;
    }
};

// Bound by the rows' way through HBM: x, y, h and n once each.  (The vectors
// come from the caches.)
template <typename T, int TPR, int CH>
__global__ __launch_bounds__(256) void k_norm_gate(NormArgs a, T *h, T *n) {
    typedef RegRow<T, TPR, CH> Row;
    __shared__ float red[8];
    const long row = (long)folded_block() * Team<TPR>::PER_BLOCK + Team<TPR>::id();
    if (row >= a.rows) return;
    const Row r(a.C);
    const long at = row * a.C, mod = row / a.rows_per_mod * a.ld;
    // Rows and modulation on their way before the first sum (30000 x 1536: 69 us, 95 with each vector read where
    // it is used), the norms' weights and biases after it; but three chunks of fp32 would leave two waves to a
    // SIMD (230400 x 320: 227 against 217), there the modulation comes after it too.
    constexpr bool EARLY = sizeof(T) == 2 || CH <= 2;
    typename Row::Raws rx, ry, rg, rs, rt;
    r.fetch((const T *)a.x + at, rx);
    r.fetch(a.y != nullptr ? (const T *)a.y + at : nullptr, ry);
    auto vectors = [&]() {
        r.fetch(a.scale != nullptr ? (const T *)a.scale + mod : nullptr, rs);
        r.fetch(a.shift != nullptr ? (const T *)a.shift + mod : nullptr, rt);
    };
    if constexpr (EARLY) {
        r.fetch(a.gate != nullptr ? (const T *)a.gate + mod : nullptr, rg);
        vectors();
    }
    typename Row::Vals v, z, w, b;
#pragma unroll
    for (int i = 0; i < CH; ++i) widen(rx[i], v[i]);
    if (a.y != nullptr) {
#pragma unroll
        for (int i = 0; i < CH; ++i) widen(ry[i], z[i]);
        r.normalise(a.post, a.post_eps, z, red);
        if (a.post_w != nullptr || a.post_b != nullptr) {
            r.load((const T *)a.post_w, w, 1.f);
            r.load((const T *)a.post_b, b, 0.f);
#pragma unroll
            for (int i = 0; i < CH; ++i)
#pragma unroll
                for (int e = 0; e < 8; ++e) z[i][e] = r.in(i) ? fmaf(z[i][e], w[i][e], b[i][e]) : 0.f;
        }
        if constexpr (!EARLY) r.fetch(a.gate != nullptr ? (const T *)a.gate + mod : nullptr, rg);
#pragma unroll
        for (int i = 0; i < CH; ++i) {
            float g[8];
            widen(rg[i], g);
#pragma unroll
            for (int e = 0; e < 8; ++e) v[i][e] = fmaf(a.gate != nullptr ? g[e] : 1.f, z[i][e], a.res_scale * v[i][e]);
        }
        if (h != nullptr) r.store(h + at, v);
    }
    if (n == nullptr) return;
    r.normalise(a.pre, a.pre_eps, v, red);
    if (a.pre_w != nullptr || a.pre_b != nullptr) {
        r.load((const T *)a.pre_w, w, 1.f);
        r.load((const T *)a.pre_b, b, 0.f);
#pragma unroll
        for (int i = 0; i < CH; ++i)
#pragma unroll
            for (int e = 0; e < 8; ++e) v[i][e] = fmaf(v[i][e], w[i][e], b[i][e]);
    }
    if constexpr (!EARLY) vectors();
    // (scale and shift that are NULL are zeros)
#pragma unroll
    for (int i = 0; i < CH; ++i) {
        float s[8], t[8];
        widen(rs[i], s);
        widen(rt[i], t);
#pragma unroll
        for (int e = 0; e < 8; ++e) v[i][e] = fmaf(v[i][e], 1.f + s[e], t[e]);
    }
    r.store(n + at, v);
}

enum { Q_GATE, Q_SCALE, Q_SHIFT, Q_POSTW, Q_POSTB, Q_PREW, Q_PREB, N_Q };

// Work of the gradients: item i is rows of one modulation row, group
// i / per_group, split into per_group items.
struct GradItems {
    float *out[N_Q];        // results, or NULL
    float *slots;           // [3][n_items][C], per_group > 1
    float *sums;            // [4][blocks][C]
    int part, per_group, n_items;   // rows of an item
};

// The gradients of rows in registers.  What a row needs of the vectors of its
// modulation row are three products,
//   P = g w_post, Q = g b_post, R = (1 + s) w:   h = rs x + P v + Q, da w = R dn, dz w_post = P H,
// and all sums over rows follow from four,
//   A = sum dn u, B = sum dn, C = sum H v, D = sum H:
//   ds = w A + b B, dt = B, dw = (1 + s) A, db = (1 + s) B,
//   dg = w_post C + b_post D, dw_post = g C, db_post = g D,
// which takes 28 operations an element instead of 63 (at 64 lanes a clock and
// unit the vector pipes would bound it) and four sums in registers instead of
// seven.  x, y, dh and dn of a team's next row are on their way while it works
// on one.  Sums leave an item through LDS (the block's teams, in order); those
// of the norms' vectors are added up per block, and k_norm_grad_join adds the
// blocks, in order.
// ALONE: modulation rows of few rows each; a team takes a whole one, with P, Q
// and R in registers, and keeps the vectors' sums there.
template <typename T, int TPR, int CH, bool SUMS, bool ALONE>
__global__ __launch_bounds__(256) void k_norm_grad(NormArgs a, const T *dh, const T *dn, T *dx, T *dy, GradItems g) {
    typedef RegRow<T, TPR, CH> Row;
    typedef typename Row::Vals Vals;
    constexpr int TEAMS = Team<TPR>::PER_BLOCK, CP = TPR * CH * 8;
    extern __shared__ __align__(16) float lds[];   // P, Q, R [2][CP / 2] each (not ALONE); [sum][team][CP]
    float *const comb = lds + (ALONE ? 0 : 3 * CP);
    __shared__ float red[8];
    const Row r(a.C);
    const int team = Team<TPR>::id(), lane = Team<TPR>::lane();
    Vals sum[SUMS ? 4 : 1], vec[SUMS && ALONE ? 4 : 1], own[ALONE ? 3 : 1];
    auto clear = [&](Vals &v) {
#pragma unroll
        for (int i = 0; i < CH; ++i)
#pragma unroll
            for (int e = 0; e < 8; ++e) v[i][e] = 0.f;
    };
    if constexpr (SUMS) {
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            clear(sum[k]);
            if constexpr (ALONE) clear(vec[k]);
        }
    }
    // P, Q and R of eight channels
    auto products = [&](long mod, int c, float (&P)[8], float (&Q)[8], float (&R)[8]) {
        float gt[8], s[8];
        load8_or((const T *)a.post_w, c, 1.f, P);
        load8_or((const T *)a.post_b, c, 0.f, Q);
        load8_or((const T *)a.pre_w, c, 1.f, R);
        load8_or((const T *)a.gate, mod + c, 1.f, gt);
        load8_or((const T *)a.scale, mod + c, 0.f, s);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            P[e] *= gt[e];
            Q[e] *= gt[e];
            R[e] *= 1.f + s[e];
        }
    };
    // (the two halves of a chunk lie apart, so that lanes read consecutive 16 bytes)
    auto cst = [&](int k, int i, float (&v)[8]) {
        if constexpr (ALONE) {
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = own[k][i][e];
        } else {
            const float *at = lds + k * CP + (lane + i * TPR) * 4;
            *reinterpret_cast<f32x4 *>(v) = *reinterpret_cast<const f32x4 *>(at);
            *reinterpret_cast<f32x4 *>(v + 4) = *reinterpret_cast<const f32x4 *>(at + CP / 2);
        }
    };
    Raw8<T> rx[CH], ry[CH], rn[CH], rh[CH];
#pragma unroll
    for (int i = 0; i < CH; ++i) rx[i] = ry[i] = rn[i] = rh[i] = Raw8<T>{};
    auto fetch = [&](const T *p, long at, Raw8<T> (&raw)[CH]) {
        if (p == nullptr) return;
#pragma unroll
        for (int i = 0; i < CH; ++i)
            if (r.in(i)) {
#pragma unroll
                for (int k = 0; k < (int)sizeof(T) / 2; ++k)
                    raw[i].v[k] = reinterpret_cast<const uint4 *>(p + at + r.at(i))[k];
            }
    };
    const bool vecs = g.out[Q_POSTW] || g.out[Q_POSTB] || g.out[Q_PREW] || g.out[Q_PREB];
    const int first = ALONE ? (int)blockIdx.x * TEAMS + team : (int)blockIdx.x;
    const int items = (int)gridDim.x * (ALONE ? TEAMS : 1);
    constexpr int STEP = ALONE ? 1 : TEAMS;
    const float rs = a.y != nullptr ? a.res_scale : 1.f, per_c = 1.f / (float)a.C;
    for (int item = first; item < g.n_items; item += items) {
        const int group = item / g.per_group;
        const long start = (long)group * a.rows_per_mod + (long)(item - group * g.per_group) * g.part;
        const long stop = min(min(start + g.part, (long)(group + 1) * a.rows_per_mod), (long)a.rows);
        const long mod = group * a.ld;
        long row = start + (ALONE ? 0 : team);
        if (row < stop) {
            fetch((const T *)a.y, row * a.C, ry);
            fetch((const T *)a.x, row * a.C, rx);
            fetch(dn, row * a.C, rn);
            fetch(dh, row * a.C, rh);
        }
        if constexpr (ALONE) {
#pragma unroll
            for (int i = 0; i < CH; ++i)
                if (r.in(i)) products(mod, r.at(i), own[0][i], own[1][i], own[2][i]);
                else {
#pragma unroll
                    for (int e = 0; e < 8; ++e) own[0][i][e] = own[1][i][e] = own[2][i][e] = 0.f;
                }
        } else {
            __syncthreads();   // the last item's products may still be read
            for (int c8 = threadIdx.x; c8 < CP / 8; c8 += 256) {
                float v[3][8] = {};
                if (c8 * 8 < a.C) products(mod, c8 * 8, v[0], v[1], v[2]);
#pragma unroll
                for (int k = 0; k < 3; ++k) {
                    *reinterpret_cast<f32x4 *>(lds + k * CP + c8 * 4) = *reinterpret_cast<const f32x4 *>(v[k]);
                    *reinterpret_cast<f32x4 *>(lds + k * CP + CP / 2 + c8 * 4) = *reinterpret_cast<const f32x4 *>(v[k] + 4);
                }
            }
            __syncthreads();
        }
        while (row < stop) {
            const long at = row * a.C;
            Vals u, v, t;
#pragma unroll
            for (int i = 0; i < CH; ++i) {
                widen(ry[i], v[i]);
                widen(rx[i], u[i]);
            }
            row += STEP;
            const long next = row * a.C;
            if (row < stop) {
                fetch((const T *)a.y, next, ry);
                fetch((const T *)a.x, next, rx);
            }
            float r_y = 1.f;
            if (a.y != nullptr) {
                r_y = r.normalise(a.post, a.post_eps, v, red);
#pragma unroll
                for (int i = 0; i < CH; ++i) {
                    float P[8], Q[8];
                    cst(0, i, P);
                    cst(1, i, Q);
#pragma unroll
                    for (int e = 0; e < 8; ++e) u[i][e] = fmaf(v[i][e], P[e], fmaf(u[i][e], rs, Q[e]));
                }
            }
            const float r_h = r.normalise(a.pre, a.pre_eps, u, red);
            float s1 = 0.f, s2 = 0.f;
#pragma unroll
            for (int i = 0; i < CH; ++i) {
                float R[8];
                cst(2, i, R);
                widen(rn[i], t[i]);
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    if constexpr (SUMS) {
                        sum[0][i][e] = fmaf(t[i][e], u[i][e], sum[0][i][e]);
                        sum[1][i][e] += t[i][e];
                    }
                    t[i][e] *= R[e];
                    s1 += t[i][e];
                    s2 = fmaf(t[i][e], u[i][e], s2);
                }
            }
            if (!ALONE && row < stop) fetch(dn, next, rn);
            // (without a norm H does not hold u, which may be infinite)
            if (a.pre != 0) {
                Team<TPR>::sum2(s1, s2, red);
                const float m1 = a.pre == NORM_LAYER ? s1 * per_c : 0.f, m2 = s2 * per_c;
#pragma unroll
                for (int i = 0; i < CH; ++i)
#pragma unroll
                    for (int e = 0; e < 8; ++e) t[i][e] = fmaf(-u[i][e], m2, t[i][e] - m1);
            }
            // t becomes H
#pragma unroll
            for (int i = 0; i < CH; ++i) {
                float o[8];
                widen(rh[i], o);
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    t[i][e] = fmaf(r_h, t[i][e], o[e]);
                    o[e] = rs * t[i][e];
                }
                if (dx != nullptr && r.in(i)) store8(dx + at + r.at(i), o);
            }
            if (row < stop) {
                if (ALONE) fetch(dn, next, rn);   // (few next rows, many registers)
                fetch(dh, next, rh);
            }
            if (a.y == nullptr) continue;
            s1 = s2 = 0.f;
#pragma unroll
            for (int i = 0; i < CH; ++i) {
                float P[8];
                cst(0, i, P);   // (0 past C, where H is the mean's share only)
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    if constexpr (SUMS) {
                        sum[2][i][e] = fmaf(t[i][e], v[i][e], sum[2][i][e]);
                        sum[3][i][e] += t[i][e];
                    }
                    t[i][e] *= P[e];
                    s1 += t[i][e];
                    s2 = fmaf(t[i][e], v[i][e], s2);
                }
            }
            if (dy == nullptr) continue;
            if (a.post != 0) {
                Team<TPR>::sum2(s1, s2, red);
                const float k1 = a.post == NORM_LAYER ? s1 * per_c : 0.f, k2 = s2 * per_c;
#pragma unroll
                for (int i = 0; i < CH; ++i)
#pragma unroll
                    for (int e = 0; e < 8; ++e) t[i][e] = r_y * fmaf(-v[i][e], k2, t[i][e] - k1);
            }
            r.store(dy + at, t);
        }
        if constexpr (SUMS) {
            if (dn == nullptr) clear(sum[0]);   // (no gradient times a u that may not be finite)
            // the sums of N channels from c on, to the gradients that they make
            auto emit = [&](int c, auto width, const float *sa, const float *sb, const float *sc, const float *sd) {
                constexpr int N = decltype(width)::value;
                float pw[N], pb[N], w[N], b[N], gt[N], s1p[N], o[3][N];
                load_or<N>((const T *)a.post_w, c, 1.f, pw);
                load_or<N>((const T *)a.post_b, c, 0.f, pb);
                load_or<N>((const T *)a.pre_w, c, 1.f, w);
                load_or<N>((const T *)a.pre_b, c, 0.f, b);
                if (vecs) {
                    load_or<N>((const T *)a.gate, mod + c, 1.f, gt);
                    load_or<N>((const T *)a.scale, mod + c, 0.f, s1p);
                }
#pragma unroll
                for (int e = 0; e < N; ++e) {
                    o[0][e] = fmaf(pw[e], sc[e], pb[e] * sd[e]);
                    o[1][e] = fmaf(w[e], sa[e], b[e] * sb[e]);
                    o[2][e] = sb[e];
                }
#pragma unroll
                for (int k = 0; k < 3; ++k) {
                    if (g.out[k] == nullptr) continue;
                    float *const to =
                        (g.per_group == 1 ? g.out[k] + (long)group * a.C : g.slots + ((long)k * g.n_items + item) * a.C) + c;
#pragma unroll
                    for (int e = 0; e < N; e += 4) *reinterpret_cast<f32x4 *>(to + e) = *reinterpret_cast<f32x4 *>(&o[k][e]);
                }
                if (!vecs) return;
                // the norms' vectors: w_post, b_post, w, b
#pragma unroll
                for (int e = 0; e < N; ++e) s1p[e] += 1.f;
                if constexpr (ALONE) {
#pragma unroll
                    for (int i = 0; i < CH; ++i)
                        if (r.at(i) == c) {
#pragma unroll
                            for (int e = 0; e < N; ++e) {
                                vec[0][i][e] = fmaf(gt[e], sc[e], vec[0][i][e]);
                                vec[1][i][e] = fmaf(gt[e], sd[e], vec[1][i][e]);
                                vec[2][i][e] = fmaf(s1p[e], sa[e], vec[2][i][e]);
                                vec[3][i][e] = fmaf(s1p[e], sb[e], vec[3][i][e]);
                            }
                        }
                } else {
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        if (g.out[3 + k] == nullptr) continue;
                        const float *const m = k < 2 ? gt : s1p, *const of = k == 0 ? sc : k == 1 ? sd : k == 2 ? sa : sb;
                        float *const to = g.sums + ((long)k * gridDim.x + blockIdx.x) * a.C + c;
#pragma unroll
                        for (int e = 0; e < N; e += 4) {
                            f32x4 v = {m[e] * of[e], m[e + 1] * of[e + 1], m[e + 2] * of[e + 2], m[e + 3] * of[e + 3]};
                            if (item != first) v += *reinterpret_cast<const f32x4 *>(to + e);
                            *reinterpret_cast<f32x4 *>(to + e) = v;
                        }
                    }
                }
            };
            if constexpr (ALONE || TEAMS == 1) {
#pragma unroll
                for (int i = 0; i < CH; ++i)
                    if (r.in(i)) emit(r.at(i), std::integral_constant<int, 8>{}, sum[0][i], sum[1][i], sum[2][i], sum[3][i]);
            } else {
                // the teams' sums: this thread's channels, four at a time (CP is a multiple of 128)
#pragma unroll
                for (int k = 0; k < 4; ++k)
#pragma unroll
                    for (int i = 0; i < CH; ++i) store8(comb + (k * TEAMS + team) * CP + r.at(i), sum[k][i]);
                __syncthreads();
                for (int c = threadIdx.x * 4; c < a.C; c += 1024) {
                    f32x4 tot[4];
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        tot[k] = *reinterpret_cast<const f32x4 *>(comb + k * TEAMS * CP + c);
#pragma unroll 3
                        for (int o = 1; o < TEAMS; ++o)
                            tot[k] += *reinterpret_cast<const f32x4 *>(comb + (k * TEAMS + o) * CP + c);
                    }
                    emit(c, std::integral_constant<int, 4>{}, (const float *)&tot[0], (const float *)&tot[1],
                         (const float *)&tot[2], (const float *)&tot[3]);
                }
                // (the next item's sums are written behind its barriers)
            }
#pragma unroll
            for (int k = 0; k < 4; ++k) clear(sum[k]);
        }
    }
    if constexpr (SUMS && ALONE) {
        // the teams' sums of the norms' vectors
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            if (g.out[3 + k] == nullptr) continue;
            __syncthreads();
#pragma unroll
            for (int i = 0; i < CH; ++i) store8(comb + team * CP + r.at(i), vec[k][i]);
            __syncthreads();
            for (int c = threadIdx.x * 4; c < a.C; c += 1024) {
                f32x4 v = *reinterpret_cast<const f32x4 *>(comb + c);
#pragma unroll
                for (int o = 1; o < TEAMS; ++o) v += *reinterpret_cast<const f32x4 *>(comb + o * CP + c);
                *reinterpret_cast<f32x4 *>(g.sums + ((long)k * gridDim.x + blockIdx.x) * a.C + c) = v;
            }
        }
    }
}

// Adds items (group blockIdx.y) or blocks: 64 slices of them by 16 threads of
// four channels each, then the slices.
__global__ __launch_bounds__(1024) void k_norm_grad_join(int C, int blocks, GradItems g) {
    __shared__ f32x4 part[64][16];
    const int k = blockIdx.z, lane = threadIdx.x & 15, slice = threadIdx.x >> 4, c = blockIdx.x * 64 + lane * 4;
    const long group = blockIdx.y;
    const bool vec = k >= 3;
    if (g.out[k] == nullptr || (vec ? group > 0 : g.per_group == 1)) return;
    const int n = vec ? blocks : g.per_group;
    const float *src = vec ? g.sums + (long)(k - 3) * blocks * C : g.slots + ((long)k * g.n_items + group * n) * C;
    f32x4 s = {0.f, 0.f, 0.f, 0.f};
    if (c < C)
        for (int i = slice; i < n; i += 64) s += *reinterpret_cast<const f32x4 *>(src + (long)i * C + c);
    part[slice][lane] = s;
    __syncthreads();
    if (slice < 8) {
#pragma unroll
        for (int i = 8; i < 64; i += 8) s += part[slice + i][lane];
        part[slice][lane] = s;
    }
    __syncthreads();
    if (slice > 0 || c >= C) return;
#pragma unroll
    for (int i = 1; i < 8; ++i) s += part[i][lane];
    *reinterpret_cast<f32x4 *>(g.out[k] + (vec ? 0 : group * C) + c) = s;
}

// Rows too long for that: read again for every pass over them.
struct Stats { float mean, rstd; };

// One row, its chunks of 8 channels spread over the block.
template <typename T>
struct NormRow {
    const NormArgs &a;
    long at, mod;
    Stats sy, sh;
    __device__ __forceinline__ NormRow(const NormArgs &args, long row)
        : a(args), at(row * args.C), mod(row / args.rows_per_mod * args.ld), sy{0.f, 1.f}, sh{0.f, 1.f} {}
    // v = (y - mean) rstd and z
    __device__ __forceinline__ void post(int c, float (&v)[8], float (&z)[8]) const {
        float w[8], b[8];
        load8((const T *)a.y + at + c, v);
        load8_or((const T *)a.post_w, c, 1.f, w);
        load8_or((const T *)a.post_b, c, 0.f, b);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            v[i] = (v[i] - sy.mean) * sy.rstd;
            z[i] = fmaf(v[i], w[i], b[i]);
        }
    }
    __device__ __forceinline__ void stream(int c, float (&h)[8]) const {
        load8((const T *)a.x + at + c, h);
        if (a.y == nullptr) return;
        float v[8], z[8], g[8];
        post(c, v, z);
        load8_or((const T *)a.gate, mod + c, 1.f, g);
#pragma unroll
        for (int i = 0; i < 8; ++i) h[i] = fmaf(g[i], z[i], a.res_scale * h[i]);
    }
    // mean and 1/deviation of f(c, values) over the row
    template <typename F>
    __device__ __forceinline__ Stats stats(int kind, float eps, float *red, F f) const {
        Stats s{0.f, 1.f};
        if (kind == 0) return s;
        float v[8], sum = 0.f;
        if (kind == NORM_LAYER) {
            for (int c = threadIdx.x * 8; c < a.C; c += 2048) {
                f(c, v);
#pragma unroll
                for (int i = 0; i < 8; ++i) sum += v[i];
            }
            s.mean = block_sum(sum, red) / (float)a.C;
            sum = 0.f;
        }
        for (int c = threadIdx.x * 8; c < a.C; c += 2048) {
            f(c, v);
#pragma unroll
            for (int i = 0; i < 8; ++i) sum = fmaf(v[i] - s.mean, v[i] - s.mean, sum);
        }
        s.rstd = 1.f / sqrtf(block_sum(sum, red) / (float)a.C + eps);
        return s;
    }
    __device__ __forceinline__ void both_stats(float *red) {
        if (a.y != nullptr)
            sy = stats(a.post, a.post_eps, red, [&](int c, float (&v)[8]) { load8((const T *)a.y + at + c, v); });
        sh = stats(a.pre, a.pre_eps, red, [&](int c, float (&v)[8]) { stream(c, v); });
    }
};

template <typename T>
__global__ __launch_bounds__(256) void k_norm_gate_wide(NormArgs a, T *h, T *n) {
    __shared__ float red[4];
    const long row = folded_block();
    if (row >= a.rows) return;
    NormRow<T> r(a, row);
    r.both_stats(red);
    for (int c = threadIdx.x * 8; c < a.C; c += 2048) {
        float v[8];
        r.stream(c, v);
        if (h != nullptr) store8(h + r.at + c, v);
        if (n == nullptr) continue;
        float w[8], b[8], s[8], t[8];
        load8_or((const T *)a.pre_w, c, 1.f, w);
        load8_or((const T *)a.pre_b, c, 0.f, b);
        load8_or((const T *)a.scale, r.mod + c, 0.f, s);
        load8_or((const T *)a.shift, r.mod + c, 0.f, t);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float m = fmaf((v[i] - r.sh.mean) * r.sh.rstd, w[i], b[i]);
            v[i] = fmaf(m, 1.f + s[i], t[i]);
        }
        store8(n + r.at + c, v);
    }
}

// Statistics of a row that the column sums need again.
struct RowStats { Stats sy, sh; float m1, m2; };

// The gradient of a row's stream, element by element, once its means are known.
template <typename T>
struct GradRow : NormRow<T> {
    using NormRow<T>::a;
    using NormRow<T>::at;
    using NormRow<T>::mod;
    using NormRow<T>::sh;
    const T *dh, *dn;
    float m1 = 0.f, m2 = 0.f;
    __device__ __forceinline__ GradRow(const NormArgs &args, long row, const T *dh_, const T *dn_)
        : NormRow<T>(args, row), dh(dh_), dn(dn_) {}
    // u, the weighted u, and da
    __device__ __forceinline__ void inner(int c, float (&u)[8], float (&av)[8], float (&da)[8]) const {
        float w[8], b[8], s[8];
        this->stream(c, u);
        load8_or((const T *)a.pre_w, c, 1.f, w);
        load8_or((const T *)a.pre_b, c, 0.f, b);
        load8_or((const T *)a.scale, mod + c, 0.f, s);
        load8_or(dn, at + c, 0.f, da);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            u[i] = (u[i] - sh.mean) * sh.rstd;
            av[i] = fmaf(u[i], w[i], b[i]);
            da[i] *= 1.f + s[i];
        }
    }
    __device__ __forceinline__ void stream_grad(int c, float (&H)[8]) const {
        float u[8], av[8], da[8], w[8];
        inner(c, u, av, da);
        load8_or((const T *)a.pre_w, c, 1.f, w);
        load8_or(dh, at + c, 0.f, H);
        if (a.pre != 0) {
#pragma unroll
            for (int i = 0; i < 8; ++i) H[i] = fmaf(sh.rstd, fmaf(da[i], w[i], -m1) - u[i] * m2, H[i]);
        } else {   // (H does not hold u, which may be infinite)
#pragma unroll
            for (int i = 0; i < 8; ++i) H[i] = fmaf(sh.rstd, fmaf(da[i], w[i], -m1), H[i]);
        }
    }
};

template <typename T>
__global__ __launch_bounds__(256) void k_norm_grad_rows_wide(NormArgs a, const T *dh, const T *dn, T *dx, T *dy,
                                                        RowStats *rows) {
    __shared__ float red[4];
    const long row = folded_block();
    if (row >= a.rows) return;
    GradRow<T> r(a, row, dh, dn);
    r.both_stats(red);
    if (a.pre != 0 && dn != nullptr) {
        float s1 = 0.f, s2 = 0.f;
        for (int c = threadIdx.x * 8; c < a.C; c += 2048) {
            float u[8], av[8], da[8], w[8];
            r.inner(c, u, av, da);
            load8_or((const T *)a.pre_w, c, 1.f, w);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                s1 = fmaf(da[i], w[i], s1);
                s2 = fmaf(da[i] * w[i], u[i], s2);
            }
        }
        if (a.pre == NORM_LAYER) r.m1 = block_sum(s1, red) / (float)a.C;
        r.m2 = block_sum(s2, red) / (float)a.C;
    }
    if (threadIdx.x == 0) rows[row] = RowStats{r.sy, r.sh, r.m1, r.m2};
    // dz w_post, the gradient of the normalised y
    auto inner_y = [&](int c, float (&H)[8], float (&v)[8], float (&d)[8]) {
        float z[8], g[8], w[8];
        r.stream_grad(c, H);
        r.post(c, v, z);
        load8_or((const T *)a.gate, r.mod + c, 1.f, g);
        load8_or((const T *)a.post_w, c, 1.f, w);
#pragma unroll
        for (int i = 0; i < 8; ++i) d[i] = H[i] * g[i] * w[i];
    };
    float k1 = 0.f, k2 = 0.f, H[8], v[8], d[8];
    if (dy != nullptr && a.post != 0) {
        float s1 = 0.f, s2 = 0.f;
        for (int c = threadIdx.x * 8; c < a.C; c += 2048) {
            inner_y(c, H, v, d);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                s1 += d[i];
                s2 = fmaf(d[i], v[i], s2);
            }
        }
        if (a.post == NORM_LAYER) k1 = block_sum(s1, red) / (float)a.C;
        k2 = block_sum(s2, red) / (float)a.C;
    }
    for (int c = threadIdx.x * 8; c < a.C; c += 2048) {
        if (dy != nullptr) {
            inner_y(c, H, v, d);
            if (a.post != 0) {
#pragma unroll
                for (int i = 0; i < 8; ++i) d[i] = r.sy.rstd * (d[i] - k1 - v[i] * k2);
            }
            store8(dy + r.at + c, d);
        } else {
            r.stream_grad(c, H);
        }
        if (dx == nullptr) continue;
        if (a.y != nullptr) {
#pragma unroll
            for (int i = 0; i < 8; ++i) H[i] *= a.res_scale;
        }
        store8(dx + r.at + c, H);
    }
}

// The vectors' gradients.  Part p sums `part` rows; a part's modulation sums go
// out at every change of the modulation row: straight to the result where the
// part holds all of its rows, else to one of two slots of the part (0: a
// modulation row that an earlier part began, 1: one that this part begins).
struct ColOut {
    float *out[N_Q];        // results, or NULL
    float *slots;           // [3][n_parts][2][C]
    float *sums;            // [4][n_parts][C]
    int part, n_parts;
};

template <typename T>
__global__ __launch_bounds__(64) void k_norm_grad_cols_wide(NormArgs a, const T *dh, const T *dn, const RowStats *rows,
                                                       ColOut o) {
    const int c = (blockIdx.y * 64 + threadIdx.x) * 8, p = blockIdx.x;
    if (c >= a.C) return;
    const long r0 = (long)p * o.part, r1 = min(r0 + o.part, (long)a.rows);
    float q[N_Q][8] = {};
    for (long row = r0; row < r1; ++row) {
        GradRow<T> r(a, row, dh, dn);
        const RowStats st = rows[row];
        r.sy = st.sy;
        r.sh = st.sh;
        r.m1 = st.m1;
        r.m2 = st.m2;
        if (dn != nullptr) {
            float u[8], av[8], da[8], d[8];
            r.inner(c, u, av, da);
            load8(dn + r.at + c, d);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                q[Q_SCALE][i] = fmaf(d[i], av[i], q[Q_SCALE][i]);
                q[Q_SHIFT][i] += d[i];
                q[Q_PREW][i] = fmaf(da[i], u[i], q[Q_PREW][i]);
                q[Q_PREB][i] += da[i];
            }
        }
        if (a.y != nullptr) {
            float H[8], v[8], z[8], g[8];
            r.stream_grad(c, H);
            r.post(c, v, z);
            load8_or((const T *)a.gate, r.mod + c, 1.f, g);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                q[Q_GATE][i] = fmaf(H[i], z[i], q[Q_GATE][i]);
                q[Q_POSTW][i] = fmaf(H[i] * g[i], v[i], q[Q_POSTW][i]);
                q[Q_POSTB][i] = fmaf(H[i], g[i], q[Q_POSTB][i]);
            }
        }
        const long m = row / a.rows_per_mod, begin = m * a.rows_per_mod;
        const long end = min(begin + a.rows_per_mod, (long)a.rows);
        if (row + 1 == end || row + 1 == r1) {
#pragma unroll
            for (int k = 0; k < 3; ++k) {
                if (o.out[k] == nullptr) continue;
                float *to = begin >= r0 && end <= r1
                                ? o.out[k] + m * a.C
                                : o.slots + (((long)k * o.n_parts + p) * 2 + (begin >= r0 ? 1 : 0)) * a.C;
                store8(to + c, q[k]);
#pragma unroll
                for (int i = 0; i < 8; ++i) q[k][i] = 0.f;
            }
        }
    }
#pragma unroll
    for (int k = 3; k < N_Q; ++k)
        if (o.out[k] != nullptr) store8(o.sums + ((long)(k - 3) * o.n_parts + p) * a.C + c, q[k]);
}

// Joins the parts, in their order: block p > 0 the modulation row that is the
// first to cross the start of part p, block 0 the vectors of all rows.
__global__ __launch_bounds__(64) void k_norm_grad_join_wide(int C, int rows, int rows_per_mod, ColOut o) {
    const int c = blockIdx.y * 64 + threadIdx.x, k = blockIdx.z;
    if (c >= C || o.out[k] == nullptr || (k < 3) != (blockIdx.x > 0)) return;
    float s = 0.f;
    long m = 0;
    if (k < 3) {
        const long edge = (long)blockIdx.x * o.part, begin = edge / rows_per_mod * rows_per_mod;
        if (begin == edge || begin < edge - o.part) return;   // none crosses, or an earlier block joins it
        m = begin / rows_per_mod;
        const long end = min(begin + rows_per_mod, (long)rows);
        for (long p = blockIdx.x - 1; p <= (end - 1) / o.part; ++p)
            s += o.slots[(((long)k * o.n_parts + p) * 2 + (p * o.part <= begin ? 1 : 0)) * C + c];
    } else {
        for (long p = 0; p < o.n_parts; ++p) s += o.sums[((long)(k - 3) * o.n_parts + p) * C + c];
    }
    o.out[k][m * C + c] = s;
}

__global__ void k_zero(float *p, int n) {
    for (int i = blockIdx.x * blockDim.x + threadIdx.x; i < n; i += gridDim.x * blockDim.x) p[i] = 0.f;
}

}  // namespace

hipError_t launch_zero(float *p, int n, hipStream_t st) {
    launch_k(k_zero, std::min(cdiv(n, 256), 1024), 256, 0, st, p, n);
    return hipGetLastError();
}

// f(threads per row, chunks per thread) of a team as constants
template <typename F>
static hipError_t with_team(NormTeam t, F f) {
    using std::integral_constant;
    constexpr integral_constant<int, 16> quarter{};
    constexpr integral_constant<int, 32> half{};
    constexpr integral_constant<int, 64> wave{};
    constexpr integral_constant<int, 256> block{};
    constexpr integral_constant<int, 1> one{};
    constexpr integral_constant<int, 2> two{};
    constexpr integral_constant<int, 3> three{};
    constexpr integral_constant<int, 4> four{};
    switch (t.threads * 8 + t.chunks) {
        case 16 * 8 + 1: return f(quarter, one);
        case 16 * 8 + 2: return f(quarter, two);
        case 16 * 8 + 3: return f(quarter, three);
        case 32 * 8 + 2: return f(half, two);
        case 32 * 8 + 3: return f(half, three);
        case 64 * 8 + 2: return f(wave, two);
        case 64 * 8 + 3: return f(wave, three);
        case 64 * 8 + 4: return f(wave, four);
        case 256 * 8 + 1: return f(block, one);
        case 256 * 8 + 2: return f(block, two);
        case 256 * 8 + 4: return f(block, four);
        case 256 * 8: return f(block, integral_constant<int, 0>{});
        default: return hipErrorInvalidValue;
    }
}

template <typename T>
static hipError_t go_norm_gate(const NormArgs &a, T *h, T *n, hipStream_t st) {
    return with_team(norm_team(a.rows, a.C), [&](auto tpr, auto ch) -> hipError_t {
        constexpr int TPR = decltype(tpr)::value, CH = decltype(ch)::value;
        if constexpr (CH == 0)
            launch_k(k_norm_gate_wide<T>, folded_grid(a.rows, 256), 256, 0, st, a, h, n);
        else
            launch_k(k_norm_gate<T, TPR, CH>, folded_grid(((long)a.rows * TPR + 255) / 256, 256), 256, 0, st, a, h, n);
        return hipGetLastError();
    });
}

hipError_t launch_norm_gate(const NormArgs &a, void *h, void *n, hipStream_t st) {
    StageScope _stage(st, "norm_gate");
    return a.bf16 ? go_norm_gate(a, (uint16_t *)h, (uint16_t *)n, st) : go_norm_gate(a, (float *)h, (float *)n, st);
}

static_assert(sizeof(RowStats) == GRAD_ROW_STATS, "the plan's statistics");

size_t norm_grad_workspace_bytes(int rows, int C, int rows_per_mod, bool bf16) {
    if (rows <= 0) return 0;
    return grad_plan(rows, C, rows_per_mod > 0 ? rows_per_mod : rows, rows_per_mod > 0, true, bf16).bytes();
}

template <typename T, int TPR, int CH, bool SUMS, bool ALONE>
static hipError_t go_norm_grad(const NormArgs &a, const T *dh, const T *dn, T *dx, T *dy, const NormGrads &q,
                               const GradPlan &p, void *ws, hipStream_t st) {
    constexpr int TEAMS = Team<TPR>::PER_BLOCK, CP = TPR * CH * 8;
    GradItems g{{q.gate, q.scale, q.shift, q.post_w, q.post_b, q.pre_w, q.pre_b}, (float *)ws,
                (float *)((char *)ws + p.slots), p.part, p.per_group, p.n_items};
    const size_t lds = ((ALONE ? 0 : 3) + (!SUMS || TEAMS == 1 ? 0 : ALONE ? TEAMS : 4 * TEAMS)) * (size_t)CP * 4;
    const hipError_t e = raise_lds_limit((const void *)k_norm_grad<T, TPR, CH, SUMS, ALONE>, lds);
    if (e != hipSuccess) return e;
    launch_k(k_norm_grad<T, TPR, CH, SUMS, ALONE>, p.blocks, 256, lds, st, a, dh, dn, dx, dy, g);
    if (p.slots > 0 || p.sums > 0)
        launch_k(k_norm_grad_join,
                 dim3((unsigned)cdiv(a.C, 64), p.slots > 0 ? (unsigned)(p.n_items / p.per_group) : 1u, N_Q), 1024, 0, st,
                 a.C, p.blocks, g);
    return hipGetLastError();
}

template <typename T>
static hipError_t go_norm_grad_wide(const NormArgs &a, const T *dh, const T *dn, T *dx, T *dy, const NormGrads &q,
                                    const GradPlan &p, void *ws, hipStream_t st) {
    RowStats *rows = (RowStats *)ws;
    const ColOut o{{q.gate, q.scale, q.shift, q.post_w, q.post_b, q.pre_w, q.pre_b}, (float *)((char *)ws + p.stats),
                   (float *)((char *)ws + p.stats + p.slots), p.part, p.n_items};
    launch_k(k_norm_grad_rows_wide<T>, folded_grid(a.rows, 256), 256, 0, st, a, dh, dn, dx, dy, rows);
    if (p.slots == 0 && p.sums == 0) return hipGetLastError();
    launch_k(k_norm_grad_cols_wide<T>, dim3((unsigned)o.n_parts, (unsigned)cdiv(a.C, 512)), 64, 0, st, a, dh, dn, rows, o);
    launch_k(k_norm_grad_join_wide, dim3((unsigned)o.n_parts, (unsigned)cdiv(a.C, 64), N_Q), 64, 0, st, a.C, a.rows,
             a.rows_per_mod, o);
    return hipGetLastError();
}

template <typename T>
static hipError_t type_norm_grad(const NormArgs &a, const T *dh, const T *dn, T *dx, T *dy, const NormGrads &q,
                                 void *ws, hipStream_t st) {
    const bool mods = q.gate || q.scale || q.shift, vecs = q.post_w || q.post_b || q.pre_w || q.pre_b;
    const GradPlan p = grad_plan(a.rows, a.C, a.rows_per_mod, mods, vecs, a.bf16);
    return with_team(p.team, [&](auto tpr, auto ch) -> hipError_t {
        constexpr int TPR = decltype(tpr)::value, CH = decltype(ch)::value;
        if constexpr (CH == 0) {
            return go_norm_grad_wide(a, dh, dn, dx, dy, q, p, ws, st);
        } else {
            // (teams that the plan takes: 32 lanes with three chunks and 64 with four are the forward's)
            if constexpr ((TPR == 32 && CH == 3) || (TPR == 64 && CH == 4)) {
                return hipErrorInvalidValue;
            } else {
                if constexpr (TPR < 256) {
                    if (p.alone)
                        return mods || vecs ? go_norm_grad<T, TPR, CH, true, true>(a, dh, dn, dx, dy, q, p, ws, st)
                                            : go_norm_grad<T, TPR, CH, false, true>(a, dh, dn, dx, dy, q, p, ws, st);
                }
                return mods || vecs ? go_norm_grad<T, TPR, CH, true, false>(a, dh, dn, dx, dy, q, p, ws, st)
                                    : go_norm_grad<T, TPR, CH, false, false>(a, dh, dn, dx, dy, q, p, ws, st);
            }
        }
    });
}

hipError_t launch_norm_gate_grad(const NormArgs &args, const void *dh, const void *dn, void *dx, void *dy,
                                 const NormGrads &q, void *ws, hipStream_t st) {
    StageScope _stage(st, "norm_gate_grad");
    NormArgs a = args;
    if (dn == nullptr) {   // n takes no part: its norm is not made, whatever the rows hold
        a.pre = 0;
        a.pre_w = a.pre_b = a.scale = nullptr;
    }
    if (a.bf16)
        return type_norm_grad(a, (const uint16_t *)dh, (const uint16_t *)dn, (uint16_t *)dx, (uint16_t *)dy, q, ws, st);
    return type_norm_grad(a, (const float *)dh, (const float *)dn, (float *)dx, (float *)dy, q, ws, st);
}

}  // namespace oc
