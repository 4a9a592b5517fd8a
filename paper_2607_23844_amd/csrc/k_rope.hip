// Rotary positions of q and k rows with up to three axes.
//
// A block turns `rows` rows.  First the cosines and sines of its rows' pairs, one
// per thread, into LDS (oc_rope.h).  Then all heads of q and k of those rows, in
// units of 8 neighbouring channels (pairs side by side) or of V channels and
// their V partners half a section further; consecutive threads take consecutive
// units, four of them loaded at a time.  Bound by q's and k's way through HBM.
#include "oc_attn_common.h"
#include "oc_device.h"
#include "oc_launch.h"
#include "oc_rope.h"
#include <cmath>
#include <cstring>

namespace oc {

namespace {

template <typename T, int V> struct Chunk { typedef T type __attribute__((ext_vector_type(V))); };

template <typename T, int V>
__device__ __forceinline__ void get(const T *p, float (&v)[V]) {
    typedef typename Chunk<T, V>::type C;
    const C c = *reinterpret_cast<const C *>(p);
#pragma unroll
    for (int i = 0; i < V; ++i) v[i] = (float)c[i];
}
template <typename T, int V>
__device__ __forceinline__ void put(T *p, const float (&v)[V]) {
    typedef typename Chunk<T, V>::type C;
    C c;
#pragma unroll
    for (int i = 0; i < V; ++i) c[i] = turned<T>(v[i]);
    *reinterpret_cast<C *>(p) = c;
}

constexpr int ROPE_ROWS = 16;   // most rows of a block

// Positions and turns of a block's rows, by all of its 256 threads.
__device__ __forceinline__ void make_turns(const RopeGeom &g, const RopeArgs &a, long row0, int rows,
                                           int (*where)[4], Turn *turns) {
    if ((int)threadIdx.x < rows) {
        const long row = row0 + threadIdx.x;
        int *const w = where[threadIdx.x];
        if (a.pos != nullptr) {
#pragma unroll
            for (int i = 0; i < 3; ++i) w[i] = a.pos[row * 3 + i];
            w[3] = 1;
        } else {
            const int4 at = rope_place(g, batch_token((int)row, a.idx, a.tF, a.tN));
            w[0] = at.x;
            w[1] = at.y;
            w[2] = at.z;
            w[3] = at.w;
        }
    }
    __syncthreads();
    for (int e = threadIdx.x; e < rows * g.P; e += 256) {
        const int r = e / g.P, p = e - r * g.P, axis = rope_axis(g, p);
        const Turn t = rope_turn(rope_fraction(where[r][axis], g.origin[axis], g.turn[p]));
        turns[r * ROPE_MAX_PAIRS + p] = Turn{t.c, a.inverse ? -t.s : t.s};
    }
    __syncthreads();
}

// PAIRS: unit u is channels 8u..8u+7 (V = 4 pairs); else channels lo.. and hi.. of V pairs
template <typename T, bool PAIRS, int V>
__global__ __launch_bounds__(256) void k_rope(RopeGeom g, RopeArgs a, int block_rows) {
    __shared__ __align__(16) Turn turns[ROPE_ROWS * ROPE_MAX_PAIRS];
    __shared__ int where[ROPE_ROWS][4];   // position on the axes; whether there is one
    const long row0 = (long)folded_block() * block_rows;
    if (row0 >= a.rows) return;
    const int rows = (int)min((long)block_rows, a.rows - row0);
    make_turns(g, a, row0, rows, where, turns);
    const int units = g.dh / 2 / V, q_units = a.q != nullptr ? a.heads * units : 0;
    const int row_units = q_units + (a.k != nullptr ? a.k_heads * units : 0);
    constexpr int N = 4, W = PAIRS ? 8 : V;   // units at a time; channels of a run
    for (int i0 = threadIdx.x; i0 < rows * row_units; i0 += 256 * N) {
        float v[N][W], w[PAIRS ? 1 : N][W];
        T *to[N];
        int first[N], gap[N], of[N];
#pragma unroll
        for (int b = 0; b < N; ++b) {
            const int i = i0 + b * 256, r = i / row_units;
            to[b] = nullptr;
            if (i >= rows * row_units || !where[r][3]) continue;
            int j = i - r * row_units;
            const bool k = j >= q_units;
            if (k) j -= q_units;
            const int h = j / units, p0 = (j - h * units) * V;
            const long row = row0 + r;
            const T *src = k ? (const T *)a.k + row * a.ld_k : (const T *)a.q + row * a.ld_q;
            to[b] = k ? (T *)a.ko + row * a.ld_ko : (T *)a.qo + row * a.ld_qo;
            int lo = 2 * p0;
            if constexpr (!PAIRS) {
                int s0 = 0, s1 = 0;
#pragma unroll
                for (int m = 0; m < 4; ++m)
                    if (p0 >= g.sect[m] && p0 < g.sect[m + 1]) {
                        s0 = g.sect[m];
                        s1 = g.sect[m + 1];
                    }
                lo = s0 + p0;
                gap[b] = s1 - s0;
            }
            src += h * g.dh + lo;
            to[b] += h * g.dh + lo;
            first[b] = p0;
            of[b] = r * ROPE_MAX_PAIRS;
            get<T, W>(src, v[b]);
            if constexpr (!PAIRS) get<T, W>(src + gap[b], w[b]);
        }
#pragma unroll
        for (int b = 0; b < N; ++b) {
            if (to[b] == nullptr) continue;
#pragma unroll
            for (int j = 0; j < V; ++j) {
                if (first[b] + j >= g.P) break;   // (not turned)
                const Turn t = turns[of[b] + first[b] + j];
                turn_pair(PAIRS ? v[b][2 * j] : v[b][j], PAIRS ? v[b][2 * j + 1] : w[PAIRS ? 0 : b][j], t);
            }
            put<T, W>(to[b], v[b]);
            if constexpr (!PAIRS) put<T, W>(to[b] + gap[b], w[b]);
        }
    }
}

// Halves whose sections fit no run of four channels: heads pass through LDS,
// read and written in 16-byte chunks, and a wave turns a head there, one pair
// per lane (access by single channels took 39 us for 4096 rows of 2 x 12 heads
// of 128).
constexpr int ROPE_LDS = 8192;   // channels at a time
template <typename T>
__global__ __launch_bounds__(256) void k_rope_lds(RopeGeom g, RopeArgs a, int block_rows) {
    __shared__ __align__(16) Turn turns[ROPE_ROWS * ROPE_MAX_PAIRS];
    __shared__ int where[ROPE_ROWS][4];
    __shared__ __align__(16) T data[ROPE_LDS];
    const long row0 = (long)folded_block() * block_rows;
    if (row0 >= a.rows) return;
    const int rows = (int)min((long)block_rows, a.rows - row0);
    make_turns(g, a, row0, rows, where, turns);
    const int q_heads = a.q != nullptr ? a.heads : 0, heads = q_heads + (a.k != nullptr ? a.k_heads : 0);
    const int total = rows * heads, most = ROPE_LDS / g.dh, cpr = g.dh / 8;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int lo, hi;   // this lane's pair
    rope_channels(g, lane, lo, hi);
    // chunk c of heads h0, h0 + 1, ... of the block's rows (nullptr: a row without a position)
    auto chunk = [&](int h0, int c, const void *q, const void *k, long ld_q, long ld_k) -> T * {
        const int s = h0 + c / cpr, r = s / heads;
        int h = s - r * heads;
        if (!where[r][3]) return nullptr;
        const bool is_k = h >= q_heads;
        if (is_k) h -= q_heads;
        return (T *)(is_k ? k : q) + (row0 + r) * (is_k ? ld_k : ld_q) + h * g.dh + (c % cpr) * 8;
    };
    typedef typename Chunk<T, 8>::type C8;
    for (int h0 = 0; h0 < total; h0 += most) {
        const int n = min(most, total - h0);
        for (int c = threadIdx.x; c < n * cpr; c += 256) {
            const T *p = chunk(h0, c, a.q, a.k, a.ld_q, a.ld_k);
            if (p != nullptr) *reinterpret_cast<C8 *>(data + c * 8) = *reinterpret_cast<const C8 *>(p);
        }
        __syncthreads();
        if (lane < g.P) {
            for (int s = wave; s < n; s += 4) {
                const Turn t = turns[(h0 + s) / heads * ROPE_MAX_PAIRS + lane];
                T &x = data[s * g.dh + lo], &y = data[s * g.dh + hi];
                float u = (float)x, v = (float)y;
                turn_pair(u, v, t);
                x = turned<T>(u);
                y = turned<T>(v);
            }
        }
        __syncthreads();
        for (int c = threadIdx.x; c < n * cpr; c += 256) {
            T *p = chunk(h0, c, a.qo, a.ko, a.ld_qo, a.ld_ko);
            if (p != nullptr) *reinterpret_cast<C8 *>(p) = *reinterpret_cast<const C8 *>(data + c * 8);
        }
        __syncthreads();
    }
}

template <typename T>
hipError_t type_rope(const RopeGeom &g, const RopeArgs &a, hipStream_t st) {
    // rows of a block: all that leave two blocks for every unit, since few units of a row leave threads idle (bf16,
    // 230400 rows of 2 x 5 heads of 64 111 us by 16 rows, 136 by four, 274 by one; 57600 rows 30, 35 and 68).  Rows of
    // many heads fill a block by themselves and would do with fewer (2 x 24 heads, 2048 rows 9.9 us by four, 8.5 by
    // one; 4096 rows 15.2 by eight, 11.9 by two).
    int rows = 1;
    while (rows < ROPE_ROWS && a.rows / (2 * rows) >= 2 * N_CUS) rows *= 2;
    auto go = [&](auto kern) {
        launch_k(kern, folded_grid((a.rows + rows - 1) / rows, 256), 256, 0, st, g, a, rows);
        return hipGetLastError();
    };
    if (g.pairs) return go(k_rope<T, true, 4>);
    return g.vec == 8 ? go(k_rope<T, false, 8>) : g.vec == 4 ? go(k_rope<T, false, 4>) : go(k_rope_lds<T>);
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
