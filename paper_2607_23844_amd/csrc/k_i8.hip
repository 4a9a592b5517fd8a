// Products in 8-bit integers: rows quantised with a scale each, and the product
// of two such matrices with a fused epilogue (scales, bias, GELU, rows written
// to their positions).
#include "oc_attn_common.h"
#include "oc_device.h"
#include "oc_gemm_epi.h"
#include "oc_i8_pick.h"
#include "oc_launch.h"
#include "oc_ops.h"
#include "oc_ring_tile.h"
#include <algorithm>

namespace oc {

namespace {

// ---------------------------------------------------------------------------
// Quantisation.  q = 127 x / m to the nearest whole number, ties to even, of the
// exact quotient (m = max|x|): with r = 1/m rounded, d = t r and one correction
// d + (t - d m) r by fused multiply-adds, a quotient that is exactly a tie
// comes out as it.  In fp32 for bf16 (t = 127 x has 15 bits; no quotient that
// is not a tie lies within 2^-17 of one), in 64 bits for fp32 (t has 31).
// ---------------------------------------------------------------------------
struct Quotient16 {
    float top, inv, mul;   // m and 127 times a power of two that keeps 1/m and 127 x in range
    __device__ __forceinline__ explicit Quotient16(float m) {
        const float f = m < 0x1p-60f ? 0x1p64f : m > 0x1p100f ? 0x1p-40f : 1.f;
        top = m * f;
        inv = 1.f / top;
        mul = 127.f * f;
    }
    __device__ __forceinline__ int operator()(float x) const {
        const float t = x * mul, d = t * inv;
        return (int)rintf(fmaf(fmaf(-d, top, t), inv, d));
    }
};
struct Quotient32 {
    double top, inv;
    __device__ __forceinline__ explicit Quotient32(float m) : top(m), inv(1.0 / (double)m) {}
    __device__ __forceinline__ int operator()(float x) const {
        const double t = 127.0 * (double)x, d = t * inv;
        return (int)rint(fma(fma(-d, top, t), inv, d));
    }
};
template <typename T> struct QuotientOf { typedef Quotient32 type; };
template <> struct QuotientOf<uint16_t> { typedef Quotient16 type; };

constexpr uint32_t INF_BITS = 0x7F800000u;   // magnitudes from here on: infinities and NaNs

// A row of 8 elements per chunk, kept as it was read.
template <typename T> struct Raw8 { uint4 v[sizeof(T) / 2]; };
template <typename T>
__device__ __forceinline__ Raw8<T> raw8(const T *p) {
    Raw8<T> r;
#pragma unroll
    for (int i = 0; i < (int)sizeof(T) / 2; ++i) r.v[i] = reinterpret_cast<const uint4 *>(p)[i];
    return r;
}
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

// A row by TPR threads (a wave, or the block of 256), read once: CH chunks of
// 8 elements per thread stay in registers between the maximum and the
// quotients.  CH = 0: rows too long for that, read twice.
template <typename T, int TPR, int CH>
__global__ __launch_bounds__(256) void k_quant(const T *__restrict__ x, long ld, int n_src, int K,
                                               const int32_t *__restrict__ idx, int rows, int8_t *__restrict__ q,
                                               float *__restrict__ scale) {
    constexpr int N = CH > 0 ? CH : 1;
    __shared__ uint32_t red[4];
    const int lane = threadIdx.x % TPR;
    const long row = (long)folded_block() * (256 / TPR) + threadIdx.x / TPR;
    if (row >= rows) return;
    const long src = idx != nullptr ? (long)idx[row] : row;
    if (src < 0 || src >= n_src) return;
    x += src * ld;
    uint32_t m = 0;
    auto widest = [&](const Raw8<T> &r) {
        float v[8];
        widen(r, v);
#pragma unroll
        for (int e = 0; e < 8; ++e) m = max(m, __float_as_uint(v[e]) & 0x7FFFFFFFu);
    };
    Raw8<T> keep[N];
    if constexpr (CH > 0) {
#pragma unroll
        for (int i = 0; i < CH; ++i) {
            const int k = (lane + i * TPR) * 8;
            if (k < K) keep[i] = raw8(x + k);
        }
#pragma unroll
        for (int i = 0; i < CH; ++i)
            if ((lane + i * TPR) * 8 < K) widest(keep[i]);
    } else {
        for (int k = lane * 8; k < K; k += TPR * 8) widest(raw8(x + k));
    }
    m = lanes_max(m);
    if constexpr (TPR > 64) {
        if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = m;
        __syncthreads();
        m = max(max(red[0], red[1]), max(red[2], red[3]));
    }
    const float top = __uint_as_float(m);
    if (lane == 0) scale[row] = m >= INF_BITS ? __uint_as_float(0x7FC00000u) : top / 127.f;
    const bool zero = m == 0 || m >= INF_BITS;
    const typename QuotientOf<T>::type quotient(zero ? 1.f : top);
    const int Kp = (K + 15) & ~15;
    q += row * Kp;
    auto write = [&](int k, const Raw8<T> &r) {
        float v[8];
        widen(r, v);
        uint32_t w[2] = {0, 0};
        if (!zero) {
#pragma unroll
            for (int e = 0; e < 8; ++e) w[e / 4] |= (uint32_t)(quotient(v[e]) & 0xFF) << (e % 4 * 8);
        }
        *reinterpret_cast<uint2 *>(q + k) = make_uint2(w[0], w[1]);
    };
    if constexpr (CH > 0) {
#pragma unroll
        for (int i = 0; i < CH; ++i) {
            const int k = (lane + i * TPR) * 8;
            if (k < K) write(k, keep[i]);
        }
    } else {
        for (int k = lane * 8; k < K; k += TPR * 8) write(k, raw8(x + k));
    }
    if (Kp > K && lane == 0) *reinterpret_cast<uint2 *>(q + K) = make_uint2(0, 0);   // (K is a multiple of 8)
}

template <typename T>
hipError_t go_quant(const T *x, long ld, int n_src, int K, const int *idx, int rows, int8_t *q, float *scale,
                    hipStream_t st) {
    auto go = [&](auto kern, int per_block) {
        launch_k(kern, folded_grid((rows + per_block - 1) / per_block, 256), 256, 0, st, x, ld, n_src, K, idx, rows, q,
                 scale);
        return hipGetLastError();
    };
    // A wave for a short row where there are rows for all units, else the block: bf16, K = 320, 100000 rows 24 us by
    // waves, 50 by blocks, K = 1536 79 and 100; 256 rows of 1536 3.7 and 3.2, of 320 3.1 and 3.2.  (Between 512 and
    // 2048 rows, in bf16 of K = 2048 up to 16000 and in fp32 from K = 1536 on the two are close or the block is ahead:
    // 1024 rows of 1536 3.9 and 3.7, 100000 of 2048 106 and 113, in fp32 188 and 167.)  Three chunks for K = 1536 take
    // as long as four (100000 rows 79.9 and 79.2); rows of up to 8192 are read once (16000 of them 69 us, read twice
    // 86, in fp32 122 and 168).
    const int c = cdiv(K, 8);
    if (c <= 256 && rows >= 2 * N_CUS) {
        if (c <= 64) return go(k_quant<T, 64, 1>, 4);
        return c <= 128 ? go(k_quant<T, 64, 2>, 4) : go(k_quant<T, 64, 4>, 4);
    }
    if (c <= 256) return go(k_quant<T, 256, 1>, 1);
    if (c <= 512) return go(k_quant<T, 256, 2>, 1);
    return c <= 1024 ? go(k_quant<T, 256, 4>, 1) : go(k_quant<T, 256, 0>, 1);
}

// GELU in its tanh form, v / (1 + exp(-2 z)), z = sqrt(2/pi) (v + 0.044715 v^3)
// (exp and reciprocal to 1 ulp)
__device__ __forceinline__ float gelu_tanh(float v) {
    constexpr double c = -2.0 * 1.4426950408889634 * 0.7978845608028654;   // -2 z log2(e) = c v + 0.044715 c v^3
    const float e = v * fmaf(v * v, (float)(c * 0.044715), (float)c);
    return v * __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(e));
}

// Scales and biases of four consecutive outputs, and these outputs of a row from
// their sums.
template <typename T>
__device__ __forceinline__ void columns4(const LinearI8Args &a, int n, f32x4 &sw, f32x4 &b) {
    sw = *reinterpret_cast<const f32x4 *>(a.sw + n);
    b = f32x4{0.f, 0.f, 0.f, 0.f};
    if (a.bias == nullptr) return;
    if constexpr (sizeof(T) == 2) {
        const u16x4 h = *reinterpret_cast<const u16x4 *>((const uint16_t *)a.bias + n);
#pragma unroll
        for (int e = 0; e < 4; ++e) b[e] = bf2f(h[e]);
    } else {
        b = *reinterpret_cast<const f32x4 *>((const float *)a.bias + n);
    }
}
__device__ __forceinline__ i32x4 four(const i32x16 &acc, int g) {
    return i32x4{acc[4 * g], acc[4 * g + 1], acc[4 * g + 2], acc[4 * g + 3]};
}
template <bool GELU>
__device__ __forceinline__ f32x4 finish4(i32x4 acc, float sq, f32x4 sw, f32x4 b) {
    f32x4 v;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        v[e] = fmaf((float)acc[e] * sq, sw[e], b[e]);
        if constexpr (GELU) v[e] = gelu_tanh(v[e]);
    }
    return v;
}
__device__ __forceinline__ u16x4 to_bf16(f32x4 v) {
    return __builtin_bit_cast(u16x4, __builtin_convertvector(v, bf16x4));
}

// Exchanges x of lanes 16..31 and 48..63 with y of lanes 0..15 and 32..47.
__device__ __forceinline__ void swap16(uint4 &x, uint4 &y) {
    const auto a = __builtin_amdgcn_permlane16_swap(x.x, y.x, false, false);
    const auto b = __builtin_amdgcn_permlane16_swap(x.y, y.y, false, false);
    const auto c = __builtin_amdgcn_permlane16_swap(x.z, y.z, false, false);
    const auto d = __builtin_amdgcn_permlane16_swap(x.w, y.w, false, false);
    x = make_uint4(a[0], b[0], c[0], d[0]);
    y = make_uint4(a[1], b[1], c[1], d[1]);
}

// Between a wave's writes and reads of LDS that no other wave touches.
__device__ __forceinline__ void wave_lds_fence() {
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
}

// y row of batch row r, or -1
__device__ __forceinline__ long out_row(const LinearI8Args &a, long r) {
    if (r >= a.rows) return -1;
    const long t = a.out_idx != nullptr ? (long)a.out_idx[r] : r;
    return t >= 0 && t < a.n_out ? t : -1;
}

// ---------------------------------------------------------------------------
// The product on ring-buffered MFMA tiles: a = weight rows, b = batch rows.  A
// lane of an accumulator of 32 x 32 has four outputs of one row in each of four
// groups.  bf16: lanes exchange them (v_permlane32_swap, v_permlane16_swap) until
// each stores 16 bytes of a row beside its partners', and waves finish one by
// one; through LDS in whole rows, after a barrier, it took 73 us (now 63) for
// 230400 x 320 x 320, 252 (246) x 1280, 330 (296) with GELU, 11.2 (10.0) for 2048
// x 1536 x 1536 and 61 (57) for 4429 x 1536 x 6144 with GELU.  fp32: through LDS
// wave by wave.
// ---------------------------------------------------------------------------
// LDS: the ring, or in its place scales and biases of the outputs, scales and
// places of the rows, and the waves' parts for fp32
constexpr int F32_LD = 36;
template <typename R>
constexpr size_t LIN_LDS = std::max<size_t>(R::RING_BYTES, (R::BA + R::BB) * 8 + R::NW * 32 * F32_LD * 4);

template <int ID, typename T, bool GELU>
__global__ __launch_bounds__(RING_THREADS<ID>) void k_linear_i8(LinearI8Args a, int n_at, int n_bt) {
    using R = typename RingShape<ID, RING_I8>::Tile;
    constexpr int BA = R::BA, BB = R::BB;
    static_assert(BA <= R::NT && BB <= R::NT && LIN_LDS<R> <= 160 * 1024, "a thread for each row and output; LDS");
    extern __shared__ __align__(16) uint16_t lds[];
    int at, bt;
    tile_order(xcd_remap(blockIdx.x, n_at * n_bt), n_at, n_bt, at, bt);
    const int a0 = at * BA, b0 = bt * BB;
    const int K2 = (a.K + 15) / 16 * 8;   // pairs of elements in a row
    // what the epilogue needs of one output and one row, loaded ahead of the operands
    const int mine_a = min(a0 + (int)threadIdx.x, a.N - 1), mine_b = min(b0 + (int)threadIdx.x, a.rows - 1);
    float my_sw = 0.f, my_bias = 0.f, my_sq = 0.f;
    int my_out = 0;
    if ((int)threadIdx.x < BA) {
        my_sw = a.sw[mine_a];
        if (a.bias != nullptr) my_bias = Elem<T>::ld((const T *)a.bias + mine_a);
    }
    if ((int)threadIdx.x < BB) {
        my_sq = a.sq[mine_b];
        my_out = a.out_idx != nullptr ? a.out_idx[mine_b] : mine_b;
    }
    typename R::RowsA ra;
    typename R::RowsB rb;
    ring_rows(ra, (const uint16_t *)a.w, a.N, K2, a0);
    ring_rows(rb, (const uint16_t *)a.q, a.rows, K2, b0);
    R t;
    t.run(lds, ra, rb, K2);
    // (in the ring, free now)
    float *const col_sw = reinterpret_cast<float *>(lds), *const col_b = col_sw + BA;
    float *const row_sq = col_b + BA;
    int *const row_out = reinterpret_cast<int *>(row_sq + BB);   // y row, or -1
    if ((int)threadIdx.x < BA) {
        col_sw[threadIdx.x] = my_sw;
        col_b[threadIdx.x] = my_bias;
    }
    if ((int)threadIdx.x < BB) {
        row_sq[threadIdx.x] = my_sq;
        row_out[threadIdx.x] = b0 + (int)threadIdx.x < a.rows && my_out >= 0 && my_out < a.n_out ? my_out : -1;
    }
    __syncthreads();
    const int lane = threadIdx.x & 63;
    float sq[R::TB];
#pragma unroll
    for (int j = 0; j < R::TB; ++j) sq[j] = row_sq[R::b_of(j)];
    if constexpr (sizeof(T) == 2) {
        // 32 bytes of a row together with GELU, whose stores come further apart, 64 without (230400 x 320 x
        // 1280: 300 us against 310, 258 against 272)
        constexpr int ROWS = GELU ? 1 : 2;   // rows that a lane stores of an accumulator
#pragma unroll
        for (int j = 0; j < R::TB; ++j) {
            uint16_t *to[ROWS];
#pragma unroll
            for (int h = 0; h < ROWS; ++h) {
                const int o = row_out[(R::b_of(j) & ~31) + (lane & (32 / ROWS - 1)) + h * (32 / ROWS)];
                to[h] = o >= 0 ? (uint16_t *)a.y + o * a.ld_y : nullptr;
            }
            auto store = [&](int h, int n, uint4 v) {
                if (to[h] != nullptr && n < a.N) *reinterpret_cast<uint4 *>(to[h] + n) = v;
            };
#pragma unroll
            for (int i = 0; i < R::TA; ++i) {
                auto group = [&](int g) {
                    const int c = R::a_of(i, g);
                    return __builtin_bit_cast(
                        uint2, to_bf16(finish4<GELU>(four(t.acc[i][j], g), sq[j], *reinterpret_cast<const f32x4 *>(col_sw + c),
                                                     *reinterpret_cast<const f32x4 *>(col_b + c))));
                };
                uint4 v[2];
#pragma unroll
                for (int h = 0; h < 2; ++h) {   // outputs 0..7 | 8..15 in the halves of the wave, and 16 further
                    const uint2 x = group(2 * h), y = group(2 * h + 1);
                    const auto p = __builtin_amdgcn_permlane32_swap(x.x, y.x, false, false);
                    const auto q = __builtin_amdgcn_permlane32_swap(x.y, y.y, false, false);
                    v[h] = make_uint4(p[0], q[0], p[1], q[1]);
                }
                const int n = a0 + (R::a_of(i, 0) & ~31) + (lane & 32) / 4;
                if constexpr (ROWS == 2) {
                    swap16(v[0], v[1]);
                    store(0, n + (lane & 16), v[0]);
                    store(1, n + (lane & 16), v[1]);
                } else {
                    store(0, n, v[0]);
                    store(0, n + 16, v[1]);
                }
            }
        }
    } else {
        // 32 rows of 32 outputs at a time through a part of LDS of the wave's own: 128 bytes of a row
        // are stored together (each lane storing its four outputs took 80 us for 4429 x 1536 x 6144; 128 bytes
        // exchanged between lanes as above 59, this 56: there the neighbours of a store are lanes apart)
        float *const mine = reinterpret_cast<float *>(row_out + BB) + (threadIdx.x >> 6) * 32 * F32_LD;
#pragma unroll
        for (int i = 0; i < R::TA; ++i) {
            const int n = a0 + (R::a_of(i, 0) & ~31) + (lane & 7) * 4;   // outputs that this lane stores
#pragma unroll
            for (int j = 0; j < R::TB; ++j) {
#pragma unroll
                for (int g = 0; g < 4; ++g) {
                    const int c = R::a_of(i, g);
                    *reinterpret_cast<f32x4 *>(mine + (lane & 31) * F32_LD + 8 * g + 4 * (lane >> 5)) =
                        finish4<GELU>(four(t.acc[i][j], g), sq[j], *reinterpret_cast<const f32x4 *>(col_sw + c),
                                      *reinterpret_cast<const f32x4 *>(col_b + c));
                }
                wave_lds_fence();
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const int r = k * 8 + (lane >> 3);
                    const f32x4 v = *reinterpret_cast<const f32x4 *>(mine + r * F32_LD + (lane & 7) * 4);
                    const int o = row_out[(R::b_of(j) & ~31) + r];
                    if (o >= 0 && n < a.N) *reinterpret_cast<f32x4 *>((T *)a.y + o * a.ld_y + n) = v;
                }
                wave_lds_fence();
            }
        }
    }
}

// ---------------------------------------------------------------------------
// The product of few rows: bound by the weights' way from HBM, so a block takes
// 16 weight rows (or OUT = 8, half of an MFMA's) and all its waves share out
// their K (the ring's tiles would be N / 64 blocks of one after another 128
// bytes).  v_mfma_i32_16x16x64_i8, a = weights, b = up to 16 RT batch rows, four
// of them from one round of loads.  The waves' sums are added in LDS (integers:
// in any order).
// ---------------------------------------------------------------------------
template <typename T, int RT, int OUT>
__global__ __launch_bounds__(1024) void k_linear_i8_thin(LinearI8Args a) {
    extern __shared__ __align__(16) int part[];   // [wave][RT][16 batch rows][16 + 4 outputs]
    constexpr int LD = 20;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, nw = blockDim.x >> 6;
    const int lr = lane & 15, lg = lane >> 4, n0 = blockIdx.x * OUT;
    const int Kp = (a.K + 15) & ~15;
    const int8_t *w = a.w + (long)min(n0 + lr, a.N - 1) * Kp;
    const int8_t *q[RT];
    i32x4 acc[RT];
    const i32x4 zero = {0, 0, 0, 0};
#pragma unroll
    for (int t = 0; t < RT; ++t) {
        q[t] = a.q + (long)min(t * 16 + lr, a.rows - 1) * Kp;
        acc[t] = zero;
    }
    for (int k0 = wave * 256; k0 < Kp; k0 += nw * 256) {
        i32x4 fw[4], fq[RT][4];
#pragma unroll
        for (int s = 0; s < 4; ++s) {
            const int k = k0 + s * 64 + lg * 16;
            fw[s] = k < Kp && (OUT == 16 || lr < OUT) ? *reinterpret_cast<const i32x4 *>(w + k) : zero;
#pragma unroll
            for (int t = 0; t < RT; ++t) fq[t][s] = k < Kp ? *reinterpret_cast<const i32x4 *>(q[t] + k) : zero;
        }
#pragma unroll
        for (int s = 0; s < 4; ++s)
#pragma unroll
            for (int t = 0; t < RT; ++t)
                acc[t] = __builtin_amdgcn_mfma_i32_16x16x64_i8(fw[s], fq[t][s], acc[t], 0, 0, 0);
    }
    // lane: batch row lr, outputs 4 lg .. 4 lg + 3
#pragma unroll
    for (int t = 0; t < RT; ++t)
        *reinterpret_cast<i32x4 *>(part + ((wave * RT + t) * 16 + lr) * LD + lg * 4) = acc[t];
    __syncthreads();
    for (int i = threadIdx.x; i < RT * 4 * OUT; i += blockDim.x) {
        const int r = i / (OUT / 4), n = i % (OUT / 4) * 4;
        const long o = out_row(a, r);
        if (o < 0 || n0 + n >= a.N) continue;
        i32x4 s = zero;
        for (int v = 0; v < nw; ++v) s += *reinterpret_cast<const i32x4 *>(part + (v * RT * 16 + r) * LD + n);
        f32x4 sw, bias;
        columns4<T>(a, n0 + n, sw, bias);
        const f32x4 f = a.gelu ? finish4<true>(s, a.sq[r], sw, bias) : finish4<false>(s, a.sq[r], sw, bias);
        T *const to = (T *)a.y + o * a.ld_y + n0 + n;
        if constexpr (sizeof(T) == 2) *reinterpret_cast<u16x4 *>(to) = to_bf16(f);
        else *reinterpret_cast<f32x4 *>(to) = f;
    }
}

template <typename T, int RT, int OUT>
hipError_t go_thin_out(const LinearI8Args &a, hipStream_t st) {
    // waves: one pass of 256 bytes of k each, or as few as 16 waves need
    const int blocks = cdiv(a.N, OUT), passes = cdiv(a.K, 256), nw = cdiv(passes, cdiv(passes, 16));
    const size_t lds = (size_t)nw * RT * 16 * 20 * 4;
    const hipError_t e = raise_lds_limit((const void *)k_linear_i8_thin<T, RT, OUT>, lds);
    if (e != hipSuccess) return e;
    launch_k(k_linear_i8_thin<T, RT, OUT>, (unsigned)blocks, nw * 64, lds, st, a);
    return hipGetLastError();
}

template <typename T, int RT>
hipError_t go_thin(const LinearI8Args &a, hipStream_t st) {
    // Eight outputs a block where these are no more blocks than units and rows are long: what bounds a block
    // is then its own weights' way (one row of K = 6144, N = 1536 5.6 us against 6.6, 32 rows 10.4 against
    // 11.2, K = 1536 3.8 against 3.9; past that the rows' second reading costs more, N = 3200 4.5 against 4.1,
    // and with K = 320 2.6 against 2.5).
    return a.N <= 8 * N_CUS && a.K >= 1024 ? go_thin_out<T, RT, 8>(a, st) : go_thin_out<T, RT, 16>(a, st);
}

template <typename T, bool GELU>
hipError_t go_ring(const LinearI8Args &a, hipStream_t st) {
    return ring_dispatch(i8_pick(a.rows, a.K, a.N), [&](auto c) -> hipError_t {
        constexpr int ID = decltype(c)::value;
        using R = typename RingShape<ID, RING_I8>::Tile;
        const hipError_t e = allow_lds(k_linear_i8<ID, T, GELU>, LIN_LDS<R>);
        if (e != hipSuccess) return e;
        const int n_at = cdiv(a.N, R::BA), n_bt = cdiv(a.rows, R::BB);
        launch_k(k_linear_i8<ID, T, GELU>, (unsigned)(n_at * n_bt), R::NT, LIN_LDS<R>, st, a, n_at, n_bt);
        return hipGetLastError();
    });
}

template <typename T>
hipError_t go_linear(const LinearI8Args &a, hipStream_t st) {
    // Up to 16 rows: 3.8 us against the ring's 6.3 for one row of K = N = 1536, 6.3 against 7.8 at N =
    // 9216.  Up to 32 while the ring's tiles of 64 outputs are few: 32 rows, K = 1536, N = 1536 5.1
    // against 6.4, N = 4608 7.3 against 6.5 (every block reads all rows from L2).
    if (a.rows <= 16) return go_thin<T, 1>(a, st);
    if (a.rows <= 32 && a.N <= 4096) return go_thin<T, 2>(a, st);
    return a.gelu ? go_ring<T, true>(a, st) : go_ring<T, false>(a, st);
}

}  // namespace

hipError_t launch_quant(bool bf16, const void *x, long ld, int n_src, int K, const int *idx, int rows, int8_t *q,
                        float *scale, hipStream_t st) {
    StageScope _stage(st, "quant_rows");
    return bf16 ? go_quant((const uint16_t *)x, ld, n_src, K, idx, rows, q, scale, st)
                : go_quant((const float *)x, ld, n_src, K, idx, rows, q, scale, st);
}

hipError_t launch_linear_i8(const LinearI8Args &a, hipStream_t st) {
    StageScope _stage(st, "linear_i8");
    return a.bf16 ? go_linear<uint16_t>(a, st) : go_linear<float>(a, st);
}

}  // namespace oc
