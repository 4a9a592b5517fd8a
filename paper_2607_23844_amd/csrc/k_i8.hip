// Products in 8-bit integers: rows quantised with a scale each, and the product
// of two such matrices with a fused epilogue (scales, bias, GELU, rows written
// to their positions).
#include "oc_attn_common.h"
#include "oc_device.h"
#include "oc_gemm_epi.h"
#include "oc_launch.h"
#include "oc_ops.h"
#include "oc_ring_tile.h"

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

template <typename T>
__global__ __launch_bounds__(256) void k_quant(const T *__restrict__ x, long ld, int n_src, int K,
                                               const int32_t *__restrict__ idx, int rows, int8_t *__restrict__ q,
                                               float *__restrict__ scale) {
    __shared__ uint32_t red[4];
    const long row = folded_block();
    if (row >= rows) return;
    const long src = idx != nullptr ? (long)idx[row] : row;
    if (src < 0 || src >= n_src) return;
    x += src * ld;
    uint32_t m = 0;
    for (int k = threadIdx.x; k < K; k += 256) m = max(m, __float_as_uint(Elem<T>::ld(x + k)) & 0x7FFFFFFFu);
    for (int o = 32; o > 0; o >>= 1) m = max(m, (uint32_t)__shfl_xor((int)m, o, WAVE));
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = m;
    __syncthreads();
    m = max(max(red[0], red[1]), max(red[2], red[3]));
    const float top = __uint_as_float(m);
    if (threadIdx.x == 0) scale[row] = m >= INF_BITS ? __uint_as_float(0x7FC00000u) : top / 127.f;
    const bool zero = m == 0 || m >= INF_BITS;
    const typename QuotientOf<T>::type quotient(zero ? 1.f : top);
    const int Kp = (K + 15) & ~15;
    for (int k = threadIdx.x; k < Kp; k += 256)
        q[row * Kp + k] = (int8_t)(zero || k >= K ? 0 : quotient(Elem<T>::ld(x + k)));
}

// GELU in its tanh form, v / (1 + exp(-2 z)) (exp and reciprocal to 1 ulp)
__device__ __forceinline__ float gelu_tanh(float v) {
    const float z = 0.7978845608028654f * fmaf(0.044715f * v, v * v, v);
    return v * __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(-2.8853900817779268f * z));
}

// Four consecutive outputs of a row from their sums.
template <typename T>
__device__ __forceinline__ f32x4 finish4(const LinearI8Args &a, const int (&acc)[4], float sq, int n) {
    const f32x4 sw = *reinterpret_cast<const f32x4 *>(a.sw + n);
    f32x4 v;
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = (float)acc[e] * sq * sw[e];
    if (a.bias != nullptr) {
        if constexpr (sizeof(T) == 2) {
            const u16x4 b = *reinterpret_cast<const u16x4 *>((const uint16_t *)a.bias + n);
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] += bf2f(b[e]);
        } else {
            v += *reinterpret_cast<const f32x4 *>((const float *)a.bias + n);
        }
    }
    if (a.gelu) {
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = gelu_tanh(v[e]);
    }
    return v;
}
__device__ __forceinline__ u16x4 to_bf16(f32x4 v) {
    bf16x4 o;
#pragma unroll
    for (int e = 0; e < 4; ++e) o[e] = (__bf16)v[e];
    return *reinterpret_cast<u16x4 *>(&o);
}

// y row of batch row r, or -1
__device__ __forceinline__ long out_row(const LinearI8Args &a, long r) {
    if (r >= a.rows) return -1;
    const long t = a.out_idx != nullptr ? (long)a.out_idx[r] : r;
    return t >= 0 && t < a.n_out ? t : -1;
}

// ---------------------------------------------------------------------------
// The product on ring-buffered MFMA tiles: a = weight rows, b = batch rows.
// bf16 tiles are staged through LDS and written in 16-byte chunks of whole
// rows; fp32 rows are stored as the accumulators hold them, four outputs at a
// time.
// ---------------------------------------------------------------------------
template <int ID, typename T>
__global__ __launch_bounds__(RING_THREADS<ID>) void k_linear_i8(LinearI8Args a, int n_at, int n_bt) {
    using R = typename RingShape<ID, RING_I8>::Tile;
    constexpr int BA = R::BA, BB = R::BB;
    extern __shared__ __align__(16) uint16_t lds[];
    int at, bt;
    tile_order(xcd_remap(blockIdx.x, n_at * n_bt), n_at, n_bt, at, bt);
    const int a0 = at * BA, b0 = bt * BB;
    const int K2 = (a.K + 15) / 16 * 8;   // pairs of elements in a row
    typename R::RowsA ra;
    typename R::RowsB rb;
    ring_rows(ra, (const uint16_t *)a.w, a.N, K2, a0);
    ring_rows(rb, (const uint16_t *)a.q, a.rows, K2, b0);
    R t;
    t.run(lds, ra, rb, K2);
#pragma unroll
    for (int j = 0; j < R::TB; ++j) {
        const int b = R::b_of(j);
        const float sq = a.sq[min(b0 + b, a.rows - 1)];
        T *to = nullptr;
        if constexpr (sizeof(T) == 4) {
            const long o = out_row(a, b0 + b);
            if (o >= 0) to = (T *)a.y + o * a.ld_y;
        }
#pragma unroll
        for (int i = 0; i < R::TA; ++i)
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                const int n = R::a_of(i, g);
                if (a0 + n >= a.N) continue;
                const int acc[4] = {t.acc[i][j][4 * g], t.acc[i][j][4 * g + 1], t.acc[i][j][4 * g + 2],
                                    t.acc[i][j][4 * g + 3]};
                const f32x4 v = finish4<T>(a, acc, sq, a0 + n);
                if constexpr (sizeof(T) == 2) *reinterpret_cast<u16x4 *>(lds + b * (BA + 8) + n) = to_bf16(v);
                else if (to != nullptr) *reinterpret_cast<f32x4 *>(to + a0 + n) = v;
            }
    }
    if constexpr (sizeof(T) == 2) {
        __syncthreads();
        write_rows<BA, BB, R::NT>(lds, min(BA, a.N - a0), [&](int b, int c0) -> uint16_t * {
            const long o = out_row(a, b0 + b);
            return o >= 0 ? (uint16_t *)a.y + o * a.ld_y + a0 + c0 : nullptr;
        });
    }
}

template <typename T>
hipError_t go_linear(const LinearI8Args &a, hipStream_t st) {
    const int K2 = (int)(i8_row(a.K) / 2);
    const int id = ring_pick(K2, [&](int BA, int BB) { return (long)cdiv(a.N, BA) * cdiv(a.rows, BB); });
    return ring_dispatch(id, [&](auto c) -> hipError_t {
        constexpr int ID = decltype(c)::value;
        using R = typename RingShape<ID, RING_I8>::Tile;
        const hipError_t e = allow_lds(k_linear_i8<ID, T>, R::LDS_BYTES);
        if (e != hipSuccess) return e;
        const int n_at = cdiv(a.N, R::BA), n_bt = cdiv(a.rows, R::BB);
        launch_k(k_linear_i8<ID, T>, (unsigned)(n_at * n_bt), R::NT, R::LDS_BYTES, st, a, n_at, n_bt);
        return hipGetLastError();
    });
}

}  // namespace

hipError_t launch_quant(bool bf16, const void *x, long ld, int n_src, int K, const int *idx, int rows, int8_t *q,
                        float *scale, hipStream_t st) {
    StageScope _stage(st, "quant_rows");
    const dim3 grid = folded_grid(rows, 256);
    if (bf16) launch_k(k_quant<uint16_t>, grid, 256, 0, st, (const uint16_t *)x, ld, n_src, K, idx, rows, q, scale);
    else launch_k(k_quant<float>, grid, 256, 0, st, (const float *)x, ld, n_src, K, idx, rows, q, scale);
    return hipGetLastError();
}

hipError_t launch_linear_i8(const LinearI8Args &a, hipStream_t st) {
    StageScope _stage(st, "linear_i8");
    return a.bf16 ? go_linear<uint16_t>(a, st) : go_linear<float>(a, st);
}

}  // namespace oc
