// Products in 8-bit integers: rows quantised with a scale each, and the product
// of two such matrices with a fused epilogue (scales, bias, GELU, rows written
// to their positions).
#include "oc_device.h"
#include "oc_launch.h"
#include "oc_ops.h"
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

__device__ __forceinline__ float gelu_tanh(float v) {
    const float z = 0.7978845608028654f * fmaf(0.044715f * v, v * v, v);
    return v / (1.0f + __builtin_amdgcn_exp2f(-2.8853900817779268f * z));
}

// A 32 x 32 tile of y per block, 16-byte steps of k through LDS, one row and
// four columns per thread.
template <typename T>
__global__ __launch_bounds__(256) void k_linear_i8(LinearI8Args a) {
    __shared__ int4 sq[32][9], sw[32][9];
    const int Kp = (a.K + 15) & ~15, n0 = blockIdx.x * 32;
    const long r0 = (long)blockIdx.y * 32;
    const int tr = threadIdx.x >> 3, tc = threadIdx.x & 7;
    int acc[4] = {};
    for (int k0 = 0; k0 < Kp; k0 += 128) {
        const int k = k0 + tc * 16;
        const int4 z = make_int4(0, 0, 0, 0);
        sq[tr][tc] = r0 + tr < a.rows && k < Kp ? *reinterpret_cast<const int4 *>(a.q + (r0 + tr) * Kp + k) : z;
        sw[tr][tc] = n0 + tr < a.N && k < Kp ? *reinterpret_cast<const int4 *>(a.w + (long)(n0 + tr) * Kp + k) : z;
        __syncthreads();
        for (int c = 0; c < 8; ++c) {
            const int4 u = sq[tr][c];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int4 v = sw[tc + 8 * j][c];
                acc[j] = __builtin_amdgcn_sdot4(u.x, v.x, acc[j], false);
                acc[j] = __builtin_amdgcn_sdot4(u.y, v.y, acc[j], false);
                acc[j] = __builtin_amdgcn_sdot4(u.z, v.z, acc[j], false);
                acc[j] = __builtin_amdgcn_sdot4(u.w, v.w, acc[j], false);
            }
        }
        __syncthreads();
    }
    const long r = r0 + tr;
    if (r >= a.rows) return;
    const long t = a.out_idx != nullptr ? (long)a.out_idx[r] : r;
    if (t < 0 || t >= a.n_out) return;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const int n = n0 + tc + 8 * j;
        if (n >= a.N) continue;
        float v = (float)acc[j] * a.sq[r] * a.sw[n];
        if (a.bias != nullptr) v += Elem<T>::ld((const T *)a.bias + n);
        if (a.gelu) v = gelu_tanh(v);
        T *const to = (T *)a.y + t * a.ld_y + n;
        if constexpr (sizeof(T) == 2) *reinterpret_cast<__bf16 *>(to) = (__bf16)v;
        else *to = v;
    }
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
    const dim3 grid((unsigned)cdiv(a.N, 32), (unsigned)cdiv(a.rows, 32));
    if (a.bf16) launch_k(k_linear_i8<uint16_t>, grid, 256, 0, st, a);
    else launch_k(k_linear_i8<float>, grid, 256, 0, st, a);
    return hipGetLastError();
}

}  // namespace oc
