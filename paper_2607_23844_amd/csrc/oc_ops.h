// Argument structures and launchers of the operators around a sublayer
// (k_norm.hip, k_rope.hip, k_i8.hip).
#pragma once
#include <cstddef>
#include <cstdint>
#include <hip/hip_runtime_api.h>

namespace oc {

// Norms before and after a sublayer with its gate, modulation and residual.
struct NormArgs {
    const void *x, *y;                                // [rows, C]; y NULL: h is x
    const void *gate, *scale, *shift;                 // rows of C, ld elements apart, or NULL
    const void *post_w, *post_b, *pre_w, *pre_b;      // [C] or NULL
    long ld;
    int rows, C, rows_per_mod;
    int post, pre;                                    // oc_norm_kind
    float post_eps, pre_eps, res_scale;
    bool bf16;
};
struct NormGrads { float *gate, *scale, *shift, *post_w, *post_b, *pre_w, *pre_b; };

hipError_t launch_norm_gate(const NormArgs &a, void *h, void *n, hipStream_t st);
hipError_t launch_norm_gate_grad(const NormArgs &a, const void *dh, const void *dn, void *dx, void *dy,
                                 const NormGrads &g, void *ws, hipStream_t st);
hipError_t launch_zero(float *p, int n, hipStream_t st);   // gradients summed over no rows
size_t norm_grad_workspace_bytes(int rows, int C, int rows_per_mod, bool bf16);


// Rotary positions, the geometry of one head as a kernel takes it: pairs 0..P
// of the axes in order, then those past the rotated channels (left alone) up
// to dh / 2.
constexpr int ROPE_MAX_PAIRS = 64;
struct RopeGeom {
    int P, dh;               // rotated pairs, head dim
    int axis1, axis2;        // first pair of the second and of the third axis
    int pairs;               // neighbours (2p, 2p + 1); else halves:
    int sect[5];             // pairs [sect[i], sect[i + 1]) lie in two halves from channel 2 sect[i] on
    int vec;                 // largest power of two <= 8 that divides every sect
    int N, W;
    long FN;                 // tokens of the grid
    double origin[3];
    double turn[ROPE_MAX_PAIRS];   // turns (of 2 pi) per position
};
// fills g from checked arguments
void rope_geom(const int *dim, int layout, int shared, const int *origin, double theta, const double *scale, int F,
               int H, int W, int head_dim, RopeGeom &g);

enum RopeType { ROPE_BF16, ROPE_F16, ROPE_F32 };
struct RopeArgs {
    const void *q, *k;       // either may be NULL
    void *qo, *ko;
    long ld_q, ld_k, ld_qo, ld_ko;
    int heads, k_heads, rows;
    const int *idx, *pos;    // row -> token, or row -> position, or NULL
    int tF, tN;              // tF > 0 (no idx): row n*tF + f is token f*tN + n
    int inverse;
};
hipError_t launch_rope(const RopeGeom &g, const RopeArgs &a, RopeType type, hipStream_t st);

// Products in 8-bit integers.
constexpr long i8_row(long K) { return (K + 15) / 16 * 16; }
hipError_t launch_quant(bool bf16, const void *x, long ld, int n_src, int K, const int *idx, int rows, int8_t *q,
                        float *scale, hipStream_t st);
struct LinearI8Args {
    const int8_t *q, *w;         // rows of i8_row(K) bytes
    const float *sq, *sw;
    const void *bias;            // [N] or NULL
    const int *out_idx;          // row -> y row, or NULL
    void *y;
    long ld_y;
    int rows, K, N, n_out;
    int gelu;
    bool bf16;
};
hipError_t launch_linear_i8(const LinearI8Args &a, hipStream_t st);

}  // namespace oc
