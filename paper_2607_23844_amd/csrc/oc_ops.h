// Argument structures and launchers of the operators around a sublayer
// (k_norm.hip).
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
size_t norm_grad_workspace_bytes(int rows, int C, int rows_per_mod);

}  // namespace oc
