// Entry points of the operators around a sublayer: argument checks and
// launches.  Nothing is enqueued before every check has passed.
#include "oc_host.h"
#include "oc_ops.h"

#include <cmath>
#include <cstring>

using namespace oc;

namespace {

oc_status launched(hipError_t e, const char *what) {
    return e == hipSuccess ? record_error(OC_OK, "") : failf(OC_ERR_HIP, "%s: %s", what, hipGetErrorString(e));
}

oc_status check_norm(const oc_norm *n, const char *which) {
    if (!n) return OC_OK;
    if (n->kind < OC_NORM_NONE || n->kind > OC_NORM_LAYER)
        return failf(OC_ERR_INVALID_ARG, "%s: unknown norm %d", which, n->kind);
    if (!(n->eps >= 0.f) || !std::isfinite(n->eps))
        return failf(OC_ERR_INVALID_ARG, "%s: eps=%g must be finite and >= 0", which, (double)n->eps);
    if (!is_aligned(n->w, 16) || !is_aligned(n->b, 16))
        return failf(OC_ERR_INVALID_ARG, "%s: w and b must be 16-byte aligned", which);
    return OC_OK;
}

struct Range { const void *p; size_t bytes; };

// What forward and gradient check alike; fills a.
oc_status norm_args(const oc_shape *shape, int32_t n_rows, const void *x, const void *y, const oc_norm *post,
                    const oc_norm *pre, const oc_mod *mod, float res_scale, NormArgs &a) {
    oc_status s = valid_shape(shape);
    if (s != OC_OK) return s;
    if (n_rows < 0 || n_rows >= (1 << 30)) return failf(OC_ERR_SHAPE, "n_rows=%d outside [0, 2^30)", n_rows);
    if ((s = check_norm(post, "post")) != OC_OK || (s = check_norm(pre, "pre")) != OC_OK) return s;
    if (!std::isfinite(res_scale)) return failf(OC_ERR_INVALID_ARG, "res_scale must be finite");
    std::memset(&a, 0, sizeof(a));
    a.bf16 = shape->dtype == OC_BF16;
    a.rows = n_rows;
    a.C = shape->C;
    a.rows_per_mod = n_rows > 0 ? n_rows : 1;
    a.x = x;
    a.y = y;
    a.res_scale = res_scale;
    if (mod) {
        if (mod->reserved != 0) return failf(OC_ERR_INVALID_ARG, "oc_mod.reserved must be 0");
        if (mod->rows_per_mod < 1) return failf(OC_ERR_INVALID_ARG, "rows_per_mod=%d must be >= 1", mod->rows_per_mod);
        const int per16 = a.bf16 ? 8 : 4;
        if (mod->ld < shape->C || mod->ld % per16)
            return failf(OC_ERR_SHAPE, "modulation rows: ld=%lld must be >= C=%d and a multiple of %d",
                         (long long)mod->ld, shape->C, per16);
        if (!is_aligned(mod->gate, 16) || !is_aligned(mod->scale, 16) || !is_aligned(mod->shift, 16))
            return failf(OC_ERR_INVALID_ARG, "gate, scale and shift must be 16-byte aligned");
        a.gate = mod->gate;
        a.scale = mod->scale;
        a.shift = mod->shift;
        a.ld = mod->ld;
        a.rows_per_mod = mod->rows_per_mod;
    }
    if (post) {
        a.post = post->kind;
        a.post_eps = post->eps;
        a.post_w = post->w;
        a.post_b = post->b;
    }
    if (pre) {
        a.pre = pre->kind;
        a.pre_eps = pre->eps;
        a.pre_w = pre->w;
        a.pre_b = pre->b;
    }
    if (n_rows > 0 && !y && (post || a.gate || res_scale != 1.f))
        return failf(OC_ERR_INVALID_ARG, "post, gate and res_scale belong to y, which is NULL");
    if (n_rows > 0 && !x) return failf(OC_ERR_INVALID_ARG, "x is NULL");
    if (!is_aligned(x, 16) || !is_aligned(y, 16)) return failf(OC_ERR_INVALID_ARG, "x and y must be 16-byte aligned");
    return OC_OK;
}

// The vectors of a call and their sizes in bytes.
int vectors(const NormArgs &a, size_t esz, Range (&v)[7]) {
    const size_t row = (size_t)a.C * esz;
    const size_t n_mod = a.rows > 0 ? ((size_t)a.rows + a.rows_per_mod - 1) / a.rows_per_mod : 0;
    const size_t mods = n_mod > 0 ? (n_mod - 1) * (size_t)a.ld * esz + row : 0;
    const Range r[7] = {{a.gate, mods}, {a.scale, mods}, {a.shift, mods}, {a.post_w, row},
                        {a.post_b, row}, {a.pre_w, row}, {a.pre_b, row}};
    std::memcpy(v, r, sizeof(r));
    return 7;
}

}  // namespace

extern "C" {

oc_status oc_norm_gate(const oc_shape *shape, int32_t n_rows, const void *x, const void *y, const oc_norm *post,
                       const oc_norm *pre, const oc_mod *mod, float res_scale, void *h, void *n, hipStream_t stream) {
    NormArgs a;
    oc_status s = norm_args(shape, n_rows, x, y, post, pre, mod, res_scale, a);
    if (s != OC_OK) return s;
    if (!y && h) return failf(OC_ERR_INVALID_ARG, "h is x where y is NULL: h must be NULL");
    if (n_rows > 0 && !h && !n) return failf(OC_ERR_INVALID_ARG, "neither h nor n is wanted");
    if (!is_aligned(h, 16) || !is_aligned(n, 16)) return failf(OC_ERR_INVALID_ARG, "h and n must be 16-byte aligned");
    const size_t esz = a.bf16 ? 2 : 4, bytes = (size_t)n_rows * a.C * esz;
    if (overlaps(h, bytes, n, bytes)) return failf(OC_ERR_INVALID_ARG, "h and n must not overlap");
    Range v[7];
    const int nv = vectors(a, esz, v);
    for (const void *o : {(const void *)h, (const void *)n}) {
        for (const void *i : {x, y})
            if (i != o && overlaps(i, bytes, o, bytes))
                return failf(OC_ERR_INVALID_ARG, "h and n may be x or y, but not overlap them otherwise");
        for (int i = 0; i < nv; ++i)
            if (overlaps(v[i].p, v[i].bytes, o, bytes))
                return failf(OC_ERR_INVALID_ARG, "h and n must not overlap the vectors");
    }
    if (n_rows == 0) return record_error(OC_OK, "");
    return launched(launch_norm_gate(a, h, n, stream), "norm_gate");
}

size_t oc_norm_gate_grad_workspace_bytes(const oc_shape *shape, int32_t n_rows, int32_t rows_per_mod) {
    if (valid_shape(shape) != OC_OK || n_rows < 0 || n_rows >= (1 << 30) || rows_per_mod < 0) return 0;
    return norm_grad_workspace_bytes(n_rows, shape->C, rows_per_mod);
}

oc_status oc_norm_gate_grad(const oc_shape *shape, int32_t n_rows, const void *x, const void *y, const oc_norm *post,
                            const oc_norm *pre, const oc_mod *mod, float res_scale, const void *dh, const void *dn,
                            void *dx, void *dy, const oc_norm_grads *grads, void *ws, size_t ws_bytes,
                            hipStream_t stream) {
    NormArgs a;
    oc_status s = norm_args(shape, n_rows, x, y, post, pre, mod, res_scale, a);
    if (s != OC_OK) return s;
    const oc_norm_grads none = {nullptr, nullptr, nullptr, nullptr, nullptr, nullptr, nullptr};
    const oc_norm_grads &g = grads ? *grads : none;
    if (n_rows > 0 && !dh && !dn) return failf(OC_ERR_INVALID_ARG, "neither dh nor dn is given");
    if (!y && dy) return failf(OC_ERR_INVALID_ARG, "dy must be NULL where y is");
    const struct { const float *grad; const void *of; const char *name; } pairs[] = {
        {g.gate, a.gate, "gate"}, {g.scale, a.scale, "scale"}, {g.shift, a.shift, "shift"},
        {g.post_w, a.post_w, "post.w"}, {g.post_b, a.post_b, "post.b"}, {g.pre_w, a.pre_w, "pre.w"},
        {g.pre_b, a.pre_b, "pre.b"}};
    for (const auto &p : pairs) {
        if (p.grad && !p.of) return failf(OC_ERR_INVALID_ARG, "a gradient of %s is asked for, but it is NULL", p.name);
        if (!is_aligned(p.grad, 16)) return failf(OC_ERR_INVALID_ARG, "the gradients must be 16-byte aligned");
    }
    if (!is_aligned(dh, 16) || !is_aligned(dn, 16) || !is_aligned(dx, 16) || !is_aligned(dy, 16))
        return failf(OC_ERR_INVALID_ARG, "dh, dn, dx and dy must be 16-byte aligned");
    const size_t esz = a.bf16 ? 2 : 4, bytes = (size_t)n_rows * a.C * esz;
    const size_t need = norm_grad_workspace_bytes(n_rows, a.C, mod ? mod->rows_per_mod : 0);
    if ((s = valid_ws(ws, ws_bytes, need)) != OC_OK) return s;
    // outputs against inputs, the vectors, the workspace and each other
    Range v[7];
    const int nv = vectors(a, esz, v);
    const size_t n_mod = ((size_t)n_rows + a.rows_per_mod - 1) / a.rows_per_mod, row = (size_t)a.C * 4;
    const Range outs[9] = {{dx, bytes}, {dy, bytes}, {g.gate, n_mod * row}, {g.scale, n_mod * row},
                           {g.shift, n_mod * row}, {g.post_w, row}, {g.post_b, row}, {g.pre_w, row}, {g.pre_b, row}};
    const Range ins[5] = {{x, bytes}, {y, bytes}, {dh, bytes}, {dn, bytes}, {ws, need}};
    for (int i = 0; i < 9; ++i) {
        for (int j = 0; j < i; ++j)
            if (overlaps(outs[i].p, outs[i].bytes, outs[j].p, outs[j].bytes))
                return failf(OC_ERR_INVALID_ARG, "the gradients must not overlap each other");
        for (const Range &r : ins)
            if (overlaps(outs[i].p, outs[i].bytes, r.p, r.bytes))
                return failf(OC_ERR_INVALID_ARG, "the gradients must not overlap an input or the workspace");
        for (int j = 0; j < nv; ++j)
            if (overlaps(outs[i].p, outs[i].bytes, v[j].p, v[j].bytes))
                return failf(OC_ERR_INVALID_ARG, "the gradients must not overlap the vectors");
    }
    if (n_rows == 0) {
        // sums over no rows: the vectors of all rows are zero, there are no modulation rows
        for (float *p : {g.post_w, g.post_b, g.pre_w, g.pre_b})
            if (p) {
                const hipError_t e = launch_zero(p, a.C, stream);
                if (e != hipSuccess) return launched(e, "norm_gate_grad");
            }
        return record_error(OC_OK, "");
    }
    const NormGrads ng{g.gate, g.scale, g.shift, g.post_w, g.post_b, g.pre_w, g.pre_b};
    return launched(launch_norm_gate_grad(a, dh, dn, dx, dy, ng, ws, stream), "norm_gate_grad");
}

}  // extern "C"
