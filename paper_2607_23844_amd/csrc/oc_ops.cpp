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

constexpr int MAX_ROWS = 1 << 30;
constexpr int64_t MAX_LD = 1LL << 40;
constexpr int MAX_I8_K = 131056;   // 128 * 128 * K stays below 2^31

oc_status check_i8(int32_t dtype, int32_t n_rows, int32_t K) {
    if (dtype != OC_F32 && dtype != OC_BF16) return failf(OC_ERR_DTYPE, "unknown dtype %d", dtype);
    if (n_rows < 0 || n_rows >= MAX_ROWS) return failf(OC_ERR_SHAPE, "n_rows=%d outside [0, 2^30)", n_rows);
    if (K < 8 || K % 8 || K > MAX_I8_K)
        return failf(OC_ERR_SHAPE, "K=%d must be a multiple of 8 in [8, %d]", K, MAX_I8_K);
    return OC_OK;
}

}  // namespace

namespace oc {

oc_status make_rope(const oc_shape *sh, const oc_rope *rope, RopeGeom &g) {
    if (!rope) return OC_OK;
    long long sum = 0;
    for (int i = 0; i < 3; ++i) {
        if (rope->dim[i] < 0 || rope->dim[i] % 2)
            return failf(OC_ERR_SHAPE, "rotary dim[%d]=%d must be even and >= 0", i, rope->dim[i]);
        if (!std::isfinite(rope->scale[i])) return failf(OC_ERR_INVALID_ARG, "rotary scale[%d] must be finite", i);
        sum += rope->dim[i];
    }
    if (sum < 2 || sum > sh->head_dim)
        return failf(OC_ERR_SHAPE, "rotary dims of %lld channels in all: outside [2, head_dim=%d]", sum, sh->head_dim);
    if (rope->layout < OC_ROPE_PAIRS || rope->layout > OC_ROPE_SPLIT)
        return failf(OC_ERR_INVALID_ARG, "unknown rotary layout %d", rope->layout);
    if (rope->shared != 0 && rope->shared != 1) return failf(OC_ERR_INVALID_ARG, "shared must be 0 or 1");
    if (!(rope->theta > 0.0) || !std::isfinite(rope->theta))
        return failf(OC_ERR_INVALID_ARG, "theta=%g must be finite and > 0", rope->theta);
    rope_geom(rope->dim, rope->layout, rope->shared, rope->origin, rope->theta, rope->scale, sh->F, sh->H, sh->W,
              sh->head_dim, g);
    for (int p = 0; p < g.P; ++p)
        if (!std::isfinite(g.turn[p] * 0x1p33))   // (any position plus origin)
            return failf(OC_ERR_INVALID_ARG, "theta=%g and the scales give pair %d no finite angle", rope->theta, p);
    return OC_OK;
}

}  // namespace oc

extern "C" {

oc_status oc_rope_qk(const oc_shape *shape, const oc_rope *rope, int32_t n_rows, const int32_t *kept_idx,
                     const int32_t *pos, const void *q, int64_t ld_q, const void *k, int64_t ld_k, int32_t k_heads,
                     void *q_out, int64_t ld_qo, void *k_out, int64_t ld_ko, int32_t inverse, hipStream_t stream) {
    oc_status s = valid_shape(shape);
    if (s != OC_OK) return s;
    if (!rope) return failf(OC_ERR_INVALID_ARG, "rope is NULL");
    RopeGeom g;
    if ((s = make_rope(shape, rope, g)) != OC_OK) return s;
    if (n_rows < 0 || n_rows >= (1 << 30)) return failf(OC_ERR_SHAPE, "n_rows=%d outside [0, 2^30)", n_rows);
    if (inverse != 0 && inverse != 1) return failf(OC_ERR_INVALID_ARG, "inverse must be 0 or 1");
    if (kept_idx && pos) return failf(OC_ERR_INVALID_ARG, "kept_idx and pos exclude each other");
    if (!kept_idx && !pos && n_rows > g.FN)
        return failf(OC_ERR_SHAPE, "n_rows=%d past the grid of %ld tokens", n_rows, g.FN);
    if (n_rows > 0 && !q && !k) return failf(OC_ERR_INVALID_ARG, "neither q nor k is given");
    if ((q && !q_out) || (!q && q_out) || (k && !k_out) || (!k && k_out))
        return failf(OC_ERR_INVALID_ARG, "q and q_out, k and k_out go together");
    if (k && (k_heads < 1 || k_heads > (1 << 20))) return failf(OC_ERR_SHAPE, "k_heads=%d outside [1, 2^20]", k_heads);
    const bool bf16 = shape->dtype == OC_BF16;
    const size_t esz = bf16 ? 2 : 4;
    struct Side { const void *p; int64_t ld; size_t width; const char *name; };
    const size_t wq = (size_t)shape->heads * shape->head_dim, wk = k ? (size_t)k_heads * shape->head_dim : 0;
    const Side in[2] = {{q, ld_q, wq, "q"}, {k, ld_k, wk, "k"}}, out[2] = {{q_out, ld_qo, wq, "q_out"},
                                                                         {k_out, ld_ko, wk, "k_out"}};
    for (const Side &d : {in[0], in[1], out[0], out[1]}) {
        if (!d.p) continue;
        if (!is_aligned(d.p, 16)) return failf(OC_ERR_INVALID_ARG, "%s must be 16-byte aligned", d.name);
        if (d.ld < (int64_t)d.width || d.ld > (1LL << 40) || d.ld * esz % 16)
            return failf(OC_ERR_SHAPE, "%s: a row stride of %lld elements is not a multiple of 16 bytes of at least %zu",
                         d.name, (long long)d.ld, d.width);
    }
    for (const Side &o : out) {
        for (const Side &i : in)
            if (!(i.p == o.p && i.ld == o.ld && i.width == o.width) &&
                rows_overlap(i.p, i.width * esz, i.ld * esz, o.p, o.width * esz, o.ld * esz, n_rows))
                return failf(OC_ERR_INVALID_ARG, "%s overlaps %s", o.name, i.name);
        if (overlaps(kept_idx, (size_t)n_rows * 4, o.p, n_rows ? ((n_rows - 1) * o.ld + o.width) * esz : 0) ||
            overlaps(pos, (size_t)n_rows * 12, o.p, n_rows ? ((n_rows - 1) * o.ld + o.width) * esz : 0))
            return failf(OC_ERR_INVALID_ARG, "%s overlaps the positions", o.name);
    }
    if (rows_overlap(q_out, wq * esz, ld_qo * esz, k_out, wk * esz, ld_ko * esz, n_rows))
        return failf(OC_ERR_INVALID_ARG, "q_out overlaps k_out");
    if (q && k && (q == k_out || k == q_out) && n_rows > 0)
        return failf(OC_ERR_INVALID_ARG, "an output is the other tensor's input");
    if (n_rows == 0) return record_error(OC_OK, "");
    const RopeArgs a{q, k, q_out, k_out, (long)ld_q, (long)ld_k, (long)ld_qo, (long)ld_ko, shape->heads, k_heads,
                     n_rows, kept_idx, pos, 0, 0, inverse};
    return launched(launch_rope(g, a, bf16 ? ROPE_BF16 : ROPE_F32, stream), "rope");
}

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
    return norm_grad_workspace_bytes(n_rows, shape->C, rows_per_mod, shape->dtype == OC_BF16);
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
    const size_t need = norm_grad_workspace_bytes(n_rows, a.C, mod ? mod->rows_per_mod : 0, a.bf16);
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
    for (int i = 0; i < 4; ++i)
        if (overlaps(ws, need, ins[i].p, ins[i].bytes))
            return failf(OC_ERR_INVALID_ARG, "the workspace must not overlap an input");
    for (int i = 0; i < nv; ++i)
        if (overlaps(ws, need, v[i].p, v[i].bytes))
            return failf(OC_ERR_INVALID_ARG, "the workspace must not overlap the vectors");
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

size_t oc_i8_row_bytes(int32_t K) { return K > 0 ? (size_t)i8_row(K) : 0; }

oc_status oc_quant_rows(int32_t dtype, const void *x, int64_t ld, int32_t n_src, int32_t K, const int32_t *row_idx,
                        int32_t n_rows, int8_t *q, float *scale, hipStream_t stream) {
    oc_status s = check_i8(dtype, n_rows, K);
    if (s != OC_OK) return s;
    const size_t esz = dtype == OC_BF16 ? 2 : 4;
    if (n_src < 0 || n_src >= MAX_ROWS) return failf(OC_ERR_SHAPE, "n_src=%d outside [0, 2^30)", n_src);
    if (!row_idx && n_rows > n_src) return failf(OC_ERR_SHAPE, "n_rows=%d of a matrix of %d rows", n_rows, n_src);
    if (ld < K || ld > MAX_LD || ld * esz % 16)
        return failf(OC_ERR_SHAPE, "x: a row stride of %lld elements is not a multiple of 16 bytes of at least K=%d",
                     (long long)ld, K);
    if (n_rows > 0 && (!q || !scale || (!x && n_src > 0))) return failf(OC_ERR_INVALID_ARG, "NULL pointer");
    if (!is_aligned(x, 16) || !is_aligned(q, 16)) return failf(OC_ERR_INVALID_ARG, "x and q must be 16-byte aligned");
    if (!is_aligned(scale, 4) || !is_aligned(row_idx, 4))
        return failf(OC_ERR_INVALID_ARG, "scale and row_idx must be 4-byte aligned");
    const size_t xb = n_src > 0 ? ((size_t)(n_src - 1) * ld + K) * esz : 0, qb = (size_t)n_rows * i8_row(K);
    const size_t sb = (size_t)n_rows * 4;
    if (overlaps(q, qb, x, xb) || overlaps(scale, sb, x, xb) || overlaps(q, qb, scale, sb) ||
        overlaps(q, qb, row_idx, sb) || overlaps(scale, sb, row_idx, sb))
        return failf(OC_ERR_INVALID_ARG, "q and scale must not overlap each other or an input");
    if (n_rows == 0 || n_src == 0) return record_error(OC_OK, "");
    return launched(launch_quant(dtype == OC_BF16, x, (long)ld, n_src, K, row_idx, n_rows, q, scale, stream),
                    "quant_rows");
}

oc_status oc_linear_i8(int32_t dtype, int32_t n_rows, int32_t K, int32_t N, const int8_t *q, const float *scale_q,
                       const int8_t *w, const float *scale_w, const void *bias, int32_t act, const int32_t *out_idx,
                       int32_t n_out, void *y, int64_t ld_y, hipStream_t stream) {
    oc_status s = check_i8(dtype, n_rows, K);
    if (s != OC_OK) return s;
    const size_t esz = dtype == OC_BF16 ? 2 : 4;
    if (N < 8 || N % 8 || N > (1 << 24)) return failf(OC_ERR_SHAPE, "N=%d must be a multiple of 8 in [8, 2^24]", N);
    if ((int64_t)n_rows * N >= 1LL << 37) return failf(OC_ERR_SHAPE, "%d rows of N=%d outputs: too many", n_rows, N);
    if (act != OC_ACT_NONE && act != OC_ACT_GELU) return failf(OC_ERR_INVALID_ARG, "unknown activation %d", act);
    if (n_out < 0 || n_out >= MAX_ROWS) return failf(OC_ERR_SHAPE, "n_out=%d outside [0, 2^30)", n_out);
    if (!out_idx && n_rows > n_out) return failf(OC_ERR_SHAPE, "n_rows=%d into %d rows", n_rows, n_out);
    if (ld_y < N || ld_y > MAX_LD || ld_y * esz % 16)
        return failf(OC_ERR_SHAPE, "y: a row stride of %lld elements is not a multiple of 16 bytes of at least N=%d",
                     (long long)ld_y, N);
    if (n_rows > 0 && (!q || !scale_q || !w || !scale_w || (!y && n_out > 0)))
        return failf(OC_ERR_INVALID_ARG, "NULL pointer");
    if (!is_aligned(q, 16) || !is_aligned(w, 16) || !is_aligned(scale_w, 16) || !is_aligned(bias, 16) ||
        !is_aligned(y, 16))
        return failf(OC_ERR_INVALID_ARG, "q, w, scale_w, bias and y must be 16-byte aligned");
    if (!is_aligned(scale_q, 4) || !is_aligned(out_idx, 4))
        return failf(OC_ERR_INVALID_ARG, "scale_q and out_idx must be 4-byte aligned");
    const size_t row = (size_t)i8_row(K), yb = n_out > 0 ? ((size_t)(n_out - 1) * ld_y + N) * esz : 0;
    const Range ins[] = {{q, n_rows * row}, {w, N * row}, {scale_q, (size_t)n_rows * 4}, {scale_w, (size_t)N * 4},
                         {bias, N * esz}, {out_idx, (size_t)n_rows * 4}};
    for (const Range &r : ins)
        if (overlaps(y, yb, r.p, r.bytes)) return failf(OC_ERR_INVALID_ARG, "y must not overlap an input");
    if (n_rows == 0 || n_out == 0) return record_error(OC_OK, "");
    const LinearI8Args a{q, w, scale_q, scale_w, bias, out_idx, y, (long)ld_y, n_rows, K, N, n_out,
                         act == OC_ACT_GELU ? 1 : 0, dtype == OC_BF16};
    return launched(launch_linear_i8(a, stream), "linear_i8");
}

}  // extern "C"
