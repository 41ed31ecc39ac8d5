// C entry points of the operators of a normalised residual block: argument checks, then the launchers of block.h.
#include <math.h>

#include "block.h"
#include "checks.h"

using namespace purine;

namespace {

bool act_ok(int act) { return act >= PURINE_ACT_NONE && act <= PURINE_ACT_GELU_TANH; }

// A matrix [rows, cols] whose rows may lie nstride elements apart.
int64_t row_stride(const purine_tensor* t) { return t->nstride ? t->nstride : t->dim[1]; }
int check_matrix(const purine_tensor* t) {
    if (!t) return PURINE_E_NULL;
    purine_tensor dense = *t;
    dense.nstride = 0;
    const int rc = check_tensor(&dense, 2);
    if (rc) return rc;
    if (!is_float_dtype(t->dtype)) return PURINE_E_DTYPE;
    if (t->nstride == 0 || t->nstride == t->dim[1]) return PURINE_OK;
    if (t->nstride < t->dim[1] || t->nstride >= (1ll << 31)) return PURINE_E_SHAPE;
    if (t->nstride & (t->dtype == PURINE_BF16 ? 7 : 3)) return PURINE_E_LAYOUT;
    return (t->dim[0] - 1) * t->nstride + t->dim[1] < (1ll << 31) ? PURINE_OK : PURINE_E_SHAPE;
}
bool is_matrix(const purine_tensor* t, int64_t rows, int64_t cols) { return t->dim[0] == rows && t->dim[1] == cols; }

struct Bytes { uintptr_t lo, hi; };
Bytes bytes_of(const purine_tensor* t) {
    const uintptr_t lo = (uintptr_t)t->data;
    const size_t e = t->dtype == PURINE_F8 ? 1 : elem_bytes(t->dtype);
    if (t->ndim == 2) return {lo, lo + (size_t)((t->dim[0] - 1) * row_stride(t) + t->dim[1]) * e};
    return {lo, lo + (size_t)span_elems(t) * e};
}
bool meet(const Bytes& a, const Bytes& b) { return a.lo < b.hi && b.lo < a.hi; }
// Matrices that share bytes, columns of one buffer aside (the same distance between rows, disjoint columns).
bool matrices_meet(const purine_tensor* a, const purine_tensor* b) {
    if (!meet(bytes_of(a), bytes_of(b))) return false;
    const uint64_t s = (uint64_t)row_stride(a) * elem_bytes(a->dtype);
    if (s != (uint64_t)row_stride(b) * elem_bytes(b->dtype)) return true;
    const uint64_t la = (uint64_t)a->dim[1] * elem_bytes(a->dtype), lb = (uint64_t)b->dim[1] * elem_bytes(b->dtype);
    const uintptr_t pa = (uintptr_t)a->data, pb = (uintptr_t)b->data;
    const uint64_t d = pa >= pb ? (pa - pb) % s : (s - (pb - pa) % s) % s;
    return d < lb || s - d < la;
}
// An output and an input that may be one and the same matrix, element by element, but not overlap otherwise.
bool aliased_badly(const purine_tensor* out, const purine_tensor* in) {
    if (out->data == in->data) return row_stride(out) != row_stride(in) || out->dtype != in->dtype;
    return matrices_meet(out, in);
}
int check_ws(const void* ws, size_t ws_bytes, size_t need, std::initializer_list<const purine_tensor*> with) {
    if (need == 0) return PURINE_OK;
    if (!ws || ws_bytes < need) return PURINE_E_WORKSPACE;
    if ((uintptr_t)ws & 15u) return PURINE_E_LAYOUT;
    for (const purine_tensor* t : with)
        if (t && meet({(uintptr_t)ws, (uintptr_t)ws + need}, bytes_of(t))) return PURINE_E_LAYOUT;
    return PURINE_OK;
}
// A vector of n elements, F32 (or of `also`'s type).
int check_vector(const purine_tensor* t, int64_t n, int also = PURINE_F32) {
    const int rc = check_tensor(t, 1);
    if (rc) return rc;
    if (t->dtype != PURINE_F32 && t->dtype != also) return PURINE_E_DTYPE;
    return t->dim[0] == n ? PURINE_OK : PURINE_E_SHAPE;
}

// ---- group normalization
int norm_axes(const purine_tensor* x) { return x->ndim >= 2 && x->ndim <= 4 ? x->ndim : -1; }
int norm_shape(const purine_tensor* x, int groups, int act, NormShape* s) {
    int rc = check_tensor(x, norm_axes(x), true);
    if (rc) return rc;
    if (!is_float_dtype(x->dtype)) return PURINE_E_DTYPE;
    if (!act_ok(act) || groups < 1) return PURINE_E_ARG;
    s->N = (int)x->dim[0];
    s->C = (int)x->dim[x->ndim - 1];
    s->S = (int)(image_elems(x) / s->C);
    if (s->C % groups) return PURINE_E_SHAPE;
    s->G = groups;
    s->act = act;
    s->x_ns = nstride_of(x);
    return PURINE_OK;
}
int norm_like(const purine_tensor* x, const purine_tensor* t) {
    const int rc = check_tensor(t, x->ndim, true);
    if (rc) return rc;
    if (t->dtype != x->dtype) return PURINE_E_DTYPE;
    return same_dims(x, t) ? PURINE_OK : PURINE_E_SHAPE;
}
int norm_stat(const purine_tensor* t, const NormShape& s) {
    const int rc = check_tensor(t, 2);
    if (rc) return rc;
    if (t->dtype != PURINE_F32) return PURINE_E_DTYPE;
    return is_matrix(t, s.N, s.G) ? PURINE_OK : PURINE_E_SHAPE;
}
const float* data_or_null(const purine_tensor* t) { return t ? (const float*)t->data : nullptr; }
bool any_meets(const purine_tensor* out, std::initializer_list<const purine_tensor*> with) {
    for (const purine_tensor* t : with)
        if (t && meet(bytes_of(out), bytes_of(t))) return true;
    return false;
}
bool norm_aliased_badly(const purine_tensor* out, const purine_tensor* in) {
    return out->data == in->data ? nstride_of(out) != nstride_of(in) : overlaps(out, in);
}

// ---- matrix products
int linear_bias(const purine_tensor* b, int64_t n, int dtype) {
    const int rc = check_vector(b, n, dtype);
    if (rc) return rc;
    return b->dtype == dtype ? PURINE_OK : PURINE_E_DTYPE;
}
int grad_vector(const purine_tensor* db, int64_t n, int dtype) { return check_vector(db, n, dtype); }

}  // namespace

extern "C" {

size_t purine_group_norm_workspace_bytes(int backward, const int64_t x_dim[4], int ndim, int groups, int32_t dtype) {
    if (!x_dim || ndim < 2 || ndim > 4 || groups < 1 || !is_float_dtype(dtype)) return 0;
    int64_t n = 1;
    for (int i = 0; i < ndim; ++i) {
        if (x_dim[i] < 1 || x_dim[i] >= (1ll << 31) || (n *= x_dim[i]) >= (1ll << 31)) return 0;
    }
    const int64_t C = x_dim[ndim - 1];
    if (C % groups) return 0;
    return group_norm_ws_bytes(x_dim[0], n / x_dim[0] / C, C, groups);
}

int purine_group_norm_fwd(const purine_tensor* x, const purine_tensor* scale, const purine_tensor* shift, purine_tensor* y,
                          purine_tensor* mean, purine_tensor* rstd, int groups, float eps, int act, void* ws,
                          size_t ws_bytes, void* hip_stream) {
    if (!x || !y) return PURINE_E_NULL;
    NormShape s{};
    int rc;
    if ((rc = norm_shape(x, groups, act, &s)) || (rc = norm_like(x, y))) return rc;
    if (!(eps > 0.0f) || !(eps < INFINITY)) return PURINE_E_ARG;
    if ((scale && (rc = check_vector(scale, s.C))) || (shift && (rc = check_vector(shift, s.C)))) return rc;
    if (!mean != !rstd) return PURINE_E_NULL;
    if (mean && ((rc = norm_stat(mean, s)) || (rc = norm_stat(rstd, s)))) return rc;
    if (norm_aliased_badly(y, x) || any_meets(y, {scale, shift, mean, rstd})) return PURINE_E_LAYOUT;
    if (mean && (any_meets(mean, {x, scale, shift, rstd}) || any_meets(rstd, {x, scale, shift}))) return PURINE_E_LAYOUT;
    const size_t need = group_norm_ws_bytes(s.N, s.S, s.C, s.G);
    if ((rc = check_ws(ws, ws_bytes, need, {x, y, scale, shift, mean, rstd}))) return rc;
    s.y_ns = nstride_of(y);
    s.eps = eps;
    return hip_status(launch_group_norm_fwd(x->dtype, s, x->data, data_or_null(scale), data_or_null(shift), y->data,
                                            (float*)data_or_null(mean), (float*)data_or_null(rstd), ws, (hipStream_t)hip_stream));
}

int purine_group_norm_bwd(const purine_tensor* x, const purine_tensor* scale, const purine_tensor* shift,
                          const purine_tensor* mean, const purine_tensor* rstd, const purine_tensor* dy, purine_tensor* dx,
                          purine_tensor* dscale, purine_tensor* dshift, int groups, int act, float beta, void* ws,
                          size_t ws_bytes, void* hip_stream) {
    if (!x || !mean || !rstd || !dy || !dx) return PURINE_E_NULL;
    NormShape s{};
    int rc;
    if ((rc = norm_shape(x, groups, act, &s)) || (rc = norm_like(x, dy)) || (rc = norm_like(x, dx)) || (rc = norm_stat(mean, s)) ||
        (rc = norm_stat(rstd, s)) || (rc = check_beta(beta)))
        return rc;
    if ((scale && (rc = check_vector(scale, s.C))) || (shift && (rc = check_vector(shift, s.C)))) return rc;
    if (!dscale != !dshift) return PURINE_E_NULL;
    if (dscale && ((rc = check_vector(dscale, s.C)) || (rc = check_vector(dshift, s.C)))) return rc;
    if (norm_aliased_badly(dx, dy) || overlaps(dx, x) || any_meets(dx, {scale, shift, mean, rstd, dscale, dshift})) return PURINE_E_LAYOUT;
    if (dscale && (any_meets(dscale, {x, scale, shift, mean, rstd, dy, dshift}) || any_meets(dshift, {x, scale, shift, mean, rstd, dy})))
        return PURINE_E_LAYOUT;
    const size_t need = group_norm_ws_bytes(s.N, s.S, s.C, s.G);
    if ((rc = check_ws(ws, ws_bytes, need, {x, scale, shift, mean, rstd, dy, dx, dscale, dshift}))) return rc;
    s.dy_ns = nstride_of(dy);
    s.dx_ns = nstride_of(dx);
    return hip_status(launch_group_norm_bwd(x->dtype, s, x->data, data_or_null(scale), data_or_null(shift), data_or_null(mean),
                                            data_or_null(rstd), dy->data, dx->data, (float*)data_or_null(dscale), (float*)data_or_null(dshift),
                                            beta, ws, (hipStream_t)hip_stream));
}

size_t purine_linear_workspace_bytes(int pass, int64_t N, int64_t C, int64_t K, int32_t dtype) {
    const int64_t lim = 1ll << 31;
    if (N < 1 || C < 1 || K < 1 || N >= lim || C >= lim || K >= lim || N * C >= lim || C * K >= lim || N * K >= lim || !is_float_dtype(dtype)) return 0;
    switch (pass) {
        case PURINE_CONV_FWD: return linear_ws_bytes(N, K, C, true, true, dtype);
        case PURINE_CONV_BWD_DATA: return linear_ws_bytes(N, C, K, true, false, dtype);
        case PURINE_CONV_BWD_WEIGHT: {
            const size_t db = act_bwd_ws_bytes(N, K), dw = linear_ws_bytes(K, C, N, false, false, dtype);
            return db > dw ? db : dw;
        }
        default: return 0;
    }
}

int purine_linear_fwd(const purine_tensor* x, const purine_tensor* w, const purine_tensor* b, const purine_tensor* r,
                      purine_tensor* y, purine_tensor* pre, int act, void* ws, size_t ws_bytes, void* hip_stream) {
    if (!x || !w || !y) return PURINE_E_NULL;
    int rc;
    if ((rc = check_matrix(x)) || (rc = check_matrix(w)) || (rc = check_matrix(y))) return rc;
    const int64_t N = x->dim[0], C = x->dim[1], K = w->dim[0];
    if (w->dtype != x->dtype || y->dtype != x->dtype) return PURINE_E_DTYPE;
    if (w->dim[1] != C || !is_matrix(y, N, K)) return PURINE_E_SHAPE;
    if (b && (rc = linear_bias(b, K, x->dtype))) return rc;
    for (const purine_tensor* t : {r, (const purine_tensor*)pre}) {
        if (!t) continue;
        if ((rc = check_matrix(t))) return rc;
        if (t->dtype != x->dtype) return PURINE_E_DTYPE;
        if (!is_matrix(t, N, K)) return PURINE_E_SHAPE;
    }
    if (!act_ok(act)) return PURINE_E_ARG;
    if (matrices_meet(y, x) || matrices_meet(y, w) || (b && meet(bytes_of(y), bytes_of(b))) || (r && aliased_badly(y, r))) return PURINE_E_LAYOUT;
    if (pre && (matrices_meet(pre, x) || matrices_meet(pre, w) || matrices_meet(pre, y) || (b && meet(bytes_of(pre), bytes_of(b))) ||
                (r && matrices_meet(pre, r))))
        return PURINE_E_LAYOUT;
    const size_t need = purine_linear_workspace_bytes(PURINE_CONV_FWD, N, C, K, x->dtype);
    if ((rc = check_ws(ws, ws_bytes, need, {x, w, b, r, y, pre}))) return rc;
    LinearCall c{};
    c.rows = N; c.cols = K; c.K = C;
    c.a = x->data; c.a_ld = row_stride(x); c.a_in = true;
    c.b = w->data; c.b_ld = row_stride(w); c.b_in = true;
    c.dtype = c.out_dtype = x->dtype;
    c.out = y->data; c.out_ld = row_stride(y);
    c.bias = b ? b->data : nullptr;
    if (r) { c.res = r->data; c.res_ld = row_stride(r); }
    if (pre) { c.pre = pre->data; c.pre_ld = row_stride(pre); }
    c.act = act;
    return hip_status(launch_linear(c, ws, (hipStream_t)hip_stream));
}

int purine_linear_bwd_data(const purine_tensor* dy, const purine_tensor* w, const purine_tensor* pre, purine_tensor* dx,
                           int act, float beta, void* ws, size_t ws_bytes, void* hip_stream) {
    if (!dy || !w || !dx) return PURINE_E_NULL;
    int rc;
    if ((rc = check_matrix(dy)) || (rc = check_matrix(w)) || (rc = check_matrix(dx))) return rc;
    const int64_t N = dy->dim[0], K = dy->dim[1], C = w->dim[1];
    if (w->dtype != dy->dtype || dx->dtype != dy->dtype) return PURINE_E_DTYPE;
    if (w->dim[0] != K || !is_matrix(dx, N, C)) return PURINE_E_SHAPE;
    if (pre) {
        if ((rc = check_matrix(pre))) return rc;
        if (pre->dtype != dy->dtype) return PURINE_E_DTYPE;
        if (!is_matrix(pre, N, C)) return PURINE_E_SHAPE;
    }
    if (!act_ok(act) || (!pre && act != PURINE_ACT_NONE)) return PURINE_E_ARG;
    if ((rc = check_beta(beta))) return rc;
    if (matrices_meet(dx, dy) || matrices_meet(dx, w) || (pre && aliased_badly(dx, pre))) return PURINE_E_LAYOUT;
    if (pre && beta != 0.0f && dx->data == pre->data) return PURINE_E_LAYOUT;
    const size_t need = purine_linear_workspace_bytes(PURINE_CONV_BWD_DATA, N, C, K, dy->dtype);
    if ((rc = check_ws(ws, ws_bytes, need, {dy, w, pre, dx}))) return rc;
    LinearCall c{};
    c.rows = N; c.cols = C; c.K = K;
    c.a = dy->data; c.a_ld = row_stride(dy); c.a_in = true;
    c.b = w->data; c.b_ld = row_stride(w); c.b_in = false;
    c.dtype = c.out_dtype = dy->dtype;
    c.out = dx->data; c.out_ld = row_stride(dx);
    if (pre && act != PURINE_ACT_NONE) { c.slope = pre->data; c.slope_ld = row_stride(pre); }
    c.act = act;
    c.accumulate = beta != 0.0f;
    return hip_status(launch_linear(c, ws, (hipStream_t)hip_stream));
}

int purine_linear_bwd_weight(const purine_tensor* x, const purine_tensor* dy, purine_tensor* dw, purine_tensor* db, float beta,
                             void* ws, size_t ws_bytes, void* hip_stream) {
    if (!x || !dy || !dw) return PURINE_E_NULL;
    int rc;
    if ((rc = check_matrix(x)) || (rc = check_matrix(dy)) || (rc = check_matrix(dw))) return rc;
    const int64_t N = x->dim[0], C = x->dim[1], K = dy->dim[1];
    if (dy->dtype != x->dtype || (dw->dtype != PURINE_F32 && dw->dtype != x->dtype)) return PURINE_E_DTYPE;
    if (dy->dim[0] != N || !is_matrix(dw, K, C)) return PURINE_E_SHAPE;
    if ((db && (rc = grad_vector(db, K, x->dtype))) || (rc = check_beta(beta))) return rc;
    if (meet(bytes_of(dw), bytes_of(x)) || meet(bytes_of(dw), bytes_of(dy))) return PURINE_E_LAYOUT;
    if (db && any_meets(db, {x, dy, dw})) return PURINE_E_LAYOUT;
    const size_t need = purine_linear_workspace_bytes(PURINE_CONV_BWD_WEIGHT, N, C, K, x->dtype);
    if ((rc = check_ws(ws, ws_bytes, need, {x, dy, dw, db}))) return rc;
    LinearCall c{};
    c.rows = K; c.cols = C; c.K = N;
    c.a = dy->data; c.a_ld = row_stride(dy); c.a_in = false;
    c.b = x->data; c.b_ld = row_stride(x); c.b_in = false;
    c.dtype = x->dtype;
    c.out = dw->data; c.out_ld = row_stride(dw); c.out_dtype = dw->dtype;
    c.accumulate = beta != 0.0f;
    hipError_t e = launch_linear(c, ws, (hipStream_t)hip_stream);
    if (e == hipSuccess && db)
        e = launch_act_bwd(dy->dtype, nullptr, 0, dy->data, row_stride(dy), nullptr, 0, db->data, db->dtype, beta != 0.0f, N, K, PURINE_ACT_NONE,
                           ws, (hipStream_t)hip_stream);
    return hip_status(e);
}

size_t purine_act_bwd_workspace_bytes(int64_t N, int64_t K) {
    const int64_t lim = 1ll << 31;
    return N < 1 || K < 1 || N >= lim || K >= lim || N * K >= lim ? 0 : act_bwd_ws_bytes(N, K);
}

int purine_act_bwd(const purine_tensor* pre, const purine_tensor* dy, purine_tensor* g, purine_tensor* db, int act, void* ws,
                   size_t ws_bytes, void* hip_stream) {
    if (!pre || !dy || !g) return PURINE_E_NULL;
    int rc;
    if ((rc = check_matrix(pre)) || (rc = check_matrix(dy)) || (rc = check_matrix(g))) return rc;
    const int64_t N = pre->dim[0], K = pre->dim[1];
    if (dy->dtype != pre->dtype || g->dtype != pre->dtype) return PURINE_E_DTYPE;
    if (!is_matrix(dy, N, K) || !is_matrix(g, N, K)) return PURINE_E_SHAPE;
    if (db && (rc = grad_vector(db, K, pre->dtype))) return rc;
    if (!act_ok(act)) return PURINE_E_ARG;
    if (aliased_badly(g, dy) || aliased_badly(g, pre) || (db && any_meets(db, {pre, dy, g}))) return PURINE_E_LAYOUT;
    if (db && (rc = check_ws(ws, ws_bytes, act_bwd_ws_bytes(N, K), {pre, dy, g, db}))) return rc;
    return hip_status(launch_act_bwd(pre->dtype, pre->data, row_stride(pre), dy->data, row_stride(dy), g->data, row_stride(g),
                                     db ? db->data : nullptr, db ? db->dtype : PURINE_F32, false, N, K, act, ws, (hipStream_t)hip_stream));
}

int purine_adamw_step(const purine_adamw_desc* d, const purine_adamw_param* params, int n_params, purine_tensor* done,
                      void* hip_stream) {
    if (!d || (n_params > 0 && !params)) return PURINE_E_NULL;
    if (n_params < 0) return PURINE_E_ARG;
    auto finite = [](double v) { return (float)v - (float)v == 0.0f; };
    if (!finite(d->lr) || !finite(d->weight_decay) || !finite(d->grad_scale) || !(d->beta1 >= 0.0 && d->beta1 < 1.0) ||
        !(d->beta2 >= 0.0 && d->beta2 < 1.0) || !((float)d->eps > 0.0f) || !finite(d->eps) || (d->dither != 0 && d->dither != 1))
        return PURINE_E_ARG;
    int rc;
    if (done) {
        if ((rc = check_tensor(done, 1))) return rc;
        if (done->dtype != PURINE_I32) return PURINE_E_DTYPE;
        if (done->dim[0] != 1) return PURINE_E_SHAPE;
    } else if (d->step < 1) {
        return PURINE_E_ARG;
    }
    for (int i = 0; i < n_params; ++i) {
        const purine_adamw_param& p = params[i];
        const bool coded = p.m.dtype == PURINE_F8;
        if ((rc = check_tensor(&p.w, p.w.ndim >= 1 && p.w.ndim <= 4 ? p.w.ndim : -1))) return rc;
        const int64_t n = numel(&p.w), blocks = (n + PURINE_ADAMW_BLOCK - 1) / PURINE_ADAMW_BLOCK;
        const purine_tensor* all[7] = {&p.w, &p.dw, &p.m, &p.v, &p.copy, &p.m_scale, &p.v_scale};
        for (int k = 1; k < 7; ++k) {
            if (k == 4 && !p.copy.data) { all[k] = nullptr; continue; }
            if (k >= 5 && !coded) { all[k] = nullptr; continue; }
            purine_tensor t = *all[k];
            if (t.dtype == PURINE_F8 && (k == 2 || k == 3)) t.dtype = PURINE_F32;      // (check_tensor knows the types of the other operators)
            if (k >= 5 && ((uintptr_t)t.data & 15u) % 4 == 0) t.data = (void*)((uintptr_t)t.data & ~(uintptr_t)15u);   // (read and written one by one)
            if ((rc = check_tensor(&t, t.ndim >= 1 && t.ndim <= 4 ? t.ndim : -1))) return rc;
            if (numel(&t) != (k >= 5 ? blocks : n)) return PURINE_E_SHAPE;
        }
        if (!is_float_dtype(p.w.dtype) || !is_float_dtype(p.dw.dtype) || (p.m.dtype != PURINE_F32 && !coded) || p.v.dtype != p.m.dtype ||
            (p.copy.data && p.copy.dtype != PURINE_BF16) || (coded && (p.m_scale.dtype != PURINE_F32 || p.v_scale.dtype != PURINE_F32)))
            return PURINE_E_DTYPE;
        if (p.w.dtype != params[0].w.dtype || p.dw.dtype != params[0].dw.dtype || p.m.dtype != params[0].m.dtype) return PURINE_E_DTYPE;
        for (int a = 0; a < 7; ++a)
            for (int b = 0; b < a; ++b)
                if (all[a] && all[b] && meet(bytes_of(all[a]), bytes_of(all[b]))) return PURINE_E_LAYOUT;
    }
    return hip_status(launch_adamw(*d, params, n_params, done ? (int*)done->data : nullptr, (hipStream_t)hip_stream));
}

}  // extern "C"
