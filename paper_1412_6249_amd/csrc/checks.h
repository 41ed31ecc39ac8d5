// Argument checks that the host entry points share (api.cpp, block_api.cpp). Everything here is host integer code.
#pragma once
#include "common.h"

namespace purine {
namespace {

int64_t numel(const purine_tensor* t) {
    int64_t n = 1;
    for (int i = 0; i < t->ndim; ++i) n *= t->dim[i];
    return n;
}

// elements of one image (all axes but the first)
int64_t image_elems(const purine_tensor* t) {
    int64_t n = 1;
    for (int i = 1; i < t->ndim; ++i) n *= t->dim[i];
    return n;
}
// elements between consecutive images: the dense distance unless the tensor is a channel-slice view
int64_t nstride_of(const purine_tensor* t) {
    return (t->ndim == 4 && t->nstride != 0) ? t->nstride : image_elems(t);
}
bool is_view(const purine_tensor* t) { return nstride_of(t) != image_elems(t); }
// elements from the first to one past the last element of the tensor
int64_t span_elems(const purine_tensor* t) { return (t->dim[0] - 1) * nstride_of(t) + image_elems(t); }

static bool is_float_dtype_(int d) { return d == PURINE_F32 || d == PURINE_BF16; }
// allow_view: the argument may be a channel-slice view (F32 or BF16, 4 axes)
int check_tensor(const purine_tensor* t, int ndim, bool allow_view = false) {
    if (!t) return PURINE_E_NULL;
    if (!t->data) return PURINE_E_NULL;
    if (t->ndim != ndim) return PURINE_E_SHAPE;
    if (t->dtype != PURINE_F32 && t->dtype != PURINE_BF16 && t->dtype != PURINE_I32) return PURINE_E_DTYPE;
    int64_t n = 1;
    for (int i = 0; i < ndim; ++i) {
        if (t->dim[i] < 1) return PURINE_E_SHAPE;
        if (t->dim[i] >= (1ll << 31)) return PURINE_E_SHAPE;
        n *= t->dim[i];
        if (n >= (1ll << 31)) return PURINE_E_SHAPE;
    }
    if (((uintptr_t)t->data) & 15u) return PURINE_E_LAYOUT;
    if (t->nstride != 0) {
        if (t->ndim != 4 || t->nstride < image_elems(t)) return PURINE_E_SHAPE;
        if (is_view(t)) {
            // images keep the 16-byte alignment of the vector loads and stores: 4 floats, 8 bfloat16
            const int64_t packet = t->dtype == PURINE_BF16 ? 7 : 3;
            if (!allow_view || !is_float_dtype_(t->dtype) || (t->nstride & packet)) return PURINE_E_LAYOUT;
            if (t->nstride >= (1ll << 31) || span_elems(t) >= (1ll << 31)) return PURINE_E_SHAPE;
        }
    }
    return PURINE_OK;
}

bool is_float_dtype(int d) { return d == PURINE_F32 || d == PURINE_BF16; }
size_t elem_bytes(int d) { return d == PURINE_BF16 ? 2 : 4; }

// Do the two tensors share a byte? Exact for dense tensors; for two views with the same distance
// between images the per-image ranges are compared modulo that distance (channel slices of one
// buffer); anything else falls back to the spans.
bool overlaps(const purine_tensor* a, const purine_tensor* b) {
    const uintptr_t a0 = (uintptr_t)a->data, a1 = a0 + (size_t)span_elems(a) * elem_bytes(a->dtype);
    const uintptr_t b0 = (uintptr_t)b->data, b1 = b0 + (size_t)span_elems(b) * elem_bytes(b->dtype);
    if (!(a0 < b1 && b0 < a1)) return false;
    const uint64_t sa = (uint64_t)nstride_of(a) * elem_bytes(a->dtype), sb = (uint64_t)nstride_of(b) * elem_bytes(b->dtype);
    if (is_view(a) && is_view(b) && sa == sb) {
        const uint64_t la = (uint64_t)image_elems(a) * elem_bytes(a->dtype), lb = (uint64_t)image_elems(b) * elem_bytes(b->dtype);
        const uint64_t d = a0 >= b0 ? (a0 - b0) % sa : (sa - (b0 - a0) % sa) % sa;   // (a0 - b0) mod s
        return d < lb || sa - d < la;
    }
    return true;
}

bool same_dims(const purine_tensor* a, const purine_tensor* b) {
    if (a->ndim != b->ndim) return false;
    for (int i = 0; i < a->ndim; ++i)
        if (a->dim[i] != b->dim[i]) return false;
    return true;
}

int check_beta(float beta) { return (beta == 0.0f || beta == 1.0f) ? PURINE_OK : PURINE_E_ARG; }

}  // namespace
}  // namespace purine
