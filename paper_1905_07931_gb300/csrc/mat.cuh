// Host checks of csrt_mat arguments, shared by the calls that take them.
#pragma once

#include "common.cuh"

namespace csrt {

inline int dt_size(int dtype) { return dtype == CSRT_DT_F32 ? 4 : 2; }

// Rows that TMA (and 16-byte vector access) can take in place.
inline bool tma_rows_ok(const void *p, int64_t ld, int size) {
    return (reinterpret_cast<uintptr_t>(p) & 15) == 0 && ld * size % 16 == 0;
}

constexpr int64_t kMaxElems = (int64_t)1 << 40;   // largest matrix extent taken (rows x ld)

inline size_t align_up(size_t v, size_t a) { return (v + a - 1) / a * a; }

inline int check_mat(const csrt_mat *m, const char *name) {
    CSRT_ARG(m != nullptr, "%s is NULL", name);
    CSRT_ARG(m->rows >= 0 && m->cols >= 0, "%s: negative size", name);
    CSRT_ARG(m->ld >= m->cols && (m->rows == 0 || m->ld < kMaxElems / ((int64_t)m->rows + 1)), "%s: bad ld", name);
    CSRT_ARG(m->dtype == CSRT_DT_F32 || m->dtype == CSRT_DT_BF16 || m->dtype == CSRT_DT_F16, "%s: unknown dtype", name);
    CSRT_ARG(m->data != nullptr || m->rows == 0 || m->cols == 0, "%s: data is NULL", name);
    CSRT_ARG(reinterpret_cast<uintptr_t>(m->data) % dt_size(m->dtype) == 0, "%s: data is not aligned to its type", name);
    return CSRT_OK;
}

inline int check_shape(const csrt_mat *m, const char *name, int32_t rows, int32_t cols) {
    CSRT_ARG(m->rows == rows && m->cols == cols, "%s is %d x %d, must be %d x %d", name, m->rows, m->cols, rows, cols);
    return CSRT_OK;
}

#define CSRT_TRY(call)                  \
    do {                                \
        const int rc_ = (call);         \
        if (rc_ != CSRT_OK) return rc_; \
    } while (0)

inline bool overlap(const csrt_mat *a, const csrt_mat *b) {
    if (a == nullptr || b == nullptr || a->rows == 0 || b->rows == 0 || a->cols == 0 || b->cols == 0) return false;
    const char *pa = static_cast<const char *>(a->data), *pb = static_cast<const char *>(b->data);
    const int64_t la = ((a->rows - 1) * a->ld + a->cols) * dt_size(a->dtype);
    const int64_t lb = ((b->rows - 1) * b->ld + b->cols) * dt_size(b->dtype);
    return pa < pb + lb && pb < pa + la;
}
inline bool same_place(const csrt_mat *a, const csrt_mat *b) {
    return a->data == b->data && a->ld == b->ld && a->dtype == b->dtype;
}

// Columns of an interleaved buffer may share its extent without sharing elements: only what an output and an input
// both name counts, so outputs are checked as whole extents except where rows interleave (equal ld).
inline bool clash(const csrt_mat *out, const csrt_mat *in) {
    if (!overlap(out, in)) return false;
    if (out->ld == in->ld && out->dtype == in->dtype) {
        const int64_t d = (static_cast<const char *>(in->data) - static_cast<const char *>(out->data)) /
                          (int64_t)dt_size(out->dtype);
        const int64_t c = ((d % out->ld) + out->ld) % out->ld;   // first column of `in` within out's rows
        return c < out->cols || c + in->cols > out->ld;
    }
    return true;
}

// Whether a float32 vector of n elements (may be NULL) shares bytes with a matrix's elements: it may lie between two rows.
inline bool vector_meets(const float *v, int64_t n, const csrt_mat *m) {
    csrt_mat flat = {};
    flat.data = const_cast<float *>(v);
    flat.rows = 1;
    flat.cols = (int32_t)n;
    flat.ld = n;
    flat.dtype = CSRT_DT_F32;
    if (v == nullptr || !overlap(m, &flat)) return false;
    const int64_t row = m->ld * dt_size(m->dtype), used = m->cols * (int64_t)dt_size(m->dtype);
    const int64_t d = reinterpret_cast<const char *>(v) - static_cast<const char *>(m->data);
    return d < 0 || d % row < used || d % row + n * 4 > row;
}
inline int check_vector(const float *v, const char *name) {
    CSRT_ARG(reinterpret_cast<uintptr_t>(v) % 4 == 0, "%s is not aligned to its type", name);
    return CSRT_OK;
}

}  // namespace csrt
