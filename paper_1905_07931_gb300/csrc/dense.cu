// Dense layers: forward product with bias, activation and residual in its epilogue, the two backward products, the
// elementwise act' and the weight update (include/csrtrain.h). The products run on gemm16_kernel (gemm16.cuh).
#include <cmath>

#include "dense_tokens.cuh"
#include "gemm16_host.cuh"

namespace csrt {
// The kernels' instances are compiled in dense_gemm_fwd.cu and dense_gemm_bwd.cu.
int dense_gemm_fwd(const GProduct &p, const GArgs &a, bool wide, cudaStream_t s);
int dense_gemm_bwd(const GProduct &p, const GArgs &a, bool wide, cudaStream_t s);
}  // namespace csrt

namespace csrt {

// ---------------------------------------------------------------------------
// Copy of an operand whose rows are not 16-byte aligned into padded rows. A thread takes the eight elements of an
// aligned 16-byte store out of the one or two aligned 16-byte words that hold them (as long as those lie within the
// matrix); short rows share a block. 4096 x 1777 adds 6.8 us to a product, 9216 x 5 2.
// ---------------------------------------------------------------------------
__global__ void pack16_kernel(const uint16_t *__restrict__ src, int64_t ld, int32_t rows, int32_t cols,
                              uint16_t *__restrict__ dst, int64_t dld) {
    pdl_enter();
    const uintptr_t first = reinterpret_cast<uintptr_t>(src);
    const uintptr_t end = reinterpret_cast<uintptr_t>(src + (int64_t)(rows - 1) * ld + cols);
    for (int64_t r = (int64_t)blockIdx.y * blockDim.y + threadIdx.y; r < rows; r += (int64_t)gridDim.y * blockDim.y)
        for (int64_t c = ((int64_t)blockIdx.x * blockDim.x + threadIdx.x) * 8; c < cols; c += (int64_t)gridDim.x * blockDim.x * 8) {
            const uint16_t *p = src + r * ld + c;
            const int count = (int)imin<int64_t>(cols - c, 8);
            const uintptr_t at = reinterpret_cast<uintptr_t>(p), word = at & ~(uintptr_t)15;
            const bool two = (at & 15) + 2 * count > 16;
            uint4 u;
            if (word >= first && word + (two ? 32 : 16) <= end) {
                const uint4 lo = __ldg(reinterpret_cast<const uint4 *>(word));
                const uint4 hi = two ? __ldg(reinterpret_cast<const uint4 *>(word) + 1) : make_uint4(0, 0, 0, 0);
                u = eight_at(lo, hi, (uint32_t)(at & 15));
            } else {
                u = eight_singly(p, count);
            }
            *reinterpret_cast<uint4 *>(dst + r * dld + c) = u;
        }
}

// Operand of a product: in place, or packed at *at (advanced).
static int operand(const csrt_mat *m, char **at, cudaStream_t s, GOperand *o) {
    o->p = m->data;
    o->rows = m->rows;
    o->cols = m->cols;
    o->ld = m->ld;
    if (tma_rows_ok(m->data, m->ld, 2) || m->rows == 0 || m->cols == 0) return CSRT_OK;   // (an empty one is not read)
    o->ld = (int64_t)align_up((size_t)m->cols, 8);
    o->p = *at;
    *at += align_up((size_t)m->rows * o->ld * 2, 256);
    unsigned bx = 1;   // threads along a row: a block of 256 takes several short rows
    while (bx < 256 && (int64_t)bx * 8 < m->cols) bx *= 2;
    const unsigned gx = (unsigned)imin<int64_t>(ceil_div<int64_t>(m->cols, 8 * bx), 64);
    const unsigned gy = (unsigned)imin<int64_t>(ceil_div<int64_t>(m->rows, 256 / bx), 65535);
    launch_pdl(pack16_kernel, dim3(gx, gy), dim3(bx, 256 / bx), 0, s, static_cast<const uint16_t *>(m->data), m->ld, m->rows,
               m->cols, static_cast<uint16_t *>(o->p), o->ld);
    count_launch();
    return check_launch("pack16_kernel");
}

static GMat epi_mat(const csrt_mat *m) {
    GMat g = {};
    if (m == nullptr) return g;
    g.p = m->data;
    g.ld = m->ld;
    g.dtype = m->dtype;
    g.vec = tma_rows_ok(m->data, m->ld, dt_size(m->dtype));
    return g;
}

static GMat out_mat(const csrt_mat *m) {
    GMat g = epi_mat(m);
    g.vec = m != nullptr && tma_store_ok(m->data, m->ld, m->cols, dt_size(m->dtype));
    return g;
}

static char *operand_space(void *ws) { return ws_scratch(ws) + kPartialBytes; }

// D = A B^T with the epilogue of the forward (kEpiFwd) or the backward products; `at`: the workspace's space for operands.
template <int EPI>
static int dense_product(const csrt_mat *am, bool a_mn, const csrt_mat *bm, bool b_mn, GArgs a, csrt_mat *out0,
                         csrt_mat *out1, void *ws, char *at, cudaStream_t s) {
    GProduct p;
    CSRT_TRY(operand(am, &at, s, &p.a));
    CSRT_TRY(operand(bm, &at, s, &p.b));
    p.a_mn = a_mn;
    p.b_mn = b_mn;
    a.f16 = am->dtype == CSRT_DT_F16;
    a.m = out0->rows;
    a.n = out0->cols;
    a.batch = 1;
    a.out0 = out_mat(out0);
    a.out1 = out_mat(out1);
    // a staging slot holds two aligned 16-bit blocks, or one block of any other kind
    if (out1 != nullptr && (out0->dtype == CSRT_DT_F32 || !a.out0.vec || !a.out1.vec)) a.out0.vec = a.out1.vec = 0;
    a.hdr = static_cast<WsHeader *>(ws);
    a.counters = ws_counters(ws);
    a.partial = reinterpret_cast<float *>(ws_scratch(ws));
    p.reduction = a_mn ? am->rows : am->cols;
    const bool wide = out0->dtype == CSRT_DT_F32;
    return EPI == kEpiFwd ? dense_gemm_fwd(p, a, wide, s) : dense_gemm_bwd(p, a, wide, s);
}

// ---------------------------------------------------------------------------
// Row sums (db), act' and update
// ---------------------------------------------------------------------------
// A warp per row.
template <bool F16>
__global__ void row_sums_kernel(const uint16_t *__restrict__ dy, int64_t ld, int32_t rows, int32_t cols, bool accumulate,
                                float *__restrict__ db) {
    pdl_enter();
    const int warps = blockDim.x >> 5, lane = threadIdx.x & 31;
    for (int64_t r = (int64_t)blockIdx.x * warps + (threadIdx.x >> 5); r < rows; r += (int64_t)gridDim.x * warps) {
        const float t = warp_row_sum<F16>(dy + r * ld, cols);
        if (lane == 0) db[r] = accumulate ? db[r] + t : t;
    }
}

// An element at a time, 2 or 4 bytes an access: 4096 x 256 takes 9.0 us with gelu' on bfloat16 and 6.6 to convert, 4096 x
// 9216 297 and 160 (33 at the measured copy rate for the former).
__global__ void act_bwd_kernel(GMat dy, GMat z, int32_t act, GMat out, int32_t rows, int32_t cols) {
    pdl_enter();
    for (int64_t r = blockIdx.y; r < rows; r += gridDim.y)
        for (int64_t c = (int64_t)blockIdx.x * blockDim.x + threadIdx.x; c < cols; c += (int64_t)gridDim.x * blockDim.x) {
            float v = load1(dy.p, r * dy.ld + c, dy.dtype);
            if (act != CSRT_ACT_NONE) v *= act_deriv(load1(z.p, r * z.ld + c, z.dtype), act);
            store1(out.p, r * out.ld + c, v, out.dtype);
        }
}

// As act_bwd_kernel: 4096 x 9216 with a float32 direction and a bfloat16 copy takes 139 us (528 MB, 78 at the measured copy
// rate), 4096 x 256 6.8.
__global__ void dense_update_kernel(GMat w, GMat d, float eta, float keep, GMat w16, int32_t rows, int32_t cols) {
    pdl_enter();
    float *wp = static_cast<float *>(w.p);
    for (int64_t r = blockIdx.y; r < rows; r += gridDim.y)
        for (int64_t c = (int64_t)blockIdx.x * blockDim.x + threadIdx.x; c < cols; c += (int64_t)gridDim.x * blockDim.x) {
            const float v = __fsub_rn(__fmul_rn(wp[r * w.ld + c], keep), __fmul_rn(eta, load1(d.p, r * d.ld + c, d.dtype)));
            wp[r * w.ld + c] = v;
            if (w16.p != nullptr) store1(w16.p, r * w16.ld + c, v, w16.dtype);
        }
}

static dim3 elementwise_grid(int32_t rows, int32_t cols) {
    const unsigned gx = (unsigned)imin<int64_t>(ceil_div<int64_t>(cols, 256), 4096);
    const unsigned gy = (unsigned)imin<int64_t>(rows, imax<int64_t>(1, imin<int64_t>(65535, (int64_t)num_sms() * 64 / gx)));
    return dim3(gx, gy);
}

static size_t operand_bytes(int64_t rows, int64_t cols) { return align_up((size_t)(rows * ((cols + 7) / 8 * 8) * 2), 256); }

static size_t dense_bytes(int64_t m, int64_t k, int64_t n) {
    return kWsReservedBytes + kPartialBytes + operand_bytes(m, k) + operand_bytes(m, n) + operand_bytes(k, n);
}

static int check_call(const csrt_mat *a, const char *an, const csrt_mat *b, const char *bn, int32_t m, int32_t k,
                      int32_t n, const void *ws, size_t ws_bytes) {
    CSRT_ARG(a->dtype != CSRT_DT_F32 && a->dtype == b->dtype, "%s and %s must have one 16-bit type", an, bn);
    CSRT_ARG(ws != nullptr, "workspace is NULL");
    CSRT_ARG((reinterpret_cast<uintptr_t>(ws) & 255) == 0, "workspace is not 256-byte aligned");
    if (ws_bytes < dense_bytes(m, k, n))
        return fail(CSRT_ERR_WORKSPACE, "workspace has %zu bytes, needs %zu", ws_bytes, dense_bytes(m, k, n));
    return CSRT_OK;
}

static int check_out(const csrt_mat *o, const char *name, int32_t dtype) {
    CSRT_ARG(o->dtype == CSRT_DT_F32 || o->dtype == dtype, "%s must be float32 or of the operands' type", name);
    return CSRT_OK;
}

}  // namespace csrt

using namespace csrt;

extern "C" {

int csrt_dense_workspace_bytes(int32_t m, int32_t k, int32_t max_n, size_t *bytes) {
    CSRT_ARG(bytes != nullptr, "bytes is NULL");
    CSRT_ARG(m >= 0 && k >= 0 && max_n >= 0, "negative size");
    *bytes = dense_bytes(m, k, max_n);
    return CSRT_OK;
}

int csrt_dense_fwd(const csrt_mat *w, const csrt_mat *x, const float *bias, int32_t act, const csrt_mat *residual,
                   csrt_mat *z, csrt_mat *y, void *ws, size_t ws_bytes, void *stream) {
    CSRT_TRY(check_mat(w, "w"));
    CSRT_TRY(check_mat(x, "x"));
    CSRT_TRY(check_mat(y, "y"));
    const int32_t m = w->rows, k = w->cols, n = x->cols;
    CSRT_TRY(check_shape(x, "x", k, n));
    CSRT_TRY(check_shape(y, "y", m, n));
    CSRT_ARG(act >= CSRT_ACT_NONE && act <= CSRT_ACT_SILU, "unknown activation %d", act);
    CSRT_TRY(check_call(w, "w", x, "x", m, k, n, ws, ws_bytes));
    CSRT_TRY(check_out(y, "y", w->dtype));
    if (residual != nullptr) {
        CSRT_TRY(check_mat(residual, "residual"));
        CSRT_TRY(check_shape(residual, "residual", m, n));
        CSRT_ARG(residual->dtype == y->dtype, "residual must have y's type");
        CSRT_ARG(same_place(residual, y) || !clash(y, residual), "y overlaps residual");
    }
    if (z != nullptr) {
        CSRT_TRY(check_mat(z, "z"));
        CSRT_TRY(check_shape(z, "z", m, n));
        CSRT_ARG(z->dtype == w->dtype, "z must have w's type");
        CSRT_ARG(!clash(z, y) && !clash(z, x) && !clash(z, w) && (residual == nullptr || !clash(z, residual)),
                 "z overlaps another matrix");
    }
    CSRT_TRY(check_vector(bias, "bias"));
    CSRT_ARG(!vector_meets(bias, m, y), "bias overlaps y");
    CSRT_ARG(z == nullptr || !vector_meets(bias, m, z), "bias overlaps z");
    CSRT_ARG(!clash(y, x) && !clash(y, w), "y overlaps an operand");
    if (m == 0 || n == 0) return CSRT_OK;
    // One to four tokens stream W past x, unless x has gaps between its rows (columns of a wider buffer): W is then read two
    // bytes a lane and x by a cache line for each element, which the tensor cores overtake once the product is large enough
    // to pay for their fixed cost and for the copy of an x that TMA cannot take (us, stream / tensor cores: x in rows of 64,
    // 1000 x 1024 one token 5.1 / 7.6, 4096 x 1024 one 10.7 / 7.8, 4096 x 4096 one 32 / 12, four 132 / 12; in rows of 61,
    // 1000 x 4096 four 13.4 / 11.7, 4096 x 2048 two 11.9 / 12.6, 4096 x 4096 two 22 / 14). With W to be copied too the
    // stream stays (4096 x 4097, one token: 16 to 32 / 26 to 29).
    const int64_t terms = (int64_t)m * k * n;
    const bool gaps = x->ld != n && tma_rows_ok(w->data, w->ld, 2) &&
                      terms >= (int64_t)1 << (tma_rows_ok(x->data, x->ld, 2) ? 22 : 25);
    if (n <= kTokensMax && !gaps) {
        TokenArgs t = {};
        t.w = static_cast<const uint16_t *>(w->data);
        t.x = static_cast<const uint16_t *>(x->data);
        t.ldw = w->ld;
        t.ldx = x->ld;
        t.m = m;
        t.k = k;
        t.bias = bias;
        t.act = act;
        t.res = epi_mat(residual);
        t.z = epi_mat(z);
        t.y = epi_mat(y);
        const bool vec = k % 8 == 0 && tma_rows_ok(w->data, w->ld, 2) && x->ld == n &&
                         (reinterpret_cast<uintptr_t>(x->data) & 15) == 0;
        return dense_tokens(t, n, w->dtype == CSRT_DT_F16, vec, as_stream(stream));
    }
    GArgs a = {};
    a.bias = bias;
    a.act = act;
    a.c1 = epi_mat(residual);
    return dense_product<kEpiFwd>(w, false, x, true, a, y, z, ws, operand_space(ws), as_stream(stream));
}

int csrt_dense_bwd_x(const csrt_mat *w, const csrt_mat *dy, const csrt_mat *z_below, int32_t act,
                     const csrt_mat *residual, csrt_mat *dx, void *ws, size_t ws_bytes, void *stream) {
    CSRT_TRY(check_mat(w, "w"));
    CSRT_TRY(check_mat(dy, "dy"));
    CSRT_TRY(check_mat(dx, "dx"));
    const int32_t m = w->rows, k = w->cols, n = dy->cols;
    CSRT_TRY(check_shape(dy, "dy", m, n));
    CSRT_TRY(check_shape(dx, "dx", k, n));
    CSRT_ARG(act >= CSRT_ACT_NONE && act <= CSRT_ACT_SILU, "unknown activation %d", act);
    CSRT_TRY(check_call(w, "w", dy, "dy", m, k, n, ws, ws_bytes));
    CSRT_TRY(check_out(dx, "dx", w->dtype));
    CSRT_ARG(z_below != nullptr || act == CSRT_ACT_NONE, "an activation needs z_below");
    if (z_below != nullptr) {
        CSRT_TRY(check_mat(z_below, "z_below"));
        CSRT_TRY(check_shape(z_below, "z_below", k, n));
        CSRT_ARG(z_below->dtype == w->dtype, "z_below must have w's type");
        CSRT_ARG(!clash(dx, z_below), "dx overlaps z_below");
    }
    if (residual != nullptr) {
        CSRT_TRY(check_mat(residual, "residual"));
        CSRT_TRY(check_shape(residual, "residual", k, n));
        CSRT_ARG(residual->dtype == dx->dtype, "residual must have dx's type");
        CSRT_ARG(same_place(residual, dx) || !clash(dx, residual), "dx overlaps residual");
    }
    CSRT_ARG(!clash(dx, dy) && !clash(dx, w), "dx overlaps an operand");
    if (k == 0 || n == 0) return CSRT_OK;
    GArgs a = {};
    a.act = act;
    if (act != CSRT_ACT_NONE) a.c0 = epi_mat(z_below);
    a.c1 = epi_mat(residual);
    return dense_product<kEpiBwd>(w, true, dy, true, a, dx, nullptr, ws, operand_space(ws), as_stream(stream));
}

int csrt_dense_bwd_w(const csrt_mat *dy, const csrt_mat *x, int32_t accumulate, csrt_mat *dw, float *db, void *ws,
                     size_t ws_bytes, void *stream) {
    CSRT_TRY(check_mat(dy, "dy"));
    CSRT_TRY(check_mat(x, "x"));
    CSRT_TRY(check_mat(dw, "dw"));
    const int32_t m = dy->rows, k = x->rows, n = dy->cols;
    CSRT_TRY(check_shape(x, "x", k, n));
    CSRT_TRY(check_shape(dw, "dw", m, k));
    CSRT_TRY(check_call(dy, "dy", x, "x", m, k, n, ws, ws_bytes));
    CSRT_TRY(check_out(dw, "dw", dy->dtype));
    CSRT_ARG(!clash(dw, dy) && !clash(dw, x), "dw overlaps an operand");
    CSRT_TRY(check_vector(db, "db"));
    CSRT_ARG(!vector_meets(db, m, dw), "db overlaps dw");
    CSRT_ARG(!vector_meets(db, m, dy), "db overlaps dy");
    CSRT_ARG(!vector_meets(db, m, x), "db overlaps x");
    cudaStream_t s = as_stream(stream);
    GArgs a = {};
    if (accumulate) a.c1 = epi_mat(dw);
    // dy's rows as the product takes them, in place or copied to aligned ones: the row sums read no others. (Read two bytes
    // at a time beside the product they outlasted it: 4096 x 4096 from 777 columns 38 us without db, 52 with it.)
    csrt_mat d = *dy;
    char *at = operand_space(ws);
    GOperand rows;
    CSRT_TRY(operand(dy, &at, s, &rows));
    d.data = rows.p;
    d.ld = rows.ld;
    if (db != nullptr && m > 0) {
        const uint16_t *p = static_cast<const uint16_t *>(d.data);
        // The product's idle warps take the row sums along (two warps an SM, about 3 KB/us each, against a kernel of
        // its own at HBM rate and a launch of 3 us) unless they would outlast it.
        bool along = false;
        if (k > 0) {
            GArgs t = {};
            t.m = m;
            t.n = k;
            t.batch = 1;
            t.out0 = out_mat(dw);
            t.c1 = a.c1;
            const GChoice c = choose_tile(t, n, aligned_set(t, dw->dtype == CSRT_DT_F32));
            const int64_t units = ceil_div<int64_t>(m, 128 * kTiles[c.tile].cg) * ceil_div<int64_t>(k, kTiles[c.tile].bn) *
                                  c.split.splits * kTiles[c.tile].cg;
            const double us = (double)m * n * 2 / (2.0 * imin<int64_t>(units, num_sms()) * 3000.0);
            along = us <= imax(c.split.us, 4.0);
        }
        if (along) {
            a.sum_src = p;
            a.sum_ld = d.ld;
            a.sum_rows = m;
            a.sum_cols = n;
            a.sum_add = accumulate != 0;
            a.sum_dst = db;
        } else {
            const dim3 grid((unsigned)imin<int64_t>(ceil_div<int64_t>(m, 4), (int64_t)num_sms() * 16)), block(128);
            if (dy->dtype == CSRT_DT_F16)
                launch_pdl(row_sums_kernel<true>, grid, block, 0, s, p, d.ld, m, n, accumulate != 0, db);
            else
                launch_pdl(row_sums_kernel<false>, grid, block, 0, s, p, d.ld, m, n, accumulate != 0, db);
            count_launch();
            CSRT_TRY(check_launch("row_sums_kernel"));
        }
    }
    if (m == 0 || k == 0) return CSRT_OK;
    return dense_product<kEpiBwd>(&d, false, x, false, a, dw, nullptr, ws, at, s);
}

int csrt_dense_act_bwd(const csrt_mat *dy, const csrt_mat *z, int32_t act, csrt_mat *dpre, void *stream) {
    CSRT_TRY(check_mat(dy, "dy"));
    CSRT_TRY(check_mat(dpre, "dpre"));
    CSRT_ARG(act >= CSRT_ACT_NONE && act <= CSRT_ACT_SILU, "unknown activation %d", act);
    CSRT_TRY(check_shape(dpre, "dpre", dy->rows, dy->cols));
    CSRT_ARG(same_place(dy, dpre) || !clash(dpre, dy), "dpre overlaps dy");
    if (act != CSRT_ACT_NONE) {
        CSRT_TRY(check_mat(z, "z"));
        CSRT_TRY(check_shape(z, "z", dy->rows, dy->cols));
        CSRT_ARG(!clash(dpre, z), "dpre overlaps z");
    }
    if (dy->rows == 0 || dy->cols == 0) return CSRT_OK;
    launch_pdl(act_bwd_kernel, elementwise_grid(dy->rows, dy->cols), dim3(256), 0, as_stream(stream), epi_mat(dy),
               act == CSRT_ACT_NONE ? GMat{} : epi_mat(z), act, epi_mat(dpre), dy->rows, dy->cols);
    count_launch();
    return check_launch("act_bwd_kernel");
}

int csrt_dense_update(csrt_mat *w, const csrt_mat *d, float eta, float decay, csrt_mat *w16, void *stream) {
    CSRT_TRY(check_mat(w, "w"));
    CSRT_TRY(check_mat(d, "d"));
    CSRT_ARG(w->dtype == CSRT_DT_F32, "w must be float32");
    CSRT_TRY(check_shape(d, "d", w->rows, w->cols));
    CSRT_ARG(std::isfinite(eta) && std::isfinite(decay) && eta >= 0.f && decay >= 0.f, "eta and decay must be finite and >= 0");
    CSRT_ARG(!clash(w, d), "w overlaps d");
    if (w16 != nullptr) {
        CSRT_TRY(check_mat(w16, "w16"));
        CSRT_TRY(check_shape(w16, "w16", w->rows, w->cols));
        CSRT_ARG(!clash(w16, d) && !clash(w16, w), "w16 overlaps another matrix");
    }
    if (w->rows == 0 || w->cols == 0) return CSRT_OK;
    const float keep = 1.f - eta * decay;
    launch_pdl(dense_update_kernel, elementwise_grid(w->rows, w->cols), dim3(256), 0, as_stream(stream), epi_mat(w),
               epi_mat(d), eta, keep, epi_mat(w16), w->rows, w->cols);
    count_launch();
    return check_launch("dense_update_kernel");
}

}  // extern "C"
