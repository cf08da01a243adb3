// The norms before and after a block of a residual network, its gate and the scaled residual, and their backward pass
// (csrt_block_norm_fwd, csrt_block_norm_bwd):
//   t = post(y),  h = r_scale r + a(g) t,  v = pre(h)
// Activations are d x n with the token index contiguous, so a norm reduces down the columns. All of it is bound by HBM
// traffic: a few tens of operations for 8 to 20 bytes.
#include <cmath>
#include <initializer_list>

#include "block_norm.cuh"
#include "mat.cuh"

namespace csrt {

// ---------------------------------------------------------------------------
// Columns of any length: a block takes 32 tokens, a lane each, its warps every 16th feature, and reads its inputs again
// for every sum it needs (mean and mean square deviation of y, then of h, which is computed anew each time).
// ---------------------------------------------------------------------------
constexpr int kColWarps = 16;

// The sum over all features of value(i) for this lane's token; every thread gets it. Runs of 64 are summed apart.
template <typename F>
__device__ __forceinline__ float column_sum(int32_t d, float (&part)[kColWarps][32], F value) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    float total = 0.f;
    for (int64_t i0 = warp; i0 < d; i0 += 64 * kColWarps) {
        float run = 0.f;
        for (int64_t i = i0; i < imin<int64_t>(d, i0 + 64 * kColWarps); i += kColWarps) run += value(i);
        total += run;
    }
    part[warp][lane] = total;
    __syncthreads();
    total = 0.f;
    for (int w = 0; w < kColWarps; ++w) total += part[w][lane];
    __syncthreads();
    return total;
}

// Statistics of x(i), written by the first warp.
template <typename F>
__device__ __forceinline__ void column_stats(const NormSide &s, int32_t d, int64_t c, bool ok,
                                             float (&part)[kColWarps][32], F x, float &mean, float &rstd) {
    mean = 0.f;
    rstd = 1.f;
    if (s.kind == CSRT_NORM_SCALE || s.kind < 0) return;
    if (s.kind == CSRT_NORM_LAYER) mean = column_sum(d, part, x) / (float)d;
    const float m = mean;
    const float sq = column_sum(d, part, [&](int64_t i) {
        const float v = x(i) - m;
        return v * v;
    });
    rstd = 1.f / sqrtf(sq / (float)d + s.eps);
    if (ok && threadIdx.x < 32) {
        if (s.mean != nullptr && s.kind == CSRT_NORM_LAYER) s.mean[c] = mean;
        if (s.rstd != nullptr) s.rstd[c] = rstd;
    }
}

__device__ __forceinline__ float normed(const NormSide &s, float x, int64_t i, float mean, float rstd) {
    if (s.kind < 0) return x;
    x = (x - mean) * rstd;
    if (s.w != nullptr) x *= __ldg(s.w + i);
    if (s.b != nullptr) x += __ldg(s.b + i);
    return x;
}

template <typename T>
__device__ __forceinline__ float at(const NormMat &m, int64_t i, int64_t c) {
    return to_f<T>(reinterpret_cast<const T *>(m.p)[i * m.ld + c]);
}
template <typename T>
__device__ __forceinline__ void put(const NormMat &m, int64_t i, int64_t c, float v) {
    reinterpret_cast<T *>(m.p)[i * m.ld + c] = from_f<T>(v);
}

template <typename TB, typename TS>
__global__ void __launch_bounds__(kColWarps * 32) norm_fwd_columns_kernel(NormArgs a) {
    pdl_enter();
    __shared__ float part[kColWarps][32];
    constexpr bool kFast = sizeof(TB) == 2;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int64_t c = (int64_t)blockIdx.x * 32 + lane;
    const bool ok = c < a.n;
    float mpost, spost, mpre, spre;
    column_stats(a.post, a.d, c, ok, part, [&](int64_t i) { return ok ? at<TB>(a.y, i, c) : 0.f; }, mpost, spost);
    auto stream = [&](int64_t i) {
        float h = 0.f;
        if (!ok) return h;
        if (a.r.p != nullptr) h = a.r_scale * at<TS>(a.r, i, c);
        if (a.y.p != nullptr) {
            float t = normed(a.post, at<TB>(a.y, i, c), i, mpost, spost);
            if (a.g.p != nullptr) t *= gate_value<kFast>(at<TB>(a.g, i, c), a.gate_act);
            h += t;
        }
        return h;
    };
    column_stats(a.pre, a.d, c, ok, part, stream, mpre, spre);
    if (!ok) return;
    for (int64_t i = warp; i < a.d; i += kColWarps) {
        const float h = stream(i);
        if (a.h.p != nullptr) put<TS>(a.h, i, c, h);   // r may be h: each element is read for the last time just above
        if (a.v.p != nullptr) put<TB>(a.v, i, c, normed(a.pre, h, i, mpre, spre));
    }
}

// Backward: with xh = (x - mean) rstd and s = weight * dout,
//   dx = rstd (s - xh mean(s xh) - [layer] mean(s)),  dweight = sum over tokens of dout xh,  dbias = of dout.
// The sums over a block's tokens are kept in its own rows of `partial`.
struct ColumnGrad {
    float along, ones;   // mean(s xh), mean(s)
};
template <typename F, typename G>
__device__ __forceinline__ ColumnGrad column_grad(const NormSide &s, int32_t d, float (&part)[kColWarps][32], F dout, G hat) {
    ColumnGrad r = {0.f, 0.f};
    if (s.kind == CSRT_NORM_SCALE || s.kind < 0) return r;
    auto scaled = [&](int64_t i) { return s.w != nullptr ? __ldg(s.w + i) * dout(i) : dout(i); };
    r.along = column_sum(d, part, [&](int64_t i) { return scaled(i) * hat(i); }) / (float)d;
    if (s.kind == CSRT_NORM_LAYER) r.ones = column_sum(d, part, scaled) / (float)d;
    return r;
}
__device__ __forceinline__ float input_grad(const NormSide &s, float dout, float hat, int64_t i, float rstd, const ColumnGrad &g) {
    if (s.kind < 0) return dout;
    const float u = s.w != nullptr ? __ldg(s.w + i) * dout : dout;
    return s.kind == CSRT_NORM_SCALE ? u : rstd * (u - hat * g.along - g.ones);
}
__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
    for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}

template <typename TB, typename TS>
__global__ void __launch_bounds__(kColWarps * 32) norm_bwd_columns_kernel(NormArgs a) {
    pdl_enter();
    __shared__ float part[kColWarps][32];
    constexpr bool kFast = sizeof(TB) == 2;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const NormSide &post = a.post, &pre = a.pre;
    const bool sums = post.dw != nullptr || post.db != nullptr || pre.dw != nullptr || pre.db != nullptr;
    float *mine = sums ? a.partial + (int64_t)blockIdx.x * 4 * a.d : nullptr;
    bool first = true;
    for (int64_t c0 = (int64_t)blockIdx.x * 32; c0 < a.n; c0 += (int64_t)a.groups * 32, first = false) {
        const int64_t c = c0 + lane;
        const bool ok = c < a.n;
        const float mpre = ok && pre.kind == CSRT_NORM_LAYER ? pre.mean[c] : 0.f;
        const float spre = ok && pre.kind > CSRT_NORM_SCALE ? pre.rstd[c] : 1.f;
        const float mpost = ok && post.kind == CSRT_NORM_LAYER ? post.mean[c] : 0.f;
        const float spost = ok && post.kind > CSRT_NORM_SCALE ? post.rstd[c] : 1.f;
        auto dv = [&](int64_t i) { return ok && a.dv.p != nullptr ? at<TB>(a.dv, i, c) : 0.f; };
        auto hhat = [&](int64_t i) { return ok && a.h.p != nullptr ? (at<TS>(a.h, i, c) - mpre) * spre : 0.f; };
        auto yhat = [&](int64_t i) { return ok && a.y.p != nullptr ? (at<TB>(a.y, i, c) - mpost) * spost : 0.f; };
        const ColumnGrad gpre = column_grad(pre, a.d, part, dv, hhat);
        auto dh = [&](int64_t i) {
            float u = ok && a.r.p != nullptr ? at<TS>(a.r, i, c) : 0.f;
            if (a.dv.p != nullptr) u += input_grad(pre, dv(i), hhat(i), i, spre, gpre);
            return u;
        };
        auto dt = [&](int64_t i) {
            return !ok ? 0.f : a.g.p != nullptr ? dh(i) * gate_value<kFast>(at<TB>(a.g, i, c), a.gate_act) : dh(i);
        };
        const ColumnGrad gpost = column_grad(post, a.d, part, dt, yhat);
        for (int64_t i = warp; i < a.d; i += kColWarps) {
            float du = dh(i), u = du;
            const float yh = yhat(i), v = dv(i), hh = hhat(i);
            if (!ok) du = u = 0.f;
            if (ok && a.g.p != nullptr) {
                float value, slope;
                gate_both<kFast>(at<TB>(a.g, i, c), a.gate_act, value, slope);
                if (a.dg.p != nullptr) {
                    float t = yh;
                    if (post.kind >= 0 && post.w != nullptr) t *= __ldg(post.w + i);
                    if (post.kind >= 0 && post.b != nullptr) t += __ldg(post.b + i);
                    put<TB>(a.dg, i, c, du * t * slope);
                }
                u *= value;
            }
            if (ok && a.dy.p != nullptr) put<TB>(a.dy, i, c, input_grad(post, u, yh, i, spost, gpost));
            if (ok && a.dr.p != nullptr) put<TS>(a.dr, i, c, a.r_scale * du);   // dh may be dr: read above
            if (sums) {
                const float q[4] = {warp_sum(ok ? u * yh : 0.f), warp_sum(u), warp_sum(ok ? v * hh : 0.f), warp_sum(v)};
                if (lane == 0)
                    for (int k = 0; k < 4; ++k) mine[(int64_t)k * a.d + i] = first ? q[k] : mine[(int64_t)k * a.d + i] + q[k];
            }
        }
    }
}

// dweight and dbias: the groups' row sums, added in order. A block takes 32 features, its warps every eighth group.
__global__ void __launch_bounds__(256) norm_sums_kernel(NormArgs a) {
    pdl_enter();
    __shared__ float part[8][32];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int64_t i = (int64_t)blockIdx.x * 32 + lane;
    float *out[4] = {a.post.dw, a.post.db, a.pre.dw, a.pre.db};
    float *dst = out[blockIdx.y];
    if (dst == nullptr) return;
    float s = 0.f;
    if (i < a.d)
#pragma unroll 8
        for (int g = warp; g < a.groups; g += 8) s += __ldcg(a.partial + ((int64_t)g * 4 + blockIdx.y) * a.d + i);
    part[warp][lane] = s;
    __syncthreads();
    if (warp != 0 || i >= a.d) return;
    s = 0.f;
#pragma unroll
    for (int w = 0; w < 8; ++w) s += part[w][lane];
    dst[i] = a.accumulate ? dst[i] + s : s;
}

// ---------------------------------------------------------------------------
// Host
// ---------------------------------------------------------------------------
static NormMat norm_mat(const csrt_mat *m) {
    NormMat r = {};
    if (m != nullptr) {
        r.p = static_cast<char *>(m->data);
        r.ld = m->ld;
    }
    return r;
}

static NormSide norm_side(const csrt_norm *s) {
    NormSide r = {};
    r.kind = -1;
    if (s == nullptr) return r;
    r.kind = s->kind;
    r.eps = s->eps;
    r.w = s->weight;
    r.b = s->bias;
    r.mean = s->mean;
    r.rstd = s->rstd;
    r.dw = s->dweight;
    r.db = s->dbias;
    return r;
}

// What a call names, for the checks of overlaps: a matrix or a float32 vector.
struct Operand {
    const char *name;
    const csrt_mat *m;
    const float *v;
    int64_t len;
    bool out;
};

static bool meet(const Operand &a, const Operand &b) {
    if (a.m != nullptr && b.m != nullptr) return clash(a.m, b.m);
    if (a.m != nullptr) return vector_meets(b.v, b.len, a.m);
    if (b.m != nullptr) return vector_meets(a.v, a.len, b.m);
    return a.v < b.v + b.len && b.v < a.v + a.len;
}

// Outputs meet nothing, but for one that may be one input itself. Extents are compared first: nearly all pairs end there.
static int check_apart(const Operand *o, int count, const csrt_mat *alias_out, const csrt_mat *alias_in) {
    struct Extent {
        const char *from, *to;
    } e[24];
    for (int i = 0; i < count; ++i) {
        const csrt_mat *m = o[i].m;
        e[i].from = m != nullptr ? static_cast<const char *>(m->data) : reinterpret_cast<const char *>(o[i].v);
        const int64_t bytes = m != nullptr ? ((m->rows - 1) * m->ld + m->cols) * dt_size(m->dtype) : o[i].len * 4;
        e[i].to = e[i].from != nullptr ? e[i].from + bytes : nullptr;
    }
    for (int i = 0; i < count; ++i) {
        if (!o[i].out) continue;
        for (int j = 0; j < count; ++j) {
            if (i == j || (o[j].out && j < i) || e[i].from >= e[j].to || e[j].from >= e[i].to) continue;
            if (o[i].m != nullptr && o[i].m == alias_out && o[j].m != nullptr && o[j].m == alias_in &&
                same_place(alias_out, alias_in))
                continue;
            CSRT_ARG(!meet(o[i], o[j]), "%s overlaps %s", o[i].name, o[j].name);
        }
    }
    return CSRT_OK;
}

static int check_norm(const csrt_norm *s, const char *name, bool backward) {
    if (s == nullptr) return CSRT_OK;
    CSRT_ARG(s->kind >= CSRT_NORM_SCALE && s->kind <= CSRT_NORM_LAYER, "%s: unknown norm %d", name, s->kind);
    CSRT_ARG(s->kind == CSRT_NORM_SCALE || (std::isfinite(s->eps) && s->eps > 0.f), "%s: eps must be finite and > 0", name);
    const float *all[] = {s->weight, s->bias, s->mean, s->rstd, s->dweight, s->dbias};
    for (const float *p : all) CSRT_TRY(check_vector(p, name));
    if (backward) {
        CSRT_ARG(s->kind == CSRT_NORM_SCALE || s->rstd != nullptr, "%s: the backward pass needs rstd", name);
        CSRT_ARG(s->kind != CSRT_NORM_LAYER || s->mean != nullptr, "%s: the backward pass needs mean", name);
    }
    return CSRT_OK;
}

// m may be NULL; the first matrix given sets the shape, the first of each of the two types sets that.
static int check_one(const csrt_mat *m, const char *name, const csrt_mat **shape, int32_t *dtype) {
    if (m == nullptr) return CSRT_OK;
    CSRT_TRY(check_mat(m, name));
    if (*shape == nullptr) *shape = m;
    CSRT_TRY(check_shape(m, name, (*shape)->rows, (*shape)->cols));
    if (*dtype < 0) *dtype = m->dtype;
    CSRT_ARG(m->dtype == *dtype, "%s has another type than the matrices it goes with", name);
    return CSRT_OK;
}

static int check_types(int32_t *tb, int32_t *ts) {
    if (*tb < 0) *tb = *ts;
    if (*ts < 0) *ts = *tb;
    CSRT_ARG(*ts == CSRT_DT_F32 || *ts == *tb, "the residual stream must be float32 or of the block's type");
    return CSRT_OK;
}

// Rows of every matrix that is given in whole 16-byte words, and no further apart than a tensor map can say.
static bool norm_vector(std::initializer_list<const csrt_mat *> all) {
    for (const csrt_mat *m : all)
        if (m != nullptr && (!tma_rows_ok(m->data, m->ld, dt_size(m->dtype)) || m->ld * dt_size(m->dtype) >= (int64_t)1 << 40)) return false;
    return true;
}

// Tiles by measured times on a GB300 (us, with gate; F x T: features a thread, tokens). Clusters of sixteen blocks leave SMs
// idle, as a GPC takes only whole ones: 4096 x 8192 takes 101 on 4 x 32 and 68 on 8 x 32. wide: the stream is wider than the
// block's matrices; in, out: aligned rows.
static NormTile norm_fwd_choice(const NormArgs &a, bool in, bool out, bool wide) {
    const int64_t d = a.d, tiles = ceil_div<int64_t>(a.n, 32);
    // one or two tokens: a token a block (one of 4096: 4.5, on 4 x 32 6.6)
    if (a.n <= 2) return d > 65536 ? kTileColumns : d <= 16384 ? kTile1x4 : kTile1x16;
    if (d > 16384) return kTileColumns;
    if (in ? d > 10240 : d > 8192) return kTile8x4;
    if (in && d > 8192) return kTile16x5;   // 9216 x 2048: 57, on 8 x 16 69
    // few blocks: small ones (784 x 256: 4.7, on 8 x 32 6.7)
    if (d <= 2048 && tiles * ceil_div<int64_t>(d, 128) <= 2 * num_sms()) return kTile32x2;
    // unaligned inputs take twice the shared memory (4096 x 8191: 152, on 4 x 32 211; 1000 x 7777: 37 and 31)
    if (!in) return d <= 2048 ? kTile32x4 : kTile16x4;
    // unaligned results stage through more of it (4096 x 8191: 111, on 8 x 32 142)
    if (d <= 4096 && (!out || tiles * ceil_div<int64_t>(d, 256) <= 2 * num_sms())) return kTile32x4;
    // 32 tokens of 512 features of a float32 stream leave one block an SM (4096 x 8192: 129, on 4 x 16 111, 109 with tiles counted in 32 bits)
    return wide && d > 2048 ? kTile16x4 : kTile32x8;
}

template <typename TB, typename TS>
static int launch_fwd(const NormArgs &a, cudaStream_t s) {
    const int64_t tiles = ceil_div<int64_t>(a.n, 32);
    launch_pdl(norm_fwd_columns_kernel<TB, TS>, dim3((unsigned)tiles), dim3(kColWarps * 32), 0, s, a);
    count_launch();
    return check_launch("norm_fwd_columns_kernel");
}

static int32_t norm_groups(int32_t n) { return (int32_t)imax<int64_t>(1, imin<int64_t>(n, kNormGroups)); }

static size_t norm_bytes(int64_t d, int32_t max_n) {
    return kWsReservedBytes + align_up((size_t)norm_groups(max_n) * 4 * d * sizeof(float), 256);
}

template <typename TB, typename TS>
static int launch_bwd(NormArgs &a, cudaStream_t s) {
    a.groups = (int32_t)imin<int64_t>(ceil_div<int64_t>(a.n, 32), kNormGroups);
    launch_pdl(norm_bwd_columns_kernel<TB, TS>, dim3((unsigned)a.groups), dim3(kColWarps * 32), 0, s, a);
    count_launch();
    return check_launch("norm_bwd_columns_kernel");
}

// As above; wide: the block's matrices are float32 too, f32_stream: the stream is.
static NormTile norm_bwd_choice(const NormArgs &a, bool in, bool wide, bool f32_stream) {
    const int64_t d = a.d, tiles = ceil_div<int64_t>(a.n, 32);
    // five float32 matrices of 1024 features a block do not fit into shared memory
    if (d > (wide ? 8192 : 16384)) return kTileColumns;
    if (a.n <= 2) return kTile1x4;
    if (d <= 2048 && (!in || tiles * ceil_div<int64_t>(d, 128) <= 2 * num_sms())) return kTile32x2;
    if (!in) return d <= 4096 ? kTile16x2 : d <= 8192 ? kTile8x2 : kTile8x4;
    // few tokens: one cluster, which writes the sums over them itself (4096 x 24 on two: 10.5)
    if (d <= 4096 && tiles * ceil_div<int64_t>(d, 256) <= num_sms()) return kTile32x4;
    // 4096 x 8192 with a float32 stream: 226, on 4 x 32, which leaves one block an SM, 238; 2048 x 8192: 96 and 122
    if (f32_stream && d <= 4096) return kTile16x2;
    // 2048 x 8192: 67 on 4 x 32, 70 on 4 x 16; 4096 x 8192: 148 and 130 (since 1 - sigmoid keeps its digits 68 and 131)
    return d <= 2048 ? kTile32x4 : d <= 8192 ? kTile16x4 : kTile8x4;
}

// dweight and dbias of no tokens: zeros, unless they are added to.
__global__ void norm_zero_kernel(NormArgs a) {
    pdl_enter();
    const int64_t i = (int64_t)blockIdx.x * blockDim.x + threadIdx.x;
    float *out[4] = {a.post.dw, a.post.db, a.pre.dw, a.pre.db};
    if (i < a.d && out[blockIdx.y] != nullptr) out[blockIdx.y][i] = 0.f;
}

#define CSRT_NORM_DISPATCH(fn, tb, ts, ...)                                                                     \
    (tb == CSRT_DT_F32 ? fn<float, float>(__VA_ARGS__)                                                          \
     : tb == CSRT_DT_BF16                                                                                       \
         ? (ts == CSRT_DT_F32 ? fn<__nv_bfloat16, float>(__VA_ARGS__) : fn<__nv_bfloat16, __nv_bfloat16>(__VA_ARGS__)) \
         : (ts == CSRT_DT_F32 ? fn<__half, float>(__VA_ARGS__) : fn<__half, __half>(__VA_ARGS__)))

#define CSRT_NORM_TILES(fn, tb, ts)                                          \
    (tb == CSRT_DT_F32    ? fn##_f32                                         \
     : tb == CSRT_DT_BF16 ? (ts == CSRT_DT_F32 ? fn##_bf16_f32 : fn##_bf16) \
                          : (ts == CSRT_DT_F32 ? fn##_f16_f32 : fn##_f16))

}  // namespace csrt

using namespace csrt;

extern "C" {

int csrt_block_norm_fwd(const csrt_mat *y, const csrt_norm *post, const csrt_mat *gate, int32_t gate_act,
                        const csrt_mat *r, float r_scale, const csrt_norm *pre, csrt_mat *h, csrt_mat *v, void *stream) {
    CSRT_ARG(y != nullptr || r != nullptr, "y and r are both NULL");
    CSRT_ARG(h != nullptr || v != nullptr, "h and v are both NULL");
    CSRT_ARG(y != nullptr || (post == nullptr && gate == nullptr), "post and gate need y");
    CSRT_ARG((pre == nullptr) == (v == nullptr), "pre and v go together");
    CSRT_ARG(gate_act >= CSRT_GATE_NONE && gate_act <= CSRT_GATE_SILU, "unknown gate activation %d", gate_act);
    CSRT_ARG(std::isfinite(r_scale), "r_scale must be finite");
    const csrt_mat *shape = nullptr;
    int32_t tb = -1, ts = -1;
    CSRT_TRY(check_one(y, "y", &shape, &tb));
    CSRT_TRY(check_one(gate, "gate", &shape, &tb));
    CSRT_TRY(check_one(v, "v", &shape, &tb));
    CSRT_TRY(check_one(r, "r", &shape, &ts));
    CSRT_TRY(check_one(h, "h", &shape, &ts));
    CSRT_TRY(check_types(&tb, &ts));
    CSRT_TRY(check_norm(post, "post", false));
    CSRT_TRY(check_norm(pre, "pre", false));
    const int32_t d = shape->rows, n = shape->cols;
    const csrt_norm none = {};
    const csrt_norm *po = post != nullptr ? post : &none, *pr = pre != nullptr ? pre : &none;
    const bool po_mean = po->kind == CSRT_NORM_LAYER, pr_mean = pr->kind == CSRT_NORM_LAYER;
    const bool po_stat = po->kind != CSRT_NORM_SCALE, pr_stat = pr->kind != CSRT_NORM_SCALE;
    if (d == 0 || n == 0) return CSRT_OK;
    const Operand all[] = {
        {"h", h, nullptr, 0, true},
        {"v", v, nullptr, 0, true},
        {"post.mean", nullptr, po_mean ? po->mean : nullptr, n, true},
        {"post.rstd", nullptr, po_stat ? po->rstd : nullptr, n, true},
        {"pre.mean", nullptr, pr_mean ? pr->mean : nullptr, n, true},
        {"pre.rstd", nullptr, pr_stat ? pr->rstd : nullptr, n, true},
        {"y", y, nullptr, 0, false},
        {"gate", gate, nullptr, 0, false},
        {"r", r, nullptr, 0, false},
        {"post.weight", nullptr, po->weight, d, false},
        {"post.bias", nullptr, po->bias, d, false},
        {"pre.weight", nullptr, pr->weight, d, false},
        {"pre.bias", nullptr, pr->bias, d, false},
    };
    CSRT_TRY(check_apart(all, (int)(sizeof(all) / sizeof(all[0])), h, r));
    NormArgs a = {};
    a.d = d;
    a.n = n;
    a.gate_act = gate_act;
    a.r_scale = r_scale;
    a.post = norm_side(post);
    a.pre = norm_side(pre);
    a.y = norm_mat(y);
    a.g = norm_mat(gate);
    a.r = norm_mat(r);
    a.h = norm_mat(h);
    a.v = norm_mat(v);
    const bool in = tb != CSRT_DT_F32 && norm_vector({y, gate, r}), out = norm_vector({h, v}) && n % 8 == 0;
    const NormTile t = norm_fwd_choice(a, in, out, ts != tb);
    if (t == kTileColumns) return CSRT_NORM_DISPATCH(launch_fwd, tb, ts, a, as_stream(stream));
    return CSRT_NORM_TILES(norm_fwd, tb, ts)(a, t, in, out, as_stream(stream));
}

int csrt_block_norm_workspace_bytes(int32_t d, int32_t max_n, size_t *bytes) {
    CSRT_ARG(bytes != nullptr, "bytes is NULL");
    CSRT_ARG(d >= 0 && max_n >= 0, "negative size");
    *bytes = norm_bytes(d, max_n);
    return CSRT_OK;
}

int csrt_block_norm_bwd(const csrt_mat *dv, const csrt_mat *dh, const csrt_mat *h, const csrt_norm *pre,
                        const csrt_mat *y, const csrt_norm *post, const csrt_mat *gate, int32_t gate_act, float r_scale,
                        int32_t accumulate, csrt_mat *dr, csrt_mat *dy, csrt_mat *dgate, void *ws, size_t ws_bytes,
                        void *stream) {
    CSRT_ARG(dv != nullptr || dh != nullptr, "dv and dh are both NULL");
    CSRT_ARG((pre == nullptr) == (dv == nullptr), "pre and dv go together");
    CSRT_ARG(pre == nullptr || h != nullptr, "pre needs h");
    CSRT_ARG(dy != nullptr || (post == nullptr && gate == nullptr && dgate == nullptr), "post and gate need dy");
    CSRT_ARG(dgate == nullptr || gate != nullptr, "dgate needs gate");
    CSRT_ARG(y != nullptr || (post == nullptr && dgate == nullptr), "post and dgate need y");
    CSRT_ARG(gate_act >= CSRT_GATE_NONE && gate_act <= CSRT_GATE_SILU, "unknown gate activation %d", gate_act);
    CSRT_ARG(std::isfinite(r_scale), "r_scale must be finite");
    const csrt_mat *shape = nullptr;
    int32_t tb = -1, ts = -1;
    CSRT_TRY(check_one(dv, "dv", &shape, &tb));
    CSRT_TRY(check_one(y, "y", &shape, &tb));
    CSRT_TRY(check_one(gate, "gate", &shape, &tb));
    CSRT_TRY(check_one(dy, "dy", &shape, &tb));
    CSRT_TRY(check_one(dgate, "dgate", &shape, &tb));
    CSRT_TRY(check_one(dh, "dh", &shape, &ts));
    CSRT_TRY(check_one(h, "h", &shape, &ts));
    CSRT_TRY(check_one(dr, "dr", &shape, &ts));
    CSRT_TRY(check_types(&tb, &ts));
    CSRT_TRY(check_norm(post, "post", true));
    CSRT_TRY(check_norm(pre, "pre", true));
    const int32_t d = shape->rows, n = shape->cols;
    CSRT_ARG(ws != nullptr, "workspace is NULL");
    CSRT_ARG((reinterpret_cast<uintptr_t>(ws) & 255) == 0, "workspace is not 256-byte aligned");
    if (ws_bytes < norm_bytes(d, n))
        return fail(CSRT_ERR_WORKSPACE, "workspace has %zu bytes, needs %zu", ws_bytes, norm_bytes(d, n));
    const csrt_norm none = {};
    const csrt_norm *po = post != nullptr ? post : &none, *pr = pre != nullptr ? pre : &none;
    const bool po_mean = po->kind == CSRT_NORM_LAYER, pr_mean = pr->kind == CSRT_NORM_LAYER;
    const bool po_stat = po->kind != CSRT_NORM_SCALE, pr_stat = pr->kind != CSRT_NORM_SCALE;
    if (d == 0) return CSRT_OK;
    const Operand all[] = {
        {"dr", dr, nullptr, 0, true},
        {"dy", dy, nullptr, 0, true},
        {"dgate", dgate, nullptr, 0, true},
        {"post.dweight", nullptr, po->dweight, d, true},
        {"post.dbias", nullptr, po->dbias, d, true},
        {"pre.dweight", nullptr, pr->dweight, d, true},
        {"pre.dbias", nullptr, pr->dbias, d, true},
        {"dv", dv, nullptr, 0, false},
        {"dh", dh, nullptr, 0, false},
        {"h", h, nullptr, 0, false},
        {"y", y, nullptr, 0, false},
        {"gate", gate, nullptr, 0, false},
        {"post.mean", nullptr, po_mean ? po->mean : nullptr, n, false},
        {"post.rstd", nullptr, po_stat ? po->rstd : nullptr, n, false},
        {"pre.mean", nullptr, pr_mean ? pr->mean : nullptr, n, false},
        {"pre.rstd", nullptr, pr_stat ? pr->rstd : nullptr, n, false},
        {"post.weight", nullptr, po->weight, d, false},
        {"post.bias", nullptr, po->bias, d, false},
        {"pre.weight", nullptr, pr->weight, d, false},
        {"pre.bias", nullptr, pr->bias, d, false},
    };
    CSRT_TRY(check_apart(all, (int)(sizeof(all) / sizeof(all[0])), dr, dh));
    NormArgs a = {};
    a.d = d;
    a.n = n;
    a.gate_act = gate_act;
    a.accumulate = accumulate != 0;
    a.r_scale = r_scale;
    a.post = norm_side(post);
    a.pre = norm_side(pre);
    a.dv = norm_mat(dv);
    a.r = norm_mat(dh);
    // what no result asks for is not read
    a.h = norm_mat(dv != nullptr ? h : nullptr);
    a.y = norm_mat(post != nullptr || dgate != nullptr ? y : nullptr);
    a.g = norm_mat(gate);
    a.dr = norm_mat(dr);
    a.dy = norm_mat(dy);
    a.dg = norm_mat(dgate);
    a.partial = reinterpret_cast<float *>(ws_scratch(ws));
    a.hdr = static_cast<WsHeader *>(ws);
    cudaStream_t s = as_stream(stream);
    if (n == 0) {
        if (accumulate || (po->dweight == nullptr && po->dbias == nullptr && pr->dweight == nullptr && pr->dbias == nullptr))
            return CSRT_OK;
        launch_pdl(norm_zero_kernel, dim3((unsigned)ceil_div<int64_t>(d, 128), 4), dim3(128), 0, s, a);
        count_launch();
        return check_launch("norm_zero_kernel");
    }
    const bool in = tb != CSRT_DT_F32 && norm_vector({dv, dh, h, y, gate}), out = norm_vector({dr, dy, dgate}) && n % 8 == 0;
    const NormTile t = norm_bwd_choice(a, in, tb == CSRT_DT_F32, ts == CSRT_DT_F32);
    CSRT_TRY(t == kTileColumns ? CSRT_NORM_DISPATCH(launch_bwd, tb, ts, a, s) : CSRT_NORM_TILES(norm_bwd, tb, ts)(a, t, in, out, s));
    if (po->dweight == nullptr && po->dbias == nullptr && pr->dweight == nullptr && pr->dbias == nullptr) return CSRT_OK;
    if (t != kTileColumns && a.groups == 1) return CSRT_OK;   // the only group has written them
    launch_pdl(norm_sums_kernel, dim3((unsigned)ceil_div<int64_t>(d, 32), 4), dim3(256), 0, s, a);
    count_launch();
    return check_launch("norm_sums_kernel");
}

}  // extern "C"
