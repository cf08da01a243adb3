// Orthogonalised update (csrt_orthogonalize): momentum, normalisation and the Newton-Schulz products
//
//   X <- a X + (b A + c A A) X,   A = X X^T  (X^T X and products on the right where X has more rows than columns)
//
// as three products per step on gemm16_kernel: A with its mirrored half, B = b A + c A A likewise, and a X + B X. One
// cooperative launch runs all of them for all matrices, a unit waiting for its own matrix only (GLaunch). A launch per
// product was slower throughout (64 x 64: 74 against 64 us; 3 x 2048 x 2048: 595, 442; 4096 x 9216: 1947, 1858).
//
// Number formats. Singular values stay in [0, 1.203] (p(s) = a s + b s^3 + c s^5 maps [0, 1.203] into itself), so
// every entry of X, A and B is bounded (1.203, 1.45, 2.81) and fits float16 once scaled by a power of two: X and A
// are stored times 2^15, B times 2^14. float16 keeps 11 significant bits where bfloat16 keeps 8, at the same
// tensor-core rate: bfloat16 operands alone would put o about 1e-2 off. X itself is carried in float32 (times 2^15) beside
// its float16 copy, so that the term a X - all there is for the small singular values - does not gather a rounding per
// step. The diagonals of A and B are kept apart, in float32: near convergence they hold nearly all of A and B, whose
// rounding would otherwise be the largest error of o (a bfloat16 o was 2.2e-3 to 2.8e-3 off with them inside, and is
// 1.7e-3 off now, its own rounding).
//
// What bounds it (measured, whole calls): 4096 x 9216 takes 1.86 ms for 2.66 TFLOP of necessary work (1.4 ms at the
// library's rate; 2.0 ms when calls follow one another for long and the power limit sets the clock): products at 1.5 to
// 1.65 PFLOP/s, waves 90% full, and 0.14 ms for the two passes over gradient and momentum, at HBM rate. Smaller ones are
// bound by latency: a product costs at least 4 us - operands from L2, the epilogue's own, the release to the other SMs -
// so fifteen of them 64 us and more, whatever the size (a 64 x 64 matrix: 64 us).
//
// The Frobenius norm is summed in float64 over float32 sums of eight squares; a sum out of float32's safe range is
// taken again in float64, so that neither tiny nor huge gradients lose it.
#include <cmath>

#include "gemm16_host.cuh"

namespace csrt {

constexpr int kPrepThreads = 256;
constexpr int kPrepBlocks = 1024;   // most blocks (norm partials) per matrix
constexpr int kOneByOne = 1 << 26;  // longest side that the matrices of a batch may have in one launch

struct PrepArgs {
    GMat g;                 // gradient
    float *mom;             // contiguous, or NULL
    float beta, eps, scale;
    int32_t nesterov, rows, cols, vec;
    double *partial;        // [batch][gridDim.x]
    __half *hi;             // X, its float16 copy
    float *x;               // and itself, or
    GMat o;                 // with no steps: the normalised direction itself
    int64_t ldx;
    int32_t direct;
    uint32_t *done;         // the products' counts per matrix, cleared here
};

// Eight consecutive elements of row r from column c: gradient, old momentum -> u (and the new momentum stored).
template <bool UPDATE>
__device__ __forceinline__ void direction8(const PrepArgs &a, int b, int r, int c, int cnt, float (&u)[8]) {
    const int64_t gi = b * a.g.stride + (int64_t)r * a.g.ld + c;
    const int64_t mi = ((int64_t)b * a.rows + r) * a.cols + c;
    float g[8], m[8];
    if (a.vec) {
        if (a.g.dtype == CSRT_DT_F32) {
            const float4 *p = reinterpret_cast<const float4 *>(static_cast<const float *>(a.g.p) + gi);
            const float4 x = p[0], y = p[1];
            g[0] = x.x, g[1] = x.y, g[2] = x.z, g[3] = x.w, g[4] = y.x, g[5] = y.y, g[6] = y.z, g[7] = y.w;
        } else {
            const uint4 x = *reinterpret_cast<const uint4 *>(static_cast<const uint16_t *>(a.g.p) + gi);
            const float2 p = unpack16(x.x, false), q = unpack16(x.y, false), s = unpack16(x.z, false),
                         t = unpack16(x.w, false);
            g[0] = p.x, g[1] = p.y, g[2] = q.x, g[3] = q.y, g[4] = s.x, g[5] = s.y, g[6] = t.x, g[7] = t.y;
        }
        if (a.mom != nullptr) {
            const float4 *p = reinterpret_cast<const float4 *>(a.mom + mi);
            const float4 x = p[0], y = p[1];
            m[0] = x.x, m[1] = x.y, m[2] = x.z, m[3] = x.w, m[4] = y.x, m[5] = y.y, m[6] = y.z, m[7] = y.w;
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            g[i] = i < cnt ? load1(a.g.p, gi + i, a.g.dtype) : 0.f;
            m[i] = a.mom != nullptr && i < cnt ? a.mom[mi + i] : 0.f;
        }
    }
    if (a.mom == nullptr) {
#pragma unroll
        for (int i = 0; i < 8; ++i) u[i] = g[i];
        return;
    }
    if (UPDATE) {
#pragma unroll
        for (int i = 0; i < 8; ++i) m[i] = __fadd_rn(__fmul_rn(a.beta, m[i]), g[i]);
        if (a.vec) {
            float4 *p = reinterpret_cast<float4 *>(a.mom + mi);
            p[0] = make_float4(m[0], m[1], m[2], m[3]);
            p[1] = make_float4(m[4], m[5], m[6], m[7]);
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (i < cnt) a.mom[mi + i] = m[i];
        }
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) u[i] = a.nesterov ? __fadd_rn(g[i], __fmul_rn(a.beta, m[i])) : m[i];
}

__device__ __forceinline__ double block_sum(double v) {
    __shared__ double s_part[kPrepThreads / 32];
#pragma unroll
    for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    if ((threadIdx.x & 31) == 0) s_part[threadIdx.x >> 5] = v;
    __syncthreads();
    double t = 0.0;
    for (int w = 0; w < kPrepThreads / 32; ++w) t += s_part[w];
    __syncthreads();
    return t;
}

// First pass over the gradients: momentum, and the squares of u summed per block.
__global__ void __launch_bounds__(kPrepThreads) ortho_momentum_kernel(PrepArgs a) {
    pdl_enter();
    const int b = blockIdx.y;
    const uint32_t per_row = ((uint32_t)a.cols + 7) / 8, total = per_row * (uint32_t)a.rows;
    double sum = 0.0;
    for (uint32_t t = blockIdx.x * kPrepThreads + threadIdx.x; t < total; t += gridDim.x * kPrepThreads) {
        const uint32_t r = t / per_row, c = (t - r * per_row) * 8;
        float u[8];
        direction8<true>(a, b, (int)r, (int)c, min(8, a.cols - (int)c), u);
        float s = 0.f, big = 0.f;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            s += u[i] * u[i];
            big = fmaxf(big, fabsf(u[i]));
        }
        if (s > 1e-24f && s < 1e37f) {
            sum += (double)s;
        } else if (big > 0.f || s != s) {
            for (int i = 0; i < 8; ++i) sum += (double)u[i] * (double)u[i];
        }
    }
    sum = block_sum(sum);
    if (threadIdx.x == 0) a.partial[(int64_t)b * gridDim.x + blockIdx.x] = sum;
}

// Second pass: X = u / max(||u||_F, eps), scaled, in float32 and float16.
__global__ void __launch_bounds__(kPrepThreads) ortho_scale_kernel(PrepArgs a) {
    pdl_enter();
    const int b = blockIdx.y;
    if (threadIdx.x == 0 && blockIdx.x == 0) a.done[b] = 0;
    double n2 = 0.0;
    for (int i = threadIdx.x; i < (int)gridDim.x; i += kPrepThreads) n2 += a.partial[(int64_t)b * gridDim.x + i];
    n2 = block_sum(n2);
    double norm = sqrt(n2);
    norm = norm < (double)a.eps ? (double)a.eps : norm;   // a NaN stays
    // A factor that float32 does not hold (a norm below 1e-34, or scale / norm out of its range) is applied in parts, powers
    // of two first: these are exact wherever the result is not zero. Products in float64 instead, even behind a branch, take
    // the kernel's registers from 32 to 40 (2048 x 2048: 250 -> 254 us for the whole call).
    double rest = (a.direct ? (double)a.scale : (double)kXScale) / norm;
    float f0 = 1.f, f1 = 1.f;
    if (fabs(rest) >= 0x1p127) {
        f0 = 0x1p120f, rest *= 0x1p-120;
        if (fabs(rest) >= 0x1p127) f1 = 0x1p60f, rest *= 0x1p-60;
    } else if (fabs(rest) < 0x1p-126) {
        f0 = 0x1p-100f, rest *= 0x1p100;
        if (fabs(rest) < 0x1p-126) f1 = 0x1p-90f, rest *= 0x1p90;
    }
    const float f = (float)rest;
    const uint32_t per_row = ((uint32_t)a.cols + 7) / 8, total = per_row * (uint32_t)a.rows;
    for (uint32_t t = blockIdx.x * kPrepThreads + threadIdx.x; t < total; t += gridDim.x * kPrepThreads) {
        const uint32_t r = t / per_row, c = (t - r * per_row) * 8;
        const int cnt = min(8, a.cols - (int)c);
        float u[8];
        direction8<false>(a, b, (int)r, (int)c, cnt, u);
#pragma unroll
        for (int i = 0; i < 8; ++i) u[i] = u[i] * f0 * f1 * f;
        if (a.direct) {
            for (int i = 0; i < cnt; ++i)
                store1(a.o.p, b * a.o.stride + (int64_t)r * a.o.ld + c + i, u[i], a.o.dtype);
            continue;
        }
        uint32_t h[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) h[i] = pack16(u[2 * i], u[2 * i + 1], true);
        // rows are padded to a multiple of eight, so the tail of a row may be written whole
        const int64_t xi = ((int64_t)b * a.rows + r) * a.ldx + c;
        *reinterpret_cast<uint4 *>(a.hi + xi) = make_uint4(h[0], h[1], h[2], h[3]);
        float4 *x = reinterpret_cast<float4 *>(a.x + xi);
        x[0] = make_float4(u[0], u[1], u[2], u[3]);
        x[1] = make_float4(u[4], u[5], u[6], u[7]);
    }
}

struct OrthoLayout {
    int64_t ldx, lds;
    size_t slices, done, partial, x0, x1, xf, a, b, diag_a, diag_b, total;   // offsets after the reserved part
};

static OrthoLayout layout(int64_t batch, int64_t rows, int64_t cols) {
    auto up = [](int64_t v, int64_t q) { return (v + q - 1) / q * q; };
    OrthoLayout l;
    const int64_t s = rows < cols ? rows : cols;
    l.ldx = up(cols, 64);
    l.lds = up(s, 64);
    size_t at = 0;
    auto take = [&](int64_t bytes) {
        const size_t r = at;
        at += (size_t)up(bytes, 256);
        return r;
    };
    l.slices = take((int64_t)kPartialBytes);
    l.done = take(batch * (int64_t)sizeof(uint32_t));
    l.partial = take(batch * kPrepBlocks * (int64_t)sizeof(double));
    l.x0 = take(batch * rows * l.ldx * 2);
    l.x1 = take(batch * rows * l.ldx * 2);
    l.xf = take(batch * rows * l.ldx * 4);
    l.a = take(batch * s * l.lds * 2);
    l.b = take(batch * s * l.lds * 2);
    l.diag_a = take(batch * l.lds * 4);
    l.diag_b = take(batch * l.lds * 4);
    l.total = at;
    return l;
}

struct NsPlan {
    int32_t first, batch, rows, cols, steps;   // matrices first .. first + batch - 1
    float scale;
    char *base;
    OrthoLayout l;
    GMat o;
    bool direct;   // the last product writes o (bfloat16, aligned); else it leaves X, and o is made of it afterwards
    void *ws;
};

// o = scale X, for results that the products' epilogue does not write itself.
__global__ void ortho_result_kernel(const float *__restrict__ x, int64_t ldx, int32_t rows, int32_t cols, float scale, GMat o) {
    pdl_enter();
    const int64_t b = blockIdx.z;
    for (int64_t r = blockIdx.y; r < rows; r += gridDim.y)
        for (int64_t c = (int64_t)blockIdx.x * blockDim.x + threadIdx.x; c < cols; c += (int64_t)gridDim.x * blockDim.x) {
            const int64_t i = (b * rows + r) * ldx + c;
            store1(o.p, b * o.stride + r * o.ld + c, scale * x[i], o.dtype);
        }
}

// Product `set` of the six that make up the steps (ns_set).
static void ns_product(const NsPlan &q, int set, GProduct &p, GArgs &a) {
    const OrthoLayout &l = q.l;
    const bool tall = q.rows > q.cols;
    const int32_t sh = tall ? q.cols : q.rows;
    auto mat = [&](size_t off, int64_t ld, int64_t n_rows) {
        GMat m = {};
        m.ld = ld;
        m.stride = ld * n_rows;
        m.dtype = off == l.xf ? CSRT_DT_F32 : CSRT_DT_F16;
        m.p = q.base + off + q.first * m.stride * dt_size(m.dtype);
        m.vec = m.pad = 1;
        return m;
    };
    auto op = [&](size_t off, int64_t r, int64_t c, int64_t ld) {
        GOperand o;
        o.rows = r;
        o.cols = c;
        o.ld = ld;
        o.stride = r * ld;
        o.p = q.base + off + q.first * o.stride * 2;
        return o;
    };
    a = GArgs{};
    a.batch = q.batch;
    a.f16 = 1;
    a.hdr = static_cast<WsHeader *>(q.ws);
    a.counters = ws_counters(q.ws);
    a.partial = reinterpret_cast<float *>(q.base + l.slices);
    a.s_pad = (int32_t)l.lds;
    a.tall = tall;
    float *diag_a = reinterpret_cast<float *>(q.base + l.diag_a) + q.first * l.lds;
    float *diag_b = reinterpret_cast<float *>(q.base + l.diag_b) + q.first * l.lds;
    const size_t x = set == 1 || set == 4 || (set == 5 && (q.steps - 1) % 2) ? l.x1 : l.x0;
    const GOperand ox = op(x, q.rows, q.cols, l.ldx), oa = op(l.a, sh, sh, l.lds), ob = op(l.b, sh, sh, l.lds);
    if (set <= 1) {          // A = X X^T or X^T X, times 2^15
        p.a = p.b = ox;
        p.a_mn = p.b_mn = tall;
        p.reduction = tall ? q.rows : q.cols;
        a.kind = kNsGram;
        a.sym = 1;
        a.m = a.n = sh;
        a.alpha = kInvXScale;
        a.diag_out = diag_a;
        a.out0 = mat(l.a, l.lds, sh);
    } else if (set == 2) {   // B = b A + c A A, times 2^14
        p.a = p.b = oa;
        p.a_mn = p.b_mn = false;
        p.reduction = sh;
        a.kind = kNsPoly;
        a.sym = 1;
        a.m = a.n = sh;
        a.alpha = kNsC * 0.5f * kInvXScale;
        a.diag_in = diag_a;
        a.diag_out = diag_b;
        a.c0 = mat(l.a, l.lds, sh);
        a.out0 = mat(l.b, l.lds, sh);
    } else {                 // X' = a X + B X, times 2^15; the last one is o
        p.a = tall ? ox : ob;
        p.b = tall ? ob : ox;
        p.a_mn = false;
        p.b_mn = !tall;
        p.reduction = sh;
        a.kind = kNsApply;
        a.m = q.rows;
        a.n = q.cols;
        a.alpha = 2.f * kInvXScale;
        const bool out = set == 5 && q.direct;
        a.gamma = out ? q.scale * kInvXScale : 1.f;
        a.diag_in = diag_b;
        a.c0 = mat(l.xf, l.ldx, q.rows);
        a.out0 = out ? q.o : mat(x == l.x0 ? l.x1 : l.x0, l.ldx, q.rows);
        if (!out) a.out1 = a.c0;
    }
}

// All steps in one cooperative launch on CG x 128 x BN tiles. LONG: a product has a long sum; the slabs of the slices are
// then those of long sums too, so that either all tiles of a product are split or, with a slab for each CTA, none.
template <int CG, int BN, bool LONG>
static int launch_ns(const NsPlan &q, const GTile &tile, cudaStream_t s) {
    GLaunch<kEpiNs> n = {};
    int32_t units = 1;
    for (int set = 0; set < kNsSets; ++set) {
        GProduct p;
        GArgs &a = n.args[set];
        ns_product(q, set, p, a);
        // slices of different matrices' phases would share their place in the workspace
        const GSplit split = q.batch == 1 ? best_splits(tile, a, p.reduction, !LONG) : GSplit{0, 1, 0.};
        a.whole = split.whole;
        a.splits = split.splits;
        const int rc = fill_set<CG, BN, kEpiNs, false>(p, a, n.maps[set]);
        if (rc != CSRT_OK) return rc;
        units = imax(units, a.units);
    }
    n.phases = 3 * q.steps;
    n.done = reinterpret_cast<uint32_t *>(q.base + q.l.done) + q.first;
    n.step_units[0] = n.args[0].units / q.batch;
    n.step_units[1] = n.args[2].units / q.batch;
    n.step_units[2] = n.args[3].units / q.batch;

    constexpr auto kernel = gemm16_kernel<CG, BN, kEpiNs, false, false, LONG>;
    constexpr int smem = gsmem_bytes<CG, BN, kEpiNs, false>();
    const int rc = allow_smem<kernel>(smem);
    if (rc != CSRT_OK) return rc;
    // CTAs (or pairs) that the GPU can hold at once: all of them have to be there, as units wait for one another
    static int resident[64] = {0};
    int dev = 0;
    CSRT_CHECK_CUDA(cudaGetDevice(&dev));
    int slots = dev >= 0 && dev < 64 ? resident[dev] : 0;
    if (slots == 0) {
        if (CG == 1) {
            CSRT_CHECK_CUDA(cudaOccupancyMaxActiveBlocksPerMultiprocessor(&slots, kernel, kGThreads, smem));
            slots *= num_sms();
        } else {
            cudaLaunchAttribute dim[1];
            dim[0].id = cudaLaunchAttributeClusterDimension;
            dim[0].val.clusterDim.x = CG;
            dim[0].val.clusterDim.y = dim[0].val.clusterDim.z = 1;
            cudaLaunchConfig_t probe = {};
            probe.gridDim = dim3(num_sms() / CG * CG);
            probe.blockDim = dim3(kGThreads);
            probe.dynamicSmemBytes = smem;
            probe.attrs = dim;
            probe.numAttrs = 1;
            CSRT_CHECK_CUDA(cudaOccupancyMaxActiveClusters(&slots, kernel, &probe));
        }
        if (slots < 1) return fail(CSRT_ERR_CUDA, "the orthogonalisation does not fit the GPU");
        if (dev >= 0 && dev < 64) resident[dev] = slots;
    }
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeCooperative;
    attr[0].val.cooperative = 1;
    cudaLaunchConfig_t cfg = {};
    slots = imin(slots, imax(1, num_sms() / CG));
    if (LONG) slots = imin(slots, (int)(kPartialBytes / (CG * 128 * BN * sizeof(float))));
    cfg.gridDim = dim3((unsigned)(imin(units, slots) * CG));
    cfg.blockDim = dim3(kGThreads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = s;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    CSRT_CHECK_CUDA(cudaLaunchKernelEx(&cfg, kernel, n));
    count_launch();
    return check_launch("gemm16_kernel (Newton-Schulz)");
}

// Whether a product would accumulate more than kLongKb stages at once on tiles t.
static bool has_long_sum(const NsPlan &q, const GTile &t) {
    if (imax(q.rows, q.cols) <= kLongKb * kGBK) return false;
    for (int set : {0, 2, 3}) {
        GProduct p;
        GArgs a;
        ns_product(q, set, p, a);
        const GSplit split = q.batch == 1 ? best_splits(t, a, p.reduction, true) : GSplit{0, 1, 0.};
        if (longest(split, p.reduction) > kLongKb) return true;
    }
    return false;
}

static int ns_products(const NsPlan &q, cudaStream_t s) {
    if (!device_is_sm10x()) return fail(CSRT_ERR_CUDA, "the orthogonalisation needs a GPU with tcgen05");
    // The units of a batch are not sliced: one that walks a side of hundreds of millions would outlast the others' bounded
    // wait for it (two seconds), so that such matrices, 0.3 s to a slice at most, go one by one.
    if (q.batch > 1 && imax(q.rows, q.cols) > kOneByOne) {
        for (int32_t b = 0; b < q.batch; ++b) {
            NsPlan one = q;
            one.first = b;
            one.batch = 1;
            one.o.p = static_cast<char *>(q.o.p) + b * q.o.stride * dt_size(q.o.dtype);
            const int rc = ns_products(one, s);
            if (rc != CSRT_OK) return rc;
        }
        return CSRT_OK;
    }
    // By the number of 128 x 128 tiles of X (measured, us for the whole call on tiles 64, 128 by pairs and 256 by pairs
    // wide): few tiles take the narrow ones, which share the work among more SMs (1024 x 1024: 123 / 147 / 217;
    // 3 x 2048 x 512: 154 / 174 / 239); from 200 tiles on pairs of SMs on 256 x 128 (2048 x 2048: 334 / 247 / 306;
    // 6 x 256 x 4096: 226 / 203 / 267; 4096 x 1000: 246 / 237 / 290); from 700 on, where L2 traffic counts most,
    // 256 x 256 (3 x 2048 x 2048: 738 / 487 / 442; 4096 x 4096: 1826 / 1188 / 1027; 4096 x 9216: 3747 / 2204 / 1858).
    // Those shapes have short sides of 256 and more. Below, tiles of 256 rows are mostly empty and a batch has one to three
    // units of A a matrix: 6 x 128 x 8192 takes 313 us and 12 x 64 x 9216 455 where one such matrix, with slices, takes 118
    // and 105.
    const int64_t tiles = (int64_t)q.batch * ceil_div<int64_t>(q.rows, 128) * ceil_div<int64_t>(q.cols, 128);
    if (has_long_sum(q, kTiles[tiles < 200 ? 2 : tiles < 700 ? 3 : 0]))
        return tiles < 700 ? launch_ns<2, 128, true>(q, kTiles[3], s) : launch_ns<2, 256, true>(q, kTiles[0], s);
    if (tiles < 200) return launch_ns<1, 64, false>(q, kTiles[2], s);
    if (tiles < 700) return launch_ns<2, 128, false>(q, kTiles[3], s);
    return launch_ns<2, 256, false>(q, kTiles[0], s);
}

static int check_batch(const csrt_mat *m, const char *name, int32_t batch, int64_t stride) {
    CSRT_ARG(m != nullptr, "%s is NULL", name);
    CSRT_ARG(m->rows >= 0 && m->cols >= 0 && (int64_t)m->rows * m->cols < (int64_t)1 << 31, "%s: bad size", name);
    CSRT_ARG(m->ld >= m->cols && m->ld < (int64_t)1 << 31, "%s: bad ld", name);
    CSRT_ARG(stride >= 0 && stride < (int64_t)1 << 40, "%s: bad batch stride", name);
    CSRT_ARG(m->dtype == CSRT_DT_F32 || m->dtype == CSRT_DT_BF16, "%s must be float32 or bfloat16", name);
    CSRT_ARG(m->data != nullptr || batch == 0 || m->rows == 0 || m->cols == 0, "%s: data is NULL", name);
    CSRT_ARG(reinterpret_cast<uintptr_t>(m->data) % dt_size(m->dtype) == 0, "%s: data is not aligned to its type", name);
    return CSRT_OK;
}

static bool extents_meet(const void *a, int64_t abytes, const void *b, int64_t bbytes) {
    const char *pa = static_cast<const char *>(a), *pb = static_cast<const char *>(b);
    return pa < pb + bbytes && pb < pa + abytes;
}

}  // namespace csrt

using namespace csrt;

extern "C" {

int csrt_orthogonalize_workspace_bytes(int32_t batch, int32_t rows, int32_t cols, size_t *bytes) {
    CSRT_ARG(bytes != nullptr, "bytes is NULL");
    CSRT_ARG(batch >= 0 && rows >= 0 && cols >= 0, "negative size");
    CSRT_ARG(batch <= 65535 && (int64_t)rows * cols < (int64_t)1 << 31, "rows*cols must be below 2^31, batch at most 65535");
    *bytes = kWsReservedBytes + layout(batch, rows, cols).total;
    return CSRT_OK;
}

int csrt_orthogonalize(const csrt_mat *g, int64_t g_stride, int32_t batch, float *momentum, float beta,
                       int32_t nesterov, int32_t steps, float eps, float scale, csrt_mat *o, int64_t o_stride,
                       void *ws, size_t ws_bytes, void *stream) {
    CSRT_ARG(batch >= 0 && batch <= 65535, "batch must be in [0, 65535]");
    int rc = check_batch(g, "g", batch, g_stride);
    if (rc != CSRT_OK) return rc;
    rc = check_batch(o, "o", batch, o_stride);
    if (rc != CSRT_OK) return rc;
    const int32_t rows = g->rows, cols = g->cols;
    CSRT_ARG(o->rows == rows && o->cols == cols, "o is %d x %d, must be %d x %d", o->rows, o->cols, rows, cols);
    CSRT_ARG(std::isfinite(beta) && beta >= 0.f && beta < 1.f, "beta must be in [0, 1)");
    CSRT_ARG(std::isfinite(eps) && eps > 0.f, "eps must be finite and > 0");
    CSRT_ARG(std::isfinite(scale), "scale must be finite");
    CSRT_ARG(steps >= 0 && steps <= 32, "steps must be in [0, 32]");
    if (batch == 0 || rows == 0 || cols == 0) return CSRT_OK;
    CSRT_ARG(batch == 1 || o_stride >= (int64_t)(rows - 1) * o->ld + cols ||
                 (o_stride >= cols && o->ld >= (batch - 1) * o_stride + cols),
             "the matrices of o overlap");
    const int64_t g_bytes = ((batch - 1) * g_stride + (int64_t)(rows - 1) * g->ld + cols) * dt_size(g->dtype);
    const int64_t o_bytes = ((batch - 1) * o_stride + (int64_t)(rows - 1) * o->ld + cols) * dt_size(o->dtype);
    const int64_t m_bytes = (int64_t)batch * rows * cols * 4;
    CSRT_ARG(!extents_meet(o->data, o_bytes, g->data, g_bytes), "o overlaps g");
    CSRT_ARG(momentum == nullptr || (!extents_meet(o->data, o_bytes, momentum, m_bytes) &&
                                     !extents_meet(g->data, g_bytes, momentum, m_bytes)),
             "momentum overlaps g or o");
    CSRT_ARG(reinterpret_cast<uintptr_t>(momentum) % 4 == 0, "momentum is not aligned to its type");
    CSRT_ARG(ws != nullptr && (reinterpret_cast<uintptr_t>(ws) & 255) == 0, "workspace is NULL or not 256-byte aligned");
    const OrthoLayout l = layout(batch, rows, cols);
    if (ws_bytes < kWsReservedBytes + l.total)
        return fail(CSRT_ERR_WORKSPACE, "workspace has %zu bytes, needs %zu", ws_bytes, kWsReservedBytes + l.total);
    cudaStream_t s = as_stream(stream);
    char *base = ws_scratch(ws);

    PrepArgs p = {};
    p.g.p = g->data;
    p.g.ld = g->ld;
    p.g.stride = g_stride;
    p.g.dtype = g->dtype;
    p.mom = momentum;
    p.beta = beta;
    p.eps = eps;
    p.scale = scale;
    p.nesterov = nesterov != 0;
    p.rows = rows;
    p.cols = cols;
    p.vec = cols % 8 == 0 && tma_rows_ok(g->data, g->ld, dt_size(g->dtype)) && (g_stride * dt_size(g->dtype)) % 16 == 0 &&
            (reinterpret_cast<uintptr_t>(momentum) & 15) == 0;
    p.partial = reinterpret_cast<double *>(base + l.partial);
    p.hi = reinterpret_cast<__half *>(base + l.x0);
    p.x = reinterpret_cast<float *>(base + l.xf);
    p.ldx = l.ldx;
    p.done = reinterpret_cast<uint32_t *>(base + l.done);
    p.direct = steps == 0;
    p.o.p = o->data;
    p.o.ld = o->ld;
    p.o.stride = o_stride;
    p.o.dtype = o->dtype;
    p.o.vec = tma_store_ok(o->data, o->ld, cols, dt_size(o->dtype)) && (batch == 1 || o_stride * dt_size(o->dtype) % 16 == 0);
    const int64_t chunks = rows * (((int64_t)cols + 7) / 8);
    int64_t blocks = imin<int64_t>(ceil_div<int64_t>(chunks, kPrepThreads), kPrepBlocks);
    blocks = imin<int64_t>(blocks, imax<int64_t>(1, (int64_t)num_sms() * 8 / batch));
    const dim3 grid((unsigned)blocks, (unsigned)batch);
    launch_pdl(ortho_momentum_kernel, grid, dim3(kPrepThreads), 0, s, p);
    launch_pdl(ortho_scale_kernel, grid, dim3(kPrepThreads), 0, s, p);
    count_launch(2);
    rc = check_launch("ortho_scale_kernel");
    if (rc != CSRT_OK || steps == 0) return rc;

    NsPlan plan;
    plan.first = 0;
    plan.batch = batch;
    plan.rows = rows;
    plan.cols = cols;
    plan.steps = steps;
    plan.scale = scale;
    plan.base = base;
    plan.l = l;
    plan.o = p.o;
    plan.direct = p.o.vec && p.o.dtype == CSRT_DT_BF16;
    plan.ws = ws;
    rc = ns_products(plan, s);
    if (rc != CSRT_OK || plan.direct) return rc;
    const unsigned gx = (unsigned)imin<int64_t>(ceil_div<int64_t>(cols, 256), 1024);
    const unsigned gy = (unsigned)imin<int64_t>(rows, imax<int64_t>(1, imin<int64_t>(65535, (int64_t)num_sms() * 64 / gx)));
    launch_pdl(ortho_result_kernel, dim3(gx, gy, (unsigned)batch), dim3(256), 0, s,
               reinterpret_cast<const float *>(base + l.xf), l.ldx, rows, cols, scale * kInvXScale, p.o);
    count_launch();
    return check_launch("ortho_result_kernel");
}

}  // extern "C"
