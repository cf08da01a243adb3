// The global norm of the gradients of a network and their clipping (csrt_grad_norm, csrt_grad_clip):
//   norm = sqrt(sum over all matrices of x^2),   out = x min(1, max_norm / norm)
// Bound by HBM traffic. A launch carries its matrices as arguments, so nothing is copied to the device first and a captured
// graph holds all it needs.
#include <cmath>

#include "block_norm.cuh"
#include "gemm16_host.cuh"
#include "mat.cuh"

namespace csrt {

constexpr int kGradUnit = 8192;     // elements that a block takes at a time
constexpr int kGradBlocks = 608;    // four blocks of 256 threads an SM
constexpr int kGradThreads = 256;

struct GradEntry {
    const char *p;
    char *o;
    int64_t ld, ldo;
    int64_t unit0;          // first unit of this matrix within the launch
    int64_t count;          // elements
    int32_t cols;
    uint8_t dt, dto;
    uint8_t flat, flat_o;   // rows follow one another without a gap: 1, and the first is 16-byte aligned: 2
};

template <int N>
struct GradArgs {
    GradEntry e[N];
    int32_t entries;
    int64_t units;
    int32_t first, last;    // of the launches of one call
    float max_norm;         // 0: only the norm
    float *norm;
    double *partial;        // kGradBlocks
    int32_t *ticket;
    WsHeader *hdr;
};

template <int N>
__device__ __forceinline__ const GradEntry &grad_entry(const GradArgs<N> &a, int64_t unit) {
    int lo = 0, hi = a.entries - 1;   // last entry with unit0 <= unit
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (a.e[mid].unit0 <= unit) lo = mid;
        else hi = mid - 1;
    }
    return a.e[lo];
}

// Element i of a matrix whose rows lie apart. Not inlined: the division takes registers from the loops that never need it.
__device__ __noinline__ int64_t strided(int64_t i, int32_t cols, int64_t ld) { return i / cols * ld + i % cols; }
template <typename T>
__device__ __forceinline__ float grad_at(const GradEntry &e, int64_t i) {
    const T *q = reinterpret_cast<const T *>(e.p);
    return to_f<T>(e.flat ? q[i] : q[strided(i, e.cols, e.ld)]);
}

// Vectors, past the first-level cache.
template <int BYTES>
__device__ __forceinline__ void load_words(const void *p, uint32_t (&w)[BYTES / 4]) {
    if constexpr (BYTES == 16)
        asm volatile("ld.global.L1::no_allocate.v4.b32 {%0, %1, %2, %3}, [%4];"
                     : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3])
                     : "l"(p));
    else
        asm volatile("ld.global.L1::no_allocate.v2.b32 {%0, %1}, [%2];" : "=r"(w[0]), "=r"(w[1]) : "l"(p));
}
template <int BYTES>
__device__ __forceinline__ void store_words(void *p, const uint32_t (&w)[BYTES / 4]) {
    if constexpr (BYTES == 16) *static_cast<uint4 *>(p) = make_uint4(w[0], w[1], w[2], w[3]);
    else *static_cast<uint2 *>(p) = make_uint2(w[0], w[1]);
}
template <typename T>
__device__ __forceinline__ float word_at(const uint32_t *w, int k) {
    if constexpr (sizeof(T) == 4) {
        return __uint_as_float(w[k]);
    } else {
        const unsigned short h = (unsigned short)(w[k >> 1] >> (16 * (k & 1)));
        return to_f<T>(*reinterpret_cast<const T *>(&h));
    }
}

// The squares of a thread's 32 elements of a unit: float32 sums unless they overflow, or underflow without being zero.
// By vectors, all fetched together, then what is left of the last one; by elements where vectors are not aligned.
// hold: shared memory that keeps the vectors, or NULL.
template <typename T>
__device__ __forceinline__ double unit_squares(const GradEntry &e, int64_t base, uint4 *hold) {
    constexpr int N = 16 / (int)sizeof(T), kEach = kGradUnit / (kGradThreads * N);
    const int count = (int)imin<int64_t>(e.count - base, kGradUnit);
    const int vectors = e.flat == 2 ? count / N : 0;
    float t[4] = {0.f};
    uint32_t some = 0;
    uint32_t w[kEach][4];
    const char *p = e.p + (base + threadIdx.x * N) * (int64_t)sizeof(T);
#pragma unroll
    for (int u = 0; u < kEach; ++u) {
        if (u * kGradThreads + (int)threadIdx.x < vectors) load_words<16>(p + u * kGradThreads * 16, w[u]);
        else w[u][0] = w[u][1] = w[u][2] = w[u][3] = 0;
    }
    if (hold != nullptr)
#pragma unroll
        for (int u = 0; u < kEach; ++u) hold[u * kGradThreads + threadIdx.x] = make_uint4(w[u][0], w[u][1], w[u][2], w[u][3]);
#pragma unroll
    for (int u = 0; u < kEach; ++u) {
#pragma unroll
        for (int k = 0; k < 4; ++k) some |= w[u][k] & (sizeof(T) == 4 ? 0x7fffffffu : 0x7fff7fffu);
#pragma unroll
        for (int k = 0; k < N; ++k) {
            const float v = word_at<T>(w[u], k);
            t[k & 3] = fmaf(v, v, t[k & 3]);
        }
    }
    float s = (t[0] + t[1]) + (t[2] + t[3]);
    for (int i = vectors * N + threadIdx.x; i < count; i += kGradThreads) {
        const float v = grad_at<T>(e, base + i);
        s = fmaf(v, v, s);
        some |= v != 0.f;
    }
    // below 2^-80 squares that float32 does not hold (under 2^-126) could matter
    if ((s >= 8.271806e-25f && s <= 3.4028235e38f) || some == 0) return s;
    double d = 0.;
    auto add = [&](int i) {
        const double v = grad_at<T>(e, base + i);
        d += v * v;
    };
    for (int u = threadIdx.x; u < vectors; u += kGradThreads)   // the same elements
        for (int k = 0; k < N; ++k) add(u * N + k);
    for (int i = vectors * N + threadIdx.x; i < count; i += kGradThreads) add(i);
    return d;
}

__device__ __forceinline__ double squares_of(const GradEntry &e, int64_t base, uint4 *hold) {
    return e.dt == CSRT_DT_F32    ? unit_squares<float>(e, base, hold)
           : e.dt == CSRT_DT_BF16 ? unit_squares<__nv_bfloat16>(e, base, hold)
                                  : unit_squares<__half>(e, base, hold);
}

// Sum over the block in a fixed order; the first thread gets it.
__device__ __forceinline__ double block_sum(double v, double (&part)[kGradThreads / 32]) {
#pragma unroll
    for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = v;
    __syncthreads();
    v = 0.;
    if (threadIdx.x == 0)
        for (int w = 0; w < kGradThreads / 32; ++w) v += part[w];
    __syncthreads();
    return v;
}

// The factor for a sum of squares; with `norm` both are written and what is not finite is flagged.
__device__ __forceinline__ float clip_factor(float max_norm, double squares, float *norm, WsHeader *hdr) {
    const double root = sqrt(squares);
    const bool finite = root <= 1.7976931348623157e308;
    const float factor = max_norm > 0.f && finite && root > max_norm ? (float)(max_norm / root) : 1.f;
    if (norm != nullptr) {
        if (!finite) dev_flag(hdr, CSRT_DEV_NONFINITE);
        norm[0] = (float)root;
        norm[1] = factor;
    }
    return factor;
}

template <int N>
__global__ void __launch_bounds__(kGradThreads, 4) grad_norm_kernel(const __grid_constant__ GradArgs<N> a) {
    pdl_enter();
    __shared__ double part[kGradThreads / 32];
    __shared__ bool last;
    double s = 0.;
    for (int64_t u = blockIdx.x; u < a.units; u += gridDim.x) {
        const GradEntry &e = grad_entry(a, u);
        s += squares_of(e, (u - e.unit0) * kGradUnit, nullptr);
    }
    s = block_sum(s, part);
    if (threadIdx.x == 0) {
        a.partial[blockIdx.x] = a.first ? s : a.partial[blockIdx.x] + s;
        last = false;
        if (a.last) {
            __threadfence();
            last = atomicAdd(a.ticket, 1) == (int)gridDim.x - 1;
        }
    }
    __syncthreads();
    if (!last) return;
    __threadfence();
    s = 0.;
    for (int b = threadIdx.x; b < gridDim.x; b += kGradThreads) s += __ldcg(a.partial + b);
    s = block_sum(s, part);
    if (threadIdx.x == 0) {
        clip_factor(a.max_norm, s, a.norm, a.hdr);
        *a.ticket = 0;
    }
}

template <typename T, typename TO, int N>
__device__ __forceinline__ void scale_vector(char *o, const uint32_t *w, float factor) {
    uint32_t x[N * sizeof(TO) / 4];
#pragma unroll
    for (int k = 0; k < N; k += 4 / (int)sizeof(TO)) {
        if constexpr (sizeof(TO) == 4) {
            x[k] = __float_as_uint(word_at<T>(w, k) * factor);
        } else {
            const TO lo = from_f<TO>(word_at<T>(w, k) * factor), hi = from_f<TO>(word_at<T>(w, k + 1) * factor);
            x[k / 2] = *reinterpret_cast<const unsigned short *>(&lo) | (uint32_t)*reinterpret_cast<const unsigned short *>(&hi) << 16;
        }
    }
    store_words<N * sizeof(TO)>(o, x);
}
// hold: the unit's vectors as unit_squares kept them, or NULL.
template <typename T, typename TO>
__device__ __forceinline__ void unit_scale(const GradEntry &e, int64_t base, float factor, const char *hold) {
    constexpr int N = sizeof(T) == 2 && sizeof(TO) == 2 ? 8 : 4, kEach = kGradUnit / (kGradThreads * N);
    constexpr int kIn = N * (int)sizeof(T), kOut = N * (int)sizeof(TO);
    const int count = (int)imin<int64_t>(e.count - base, kGradUnit);
    const int vectors = e.flat == 2 && e.flat_o == 2 ? count / N : 0;
    const char *p = e.p + (base + threadIdx.x * N) * (int64_t)sizeof(T);
    char *o = e.o + (base + threadIdx.x * N) * (int64_t)sizeof(TO);
    if (hold != nullptr) {
        const int held = imin(vectors, count / (16 / (int)sizeof(T)) * (16 / (int)sizeof(T)) / N);
#pragma unroll 4
        for (int u = threadIdx.x; u < held; u += kGradThreads) {
            uint32_t w[kIn / 4];
#pragma unroll
            for (int k = 0; k < kIn / 4; ++k) w[k] = reinterpret_cast<const uint32_t *>(hold + u * kIn)[k];
            scale_vector<T, TO, N>(e.o + (base + u * N) * (int64_t)sizeof(TO), w, factor);
        }
        for (int u = held + threadIdx.x; u < vectors; u += kGradThreads) {   // beyond the last whole 16 bytes
            uint32_t w[kIn / 4];
            load_words<kIn>(e.p + (base + u * N) * (int64_t)sizeof(T), w);
            scale_vector<T, TO, N>(e.o + (base + u * N) * (int64_t)sizeof(TO), w, factor);
        }
    } else if (vectors == kGradUnit / N) {
        uint32_t w[kEach][kIn / 4];
#pragma unroll
        for (int u = 0; u < kEach; ++u) load_words<kIn>(p + u * kGradThreads * kIn, w[u]);
#pragma unroll
        for (int u = 0; u < kEach; ++u) scale_vector<T, TO, N>(o + u * kGradThreads * kOut, w[u], factor);
        return;
    } else {
#pragma unroll 2
        for (int u = 0; u < kEach; ++u) {
            if (u * kGradThreads + (int)threadIdx.x >= vectors) break;
            uint32_t w[kIn / 4];
            load_words<kIn>(p + u * kGradThreads * kIn, w);
            scale_vector<T, TO, N>(o + u * kGradThreads * kOut, w, factor);
        }
    }
    TO *out = reinterpret_cast<TO *>(e.o);
    for (int i = vectors * N + threadIdx.x; i < count; i += kGradThreads) {
        const int64_t at = base + i;
        out[e.flat_o ? at : strided(at, e.cols, e.ldo)] = from_f<TO>(grad_at<T>(e, at) * factor);
    }
}
template <typename T>
__device__ __forceinline__ void unit_scale_to(const GradEntry &e, int64_t base, float factor, const char *hold) {
    if (e.dto == CSRT_DT_F32) unit_scale<T, float>(e, base, factor, hold);
    else if (e.dto == CSRT_DT_BF16) unit_scale<T, __nv_bfloat16>(e, base, factor, hold);
    else unit_scale<T, __half>(e, base, factor, hold);
}
__device__ __forceinline__ void scale_of(const GradEntry &e, int64_t base, float factor, const char *hold) {
    if (factor == 1.f && e.o == e.p && e.dt == e.dto) return;
    if (e.dt == CSRT_DT_F32) unit_scale_to<float>(e, base, factor, hold);
    else if (e.dt == CSRT_DT_BF16) unit_scale_to<__nv_bfloat16>(e, base, factor, hold);
    else unit_scale_to<__half>(e, base, factor, hold);
}

// From the last unit to the first: the norm's pass has left some of the last ones in the second-level cache (25 of 235 MB).
// Loads marked to leave it last brought 4% (58.7M float32 gradients 113 -> 108 us) and would have stayed in other calls' way.
template <int N>
__global__ void __launch_bounds__(kGradThreads, 4) grad_scale_kernel(const __grid_constant__ GradArgs<N> a) {
    pdl_enter();
    const float factor = __ldcg(a.norm + 1);
    for (int64_t u = a.units - 1 - blockIdx.x; u >= 0; u -= gridDim.x) {
        const GradEntry &e = grad_entry(a, u);
        scale_of(e, (u - e.unit0) * kGradUnit, factor, nullptr);
    }
}

// Norm and scaling in one launch, for no more units than two blocks an SM: each block keeps its unit in shared memory, waits
// for the others' sums (cooperative launch: all run at the same time), adds them all by itself in one order and scales.
// 60 tensors of 1 to 100000: 7.2 us, in two launches 9.2. With four blocks an SM it is no faster (4.8M float32 in 18 tensors
// 16.4 in a stream, two launches 15.0), nor with several units a block (58.7M: 111 us, two launches 110): the second launch
// reads and writes at the copy rate.
constexpr int kHoldBytes = kGradUnit * (int)sizeof(float);
constexpr int kGaveUp = 1 << 30;   // in the count of sums that have come: a wait for them ran out

template <int N>
__global__ void __launch_bounds__(kGradThreads, 2) grad_clip_kernel(const __grid_constant__ GradArgs<N> a) {
    pdl_enter();
    extern __shared__ __align__(16) char hold[];
    __shared__ double part[kGradThreads / 32];
    __shared__ float scale;
    const GradEntry &e = grad_entry(a, blockIdx.x);
    const int64_t base = (blockIdx.x - e.unit0) * kGradUnit;
    double s = squares_of(e, base, reinterpret_cast<uint4 *>(hold));
    s = block_sum(s, part);
    if (threadIdx.x == 0) {
        const int all = (int)gridDim.x;
        a.partial[blockIdx.x] = s;
        __threadfence();
        atomicAdd(a.ticket, 1);
        int seen = 0;
        for (unsigned spin = 0; spin < kSpinLimit; ++spin) {
            asm volatile("ld.acquire.gpu.global.s32 %0, [%1];" : "=r"(seen) : "l"(a.ticket) : "memory");
            if (seen == all || (seen & kGaveUp) != 0) break;
            if (spin > 16) __nanosleep(20);
        }
        // one outcome for all blocks: the count is complete and stays so, or it is marked before that (each try that fails
        // met another block's arrival)
        while (seen != all && (seen & kGaveUp) == 0) {
            const int old = atomicCAS(a.ticket, seen, seen | kGaveUp);
            seen = old == seen ? seen | kGaveUp : old;
            __threadfence();
        }
        if (seen != all) dev_flag(a.hdr, CSRT_DEV_TIMEOUT);
        scale = seen == all ? 1.f : -1.f;
    }
    __syncthreads();
    const bool come = scale > 0.f;   // else the others' sums never came: nothing is written
    s = 0.;
    for (int b = threadIdx.x; come && b < gridDim.x; b += kGradThreads) s += __ldcg(a.partial + b);
    s = block_sum(s, part);
    if (threadIdx.x == 0) {
        if (come) scale = clip_factor(a.max_norm, s, blockIdx.x == 0 ? a.norm : nullptr, a.hdr);
        else if (blockIdx.x == 0) a.norm[0] = a.norm[1] = NAN;
        // the last block to have read the first counter leaves both as they were
        if (atomicAdd(a.ticket + 1, 1) == (int)gridDim.x - 1) {
            a.ticket[1] = 0;
            a.ticket[0] = 0;
        }
    }
    __syncthreads();
    if (!come) return;
    scale_of(e, base, scale, hold);
}

// ---------------------------------------------------------------------------
// Host
// ---------------------------------------------------------------------------
static size_t grad_bytes() { return kWsReservedBytes + align_up(kGradBlocks * sizeof(double), 256); }

static int check_grads(const csrt_mat *g, int32_t count, const csrt_mat *out, float *norm, void *ws, size_t ws_bytes) {
    CSRT_ARG(count >= 0, "count is negative");
    CSRT_ARG(count == 0 || g != nullptr, "g is NULL");
    CSRT_ARG(norm != nullptr, "norm is NULL");
    CSRT_TRY(check_vector(norm, "norm"));
    for (int32_t k = 0; k < count; ++k) {
        CSRT_TRY(check_mat(g + k, "g"));
        CSRT_ARG(!vector_meets(norm, 2, g + k), "norm overlaps g[%d]", k);
        if (out == nullptr) continue;
        CSRT_TRY(check_mat(out + k, "out"));
        CSRT_TRY(check_shape(out + k, "out", g[k].rows, g[k].cols));
        CSRT_ARG(same_place(out + k, g + k) || !clash(out + k, g + k), "out[%d] overlaps g[%d]", k, k);
        CSRT_ARG(!vector_meets(norm, 2, out + k), "norm overlaps out[%d]", k);
    }
    CSRT_ARG(ws != nullptr, "workspace is NULL");
    CSRT_ARG((reinterpret_cast<uintptr_t>(ws) & 255) == 0, "workspace is not 256-byte aligned");
    if (ws_bytes < grad_bytes()) return fail(CSRT_ERR_WORKSPACE, "workspace has %zu bytes, needs %zu", ws_bytes, grad_bytes());
    return CSRT_OK;
}

static uint8_t flatness(const csrt_mat &m) {
    if (m.rows > 1 && m.ld != m.cols) return 0;
    return (reinterpret_cast<uintptr_t>(m.data) & 15) == 0 ? 2 : 1;
}

template <int N>
static int grad_once(const GradArgs<N> &a, cudaStream_t s) {
    CSRT_TRY(allow_smem<grad_clip_kernel<N>>(kHoldBytes));
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeCooperative;
    attr[0].val.cooperative = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)a.units);
    cfg.blockDim = dim3(kGradThreads);
    cfg.dynamicSmemBytes = kHoldBytes;
    cfg.stream = s;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    CSRT_CHECK_CUDA(cudaLaunchKernelEx(&cfg, grad_clip_kernel<N>, a));
    count_launch();
    return CSRT_OK;
}

template <int N>
static int grad_launch(const csrt_mat *g, int32_t count, float max_norm, const csrt_mat *out, float *norm, void *ws,
                       cudaStream_t s) {
    // matrices that hold something, N a launch; the norm's launches come first
    int32_t full = 0;
    int64_t all = 0;
    for (int32_t k = 0; k < count; ++k) {
        const int64_t c = (int64_t)g[k].rows * g[k].cols;
        full += c > 0;
        all += ceil_div<int64_t>(c, kGradUnit);
    }
    const unsigned blocks = (unsigned)imax<int64_t>(1, imin<int64_t>(all, kGradBlocks));
    const bool once = max_norm > 0.f && full <= N && full > 0 && all <= 2 * num_sms();
    for (int pass = 0; pass < (max_norm > 0.f ? 2 : 1); ++pass) {
        int32_t done = 0, k = 0;
        do {
            GradArgs<N> a;
            a.entries = 0;
            a.units = 0;
            for (; k < count && a.entries < N; ++k) {
                const csrt_mat &m = g[k], &o = out != nullptr ? out[k] : g[k];
                const int64_t c = (int64_t)m.rows * m.cols;
                if (c == 0) continue;
                GradEntry &e = a.e[a.entries++];
                e.p = static_cast<const char *>(m.data);
                e.o = static_cast<char *>(o.data);
                e.ld = m.ld;
                e.ldo = o.ld;
                e.unit0 = a.units;
                e.count = c;
                e.cols = m.cols;
                e.dt = (uint8_t)m.dtype;
                e.dto = (uint8_t)o.dtype;
                e.flat = flatness(m);
                e.flat_o = flatness(o);
                a.units += ceil_div<int64_t>(c, kGradUnit);
                ++done;
            }
            a.first = done == a.entries;
            a.last = done == full;
            a.max_norm = max_norm;
            a.norm = norm;
            a.partial = reinterpret_cast<double *>(ws_scratch(ws));
            a.ticket = ws_counters(ws);
            a.hdr = static_cast<WsHeader *>(ws);
            if (once) return grad_once(a, s);
            if (pass == 0) {
                launch_pdl(grad_norm_kernel<N>, dim3(blocks), dim3(kGradThreads), 0, s, a);
                count_launch();
                CSRT_TRY(check_launch("grad_norm_kernel"));
            } else if (a.units > 0) {
                launch_pdl(grad_scale_kernel<N>, dim3((unsigned)imin<int64_t>(a.units, kGradBlocks)), dim3(kGradThreads), 0, s, a);
                count_launch();
                CSRT_TRY(check_launch("grad_scale_kernel"));
            }
        } while (done < full);
    }
    return CSRT_OK;
}

static int grad_call(const csrt_mat *g, int32_t count, float max_norm, const csrt_mat *out, float *norm, void *ws,
                     void *stream) {
    if (count <= 16) return grad_launch<16>(g, count, max_norm, out, norm, ws, as_stream(stream));
    return grad_launch<256>(g, count, max_norm, out, norm, ws, as_stream(stream));
}

}  // namespace csrt

using namespace csrt;

extern "C" {

int csrt_grad_workspace_bytes(size_t *bytes) {
    CSRT_ARG(bytes != nullptr, "bytes is NULL");
    *bytes = grad_bytes();
    return CSRT_OK;
}

int csrt_grad_norm(const csrt_mat *g, int32_t count, float *norm, void *ws, size_t ws_bytes, void *stream) {
    CSRT_TRY(check_grads(g, count, nullptr, norm, ws, ws_bytes));
    return grad_call(g, count, 0.f, nullptr, norm, ws, stream);
}

int csrt_grad_clip(const csrt_mat *g, int32_t count, float max_norm, const csrt_mat *out, float *norm, void *ws,
                   size_t ws_bytes, void *stream) {
    CSRT_TRY(check_grads(g, count, out, norm, ws, ws_bytes));
    CSRT_ARG(std::isfinite(max_norm) && max_norm > 0.f, "max_norm must be finite and > 0");
    return grad_call(g, count, max_norm, out, norm, ws, stream);
}

}  // extern "C"
