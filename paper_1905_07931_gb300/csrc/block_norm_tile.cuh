// The kernels of the norms around a block that read every matrix once (block_norm.cuh has the arguments).
//
// A norm reduces down the columns of a feature-major matrix, so a tile is TT tokens wide and as high as the matrix: d
// features are split over the blocks of a cluster, which exchange their sums through distributed shared memory. Each thread
// holds V tokens (a vector of 16 bytes, or one) of F features, the same from the first load to the last store; what it
// loads goes by cp.async into shared memory that no other thread reads. A cluster walks over the tiles of tokens, and the
// next tile's loads are issued as soon as the present one's are in registers: they run while sums are exchanged and results
// stored.
//
// Rows that are not 16-byte aligned take V = 1: an element's aligned 4-byte word is fetched, and its half picked.
#pragma once

#include <cmath>
#include <mutex>
#include <type_traits>

#include "block_norm.cuh"
#include "mat.cuh"

namespace csrt {

constexpr int kNormWarps = 8;
constexpr int kNormThreads = kNormWarps * 32;
constexpr int kNormClusterMax = 16;

// V tokens as packed pairs (two float32 operations an instruction), or one.
typedef unsigned long long f32x2;
__device__ __forceinline__ f32x2 pack2(float a, float b) {
    f32x2 r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
    return r;
}
__device__ __forceinline__ void unpack2(f32x2 v, float &a, float &b) { asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(v)); }
__device__ __forceinline__ f32x2 fma2(f32x2 a, f32x2 b, f32x2 c) {
    f32x2 r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
    return r;
}
__device__ __forceinline__ f32x2 mul2(f32x2 a, f32x2 b) {
    f32x2 r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ f32x2 add2(f32x2 a, f32x2 b) {
    f32x2 r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ float fma2(float a, float b, float c) { return fmaf(a, b, c); }
__device__ __forceinline__ float mul2(float a, float b) { return a * b; }
__device__ __forceinline__ float add2(float a, float b) { return a + b; }

template <int V>
struct Tok;
template <>
struct Tok<8> {
    static constexpr int N = 4;
    typedef f32x2 P;
    static __device__ __forceinline__ P all(float v) { return pack2(v, v); }
    static __device__ __forceinline__ P get(const float *v, int k) { return pack2(v[2 * k], v[2 * k + 1]); }
    static __device__ __forceinline__ void put(float *v, int k, P p) { unpack2(p, v[2 * k], v[2 * k + 1]); }
    static __device__ __forceinline__ float sum(P p) {
        float a, b;
        unpack2(p, a, b);
        return a + b;
    }
};
template <>
struct Tok<1> {
    static constexpr int N = 1;
    typedef float P;
    static __device__ __forceinline__ P all(float v) { return v; }
    static __device__ __forceinline__ P get(const float *v, int) { return *v; }
    static __device__ __forceinline__ void put(float *v, int, P p) { *v = p; }
    static __device__ __forceinline__ float sum(P p) { return p; }
};

__device__ __forceinline__ void cp_async16(uint32_t dst, const char *src, int bytes) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(bytes) : "memory");
}
__device__ __forceinline__ void cp_async4(uint32_t dst, const char *src, int bytes) {
    asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(dst), "l"(src), "r"(bytes) : "memory");
}
__device__ __forceinline__ void cp_async_wait() { asm volatile("cp.async.wait_all;" ::: "memory"); }

// Where a thread stands: its features are row0 + f * kStep of the block's `rows`, from feature i0 on.
template <int TT, int V>
struct Place {
    static constexpr int kLanes = TT / V;              // lanes along a row
    static constexpr int kRowsWarp = 32 / kLanes;      // features a warp spans at a time
    static constexpr int kStep = kRowsWarp * kNormWarps;
    int row0, q;
    __device__ __forceinline__ Place() {
        const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
        row0 = warp * kRowsWarp + lane / kLanes;
        q = (lane % kLanes) * V;
    }
};

// A thread's own copies of one matrix: F x V elements of type T in shared memory.
template <typename T, int TT, int V, int F>
struct Held {
    static constexpr int kWords = V == 8 ? (int)sizeof(T) / 2 : 1;       // of 16 bytes (V = 8) or 4, for one feature
    static constexpr int kTotal = kWords * (V == 8 ? 16 : 4) * F * kNormThreads;
    // `src` is the matrix's first element of this thread's column and first feature. Where not all of the tile exists
    // (!full), nv tokens and the features below `rows` are fetched and the rest is zeros.
    static __device__ __forceinline__ void fetch(char *base, const char *src, int64_t ld, bool full, int rows, int row0, int nv) {
        uint32_t dst = (uint32_t)__cvta_generic_to_shared(base) + threadIdx.x * (V == 8 ? 16 : 4);
        const int64_t step = ld * (int64_t)(sizeof(T) * Place<TT, V>::kStep);
        // V = 1: the high half of a word lies behind bytes before it, the low half is fetched alone: nothing past the element
        const bool high = V == 1 && sizeof(T) == 2 && (reinterpret_cast<uintptr_t>(src) & 2) != 0;
        const int bytes = sizeof(T) == 4 || high ? 4 : 2;
        if (high) src -= 2;
        const char *none = reinterpret_cast<const char *>(reinterpret_cast<uintptr_t>(src) & ~(uintptr_t)15);
#pragma unroll
        for (int f = 0; f < F; ++f, src += step) {
            if constexpr (V == 8) {
                if (full) {
#pragma unroll
                    for (int k = 0; k < kWords; ++k) cp_async16(dst + (f * kWords + k) * kNormThreads * 16, src + 16 * k, 16);
                } else {
                    constexpr int each = 16 / (int)sizeof(T);
                    const int have = row0 + f * Place<TT, V>::kStep < rows ? nv : 0;
#pragma unroll
                    for (int k = 0; k < kWords; ++k) {
                        const int here = imin(imax(have - k * each, 0), each);
                        cp_async16(dst + (f * kWords + k) * kNormThreads * 16, here > 0 ? src + 16 * k : none, here * (int)sizeof(T));
                    }
                }
            } else {
                const bool have = full || (nv > 0 && row0 + f * Place<TT, V>::kStep < rows);
                cp_async4(dst + f * kNormThreads * 4, have ? src : none, have ? bytes : 0);
            }
        }
    }
    // `odd`: V = 1 and 2-byte elements: bit 1 of this element's address
    static __device__ __forceinline__ void read(const char *base, int f, bool odd, typename Tok<V>::P (&x)[Tok<V>::N]) {
        if constexpr (V == 1) {
            const uint32_t w = reinterpret_cast<const uint32_t *>(base)[f * kNormThreads + threadIdx.x];
            if constexpr (sizeof(T) == 4) x[0] = __uint_as_float(w);
            else if constexpr (std::is_same<T, __nv_bfloat16>::value) x[0] = __uint_as_float(odd ? w & 0xffff0000u : w << 16);
            else x[0] = __half2float(__ushort_as_half((unsigned short)(odd ? w >> 16 : w & 0xffffu)));
        } else if constexpr (sizeof(T) == 4) {
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                const float4 w = reinterpret_cast<const float4 *>(base)[(f * 2 + k) * kNormThreads + threadIdx.x];
                x[2 * k] = pack2(w.x, w.y);
                x[2 * k + 1] = pack2(w.z, w.w);
            }
        } else {
            const uint4 w = reinterpret_cast<const uint4 *>(base)[f * kNormThreads + threadIdx.x];
            const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                if constexpr (std::is_same<T, __nv_bfloat16>::value) {
                    x[k] = pack2(__uint_as_float(u[k] << 16), __uint_as_float(u[k] & 0xffff0000u));
                } else {
                    const float2 v = __half22float2(*reinterpret_cast<const __half2 *>(&u[k]));
                    x[k] = pack2(v.x, v.y);
                }
            }
        }
    }
};

// V values to a row's place; nv of them exist.
template <typename T, int V>
__device__ __forceinline__ void put_tokens(char *dst, const typename Tok<V>::P (&x)[Tok<V>::N], int nv) {
    T *o = reinterpret_cast<T *>(dst);
    if constexpr (V == 1) {
        if (nv > 0) *o = from_f<T>(x[0]);
    } else {
        float v[8];
#pragma unroll
        for (int k = 0; k < 4; ++k) unpack2(x[k], v[2 * k], v[2 * k + 1]);
        if (nv == 8) {
            if constexpr (sizeof(T) == 4) {
                reinterpret_cast<float4 *>(dst)[0] = make_float4(v[0], v[1], v[2], v[3]);
                reinterpret_cast<float4 *>(dst)[1] = make_float4(v[4], v[5], v[6], v[7]);
            } else {
                uint32_t u[4];
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    if constexpr (std::is_same<T, __nv_bfloat16>::value) {
                        const __nv_bfloat162 h = __floats2bfloat162_rn(v[2 * k], v[2 * k + 1]);
                        u[k] = *reinterpret_cast<const uint32_t *>(&h);
                    } else {
                        const __half2 h = __floats2half2_rn(v[2 * k], v[2 * k + 1]);
                        u[k] = *reinterpret_cast<const uint32_t *>(&h);
                    }
                }
                *reinterpret_cast<uint4 *>(dst) = make_uint4(u[0], u[1], u[2], u[3]);
            }
        } else {
#pragma unroll
            for (int k = 0; k < 8; ++k)
                if (k < nv) o[k] = from_f<T>(v[k]);
        }
    }
}

// ---------------------------------------------------------------------------
// Sums over all features of a token: over a thread's features, the lanes that hold the same tokens, the warps, the
// cluster's blocks. One or two sums a token, or its mean and sum of square deviations, which are merged by the formula of
// Chan, Golub and LeVeque: no cancellation, and one exchange instead of two.
//
// Blocks write their totals into each other's shared memory by st.async, which counts on the receiver's mbarrier: a cluster
// barrier in its place waits for the stores of results in flight too (a fifth of the forward kernel's stalls).
// ---------------------------------------------------------------------------
enum { kOneSum, kTwoSums, kMoments };

template <int MODE>
__device__ __forceinline__ void merge(float &a, float &b, float na, float a2, float b2, float nb) {
    if (MODE != kMoments) {
        a += a2;
        if (MODE == kTwoSums) b += b2;
        return;
    }
    const float n = na + nb;
    const float share = n > 0.f ? __fdividef(nb, n) : 0.f, delta = a2 - a;
    a = fmaf(delta, share, a);
    b = b + b2 + delta * delta * (na * share);
}

template <int TT>
struct Exchange {
    float2 *slots;    // [2][cluster][TT], written by the cluster's blocks
    float2 *part;     // [2][warps][TT]; a warp's row of the half that is not in use takes its results to its threads
    float *part_n;    // [2][warps]
    uint64_t *bar;    // [2]
    int turn;         // exchanges so far: halves alternate, as a block may be one exchange ahead of another
    int size, rank, chunk, d;
    float inv_d;

    static constexpr int bytes(int size) {
        return (int)sizeof(float2) * TT * (2 * kNormWarps + 2 * size) + 2 * kNormWarps * (int)sizeof(float) + 2 * (int)sizeof(uint64_t);
    }
    __device__ __forceinline__ Exchange(char *base, int size_, int rank_, int chunk_, int d_)
        : turn(0), size(size_), rank(rank_), chunk(chunk_), d(d_), inv_d(1.f / (float)d_) {
        slots = reinterpret_cast<float2 *>(base);
        part = slots + 2 * size * TT;
        bar = reinterpret_cast<uint64_t *>(part + 2 * kNormWarps * TT);
        part_n = reinterpret_cast<float *>(bar + 2);
        if (size > 1) {
            if (threadIdx.x == 0) {
                for (int k = 0; k < 2; ++k)
                    asm volatile("mbarrier.init.shared::cta.b64 [%0], 1;" ::"r"((uint32_t)__cvta_generic_to_shared(bar + k)) : "memory");
                asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
            }
            __syncthreads();
            asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
        }
    }
    // Every block has started and its barriers are set; before the first exchange.
    __device__ __forceinline__ void started() const {
        if (size > 1) asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
    }
    // No block leaves while another may still write to it.
    __device__ __forceinline__ void leave() const {
        if (size > 1) {
            asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory");
            asm volatile("barrier.cluster.wait.aligned;" ::: "memory");
        }
    }
};

// a, b: this thread's values for its V tokens, over n of its features. Returns the totals for token (lane % TT).
template <int MODE, int TT, int V>
__device__ __forceinline__ float2 cluster_total(Exchange<TT> &x, float (&a)[V], float (&b)[V], float n) {
    constexpr int kLanes = Place<TT, V>::kLanes;
    static_assert(V == 1 || Place<TT, V>::kRowsWarp >= V, "a lane ends with one token");
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const unsigned full = 0xffffffffu;
    int token = (lane % kLanes) * V, copy = 0;   // the first token still held; lanes with `copy` hold another's
    int held = V;
#pragma unroll
    for (int o = 16; o >= kLanes; o >>= 1) {
        const float nb = MODE == kMoments ? __shfl_xor_sync(full, n, o) : 0.f;
        if (held > 1) {   // each of the two lanes goes on with half of the tokens
            const bool up = (lane & o) != 0;
            held >>= 1;
#pragma unroll
            for (int j = 0; j < V / 2; ++j) {
                if (j >= held) break;
                float a2 = up ? a[j] : a[j + held], b2 = 0.f;
                a[j] = up ? a[j + held] : a[j];
                a2 = __shfl_xor_sync(full, a2, o);
                if (MODE != kOneSum) {
                    b2 = up ? b[j] : b[j + held];
                    b[j] = up ? b[j + held] : b[j];
                    b2 = __shfl_xor_sync(full, b2, o);
                }
                merge<MODE>(a[j], b[j], n, a2, b2, nb);
            }
            if (up) token += held;
        } else {
            const float a2 = __shfl_xor_sync(full, a[0], o), b2 = MODE != kOneSum ? __shfl_xor_sync(full, b[0], o) : 0.f;
            merge<MODE>(a[0], b[0], n, a2, b2, nb);
            copy |= lane & o;
        }
        n += nb;
    }
    const int half = x.turn & 1;
    float2 *part = x.part + half * kNormWarps * TT;
    if (copy == 0) part[warp * TT + token] = make_float2(a[0], MODE != kOneSum ? b[0] : 0.f);
    if (MODE == kMoments && lane == 0) x.part_n[half * kNormWarps + warp] = n;
    const uint32_t bar = (uint32_t)__cvta_generic_to_shared(x.bar + half);
    if (x.size > 1 && threadIdx.x == 0)
        asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(x.size * TT * 8) : "memory");
    __syncthreads();
    const int t = lane % TT;
    float2 s = part[t];
    float sn = MODE == kMoments ? x.part_n[half * kNormWarps] : 0.f;
#pragma unroll
    for (int w = 1; w < kNormWarps; ++w) {
        const float2 v = part[w * TT + t];
        const float nb = MODE == kMoments ? x.part_n[half * kNormWarps + w] : 0.f;
        merge<MODE>(s.x, s.y, sn, v.x, v.y, nb);
        sn += nb;
    }
    const int parity = (x.turn >> 1) & 1;
    ++x.turn;
    if (x.size == 1) return s;
    float2 *slots = x.slots + half * x.size * TT;
    const uint32_t own = (uint32_t)__cvta_generic_to_shared(slots + x.rank * TT + t);
    for (int r = warp; r < x.size; r += kNormWarps)
        if (lane < TT) {
            uint32_t at, there;
            asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(at) : "r"(own), "r"(r));
            asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(there) : "r"(bar), "r"(r));
            asm volatile("st.async.shared::cluster.mbarrier::complete_tx::bytes.b64 [%0], %1, [%2];" ::"r"(at),
                         "l"(pack2(s.x, s.y)), "r"(there)
                         : "memory");
        }
    // never runs out while the cluster lives; the results of a wait that did are NaN
    if (!mbar_wait_bounded(x.bar + half, parity)) return make_float2(NAN, NAN);
    s = slots[t];
    sn = (float)imin(x.chunk, x.d);
    for (int r = 1; r < x.size; ++r) {
        const float2 v = slots[r * TT + t];
        const float nb = (float)imax(0, imin(x.chunk, x.d - r * x.chunk));
        merge<MODE>(s.x, s.y, sn, v.x, v.y, nb);
        sn += nb;
    }
    return s;
}

// Two values for each token (a lane's, for token lane % TT) to the threads that hold it, after cluster_total. The row of
// `part` is this warp's own: others read it only before the barrier of the last exchange and after that of the next.
template <int TT, int V>
__device__ __forceinline__ void to_tokens(Exchange<TT> &x, float2 own, int q, float (&a)[V], float (&b)[V]) {
    const int lane = threadIdx.x & 31;
    float2 *mine = x.part + ((x.turn & 1) * kNormWarps + (threadIdx.x >> 5)) * TT;
    __syncwarp();
    if (lane < TT) mine[lane] = own;
    __syncwarp();
#pragma unroll
    for (int k = 0; k < V; ++k) {
        const float2 v = mine[q + k];
        a[k] = v.x;
        b[k] = v.y;
    }
    __syncwarp();
}

// 1 / sqrt(v): the approximation and a Newton step
__device__ __forceinline__ float rsqrt_near(float v) {
    const float r = rsqrtf(v);
    return v <= 3.4028235e38f ? r * fmaf(-0.5f * v * r, r, 1.5f) : r;
}

// exp and quotient of the fast sigmoid: 2^-22 and 2^-23 of the result, 2^-24 |g| from the rounded argument
__device__ __forceinline__ float exp2_fast(float v) {
    asm("ex2.approx.ftz.f32 %0, %0;" : "+f"(v));
    return v;
}
__device__ __forceinline__ float rcp_fast(float v) {
    asm("rcp.approx.ftz.f32 %0, %0;" : "+f"(v));
    return v;
}
template <bool FAST>
__device__ __forceinline__ f32x2 sigmoid2(f32x2 g) {
    float a, b;
    if (FAST) {
        unpack2(mul2(g, pack2(-1.44269504f, -1.44269504f)), a, b);
        f32x2 e = add2(pack2(exp2_fast(a), exp2_fast(b)), pack2(1.f, 1.f));
        unpack2(e, a, b);
        return pack2(rcp_fast(a), rcp_fast(b));
    }
    unpack2(g, a, b);
    return pack2(sigmoid_of<false>(a), sigmoid_of<false>(b));
}
template <bool FAST>
__device__ __forceinline__ float sigmoid2(float g) {
    return FAST ? rcp_fast(1.f + exp2_fast(g * -1.44269504f)) : sigmoid_of<false>(g);
}

// ---------------------------------------------------------------------------
// Host: the cluster that d features take, and how many of them a GPU holds at once.
// ---------------------------------------------------------------------------
template <int TT, int V, int F>
struct TileShape {
    static constexpr int kFeatures = Place<TT, V>::kStep * F;   // of a block
    static int cluster(int32_t d) {
        const int64_t c = ceil_div<int64_t>(d, kFeatures);
        return c <= 8 ? (int)c : c <= kNormClusterMax ? kNormClusterMax : 0;
    }
};

// Launches `kernel` on clusters of `size` blocks, as many as fit or as there are tiles.
template <auto kernel>
int launch_clusters(NormArgs a, int size, int64_t tiles, int smem, cudaStream_t s) {
    static std::mutex lock;
    static int fit[64][kNormClusterMax + 1] = {{0}};
    int dev = 0;
    CSRT_CHECK_CUDA(cudaGetDevice(&dev));
    CSRT_ARG(dev >= 0 && dev < 64, "device %d is out of range", dev);
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = (unsigned)size;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[1].val.programmaticStreamSerializationAllowed = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)size);
    cfg.blockDim = dim3(kNormThreads);
    cfg.dynamicSmemBytes = (size_t)smem;
    cfg.stream = s;
    cfg.attrs = attr;
    int resident;
    {
        std::lock_guard<std::mutex> hold(lock);
        if (fit[dev][size] == 0) {
            CSRT_CHECK_CUDA(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, 227 * 1024));
            CSRT_CHECK_CUDA(cudaFuncSetAttribute(kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1));
            cfg.numAttrs = 1;
            int n = 0;
            CSRT_CHECK_CUDA(cudaOccupancyMaxActiveClusters(&n, kernel, &cfg));
            fit[dev][size] = imax(1, n);
        }
        resident = fit[dev][size];
    }
    a.cluster = size;
    a.groups = (int32_t)imin<int64_t>(imin<int64_t>(tiles, resident), kNormGroups);
    cfg.gridDim = dim3((unsigned)(a.groups * size));
    cfg.numAttrs = 2;
    CSRT_CHECK_CUDA(cudaLaunchKernelEx(&cfg, kernel, a));
    count_launch();
    return CSRT_OK;
}

}  // namespace csrt
