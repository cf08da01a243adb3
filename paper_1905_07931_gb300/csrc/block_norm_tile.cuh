// The kernels of the norms around a block that read every matrix once (block_norm.cuh has the arguments).
//
// A norm reduces down the columns of a feature-major matrix, so a tile is TT tokens wide and as high as the matrix: d
// features are split over the blocks of a cluster, which exchange their sums through distributed shared memory. Each thread
// holds V tokens (eight, or one where there are one or two in all) of F features, the same from the first load to the last
// store. A cluster walks over the tiles of tokens, and the next tile's loads are issued as soon as the present one's are in
// registers: they run while sums are exchanged and results stored.
//
// Aligned inputs (16-byte rows) come by TMA. Fetched by cp.async, with the same overlap, the threads stood at the issue of
// their loads for 15% to 35% of the time, as the memory pipe takes only so many.
// Other rows (U): a thread fetches the aligned words that its eight tokens touch by cp.async, into shared memory that no
// other thread reads, and shifts them into place by its row's offset, which is the same for all of its features and tiles.
// Results whose rows are unaligned, or end inside a vector (UOUT), pass through shared memory of the warp's and leave by single elements, 32 tokens of
// a row (or fewer of several) a store.
#pragma once

#include <atomic>
#include <cmath>
#include <type_traits>

#include "block_norm.cuh"
#include "gemm16_host.cuh"

namespace csrt {

constexpr int kNormWarps = 8;
constexpr int kNormThreads = kNormWarps * 32;
constexpr int kNormClusterMax = 16;
constexpr int kLoader = kNormThreads - 32;   // the thread that issues TMA loads

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

// V values that lie side by side, on a 16-byte boundary where V is eight.
template <int V>
__device__ __forceinline__ void load_tokens(const float *p, typename Tok<V>::P (&x)[Tok<V>::N]) {
    if constexpr (V == 1) {
        x[0] = *p;
    } else {
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            const ulonglong2 v = reinterpret_cast<const ulonglong2 *>(p)[k];
            x[2 * k] = v.x;
            x[2 * k + 1] = v.y;
        }
    }
}

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

// Eight elements, from the 32-bit words that hold them.
template <typename T>
__device__ __forceinline__ void unpack_words(const uint32_t *u, f32x2 (&x)[4]) {
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        if constexpr (sizeof(T) == 4) {
            x[k] = pack2(__uint_as_float(u[2 * k]), __uint_as_float(u[2 * k + 1]));
        } else if constexpr (std::is_same<T, __nv_bfloat16>::value) {
            x[k] = pack2(__uint_as_float(u[k] << 16), __uint_as_float(u[k] & 0xffff0000u));
        } else {
            const float2 v = __half22float2(*reinterpret_cast<const __half2 *>(u + k));
            x[k] = pack2(v.x, v.y);
        }
    }
}
template <typename T>
__device__ __forceinline__ void unpack_words(const uint4 *w, f32x2 (&x)[4]) {
    uint32_t u[8];
#pragma unroll
    for (int k = 0; k < (int)sizeof(T) / 2; ++k) {
        const uint4 v = w[k];
        u[4 * k] = v.x;
        u[4 * k + 1] = v.y;
        u[4 * k + 2] = v.z;
        u[4 * k + 3] = v.w;
    }
    unpack_words<T>(u, x);
}

// Inputs by TMA: the block's features x TT tokens of one matrix, a row after the other.
template <typename T, int TT, int F>
struct Tiled {
    static constexpr int kSize = (int)sizeof(T);
    static constexpr int kRow = TT * kSize;
    static constexpr int kTotal = Place<TT, 8>::kStep * F * kRow;
    static __device__ __forceinline__ int offset(const char *) { return 0; }
    static __device__ __forceinline__ void read(const char *base, int f, int, f32x2 (&x)[4]) {
        const Place<TT, 8> at;
        unpack_words<T>(reinterpret_cast<const uint4 *>(base + (at.row0 + f * at.kStep) * kRow + at.q * kSize), x);
    }
};

// A thread's own copies of one matrix: F x V elements of type T in shared memory, 16-byte words of it (V = 8, one more than
// they fill) or 4-byte ones (V = 1).
template <typename T, int TT, int V, int F>
struct Held {
    static constexpr int kSize = (int)sizeof(T);
    static constexpr int kWord = V == 8 ? 16 : 4;
    static constexpr int kWords = V == 8 ? kSize / 2 + 1 : 1;   // for one feature
    static constexpr int kTotal = kWords * kWord * F * kNormThreads;
    // How far a row's first token of this thread lies behind an aligned word, in elements.
    static __device__ __forceinline__ int offset(const char *src) {
        return (int)(reinterpret_cast<uintptr_t>(src) & (kWord - 1)) / kSize;
    }
    // `src` is the matrix's first element of this thread's column and first feature. nv tokens and the features below `rows`
    // are fetched and the rest is zeros. What shares an aligned word with an element in front of it is read too, nothing
    // behind a row's last element.
    static __device__ __forceinline__ void fetch(char *base, const char *src, int64_t ld, int rows, int row0, int nv) {
        const uint32_t dst = (uint32_t)__cvta_generic_to_shared(base) + threadIdx.x * kWord;
        const int64_t step = ld * (int64_t)(kSize * Place<TT, V>::kStep);
        const int before = offset(src) * kSize;
        src -= before;
        const char *none = reinterpret_cast<const char *>(reinterpret_cast<uintptr_t>(src) & ~(uintptr_t)15);
        int bytes[kWords];
#pragma unroll
        for (int k = 0; k < kWords; ++k) bytes[k] = nv > 0 ? imin(imax(before + nv * kSize - k * kWord, 0), kWord) : 0;
#pragma unroll
        for (int f = 0; f < F; ++f, src += step) {
            const bool have = row0 + f * Place<TT, V>::kStep < rows;
#pragma unroll
            for (int k = 0; k < kWords; ++k) {
                const int here = have ? bytes[k] : 0;
                const char *at = here > 0 ? src + kWord * k : none;
                if (V == 8) cp_async16(dst + (f * kWords + k) * kNormThreads * 16, at, here);
                else cp_async4(dst + f * kNormThreads * 4, at, here);
            }
        }
    }
    // off: offset() of the thread's elements
    static __device__ __forceinline__ void read(const char *base, int f, int off, typename Tok<V>::P (&x)[Tok<V>::N]) {
        if constexpr (V == 1) {
            const uint32_t w = reinterpret_cast<const uint32_t *>(base)[f * kNormThreads + threadIdx.x];
            if constexpr (kSize == 4) x[0] = __uint_as_float(w);
            else if constexpr (std::is_same<T, __nv_bfloat16>::value) x[0] = __uint_as_float(off ? w & 0xffff0000u : w << 16);
            else x[0] = __half2float(__ushort_as_half((unsigned short)(off ? w >> 16 : w & 0xffffu)));
        } else {
            constexpr int kOut = kSize * 2;      // 32-bit words of eight elements
            uint32_t u[kWords * 4];
#pragma unroll
            for (int k = 0; k < kWords; ++k) {
                const uint4 w = reinterpret_cast<const uint4 *>(base)[(f * kWords + k) * kNormThreads + threadIdx.x];
                u[4 * k] = w.x;
                u[4 * k + 1] = w.y;
                u[4 * k + 2] = w.z;
                u[4 * k + 3] = w.w;
            }
            const int words = kSize == 4 ? off : off >> 1;
            if (words & 2)
#pragma unroll
                for (int k = 0; k < kOut + 2; ++k) u[k] = u[k + 2];
            if (words & 1)
#pragma unroll
                for (int k = 0; k < kOut + 1; ++k) u[k] = u[k + 1];
            if constexpr (kSize == 2) {
                const int bits = (off & 1) * 16;
#pragma unroll
                for (int k = 0; k < kOut; ++k) u[k] = __funnelshift_r(u[k], u[k + 1], bits);
            }
            unpack_words<T>(u, x);
        }
    }
};

template <bool TMA, typename T, int TT, int V, int F>
struct InputOf {
    typedef Held<T, TT, V, F> type;
};
template <typename T, int TT, int F>
struct InputOf<true, T, TT, 8, F> {
    typedef Tiled<T, TT, F> type;
};

// One result matrix: where a thread's elements of a tile go.
template <typename T, int TT, int V, bool U>
struct Result {
    static constexpr int kSize = (int)sizeof(T);
    static constexpr int kStageBytes = U && V == 8 ? 32 * 8 * kSize : 0;   // of a warp
    static constexpr int kRowsStore = V == 8 && U ? 32 / TT : 1;           // features that one store of the warp spans
    char *p;        // this lane's first element
    int64_t row;    // bytes from a feature to the next
    int tokens;     // this lane's that exist
    // first: the warp's first feature in the matrix; c0: the tile's first token
    __device__ __forceinline__ Result(const NormMat &m, int64_t first, int64_t c0, int32_t n) {
        const int lane = threadIdx.x & 31;
        constexpr int each = U ? 1 : V, lanes = TT / each;
        const int64_t c = c0 + (lane % lanes) * each;
        row = m.ld * kSize;
        p = m.p + (first + lane / lanes) * row + c * kSize;
        tokens = (int)imax<int64_t>(0, imin<int64_t>(each, n - c));
    }
    // Feature f of the thread (row0 its first within the block, of `rows`; none of 0); `stage` is the warp's.
    __device__ __forceinline__ void put(char *stage, int f, int row0, int rows, const typename Tok<V>::P (&x)[Tok<V>::N]) {
        char *dst = p + f * Place<TT, V>::kStep * row;
        if constexpr (V == 1) {
            if (tokens > 0 && row0 + f * Place<TT, V>::kStep < rows) *reinterpret_cast<T *>(dst) = from_f<T>(x[0]);
        } else {
            uint4 w[kSize / 2];
            if constexpr (kSize == 4) {
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    float a, b, c, d;
                    unpack2(x[2 * k], a, b);
                    unpack2(x[2 * k + 1], c, d);
                    w[k] = make_uint4(__float_as_uint(a), __float_as_uint(b), __float_as_uint(c), __float_as_uint(d));
                }
            } else {
                uint32_t u[4];
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    float a, b;
                    unpack2(x[k], a, b);
                    if constexpr (std::is_same<T, __nv_bfloat16>::value) {
                        const __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
                        u[k] = *reinterpret_cast<const uint32_t *>(&h);
                    } else {
                        const __half2 h = __floats2half2_rn(a, b);
                        u[k] = *reinterpret_cast<const uint32_t *>(&h);
                    }
                }
                w[0] = make_uint4(u[0], u[1], u[2], u[3]);
            }
            if constexpr (U) {
                const int lane = threadIdx.x & 31;
                const int own = (threadIdx.x >> 5) * Place<TT, V>::kRowsWarp + f * Place<TT, V>::kStep + lane / TT;
#pragma unroll
                for (int k = 0; k < kSize / 2; ++k) reinterpret_cast<uint4 *>(stage)[lane * (kSize / 2) + k] = w[k];
                __syncwarp();
#pragma unroll
                for (int j = 0; j < 8; ++j, dst += kRowsStore * row) {
                    const T v = reinterpret_cast<const T *>(stage)[lane + 32 * j];
                    if (tokens > 0 && own + j * kRowsStore < rows) *reinterpret_cast<T *>(dst) = v;
                }
                __syncwarp();
            } else if (tokens > 0 && row0 + f * Place<TT, V>::kStep < rows) {   // eight exist, or none
#pragma unroll
                for (int k = 0; k < kSize / 2; ++k) reinterpret_cast<uint4 *>(dst)[k] = w[k];
            }
        }
    }
};

// ---------------------------------------------------------------------------
// Sums over all features of a token: over a thread's features, the lanes that hold the same tokens, the warps, the
// cluster's blocks. One or two sums a token, or its mean and sum of square deviations, which are merged by the formula of
// Chan, Golub and LeVeque: no cancellation, and one exchange instead of two.
//
// Blocks write their totals into each other's shared memory by st.async, which counts on the receiver's mbarrier: a cluster
// barrier in its place waits for the stores of results in flight too (a tenth of the forward kernel's stalls).
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

// Bounded wait for a phase of an mbarrier: about a second, as try_wait suspends the thread for a microsecond at most. It never
// runs out while the cluster lives: results of a wait that did are NaN.
#ifndef CSRT_NORM_IN_TIME
#define CSRT_NORM_IN_TIME true   // a test takes every wait as one that ran out, once it is over
#endif
constexpr unsigned kNormWaits = 1u << 20;
__device__ __forceinline__ bool norm_wait(uint64_t *bar, uint32_t parity, WsHeader *hdr) {
    const uint32_t addr = smem_u32(bar);
    for (unsigned i = 0; i < kNormWaits; ++i) {
        uint32_t done;
        asm volatile(
            "{\n .reg .pred p;\n mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2, %3;\n"
            " selp.u32 %0, 1, 0, p;\n}\n"
            : "=r"(done)
            : "r"(addr), "r"(parity), "r"(1000u)
            : "memory");
        if (done && CSRT_NORM_IN_TIME) return true;
        if (done) break;
    }
    if (hdr != nullptr) dev_flag(hdr, CSRT_DEV_TIMEOUT);
    return false;
}

template <int TT>
struct Exchange {
    static constexpr int kTokensWarp = TT >= kNormWarps ? TT / kNormWarps : 1;   // tokens that a warp sums up
    float2 *slots;    // [2][cluster][TT], written by the cluster's blocks
    float2 *part;     // [warps][TT]
    float *last;      // [2][2][TT]: two results a token
    uint64_t *bar;    // [2]; behind them two for loads
    float *part_n;    // [warps]
    WsHeader *hdr;    // takes a flag if a wait runs out, may be NULL
    int turn;         // exchanges so far: halves alternate, as a block may be one exchange ahead of another
    int size, rank, chunk, d;
    float inv_d;

    static constexpr int bytes(int size) {
        return (int)sizeof(float2) * TT * (kNormWarps + 2 * size + 2) + kNormWarps * (int)sizeof(float) + 4 * (int)sizeof(uint64_t);
    }
    __device__ __forceinline__ Exchange(char *base, int size_, int rank_, int chunk_, int d_, WsHeader *hdr_)
        : hdr(hdr_), turn(0), size(size_), rank(rank_), chunk(chunk_), d(d_), inv_d(1.f / (float)d_) {
        slots = reinterpret_cast<float2 *>(base);
        part = slots + 2 * size * TT;
        last = reinterpret_cast<float *>(part + kNormWarps * TT);
        bar = reinterpret_cast<uint64_t *>(last + 4 * TT);
        part_n = reinterpret_cast<float *>(bar + 4);
        if (threadIdx.x == 0) {
            for (int k = 0; k < 4; ++k) mbar_init(bar + k, 1);
            asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        }
        __syncthreads();
        if (size > 1) asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
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

// Joins the values of the eight lanes that differ in the lowest three bits; all get one result.
template <int MODE>
__device__ __forceinline__ void join_lanes(float &a, float &b, float &n) {
    const unsigned full = 0xffffffffu;
#pragma unroll
    for (int o = 1; o < 8; o <<= 1) {
        const float nb = MODE == kMoments ? __shfl_xor_sync(full, n, o) : 0.f;
        const float a2 = __shfl_xor_sync(full, a, o), b2 = MODE != kOneSum ? __shfl_xor_sync(full, b, o) : 0.f;
        merge<MODE>(a, b, n, a2, b2, nb);
        n += nb;
    }
    if (MODE == kMoments) {   // the merge is not symmetric to the last bit
        const int first = threadIdx.x & 24;
        a = __shfl_sync(full, a, first);
        b = __shfl_sync(full, b, first);
    }
}

// a, b: this thread's values for its V tokens, over n of its features. finish(token, total) turns a token's totals into two
// results, which every thread gets for its tokens (x, y). freed() runs once all threads of the block have come here.
template <int MODE, int TT, int V, typename FIN, typename FREED>
__device__ __forceinline__ void exchange(Exchange<TT> &e, float (&a)[V], float (&b)[V], float n, int q, FIN finish, FREED freed,
                                         typename Tok<V>::P (&x)[Tok<V>::N], typename Tok<V>::P (&y)[Tok<V>::N]) {
    constexpr int kLanes = Place<TT, V>::kLanes;
    static_assert(V == 1 || Place<TT, V>::kRowsWarp >= V || kLanes * Place<TT, V>::kRowsWarp == 32, "lanes");
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
    const int half = e.turn & 1, parity = (e.turn >> 1) & 1;
    ++e.turn;
    if (copy == 0) e.part[warp * TT + token] = make_float2(a[0], MODE != kOneSum ? b[0] : 0.f);
    if (MODE == kMoments && lane == 0) e.part_n[warp] = n;
    const uint32_t bar = (uint32_t)__cvta_generic_to_shared(e.bar + half);
    if (e.size > 1 && threadIdx.x == 0)
        asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(e.size * TT * 8) : "memory");
    __syncthreads();
    freed();
    // a warp joins its tokens' eight parts, a lane each
    constexpr int kMine = Exchange<TT>::kTokensWarp;
    const int j = lane & 7, t = (TT >= kNormWarps ? warp * kMine : 0) + (lane >> 3) % kMine;
    const bool mine = lane < 8 * kMine && (TT >= kNormWarps || warp == 0);   // the others hold copies
    float2 s = e.part[j * TT + t];
    float sn = MODE == kMoments ? e.part_n[j] : 0.f;
    join_lanes<MODE>(s.x, s.y, sn);
    if (e.size > 1) {
        float2 *slots = e.slots + half * e.size * TT;
        if (mine) {
            const uint32_t own = (uint32_t)__cvta_generic_to_shared(slots + e.rank * TT + t);
            for (int r = j; r < e.size; r += 8) {
                uint32_t at, there;
                asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(at) : "r"(own), "r"(r));
                asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(there) : "r"(bar), "r"(r));
                asm volatile("st.async.shared::cluster.mbarrier::complete_tx::bytes.b64 [%0], %1, [%2];" ::"r"(at),
                             "l"(pack2(s.x, s.y)), "r"(there)
                             : "memory");
            }
        }
        const bool ok = norm_wait(e.bar + half, parity, e.hdr);
        s = make_float2(0.f, 0.f);
        sn = 0.f;
        for (int r = j; r < e.size; r += 8) {
            const float2 v = slots[r * TT + t];
            const float nb = (float)imax(0, imin(e.chunk, e.d - r * e.chunk));
            merge<MODE>(s.x, s.y, sn, v.x, v.y, nb);
            sn += nb;
        }
        __syncwarp();
        join_lanes<MODE>(s.x, s.y, sn);
        if (!ok) s = make_float2(NAN, NAN);
    }
    s = finish(t, s);
    float *out = e.last + half * 2 * TT;
    if (mine && j == 0) {
        out[t] = s.x;
        out[TT + t] = s.y;
    }
    __syncthreads();
    load_tokens<V>(out + q, x);
    load_tokens<V>(out + TT + q, y);
}

// 1 / sqrt(v): the approximation and a Newton step (r first: half of a subnormal v would not be exact)
__device__ __forceinline__ float rsqrt_near(float v) {
    const float r = rsqrtf(v);
    return v <= 3.4028235e38f ? r * fmaf(-0.5f * r * v, r, 1.5f) : r;
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
// p = sigmoid(g) and q = 1 - p = e^-g p, which keeps its digits where p is near 1 (the product is NaN where e^-g is infinite
// and p is 0: the minimum takes 1).
template <bool FAST>
__device__ __forceinline__ void sigmoid2(f32x2 g, f32x2 &p, f32x2 &q) {
    float a, b, c, d;
    f32x2 e;
    if (FAST) {
        unpack2(mul2(g, pack2(-1.44269504f, -1.44269504f)), a, b);
        e = pack2(exp2_fast(a), exp2_fast(b));
        unpack2(add2(e, pack2(1.f, 1.f)), a, b);
        p = pack2(rcp_fast(a), rcp_fast(b));
    } else {
        unpack2(g, a, b);
        a = expf(-a);
        b = expf(-b);
        e = pack2(a, b);
        p = pack2(1.f / (1.f + a), 1.f / (1.f + b));
    }
    unpack2(mul2(e, p), c, d);
    q = pack2(fminf(c, 1.f), fminf(d, 1.f));
}
template <bool FAST>
__device__ __forceinline__ void sigmoid2(float g, float &p, float &q) {
    const float e = FAST ? exp2_fast(g * -1.44269504f) : expf(-g);
    p = FAST ? rcp_fast(1.f + e) : 1.f / (1.f + e);
    q = fminf(e * p, 1.f);
}

__device__ __forceinline__ f32x2 above_m128(f32x2 g) {
    float a, b;
    unpack2(g, a, b);
    return pack2(above_m128(a), above_m128(b));
}
__device__ __forceinline__ f32x2 within_128(f32x2 g) {
    float a, b;
    unpack2(g, a, b);
    return pack2(within_128(a), within_128(b));
}

// a(g) and a'(g) of V tokens. GATE: CSRT_GATE_*, known to the compiler, so that the features of a thread's loop are not
// separated by branches and their latencies overlap.
template <int GATE, bool FAST, typename P>
__device__ __forceinline__ void gate_of(P g, P one, P &value, P &slope) {
    value = g;
    slope = one;
    if (GATE == CSRT_GATE_NONE) return;
    if (GATE == CSRT_GATE_SILU) g = above_m128(g);   // before the sigmoid, which is the same: no second copy of g lives
    P p, q;
    sigmoid2<FAST>(g, p, q);
    value = GATE == CSRT_GATE_SILU ? mul2(p, g) : p;
    slope = GATE == CSRT_GATE_SILU ? mul2(p, fma2(within_128(g), q, one)) : mul2(p, q);
}
template <typename F>
__device__ __forceinline__ void with_gate(int act, F body) {
    if (act == CSRT_GATE_SIGMOID) body(std::integral_constant<int, CSRT_GATE_SIGMOID>());
    else if (act == CSRT_GATE_SILU) body(std::integral_constant<int, CSRT_GATE_SILU>());
    else body(std::integral_constant<int, CSRT_GATE_NONE>());
}

// ---------------------------------------------------------------------------
// Host: the cluster that d features take, and how many of them a GPU holds at once.
// ---------------------------------------------------------------------------
template <int TT, int V, int F>
struct TileShape {
    static constexpr int kFeatures = Place<TT, V>::kStep * F;   // of a block
    static int cluster(int32_t d) {
        const int64_t c = ceil_div<int64_t>(d, kFeatures);
        return c <= kNormClusterMax ? (int)c : 0;
    }
};

// A block's share of the features: `box` of them a TMA load, `boxes` loads.
struct Share {
    int chunk, box, boxes;
};
inline Share norm_share(int32_t d, int size, int most, bool tma) {
    Share s = {(int)ceil_div<int64_t>(d, size), 0, 0};
    if (!tma) return s;
    for (s.boxes = ceil_div(s.chunk, 256);; ++s.boxes) {   // a box is at most 256 rows, of whole 128 bytes of shared memory
        s.box = ceil_div(ceil_div(s.chunk, s.boxes), 8) * 8;
        if (s.box * s.boxes <= most) break;
    }
    s.chunk = s.box * s.boxes;
    return s;
}

struct NormMaps {
    CUtensorMap m[5];
};
inline bool norm_map(CUtensorMap *map, const NormMat &m, int dtype, const NormArgs &a, int width) {
    return m.p == nullptr || make_map3(map, m.p, dtype, a.d, a.n, m.ld, 1, 0, width, a.box, CU_TENSOR_MAP_SWIZZLE_NONE);
}
template <typename T>
constexpr int dtype_of() {
    return sizeof(T) == 4 ? CSRT_DT_F32 : std::is_same<T, __half>::value ? CSRT_DT_F16 : CSRT_DT_BF16;
}
// All boxes of one matrix's tile, by one thread.
__device__ __forceinline__ void load_tile(char *dst, const CUtensorMap *map, const NormArgs &a, int rank, int64_t token, int row_bytes,
                                          uint64_t *bar) {
    for (int k = 0; k < a.boxes; ++k)
        asm volatile(
            "cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];" ::"r"(
                smem_u32(dst + k * a.box * row_bytes)),
            "l"(reinterpret_cast<uint64_t>(map)), "r"((int)token), "r"(rank * a.chunk + k * a.box), "r"(0), "r"(smem_u32(bar))
            : "memory");
}

// Zeros in the features of a tile that no box brings.
template <typename H>
__device__ __forceinline__ void clear_rows(char *tile, int chunk) {
    for (int i = chunk * H::kRow + (int)threadIdx.x * 4; i < H::kTotal; i += kNormThreads * 4) *reinterpret_cast<uint32_t *>(tile + i) = 0;
}

// Launches `kernel` on clusters of `size` blocks, as many as fit or as there are tiles (a.groups).
template <auto kernel>
int launch_clusters(NormArgs &a, const NormMaps &maps, int size, int64_t tiles, int smem, cudaStream_t s) {
    // by what a block holds, so that a call gives the same clusters (and sums over tokens the same order) whatever came before;
    // threads that come first at the same time find the same
    static std::atomic<uint16_t> fit[64][kNormClusterMax + 1][32];
    const int holds = (a.y.p != nullptr) | (a.g.p != nullptr) << 1 | (a.r.p != nullptr) << 2 | (a.h.p != nullptr) << 3 |
                      (a.dv.p != nullptr) << 4;
    int dev = 0;
    CSRT_ARG(size > 0, "a cluster cannot hold %d features", a.d);
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
    int resident = fit[dev][size][holds].load(std::memory_order_relaxed);
    if (resident == 0) {
        CSRT_CHECK_CUDA(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, 226 * 1024));
        CSRT_CHECK_CUDA(cudaFuncSetAttribute(kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1));
        cfg.numAttrs = 1;
        int n = 0;
        CSRT_CHECK_CUDA(cudaOccupancyMaxActiveClusters(&n, kernel, &cfg));
        resident = imin(imax(1, n), 65535);
        fit[dev][size][holds].store((uint16_t)resident, std::memory_order_relaxed);
    }
    a.cluster = size;
    a.groups = (int32_t)imin<int64_t>(imin<int64_t>(tiles, resident), kNormGroups);
    cfg.gridDim = dim3((unsigned)(a.groups * size));
    cfg.numAttrs = 2;
    CSRT_CHECK_CUDA(cudaLaunchKernelEx(&cfg, kernel, a, maps));
    count_launch();
    return CSRT_OK;
}

}  // namespace csrt
