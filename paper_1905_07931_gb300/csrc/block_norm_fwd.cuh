// Forward kernel of the norms around a block (block_norm_tile.cuh says how a tile is held).
#pragma once

#include "block_norm_tile.cuh"

namespace csrt {

// Mean (negated) and reciprocal deviation of this thread's V tokens, over all features; `rows` of the block's features
// exist, x is zero beyond them. Written out by the cluster's first block.
template <int TT, int V, int F>
__device__ __forceinline__ void tile_stats(Exchange<TT> &ex, const NormSide &s, const Place<TT, V> &at, int rows, int64_t c0,
                                           int32_t n, const typename Tok<V>::P (&x)[F][Tok<V>::N],
                                           typename Tok<V>::P (&m)[Tok<V>::N], typename Tok<V>::P (&r)[Tok<V>::N]) {
    typedef Tok<V> T;
    float a[V], b[V];
    float2 own;
    typename T::P sq[T::N];
#pragma unroll
    for (int k = 0; k < T::N; ++k) sq[k] = T::all(0.f);
    if (s.kind == CSRT_NORM_LAYER) {
        float cnt = 0.f;
        typename T::P sum[T::N];
#pragma unroll
        for (int k = 0; k < T::N; ++k) sum[k] = T::all(0.f);
#pragma unroll
        for (int f = 0; f < F; ++f) {
            cnt += at.row0 + f * at.kStep < rows ? 1.f : 0.f;
#pragma unroll
            for (int k = 0; k < T::N; ++k) sum[k] = add2(sum[k], x[f][k]);
        }
        const float inv = cnt > 0.f ? -1.f / cnt : 0.f;
#pragma unroll
        for (int k = 0; k < T::N; ++k) sum[k] = mul2(sum[k], T::all(inv));
#pragma unroll
        for (int f = 0; f < F; ++f)
            if (at.row0 + f * at.kStep < rows)
#pragma unroll
                for (int k = 0; k < T::N; ++k) {
                    const typename T::P v = add2(x[f][k], sum[k]);
                    sq[k] = fma2(v, v, sq[k]);
                }
#pragma unroll
        for (int k = 0; k < T::N; ++k) {
            T::put(a, k, mul2(sum[k], T::all(-1.f)));
            T::put(b, k, sq[k]);
        }
        own = cluster_total<kMoments>(ex, a, b, cnt);
    } else {
#pragma unroll
        for (int f = 0; f < F; ++f)
#pragma unroll
            for (int k = 0; k < T::N; ++k) sq[k] = fma2(x[f][k], x[f][k], sq[k]);
#pragma unroll
        for (int k = 0; k < T::N; ++k) T::put(a, k, sq[k]);
        own = make_float2(0.f, cluster_total<kOneSum>(ex, a, b, 0.f).x);
    }
    own.y = rsqrt_near(fmaf(own.y, ex.inv_d, s.eps));
    const int64_t c = c0 + (threadIdx.x & 31);
    if (ex.rank == 0 && threadIdx.x < TT && c < n) {
        if (s.mean != nullptr && s.kind == CSRT_NORM_LAYER) s.mean[c] = own.x;
        if (s.rstd != nullptr) s.rstd[c] = own.y;
    }
    own.x = -own.x;
    to_tokens(ex, own, at.q, a, b);
#pragma unroll
    for (int k = 0; k < T::N; ++k) {
        m[k] = T::get(a, k);
        r[k] = T::get(b, k);
    }
}

template <typename TB, typename TS, int TT, int V, int F>
__global__ void __launch_bounds__(kNormThreads, 2) norm_fwd_tile_kernel(const __grid_constant__ NormArgs a) {
    pdl_enter();
    extern __shared__ __align__(16) char held[];
    typedef Tok<V> T;
    typedef Held<TB, TT, V, F> HB;
    typedef Held<TS, TT, V, F> HS;
    typedef typename T::P P;
    constexpr bool kFast = sizeof(TB) == 2;
    constexpr int kFeatures = Place<TT, V>::kStep * F;
    const Place<TT, V> at;
    const int size = a.cluster;
    const int rank = size > 1 ? (int)(blockIdx.x % size) : 0;
    const int chunk = (a.d + size - 1) / size;
    const int rows = imax(0, imin(chunk, a.d - rank * chunk));
    const int64_t i0 = (int64_t)rank * chunk + (at.row0 < rows ? at.row0 : 0);
    char *sy = held, *sg = sy + (a.y.p ? HB::kTotal : 0), *sr = sg + (a.g.p ? HB::kTotal : 0);
    float2 *wpost = reinterpret_cast<float2 *>(sr + (a.r.p ? HS::kTotal : 0)), *wpre = wpost + kFeatures;   // weight, bias
    Exchange<TT> ex(reinterpret_cast<char *>(wpre + kFeatures), size, rank, chunk, a.d);
    const int64_t tiles = ((int64_t)a.n + TT - 1) / TT;
    int64_t tile = blockIdx.x / size;

    auto column = [&](int64_t t) { return t * TT + at.q; };
    auto exist = [&](int64_t t) { return (int)imax<int64_t>(0, imin<int64_t>(V, a.n - column(t))); };
    auto fetch = [&](int64_t t) {
        const int nv = exist(t);
        const int64_t c = nv > 0 ? column(t) : 0;
        const bool full = rows == kFeatures && (t + 1) * TT <= a.n;
        if (a.y.p) HB::fetch(sy, a.y.p + (i0 * a.y.ld + c) * sizeof(TB), a.y.ld, full, rows, at.row0, nv);
        if (a.g.p) HB::fetch(sg, a.g.p + (i0 * a.g.ld + c) * sizeof(TB), a.g.ld, full, rows, at.row0, nv);
        if (a.r.p) HS::fetch(sr, a.r.p + (i0 * a.r.ld + c) * sizeof(TS), a.r.ld, full, rows, at.row0, nv);
    };
    // bit 1 of the address of a 2-byte element: the same for all of a thread's features and tiles (kStep and TT are even,
    // or TT is 1)
    auto odd = [&](const NormMat &m, int64_t c) {
        return V == 1 && (((reinterpret_cast<uintptr_t>(m.p) >> 1) + (uint32_t)(i0 * m.ld + c)) & 1) != 0;
    };
    fetch(tile);
    // weights; zeros beyond `rows`, so that what is computed there is zero
    for (int i = threadIdx.x; i < kFeatures; i += kNormThreads) {
        const int64_t j = (int64_t)rank * chunk + i;
        float2 p = make_float2(0.f, 0.f), q = p;
        if (i < rows) {
            p.x = a.post.w != nullptr ? a.post.w[j] : 1.f;
            q.x = a.pre.w != nullptr ? a.pre.w[j] : 1.f;
            if (a.post.b != nullptr) p.y = a.post.b[j];
            if (a.pre.b != nullptr) q.y = a.pre.b[j];
        }
        wpost[i] = p;
        wpre[i] = q;
    }
    __syncthreads();
    ex.started();

    for (; tile < tiles; tile += a.groups) {
        const int nv = exist(tile);
        const int64_t c = column(tile);
        P x[F][T::N], m[T::N], r[T::N];
        char *ph = a.h.p + (i0 * a.h.ld + c) * sizeof(TS);
        const int64_t step_h = a.h.ld * (int64_t)(sizeof(TS) * at.kStep);
        auto put_h = [&](int f) {
            if (a.h.p) {
                if (at.row0 + f * at.kStep < rows) put_tokens<TS, V>(ph, x[f], nv);
                ph += step_h;
            }
        };
        cp_async_wait();
        const bool odd_r = odd(a.r, c);
        if (a.y.p) {
            const bool odd_y = odd(a.y, c), odd_g = odd(a.g, c);
#pragma unroll
            for (int f = 0; f < F; ++f) HB::read(sy, f, odd_y, x[f]);
#pragma unroll
            for (int k = 0; k < T::N; ++k) {
                m[k] = T::all(0.f);
                r[k] = T::all(1.f);
            }
            if (a.post.kind > CSRT_NORM_SCALE) tile_stats<TT, V, F>(ex, a.post, at, rows, tile * TT, a.n, x, m, r);
#pragma unroll
            for (int f = 0; f < F; ++f) {
                const float2 w = wpost[at.row0 + f * at.kStep];
#pragma unroll
                for (int k = 0; k < T::N; ++k)
                    x[f][k] = fma2(add2(x[f][k], m[k]), mul2(r[k], T::all(w.x)), T::all(w.y));
                if (a.g.p) {
                    P g[T::N], v[T::N];
                    HB::read(sg, f, odd_g, g);
                    if (a.gate_act != CSRT_GATE_NONE) {
#pragma unroll
                        for (int k = 0; k < T::N; ++k) v[k] = sigmoid2<kFast>(g[k]);
                        if (a.gate_act == CSRT_GATE_SILU)
#pragma unroll
                            for (int k = 0; k < T::N; ++k) v[k] = mul2(v[k], g[k]);
                    } else {
#pragma unroll
                        for (int k = 0; k < T::N; ++k) v[k] = g[k];
                    }
#pragma unroll
                    for (int k = 0; k < T::N; ++k) x[f][k] = mul2(x[f][k], v[k]);
                }
                if (a.r.p) {
                    P r0[T::N];
                    HS::read(sr, f, odd_r, r0);
#pragma unroll
                    for (int k = 0; k < T::N; ++k) x[f][k] = fma2(r0[k], T::all(a.r_scale), x[f][k]);
                }
                put_h(f);
            }
        } else {
#pragma unroll
            for (int f = 0; f < F; ++f) {
                HS::read(sr, f, odd_r, x[f]);
#pragma unroll
                for (int k = 0; k < T::N; ++k) x[f][k] = mul2(x[f][k], T::all(a.r_scale));
                put_h(f);
            }
        }
        if (tile + a.groups < tiles) fetch(tile + a.groups);
        if (!a.v.p) continue;
#pragma unroll
        for (int k = 0; k < T::N; ++k) {
            m[k] = T::all(0.f);
            r[k] = T::all(1.f);
        }
        if (a.pre.kind > CSRT_NORM_SCALE) tile_stats<TT, V, F>(ex, a.pre, at, rows, tile * TT, a.n, x, m, r);
        char *pv = a.v.p + (i0 * a.v.ld + c) * sizeof(TB);
        const int64_t step_v = a.v.ld * (int64_t)(sizeof(TB) * at.kStep);
#pragma unroll
        for (int f = 0; f < F; ++f, pv += step_v) {
            const float2 w = wpre[at.row0 + f * at.kStep];
            P v[T::N];
#pragma unroll
            for (int k = 0; k < T::N; ++k) v[k] = fma2(add2(x[f][k], m[k]), mul2(r[k], T::all(w.x)), T::all(w.y));
            if (at.row0 + f * at.kStep < rows) put_tokens<TB, V>(pv, v, nv);
        }
    }
    ex.leave();
}

template <typename TB, typename TS, int TT, int V, int F>
int norm_fwd_tile(const NormArgs &a, cudaStream_t s) {
    const int size = TileShape<TT, V, F>::cluster(a.d);
    const int smem = (a.y.p ? Held<TB, TT, V, F>::kTotal : 0) + (a.g.p ? Held<TB, TT, V, F>::kTotal : 0) +
                     (a.r.p ? Held<TS, TT, V, F>::kTotal : 0) + TileShape<TT, V, F>::kFeatures * 16 +
                     Exchange<TT>::bytes(size);
    return launch_clusters<norm_fwd_tile_kernel<TB, TS, TT, V, F>>(a, size, ceil_div<int64_t>(a.n, TT), smem, s);
}

template <typename TB, typename TS>
int norm_fwd_tiles(const NormArgs &a, NormTile t, cudaStream_t s) {
    if constexpr (sizeof(TB) == 2) {
        switch (t) {
            case kTile32x8x8: return norm_fwd_tile<TB, TS, 32, 8, 8>(a, s);
            case kTile32x8x4: return norm_fwd_tile<TB, TS, 32, 8, 4>(a, s);
            case kTile32x8x2: return norm_fwd_tile<TB, TS, 32, 8, 2>(a, s);
            case kTile16x8x8: return norm_fwd_tile<TB, TS, 16, 8, 8>(a, s);
            default: break;
        }
    }
    switch (t) {
        case kTile32x1x32: return norm_fwd_tile<TB, TS, 32, 1, 32>(a, s);
        case kTile32x1x16: return norm_fwd_tile<TB, TS, 32, 1, 16>(a, s);
        case kTile16x1x32: return norm_fwd_tile<TB, TS, 16, 1, 32>(a, s);
        case kTile8x1x32: return norm_fwd_tile<TB, TS, 8, 1, 32>(a, s);
        case kTile1x1x16: return norm_fwd_tile<TB, TS, 1, 1, 16>(a, s);
        case kTile1x1x4: return norm_fwd_tile<TB, TS, 1, 1, 4>(a, s);
        default: return fail(CSRT_ERR_ARG, "unknown tile %d", (int)t);
    }
}

}  // namespace csrt
