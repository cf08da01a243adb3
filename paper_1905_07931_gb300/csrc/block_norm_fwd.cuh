// Forward kernel of the norms around a block (block_norm_tile.cuh says how a tile is held).
#pragma once

#include "block_norm_tile.cuh"

namespace csrt {

// Mean and reciprocal deviation of this thread's V tokens, over all features; x as above, `rows` of the block's features
// exist. Written out by the cluster's first block.
template <int TT, int V, int F>
__device__ __forceinline__ void tile_stats(Exchange<TT> &ex, const NormSide &s, const Place<TT, V> &at, int rows, int64_t c0,
                                           int32_t n, const typename Tok<V>::P (&x)[F][Tok<V>::N], float (&mean)[V],
                                           float (&rstd)[V]) {
    typedef Tok<V> T;
    float a[V], b[V];
    float2 own;
    if (s.kind == CSRT_NORM_LAYER) {
        float cnt = 0.f;
        typename T::P sum[T::N], sq[T::N];
#pragma unroll
        for (int k = 0; k < T::N; ++k) sum[k] = sq[k] = T::all(0.f);
#pragma unroll
        for (int f = 0; f < F; ++f) {
            cnt += at.row0 + f * at.kStep < rows ? 1.f : 0.f;
#pragma unroll
            for (int k = 0; k < T::N; ++k) sum[k] = add2(sum[k], x[f][k]);   // features beyond `rows` are zeros
        }
        const float inv = cnt > 0.f ? 1.f / cnt : 0.f;
#pragma unroll
        for (int k = 0; k < T::N; ++k) sum[k] = mul2(sum[k], T::all(-inv));
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
        own = cluster_total<true>(ex, a, b, cnt);
    } else {
        typename T::P sq[T::N];
#pragma unroll
        for (int k = 0; k < T::N; ++k) sq[k] = T::all(0.f);
#pragma unroll
        for (int f = 0; f < F; ++f)
#pragma unroll
            for (int k = 0; k < T::N; ++k) sq[k] = fma2(x[f][k], x[f][k], sq[k]);
#pragma unroll
        for (int k = 0; k < V; ++k) a[k] = 0.f;
#pragma unroll
        for (int k = 0; k < T::N; ++k) T::put(b, k, sq[k]);
        own = cluster_total<false>(ex, a, b, 0.f);
    }
    own.y = 1.f / sqrtf(own.y / (float)ex.d + s.eps);
    const int64_t c = c0 + (threadIdx.x & 31);
    if (ex.rank == 0 && threadIdx.x < TT && c < n) {
        if (s.mean != nullptr && s.kind == CSRT_NORM_LAYER) s.mean[c] = own.x;
        if (s.rstd != nullptr) s.rstd[c] = own.y;
    }
    to_tokens(ex, own, at.q, mean, rstd);
}

template <typename TB, typename TS, int TT, int V, int F>
__global__ void __launch_bounds__(kNormThreads, 2) norm_fwd_tile_kernel(const __grid_constant__ NormArgs a) {
    pdl_enter();
    extern __shared__ __align__(16) char held[];
    typedef Tok<V> T;
    typedef Held<TB, TT, V, F> HB;
    typedef Held<TS, TT, V, F> HS;
    constexpr bool kFast = sizeof(TB) == 2;
    const int size = a.cluster;
    const Place<TT, V> at;
    const int rank = size > 1 ? (int)(blockIdx.x % size) : 0;
    const int chunk = (a.d + size - 1) / size;
    const int rows = imax(0, imin(chunk, a.d - rank * chunk));
    const int64_t i0 = (int64_t)rank * chunk + at.row0;
    char *sy = held, *sg = sy + (a.y.p ? HB::kTotal : 0), *sr = sg + (a.g.p ? HB::kTotal : 0),
         *end = sr + (a.r.p ? HS::kTotal : 0);
    Exchange<TT> ex(end, size, rank, chunk, a.d);
    const int64_t tiles = ((int64_t)a.n + TT - 1) / TT;
    int64_t tile = blockIdx.x / size;
    if (size > 1) cluster_arrive();   // every block has started before another writes into its shared memory

    auto column = [&](int64_t t) { return t * TT + at.q; };
    auto exist = [&](int64_t t) { return (int)imax<int64_t>(0, imin<int64_t>(V, a.n - column(t))); };
    auto fetch = [&](int64_t t) {
        const int nv = exist(t);
        const int64_t c = nv > 0 ? column(t) : 0;
        const int64_t i = at.row0 < rows ? i0 : 0;
        if (a.y.p) HB::fetch(sy, a.y.p + (i * a.y.ld + c) * sizeof(TB), a.y.ld, rows, at.row0, nv);
        if (a.g.p) HB::fetch(sg, a.g.p + (i * a.g.ld + c) * sizeof(TB), a.g.ld, rows, at.row0, nv);
        if (a.r.p) HS::fetch(sr, a.r.p + (i * a.r.ld + c) * sizeof(TS), a.r.ld, rows, at.row0, nv);
    };
    // bit 1 of an element's address
    auto odd = [&](const NormMat &m, int64_t c, int f, int bytes) {
        return V == 1 && bytes == 2 && ((reinterpret_cast<uintptr_t>(m.p) >> 1) + (uint32_t)((i0 + f * at.kStep) * m.ld + c)) & 1;
    };
    fetch(tile);
    if (size > 1) cluster_wait();

    for (; tile < tiles; tile += a.groups) {
        const int nv = exist(tile);
        const int64_t c = column(tile);
        typename T::P x[F][T::N];
        cp_async_wait();
        float mean[V], rstd[V];
        if (a.y.p) {
#pragma unroll
            for (int f = 0; f < F; ++f) HB::read(sy, f, odd(a.y, c, f, sizeof(TB)), x[f]);
            typename T::P m[T::N], r[T::N];
            if (a.post.kind > CSRT_NORM_SCALE) {
                tile_stats<TT, V, F>(ex, a.post, at, rows, tile * TT, a.n, x, mean, rstd);
#pragma unroll
                for (int k = 0; k < T::N; ++k) {
                    m[k] = mul2(T::get(mean, k), T::all(-1.f));
                    r[k] = T::get(rstd, k);
                }
            }
#pragma unroll
            for (int f = 0; f < F; ++f) {
                const bool in = at.row0 + f * at.kStep < rows;
                const int64_t i = in ? i0 + f * at.kStep : 0;
                const float w = a.post.w != nullptr ? __ldg(a.post.w + i) : 1.f;
                const float b = a.post.b != nullptr ? __ldg(a.post.b + i) : 0.f;
                if (a.post.kind > CSRT_NORM_SCALE)
#pragma unroll
                    for (int k = 0; k < T::N; ++k) x[f][k] = mul2(add2(x[f][k], m[k]), r[k]);
#pragma unroll
                for (int k = 0; k < T::N; ++k) x[f][k] = fma2(x[f][k], T::all(w), T::all(b));
                if (a.g.p) {
                    typename T::P g[T::N];
                    HB::read(sg, f, odd(a.g, c, f, sizeof(TB)), g);
#pragma unroll
                    for (int k = 0; k < T::N; ++k) {
                        typename T::P v = g[k];
                        if (a.gate_act != CSRT_GATE_NONE) {
                            v = sigmoid2<kFast>(g[k]);
                            if (a.gate_act == CSRT_GATE_SILU) v = mul2(v, g[k]);
                        }
                        x[f][k] = mul2(x[f][k], v);
                    }
                }
                if (a.r.p) {
                    typename T::P r0[T::N];
                    HS::read(sr, f, odd(a.r, c, f, sizeof(TS)), r0);
#pragma unroll
                    for (int k = 0; k < T::N; ++k) x[f][k] = fma2(r0[k], T::all(a.r_scale), x[f][k]);
                }
                if (!in)   // a bias or a mean moved them off zero
#pragma unroll
                    for (int k = 0; k < T::N; ++k) x[f][k] = T::all(0.f);
            }
        } else {
#pragma unroll
            for (int f = 0; f < F; ++f) {
                HS::read(sr, f, odd(a.r, c, f, sizeof(TS)), x[f]);
#pragma unroll
                for (int k = 0; k < T::N; ++k) x[f][k] = mul2(x[f][k], T::all(a.r_scale));
            }
        }
        if (tile + a.groups < tiles) fetch(tile + a.groups);
        typename T::P m[T::N], r[T::N];
        if (a.pre.kind > CSRT_NORM_SCALE) {
            tile_stats<TT, V, F>(ex, a.pre, at, rows, tile * TT, a.n, x, mean, rstd);
#pragma unroll
            for (int k = 0; k < T::N; ++k) {
                m[k] = mul2(T::get(mean, k), T::all(-1.f));
                r[k] = T::get(rstd, k);
            }
        }
        char *ph = a.h.p + (i0 * a.h.ld + c) * sizeof(TS), *pv = a.v.p + (i0 * a.v.ld + c) * sizeof(TB);
#pragma unroll
        for (int f = 0; f < F; ++f) {
            if (at.row0 + f * at.kStep < rows) {
                if (a.h.p) put_tokens<TS, V>(ph + f * at.kStep * a.h.ld * (int64_t)sizeof(TS), x[f], nv);
                if (a.v.p) {
                    const int64_t i = i0 + f * at.kStep;
                    const float w = a.pre.w != nullptr ? __ldg(a.pre.w + i) : 1.f;
                    const float b = a.pre.b != nullptr ? __ldg(a.pre.b + i) : 0.f;
                    typename T::P v[T::N];
#pragma unroll
                    for (int k = 0; k < T::N; ++k) {
                        v[k] = a.pre.kind > CSRT_NORM_SCALE ? mul2(add2(x[f][k], m[k]), r[k]) : x[f][k];
                        v[k] = fma2(v[k], T::all(w), T::all(b));
                    }
                    put_tokens<TB, V>(pv + f * at.kStep * a.v.ld * (int64_t)sizeof(TB), v, nv);
                }
            }
        }
    }
}

template <typename TB, typename TS, int TT, int V, int F>
int norm_fwd_tile(const NormArgs &a, cudaStream_t s) {
    const int size = TileShape<TT, V, F>::cluster(a.d);
    const int smem = (a.y.p ? Held<TB, TT, V, F>::kTotal : 0) + (a.g.p ? Held<TB, TT, V, F>::kTotal : 0) +
                     (a.r.p ? Held<TS, TT, V, F>::kTotal : 0) + Exchange<TT>::bytes(size);
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
