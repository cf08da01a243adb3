// Forward kernel of the norms around a block (block_norm_tile.cuh says how a tile is held).
#pragma once

#include "block_norm_tile.cuh"

namespace csrt {

// Mean (negated) and reciprocal deviation of this thread's V tokens, over all features; `rows` of the block's features
// exist, x is zero beyond them. Written out by the cluster's first block. zero: 0, or NaN where a wait for x ran out.
template <int TT, int V, int F, typename FREED>
__device__ __forceinline__ void tile_stats(Exchange<TT> &ex, const NormSide &s, const Place<TT, V> &at, int rows, int64_t c0,
                                           int32_t n, float zero, FREED freed, const typename Tok<V>::P (&x)[F][Tok<V>::N],
                                           typename Tok<V>::P (&m)[Tok<V>::N], typename Tok<V>::P (&r)[Tok<V>::N]) {
    typedef Tok<V> T;
    float a[V], b[V];
    auto finish = [&](int t, float2 own) {
        own.y = rsqrt_near(fmaf(own.y, ex.inv_d, s.eps));
        const int64_t c = c0 + t;
        if (ex.rank == 0 && c < n) {   // the lanes that hold copies write the same
            if (s.mean != nullptr && s.kind == CSRT_NORM_LAYER) s.mean[c] = own.x;
            if (s.rstd != nullptr) s.rstd[c] = own.y;
        }
        own.x = -own.x;
        return own;
    };
    typename T::P sq[T::N];
#pragma unroll
    for (int k = 0; k < T::N; ++k) sq[k] = T::all(zero);
    if (s.kind == CSRT_NORM_LAYER) {
        float cnt = 0.f;
        typename T::P sum[T::N];
#pragma unroll
        for (int k = 0; k < T::N; ++k) sum[k] = T::all(zero);
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
        exchange<kMoments>(ex, a, b, cnt, at.q, finish, freed, m, r);
    } else {
#pragma unroll
        for (int f = 0; f < F; ++f)
#pragma unroll
            for (int k = 0; k < T::N; ++k) sq[k] = fma2(x[f][k], x[f][k], sq[k]);
#pragma unroll
        for (int k = 0; k < T::N; ++k) T::put(a, k, sq[k]);
        exchange<kOneSum>(ex, a, b, 0.f, at.q, [&](int t, float2 own) { return finish(t, make_float2(0.f, own.x)); }, freed, m, r);
    }
}

template <typename TB, typename TS, int TT, int V, int F, bool TMA, bool UOUT, int BLOCKS>
__global__ void __launch_bounds__(kNormThreads, BLOCKS) norm_fwd_tile_kernel(const __grid_constant__ NormArgs a,
                                                                             const __grid_constant__ NormMaps maps) {
    pdl_enter();
    extern __shared__ __align__(128) char held[];
    typedef Tok<V> T;
    typedef typename InputOf<TMA, TB, TT, V, F>::type HB;
    typedef typename InputOf<TMA, TS, TT, V, F>::type HS;
    typedef Result<TB, TT, V, UOUT> RB;
    typedef Result<TS, TT, V, UOUT> RS;
    typedef typename T::P P;
    constexpr bool kFast = sizeof(TB) == 2;
    constexpr int kFeatures = Place<TT, V>::kStep * F;
    const Place<TT, V> at;
    const int size = a.cluster;
    const int rank = size > 1 ? (int)(blockIdx.x % size) : 0;
    const int chunk = a.chunk;
    const int rows = imax(0, imin(chunk, a.d - rank * chunk));
    const int64_t i0 = (int64_t)rank * chunk + (at.row0 < rows ? at.row0 : 0);
    char *sy = held, *sg = sy + (a.y.p ? HB::kTotal : 0), *sr = sg + (a.g.p ? HB::kTotal : 0);
    float2 *wpost = reinterpret_cast<float2 *>(sr + (a.r.p ? HS::kTotal : 0)), *wpre = wpost + kFeatures;   // weight, bias
    char *stage = reinterpret_cast<char *>(wpre + kFeatures) + (threadIdx.x >> 5) * RS::kStageBytes;   // this warp's
    Exchange<TT> ex(reinterpret_cast<char *>(wpre + kFeatures) + kNormWarps * RS::kStageBytes, size, rank, chunk, a.d, a.hdr);
    const int64_t first = (int64_t)rank * chunk + (threadIdx.x >> 5) * at.kRowsWarp;   // the warp's first feature
    const int tiles = (int)(((int64_t)a.n + TT - 1) / TT);   // n <= 2 where TT is 1
    int tile = (int)(blockIdx.x / size);

    auto column = [&](int t) { return (int64_t)t * TT + at.q; };
    auto exist = [&](int t) { return (int)imax<int64_t>(0, imin<int64_t>(V, a.n - column(t))); };
    auto fetch = [&](int t) {
        if constexpr (TMA) {
            if (threadIdx.x != kLoader) return;
            uint64_t *bar = ex.bar + 2;
            const int tokens = a.box * a.boxes * TT;
            mbar_expect_tx(bar, tokens * ((a.y.p ? HB::kSize : 0) + (a.g.p ? HB::kSize : 0) + (a.r.p ? HS::kSize : 0)));
            if (a.y.p) load_tile(sy, maps.m, a, rank, (int64_t)t * TT, HB::kRow, bar);
            if (a.g.p) load_tile(sg, maps.m + 1, a, rank, (int64_t)t * TT, HB::kRow, bar);
            if (a.r.p) load_tile(sr, maps.m + 2, a, rank, (int64_t)t * TT, HS::kRow, bar);
        } else {
            const int nv = exist(t);
            const int64_t c = nv > 0 ? column(t) : 0;
            if (a.y.p) HB::fetch(sy, a.y.p + (i0 * a.y.ld + c) * sizeof(TB), a.y.ld, rows, at.row0, nv);
            if (a.g.p) HB::fetch(sg, a.g.p + (i0 * a.g.ld + c) * sizeof(TB), a.g.ld, rows, at.row0, nv);
            if (a.r.p) HS::fetch(sr, a.r.p + (i0 * a.r.ld + c) * sizeof(TS), a.r.ld, rows, at.row0, nv);
        }
    };
    auto offset = [&](auto held_type, const NormMat &m, int64_t c) {
        return decltype(held_type)::offset(m.p + (i0 * m.ld + c) * decltype(held_type)::kSize);
    };
    fetch(tile);
    if constexpr (TMA) {
        if (a.y.p) clear_rows<HB>(sy, chunk);
        if (a.g.p) clear_rows<HB>(sg, chunk);
        if (a.r.p) clear_rows<HS>(sr, chunk);
    }
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

    for (int turn = 0; tile < tiles; tile += a.groups, ++turn) {
        const int64_t c = column(tile);
        P x[F][T::N], m[T::N], r[T::N];
        RS out_h(a.h, first, (int64_t)tile * TT, a.n);
        float one = 1.f;   // NaN where the wait ran out: all that follows from the inputs is
        if constexpr (TMA) one = norm_wait(ex.bar + 2, turn & 1, ex.hdr) ? 1.f : NAN;
        else cp_async_wait();
        const int off_r = offset(HS(), a.r, c);
        if (a.y.p) {
            const int off_y = offset(HB(), a.y, c), off_g = offset(HB(), a.g, c);
#pragma unroll
            for (int f = 0; f < F; ++f) HB::read(sy, f, off_y, x[f]);
#pragma unroll
            for (int k = 0; k < T::N; ++k) {
                m[k] = T::all(0.f);
                r[k] = T::all(one);
            }
            if (a.post.kind > CSRT_NORM_SCALE) tile_stats<TT, V, F>(ex, a.post, at, rows, (int64_t)tile * TT, a.n, one - 1.f, [] {}, x, m, r);
            // GATE: CSRT_GATE_*, or -1 for no gate. Stores are spread over the features: in a loop of their own they held up
            // the loads behind them (float32 stream 127 -> 150 us).
            auto pass = [&](auto gate) {
                constexpr int kGate = decltype(gate)::value;
#pragma unroll
                for (int f = 0; f < F; ++f) {
                    const float2 w = wpost[at.row0 + f * at.kStep];
#pragma unroll
                    for (int k = 0; k < T::N; ++k)
                        x[f][k] = fma2(add2(x[f][k], m[k]), mul2(r[k], T::all(w.x)), T::all(w.y));
                    if constexpr (kGate >= 0) {
                        P g[T::N];
                        HB::read(sg, f, off_g, g);
#pragma unroll
                        for (int k = 0; k < T::N; ++k) {
                            P value, slope;
                            gate_of<kGate, kFast>(g[k], T::all(1.f), value, slope);
                            x[f][k] = mul2(x[f][k], value);
                        }
                    }
                    if (a.r.p) {
                        P r0[T::N];
                        HS::read(sr, f, off_r, r0);
#pragma unroll
                        for (int k = 0; k < T::N; ++k) x[f][k] = fma2(r0[k], T::all(a.r_scale), x[f][k]);
                    }
                    if (a.h.p) out_h.put(stage, f, at.row0, rows, x[f]);
                }
            };
            if (a.g.p) with_gate(a.gate_act, pass);
            else pass(std::integral_constant<int, -1>());
        } else {
#pragma unroll
            for (int f = 0; f < F; ++f) {
                HS::read(sr, f, off_r, x[f]);
#pragma unroll
                for (int k = 0; k < T::N; ++k) x[f][k] = mul2(x[f][k], T::all(a.r_scale * one));
                if (a.h.p) out_h.put(stage, f, at.row0, rows, x[f]);
            }
        }
        auto next = [&] {   // the inputs are in registers
            if (tile + a.groups < tiles) fetch(tile + a.groups);
        };
        const bool stats = a.pre.kind > CSRT_NORM_SCALE;
        if (!TMA || !stats) {
            if (TMA) __syncthreads();   // of all threads
            next();
        }
        if (!a.v.p) continue;
#pragma unroll
        for (int k = 0; k < T::N; ++k) {
            m[k] = T::all(0.f);
            r[k] = T::all(1.f);
        }
        if (stats)
            tile_stats<TT, V, F>(ex, a.pre, at, rows, (int64_t)tile * TT, a.n, 0.f, [&] { if (TMA) next(); }, x, m, r);
        RB out_v(a.v, first, (int64_t)tile * TT, a.n);
#pragma unroll
        for (int f = 0; f < F; ++f) {
            const float2 w = wpre[at.row0 + f * at.kStep];
            P v[T::N];
#pragma unroll
            for (int k = 0; k < T::N; ++k) v[k] = fma2(add2(x[f][k], m[k]), mul2(r[k], T::all(w.x)), T::all(w.y));
            out_v.put(stage, f, at.row0, rows, v);
        }
    }
    ex.leave();
}

template <typename TB, typename TS, int TT, int V, int F, bool TMA, bool UOUT, int BLOCKS = 2>
int norm_fwd_tile(NormArgs a, cudaStream_t s) {
    typedef typename InputOf<TMA, TB, TT, V, F>::type HB;
    typedef typename InputOf<TMA, TS, TT, V, F>::type HS;
    const int size = TileShape<TT, V, F>::cluster(a.d);
    CSRT_ARG(size > 0, "a cluster cannot hold %d features", a.d);
    const Share share = norm_share(a.d, size, TileShape<TT, V, F>::kFeatures, TMA);
    a.chunk = share.chunk;
    a.box = share.box;
    a.boxes = share.boxes;
    NormMaps maps;
    if (TMA && (!norm_map(maps.m, a.y, dtype_of<TB>(), a, TT) || !norm_map(maps.m + 1, a.g, dtype_of<TB>(), a, TT) ||
                !norm_map(maps.m + 2, a.r, dtype_of<TS>(), a, TT)))
        return fail(CSRT_ERR_CUDA, "cuTensorMapEncodeTiled refused a matrix");
    const int smem = (a.y.p ? HB::kTotal : 0) + (a.g.p ? HB::kTotal : 0) + (a.r.p ? HS::kTotal : 0) +
                     TileShape<TT, V, F>::kFeatures * 16 + kNormWarps * Result<TS, TT, V, UOUT>::kStageBytes + Exchange<TT>::bytes(size);
    return launch_clusters<norm_fwd_tile_kernel<TB, TS, TT, V, F, TMA, UOUT, BLOCKS>>(a, maps, size, ceil_div<int64_t>(a.n, TT), smem, s);
}

template <typename TB, typename TS, int TT, int F, int BLOCKS = 2>
int norm_fwd_aligned(const NormArgs &a, bool out, cudaStream_t s) {
    return out ? norm_fwd_tile<TB, TS, TT, 8, F, true, false, BLOCKS>(a, s) : norm_fwd_tile<TB, TS, TT, 8, F, true, true, BLOCKS>(a, s);
}

// in, out: all rows of the inputs, or of the results, are 16-byte aligned.
template <typename TB, typename TS>
int norm_fwd_tiles(const NormArgs &a, NormTile t, bool in, bool out, cudaStream_t s) {
    switch (t) {
        case kTile1x4: return norm_fwd_tile<TB, TS, 1, 1, 4, false, true>(a, s);
        case kTile1x16: return norm_fwd_tile<TB, TS, 1, 1, 16, false, true>(a, s);
        default: break;
    }
    if constexpr (sizeof(TB) == 2) {
        if (in) switch (t) {
                case kTile32x8: return norm_fwd_aligned<TB, TS, 32, 8>(a, out, s);
                case kTile32x4: return norm_fwd_aligned<TB, TS, 32, 4>(a, out, s);
                case kTile32x2: return norm_fwd_aligned<TB, TS, 32, 2>(a, out, s);
                case kTile16x5: return norm_fwd_aligned<TB, TS, 16, 5>(a, out, s);
                case kTile16x4: return norm_fwd_aligned<TB, TS, 16, 4, 3>(a, out, s);
                default: break;
            }
    }
    switch (t) {
        case kTile32x4: return norm_fwd_tile<TB, TS, 32, 8, 4, false, true>(a, s);
        case kTile32x2: return norm_fwd_tile<TB, TS, 32, 8, 2, false, true>(a, s);
        case kTile16x4: return norm_fwd_tile<TB, TS, 16, 8, 4, false, true>(a, s);
        case kTile8x4: return norm_fwd_tile<TB, TS, 8, 8, 4, false, true>(a, s);
        default: return fail(CSRT_ERR_ARG, "unknown tile %d", (int)t);
    }
}

}  // namespace csrt
