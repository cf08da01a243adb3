// Backward kernel of the norms around a block (block_norm_tile.cuh says how a tile is held).
//
// With xh = (x - mean) rstd and s = weight dout:  dx = rstd (s - xh mean(s xh) - [layer] mean(s)),
// dweight = sum over tokens of dout xh,  dbias = sum over tokens of dout.
#pragma once

#include "block_norm_tile.cuh"

namespace csrt {

// Sums over the tokens of four values of each of a thread's features, carried in registers from tile to tile: a thread's own
// tokens, joined along the row at the end.
template <int TT, int V, int F>
struct TokenSums {
    static constexpr int kLanes = Place<TT, V>::kLanes;
    float v[4][F];
    __device__ __forceinline__ TokenSums() {
#pragma unroll
        for (int k = 0; k < 4; ++k)
#pragma unroll
            for (int f = 0; f < F; ++f) v[k][f] = 0.f;
    }
    __device__ __forceinline__ void add(int k, int f, float x) { v[k][f] += x; }
    // To the group's part of a.partial, or, by the only group, to where they belong; i0: the thread's first feature.
    __device__ __forceinline__ void store(const NormArgs &a, int64_t group, int64_t i0, int row0, int rows) {
        const int lane = threadIdx.x & 31;
        float *const out[4] = {a.post.dw, a.post.db, a.pre.dw, a.pre.db};
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            if (out[k] == nullptr) continue;
            float *p = a.groups == 1 ? out[k] : a.partial + (group * 4 + k) * a.d;
#pragma unroll
            for (int f = 0; f < F; ++f) {
                float s = v[k][f];
#pragma unroll
                for (int o = 1; o < kLanes; o <<= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
                const int64_t i = i0 + f * Place<TT, V>::kStep;
                if (lane % kLanes == 0 && row0 + f * Place<TT, V>::kStep < rows) p[i] = a.groups == 1 && a.accumulate ? p[i] + s : s;
            }
        }
    }
};

template <typename TB, typename TS, int TT, int V, int F, bool TMA, bool UOUT, int BLOCKS>
__global__ void __launch_bounds__(kNormThreads, BLOCKS) norm_bwd_tile_kernel(const __grid_constant__ NormArgs a,
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
    const int lane = threadIdx.x & 31;
    const int size = a.cluster;
    const int rank = size > 1 ? (int)(blockIdx.x % size) : 0;
    const int chunk = a.chunk;
    const int rows = imax(0, imin(chunk, a.d - rank * chunk));
    const int64_t i0 = (int64_t)rank * chunk + (at.row0 < rows ? at.row0 : 0);
    char *p = held;
    auto take = [&](const NormMat &m, int bytes) {
        char *q = p;
        if (m.p) p += bytes;
        return q;
    };
    char *sv = take(a.dv, HB::kTotal), *su = take(a.r, HS::kTotal), *sh = take(a.h, HS::kTotal), *sy = take(a.y, HB::kTotal),
         *sg = take(a.g, HB::kTotal);
    if (!a.y.p) sy = a.dv.p ? sv : su;   // read, and no result depends on it
    float4 *weights = reinterpret_cast<float4 *>(p);   // post weight, post bias, pre weight
    // this warp's: statistics of the tile's tokens (pre mean, negated, and rstd, post likewise), and the stage of results
    float *mine = reinterpret_cast<float *>(weights + kFeatures) + (threadIdx.x >> 5) * 4 * TT;
    char *stage = reinterpret_cast<char *>(weights + kFeatures + kNormWarps * TT) + (threadIdx.x >> 5) * RS::kStageBytes;
    Exchange<TT> ex(reinterpret_cast<char *>(weights + kFeatures + kNormWarps * TT) + kNormWarps * RS::kStageBytes, size, rank,
                    chunk, a.d, a.hdr);
    const int64_t first = (int64_t)rank * chunk + (threadIdx.x >> 5) * at.kRowsWarp;   // the warp's first feature
    const int64_t tiles = ((int64_t)a.n + TT - 1) / TT;
    int64_t tile = blockIdx.x / size;

    auto column = [&](int64_t t) { return t * TT + at.q; };
    auto exist = [&](int64_t t) { return (int)imax<int64_t>(0, imin<int64_t>(V, a.n - column(t))); };
    // TMA: by the first thread, once it has announced the bytes
    auto fetch = [&](auto held_type, const NormMat &m, int k, char *dst, int64_t t) {
        if (!m.p) return;
        if constexpr (TMA) {
            load_tile(dst, maps.m + k, a, rank, t * TT, decltype(held_type)::kRow, ex.bar + (k == 3 ? 3 : 2));
        } else {
            const int nv = exist(t);
            const int64_t c = nv > 0 ? column(t) : 0;
            decltype(held_type)::fetch(dst, m.p + (i0 * m.ld + c) * decltype(held_type)::kSize, m.ld, rows, at.row0, nv);
        }
    };
    const int tokens = TMA ? a.box * a.boxes * TT : 0;
    auto fetch_all = [&](int64_t t) {
        if (TMA) {
            if (threadIdx.x != kLoader) return;
            mbar_expect_tx(ex.bar + 2, tokens * ((a.dv.p ? HB::kSize : 0) + (a.h.p ? HS::kSize : 0) + (a.r.p ? HS::kSize : 0) +
                                                 (a.g.p ? HB::kSize : 0)));
        }
        fetch(HB(), a.dv, 0, sv, t);
        fetch(HS(), a.h, 1, sh, t);
        fetch(HS(), a.r, 2, su, t);
        fetch(HB(), a.g, 4, sg, t);
    };
    auto fetch_y = [&](int64_t t) {
        if (!a.y.p) return;
        if (TMA) {
            if (threadIdx.x != kLoader) return;
            mbar_expect_tx(ex.bar + 3, tokens * HB::kSize);
        }
        fetch(HB(), a.y, 3, sy, t);
    };
    auto offset = [&](auto held_type, const NormMat &m, int64_t c) {
        return decltype(held_type)::offset(m.p + (i0 * m.ld + c) * decltype(held_type)::kSize);
    };
    // a lane's token: pre mean (negated) and rstd, post likewise
    auto statistics = [&](int64_t t) {
        const int64_t c = t * TT + lane;
        float4 s = make_float4(0.f, 1.f, 0.f, 1.f);
        if (lane < TT && c < a.n) {
            if (a.pre.kind == CSRT_NORM_LAYER) s.x = -a.pre.mean[c];
            if (a.pre.kind > CSRT_NORM_SCALE) s.y = a.pre.rstd[c];
            if (a.post.kind == CSRT_NORM_LAYER) s.z = -a.post.mean[c];
            if (a.post.kind > CSRT_NORM_SCALE) s.w = a.post.rstd[c];
        }
        return s;
    };
    fetch_all(tile);
    fetch_y(tile);
    if constexpr (TMA) {
        if (a.dv.p) clear_rows<HB>(sv, chunk);
        if (a.h.p) clear_rows<HS>(sh, chunk);
        if (a.r.p) clear_rows<HS>(su, chunk);
        if (a.y.p) clear_rows<HB>(sy, chunk);
        if (a.g.p) clear_rows<HB>(sg, chunk);
    }
    float4 stat = statistics(tile);
    for (int i = threadIdx.x; i < kFeatures; i += kNormThreads) {
        const int64_t j = (int64_t)rank * chunk + i;
        float4 w = make_float4(0.f, 0.f, 0.f, 0.f);
        if (i < rows) {
            w.x = a.post.w != nullptr ? a.post.w[j] : 1.f;
            w.y = a.post.b != nullptr ? a.post.b[j] : 0.f;
            w.z = a.pre.w != nullptr ? a.pre.w[j] : 1.f;
        }
        weights[i] = w;
    }
    __syncthreads();
    ex.started();
    const bool sums_post = a.post.dw != nullptr || a.post.db != nullptr, sums_pre = a.pre.dw != nullptr || a.pre.db != nullptr;
    TokenSums<TT, V, F> sums;

    for (int turn = 0; tile < tiles; tile += a.groups, ++turn) {
        const int64_t c = column(tile);
        const int off_v = offset(HB(), a.dv, c), off_u = offset(HS(), a.r, c), off_h = offset(HS(), a.h, c),
                  off_y = offset(HB(), a.y, c), off_g = offset(HB(), a.g, c);
        bool ok = true;
        if constexpr (TMA) ok = norm_wait(ex.bar + 2, turn & 1, ex.hdr);
        else cp_async_wait();
        __syncwarp();
        if (lane < TT) {
            mine[lane] = stat.x;
            mine[TT + lane] = stat.y;
            mine[2 * TT + lane] = stat.z;
            mine[3 * TT + lane] = stat.w;
        }
        __syncwarp();
        float va[V], vb[V];
        P al[T::N], on[T::N];
#pragma unroll
        for (int k = 0; k < T::N; ++k) al[k] = on[k] = T::all(0.f);
        P m[T::N], r[T::N];
        auto own_stats = [&](int post) {
            load_tokens<V>(mine + 2 * post * TT + at.q, m);
            load_tokens<V>(mine + (2 * post + 1) * TT + at.q, r);
        };
        // the means of s xh and of s, negated, from this thread's sums
        auto means = [&](const P (&sa)[T::N], const P (&sb)[T::N], bool layer, auto freed) {
#pragma unroll
            for (int k = 0; k < T::N; ++k) {
                T::put(va, k, sa[k]);
                T::put(vb, k, sb[k]);
            }
            auto finish = [&](int, float2 own) { return make_float2(own.x * -ex.inv_d, layer ? own.y * -ex.inv_d : 0.f); };
            if (layer) exchange<kTwoSums>(ex, va, vb, 0.f, at.q, finish, freed, al, on);
            else exchange<kOneSum>(ex, va, vb, 0.f, at.q, finish, freed, al, on);
        };
        own_stats(0);
        if (a.pre.kind > CSRT_NORM_SCALE) {
            P sa[T::N], sb[T::N];
#pragma unroll
            for (int k = 0; k < T::N; ++k) sa[k] = sb[k] = T::all(ok ? 0.f : NAN);
#pragma unroll
            for (int f = 0; f < F; ++f) {
                const float w = weights[at.row0 + f * at.kStep].z;
                P v[T::N], h[T::N];
                HB::read(sv, f, off_v, v);
                HS::read(sh, f, off_h, h);
#pragma unroll
                for (int k = 0; k < T::N; ++k) {
                    const P s = mul2(v[k], T::all(w));
                    sb[k] = add2(sb[k], s);
                    sa[k] = fma2(mul2(add2(h[k], m[k]), r[k]), s, sa[k]);
                }
            }
            means(sa, sb, a.pre.kind == CSRT_NORM_LAYER, [] {});
            own_stats(0);
        }
        P x[F][T::N], sa[T::N], sb[T::N];
        // dh' and with it dr
        if (a.r.p) {
#pragma unroll
            for (int f = 0; f < F; ++f) HS::read(su, f, off_u, x[f]);
        } else {
#pragma unroll
            for (int f = 0; f < F; ++f)
#pragma unroll
                for (int k = 0; k < T::N; ++k) x[f][k] = T::all(0.f);
        }
        if (a.dv.p)
#pragma unroll
            for (int f = 0; f < F; ++f) {
                const float w = weights[at.row0 + f * at.kStep].z;
                P v[T::N], h[T::N];
                HB::read(sv, f, off_v, v);
                HS::read(sh, f, off_h, h);
                P tw = T::all(0.f), tb = tw;
#pragma unroll
                for (int k = 0; k < T::N; ++k) {
                    const P hat = mul2(add2(h[k], m[k]), r[k]);
                    const P q = fma2(hat, al[k], fma2(v[k], T::all(w), on[k]));
                    x[f][k] = fma2(q, r[k], x[f][k]);
                    tw = fma2(v[k], hat, tw);
                    tb = add2(tb, v[k]);
                }
                sums.add(kSumPreW, f, T::sum(tw));
                sums.add(kSumPreB, f, T::sum(tb));
            }
        if (!ok)
#pragma unroll
            for (int f = 0; f < F; ++f)
#pragma unroll
                for (int k = 0; k < T::N; ++k) x[f][k] = T::all(NAN);
        if (a.dr.p) {
            RS out_dr(a.dr, first, tile * TT, a.n);
#pragma unroll
            for (int f = 0; f < F; ++f) {
                P o[T::N];
#pragma unroll
                for (int k = 0; k < T::N; ++k) o[k] = mul2(x[f][k], T::all(a.r_scale));
                out_dr.put(stage, f, at.row0, rows, o);
            }
        }
        const bool more = tile + a.groups < tiles;
        const bool stats = a.dy.p && a.post.kind > CSRT_NORM_SCALE;
        auto next = [&] {   // all inputs but y are in registers
            if (more) {
                fetch_all(tile + a.groups);
                stat = statistics(tile + a.groups);
            }
        };
        if (a.dy.p) {
            if constexpr (TMA)
                if (a.y.p) ok = norm_wait(ex.bar + 3, turn & 1, ex.hdr) && ok;
            own_stats(1);
            if (!ok)
#pragma unroll
                for (int k = 0; k < T::N; ++k) r[k] = T::all(NAN);
#pragma unroll
            for (int k = 0; k < T::N; ++k) sa[k] = sb[k] = T::all(0.f);
            RB out_dg(a.dg, first, tile * TT, a.n);
            const int rows_dg = a.dg.p ? rows : 0;
            // GATE: CSRT_GATE_*, or -1 for no gate
            auto pass = [&](auto gate) {
                constexpr int kGate = decltype(gate)::value;
#pragma unroll
                for (int f = 0; f < F; ++f) {
                    const float4 w = weights[at.row0 + f * at.kStep];
                    P hat[T::N];
                    HB::read(sy, f, off_y, hat);
#pragma unroll
                    for (int k = 0; k < T::N; ++k) hat[k] = mul2(add2(hat[k], m[k]), r[k]);
                    if constexpr (kGate >= 0) {
                        P g[T::N], o[T::N];
                        HB::read(sg, f, off_g, g);
#pragma unroll
                        for (int k = 0; k < T::N; ++k) {
                            P value, slope;
                            gate_of<kGate, kFast>(g[k], T::all(1.f), value, slope);
                            o[k] = mul2(mul2(x[f][k], fma2(hat[k], T::all(w.x), T::all(w.y))), slope);
                            x[f][k] = mul2(x[f][k], value);
                        }
                        out_dg.put(stage, f, at.row0, rows_dg, o);
                    }
                    P tw = T::all(0.f), tb = tw;
#pragma unroll
                    for (int k = 0; k < T::N; ++k) {
                        tw = fma2(x[f][k], hat[k], tw);
                        tb = add2(tb, x[f][k]);
                        x[f][k] = mul2(x[f][k], T::all(w.x));
                        sa[k] = fma2(x[f][k], hat[k], sa[k]);
                        sb[k] = add2(sb[k], x[f][k]);
                    }
                    sums.add(kSumPostW, f, T::sum(tw));
                    sums.add(kSumPostB, f, T::sum(tb));
                }
            };
            if (a.g.p) with_gate(a.gate_act, pass);
            else pass(std::integral_constant<int, -1>());
            if (!TMA || !stats) {
                if (TMA) __syncthreads();   // of all threads
                next();
            }
            if (stats) {
                means(sa, sb, a.post.kind == CSRT_NORM_LAYER, [&] { if (TMA) next(); });
                own_stats(1);
                if (!ok)
#pragma unroll
                    for (int k = 0; k < T::N; ++k) r[k] = T::all(NAN);
            } else {
#pragma unroll
                for (int k = 0; k < T::N; ++k) al[k] = on[k] = T::all(0.f);
            }
            RB out_dy(a.dy, first, tile * TT, a.n);
            if (stats)
#pragma unroll
                for (int f = 0; f < F; ++f) {
                    P y[T::N];
                    HB::read(sy, f, off_y, y);
#pragma unroll
                    for (int k = 0; k < T::N; ++k)
                        x[f][k] = mul2(fma2(mul2(add2(y[k], m[k]), r[k]), al[k], add2(x[f][k], on[k])), r[k]);
                }
#pragma unroll
            for (int f = 0; f < F; ++f) out_dy.put(stage, f, at.row0, rows, x[f]);
            if (TMA) __syncthreads();   // all threads have read y
            if (more) fetch_y(tile + a.groups);
        } else {
            if (TMA) __syncthreads();
            next();
        }
    }
    if (sums_post || sums_pre) sums.store(a, blockIdx.x / size, i0, at.row0, rows);
    ex.leave();
}

template <typename TB, typename TS, int TT, int V, int F, bool TMA, bool UOUT, int BLOCKS>
int norm_bwd_tile(NormArgs &a, cudaStream_t s) {
    typedef typename InputOf<TMA, TB, TT, V, F>::type HB;
    typedef typename InputOf<TMA, TS, TT, V, F>::type HS;
    const int size = TileShape<TT, V, F>::cluster(a.d);
    CSRT_ARG(size > 0, "a cluster cannot hold %d features", a.d);
    const Share share = norm_share(a.d, size, TileShape<TT, V, F>::kFeatures, TMA);
    a.chunk = share.chunk;
    a.box = share.box;
    a.boxes = share.boxes;
    NormMaps maps;
    if (TMA && (!norm_map(maps.m, a.dv, dtype_of<TB>(), a, TT) || !norm_map(maps.m + 1, a.h, dtype_of<TS>(), a, TT) ||
                !norm_map(maps.m + 2, a.r, dtype_of<TS>(), a, TT) || !norm_map(maps.m + 3, a.y, dtype_of<TB>(), a, TT) ||
                !norm_map(maps.m + 4, a.g, dtype_of<TB>(), a, TT)))
        return fail(CSRT_ERR_CUDA, "cuTensorMapEncodeTiled refused a matrix");
    constexpr int b = HB::kTotal, w = HS::kTotal;
    const int smem = (a.dv.p ? b : 0) + (a.r.p ? w : 0) + (a.h.p ? w : 0) + (a.y.p ? b : 0) + (a.g.p ? b : 0) +
                     (TileShape<TT, V, F>::kFeatures + kNormWarps * TT) * (int)sizeof(float4) +
                     kNormWarps * Result<TS, TT, V, UOUT>::kStageBytes + Exchange<TT>::bytes(size);
    return launch_clusters<norm_bwd_tile_kernel<TB, TS, TT, V, F, TMA, UOUT, BLOCKS>>(a, maps, size, ceil_div<int64_t>(a.n, TT),
                                                                                      smem, s);
}

template <typename TB, typename TS, int TT, int F>
int norm_bwd_aligned(NormArgs &a, bool out, cudaStream_t s) {
    return out ? norm_bwd_tile<TB, TS, TT, 8, F, true, false, 2>(a, s) : norm_bwd_tile<TB, TS, TT, 8, F, true, true, 2>(a, s);
}

// in, out: all rows of the inputs, or of the results, are 16-byte aligned.
template <typename TB, typename TS>
int norm_bwd_tiles(NormArgs &a, NormTile t, bool in, bool out, cudaStream_t s) {
    if (t == kTile1x4) return norm_bwd_tile<TB, TS, 1, 1, 4, false, true, 2>(a, s);
    if constexpr (sizeof(TB) == 2) {
        if (in) switch (t) {
                case kTile32x4: return norm_bwd_aligned<TB, TS, 32, 4>(a, out, s);
                case kTile32x2: return norm_bwd_aligned<TB, TS, 32, 2>(a, out, s);
                case kTile16x4: return norm_bwd_aligned<TB, TS, 16, 4>(a, out, s);
                case kTile8x4: return norm_bwd_aligned<TB, TS, 8, 4>(a, out, s);
                case kTile16x2: return norm_bwd_aligned<TB, TS, 16, 2>(a, out, s);
                default: break;
            }
    }
    switch (t) {
        case kTile32x2: return norm_bwd_tile<TB, TS, 32, 8, 2, false, true, 2>(a, s);
        case kTile16x2: return norm_bwd_tile<TB, TS, 16, 8, 2, false, true, 2>(a, s);
        case kTile8x2: return norm_bwd_tile<TB, TS, 8, 8, 2, false, true, 2>(a, s);
        case kTile8x4: return norm_bwd_tile<TB, TS, 8, 8, 4, false, true, 1>(a, s);
        default: return fail(CSRT_ERR_ARG, "unknown tile %d", (int)t);
    }
}

}  // namespace csrt
