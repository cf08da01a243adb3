// Embedding lookup into feature-major activations and the gradient of its table (csrt_embed_fwd, csrt_embed_bwd):
//   x[:, c] = scale table[token c, :],   dtable[v, :] (+)= scale sum_{c: token c = v} dx[:, c]
// The table holds a token in a row, activations hold it in a column: both directions transpose on the way.
#include <cmath>

#include "block_norm.cuh"
#include "mat.cuh"

namespace csrt {

struct EmbedArgs {
    const char *table;         // forward: table; backward: dx
    int64_t ld;
    char *out;                 // forward: x; backward: dtable
    int64_t ldo;
    const int32_t *tokens;
    int32_t vocab, d, n;
    float scale;
    int32_t accumulate;
    int32_t in_vec, out_vec;   // rows of the input, the output allow vectors (as each kernel says)
    WsHeader *hdr;
    // backward
    int32_t *key[2], *idx[2];  // sorted tokens (vocab: none) and their columns; the second pair is scratch
    char *rows;                // dx with a token in a row of `pitch` elements
    int64_t pitch;
    float *partial;            // [chunk][2][pitch]: sums of tokens that go on from the chunk before, into the chunk after
    int32_t chunks;
    int64_t tiles;             // blocks that transpose
    int32_t lanes;             // threads along a row
    int64_t sum_blocks;
};

// ---------------------------------------------------------------------------
// Lookup: a tile of 64 tokens x 64 features passes through shared memory, read along the table's rows and written along
// x's. Blocks that follow one another share their tokens, so that a row's pieces are fetched together; the rows of repeated
// tokens come from L2. in_vec: pairs of features, out_vec: pairs of tokens.
// ---------------------------------------------------------------------------
template <typename T>
struct alignas(2 * sizeof(T)) Pair {
    T a, b;
};
template <typename T>
__device__ __forceinline__ void put_pair(T *p, T a, T b) {
    if constexpr (sizeof(T) == 4) {
        *reinterpret_cast<float2 *>(p) = make_float2(a, b);
    } else {
        const Pair<T> w = {a, b};
        *reinterpret_cast<uint32_t *>(p) = *reinterpret_cast<const uint32_t *>(&w);
    }
}
template <typename TT, typename TX>
__global__ void __launch_bounds__(256) embed_fwd_kernel(EmbedArgs a) {
    pdl_enter();
    __shared__ float tile[64][65];
    __shared__ int32_t tok[64];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int64_t across = ceil_div<int64_t>(a.d, 64);
    const int64_t c0 = blockIdx.x / across * 64, i0 = blockIdx.x % across * 64;
    if (threadIdx.x < 64) {
        const int64_t c = c0 + threadIdx.x;
        int32_t t = c < a.n ? a.tokens[c] : -1;
        if (t >= a.vocab) {
            dev_flag(a.hdr, CSRT_DEV_INVALID);
            t = -1;
        }
        tok[threadIdx.x] = t;
    }
    __syncthreads();
    const TT *table = reinterpret_cast<const TT *>(a.table);
    Pair<TT> v[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) {
        const int32_t t = tok[warp + 8 * k];
        const int64_t i = i0 + 2 * lane;
        const TT *p = table + (int64_t)t * a.ld + i;
        v[k].a = v[k].b = from_f<TT>(0.f);
        if (t >= 0 && i + 1 < a.d && a.in_vec) {
            if constexpr (sizeof(TT) == 4) {
                const float2 w = __ldg(reinterpret_cast<const float2 *>(p));
                v[k] = {w.x, w.y};
            } else {
                const uint32_t w = __ldg(reinterpret_cast<const unsigned int *>(p));
                v[k] = *reinterpret_cast<const Pair<TT> *>(&w);
            }
        } else if (t >= 0) {
            if (i < a.d) v[k].a = p[0];
            if (i + 1 < a.d) v[k].b = p[1];
        }
    }
#pragma unroll
    for (int k = 0; k < 8; ++k) {
        tile[2 * lane][warp + 8 * k] = a.scale * to_f<TT>(v[k].a);
        tile[2 * lane + 1][warp + 8 * k] = a.scale * to_f<TT>(v[k].b);
    }
    __syncthreads();
    TX *x = reinterpret_cast<TX *>(a.out);
    const int64_t c = c0 + 2 * lane;
#pragma unroll
    for (int k = 0; k < 8; ++k) {
        const int64_t i = i0 + warp + 8 * k;
        if (i >= a.d) break;
        const Pair<TX> w = {from_f<TX>(tile[warp + 8 * k][2 * lane]), from_f<TX>(tile[warp + 8 * k][2 * lane + 1])};
        TX *p = x + i * a.ldo + c;
        if (a.out_vec && c + 1 < a.n) {
            put_pair(p, w.a, w.b);
        } else {
            if (c < a.n) p[0] = w.a;
            if (c + 1 < a.n) p[1] = w.b;
        }
    }
}

// ---------------------------------------------------------------------------
// Gradient, first launch: the first block sorts the tokens, the others turn dx into rows, a token each (read from its columns
// the gradient would fetch 32 bytes for every two).
//
// The sort is a stable radix sort, 8 bits a pass. Each warp owns a contiguous run of tokens; counts are kept per digit and
// warp, so that a scan of them in that order gives every warp its places. It is done before the others are from some tens of
// thousands of elements a token on.
// ---------------------------------------------------------------------------
constexpr int kSortWarps = 16;
constexpr int kTurnThreads = kSortWarps * 32;
constexpr int kTurnTokens = 128, kTurnFeatures = 64;   // a tile of the others

__device__ __forceinline__ int embed_passes(int32_t vocab) {   // digits of the values 0 .. vocab
    int p = 1;
    while (p < 4 && ((int64_t)vocab >> (8 * p)) != 0) ++p;
    return p;
}

__device__ void embed_sort(const EmbedArgs &a, int32_t (*count)[kSortWarps]) {
    constexpr int kAhead = 4;   // rounds whose tokens are fetched together
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const unsigned full = 0xffffffffu;
    const int64_t per = ceil_div<int64_t>(ceil_div<int64_t>(a.n, 32), kSortWarps) * 32;
    const int64_t k0 = imin<int64_t>(a.n, per * warp), k1 = imin<int64_t>(a.n, per * (warp + 1));
    __shared__ int32_t warp_total[kSortWarps];
    const int passes = embed_passes(a.vocab);
    // the last pass ends in the first pair of buffers
    for (int p = 0; p < passes; ++p) {
        const int to = (passes - 1 - p) & 1;
        const int32_t *kin = a.key[to ^ 1], *iin = a.idx[to ^ 1];
        int32_t *kout = a.key[to], *iout = a.idx[to];
        auto fetch = [&](int64_t k) -> int32_t {
            if (p > 0) return kin[k];
            const int32_t t = a.tokens[k];
            if (t >= a.vocab) dev_flag(a.hdr, CSRT_DEV_INVALID);
            return t < 0 || t >= a.vocab ? a.vocab : t;
        };
        for (int j = lane; j < 256; j += 32) count[j][warp] = 0;
        __syncwarp();
        for (int64_t k = k0; k < k1; k += 32 * kAhead) {
            int32_t key[kAhead];
#pragma unroll
            for (int u = 0; u < kAhead; ++u) key[u] = k + 32 * u + lane < k1 ? fetch(k + 32 * u + lane) : -1;
#pragma unroll
            for (int u = 0; u < kAhead; ++u) {
                const int digit = key[u] >= 0 ? (key[u] >> (8 * p)) & 255 : 256;
                const unsigned same = __match_any_sync(full, digit);
                if (digit < 256 && (same & ((1u << lane) - 1)) == 0) count[digit][warp] += __popc(same);
                __syncwarp();
            }
        }
        __syncthreads();
        // exclusive scan of the counts in digit-major order, eight a thread
        int32_t own[8], sum = 0;
        int32_t *flat = &count[0][0];
        for (int j = 0; j < 8; ++j) {
            own[j] = sum;
            sum += flat[threadIdx.x * 8 + j];
        }
        int32_t incl = sum;
        for (int o = 1; o < 32; o <<= 1) {
            const int32_t v = __shfl_up_sync(full, incl, o);
            if (lane >= o) incl += v;
        }
        if (lane == 31) warp_total[warp] = incl;
        __syncthreads();
        int32_t base = incl - sum;
        for (int w = 0; w < warp; ++w) base += warp_total[w];
        for (int j = 0; j < 8; ++j) flat[threadIdx.x * 8 + j] = base + own[j];
        __syncthreads();
        for (int64_t k = k0; k < k1; k += 32 * kAhead) {
            int32_t key[kAhead], col[kAhead];
#pragma unroll
            for (int u = 0; u < kAhead; ++u) {
                const int64_t at = k + 32 * u + lane;
                key[u] = at < k1 ? fetch(at) : -1;
                col[u] = p > 0 && at < k1 ? iin[at] : (int32_t)at;
            }
#pragma unroll
            for (int u = 0; u < kAhead; ++u) {
                const int digit = key[u] >= 0 ? (key[u] >> (8 * p)) & 255 : 256;
                const unsigned same = __match_any_sync(full, digit);
                const int before = __popc(same & ((1u << lane) - 1));
                const int32_t at = digit < 256 ? count[digit][warp] : 0;
                __syncwarp();
                if (digit < 256) {
                    kout[at + before] = key[u];
                    iout[at + before] = col[u];
                    if (before == 0) count[digit][warp] = at + __popc(same);
                }
                __syncwarp();
            }
        }
        __syncthreads();
    }
}

// A tile of dx into rows: in_vec says that four tokens make an aligned vector.
template <typename TX>
__device__ __forceinline__ void embed_turn(const EmbedArgs &a, int64_t unit, TX *tile) {
    constexpr int kPitch = kTurnTokens + (sizeof(TX) == 4 ? 1 : 2);
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int64_t along = ceil_div<int64_t>(a.n, kTurnTokens);
    const int64_t c0 = unit % along * kTurnTokens, i0 = unit / along * kTurnFeatures;
    const TX *dx = reinterpret_cast<const TX *>(a.table);
    const bool vec = a.in_vec && c0 + kTurnTokens <= a.n;
    TX v[kTurnFeatures / kSortWarps][4];
#pragma unroll
    for (int k = 0; k < kTurnFeatures / kSortWarps; ++k) {
        const int64_t i = i0 + warp + k * kSortWarps;
        const TX *p = dx + i * a.ld + c0;
        if (i < a.d && vec) {
            if constexpr (sizeof(TX) == 4) {
                *reinterpret_cast<float4 *>(v[k]) = __ldg(reinterpret_cast<const float4 *>(p) + lane);
            } else {
                const uint2 w = __ldg(reinterpret_cast<const uint2 *>(p) + lane);
                const uint32_t u[2] = {w.x, w.y};
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const unsigned short h = (unsigned short)(u[j >> 1] >> (16 * (j & 1)));
                    v[k][j] = *reinterpret_cast<const TX *>(&h);
                }
            }
        } else {
#pragma unroll
            for (int j = 0; j < 4; ++j) v[k][j] = i < a.d && c0 + lane + 32 * j < a.n ? p[lane + 32 * j] : from_f<TX>(0.f);
        }
    }
#pragma unroll
    for (int k = 0; k < kTurnFeatures / kSortWarps; ++k)
#pragma unroll
        for (int j = 0; j < 4; ++j) tile[(warp + k * kSortWarps) * kPitch + (vec ? 4 * lane + j : lane + 32 * j)] = v[k][j];
    __syncthreads();
    TX *out = reinterpret_cast<TX *>(a.rows);
#pragma unroll
    for (int k = 0; k < kTurnTokens / kSortWarps; ++k) {
        const int t = warp + k * kSortWarps;
        const int64_t c = c0 + t, i = i0 + 2 * lane;
        if (c < a.n && i < a.pitch)
            put_pair(out + c * a.pitch + i, tile[2 * lane * kPitch + t], tile[(2 * lane + 1) * kPitch + t]);
    }
}

template <typename TX>
__global__ void __launch_bounds__(kTurnThreads) embed_turn_kernel(EmbedArgs a) {
    pdl_enter();
    constexpr size_t kTile = kTurnFeatures * (kTurnTokens + 2) * sizeof(TX), kCounts = 256 * kSortWarps * sizeof(int32_t);
    __shared__ __align__(16) char space[kTile > kCounts ? kTile : kCounts];
    if (blockIdx.x == 0) embed_sort(a, reinterpret_cast<int32_t(*)[kSortWarps]>(space));
    else embed_turn<TX>(a, (int64_t)blockIdx.x - 1, reinterpret_cast<TX *>(space));
}

// ---------------------------------------------------------------------------
// Second launch: sums over the sorted tokens, kChunk of them by `lanes` threads with eight features each, so that a token
// that comes often is shared among many. A token's run that lies within a chunk is finished there; the parts of one that does
// not are kept, and added in order by the third launch. Other blocks write zeros into the rows that no token is.
// ---------------------------------------------------------------------------
constexpr int kChunk = 64, kSumThreads = 128, kZeroRows = 32;

template <typename T>
__device__ __forceinline__ void load8(const char *p, float (&v)[8]) {
    if constexpr (sizeof(T) == 4) {
        const float4 x = __ldg(reinterpret_cast<const float4 *>(p)), y = __ldg(reinterpret_cast<const float4 *>(p) + 1);
        v[0] = x.x; v[1] = x.y; v[2] = x.z; v[3] = x.w;
        v[4] = y.x; v[5] = y.y; v[6] = y.z; v[7] = y.w;
    } else {
        const uint4 x = __ldg(reinterpret_cast<const uint4 *>(p));
        const uint32_t u[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const unsigned short lo = (unsigned short)u[k], hi = (unsigned short)(u[k] >> 16);
            v[2 * k] = to_f<T>(*reinterpret_cast<const T *>(&lo));
            v[2 * k + 1] = to_f<T>(*reinterpret_cast<const T *>(&hi));
        }
    }
}

// Eight features of a table row from i on: scale * s, or that added to them. out_vec: rows of whole 16-byte words.
template <typename T>
__device__ __forceinline__ void put_row(const EmbedArgs &a, int64_t v, int64_t i, const float (&s)[8]) {
    T *o = reinterpret_cast<T *>(a.out) + v * a.ldo + i;
    if (a.out_vec && i + 8 <= a.d) {
        float w[8];
        if (a.accumulate) {
            load8<T>(reinterpret_cast<const char *>(o), w);
#pragma unroll
            for (int k = 0; k < 8; ++k) w[k] += s[k] * a.scale;
        } else {
#pragma unroll
            for (int k = 0; k < 8; ++k) w[k] = s[k] * a.scale;
        }
        if constexpr (sizeof(T) == 4) {
            reinterpret_cast<float4 *>(o)[0] = make_float4(w[0], w[1], w[2], w[3]);
            reinterpret_cast<float4 *>(o)[1] = make_float4(w[4], w[5], w[6], w[7]);
        } else {
            uint32_t u[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const Pair<T> h = {from_f<T>(w[2 * k]), from_f<T>(w[2 * k + 1])};
                u[k] = *reinterpret_cast<const uint32_t *>(&h);
            }
            *reinterpret_cast<uint4 *>(o) = make_uint4(u[0], u[1], u[2], u[3]);
        }
        return;
    }
#pragma unroll
    for (int k = 0; k < 8; ++k)
        if (i + k < a.d) o[k] = from_f<T>(a.accumulate ? to_f<T>(o[k]) + s[k] * a.scale : s[k] * a.scale);
}

template <typename TX, typename TT>
__device__ __forceinline__ void embed_chunk(const EmbedArgs &a, int64_t chunk, int64_t i) {
    constexpr int kAhead = 4;
    const int32_t *key = a.key[0], *idx = a.idx[0];
    const int64_t k0 = chunk * kChunk, k1 = imin<int64_t>(a.n, k0 + kChunk);
    int32_t v = __ldg(key + k0);
    bool head = k0 > 0 && __ldg(key + k0 - 1) == v;   // the run began before this chunk
    const int32_t after = k1 < a.n ? __ldg(key + k1) : -1;
    float s[8] = {0.f};
    auto keep = [&](int slot) {
        float *o = a.partial + (chunk * 2 + slot) * a.pitch + i;
        reinterpret_cast<float4 *>(o)[0] = make_float4(s[0], s[1], s[2], s[3]);
        reinterpret_cast<float4 *>(o)[1] = make_float4(s[4], s[5], s[6], s[7]);
    };
    for (int64_t k = k0; k < k1; k += kAhead) {
        int32_t token[kAhead];
        float x[kAhead][8];
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            token[u] = k + u < k1 ? __ldg(key + k + u) : a.vocab;
            if (token[u] < a.vocab) load8<TX>(a.rows + ((int64_t)__ldg(idx + k + u) * a.pitch + i) * sizeof(TX), x[u]);
        }
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            if (token[u] != v) {   // the run of v is over (none of padding, which sorts last)
                if (head) keep(0);
                else if (v < a.vocab) put_row<TT>(a, v, i, s);
                head = false;
                v = token[u];
#pragma unroll
                for (int j = 0; j < 8; ++j) s[j] = 0.f;
            }
            if (v < a.vocab)
#pragma unroll
                for (int j = 0; j < 8; ++j) s[j] += x[u][j];
        }
    }
    if (v >= a.vocab) return;
    if (head) keep(0);   // all of the chunk, or its end as well as its beginning
    else if (after == v) keep(1);
    else put_row<TT>(a, v, i, s);
}

template <typename TX, typename TT>
__global__ void __launch_bounds__(kSumThreads) embed_sum_kernel(EmbedArgs a) {
    pdl_enter();
    if (blockIdx.x < a.sum_blocks) {
        const int64_t across = ceil_div<int64_t>(a.pitch, (int64_t)a.lanes * 8);
        const int64_t i = ((int64_t)blockIdx.x % across * a.lanes + threadIdx.x % a.lanes) * 8;
        const int64_t chunk = (int64_t)blockIdx.x / across * (kSumThreads / a.lanes) + threadIdx.x / a.lanes;
        if (i < a.pitch && chunk < a.chunks) embed_chunk<TX, TT>(a, chunk, i);
        return;
    }
    __shared__ int32_t used[kZeroRows];
    const int64_t v0 = ((int64_t)blockIdx.x - a.sum_blocks) * kZeroRows;
    const int rows = (int)imin<int64_t>(kZeroRows, a.vocab - v0);
    if (threadIdx.x < kZeroRows) {
        used[threadIdx.x] = 0;
        __syncwarp();
        const int32_t *key = a.key[0];
        int64_t from, to;
        warp_first_false2(0, a.n, [&](int64_t k) { return __ldg(key + k) < v0; }, 0, a.n,
                          [&](int64_t k) { return __ldg(key + k) < v0 + rows; }, from, to);
        for (int64_t k = from + threadIdx.x; k < to; k += 32) used[__ldg(key + k) - v0] = 1;
    }
    __syncthreads();
    const float zero[8] = {0.f};
    for (int r = 0; r < rows; ++r)
        if (!used[r])
            for (int64_t i = threadIdx.x * 8; i < a.d; i += kSumThreads * 8) put_row<TT>(a, v0 + r, i, zero);
}

// Third launch: the runs that begin in a chunk and go on after it.
template <typename TT>
__global__ void __launch_bounds__(kSumThreads) embed_join_kernel(EmbedArgs a) {
    pdl_enter();
    const int64_t across = ceil_div<int64_t>(a.pitch, (int64_t)a.lanes * 8);
    const int64_t i = ((int64_t)blockIdx.x % across * a.lanes + threadIdx.x % a.lanes) * 8;
    const int64_t chunk = (int64_t)blockIdx.x / across * (kSumThreads / a.lanes) + threadIdx.x / a.lanes;
    if (i >= a.pitch || chunk + 1 >= a.chunks) return;
    const int32_t *key = a.key[0];
    const int64_t k0 = chunk * kChunk, next = k0 + kChunk;
    const int32_t v = __ldg(key + next - 1);
    if (v >= a.vocab || __ldg(key + next) != v || (__ldg(key + k0) == v && k0 > 0 && __ldg(key + k0 - 1) == v)) return;
    float s[8], x[8];
    load8<float>(reinterpret_cast<const char *>(a.partial + (chunk * 2 + 1) * a.pitch + i), s);
#pragma unroll 4
    for (int64_t c = chunk + 1; c < a.chunks && __ldg(key + c * kChunk) == v; ++c) {
        load8<float>(reinterpret_cast<const char *>(a.partial + c * 2 * a.pitch + i), x);
#pragma unroll
        for (int k = 0; k < 8; ++k) s[k] += x[k];
    }
    put_row<TT>(a, v, i, s);
}

// ---------------------------------------------------------------------------
// Host
// ---------------------------------------------------------------------------
static size_t embed_list_bytes(int64_t n) { return align_up((size_t)n * sizeof(int32_t), 256); }
static int64_t embed_pitch(int64_t d) { return ceil_div<int64_t>(d, 8) * 8; }
// the sorted tokens, dx in rows (float32 at most), the parts of runs
static size_t embed_bytes(int64_t d, int64_t n) {
    const size_t row = (size_t)embed_pitch(d) * sizeof(float);
    return kWsReservedBytes + 4 * embed_list_bytes(n) + align_up((size_t)n * row, 256) + align_up(ceil_div<int64_t>(n, kChunk) * 2 * row, 256);
}

static int check_embed(const int32_t *tokens, float scale, int32_t vocab, int32_t d, int32_t n, const csrt_mat *out,
                       const char *out_name, void *ws, size_t ws_bytes) {
    CSRT_ARG(n == 0 || tokens != nullptr, "tokens is NULL");
    CSRT_TRY(check_vector(reinterpret_cast<const float *>(tokens), "tokens"));
    CSRT_ARG(!vector_meets(reinterpret_cast<const float *>(tokens), n, out), "tokens overlap %s", out_name);
    CSRT_ARG(std::isfinite(scale), "scale must be finite");
    CSRT_ARG(vocab < INT32_MAX, "the table has too many rows");
    CSRT_ARG(ws != nullptr, "workspace is NULL");
    CSRT_ARG((reinterpret_cast<uintptr_t>(ws) & 255) == 0, "workspace is not 256-byte aligned");
    if (ws_bytes < embed_bytes(d, n))
        return fail(CSRT_ERR_WORKSPACE, "workspace has %zu bytes, needs %zu", ws_bytes, embed_bytes(d, n));
    return CSRT_OK;
}

// Rows whose elements 0, k, 2k .. begin on a multiple of k elements.
static bool rows_of(const csrt_mat *m, int k) {
    return reinterpret_cast<uintptr_t>(m->data) % (k * dt_size(m->dtype)) == 0 && (m->ld % k == 0 || m->rows <= 1);
}

static EmbedArgs embed_args(const csrt_mat *in, const csrt_mat *out, const int32_t *tokens, int32_t vocab, int32_t d,
                            int32_t n, float scale, void *ws) {
    EmbedArgs a = {};
    a.table = static_cast<const char *>(in->data);
    a.ld = in->ld;
    a.out = static_cast<char *>(out->data);
    a.ldo = out->ld;
    a.tokens = tokens;
    a.vocab = vocab;
    a.d = d;
    a.n = n;
    a.scale = scale;
    a.hdr = static_cast<WsHeader *>(ws);
    char *at = ws_scratch(ws);
    for (int k = 0; k < 2; ++k) {
        a.key[k] = reinterpret_cast<int32_t *>(at);
        a.idx[k] = reinterpret_cast<int32_t *>(at + embed_list_bytes(n));
        at += 2 * embed_list_bytes(n);
    }
    a.pitch = embed_pitch(d);
    a.rows = at;
    a.partial = reinterpret_cast<float *>(at + align_up((size_t)n * a.pitch * sizeof(float), 256));
    a.chunks = (int32_t)ceil_div<int64_t>(n, kChunk);
    return a;
}

template <typename TT, typename TX>
static int launch_embed_fwd(const EmbedArgs &a, cudaStream_t s) {
    const int64_t blocks = ceil_div<int64_t>(a.n, 64) * ceil_div<int64_t>(a.d, 64);
    CSRT_ARG(blocks <= INT32_MAX, "x is too large");
    launch_pdl(embed_fwd_kernel<TT, TX>, dim3((unsigned)blocks), dim3(256), 0, s, a);
    count_launch();
    return check_launch("embed_fwd_kernel");
}

template <typename TX, typename TT>
static int launch_embed_bwd(EmbedArgs a, cudaStream_t s) {
    a.tiles = ceil_div<int64_t>(a.n, kTurnTokens) * ceil_div<int64_t>(a.d, kTurnFeatures);
    for (a.lanes = 1; a.lanes < kSumThreads && a.lanes * 8 < a.pitch;) a.lanes *= 2;
    const int64_t across = ceil_div<int64_t>(a.pitch, (int64_t)a.lanes * 8);
    a.sum_blocks = across * ceil_div<int64_t>(a.chunks, kSumThreads / a.lanes);
    const int64_t zero_blocks = a.accumulate ? 0 : ceil_div<int64_t>(a.vocab, kZeroRows);
    CSRT_ARG(a.tiles < INT32_MAX && a.sum_blocks + zero_blocks < INT32_MAX, "dx is too large");
    launch_pdl(embed_turn_kernel<TX>, dim3((unsigned)(1 + a.tiles)), dim3(kTurnThreads), 0, s, a);
    count_launch();
    CSRT_TRY(check_launch("embed_turn_kernel"));
    if (a.sum_blocks + zero_blocks > 0) {
        launch_pdl(embed_sum_kernel<TX, TT>, dim3((unsigned)(a.sum_blocks + zero_blocks)), dim3(kSumThreads), 0, s, a);
        count_launch();
        CSRT_TRY(check_launch("embed_sum_kernel"));
    }
    if (a.chunks < 2) return CSRT_OK;
    launch_pdl(embed_join_kernel<TT>, dim3((unsigned)a.sum_blocks), dim3(kSumThreads), 0, s, a);
    count_launch();
    return check_launch("embed_join_kernel");
}

#define CSRT_EMBED_DISPATCH(fn, from, to, ...)                                                                          \
    (from == CSRT_DT_F32                                                                                                \
         ? (to == CSRT_DT_F32 ? fn<float, float>(__VA_ARGS__)                                                           \
            : to == CSRT_DT_BF16 ? fn<float, __nv_bfloat16>(__VA_ARGS__) : fn<float, __half>(__VA_ARGS__))              \
     : from == CSRT_DT_BF16                                                                                             \
         ? (to == CSRT_DT_F32 ? fn<__nv_bfloat16, float>(__VA_ARGS__)                                                   \
            : to == CSRT_DT_BF16 ? fn<__nv_bfloat16, __nv_bfloat16>(__VA_ARGS__) : fn<__nv_bfloat16, __half>(__VA_ARGS__)) \
         : (to == CSRT_DT_F32 ? fn<__half, float>(__VA_ARGS__)                                                          \
            : to == CSRT_DT_BF16 ? fn<__half, __nv_bfloat16>(__VA_ARGS__) : fn<__half, __half>(__VA_ARGS__)))

}  // namespace csrt

using namespace csrt;

extern "C" {

int csrt_embed_workspace_bytes(int32_t vocab, int32_t d, int32_t max_n, size_t *bytes) {
    CSRT_ARG(bytes != nullptr, "bytes is NULL");
    CSRT_ARG(vocab >= 0 && d >= 0 && max_n >= 0, "negative size");
    *bytes = embed_bytes(d, max_n);
    return CSRT_OK;
}

int csrt_embed_fwd(const csrt_mat *table, const int32_t *tokens, float scale, csrt_mat *x, void *ws, size_t ws_bytes,
                   void *stream) {
    CSRT_TRY(check_mat(table, "table"));
    CSRT_TRY(check_mat(x, "x"));
    const int32_t vocab = table->rows, d = table->cols, n = x->cols;
    CSRT_TRY(check_shape(x, "x", d, n));
    CSRT_ARG(!clash(x, table), "x overlaps table");
    CSRT_TRY(check_embed(tokens, scale, vocab, d, n, x, "x", ws, ws_bytes));
    if (d == 0 || n == 0) return CSRT_OK;
    EmbedArgs a = embed_args(table, x, tokens, vocab, d, n, scale, ws);
    a.in_vec = rows_of(table, 2);
    a.out_vec = rows_of(x, 2);
    return CSRT_EMBED_DISPATCH(launch_embed_fwd, table->dtype, x->dtype, a, as_stream(stream));
}

int csrt_embed_bwd(const csrt_mat *dx, const int32_t *tokens, float scale, int32_t accumulate, csrt_mat *dtable,
                   void *ws, size_t ws_bytes, void *stream) {
    CSRT_TRY(check_mat(dx, "dx"));
    CSRT_TRY(check_mat(dtable, "dtable"));
    const int32_t vocab = dtable->rows, d = dx->rows, n = dx->cols;
    CSRT_TRY(check_shape(dtable, "dtable", vocab, d));
    CSRT_ARG(!clash(dtable, dx), "dtable overlaps dx");
    CSRT_TRY(check_embed(tokens, scale, vocab, d, n, dtable, "dtable", ws, ws_bytes));
    if (d == 0 || vocab == 0) return CSRT_OK;
    EmbedArgs a = embed_args(dx, dtable, tokens, vocab, d, n, scale, ws);
    a.accumulate = accumulate != 0;
    a.in_vec = rows_of(dx, 4);
    a.out_vec = tma_rows_ok(dtable->data, dtable->ld, dt_size(dtable->dtype));
    return CSRT_EMBED_DISPATCH(launch_embed_bwd, dx->dtype, dtable->dtype, a, as_stream(stream));
}

}  // extern "C"
