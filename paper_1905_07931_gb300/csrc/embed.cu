// Embedding lookup into feature-major activations and the gradient of its table (csrt_embed_fwd, csrt_embed_bwd):
//   x[:, c] = scale table[token c, :],   dtable[v, :] (+)= scale sum_{c: token c = v} dx[:, c]
// The table holds a token in a row, activations hold it in a column: both directions transpose on the way.
#include <cmath>
#include <type_traits>

#include "block_norm.cuh"
#include "gemm16_host.cuh"
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
    int32_t steps;             // lookup: tiles of a block
    int32_t in_vec, out_vec;   // rows of the input, the output allow vectors
    WsHeader *hdr;
    // backward
    int32_t *key[2], *idx[2];  // sorted tokens (vocab: none) and their columns; the second pair is scratch
    char *rows;                // dx with a token in a row of `pitch` elements
    int64_t pitch;
    float *partial;            // [chunk][2][pitch]: sums of tokens that go on from the chunk before, into the chunk after
    int32_t chunk, chunks;     // tokens of a chunk
    int32_t sort_blocks;       // of the first launch, in front of those that turn
    int32_t lanes;             // threads along a row; few tokens: elements between two features in shared memory
    int64_t sum_blocks;
};

// ---------------------------------------------------------------------------
// Lookup: a tile of 64 tokens x 64 features passes through shared memory. A thread reads one feature of eight tokens along
// the table's rows and leaves them as one vector in the feature's row; x is written in vectors of eight tokens where its rows
// allow it (out_vec), else by single elements, 32 tokens a store. Blocks that follow one another share their tokens, so that
// a row's pieces are fetched together; the rows of repeated tokens come from L2.
// ---------------------------------------------------------------------------
constexpr int kTile = 64, kSteps = 4;

// Two 16-bit values in a word.
template <typename T>
__device__ __forceinline__ uint32_t two_of(float lo, float hi) {
    if constexpr (std::is_same<T, __nv_bfloat16>::value) {
        const __nv_bfloat162 h = __floats2bfloat162_rn(lo, hi);
        return *reinterpret_cast<const uint32_t *>(&h);
    } else {
        const __half2 h = __floats2half2_rn(lo, hi);
        return *reinterpret_cast<const uint32_t *>(&h);
    }
}

// A block takes a.steps tiles of the same tokens: the next one's rows are on their way while one is stored.
template <typename TT, typename TX>
__global__ void __launch_bounds__(256) embed_fwd_kernel(EmbedArgs a) {
    pdl_enter();
    constexpr int kWords = sizeof(TX) / 2;                 // 16-byte words of eight elements
    constexpr int kPitch = kTile * sizeof(TX) + 16;        // bytes: rows of odd 16-byte words, without bank conflicts
    __shared__ __align__(16) char tiles[2][kTile * kPitch];
    __shared__ int32_t tok[kTile];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int64_t across = ceil_div<int64_t>(a.d, kTile * a.steps);
    const int64_t c0 = blockIdx.x / across * kTile;
    int64_t i0 = blockIdx.x % across * kTile * a.steps;
    if (threadIdx.x < kTile) {
        const int64_t c = c0 + threadIdx.x;
        int32_t t = c < a.n ? a.tokens[c] : -1;
        if (t >= a.vocab) {
            dev_flag(a.hdr, CSRT_DEV_INVALID);
            t = -1;
        }
        tok[threadIdx.x] = t;
    }
    __syncthreads();
    TT v[2][8];
    auto fetch = [&](int64_t at) {
        const TT *table = reinterpret_cast<const TT *>(a.table) + at + lane;
        const bool in[2] = {at + lane < a.d, at + lane + 32 < a.d};
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const int32_t t = tok[warp * 8 + k];
            const TT *p = table + (int64_t)t * a.ld;
#pragma unroll
            for (int u = 0; u < 2; ++u) v[u][k] = t >= 0 && in[u] ? __ldg(p + 32 * u) : from_f<TT>(0.f);
        }
    };
    fetch(i0);
    TX *x = reinterpret_cast<TX *>(a.out);
    const bool whole = a.out_vec && c0 + kTile <= a.n;
    for (int s = 0; s < a.steps && i0 < a.d; ++s, i0 += kTile) {
        char *tile = tiles[s & 1];
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            uint32_t w[4 * kWords];
#pragma unroll
            for (int k = 0; k < 8; k += 2) {
                const float lo = a.scale * to_f<TT>(v[u][k]), hi = a.scale * to_f<TT>(v[u][k + 1]);
                if constexpr (sizeof(TX) == 4) {
                    w[k] = __float_as_uint(lo);
                    w[k + 1] = __float_as_uint(hi);
                } else {
                    w[k / 2] = two_of<TX>(lo, hi);
                }
            }
            uint4 *row = reinterpret_cast<uint4 *>(tile + (lane + 32 * u) * kPitch + warp * 8 * sizeof(TX));
#pragma unroll
            for (int k = 0; k < kWords; ++k) row[k] = make_uint4(w[4 * k], w[4 * k + 1], w[4 * k + 2], w[4 * k + 3]);
        }
        __syncthreads();   // the other tile has been read before the last one of these
        if (s + 1 < a.steps && i0 + kTile < a.d) fetch(i0 + kTile);
        if (whole) {
            constexpr int kLanes = 8 * kWords, kRows = 32 / kLanes;   // lanes along a row of the tile
#pragma unroll
            for (int k = 0; k < kTile / 8 / kRows; ++k) {
                const int r = (k * 8 + warp) * kRows + lane / kLanes, w = lane % kLanes;
                if (i0 + r < a.d)
                    reinterpret_cast<uint4 *>(x + (i0 + r) * a.ldo + c0)[w] = reinterpret_cast<const uint4 *>(tile + r * kPitch)[w];
            }
        } else {
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                const int r = warp + 8 * k;
#pragma unroll
                for (int u = 0; u < 2; ++u) {
                    const int64_t c = c0 + lane + 32 * u;
                    if (i0 + r < a.d && c < a.n) x[(i0 + r) * a.ldo + c] = reinterpret_cast<const TX *>(tile + r * kPitch)[lane + 32 * u];
                }
            }
        }
    }
}

// ---------------------------------------------------------------------------
// Gradient, first launch: some blocks sort the tokens, the others turn dx into rows, a token each (read from its columns the
// gradient would fetch 32 bytes for every two).
//
// Up to kRankTokens tokens are sorted by counting: a token's place is the number of tokens that come before it. That is n^2
// comparisons, spread over all SMs: the launch takes 5 us for 777 tokens of 1000 features, 24 for 8000 of 200 and 28 for 8192 of
// 4096, where the turn is longer. The radix sort below takes 28 us a digit of 16385 tokens and 44 of 32768, in one block. Around
// the limit, two digits: 16384 tokens of 4096 features take 71 us by counting and 79 by digits, of 512 features 63 and 50. The
// turn of dx hides neither.
//
// The radix sort is stable, 8 bits a pass, by one block. Each warp owns a contiguous run of tokens; counts are kept per digit
// and warp, so that a scan of them in that order gives every warp its places.
// ---------------------------------------------------------------------------
constexpr int kRankTokens = 16384;
constexpr int kSortWarps = 16;
constexpr int kSortPitch = 257;   // of a warp's counts: no bank conflicts when the scan reads across warps
constexpr int kTurnThreads = kSortWarps * 32;
static_assert(kTurnThreads == 512, "two threads scan a digit");
constexpr int kTurnTokens = 128, kTurnFeatures = 64;   // a tile of the others

__device__ __forceinline__ int embed_passes(int32_t vocab) {   // digits of the values 0 .. vocab
    int p = 1;
    while (p < 4 && ((int64_t)vocab >> (8 * p)) != 0) ++p;
    return p;
}

// The lanes of this warp with the same digit, by eight ballots (with a match in their place the launch takes 42 for 50 us, two
// digits of 16385 tokens as frequent as in text).
__device__ __forceinline__ unsigned same_digit(int digit, bool in) {
    unsigned m = __ballot_sync(0xffffffffu, in);
    if (!in) m = ~m;
#pragma unroll
    for (int b = 0; b < 8; ++b) {
        const bool set = (digit >> b) & 1;
        const unsigned v = __ballot_sync(0xffffffffu, set);
        m &= set ? v : ~v;
    }
    return m;
}

__device__ void embed_sort(const EmbedArgs &a, int32_t (*count)[kSortPitch]) {
    constexpr int kAhead = 8;   // rounds whose tokens are fetched together
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
        const int32_t *source = p > 0 ? kin : a.tokens;
        int32_t key[kAhead];
        auto fetch = [&](int64_t k) {
#pragma unroll
            for (int u = 0; u < kAhead; ++u) {
                const int64_t at = k + 32 * u + lane;
                key[u] = at < k1 ? source[at] : -1;
            }
            if (p > 0) return;
            bool beyond = false;   // once for all: a branch at each token would keep them from being fetched together
#pragma unroll
            for (int u = 0; u < kAhead; ++u) {
                beyond |= key[u] >= a.vocab;
                const bool pad = key[u] < 0 || key[u] >= a.vocab;
                key[u] = k + 32 * u + lane >= k1 ? -1 : pad ? a.vocab : key[u];
            }
            if (beyond) dev_flag(a.hdr, CSRT_DEV_INVALID);
        };
        for (int j = lane; j < 256; j += 32) count[warp][j] = 0;
        __syncwarp();
        for (int64_t k = k0; k < k1; k += 32 * kAhead) {
            fetch(k);
#pragma unroll
            for (int u = 0; u < kAhead; ++u)
                if (key[u] >= 0) atomicAdd(&count[warp][(key[u] >> (8 * p)) & 255], 1);
        }
        __syncthreads();
        // exclusive scan of the counts in digit-major order: half a digit's warps a thread
        constexpr int kHalf = kSortWarps / 2;
        const int digit = threadIdx.x >> 1, w0 = (threadIdx.x & 1) * kHalf;
        int32_t own[kHalf], sum = 0;
#pragma unroll
        for (int j = 0; j < kHalf; ++j) {
            own[j] = sum;
            sum += count[w0 + j][digit];
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
#pragma unroll
        for (int j = 0; j < kHalf; ++j) count[w0 + j][digit] = base + own[j];
        __syncthreads();
        for (int64_t k = k0; k < k1; k += 32 * kAhead) {
            int32_t col[kAhead];
            fetch(k);
#pragma unroll
            for (int u = 0; u < kAhead; ++u) {
                const int64_t at = k + 32 * u + lane;
                col[u] = p > 0 && at < k1 ? iin[at] : (int32_t)at;
            }
            // apart from the places, which depend on the rounds before, so that the ballots of all rounds overlap
            unsigned same[kAhead];
#pragma unroll
            for (int u = 0; u < kAhead; ++u) same[u] = same_digit((key[u] >> (8 * p)) & 255, key[u] >= 0);
#pragma unroll
            for (int u = 0; u < kAhead; ++u) {
                if (k + 32 * u >= k1) break;
                const int d = (key[u] >> (8 * p)) & 255;
                const int before = __popc(same[u] & ((1u << lane) - 1));
                const int32_t at = count[warp][d];
                __syncwarp();
                if (key[u] >= 0) {
                    kout[at + before] = key[u];
                    iout[at + before] = col[u];
                    if (before == 0) count[warp][d] = at + __popc(same[u]);
                }
                __syncwarp();
            }
        }
        __syncthreads();
    }
}

// The places of 64 tokens: eight slices of the threads compare them with an eighth of all tokens each.
constexpr int kRankColumns = 64, kRankKeys = 4096;

__device__ __forceinline__ void embed_rank(const EmbedArgs &a, int32_t block, int32_t *keys) {
    __shared__ int32_t part[kTurnThreads / kRankColumns][kRankColumns];
    constexpr int kSlices = kTurnThreads / kRankColumns;
    const int slice = threadIdx.x / kRankColumns, column = threadIdx.x % kRankColumns;
    const int32_t c0 = block * kRankColumns, c = c0 + column;
    auto token = [&](int32_t k) {
        const int32_t t = a.tokens[k];
        return t < 0 || t >= a.vocab ? a.vocab : t;
    };
    const int32_t mine = c < a.n ? token(c) : 0;
    if (slice == 0 && c < a.n && a.tokens[c] >= a.vocab) dev_flag(a.hdr, CSRT_DEV_INVALID);
    int32_t before = 0;
    for (int32_t base = 0; base < a.n; base += kRankKeys) {
        __syncthreads();
#pragma unroll
        for (int k = 0; k < kRankKeys / kTurnThreads; ++k) {
            const int32_t at = base + k * kTurnThreads + threadIdx.x;
            keys[k * kTurnThreads + threadIdx.x] = at < a.n ? token(at) : INT32_MAX;
        }
        __syncthreads();
        // each slice's keys, a multiple of four; behind the last are INT32_MAX
        const int length = (imin(kRankKeys, a.n - base) + 4 * kSlices - 1) / (4 * kSlices) * 4;
        const int32_t first = base + slice * length;
        const int4 *p = reinterpret_cast<const int4 *>(keys + slice * length);
        if (first + length <= c0 || first >= c0 + kRankColumns) {
            // equal tokens count where they lie in front
            const int32_t below = first < c0 ? mine + 1 : mine;
#pragma unroll 8
            for (int k = 0; k < length / 4; ++k) {
                const int4 v = p[k];
                before += (v.x < below) + (v.y < below) + (v.z < below) + (v.w < below);
            }
        } else {
#pragma unroll 2
            for (int k = 0; k < length / 4; ++k) {
                const int4 v = p[k];
                const int32_t at = first + 4 * k;
                before += (v.x < mine + (at < c)) + (v.y < mine + (at + 1 < c)) + (v.z < mine + (at + 2 < c)) + (v.w < mine + (at + 3 < c));
            }
        }
    }
    part[slice][column] = before;
    __syncthreads();
    if (slice != 0 || c >= a.n) return;
    int32_t place = 0;
#pragma unroll
    for (int s = 0; s < kSlices; ++s) place += part[s][column];
    a.key[0][place] = mine;
    a.idx[0][place] = c;
}

// A tile of 64 features x 128 tokens of dx into rows. 16-bit elements: eight tokens of a feature go into shared memory as a
// word of 16 bytes, words of eight features being permuted so that a warp reads eight features of eight tokens without bank
// conflicts; a thread takes two tokens of eight features from there and writes 16 bytes of each token's row (the same with
// 2-byte accesses throughout: 43 us for 4096 x 8192). in_vec: rows of whole 16-byte words; else they are read by elements.
template <typename TX>
__device__ __forceinline__ void embed_turn(const EmbedArgs &a, int64_t unit, char *space) {
    const int64_t along = ceil_div<int64_t>(a.n, kTurnTokens);
    const int64_t c0 = unit % along * kTurnTokens, i0 = unit / along * kTurnFeatures;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const TX *dx = reinterpret_cast<const TX *>(a.table);
    TX *out = reinterpret_cast<TX *>(a.rows);
    if constexpr (sizeof(TX) == 2) {
        constexpr int kWords = kTurnTokens / 8;   // of a feature
        uint4 *tile = reinterpret_cast<uint4 *>(space);
        if (a.in_vec && c0 + kTurnTokens <= a.n) {
            uint4 v[kTurnFeatures * kWords / kTurnThreads];
#pragma unroll
            for (int k = 0; k < kTurnFeatures * kWords / kTurnThreads; ++k) {
                const int u = k * kTurnThreads + threadIdx.x, f = u / kWords, w = u % kWords;
                v[k] = make_uint4(0, 0, 0, 0);
                if (i0 + f < a.d) v[k] = __ldg(reinterpret_cast<const uint4 *>(dx + (i0 + f) * a.ld + c0) + w);
            }
#pragma unroll
            for (int k = 0; k < kTurnFeatures * kWords / kTurnThreads; ++k) {
                const int u = k * kTurnThreads + threadIdx.x, f = u / kWords, w = u % kWords;
                tile[f * kWords + (w ^ (f >> 3))] = v[k];
            }
        } else {
            TX v[kTurnFeatures * kTurnTokens / kTurnThreads];
#pragma unroll
            for (int k = 0; k < kTurnFeatures * kTurnTokens / kTurnThreads; ++k) {
                const int u = k * kTurnThreads + threadIdx.x, f = u / kTurnTokens, t = u % kTurnTokens;
                v[k] = i0 + f < a.d && c0 + t < a.n ? dx[(i0 + f) * a.ld + c0 + t] : from_f<TX>(0.f);
            }
#pragma unroll
            for (int k = 0; k < kTurnFeatures * kTurnTokens / kTurnThreads; ++k) {
                const int u = k * kTurnThreads + threadIdx.x, f = u / kTurnTokens, t = u % kTurnTokens;
                reinterpret_cast<TX *>(space)[f * kTurnTokens + (((t >> 3) ^ (f >> 3)) << 3) + (t & 7)] = v[k];
            }
        }
        __syncthreads();
        const int g = lane & 7, t = warp * 8 + (lane >> 3) * 2;   // eight features, two tokens
        const uint32_t *word = reinterpret_cast<const uint32_t *>(space) + g * 8 * (kTurnTokens / 2) + (((t >> 3) ^ g) << 2) + ((t & 7) >> 1);
        uint32_t x[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) x[j] = word[j * (kTurnTokens / 2)];
        uint4 lo, hi;
        lo.x = __byte_perm(x[0], x[1], 0x5410); hi.x = __byte_perm(x[0], x[1], 0x7632);
        lo.y = __byte_perm(x[2], x[3], 0x5410); hi.y = __byte_perm(x[2], x[3], 0x7632);
        lo.z = __byte_perm(x[4], x[5], 0x5410); hi.z = __byte_perm(x[4], x[5], 0x7632);
        lo.w = __byte_perm(x[6], x[7], 0x5410); hi.w = __byte_perm(x[6], x[7], 0x7632);
        const int64_t c = c0 + t, i = i0 + g * 8;
        if (i >= a.pitch) return;
        if (c < a.n) *reinterpret_cast<uint4 *>(out + c * a.pitch + i) = lo;
        if (c + 1 < a.n) *reinterpret_cast<uint4 *>(out + (c + 1) * a.pitch + i) = hi;
    } else {
        constexpr int kPitch = kTurnTokens + 1;
        TX *tile = reinterpret_cast<TX *>(space);
#pragma unroll
        for (int k = 0; k < kTurnFeatures / kSortWarps; ++k) {
            const int f = warp + k * kSortWarps;
#pragma unroll
            for (int j = 0; j < 4; ++j)
                tile[f * kPitch + lane + 32 * j] =
                    i0 + f < a.d && c0 + lane + 32 * j < a.n ? dx[(i0 + f) * a.ld + c0 + lane + 32 * j] : 0.f;
        }
        __syncthreads();
#pragma unroll
        for (int k = 0; k < kTurnTokens / kSortWarps; ++k) {
            const int t = warp + k * kSortWarps;
            const int64_t c = c0 + t, i = i0 + 2 * lane;
            if (c < a.n && i < a.pitch)
                *reinterpret_cast<float2 *>(out + c * a.pitch + i) =
                    make_float2(tile[2 * lane * kPitch + t], tile[(2 * lane + 1) * kPitch + t]);
        }
    }
}

template <typename TX, bool RANK>
__global__ void __launch_bounds__(kTurnThreads, RANK ? 4 : 2) embed_turn_kernel(EmbedArgs a) {
    pdl_enter();
    constexpr size_t kTile = kTurnFeatures * (kTurnTokens + 2) * sizeof(TX);
    constexpr size_t kSort = (RANK ? kRankKeys : kSortPitch * kSortWarps) * sizeof(int32_t);
    __shared__ __align__(16) char space[kTile > kSort ? kTile : kSort];
    const int64_t unit = (int64_t)blockIdx.x - a.sort_blocks;
    if (unit >= 0) embed_turn<TX>(a, unit, space);
    else if (RANK) embed_rank(a, (int32_t)blockIdx.x, reinterpret_cast<int32_t *>(space));
    else embed_sort(a, reinterpret_cast<int32_t(*)[kSortPitch]>(space));
}

// ---------------------------------------------------------------------------
// Second launch: sums over the sorted tokens, kChunk of them by `lanes` threads with eight features each, so that a token
// that comes often is shared among many. A token's run that lies within a chunk is finished there; the parts of one that does
// not are kept, and added in order by the third launch. Other blocks write zeros into the rows that no token is.
// VEC: a thread's features lie side by side and are stored by 16-byte words; else (rows of the table that are not aligned)
// they lie `lanes` apart, so that the threads' stores do.
// ---------------------------------------------------------------------------
constexpr int kSumThreads = 128, kZeroRows = 32;
constexpr int kFewTokens = 4096;   // up to which chunks are short: few tokens leave threads idle
constexpr int kShortChunk = 8, kLongChunk = 32;

template <typename T, bool VEC>
struct Row8 {
    static constexpr int kWords = VEC ? (int)sizeof(T) * 2 : 8;
    uint32_t w[kWords];
    // non-VEC: the first `count` of eight elements that lie `step` apart
    __device__ __forceinline__ void load(const T *p, int step, int count) {
        if constexpr (VEC) {
#pragma unroll
            for (int k = 0; k < kWords / 4; ++k) {
                const uint4 x = __ldg(reinterpret_cast<const uint4 *>(p) + k);
                w[4 * k] = x.x;
                w[4 * k + 1] = x.y;
                w[4 * k + 2] = x.z;
                w[4 * k + 3] = x.w;
            }
        } else {
#pragma unroll
            for (int k = 0; k < 8; ++k) w[k] = k < count ? __float_as_uint(to_f<T>(p[k * step])) : 0u;
        }
    }
    __device__ __forceinline__ void set(const float (&v)[8]) {
#pragma unroll
        for (int k = 0; k < kWords; ++k) {
            if constexpr (!VEC || sizeof(T) == 4) {
                w[k] = __float_as_uint(v[k]);
            } else {
                const T lo = from_f<T>(v[2 * k]), hi = from_f<T>(v[2 * k + 1]);
                w[k] = *reinterpret_cast<const unsigned short *>(&lo) | (uint32_t)*reinterpret_cast<const unsigned short *>(&hi) << 16;
            }
        }
    }
    __device__ __forceinline__ float get(int k) const {
        if constexpr (!VEC || sizeof(T) == 4) return __uint_as_float(w[k]);
        else {
            const unsigned short h = (unsigned short)(w[k >> 1] >> (16 * (k & 1)));
            return to_f<T>(*reinterpret_cast<const T *>(&h));
        }
    }
};

// A thread's eight features: i + k * step; the first `count` lie within a row's pitch.
struct Features {
    int64_t i;
    int step, count;
};
template <bool VEC>
__device__ __forceinline__ Features embed_features(const EmbedArgs &a, int64_t group) {
    const int t = threadIdx.x % a.lanes;
    if (VEC) return Features{(group * a.lanes + t) * 8, 1, 8};
    const int64_t i = group * a.lanes * 8 + t;
    return Features{i, a.lanes, (int)imin<int64_t>(8, (a.pitch - i + a.lanes - 1) / a.lanes)};
}

// scale * s into a row of the table, or added to `old`, what is there.
template <typename T, bool VEC, bool ADD>
__device__ __forceinline__ void put_row(const EmbedArgs &a, int64_t v, Features f, const float (&s)[8], const Row8<T, VEC> &old) {
    T *o = reinterpret_cast<T *>(a.out) + v * a.ldo + f.i;
    float w[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) w[k] = ADD ? fmaf(s[k], a.scale, old.get(k)) : s[k] * a.scale;
    if (VEC && f.i + 8 <= a.d) {
        if constexpr (sizeof(T) == 4) {
            reinterpret_cast<float4 *>(o)[0] = make_float4(w[0], w[1], w[2], w[3]);
            reinterpret_cast<float4 *>(o)[1] = make_float4(w[4], w[5], w[6], w[7]);
        } else {
            alignas(16) T h[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) h[k] = from_f<T>(w[k]);
            *reinterpret_cast<uint4 *>(o) = *reinterpret_cast<const uint4 *>(h);
        }
        return;
    }
#pragma unroll
    for (int k = 0; k < 8; ++k)
        if (f.i + k * f.step < a.d) o[k * f.step] = from_f<T>(w[k]);
}
// What is there: the elements of row v that lie within the table.
template <typename T, bool VEC>
__device__ __forceinline__ void load_row(const EmbedArgs &a, int64_t v, Features f, Row8<T, VEC> &old) {
    const T *o = reinterpret_cast<const T *>(a.out) + v * a.ldo + f.i;
    if (VEC && f.i + 8 > a.d) {   // the row's end: by elements
        float w[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) w[k] = f.i + k < a.d ? to_f<T>(o[k]) : 0.f;
        old.set(w);
    } else {
        old.load(o, f.step, VEC ? 8 : (int)imin<int64_t>(f.count, (a.d - f.i + f.step - 1) / f.step));
    }
}

// ADD: the rows that the sums are added to are fetched with dx's.
template <typename TX, typename TT, bool VEC, bool ADD>
__device__ __forceinline__ void embed_chunk(const EmbedArgs &a, int64_t chunk, Features f) {
    constexpr int kAhead = ADD || sizeof(TX) == 4 ? 4 : 8;
    const int32_t *key = a.key[0], *idx = a.idx[0];
    const TX *rows = reinterpret_cast<const TX *>(a.rows) + f.i;
    const int64_t k0 = chunk * a.chunk, k1 = imin<int64_t>(a.n, k0 + a.chunk);
    int32_t v = __ldg(key + k0);
    bool head = k0 > 0 && __ldg(key + k0 - 1) == v;   // the run began before this chunk
    float s[8] = {0.f};
    auto keep = [&](int slot) {
        float *o = a.partial + (chunk * 2 + slot) * a.pitch + f.i;
#pragma unroll
        for (int k = 0; k < 8; ++k)
            if (k < f.count) o[k * f.step] = s[k];
    };
    for (int64_t k = k0; k < k1; k += kAhead) {
        int32_t token[kAhead + 1];   // and the one behind them
        Row8<TX, VEC> x[kAhead];
        Row8<TT, VEC> old[ADD ? kAhead : 1];
#pragma unroll
        for (int u = 0; u <= kAhead; ++u) token[u] = k + u < a.n ? __ldg(key + k + u) : a.vocab;
        // without conditions, so that all are on their way together: a row beyond the chunk's end is fetched for nothing
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            x[u].load(rows + (int64_t)__ldg(idx + imin<int64_t>(k + u, k1 - 1)) * a.pitch, f.step, f.count);
            if (ADD) load_row<TT, VEC>(a, imin(token[u], a.vocab - 1), f, old[ADD ? u : 0]);
        }
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            if (k + u >= k1 || token[u] >= a.vocab) break;   // padding sorts last
#pragma unroll
            for (int j = 0; j < 8; ++j) s[j] += x[u].get(j);
            if (token[u] != token[u + 1]) {   // the run is over
                if (head) keep(0);
                else put_row<TT, VEC, ADD>(a, token[u], f, s, old[ADD ? u : 0]);
                head = false;
#pragma unroll
                for (int j = 0; j < 8; ++j) s[j] = 0.f;
            } else if (k + u + 1 == k1) {
                keep(head ? 0 : 1);
            }
        }
    }
}

// A row of zeros by `threads` threads (eight at least): 16-byte words, and the elements in front of the first and behind the
// last.
template <typename T>
__device__ __forceinline__ void zero_row(T *row, int64_t d, int thread, int threads) {
    constexpr int each = 16 / (int)sizeof(T);
    const int64_t front = imin<int64_t>(d, (int64_t)(-reinterpret_cast<uintptr_t>(row) & 15) / (int64_t)sizeof(T));
    const int64_t words = (d - front) / each, back = front + words * each;
    for (int64_t j = thread; j < words; j += threads) reinterpret_cast<uint4 *>(row + front)[j] = make_uint4(0, 0, 0, 0);
    if (thread < front) row[thread] = from_f<T>(0.f);
    if (thread < d - back) row[back + thread] = from_f<T>(0.f);
}

// The group of features and the chunk that a thread of the second and third launch works on.
template <bool VEC>
__device__ __forceinline__ bool embed_place(const EmbedArgs &a, Features &f, int64_t &chunk) {
    const int64_t across = ceil_div<int64_t>(a.pitch, (int64_t)a.lanes * 8);
    f = embed_features<VEC>(a, (int64_t)blockIdx.x % across);
    chunk = (int64_t)blockIdx.x / across * (kSumThreads / a.lanes) + threadIdx.x / a.lanes;
    return f.i < a.pitch && chunk < a.chunks;
}

template <typename TX, typename TT, bool VEC, bool ADD>
__global__ void __launch_bounds__(kSumThreads) embed_sum_kernel(EmbedArgs a) {
    pdl_enter();
    if (blockIdx.x < a.sum_blocks) {
        Features f;
        int64_t chunk;
        if (embed_place<VEC>(a, f, chunk)) embed_chunk<TX, TT, VEC, ADD>(a, chunk, f);
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
    TT *out = reinterpret_cast<TT *>(a.out) + v0 * a.ldo;
    for (int r = 0; r < rows; ++r, out += a.ldo) {
        if (used[r]) continue;
        zero_row(out, a.d, threadIdx.x, kSumThreads);
    }
}

// Third launch: the runs that begin in a chunk and go on after it.
template <typename TT, bool VEC>
__global__ void __launch_bounds__(kSumThreads) embed_join_kernel(EmbedArgs a) {
    pdl_enter();
    Features f;
    int64_t chunk;
    if (!embed_place<VEC>(a, f, chunk) || chunk + 1 >= a.chunks) return;
    const int32_t *key = a.key[0];
    const int64_t k0 = chunk * a.chunk, next = k0 + a.chunk;
    const int32_t v = __ldg(key + next - 1), after = __ldg(key + next), before = k0 > 0 ? __ldg(key + k0 - 1) : -1;
    if (v >= a.vocab || after != v || before == v) return;   // sorted: if the token before is v, all of the chunk is
    constexpr int kAhead = 4;   // chunks whose part is fetched before it is known whether v reaches them
    float s[8];
    Row8<float, VEC> x[kAhead];
    Row8<TT, VEC> old;
    if (a.accumulate) load_row<TT, VEC>(a, v, f, old);
    x[0].load(a.partial + (chunk * 2 + 1) * a.pitch + f.i, f.step, f.count);
#pragma unroll
    for (int k = 0; k < 8; ++k) s[k] = x[0].get(k);
    bool more = true;
    for (int64_t c = chunk + 1; more && c < a.chunks; c += kAhead) {
        int32_t token[kAhead];
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            const int64_t at = imin<int64_t>(c + u, a.chunks - 1);
            token[u] = __ldg(key + at * a.chunk);
            x[u].load(a.partial + at * 2 * a.pitch + f.i, f.step, f.count);
        }
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            more = more && c + u < a.chunks && token[u] == v;
            if (!more) break;
#pragma unroll
            for (int k = 0; k < 8; ++k) s[k] += x[u].get(k);
        }
    }
    if (a.accumulate) put_row<TT, VEC, true>(a, v, f, s, old);
    else put_row<TT, VEC, false>(a, v, f, s, old);
}

// ---------------------------------------------------------------------------
// Gradient of few tokens, one launch: a block takes 32 features, keeps them for all tokens in shared memory and sorts the
// tokens itself; a warp adds the runs that begin in its share of the sorted tokens, a feature a lane, and writes 32 features
// of their rows. Other blocks write the zeros. 64 tokens of 4096 features added to a table: 4.5 us, in three launches 8.1; 200
// of 300 into 5000 rows 8.0 and 12.5; 512 of 4096 17.7 and 9.4, as every block sorts for itself and holds all tokens.
// ---------------------------------------------------------------------------
constexpr int kSmallTokens = 256, kSmallFeatures = 32, kSmallThreads = 1024;
static_assert(kSmallThreads == 32 * kSmallFeatures, "a warp fetches a feature");

template <typename TX>
constexpr int small_pitch(int n) {   // elements: rows of an odd number of 4-byte words, a lane each without bank conflicts
    return sizeof(TX) == 4 ? n | 1 : ((n + 1) / 2 | 1) * 2;
}

template <typename TX, typename TT>
__global__ void __launch_bounds__(kSmallThreads) embed_bwd_small_kernel(EmbedArgs a) {
    pdl_enter();
    constexpr int kAhead = 8;   // runs whose rows are fetched together
    extern __shared__ __align__(16) char space[];
    constexpr int32_t kPad = INT32_MAX - 1;                 // above every token, below what lies behind the last one
    __shared__ __align__(16) int32_t keys[kSmallThreads];   // tokens, kPad, INT32_MAX
    __shared__ int32_t place[kSmallThreads], sorted[kSmallThreads], column[kSmallThreads];
    __shared__ int32_t used[kZeroRows];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int64_t groups = ceil_div<int64_t>(a.d, kSmallFeatures);
    TT *out = reinterpret_cast<TT *>(a.out);
    const int t = threadIdx.x;
    int32_t token = t < a.n ? a.tokens[t] : -1;
    if (token >= a.vocab) {
        if (blockIdx.x == 0) dev_flag(a.hdr, CSRT_DEV_INVALID);
        token = -1;
    }
    if (blockIdx.x >= groups) {
        const int64_t v0 = ((int64_t)blockIdx.x - groups) * kZeroRows;
        const int rows = (int)imin<int64_t>(kZeroRows, a.vocab - v0);
        if (t < kZeroRows) used[t] = 0;
        __syncthreads();
        if (token >= v0 && token < v0 + rows) used[token - v0] = 1;
        __syncthreads();
        for (int r = warp; r < rows; r += kSmallThreads / 32)
            if (!used[r]) zero_row(out + (v0 + r) * a.ldo, a.d, lane, 32);
        return;
    }
    const int64_t i0 = (int64_t)blockIdx.x * kSmallFeatures;
    const int features = (int)imin<int64_t>(kSmallFeatures, a.d - i0), pitch = a.lanes;
    TX *tile = reinterpret_cast<TX *>(space);
    const TX *dx = reinterpret_cast<const TX *>(a.table) + i0 * a.ld;
    if (warp < features)
#pragma unroll 16
        for (int c = lane; c < a.n; c += 32) tile[warp * pitch + c] = dx[warp * a.ld + c];
    // a token's place: the tokens that come before it, counted by size columns x slices of threads
    keys[t] = t >= a.n ? INT32_MAX : token < 0 ? kPad : token;
    place[t] = 0;
    int size = 32;
    while (size < a.n) size <<= 1;
    const int slices = kSmallThreads / size, c = t % size, length = (a.n + 4 * slices - 1) / (4 * slices) * 4;
    __syncthreads();
    if (c < a.n) {
        const int32_t mine = keys[c];
        const int from = t / size * length;
        int before = 0;
#pragma unroll 4
        for (int k = from; k < imin(from + length, a.n); k += 4) {   // equal ones count where they lie in front
            const int4 v = *reinterpret_cast<const int4 *>(keys + k);
            before += (v.x < mine + (k < c)) + (v.y < mine + (k + 1 < c)) + (v.z < mine + (k + 2 < c)) + (v.w < mine + (k + 3 < c));
        }
        atomicAdd(place + c, before);
    }
    __syncthreads();
    if (t < a.n) {
        sorted[place[t]] = keys[t];
        column[place[t]] = t;
    }
    __syncthreads();
    const int per = (a.n + 31) / 32, p0 = imin(a.n, warp * per), p1 = imin(a.n, p0 + per);
    const bool in = lane < features;
    auto token_at = [&](int p) { return p < a.n ? sorted[p] : kPad; };
    for (int p = p0; p < p1; p += kAhead) {
        TT old[kAhead];
        int32_t v[kAhead];
        bool first[kAhead];
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            v[u] = p + u < p1 ? token_at(p + u) : kPad;
            first[u] = v[u] != kPad && (p + u == 0 || token_at(p + u - 1) != v[u]);
            old[u] = from_f<TT>(0.f);
            if (first[u] && a.accumulate && in) old[u] = out[(int64_t)v[u] * a.ldo + i0 + lane];
        }
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            if (!first[u]) continue;
            float s = 0.f;
            for (int q = p + u; token_at(q) == v[u]; ++q)
                if (in) s += to_f<TX>(tile[lane * pitch + column[q]]);
            if (in)
                out[(int64_t)v[u] * a.ldo + i0 + lane] = from_f<TT>(a.accumulate ? fmaf(s, a.scale, to_f<TT>(old[u])) : s * a.scale);
        }
    }
}

// ---------------------------------------------------------------------------
// Host
// ---------------------------------------------------------------------------
static size_t embed_list_bytes(int64_t n) { return align_up((size_t)n * sizeof(int32_t), 256); }
static int64_t embed_pitch(int64_t d) { return ceil_div<int64_t>(d, 8) * 8; }
// the sorted tokens, dx in rows (float32 at most), the parts of runs
static size_t embed_bytes(int64_t d, int64_t n) {
    const size_t row = (size_t)embed_pitch(d) * sizeof(float);
    const int64_t chunks = imax(ceil_div<int64_t>(imin<int64_t>(n, kFewTokens), kShortChunk), ceil_div<int64_t>(n, kLongChunk));
    return kWsReservedBytes + 4 * embed_list_bytes(n) + align_up((size_t)n * row, 256) + align_up(chunks * 2 * row, 256);
}

static int check_embed(const int32_t *tokens, float scale, int32_t vocab, int32_t n, const csrt_mat *out,
                       const char *out_name, void *ws, size_t ws_bytes, size_t need) {
    CSRT_ARG(n == 0 || tokens != nullptr, "tokens is NULL");
    CSRT_TRY(check_vector(reinterpret_cast<const float *>(tokens), "tokens"));
    CSRT_ARG(!vector_meets(reinterpret_cast<const float *>(tokens), n, out), "tokens overlap %s", out_name);
    CSRT_ARG(std::isfinite(scale), "scale must be finite");
    CSRT_ARG(vocab < INT32_MAX, "the table has too many rows");
    CSRT_ARG(ws != nullptr, "workspace is NULL");
    CSRT_ARG((reinterpret_cast<uintptr_t>(ws) & 255) == 0, "workspace is not 256-byte aligned");
    if (ws_bytes < need) return fail(CSRT_ERR_WORKSPACE, "workspace has %zu bytes, needs %zu", ws_bytes, need);
    return CSRT_OK;
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
    a.chunk = n <= kFewTokens ? kShortChunk : kLongChunk;
    a.chunks = (int32_t)ceil_div<int64_t>(n, a.chunk);
    return a;
}

template <typename TT, typename TX>
static int launch_embed_fwd(EmbedArgs a, cudaStream_t s) {
    const int64_t tiles = ceil_div<int64_t>(a.n, kTile) * ceil_div<int64_t>(a.d, kTile);
    a.steps = (int32_t)imin<int64_t>(kSteps, imax<int64_t>(1, tiles / (num_sms() * 6)));
    const int64_t blocks = ceil_div<int64_t>(a.n, kTile) * ceil_div<int64_t>(a.d, kTile * a.steps);
    CSRT_ARG(blocks <= INT32_MAX, "x is too large");
    launch_pdl(embed_fwd_kernel<TT, TX>, dim3((unsigned)blocks), dim3(256), 0, s, a);
    count_launch();
    return check_launch("embed_fwd_kernel");
}

template <typename TX, typename TT, bool VEC>
static int launch_embed_sums(const EmbedArgs &a, cudaStream_t s) {
    const int64_t zero_blocks = a.accumulate ? 0 : ceil_div<int64_t>(a.vocab, kZeroRows);
    CSRT_ARG(a.sum_blocks + zero_blocks < INT32_MAX, "dx is too large");
    if (a.sum_blocks + zero_blocks > 0) {
        launch_pdl(a.accumulate ? embed_sum_kernel<TX, TT, VEC, true> : embed_sum_kernel<TX, TT, VEC, false>, dim3((unsigned)(a.sum_blocks + zero_blocks)), dim3(kSumThreads), 0, s, a);
        count_launch();
        CSRT_TRY(check_launch("embed_sum_kernel"));
    }
    if (a.chunks < 2) return CSRT_OK;
    launch_pdl(embed_join_kernel<TT, VEC>, dim3((unsigned)a.sum_blocks), dim3(kSumThreads), 0, s, a);
    count_launch();
    return check_launch("embed_join_kernel");
}

template <typename TX, typename TT>
static int launch_embed_small(EmbedArgs a, cudaStream_t s) {
    a.lanes = small_pitch<TX>(a.n);
    const int smem = kSmallFeatures * a.lanes * (int)sizeof(TX);
    constexpr auto kernel = embed_bwd_small_kernel<TX, TT>;
    CSRT_TRY(allow_smem<kernel>(kSmallFeatures * small_pitch<TX>(kSmallTokens) * (int)sizeof(TX)));
    const int64_t blocks = ceil_div<int64_t>(a.d, kSmallFeatures) + (a.accumulate ? 0 : ceil_div<int64_t>(a.vocab, kZeroRows));
    CSRT_ARG(blocks < INT32_MAX, "dtable is too large");
    launch_pdl(kernel, dim3((unsigned)blocks), dim3(kSmallThreads), (size_t)smem, s, a);
    count_launch();
    return check_launch("embed_bwd_small_kernel");
}

template <typename TX, typename TT>
static int launch_embed_bwd(EmbedArgs a, cudaStream_t s) {
    if (a.n <= kSmallTokens) return launch_embed_small<TX, TT>(a, s);
    const bool rank = a.n <= kRankTokens;
    const int64_t tiles = ceil_div<int64_t>(a.n, kTurnTokens) * ceil_div<int64_t>(a.d, kTurnFeatures);
    a.sort_blocks = rank ? imax(1, ceil_div(a.n, kRankColumns)) : 1;
    for (a.lanes = 1; a.lanes < kSumThreads && a.lanes * 8 < a.pitch;) a.lanes *= 2;
    a.sum_blocks = ceil_div<int64_t>(a.pitch, (int64_t)a.lanes * 8) * ceil_div<int64_t>(a.chunks, kSumThreads / a.lanes);
    CSRT_ARG(a.sort_blocks + tiles < INT32_MAX, "dx is too large");
    launch_pdl(rank ? embed_turn_kernel<TX, true> : embed_turn_kernel<TX, false>, dim3((unsigned)(a.sort_blocks + tiles)),
               dim3(kTurnThreads), 0, s, a);
    count_launch();
    CSRT_TRY(check_launch("embed_turn_kernel"));
    return a.out_vec ? launch_embed_sums<TX, TT, true>(a, s) : launch_embed_sums<TX, TT, false>(a, s);
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
    CSRT_ARG((int64_t)d * max_n <= kMaxElems, "%d x %d activations are too large", d, max_n);   // no call takes them
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
    CSRT_TRY(check_embed(tokens, scale, vocab, n, x, "x", ws, ws_bytes, kWsReservedBytes));
    if (d == 0 || n == 0) return CSRT_OK;
    EmbedArgs a = embed_args(table, x, tokens, vocab, d, n, scale, ws);
    a.out_vec = tma_rows_ok(x->data, x->ld, dt_size(x->dtype));
    return CSRT_EMBED_DISPATCH(launch_embed_fwd, table->dtype, x->dtype, a, as_stream(stream));
}

int csrt_embed_bwd(const csrt_mat *dx, const int32_t *tokens, float scale, int32_t accumulate, csrt_mat *dtable,
                   void *ws, size_t ws_bytes, void *stream) {
    CSRT_TRY(check_mat(dx, "dx"));
    CSRT_TRY(check_mat(dtable, "dtable"));
    const int32_t vocab = dtable->rows, d = dx->rows, n = dx->cols;
    CSRT_TRY(check_shape(dtable, "dtable", vocab, d));
    CSRT_ARG(!clash(dtable, dx), "dtable overlaps dx");
    CSRT_TRY(check_embed(tokens, scale, vocab, n, dtable, "dtable", ws, ws_bytes, embed_bytes(d, n)));
    if (d == 0 || vocab == 0) return CSRT_OK;
    EmbedArgs a = embed_args(dx, dtable, tokens, vocab, d, n, scale, ws);
    a.accumulate = accumulate != 0;
    a.in_vec = tma_rows_ok(dx->data, dx->ld, dt_size(dx->dtype));
    a.out_vec = tma_rows_ok(dtable->data, dtable->ld, dt_size(dtable->dtype));
    return CSRT_EMBED_DISPATCH(launch_embed_bwd, dx->dtype, dtable->dtype, a, as_stream(stream));
}

}  // extern "C"
