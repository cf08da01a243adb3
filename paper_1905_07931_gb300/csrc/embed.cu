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
    int32_t *key[2], *idx[2];  // backward: sorted tokens (vocab: none) and their columns; the second pair is scratch
    WsHeader *hdr;
};

// ---------------------------------------------------------------------------
// Lookup: a tile of 64 tokens x 64 features passes through shared memory, read along the table's rows and written along
// x's. The rows of repeated tokens come from L2.
// ---------------------------------------------------------------------------
template <typename TT, typename TX>
__global__ void __launch_bounds__(256) embed_fwd_kernel(EmbedArgs a) {
    pdl_enter();
    __shared__ float tile[64][65];
    __shared__ int32_t tok[64];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int64_t c0 = (int64_t)blockIdx.x * 64, i0 = (int64_t)blockIdx.y * 64;
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
#pragma unroll
    for (int k = 0; k < 8; ++k) {
        const int32_t t = tok[warp + 8 * k];
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const int64_t i = i0 + lane + 32 * u;
            tile[lane + 32 * u][warp + 8 * k] = t >= 0 && i < a.d ? a.scale * to_f<TT>(table[(int64_t)t * a.ld + i]) : 0.f;
        }
    }
    __syncthreads();
    TX *x = reinterpret_cast<TX *>(a.out);
#pragma unroll
    for (int k = 0; k < 8; ++k) {
        const int64_t i = i0 + warp + 8 * k;
        if (i >= a.d) break;
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const int64_t c = c0 + lane + 32 * u;
            if (c < a.n) x[i * a.ldo + c] = from_f<TX>(tile[warp + 8 * k][lane + 32 * u]);
        }
    }
}

// ---------------------------------------------------------------------------
// Stable radix sort of the tokens by one block, 8 bits a pass. Each of the 32 warps owns a contiguous run of them; counts
// are kept per digit and warp, so that a scan of them in that order gives every warp its places.
// ---------------------------------------------------------------------------
constexpr int kSortWarps = 32;

__device__ __forceinline__ int embed_passes(int32_t vocab) {   // digits of the values 0 .. vocab
    int p = 1;
    while (p < 4 && ((int64_t)vocab >> (8 * p)) != 0) ++p;
    return p;
}

__device__ void embed_sort(const EmbedArgs &a, int32_t (*count)[kSortWarps]) {
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
        for (int64_t k = k0; k < k1; k += 32) {
            const bool in = k + lane < k1;
            const int digit = in ? (fetch(k + lane) >> (8 * p)) & 255 : 256;
            const unsigned same = __match_any_sync(full, digit);
            if (in && (same & ((1u << lane) - 1)) == 0) count[digit][warp] += __popc(same);
            __syncwarp();
        }
        __syncthreads();
        // exclusive scan of the 8192 counts in digit-major order, eight a thread
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
        for (int64_t k = k0; k < k1; k += 32) {
            const bool in = k + lane < k1;
            const int32_t key = in ? fetch(k + lane) : 0;
            const int32_t c = !in ? 0 : p > 0 ? iin[k + lane] : (int32_t)(k + lane);
            const int digit = in ? (key >> (8 * p)) & 255 : 256;
            const unsigned same = __match_any_sync(full, digit);
            const int before = __popc(same & ((1u << lane) - 1));
            const int32_t at = in ? count[digit][warp] : 0;
            __syncwarp();
            if (in) {
                kout[at + before] = key;
                iout[at + before] = c;
                if (before == 0) count[digit][warp] = at + __popc(same);
            }
            __syncwarp();
        }
        __syncthreads();
    }
}

__global__ void __launch_bounds__(1024) embed_sort_kernel(EmbedArgs a) {
    pdl_enter();
    __shared__ int32_t count[256][kSortWarps];
    embed_sort(a, count);
}

// ---------------------------------------------------------------------------
// Gradient: a warp takes rows of the table, finds each one's tokens in the sorted list and adds their columns.
// ---------------------------------------------------------------------------
template <typename TX, typename TT>
__global__ void __launch_bounds__(256) embed_bwd_kernel(EmbedArgs a) {
    pdl_enter();
    const int lane = threadIdx.x & 31;
    const int32_t *key = a.key[0], *idx = a.idx[0];
    const TX *dx = reinterpret_cast<const TX *>(a.table);
    TT *dt = reinterpret_cast<TT *>(a.out);
    for (int64_t v = (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5); v < a.vocab; v += (int64_t)gridDim.x * 8) {
        const int64_t k0 = warp_lower_bound(key, 0, a.n, (int32_t)v);
        const int64_t k1 = k0 + (warp_lower_bound(key + k0, 0, a.n - k0, (int32_t)v + 1));
        if (k0 == k1 && a.accumulate) continue;
        for (int64_t i = lane; i < a.d; i += 32) {
            float s = 0.f;
            for (int64_t k = k0; k < k1; ++k) s += to_f<TX>(dx[i * a.ld + idx[k]]);
            s *= a.scale;
            TT *o = dt + v * a.ldo + i;
            *o = from_f<TT>(a.accumulate ? to_f<TT>(*o) + s : s);
        }
    }
}

// ---------------------------------------------------------------------------
// Host
// ---------------------------------------------------------------------------
static size_t embed_list_bytes(int64_t n) { return align_up((size_t)n * sizeof(int32_t), 256); }
static size_t embed_bytes(int64_t d, int64_t n) { return kWsReservedBytes + 4 * embed_list_bytes(n); }

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
    return a;
}

template <typename TT, typename TX>
static int launch_embed_fwd(const EmbedArgs &a, cudaStream_t s) {
    const dim3 grid((unsigned)ceil_div<int64_t>(a.n, 64), (unsigned)ceil_div<int64_t>(a.d, 64));
    launch_pdl(embed_fwd_kernel<TT, TX>, grid, dim3(256), 0, s, a);
    count_launch();
    return check_launch("embed_fwd_kernel");
}

template <typename TX, typename TT>
static int launch_embed_bwd(const EmbedArgs &a, cudaStream_t s) {
    launch_pdl(embed_sort_kernel, dim3(1), dim3(1024), 0, s, a);
    count_launch();
    CSRT_TRY(check_launch("embed_sort_kernel"));
    const unsigned grid = (unsigned)imin<int64_t>(ceil_div<int64_t>(a.vocab, 8), (int64_t)num_sms() * 64);
    launch_pdl(embed_bwd_kernel<TX, TT>, dim3(grid), dim3(256), 0, s, a);
    count_launch();
    return check_launch("embed_bwd_kernel");
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
    CSRT_ARG(d <= 65535 * 64, "table has too many columns");
    if (d == 0 || n == 0) return CSRT_OK;
    const EmbedArgs a = embed_args(table, x, tokens, vocab, d, n, scale, ws);
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
    return CSRT_EMBED_DISPATCH(launch_embed_bwd, dx->dtype, dtable->dtype, a, as_stream(stream));
}

}  // extern "C"
