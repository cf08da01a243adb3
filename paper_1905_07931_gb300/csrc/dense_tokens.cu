// Forward product of one to four tokens (csrt_dense_fwd with n <= kTokensMax): every weight is used n times only, so
// the call is a stream over W and the tensor cores have nothing to gain. (Large products whose tokens are columns of a
// wider buffer are theirs: the rule in csrt_dense_fwd.)
//
// A warp takes two rows of W (or, where there are few rows, a share of two rows' K: the block's warps then join in
// shared memory). Per step each lane loads 16 bytes of either row and the 8 n values of x that belong to them - x is
// K x n with the tokens contiguous, so they are consecutive too, and all warps of an SM find them in L1 - and runs
// 16 n float32 FMAs. Bound by the stream: 4096 x 4096 at n = 1 reads 33.6 MB in 7.4 us (4.5 TB/s with the launch; 5.0 us
// at the measured copy rate), 4096 x 9216 75.5 MB in 13.8 us. Two rows per warp halve the x traffic in L1 and double the
// loads in flight: one row takes 8.0 and 15.3 us, four rows 7.3 and 13.7 but 3.7 instead of 2.8 us on 300 x 784. Above
// four tokens the float32 FMAs (n per weight) no longer fit beside the stream and the tensor cores take over.
//
// That is the vector form. Where K is no multiple of eight, W's rows are not 16-byte aligned or x has gaps, a lane reads
// two bytes at a time: 4096 x 4097 takes 11.7 us for one token, 17.8 for four (tight x), 300 x 784 with x in rows of 64
// 6.8 and 15.1.
#include "gemm16.cuh"
#include "dense_tokens.cuh"

namespace csrt {

constexpr int kTokWarps = 8;
constexpr int kTokRows = 2;

// Blocks an SM holds, by the registers n tokens take. Two tokens are held to fewer than the 40 they would take (17.7 ->
// 15.7 us on 4096 x 9216), more tokens spill in their loop then; one token takes 32 by itself, and a bound makes the
// compiler order its loads worse (4096 x 4096: 7.6 us without one, 15 with the weakest).
__host__ __device__ constexpr int tok_blocks(int n) {
    return n == 1 ? 8 : n == 2 ? 7 : n == 3 ? 5 : 4;
}


template <int N, bool VEC, bool F16>
__global__ void __launch_bounds__(kTokWarps * 32, N == 1 ? 0 : tok_blocks(N)) dense_tokens_kernel(const __grid_constant__ TokenArgs a) {
    pdl_enter();
    __shared__ float s_part[kTokWarps][kTokRows * N];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int group = warp / a.wpr, part = warp % a.wpr;       // wpr warps share a group of rows
    const int row0 = (blockIdx.x * (kTokWarps / a.wpr) + group) * kTokRows;
    const int dtype = F16 ? CSRT_DT_F16 : CSRT_DT_BF16;
    float acc[kTokRows][N];
#pragma unroll
    for (int r = 0; r < kTokRows; ++r)
#pragma unroll
        for (int c = 0; c < N; ++c) acc[r][c] = 0.f;
    if (row0 < a.m) {
        const uint16_t *w[kTokRows];
#pragma unroll
        for (int r = 0; r < kTokRows; ++r) w[r] = a.w + (int64_t)min(row0 + r, a.m - 1) * a.ldw;
        if constexpr (VEC) {
            const int steps = a.k / 8;   // k % 8 == 0 here
#pragma unroll 8
            for (int t = part * 32 + lane; t < steps; t += a.wpr * 32) {
                uint4 u[kTokRows];
#pragma unroll
                for (int r = 0; r < kTokRows; ++r) u[r] = ld_stream_u4(w[r] + (int64_t)t * 8);
                uint32_t x[4 * N];
                const uint4 *xp = reinterpret_cast<const uint4 *>(a.x + (int64_t)t * 8 * N);
#pragma unroll
                for (int i = 0; i < N; ++i) {
                    const uint4 q = __ldg(xp + i);
                    x[4 * i] = q.x, x[4 * i + 1] = q.y, x[4 * i + 2] = q.z, x[4 * i + 3] = q.w;
                }
                float xf[8 * N];
#pragma unroll
                for (int i = 0; i < 4 * N; ++i) {
                    const float2 p = unpack16(x[i], F16);
                    xf[2 * i] = p.x;
                    xf[2 * i + 1] = p.y;
                }
#pragma unroll
                for (int r = 0; r < kTokRows; ++r) {
                    const uint32_t uw[4] = {u[r].x, u[r].y, u[r].z, u[r].w};
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const float2 p = unpack16(uw[i], F16);
#pragma unroll
                        for (int c = 0; c < N; ++c) {
                            acc[r][c] = fmaf(p.x, xf[(2 * i) * N + c], acc[r][c]);
                            acc[r][c] = fmaf(p.y, xf[(2 * i + 1) * N + c], acc[r][c]);
                        }
                    }
                }
            }
        } else {
#pragma unroll 8
            for (uint32_t t = part * 32 + lane; t < (uint32_t)a.k; t += a.wpr * 32) {   // t may pass 2^31 on its last step
                float xf[N];
#pragma unroll
                for (int c = 0; c < N; ++c) xf[c] = load1(a.x, (int64_t)t * a.ldx + c, dtype);
#pragma unroll
                for (int r = 0; r < kTokRows; ++r) {
                    const float p = load1(w[r], t, dtype);
#pragma unroll
                    for (int c = 0; c < N; ++c) acc[r][c] = fmaf(p, xf[c], acc[r][c]);
                }
            }
        }
    }
#pragma unroll
    for (int r = 0; r < kTokRows; ++r)
#pragma unroll
        for (int c = 0; c < N; ++c)
#pragma unroll
            for (int o = 16; o; o >>= 1) acc[r][c] += __shfl_xor_sync(0xffffffffu, acc[r][c], o);
    if (lane == 0) {
#pragma unroll
        for (int r = 0; r < kTokRows; ++r)
#pragma unroll
            for (int c = 0; c < N; ++c) s_part[warp][r * N + c] = acc[r][c];
    }
    __syncthreads();
    if (part == 0 && lane < kTokRows * N) {
        const int row = row0 + lane / N, c = lane % N;
        if (row < a.m) {
            float v = 0.f;
            for (int p = 0; p < a.wpr; ++p) v += s_part[warp + p][lane];
            if (a.bias != nullptr) v += a.bias[row];
            if (a.z.p != nullptr) store1(a.z.p, (int64_t)row * a.z.ld + c, v, a.z.dtype);
            v = act_value(v, a.act);
            if (a.res.p != nullptr) v += load1(a.res.p, (int64_t)row * a.res.ld + c, a.res.dtype);
            store1(a.y.p, (int64_t)row * a.y.ld + c, v, a.y.dtype);
        }
    }
}

template <int N, bool VEC>
static void launch_tokens(const TokenArgs &a, bool f16, unsigned grid, cudaStream_t s) {
    if (f16)
        launch_pdl(dense_tokens_kernel<N, VEC, true>, dim3(grid), dim3(kTokWarps * 32), 0, s, a);
    else
        launch_pdl(dense_tokens_kernel<N, VEC, false>, dim3(grid), dim3(kTokWarps * 32), 0, s, a);
}

int dense_tokens(TokenArgs a, int n, bool f16, bool vec, cudaStream_t s) {
    // As many warps as the GPU holds at once where the rows do not give them: up to eight share two rows, as long as
    // each keeps a few steps of K (one token of 4096 x 4096: 7.6 us at 54 warps an SM, 8.3 at 27). A second wave costs
    // more than its warps bring (three tokens: 10.3 against 9.2 us).
    const int64_t pairs = ceil_div<int64_t>(a.m, kTokRows), held = (int64_t)num_sms() * tok_blocks(n) * kTokWarps;
    a.wpr = 1;
    while (a.wpr < kTokWarps && pairs * a.wpr * 2 <= held && a.k / (a.wpr * 2) >= 512) a.wpr *= 2;
    const unsigned grid = (unsigned)ceil_div<int64_t>(pairs, kTokWarps / a.wpr);
    switch (n) {
        case 1: vec ? launch_tokens<1, true>(a, f16, grid, s) : launch_tokens<1, false>(a, f16, grid, s); break;
        case 2: vec ? launch_tokens<2, true>(a, f16, grid, s) : launch_tokens<2, false>(a, f16, grid, s); break;
        case 3: vec ? launch_tokens<3, true>(a, f16, grid, s) : launch_tokens<3, false>(a, f16, grid, s); break;
        default: vec ? launch_tokens<4, true>(a, f16, grid, s) : launch_tokens<4, false>(a, f16, grid, s); break;
    }
    count_launch();
    return check_launch("dense_tokens_kernel");
}

}  // namespace csrt
