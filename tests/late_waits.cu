// The norms around a block with every wait reported as one that ran out (each is waited for to its end, as ever): one tile of
// 16-bit matrices in either direction, by TMA and by cp.async. test_gpu_block_norm.py builds it beside the library.
#define CSRT_NORM_IN_TIME false
#include "block_norm.cu"
#include "block_norm_bwd.cuh"
#include "block_norm_fwd.cuh"

namespace csrt {

typedef __nv_bfloat16 B;

int norm_fwd_bf16(const NormArgs &a, NormTile, bool in, bool out, cudaStream_t s) {
    return in && out ? norm_fwd_tile<B, B, 32, 8, 2, true, false>(a, s) : norm_fwd_tile<B, B, 32, 8, 2, false, true>(a, s);
}
int norm_bwd_bf16(NormArgs &a, NormTile, bool in, bool out, cudaStream_t s) {
    return in && out ? norm_bwd_tile<B, B, 32, 8, 2, true, false, 2>(a, s) : norm_bwd_tile<B, B, 32, 8, 2, false, true, 2>(a, s);
}

#define CSRT_NOT_HERE(fwd, bwd)                                                                                          \
    int fwd(const NormArgs &, NormTile, bool, bool, cudaStream_t) { return fail(CSRT_ERR_ARG, "16-bit matrices only"); } \
    int bwd(NormArgs &, NormTile, bool, bool, cudaStream_t) { return fail(CSRT_ERR_ARG, "16-bit matrices only"); }
CSRT_NOT_HERE(norm_fwd_bf16_f32, norm_bwd_bf16_f32)
CSRT_NOT_HERE(norm_fwd_f16, norm_bwd_f16)
CSRT_NOT_HERE(norm_fwd_f16_f32, norm_bwd_f16_f32)
CSRT_NOT_HERE(norm_fwd_f32, norm_bwd_f32)

}  // namespace csrt
