// Backward norms around a block of bfloat16 matrices.
#include "block_norm_bwd.cuh"

namespace csrt {

int norm_bwd_bf16(NormArgs &a, bool wide, NormTile t, bool in, bool out, cudaStream_t s) {
    return wide ? norm_bwd_tiles<__nv_bfloat16, float>(a, t, in, out, s) : norm_bwd_tiles<__nv_bfloat16, __nv_bfloat16>(a, t, in, out, s);
}

}  // namespace csrt
