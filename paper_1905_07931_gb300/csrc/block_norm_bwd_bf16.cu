// Backward norms around a block of bfloat16 matrices, in a stream of the same.
#include "block_norm_bwd.cuh"

namespace csrt {

int norm_bwd_bf16(NormArgs &a, NormTile t, bool in, bool out, cudaStream_t s) {
    return norm_bwd_tiles<__nv_bfloat16, __nv_bfloat16>(a, t, in, out, s);
}

}  // namespace csrt
