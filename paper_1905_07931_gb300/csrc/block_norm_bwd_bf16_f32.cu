// Backward norms around a block of bfloat16 matrices, in a float32 stream.
#include "block_norm_bwd.cuh"

namespace csrt {

int norm_bwd_bf16_f32(NormArgs &a, NormTile t, bool in, bool out, cudaStream_t s) {
    return norm_bwd_tiles<__nv_bfloat16, float>(a, t, in, out, s);
}

}  // namespace csrt
