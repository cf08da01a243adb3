// Backward norms around a block of float16 matrices, in a float32 stream.
#include "block_norm_bwd.cuh"

namespace csrt {

int norm_bwd_f16_f32(NormArgs &a, NormTile t, bool in, bool out, cudaStream_t s) {
    return norm_bwd_tiles<__half, float>(a, t, in, out, s);
}

}  // namespace csrt
