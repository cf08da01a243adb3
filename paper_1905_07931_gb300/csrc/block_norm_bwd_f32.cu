// Backward norms around a block of float32 matrices.
#include "block_norm_bwd.cuh"

namespace csrt {

int norm_bwd_f32(NormArgs &a, NormTile t, bool in, bool out, cudaStream_t s) {
    return norm_bwd_tiles<float, float>(a, t, in, out, s);
}

}  // namespace csrt
