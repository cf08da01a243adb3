// Backward norms around a block of float32 matrices.
#include "block_norm_bwd.cuh"

namespace csrt {

int norm_bwd_f32(NormArgs &a, NormTile t, cudaStream_t s) { return norm_bwd_tiles<float, float>(a, t, false, false, s); }

}  // namespace csrt
