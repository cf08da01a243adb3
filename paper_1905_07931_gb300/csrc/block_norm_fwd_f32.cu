// Forward norms around a block of float32 matrices.
#include "block_norm_fwd.cuh"

namespace csrt {

int norm_fwd_f32(const NormArgs &a, NormTile t, bool in, bool out, cudaStream_t s) {
    return norm_fwd_tiles<float, float>(a, t, in, out, s);
}

}  // namespace csrt
