// Forward norms around a block of float16 matrices, in a float32 stream.
#include "block_norm_fwd.cuh"

namespace csrt {

int norm_fwd_f16_f32(const NormArgs &a, NormTile t, bool in, bool out, cudaStream_t s) {
    return norm_fwd_tiles<__half, float>(a, t, in, out, s);
}

}  // namespace csrt
