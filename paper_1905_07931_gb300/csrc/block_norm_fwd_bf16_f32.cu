// Forward norms around a block of bfloat16 matrices, in a float32 stream.
#include "block_norm_fwd.cuh"

namespace csrt {

int norm_fwd_bf16_f32(const NormArgs &a, NormTile t, bool in, bool out, cudaStream_t s) {
    return norm_fwd_tiles<__nv_bfloat16, float>(a, t, in, out, s);
}

}  // namespace csrt
