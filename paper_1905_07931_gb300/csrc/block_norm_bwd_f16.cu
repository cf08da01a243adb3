// Backward norms around a block of float16 matrices, in a stream of the same.
#include "block_norm_bwd.cuh"

namespace csrt {

int norm_bwd_f16(NormArgs &a, NormTile t, bool in, bool out, cudaStream_t s) {
    return norm_bwd_tiles<__half, __half>(a, t, in, out, s);
}

}  // namespace csrt
