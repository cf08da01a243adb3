// Backward norms around a block of float16 matrices.
#include "block_norm_bwd.cuh"

namespace csrt {

int norm_bwd_f16(NormArgs &a, bool wide, NormTile t, bool in, bool out, cudaStream_t s) {
    return wide ? norm_bwd_tiles<__half, float>(a, t, in, out, s) : norm_bwd_tiles<__half, __half>(a, t, in, out, s);
}

}  // namespace csrt
