// Forward norms around a block of float16 matrices.
#include "block_norm_fwd.cuh"

namespace csrt {

int norm_fwd_f16(const NormArgs &a, bool wide, NormTile t, cudaStream_t s) {
    return wide ? norm_fwd_tiles<__half, float>(a, t, s) : norm_fwd_tiles<__half, __half>(a, t, s);
}

}  // namespace csrt
