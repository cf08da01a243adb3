// Forward norms around a block of float16 matrices.
#include "block_norm_fwd.cuh"

namespace csrt {

int norm_fwd_f16(const NormArgs &a, bool wide, NormTile t, bool in, bool out, cudaStream_t s) {
    return wide ? norm_fwd_tiles<__half, float>(a, t, in, out, s) : norm_fwd_tiles<__half, __half>(a, t, in, out, s);
}

}  // namespace csrt
