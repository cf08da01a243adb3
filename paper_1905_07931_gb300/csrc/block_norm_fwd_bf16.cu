// Forward norms around a block of bfloat16 matrices.
#include "block_norm_fwd.cuh"

namespace csrt {

int norm_fwd_bf16(const NormArgs &a, bool wide, NormTile t, bool in, bool out, cudaStream_t s) {
    return wide ? norm_fwd_tiles<__nv_bfloat16, float>(a, t, in, out, s) : norm_fwd_tiles<__nv_bfloat16, __nv_bfloat16>(a, t, in, out, s);
}

}  // namespace csrt
