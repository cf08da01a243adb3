// Instances of gemm16_kernel for the dense layer's forward product (16-bit and float32 outputs).
#include "gemm16_host.cuh"

namespace csrt {

int dense_gemm_fwd(const GProduct &p, const GArgs &a, bool wide, cudaStream_t s) {
    return wide ? launch_gemm16<kEpiFwd, true>(p, a, s) : launch_gemm16<kEpiFwd, false>(p, a, s);
}

}  // namespace csrt
