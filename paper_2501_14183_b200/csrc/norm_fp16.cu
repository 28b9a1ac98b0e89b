// The norms' kernels for fp16.
#include "norm_kernels.cuh"

namespace vardrop {

// Vectors as wide as the beginnings of all rows allow: 16 bytes, 4 bytes, an element.
cudaError_t norm_launch_fp16(bool bwd, int grid, const NormParams& P, cudaStream_t s) {
    return P.C % 8 == 0 ? launch_layer<__half, 8>(bwd, grid, P, s) : P.C % 2 == 0 ? launch_layer<__half, 2>(bwd, grid, P, s) : launch_layer<__half, 1>(bwd, grid, P, s);
}

}  // namespace vardrop
