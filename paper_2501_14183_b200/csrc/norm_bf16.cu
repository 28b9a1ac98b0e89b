// The norms' kernels for bf16.
#include "norm_kernels.cuh"

namespace vardrop {

// Vectors as wide as the beginnings of all rows allow: 16 bytes, 4 bytes, an element.
cudaError_t norm_launch_bf16(bool bwd, int grid, const NormParams& P, cudaStream_t s) {
    return P.C % 8 == 0 ? launch_layer<__nv_bfloat16, 8>(bwd, grid, P, s) : P.C % 2 == 0 ? launch_layer<__nv_bfloat16, 2>(bwd, grid, P, s) : launch_layer<__nv_bfloat16, 1>(bwd, grid, P, s);
}

}  // namespace vardrop
