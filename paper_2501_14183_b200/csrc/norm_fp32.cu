// The norms' kernels for fp32.
#include "norm_kernels.cuh"

namespace vardrop {

// Vectors of 16 bytes where every row begins on such a boundary, single elements otherwise.
cudaError_t norm_launch_fp32(bool bwd, int grid, const NormParams& P, cudaStream_t s) {
    return P.C % 4 == 0 ? launch_layer<float, 4>(bwd, grid, P, s) : launch_layer<float, 1>(bwd, grid, P, s);
}

}  // namespace vardrop
