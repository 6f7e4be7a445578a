// The tiled kernels with weights through registers and an epilogue: bias, activation and residual.
#include "gemm_large_kernels.h"

namespace nfp {

void launch_nested_full(int kind, const FusedLargeParams &p, const LargeConfig &c, dim3 grid, hipStream_t stream) {
    launch_nested_t<kEpiFull>(kind, p, c, grid, stream);
}

}  // namespace nfp
