// The tiled kernels with weights through LDS and an epilogue: bias, activation and residual.
#include "gemm_large_kernels.h"

namespace nfp {

void launch_staged_full(int kind, const FusedLargeParams &p, const LargeConfig &c, dim3 grid, hipStream_t stream) {
    launch_staged_t<kEpiFull>(kind, p, c, grid, stream);
}

}  // namespace nfp
