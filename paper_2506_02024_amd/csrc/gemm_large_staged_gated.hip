// The tiled kernels with weights through LDS and an epilogue: the product of an activated gate row and an up row.
#include "gemm_large_kernels.h"

namespace nfp {

void launch_staged_gated(int kind, const FusedLargeParams &p, const LargeConfig &c, dim3 grid, hipStream_t stream) {
    launch_staged_t<kEpiGated>(kind, p, c, grid, stream);
}

}  // namespace nfp
