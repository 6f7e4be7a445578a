// The tiled kernels with an epilogue: the product of an activated gate row and an up row.
#include "gemm_large_kernels.h"

namespace nfp {

void launch_tiles_gated(int kind, const LargeParams &p, const LargeConfig &c, dim3 grid, hipStream_t stream) {
    launch_tiles_t<kEpiGated>(kind, p, c, grid, stream);
}

}  // namespace nfp
