// The streaming kernel with an epilogue: bias, activation and residual.
#include "gemm_small_kernels.h"

namespace nfp {

void launch_stream_full(int kind, const FusedSmallParams &p, const SmallConfig &c, dim3 grid, hipStream_t stream) {
    launch_stream_t<kEpiFull>(kind, p, c, grid, stream);
}

}  // namespace nfp
