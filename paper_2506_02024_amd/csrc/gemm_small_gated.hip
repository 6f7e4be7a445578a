// The streaming kernel with an epilogue: the product of an activated gate row and an up row.
#include "gemm_small_kernels.h"

namespace nfp {

void launch_stream_gated(int kind, const FusedSmallParams &p, const SmallConfig &c, dim3 grid, hipStream_t stream) {
    launch_stream_t<kEpiGated>(kind, p, c, grid, stream);
}

}  // namespace nfp
