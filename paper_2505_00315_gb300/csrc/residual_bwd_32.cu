// The residual step's backward in blocks of 8 warps, 32 columns a thread (rows of more than 4096); the kernel: residual_bwd.cuh.
#include "residual_bwd.cuh"

namespace mosa {
namespace blk {

cudaError_t residual_bwd_32(const Args &p, int blocks, int bytes, cudaStream_t s) {
    return go_by_places<4, kWarps / 2, true>(p, blocks, bytes, s);
}

}  // namespace blk
}  // namespace mosa
