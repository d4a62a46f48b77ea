// The residual step's backward for sequences that lie apart, blocks of 8 warps, 16 columns a thread; the kernel: residual_bwd.cuh.
#include "residual_bwd.cuh"

namespace mosa {
namespace blk {

cudaError_t residual_bwd_16_cut(const Args &p, int blocks, int bytes, cudaStream_t s) {
    return go_by_types<2, kWarps / 2, true, true>(p, blocks, bytes, s);
}

}  // namespace blk
}  // namespace mosa
