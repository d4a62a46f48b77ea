// The residual step's backward without a gradient of h; the kernel: residual_bwd.cuh.
#include "residual_bwd.cuh"

namespace mosa {
namespace blk {

cudaError_t residual_bwd_alone(const Args &p, int times, int blocks, int bytes, cudaStream_t s) {
    return times == 1 ? go_by_places<1, kWarps, false>(p, blocks, bytes, s)
           : times == 2 ? go_by_places<2, kWarps / 2, false>(p, blocks, bytes, s)
                        : go_by_places<4, kWarps / 2, false>(p, blocks, bytes, s);
}

}  // namespace blk
}  // namespace mosa
