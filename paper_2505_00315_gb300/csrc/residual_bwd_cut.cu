// The residual step's backward for sequences that lie apart; the kernel: residual_bwd.cuh.
#include "residual_bwd.cuh"

namespace mosa {
namespace blk {

cudaError_t residual_bwd_cut(const Args &p, int times, int blocks, int bytes, cudaStream_t s) {
    return times == 1 ? go_by_types<1, kWarps, true, true>(p, blocks, bytes, s)
           : times == 2 ? residual_bwd_16_cut(p, blocks, bytes, s) : go_by_types<4, kWarps / 2, true, true>(p, blocks, bytes, s);
}

}  // namespace blk
}  // namespace mosa
