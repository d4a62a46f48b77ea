// The residual step's backward in blocks of 16 warps, its sums over tokens and its launch; the kernel: residual_bwd.cuh.
#include "residual_bwd.cuh"

namespace mosa {
namespace blk {
namespace {

// The sums over tokens from the blocks': 32 columns a block, 32 runs of blocks each, in a fixed order.
__global__ void __launch_bounds__(1024) residual_sums_kernel(const float *partial, int blocks, int d,
                                                             float *dgpost, float *dgpre, float *dgate) {
    asm volatile("griddepcontrol.wait;" ::: "memory");
    __shared__ float red[32][33];
    const int cc = threadIdx.x & 31, run = threadIdx.x >> 5, col = blockIdx.x * 32 + cc;
    float sum = 0.f, v[kSms / 32 + 1];   // (all loads first)
#pragma unroll
    for (int i = 0; i < kSms / 32 + 1; ++i) {
        const int b = run + 32 * i;
        v[i] = b < blocks && col < 3 * d ? partial[(long long)b * 3 * d + col] : 0.f;
    }
#pragma unroll
    for (int i = 0; i < kSms / 32 + 1; ++i) sum += v[i];
    red[run][cc] = sum;
    __syncthreads();
    if (run == 0 && col < 3 * d) {
        float t = 0.f;
        for (int u = 0; u < 32; ++u) t += red[u][cc];
        const int i = col / d;
        float *out = i == 0 ? dgpost : i == 1 ? dgpre : dgate;
        if (out != nullptr) out[col - i * d] = t;
    }
}

}  // namespace

size_t residual_workspace(const Residual &r) {
    return (size_t)std::min<long long>((long long)r.B * r.T, kSms) * 3 * r.d * sizeof(float);
}

cudaError_t launch_residual_bwd(const Residual &r, float *partial, cudaStream_t s) {
    Args p{};
    p.r = r;
    const bool sums = r.dgpost != nullptr || r.dgpre != nullptr || r.dgate != nullptr;
    p.partial = sums ? partial : nullptr;
    int blocks, times, bytes;
    shape(p, true, &blocks, &times, &bytes);
    cudaError_t e = r.dh.p == nullptr ? residual_bwd_alone(p, times, blocks, bytes, s)
                    : times == 1 ? go_by_places<1, kWarps, true>(p, blocks, bytes, s)
                    : times == 2 ? residual_bwd_16(p, blocks, bytes, s) : residual_bwd_32(p, blocks, bytes, s);
    if (e != cudaSuccess || !sums) return e;
    note_launches(1);
    return launch_pdl(residual_sums_kernel, dim3((3 * r.d + 31) / 32), dim3(1024), 0, s, (const float *)partial,
                      blocks, r.d, r.dgpost, r.dgpre, r.dgate);
}

}  // namespace blk
}  // namespace mosa
