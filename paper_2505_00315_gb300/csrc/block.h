// Block operators (internal): sizes and tensors as the kernels take them, and the launchers behind
// the mosa_residual_*, mosa_dropout and mosa_token_logprobs* calls.
#pragma once

#include "../../include/mosa.h"
#include "common.cuh"
#include "philox.cuh"

namespace mosa {
namespace blk {

// Strides in elements of a tensor [B, T, n].
struct Str {
    long long b, t, h;
};

// A tensor [B, T, n] of rows: fp32 (wide) or bf16.
struct Rows {
    char *p;               // null: not there
    long long b, t;        // strides in bytes
    int wide;
    int vec;               // every row starts at a multiple of 16 bytes
    int jump;              // residual step: bytes from a sequence's end to the next one's beginning
    __host__ __device__ char *at(int ib, int it) const { return p + ib * b + it * t; }
};

inline Rows rows_of(const void *p, const Str &s, int dtype) {
    const int wide = dtype == MOSA_F32, e = wide ? 4 : 2;
    return Rows{(char *)p, s.b * e, s.t * e, wide,
                ((uintptr_t)p % 16 == 0) && s.b * e % 16 == 0 && s.t * e % 16 == 0, 0};
}

// A vector [d]; null: not there.
struct Vec {
    const void *p;
    int wide;
    int vec;   // starts at a multiple of 16 bytes
};

struct Residual {
    int B, T, d;
    int post, pre, gate, sigmoid;
    int storage_wide;      // gammas, gate, h, dy and a gate's gradient are fp32
    float scale, eps;
    Drop drop;
    Rows x, y, g;          // inputs; g: a gate per token
    Rows xo, h;            // forward's outputs
    Rows dxo, dh;          // backward: gradients of the outputs
    Rows dx, dy, dg;       // backward's outputs
    Vec gpost, gpre, gch;  // gch: a gate per channel
    float *stats;
    float *dgate, *dgpost, *dgpre;   // sums over tokens
};

size_t residual_workspace(const Residual &r);
cudaError_t launch_residual(const Residual &r, cudaStream_t s);
cudaError_t launch_residual_bwd(const Residual &r, float *partial, cudaStream_t s);

cudaError_t launch_dropout(int B, int T, int d, const Rows &x, const Rows &y, const Drop &drop,
                           cudaStream_t s);

struct LogProb {
    int B, T, V;
    int target64, top, stats;
    float scale;
    Rows z, dz;
    const void *targets;
    float *logp, *entropy, *lse;             // forward's outputs; backward: entropy and lse are read.  stats: lse is [3][rows],
                                             // with the largest entry and the sum of powers relative to it
    int32_t *top_index;
    float *top_logp;
    const float *dlogp, *dentropy, *dlse, *dtop;   // backward
};

size_t logprob_workspace(const LogProb &l);
cudaError_t launch_logprob(const LogProb &l, void *ws, cudaStream_t s);
cudaError_t launch_logprob_bwd(const LogProb &l, cudaStream_t s);

}  // namespace blk
}  // namespace mosa
