// Window heads: which keys a tile of queries meets, and which queries a tile of
// keys, shared by the CUDA-core and the tensor-core kernels.
//
// Query positions p (of the Tk tokens) see tokens t <= p with p - t < window or
// t < sinks, both below the sequence's length.
#pragma once

#include "window.h"

namespace mosa {
namespace win {

__device__ __forceinline__ int seq_len(const int32_t *lens, int b, int Tk) {
    return lens == nullptr ? Tk : min(max(lens[b], 0), Tk);
}

// Key blocks of NK tokens for the queries at positions pf .. pl (pf <= pl < len), in the
// order of their tokens: blocks 0 .. far-1 hold the sinks below the window, from token 0 up,
// the others lead up to the last query's own position, the end of the last block, so
// that window + tile tokens take as few blocks as can be wherever the tile starts.
// Sinks come first because weight often lies on them: a softmax whose running
// maximum starts there seldom has to be rescaled, and their weights are powers of two then,
// which a rounding to bf16 leaves as they are.
template <int NK>
struct KeyBlocks {
    int top, near, far, slim;   // slim: sinks [0, slim) are left to the far blocks
    __device__ __forceinline__ KeyBlocks(int pf, int pl, int window, int sinks) {
        const int lo = pf >= window ? pf - window + 1 : 0;
        top = pl + 1;
        near = (top - lo + NK - 1) / NK;
        slim = min(sinks, max(top - NK * near, 0));
        far = (slim + NK - 1) / NK;
    }
    __device__ __forceinline__ int count() const { return near + far; }
    __device__ __forceinline__ bool is_far(int j) const { return j < far; }
    __device__ __forceinline__ int start(int j) const {
        return is_far(j) ? NK * j : top - NK * (far + near - j);
    }
    // Every query pf .. pl sees every key of block j.
    __device__ __forceinline__ bool whole(int j, int pf, int pl, int window) const {
        const int ks = start(j);
        if (is_far(j)) return ks + NK <= slim;
        return ks >= 0 && ks + NK - 1 <= pf && pl - ks < window;
    }
    // Whether position p (in pf .. pl) sees column c of block j, which starts at ks.
    __device__ __forceinline__ bool sees(int j, int ks, int c, int p, int window, int sinks) const {
        const int t = ks + c;
        if (is_far(j)) return t < slim;
        return t >= 0 && t <= p && (p - t < window || t < sinks);
    }
};

// A query that sees one token only has P = 1: its scores have no gradient.  Set to
// exactly zero there, where rounding would leave a remainder of dP - D.
__device__ __forceinline__ bool sees_one(int p, int window, int sinks) {
    return p == 0 || (window == 1 && sinks == 0);
}

}  // namespace win
}  // namespace mosa
