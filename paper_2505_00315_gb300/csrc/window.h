// Window heads (internal): sizes and strides as the kernels take them, and the
// launchers behind the mosa_qk_* and mosa_window_* calls.
#pragma once

#include "../../include/mosa.h"
#include "common.cuh"

namespace mosa {
namespace win {

// Strides in elements of one tensor [B, T, heads, hp].
struct Str {
    long long b, t, h;
    __host__ __device__ long long at(long long ib, long long it, long long ih) const {
        return ib * b + it * t + ih * h;
    }
};

struct Attn {
    int B, Tq, Tk, H, Hkv, hp;
    bool bf16;
    int window;   // >= 1 (no limit: Tk)
    int sinks;    // <= Tk
    float scale;
    Str q, k, v, o, go, dq, dk, dv;
    __host__ __device__ int G() const { return H / Hkv; }
    // of a packed tensor [B, Tq, H, hp]
    __host__ __device__ Str packed() const { return Str{(long long)Tq * H * hp, (long long)H * hp, hp}; }
};

// Fixed-point turns per position of each rotated pair (see rope_turn).
struct Turns {
    uint64_t phi[64];
};
Turns make_turns(int rotary, double theta);

struct Norm {
    int B, T, H, Hkv, hp;
    bool bf16;
    int rotary, halves;
    float theta, eps;
    Str q, k, yq, yk, dq, dk;
};

struct Decode {
    int B, C, H, Hkv, hp;
    bool bf16;
    int window, sinks;   // window >= 1 and <= C - sinks
    int norm, rotary, halves;
    float scale, theta, eps;
    Str q, k, v, o, kc, vc;
};

constexpr int kTcTile = 128;   // queries and keys of a tile on the tensor cores

// True when every row of the tensor starts at a multiple of 16 bytes.
inline bool rows16(const void *p, const Str &s, bool bf16) {
    const long long per = bf16 ? 8 : 4;
    return (reinterpret_cast<uintptr_t>(p) & 15) == 0 && s.b % per == 0 && s.t % per == 0 &&
           s.h % per == 0;
}

// mosa_qk_norm_rope and its backward (qk_norm.cu).
size_t norm_workspace(const Norm &n);
cudaError_t launch_norm(const Norm &n, const void *q, const void *k, const void *gq, const void *gk,
                        const int32_t *pos, void *yq, void *yk, cudaStream_t s);
cudaError_t launch_norm_bwd(const Norm &n, const void *q, const void *k, const void *gq,
                            const void *gk, const int32_t *pos, const void *dyq, const void *dyk,
                            void *dq, void *dk, float *dgq, float *dgk, void *ws, cudaStream_t s);

// Attention on CUDA cores, any strides and alignment (window_simt.cu).  delta:
// [B,H,Tq] fp32 scratch.  rest (bf16 storage, or null): [B,Tq,H,hp], what O lost when it was
// rounded, as bf16, so that the backward's D = sum(dO o O) is not off by O's rounding: dP - D cancels
// where a query's weight lies on one token, as on a sink.
cudaError_t simt_window_fwd(const Attn &a, const void *q, const void *k, const void *v,
                            const int32_t *lens, void *O, float *lse, bf16 *rest, cudaStream_t s);
cudaError_t simt_window_bwd(const Attn &a, const void *q, const void *k, const void *v,
                            const int32_t *lens, const float *lse, const void *dO,
                            const float *delta, void *dq, void *dk, void *dv, float *partial,
                            cudaStream_t s);
// Bytes of the backward's `partial`, and dk and dv of the sink rows from it (window_tiles.cuh).
size_t window_bwd_bytes(const Attn &a);
cudaError_t add_sink_rows(const Attn &a, const float *partial, int extra, void *dk, void *dv,
                          cudaStream_t s);
// delta[b,h,i] = sum over the head of dO o (O + rest), in fp32.
cudaError_t window_delta(const Attn &a, const void *O, const bf16 *rest, const void *dO, float *delta,
                         cudaStream_t s);

// The same on the tensor cores (bf16, window_tc_*.cu); false, and nothing launched, where
// the tensors' places or strides do not suit.
bool tc_window_fwd(const Attn &a, const void *q, const void *k, const void *v, const int32_t *lens,
                   void *O, float *lse, bf16 *rest, uint32_t *status, cudaStream_t s, cudaError_t *err);
bool tc_window_bwd(const Attn &a, const void *q, const void *k, const void *v, const int32_t *lens,
                   const float *lse, const void *dO, const float *delta, void *dq, void *dk, void *dv,
                   float *partial, uint32_t *status, cudaStream_t s, cudaError_t *err);

size_t decode_workspace(const Decode &d);
cudaError_t launch_decode(const Decode &d, const void *q, const void *k, const void *v,
                          const void *gq, const void *gk, const int32_t *lens, void *Kc, void *Vc,
                          void *O, void *ws, cudaStream_t s);

}  // namespace win
}  // namespace mosa
