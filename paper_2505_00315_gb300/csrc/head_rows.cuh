// Eight values a lane of a head's row: loads and stores, sums over the row's lanes and
// the rotation of qk_norm.cu, shared with the decoding step.
#pragma once

#include "common.cuh"

namespace mosa {
namespace win {

template <class T, bool VEC>
__device__ __forceinline__ void load8(const T *p, float (&v)[8]) {
    if (VEC) {
        alignas(16) T w[8];
#pragma unroll
        for (int i = 0; i < (int)(8 * sizeof(T) / 16); ++i)
            reinterpret_cast<uint4 *>(w)[i] = reinterpret_cast<const uint4 *>(p)[i];
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = to_f32(w[i]);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = to_f32(p[i]);
    }
}

template <class T, bool VEC>
__device__ __forceinline__ void store8(T *p, const float (&v)[8]) {
    if (VEC) {
        alignas(16) T w[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) w[i] = from_f32<T>(v[i]);
#pragma unroll
        for (int i = 0; i < (int)(8 * sizeof(T) / 16); ++i)
            reinterpret_cast<uint4 *>(p)[i] = reinterpret_cast<const uint4 *>(w)[i];
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) p[i] = from_f32<T>(v[i]);
    }
}

// Turns the head whose values c .. c+7 this lane holds by the angles of cs (dir =
// -1: back).  Every lane of the warp takes part.
__device__ __forceinline__ void turn8(float (&v)[8], int c, int rotary, int halves,
                                      const float2 *cs, float dir, int lane) {
    if (!halves) {
#pragma unroll
        for (int e = 0; e < 8; e += 2)
            if (c + e < rotary) {
                const float2 a = cs[(c + e) >> 1];
                const float x0 = v[e], x1 = v[e + 1], sn = a.y * dir;
                v[e] = x0 * a.x - x1 * sn;
                v[e + 1] = x0 * sn + x1 * a.x;
            }
        return;
    }
    const int half = rotary >> 1;
    if (half == 4) {   // both partners on this lane
        if (c == 0) {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float2 a = cs[e];
                const float x0 = v[e], x1 = v[e + 4], sn = a.y * dir;
                v[e] = x0 * a.x - x1 * sn;
                v[e + 4] = x0 * sn + x1 * a.x;
            }
        }
        return;
    }
    const bool low = c < half, turned = c < rotary;
    const int other = turned ? (low ? lane + (half >> 3) : lane - (half >> 3)) : lane;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const float x = __shfl_sync(0xffffffffu, v[e], other);
        if (turned) {
            const float2 a = cs[(low ? c : c - half) + e];
            v[e] = fmaf(low ? -x : x, a.y * dir, v[e] * a.x);
        }
    }
}

// (cos, sin) of the angle of t positions at phi turns (2^-64) each.
__device__ __forceinline__ float2 angle_of(uint64_t phi, int t) {
    const uint64_t turns = phi * (uint64_t)(int64_t)t;   // mod one turn
    float sn, co;
    // half turns in [-1, 1): no large angle reaches the sine
    sincospif((float)(int32_t)(turns >> 32) * 4.656612873077393e-10f, &sn, &co);
    return make_float2(co, sn);
}

// Sum over the `lanes` (a power of two) neighbouring lanes of a row.
__device__ __forceinline__ float group_sum(float x, int lanes) {
    for (int o = lanes >> 1; o > 0; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
    return x;
}

}  // namespace win
}  // namespace mosa
