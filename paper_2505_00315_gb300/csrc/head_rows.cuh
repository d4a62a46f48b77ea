// Eight values a lane of a head's row: loads and stores, sums over the row's lanes and
// the rotation of qk_norm.cu, shared with the decoding step.
#pragma once

#include "common.cuh"

namespace mosa {
namespace win {

// The values of lane li of a row: lo .. lo+3 and hi .. hi+3, so that both values of each
// rotated pair lie on one lane: neighbours, or with halves the same places of the
// two halves of the rotated dimensions (whose number is a multiple of 8 then).
struct Part {
    int lo, hi;
    __device__ __forceinline__ Part(int li, int rotary, int halves) {
        const bool split = halves && 8 * li < rotary;
        lo = split ? 4 * li : 8 * li;
        hi = split ? 4 * li + (rotary >> 1) : 8 * li + 4;
    }
};

// Four consecutive values, in one access where VEC.
template <class T, bool VEC>
__device__ __forceinline__ void load4(const T *p, float *v) {
    if (!VEC) {
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = to_f32(p[i]);
    } else if constexpr (sizeof(T) == 4) {
        const float4 w = *reinterpret_cast<const float4 *>(p);
        v[0] = w.x; v[1] = w.y; v[2] = w.z; v[3] = w.w;
    } else {
        const uint2 w = *reinterpret_cast<const uint2 *>(p);
        v[0] = __uint_as_float(w.x << 16); v[1] = __uint_as_float(w.x & 0xFFFF0000u);
        v[2] = __uint_as_float(w.y << 16); v[3] = __uint_as_float(w.y & 0xFFFF0000u);
    }
}

// Two bf16 values of a word, rounded to nearest even (the first in the low half).
__device__ __forceinline__ uint32_t two_bf16(float a, float b) {
    uint32_t w;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(w) : "f"(b), "f"(a));
    return w;
}

template <class T, bool VEC>
__device__ __forceinline__ void store4(T *p, const float *v) {
    if (!VEC) {
#pragma unroll
        for (int i = 0; i < 4; ++i) p[i] = from_f32<T>(v[i]);
    } else if constexpr (sizeof(T) == 4) {
        *reinterpret_cast<float4 *>(p) = make_float4(v[0], v[1], v[2], v[3]);
    } else {
        *reinterpret_cast<uint2 *>(p) = make_uint2(two_bf16(v[0], v[1]), two_bf16(v[2], v[3]));
    }
}

// A lane's eight values of the row at p: one access of 16 bytes of bf16 where they are neighbours.
template <class T, bool VEC>
__device__ __forceinline__ void load8(const T *p, const Part &at, float (&v)[8]) {
    if (VEC && sizeof(T) == 2 && at.hi == at.lo + 4) {
        const uint4 w = *reinterpret_cast<const uint4 *>(p + at.lo);
        v[0] = __uint_as_float(w.x << 16); v[1] = __uint_as_float(w.x & 0xFFFF0000u);
        v[2] = __uint_as_float(w.y << 16); v[3] = __uint_as_float(w.y & 0xFFFF0000u);
        v[4] = __uint_as_float(w.z << 16); v[5] = __uint_as_float(w.z & 0xFFFF0000u);
        v[6] = __uint_as_float(w.w << 16); v[7] = __uint_as_float(w.w & 0xFFFF0000u);
        return;
    }
    load4<T, VEC>(p + at.lo, v);
    load4<T, VEC>(p + at.hi, v + 4);
}

template <class T, bool VEC>
__device__ __forceinline__ void store8(T *p, const Part &at, const float (&v)[8]) {
    if (VEC && sizeof(T) == 2 && at.hi == at.lo + 4) {
        *reinterpret_cast<uint4 *>(p + at.lo) = make_uint4(two_bf16(v[0], v[1]), two_bf16(v[2], v[3]),
                                                           two_bf16(v[4], v[5]), two_bf16(v[6], v[7]));
        return;
    }
    store4<T, VEC>(p + at.lo, v);
    store4<T, VEC>(p + at.hi, v + 4);
}

// A lane's eight values as they lie in memory, to be kept in flight (VEC rows).
template <class T>
struct Raw8 {
    uint4 w[sizeof(T) / 2];
};
template <class T, bool VEC>
__device__ __forceinline__ void load_raw(const T *p, const Part &at, Raw8<T> &r) {
    if constexpr (!VEC) {
        T v[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = p[i < 4 ? at.lo + i : at.hi + i - 4];
        if constexpr (sizeof(T) == 4) {
#pragma unroll
            for (int i = 0; i < 2; ++i)
                r.w[i] = make_uint4(__float_as_uint(v[4 * i]), __float_as_uint(v[4 * i + 1]),
                                    __float_as_uint(v[4 * i + 2]), __float_as_uint(v[4 * i + 3]));
        } else {
            uint32_t u[4];
#pragma unroll
            for (int i = 0; i < 4; ++i)
                u[i] = (uint32_t)__bfloat16_as_ushort(v[2 * i]) | (uint32_t)__bfloat16_as_ushort(v[2 * i + 1]) << 16;
            r.w[0] = make_uint4(u[0], u[1], u[2], u[3]);
        }
    } else if constexpr (sizeof(T) == 4) {
        r.w[0] = *reinterpret_cast<const uint4 *>(p + at.lo);
        r.w[1] = *reinterpret_cast<const uint4 *>(p + at.hi);
    } else if (at.hi == at.lo + 4) {
        r.w[0] = *reinterpret_cast<const uint4 *>(p + at.lo);
    } else {
        const uint2 a = *reinterpret_cast<const uint2 *>(p + at.lo), b = *reinterpret_cast<const uint2 *>(p + at.hi);
        r.w[0] = make_uint4(a.x, a.y, b.x, b.y);
    }
}
template <class T>
__device__ __forceinline__ void unpack(const Raw8<T> &r, float (&v)[8]) {
    if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            v[4 * i] = __uint_as_float(r.w[i].x);
            v[4 * i + 1] = __uint_as_float(r.w[i].y);
            v[4 * i + 2] = __uint_as_float(r.w[i].z);
            v[4 * i + 3] = __uint_as_float(r.w[i].w);
        }
    } else {
        const uint32_t u[4] = {r.w[0].x, r.w[0].y, r.w[0].z, r.w[0].w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            v[2 * i] = __uint_as_float(u[i] << 16);
            v[2 * i + 1] = __uint_as_float(u[i] & 0xFFFF0000u);
        }
    }
}

// Turns lane li's eight values by the angles of cs (dir = -1: back).
__device__ __forceinline__ void turn8(float (&v)[8], int li, int rotary, int halves, const float2 *cs,
                                      float dir) {
    if (8 * li >= rotary) return;
    const float4 a = reinterpret_cast<const float4 *>(cs)[2 * li];
    const float4 b = reinterpret_cast<const float4 *>(cs)[2 * li + 1];
    const float co[4] = {a.x, a.z, b.x, b.z}, sn[4] = {a.y * dir, a.w * dir, b.y * dir, b.w * dir};
    if (halves) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const float x0 = v[e], x1 = v[e + 4];
            v[e] = x0 * co[e] - x1 * sn[e];
            v[e + 4] = x0 * sn[e] + x1 * co[e];
        }
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (8 * li + 2 * e < rotary) {
                const float x0 = v[2 * e], x1 = v[2 * e + 1];
                v[2 * e] = x0 * co[e] - x1 * sn[e];
                v[2 * e + 1] = x0 * sn[e] + x1 * co[e];
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
