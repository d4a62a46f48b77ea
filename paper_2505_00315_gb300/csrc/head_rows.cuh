// Some values a lane of a head's row: loads and stores, sums over the row's lanes and
// the rotation of qk_norm.cu, shared with the decoding step.
#pragma once

#include "common.cuh"

namespace mosa {
namespace win {

// The W values of lane li of a row: lo .. lo+W/2-1 and hi .. hi+W/2-1, so that both values of
// each rotated pair lie on one lane: neighbours, or with halves the same places of the
// two halves of the rotated dimensions (whose number is a multiple of W then).
template <int W>
struct Part {
    int lo, hi;
    __device__ __forceinline__ Part(int li, int rotary, int halves) {
        const bool split = halves && W * li < rotary;
        lo = split ? W / 2 * li : W * li;
        hi = split ? W / 2 * li + (rotary >> 1) : W * li + W / 2;
    }
    __device__ __forceinline__ int at(int e) const { return e < W / 2 ? lo + e : hi + e - W / 2; }
};

// Two bf16 values of a word, rounded to nearest even (the first in the low half).
__device__ __forceinline__ uint32_t two_bf16(float a, float b) {
    uint32_t w;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(w) : "f"(b), "f"(a));
    return w;
}

// A lane's values as they lie in memory, to be kept in flight.
template <class T, int W>
struct Raw {
    uint32_t w[W * sizeof(T) / 4];
};

// N words from or to p, in the widest pieces that its alignment (VEC: 16 bytes of W/2 values) allows.
template <int N>
__device__ __forceinline__ void words_in(const void *p, uint32_t *w) {
    if constexpr (N == 2) {
        const uint2 x = *static_cast<const uint2 *>(p);
        w[0] = x.x; w[1] = x.y;
    } else {
#pragma unroll
        for (int i = 0; i < N; i += 4) {
            const uint4 x = static_cast<const uint4 *>(p)[i / 4];
            w[i] = x.x; w[i + 1] = x.y; w[i + 2] = x.z; w[i + 3] = x.w;
        }
    }
}
template <int N>
__device__ __forceinline__ void words_out(void *p, const uint32_t *w) {
    if constexpr (N == 2) {
        *static_cast<uint2 *>(p) = make_uint2(w[0], w[1]);
    } else {
#pragma unroll
        for (int i = 0; i < N; i += 4) static_cast<uint4 *>(p)[i / 4] = make_uint4(w[i], w[i + 1], w[i + 2], w[i + 3]);
    }
}

template <class T, bool VEC, int W>
__device__ __forceinline__ void load_raw(const T *p, const Part<W> &at, Raw<T, W> &r) {
    constexpr int H = W * (int)sizeof(T) / 8;   // words of half of them
    if constexpr (!VEC) {
        T v[W];
#pragma unroll
        for (int i = 0; i < W; ++i) v[i] = p[at.at(i)];
#pragma unroll
        for (int i = 0; i < 2 * H; ++i) {
            if constexpr (sizeof(T) == 4)
                r.w[i] = __float_as_uint(v[i]);
            else
                r.w[i] = (uint32_t)__bfloat16_as_ushort(v[2 * i]) | (uint32_t)__bfloat16_as_ushort(v[2 * i + 1]) << 16;
        }
    } else if (H < 4 && at.hi == at.lo + W / 2) {   // 16 bytes of neighbours
        words_in<2 * H>(p + at.lo, r.w);
    } else {
        words_in<H>(p + at.lo, r.w);
        words_in<H>(p + at.hi, r.w + H);
    }
}

template <class T, int W>
__device__ __forceinline__ void unpack(const Raw<T, W> &r, float (&v)[W]) {
#pragma unroll
    for (int i = 0; i < W * (int)sizeof(T) / 4; ++i) {
        if constexpr (sizeof(T) == 4) {
            v[i] = __uint_as_float(r.w[i]);
        } else {
            v[2 * i] = __uint_as_float(r.w[i] << 16);
            v[2 * i + 1] = __uint_as_float(r.w[i] & 0xFFFF0000u);
        }
    }
}

template <class T, bool VEC, int W>
__device__ __forceinline__ void load_part(const T *p, const Part<W> &at, float (&v)[W]) {
    Raw<T, W> r;
    load_raw<T, VEC, W>(p, at, r);
    unpack<T, W>(r, v);
}

template <class T, bool VEC, int W>
__device__ __forceinline__ void store_part(T *p, const Part<W> &at, const float (&v)[W]) {
    constexpr int H = W * (int)sizeof(T) / 8;
    if constexpr (!VEC) {
#pragma unroll
        for (int i = 0; i < W; ++i) p[at.at(i)] = from_f32<T>(v[i]);
        return;
    }
    uint32_t w[2 * H];
#pragma unroll
    for (int i = 0; i < 2 * H; ++i) {
        if constexpr (sizeof(T) == 4) w[i] = __float_as_uint(v[i]);
        else w[i] = two_bf16(v[2 * i], v[2 * i + 1]);
    }
    if (H < 4 && at.hi == at.lo + W / 2) {
        words_out<2 * H>(p + at.lo, w);
    } else {
        words_out<H>(p + at.lo, w);
        words_out<H>(p + at.hi, w + H);
    }
}

// Where the (cos, sin) of pair a of a row on LG lanes lies: two pairs of a lane together, the lanes
// side by side, so that 16-byte reads of neighbouring lanes meet no bank twice.
template <int W, int LG>
__device__ __forceinline__ int angle_at(int a) {
    const int li = a / (W / 2), e = a % (W / 2);
    return 2 * ((e >> 1) * LG + li) + (e & 1);
}

// Turns lane li's values by the angles of cs (laid out by angle_at, 16-byte aligned; dir = -1: back).
template <int W, int LG>
__device__ __forceinline__ void turn(float (&v)[W], int li, int rotary, int halves, const float2 *cs, float dir) {
    if (W * li >= rotary) return;
#pragma unroll
    for (int e = 0; e < W / 2; e += 2) {
        const float4 a = reinterpret_cast<const float4 *>(cs)[(e >> 1) * LG + li];
        const float s0 = a.y * dir, s1 = a.w * dir;
        if (halves) {
            const float x0 = v[e], x1 = v[e + W / 2], y0 = v[e + 1], y1 = v[e + 1 + W / 2];
            v[e] = x0 * a.x - x1 * s0;
            v[e + W / 2] = x0 * s0 + x1 * a.x;
            v[e + 1] = y0 * a.z - y1 * s1;
            v[e + 1 + W / 2] = y0 * s1 + y1 * a.z;
        } else if (W * li + 2 * e < rotary) {
            const float x0 = v[2 * e], x1 = v[2 * e + 1];
            v[2 * e] = x0 * a.x - x1 * s0;
            v[2 * e + 1] = x0 * s0 + x1 * a.x;
            if (W * li + 2 * e + 2 < rotary) {
                const float y0 = v[2 * e + 2], y1 = v[2 * e + 3];
                v[2 * e + 2] = y0 * a.z - y1 * s1;
                v[2 * e + 3] = y0 * s1 + y1 * a.z;
            }
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
#pragma unroll
    for (int o = lanes >> 1; o > 0; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
    return x;
}

}  // namespace win
}  // namespace mosa
