// Checks of arguments that the C entry points of the window heads and of the block operators share.
#pragma once

#include <algorithm>
#include <cstdint>
#include <initializer_list>

#include "../../include/mosa.h"

namespace mosa {

// Strides with those of sizes of 1 set to 0; false where one is negative or the
// last element lies beyond 2^62.
template <class Str>
inline bool strides(const mosa_strides &s, int B, int T, int H, Str *out) {
    *out = Str{B > 1 ? s.b : 0, T > 1 ? s.t : 0, H > 1 ? s.h : 0};
    const long long lim = 1LL << 60;
    if (out->b < 0 || out->t < 0 || out->h < 0) return false;
    return out->b <= lim / B && out->t <= lim / T && out->h <= lim / H;
}

// An output may not meet itself: no two of its elements share a place.  Where each stride passes
// what the smaller ones reach, as in every layout that is some order of the dimensions, that is
// plain; else two rows less than hp apart are looked for, by the differences of their sequences
// and heads (2^20 of those at most: what has more is refused).
template <class Str>
inline bool output(const Str &s, int B, int T, int H, int hp) {
    struct Dim {
        long long stride, n;
    } d[3] = {{s.b, B}, {s.t, T}, {s.h, H}};
    std::sort(d, d + 3, [](const Dim &x, const Dim &y) { return x.stride < y.stride; });
    long long reach = hp;
    bool nested = true;
    for (const Dim &x : d) {
        if (x.n <= 1) continue;
        if (x.stride < hp) return false;
        nested = nested && x.stride >= reach;
        reach += (x.n - 1) * x.stride;
    }
    if (nested) return true;
    if ((long long)B * H > 1 << 20) return false;
    for (long long b = 0; b < B; ++b)
        for (long long h = b == 0 ? 0 : 1 - H; h < H; ++h) {
            const long long x = b * s.b + h * s.h;
            const long long t = T <= 1 ? 0 : std::min((x < 0 ? -x : x) / s.t, T - 1LL);   // tokens that lead back
            for (long long dt = t; dt <= t + 1 && dt < T; ++dt) {
                const long long apart = (x < 0 ? -x : x) - dt * s.t;
                if ((b != 0 || h != 0 || dt != 0) && apart < hp && -apart < hp) return false;
            }
        }
    return true;
}

inline bool aligned(const void *p, int dtype) {
    return (reinterpret_cast<uintptr_t>(p) & (dtype == MOSA_BF16 ? 1 : 3)) == 0;
}

// Pointers: none null, all at a multiple of the element size.
inline mosa_status check_ptrs(int dtype, std::initializer_list<const void *> ps) {
    for (const void *p : ps)
        if (p == nullptr || !aligned(p, dtype)) return MOSA_ERR_INVALID_ARG;
    return MOSA_OK;
}

inline mosa_status check_space(const void *ws, size_t bytes, size_t need) {
    return ws != nullptr && (reinterpret_cast<uintptr_t>(ws) & 255) == 0 && bytes >= need
               ? MOSA_OK : MOSA_ERR_WORKSPACE;
}

}  // namespace mosa
