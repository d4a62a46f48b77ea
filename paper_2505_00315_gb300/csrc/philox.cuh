// Random words without a state: Philox 4x32 (J. Salmon, M. Moraes, R. Dror, D. Shaw, "Parallel random
// numbers: as easy as 1, 2, 3", SC 2011), four 32-bit words from a 128-bit counter and a 64-bit key.
// Seven rounds, the least that the authors found to pass every test of BigCrush.
#pragma once

#include <cstdint>

namespace mosa {

struct Word4 {
    uint32_t w[4];
};

// (One round: the low and high words of two products, keys added up by Weyl sequences.)
__host__ __device__ __forceinline__ Word4 philox(uint32_t c0, uint32_t c1, uint32_t c2, uint32_t c3,
                                                 uint32_t k0, uint32_t k1) {
#pragma unroll
    for (int r = 0; r < 7; ++r) {
        const uint64_t a = 0xD2511F53ull * c0, b = 0xCD9E8D57ull * c2;
        c0 = (uint32_t)(b >> 32) ^ c1 ^ k0;
        c1 = (uint32_t)b;
        c2 = (uint32_t)(a >> 32) ^ c3 ^ k1;
        c3 = (uint32_t)a;
        k0 += 0x9E3779B9u;
        k1 += 0xBB67AE85u;
    }
    return Word4{{c0, c1, c2, c3}};
}

// What a call's dropout needs: the state on the device, and the least word that is kept.
struct Drop {
    const int64_t *rng;     // null: nothing is dropped
    int32_t site;
    uint64_t least;         // round(p 2^32), 2^32 with p = 1
    float scale;            // 1 / (1 - p), 0 with p = 1
};

struct DropKey {
    uint32_t k0, k1, o0, o1;
};

__device__ __forceinline__ DropKey drop_key(const Drop &d) {
    if (d.rng == nullptr) return DropKey{0, 0, 0, 0};
    const uint64_t s = (uint64_t)d.rng[0], o = (uint64_t)d.rng[1] + (uint64_t)(int64_t)d.site;
    return DropKey{(uint32_t)s, (uint32_t)(s >> 32), (uint32_t)o, (uint32_t)(o >> 32)};
}

// Which of the columns 8 j8 .. 8 j8 + 7 of a row are kept (bit e: column 8 j8 + e).
__device__ __forceinline__ uint32_t kept8(const Drop &d, const DropKey &k, uint32_t row, uint32_t j8) {
    const Word4 a = philox(2 * j8, row, k.o0, k.o1, k.k0, k.k1);
    const Word4 b = philox(2 * j8 + 1, row, k.o0, k.o1, k.k0, k.k1);
    // (a word w is kept where w >= least, that is w > least - 1; with p = 0 every word)
    const uint32_t last = (uint32_t)(d.least - 1);
    uint32_t bits = 0;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        bits |= a.w[e] > last ? 1u << e : 0u;
        bits |= b.w[e] > last ? 16u << e : 0u;
    }
    return d.least == 0 ? 0xFFu : bits;
}

}  // namespace mosa
