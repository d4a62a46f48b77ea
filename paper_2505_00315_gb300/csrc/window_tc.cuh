// Window attention on the tensor cores: what the forward and backward kernels
// share (tensor maps over [B, T, heads, hp] tensors of any strides, bounded
// waits, TMEM loads whose values cannot be used early, bf16 packing).
#pragma once

#include <cstdlib>

#include "tc_common.cuh"
#include "tc_tiles.cuh"
#include "tmap.h"
#include "window_tiles.cuh"

namespace mosa {
namespace win {

using namespace tc;

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.69314718055994531f;

// A tensor map and which coordinates count (a stride of 0 repeats one row).
struct Map {
    CUtensorMap m;
    int h, b;
};

// Map of a bf16 tensor [B, T, heads, hp] with boxes of 64 columns by 128 tokens, columns
// past hp and tokens outside read as zeros and not written.  False where the
// strides or the base do not suit (rows16, and tokens that do not repeat).
inline bool make_map(Map *out, const void *p, const Str &s, int B, int T, int heads, int hp) {
    if (!rows16(p, s, true) || (T > 1 && s.t == 0)) return false;
    out->h = heads > 1 && s.h != 0;
    out->b = B > 1 && s.b != 0;
    const uint64_t dims[4] = {(uint64_t)hp, (uint64_t)T, out->h ? (uint64_t)heads : 1,
                              out->b ? (uint64_t)B : 1};
    const uint64_t row = (uint64_t)hp * 2;
    const uint64_t str[3] = {T > 1 ? (uint64_t)s.t * 2 : row, out->h ? (uint64_t)s.h * 2 : row,
                             out->b ? (uint64_t)s.b * 2 : row};
    const uint32_t box[4] = {64, 128, 1, 1};
    for (uint64_t x : str)
        if (x >= (1ull << 40)) return false;
    return tmap_bf16(&out->m, p, 4, dims, str, box);
}

__device__ __forceinline__ void load_box(uint32_t dst, const Map &m, uint32_t bar, int c, int t,
                                         int h, int b) {
    tma_load_4d(dst, &m.m, bar, c, t, h * m.h, b * m.b);
}
__device__ __forceinline__ void store_box(const Map &m, uint32_t src, int c, int t, int h, int b) {
    asm volatile(
        "cp.async.bulk.tensor.4d.global.shared::cta.bulk_group [%0, {%2, %3, %4, %5}], [%1];" ::"l"(&m.m),
        "r"(src), "r"(c), "r"(t), "r"(h * m.h), "r"(b * m.b)
        : "memory");
}

// The longest that a wait of the kernels lasts, in ns: kWaitLimitNs, or for tests of giving up the value of
// MOSA_TEST_WINDOW_WAIT_NS (> 0 and less than that).
static_assert(kWaitLimitNs < 1ull << 32, "32 bits");
inline uint32_t wait_limit() {
    const char *v = std::getenv("MOSA_TEST_WINDOW_WAIT_NS");
    const unsigned long long ns = v == nullptr ? 0 : std::strtoull(v, nullptr, 10);
    return (uint32_t)(ns > 0 && ns < kWaitLimitNs ? ns : kWaitLimitNs);
}

// Waits for a phase; gives up (false) when the CTA is giving up, and after the limit,
// which sets the status.  Looks at the clock on every 16th try (a shorter limit: every one), as waiting
// warps share their issue slots with those that compute: one by one the prompt of 16384 tokens took 2%
// longer.
__device__ __forceinline__ bool wait_or_abort(uint64_t &bar, uint32_t parity, int *abort, uint32_t *status,
                                              uint32_t limit_ns) {
    const uint32_t at = smem_u32(&bar);
    if (mbar_try_wait(at, parity)) return true;
    unsigned long long t0 = 0;
    for (uint32_t n = 1; !mbar_try_wait(at, parity); ++n) {
        if ((n & 15) != 0 && limit_ns == kWaitLimitNs) continue;
        if (*(volatile int *)abort) return false;
        const unsigned long long now = globaltimer();
        if (t0 == 0) t0 = now;
        if (now - t0 > limit_ns) {
            atomicOr(status, kStatusTimeout);
            *(volatile int *)abort = 1;
            return false;
        }
    }
    return true;
}

// Whether a query sees few tokens (by the shape: lengths are on the device): P and dS are then taken in two
// parts, what bf16 holds of them and what that leaves, in every product.  Where few weights add up,
// some of them are large, and their rounding shows in O, in the backward's D and, where dP - D
// cancels, in dq and dk.  Errors of dq / dk over those of a form that rounds only what it stores, T 1000, scores
// of standard deviation 3: window 2 and 1 sink 2.0 / 2.2 in one part, 1.0 / 1.0 in two; 16 and 4 1.5 / 1.8,
// 1.0 / 1.0; 64 and 4 1.3 / 1.6, 1.0 / 1.0; in one part 256 and 4 1.2 / 1.6 still, no window 1.2 / 1.5.  Times in
// one part / two, window 64: B2 T8192, 4 heads of 64, forward 20.5 / 24.8 us, backward 58 / 63; B4 T4096, 16 + 4
// heads of 128 88 / 107, 217 / 236.
inline bool few_terms(const Attn &a) { return std::min((long long)a.Tk, (long long)a.window + a.sinks) <= 128; }

// Whether the CTA is giving up, the same answer for all lanes of a warp: some may have read the word before it
// was set, and what follows is for whole warps.
__device__ __forceinline__ bool giving_up(const int *abort) {
    return __any_sync(0xffffffffu, *(const volatile int *)abort != 0);
}

// The same for the `threads` that meet at named barrier id.
__device__ __forceinline__ bool giving_up_at(int id, int threads, const int *abort) {
    uint32_t any;
    asm volatile(
        "{\n\t.reg .pred p, q;\n\t"
        "setp.ne.s32 q, %3, 0;\n\t"
        "barrier.cta.red.or.pred p, %1, %2, q;\n\t"
        "selp.u32 %0, 1, 0, p;\n\t}"
        : "=r"(any)
        : "r"(id), "r"(threads), "r"(*(const volatile int *)abort)
        : "memory");
    return any != 0;
}

// Products of whole tiles, issued by one thread.  Operand tiles are NB 64-column blocks of 128
// rows, kBlk bytes apart; their descriptors differ by constants from the first, so that a
// product costs the issuing thread a few instructions and not the dozen of a descriptor made
// anew (8 products then take longer to issue than to run).
constexpr int kBlk = 128 * 64 * 2;

// D = A B^T over 64 NB columns, both K-major.
template <int NB>
__device__ __forceinline__ void mma_scores(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc) {
#pragma unroll
    for (int c = 0; c < NB; ++c)
#pragma unroll
        for (int kk = 0; kk < 4; ++kk)
            mma_bf16(d, a + (uint32_t)(c * (kBlk >> 4) + 2 * kk), b + (uint32_t)(c * (kBlk >> 4) + 2 * kk),
                     idesc, (c > 0 || kk > 0) ? 1u : 0u);
}
// D (+)= W X: W bf16 in TMEM, 128 columns of 16 bits, 2^lg of them every 2^lg TMEM columns (a
// worker's columns start where its scores did); X 128 rows read MN-major.
template <int lg>
__device__ __forceinline__ void mma_weights(uint32_t d, uint32_t w, uint64_t x, uint32_t idesc, bool more) {
#pragma unroll
    for (int kk = 0; kk < 8; ++kk)
        mma_bf16_ts(d, w + ((16 * kk) >> lg << lg) + (((16 * kk) & ((1 << lg) - 1)) >> 1), x + 128u * kk,
                    idesc, (more || kk > 0) ? 1u : 0u);
}
__device__ __forceinline__ uint64_t k_major(const void *tile) {
    return smem_desc_sw128(smem_u32(tile), 16, 1024);
}
__device__ __forceinline__ uint64_t mn_major(const void *tile) {
    return smem_desc_sw128(smem_u32(tile), kBlk, 1024);
}

// One arrival for the whole warp, after what its lanes did before (an arrival of every lane goes
// through the barrier's word one by one).
__device__ __forceinline__ void warp_arrive(uint64_t &bar, int lane) {
    __syncwarp();
    if (lane == 0) mbar_arrive(smem_u32(&bar));
}

// 32 columns of this thread's TMEM lane.  One statement, so that no value can be used before the
// wait and none has to be moved to be tied to it.
__device__ __forceinline__ void tmem_get32(uint32_t taddr, float (&v)[32]) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 "
        "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
        "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];\n\t"
        "tcgen05.wait::ld.sync.aligned;"
        : "=f"(v[0]), "=f"(v[1]), "=f"(v[2]), "=f"(v[3]), "=f"(v[4]), "=f"(v[5]), "=f"(v[6]),
          "=f"(v[7]), "=f"(v[8]), "=f"(v[9]), "=f"(v[10]), "=f"(v[11]), "=f"(v[12]),
          "=f"(v[13]), "=f"(v[14]), "=f"(v[15]), "=f"(v[16]), "=f"(v[17]), "=f"(v[18]),
          "=f"(v[19]), "=f"(v[20]), "=f"(v[21]), "=f"(v[22]), "=f"(v[23]), "=f"(v[24]),
          "=f"(v[25]), "=f"(v[26]), "=f"(v[27]), "=f"(v[28]), "=f"(v[29]), "=f"(v[30]),
          "=f"(v[31])
        : "r"(taddr)
        : "memory");
}
// The largest of three.
__device__ __forceinline__ float max3(float a, float b, float c) {
    float d;
    asm("max.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
    return d;
}
// 16 columns of raw words, without waiting (tmem_stored waits).
__device__ __forceinline__ void tmem_st16_async(uint32_t taddr, const uint32_t (&v)[16]) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], "
        "{%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};" ::"r"(taddr),
        "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7]),
        "r"(v[8]), "r"(v[9]), "r"(v[10]), "r"(v[11]), "r"(v[12]), "r"(v[13]), "r"(v[14]), "r"(v[15])
        : "memory");
}
__device__ __forceinline__ void tmem_stored() {
    asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory");
}

// Two fp32 operations in one instruction.
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c) {
    float2 d;
    asm("fma.rn.f32x2 %0, %1, %2, %3;"
        : "=l"(reinterpret_cast<unsigned long long &>(d))
        : "l"(reinterpret_cast<unsigned long long &>(a)), "l"(reinterpret_cast<unsigned long long &>(b)),
          "l"(reinterpret_cast<unsigned long long &>(c)));
    return d;
}
__device__ __forceinline__ float2 add2(float2 a, float2 b) {
    float2 d;
    asm("add.rn.f32x2 %0, %1, %2;"
        : "=l"(reinterpret_cast<unsigned long long &>(d))
        : "l"(reinterpret_cast<unsigned long long &>(a)), "l"(reinterpret_cast<unsigned long long &>(b)));
    return d;
}
__device__ __forceinline__ float2 mul2(float2 a, float2 b) {
    float2 d;
    asm("mul.rn.f32x2 %0, %1, %2;"
        : "=l"(reinterpret_cast<unsigned long long &>(d))
        : "l"(reinterpret_cast<unsigned long long &>(a)), "l"(reinterpret_cast<unsigned long long &>(b)));
    return d;
}

// Bits lo .. hi of 32 (any of them may lie outside).
__device__ __forceinline__ uint32_t bits(int lo, int hi) {
    const uint32_t a = lo <= 0 ? ~0u : lo > 31 ? 0u : ~0u << lo;
    return hi < 0 ? 0u : hi >= 31 ? a : a & ((2u << hi) - 1u);
}
// The blocks that all of the queries pf .. pl see whole are far blocks 0 .. far_whole-1 and near blocks
// lo .. hi-1.
struct WholeBlocks {
    int far_whole, lo, hi;
    __device__ __forceinline__ WholeBlocks(const KeyBlocks<128> &kb, int pf, int pl, int window) {
        far_whole = kb.slim / 128;
        lo = kb.far;
        while (lo < kb.count() && !kb.whole(lo, pf, pl, window)) ++lo;
        hi = kb.count();
        while (hi > lo && !kb.whole(hi - 1, pf, pl, window)) --hi;
    }
    __device__ __forceinline__ bool has(int j) const { return j < far_whole || (j >= lo && j < hi); }
};
// Zeroes (or `hidden`) the values whose bit of `seen` is not set; warps whose lanes see all of
// theirs, as most of a partly seen block's do, pass by.
__device__ __forceinline__ void hide(float (&v)[32], uint32_t seen, float hidden) {
    if (__all_sync(0xffffffffu, seen == ~0u)) return;
#pragma unroll
    for (int c = 0; c < 32; ++c)
        if (((seen >> c) & 1u) == 0) v[c] = hidden;
}

// Which of the 32 columns from c0 on of key block j (start ks) position pos sees, as bits.
__device__ __forceinline__ uint32_t seen_bits(const KeyBlocks<128> &kb, int j, int ks, int c0, int pos,
                                              int window, int sinks) {
    if (kb.is_far(j)) return bits(0, kb.slim - ks - 1 - c0);
    const int low = max(-ks, 0) - c0, last = pos - ks - c0;
    return bits(max(max(pos - window + 1, 0) - ks - c0, low), last) |
           bits(low, min(sinks - ks - 1 - c0, last));
}

// Two values as a bf16x2 word, rounded to nearest even, a in the low half.
__device__ __forceinline__ uint32_t pack_bf16x2(float a, float b) {
    uint32_t w;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(w) : "f"(b), "f"(a));
    return w;
}

// 32 bytes in one store (a whole sector), or two of 16.
__device__ __forceinline__ void store32(void *p, const uint32_t (&w)[8], bool wide) {
    if (wide) {
        asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(p), "r"(w[0]), "r"(w[1]),
                     "r"(w[2]), "r"(w[3]), "r"(w[4]), "r"(w[5]), "r"(w[6]), "r"(w[7])
                     : "memory");
    } else {
        static_cast<uint4 *>(p)[0] = make_uint4(w[0], w[1], w[2], w[3]);
        static_cast<uint4 *>(p)[1] = make_uint4(w[4], w[5], w[6], w[7]);
    }
}

// Whether a bf16x2 word holds a NaN or an infinity.
__device__ __forceinline__ bool odd_bf16x2(uint32_t w) {
    return (w & 0x7F80u) == 0x7F80u || (w & 0x7F800000u) == 0x7F800000u;
}

// Zeroes row r of a tile of NB blocks where it holds a NaN or an infinity; says whether it did.
template <int NB>
__device__ __forceinline__ bool clean_row(uint8_t *tile, int r) {
    bool odd = false;
#pragma unroll 1
    for (int u = 0; u < 8 * NB; ++u) {
        const uint4 w = *reinterpret_cast<const uint4 *>(tile + (u >> 3) * kBlk + r * 128 + (u & 7) * 16);
        odd = odd || odd_bf16x2(w.x) || odd_bf16x2(w.y) || odd_bf16x2(w.z) || odd_bf16x2(w.w);
    }
    if (odd)
#pragma unroll 1
        for (int u = 0; u < 8 * NB; ++u)
            *reinterpret_cast<uint4 *>(tile + (u >> 3) * kBlk + r * 128 + (u & 7) * 16) = make_uint4(0, 0, 0, 0);
    return odd;
}

}  // namespace win
}  // namespace mosa
