// Window attention on the tensor cores: what the forward and backward kernels
// share (tensor maps over [B, T, heads, hp] tensors of any strides, bounded
// waits, TMEM loads whose values cannot be used early, bf16 packing).
#pragma once

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

// Waits for a phase; gives up (false) at once when the CTA is giving up, and after the
// usual limit, which sets the status.
__device__ __forceinline__ bool wait_or_abort(uint64_t &bar, uint32_t parity, int *abort,
                                              uint32_t *status) {
    if (*(volatile int *)abort) return false;
    if (mbar_wait(smem_u32(&bar), parity)) return true;
    atomicOr(status, kStatusTimeout);
    *(volatile int *)abort = 1;
    return false;
}

// 32 columns of this thread's TMEM lane, without waiting: the values may be used only
// after tmem_ready of the same registers.
__device__ __forceinline__ void tmem_ld32_async(uint32_t taddr, uint32_t (&r)[32]) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 "
        "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
        "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]),
          "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]),
          "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]), "=r"(r[18]),
          "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]),
          "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]),
          "=r"(r[31])
        : "r"(taddr));
}
// All earlier TMEM loads of this thread are done; ties the registers to that point.
__device__ __forceinline__ void tmem_ready(uint32_t (&r)[32]) {
    asm volatile(
        "tcgen05.wait::ld.sync.aligned;"
        : "+r"(r[0]), "+r"(r[1]), "+r"(r[2]), "+r"(r[3]), "+r"(r[4]), "+r"(r[5]), "+r"(r[6]),
          "+r"(r[7]), "+r"(r[8]), "+r"(r[9]), "+r"(r[10]), "+r"(r[11]), "+r"(r[12]), "+r"(r[13]),
          "+r"(r[14]), "+r"(r[15]), "+r"(r[16]), "+r"(r[17]), "+r"(r[18]), "+r"(r[19]),
          "+r"(r[20]), "+r"(r[21]), "+r"(r[22]), "+r"(r[23]), "+r"(r[24]), "+r"(r[25]),
          "+r"(r[26]), "+r"(r[27]), "+r"(r[28]), "+r"(r[29]), "+r"(r[30]), "+r"(r[31])
        :
        : "memory");
}
// 32 columns of raw words, without waiting (tmem_stored waits).
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

// Two values as a bf16x2 word, rounded to nearest even, a in the low half.
__device__ __forceinline__ uint32_t pack_bf16x2(float a, float b) {
    uint32_t w;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(w) : "f"(b), "f"(a));
    return w;
}

// Whether a bf16x2 word holds a NaN or an infinity.
__device__ __forceinline__ bool odd_bf16x2(uint32_t w) {
    return (w & 0x7F80u) == 0x7F80u || (w & 0x7F800000u) == 0x7F800000u;
}

// Zeroes row r of a tile of NB 64-column blocks (128-byte rows, 16 KB apart) where it
// holds a NaN or an infinity; says whether it did.
template <int NB>
__device__ __forceinline__ bool clean_row(uint8_t *(&blk)[NB], int r) {
    bool odd = false;
#pragma unroll 1
    for (int n = 0; n < NB; ++n)
#pragma unroll 1
        for (int u = 0; u < 8; ++u) {
            const uint4 w = *reinterpret_cast<const uint4 *>(blk[n] + r * 128 + u * 16);
            odd = odd || odd_bf16x2(w.x) || odd_bf16x2(w.y) || odd_bf16x2(w.z) || odd_bf16x2(w.w);
        }
    if (odd)
#pragma unroll 1
        for (int n = 0; n < NB; ++n)
#pragma unroll 1
            for (int u = 0; u < 8; ++u)
                *reinterpret_cast<uint4 *>(blk[n] + r * 128 + u * 16) = make_uint4(0, 0, 0, 0);
    return odd;
}

}  // namespace win
}  // namespace mosa
