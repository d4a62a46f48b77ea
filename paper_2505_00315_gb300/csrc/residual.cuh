// The residual step's shared parts: how a row lies on warps, arrives and leaves, and the arithmetic on
// eight columns (residual_fwd.cu, residual_bwd.cu).
//
// A row lies on W warps, C times eight neighbouring columns on a thread; a block has G such groups,
// each with its own rows.  Rows arrive by asynchronous copies, some ahead, in a ring of the warp's own
// in shared memory, so that no registers hold what is under way; gammas and a gate per channel
// stay in shared memory as fp32.  Values are worked on in pairs.
#pragma once

#include <algorithm>

#include "block.h"
#include "launch.h"
#include "pairs.cuh"
#include "profile.h"

namespace mosa {
namespace blk {

constexpr int kWarps = 16, kThreads = kWarps * 32, kSms = 152;
constexpr int kIn = 5;              // tensors that may arrive: x, y, dx_out, dh, a gate per token
constexpr int kMaxStages = 4;
constexpr int kSmem = 227 * 1024;   // what a block may have
constexpr int kScratch = 1024;      // bytes of a warp: 256 columns on their way out

struct Args {
    Residual r;
    float *partial;     // backward: [blocks][3][d] sums over tokens, of gamma_post, gamma_pre, gate
    int warps, groups;  // W, G
    int most;           // warps of a block at most: 16, or 8 where each has 256 registers a thread
    int stages, stage_bytes;
    int off[kIn];       // of each tensor within a warp's stage
    int flat;           // every tensor's rows lie one stride apart, sequences too
    int near;           // strides and jumps fit 32 bits
    int held;           // gammas and gate are in shared memory (all but the widest fp32 rows' backward)
};

// Which of the tensors are fp32: 0 or 1, or -1 where that is only known at run time.  Such kernels
// also take rows of any place, stride and number of columns (16-byte pieces arrive as they lie in memory,
// and what is read from them is shifted); those of known types take rows of whole pieces and near
// strides, and have gammas and gate in shared memory: no branch stands between their loads.
// (kHeld 0: gammas and gate are not there, and are read where they lie.)
template <int kX, int kY, int kDh, int kStorage, int kHeld_ = 1>
struct Types {
    static constexpr bool kFast = kX >= 0, kHeld = kFast && kHeld_;   // kHeld: known to be held
    static constexpr bool kLies = kFast && !kHeld_;                   // known not to be
    static constexpr int x = kX, y = kY, dh = kDh, storage = kStorage;
};
__device__ __forceinline__ int wide_of(int known, const Rows &m) { return known < 0 ? m.wide : known; }
// Bytes of a warp's columns of a tensor.
__host__ __device__ constexpr int bytes_of(int wide, int times) { return times * (wide ? 1024 : 512); }

__device__ __forceinline__ uint32_t smem_at(const void *p) { return (uint32_t)__cvta_generic_to_shared(p); }

// 16 bytes on their way to shared memory.
__device__ __forceinline__ void copy16(uint32_t dst, const void *src) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}
// `bytes` of them from src, the others 0.
__device__ __forceinline__ void copy16(uint32_t dst, const void *src, int bytes) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(bytes) : "memory");
}
__device__ __forceinline__ void copies_end() { asm volatile("cp.async.commit_group;" ::: "memory"); }
// All but the last n rounds of copies have arrived.
__device__ __forceinline__ void copies_wait(int n) {
    if (n == 1) asm volatile("cp.async.wait_group 1;" ::: "memory");
    else if (n == 2) asm volatile("cp.async.wait_group 2;" ::: "memory");
    else if (n == 3) asm volatile("cp.async.wait_group 3;" ::: "memory");
    else asm volatile("cp.async.wait_group 0;" ::: "memory");
}

// 256 columns of a warp in shared memory: 16-byte pieces in order, those of fp32 with every second run
// of eight swapped in pairs, so that lanes that read two neighbouring pieces each meet no bank twice.
__device__ __forceinline__ int piece_at(int j) { return 16 * (j ^ ((j >> 3) & 1)); }

// Eight values in pairs.
struct Oct {
    Pair v[4];
};

#define MOSA_OCT _Pragma("unroll") for (int e = 0; e < 4; ++e)

__device__ __forceinline__ Oct times(const Oct &a, const Oct &b) {
    Oct r;
    MOSA_OCT r.v[e] = mul2(a.v[e], b.v[e]);
    return r;
}
__device__ __forceinline__ Oct times(const Oct &a, float b) {
    Oct r;
    const Pair k = both(b);
    MOSA_OCT r.v[e] = mul2(a.v[e], k);
    return r;
}
// a b + c
__device__ __forceinline__ Oct fused(const Oct &a, const Oct &b, const Oct &c) {
    Oct r;
    MOSA_OCT r.v[e] = fma2(a.v[e], b.v[e], c.v[e]);
    return r;
}
__device__ __forceinline__ Oct fused(const Oct &a, float b, const Oct &c) {
    Oct r;
    const Pair k = both(b);
    MOSA_OCT r.v[e] = fma2(a.v[e], k, c.v[e]);
    return r;
}
__device__ __forceinline__ Oct plus(const Oct &a, const Oct &b) {
    Oct r;
    MOSA_OCT r.v[e] = add2(a.v[e], b.v[e]);
    return r;
}
__device__ __forceinline__ void add_products(Pair &s, const Oct &a, const Oct &b) {
    MOSA_OCT s = fma2(a.v[e], b.v[e], s);
}
__device__ __forceinline__ Oct zeros() {
    Oct r;
    MOSA_OCT r.v[e] = 0;
    return r;
}
__device__ __forceinline__ Oct all_of(float v) {
    Oct r;
    MOSA_OCT r.v[e] = both(v);
    return r;
}
// The values whose bit is set; 0 for the others, whatever they are.
__device__ __forceinline__ Oct chosen(const Oct &a, uint32_t bits) {
    Oct r;
    MOSA_OCT {
        const F2 f = of_two(a.v[e]);
        r.v[e] = two(bits >> (2 * e) & 1 ? f.x : 0.f, bits >> (2 * e + 1) & 1 ? f.y : 0.f);
    }
    return r;
}

__device__ __forceinline__ Oct unpacked(uint4 a) {
    Oct r;
    r.v[0] = two(low(a.x), high(a.x));
    r.v[1] = two(low(a.y), high(a.y));
    r.v[2] = two(low(a.z), high(a.z));
    r.v[3] = two(low(a.w), high(a.w));
    return r;
}

// The lane's eight columns of 256 in shared memory.
__device__ __forceinline__ Oct take(const char *from, int wide, int lane) {
    if (!wide) return unpacked(*reinterpret_cast<const uint4 *>(from + 16 * lane));
    Oct r;
    const int at = piece_at(2 * lane);   // (the other piece is the one beside it)
    const ulonglong2 a = *reinterpret_cast<const ulonglong2 *>(from + at);
    const ulonglong2 b = *reinterpret_cast<const ulonglong2 *>(from + (at ^ 16));
    r.v[0] = a.x; r.v[1] = a.y; r.v[2] = b.x; r.v[3] = b.y;
    return r;
}
// The same, c times 256 columns on, of a row whose columns begin `shift` bytes into the first piece.
__device__ __forceinline__ Oct take_shifted(const char *from, int wide, int lane, int c, int shift) {
    uint32_t w[12];
#pragma unroll
    for (int i = 0; i < 3; ++i) {
        if (i == 2 && !wide) break;
        const int j = wide ? 64 * c + 2 * lane + i : 32 * c + lane + i;
        const uint4 a = *reinterpret_cast<const uint4 *>(from + (wide ? piece_at(j) : 16 * j));
        w[4 * i] = a.x; w[4 * i + 1] = a.y; w[4 * i + 2] = a.z; w[4 * i + 3] = a.w;
    }
    const int n = wide ? 12 : 8;
    if (shift & 4) {
#pragma unroll
        for (int i = 0; i < 11; ++i) w[i] = i + 1 < n ? w[i + 1] : 0u;
    }
    if (shift & 8) {
#pragma unroll
        for (int i = 0; i < 10; ++i) w[i] = i + 2 < n ? w[i + 2] : 0u;
    }
    if (!wide) {
        if (shift & 2) {
#pragma unroll
            for (int i = 0; i < 4; ++i) w[i] = __funnelshift_r(w[i], w[i + 1], 16);
        }
        return unpacked(make_uint4(w[0], w[1], w[2], w[3]));
    }
    Oct r;
    MOSA_OCT r.v[e] = two(__uint_as_float(w[2 * e]), __uint_as_float(w[2 * e + 1]));
    return r;
}
__device__ __forceinline__ void keep(char *to, int lane, const Oct &v) {   // as fp32
    *reinterpret_cast<ulonglong2 *>(to + piece_at(2 * lane)) = make_ulonglong2(v.v[0], v.v[1]);
    *reinterpret_cast<ulonglong2 *>(to + piece_at(2 * lane + 1)) = make_ulonglong2(v.v[2], v.v[3]);
}

// What put does where a row has no 16-byte pieces or ends within the 256 columns.
__device__ __forceinline__ void put_values(int wide, char *row, int col, int d, const char *scratch, int lane) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int e = 32 * i + lane;
        if (col + e >= d) continue;
        if (wide)
            reinterpret_cast<float *>(row)[col + e] = *reinterpret_cast<const float *>(scratch + piece_at(e >> 2) + 4 * (e & 3));
        else
            reinterpret_cast<unsigned short *>(row)[col + e] = *reinterpret_cast<const unsigned short *>(scratch + 2 * e);
    }
}

// The warp's 256 columns from `col` on to a row, through its scratch where lanes' own eight columns
// are not the pieces that leave together.  kDirect: fp32 columns without it, 32 bytes a lane, which pays where they are
// one of several outputs (the backward beside a bf16 dy, B2 T8192 d4096: 251 -> 239 us), not where all are fp32 (16384
// rows of 2048: 127 -> 142).
template <bool kVec, int kWide, bool kDirect = false>
__device__ __forceinline__ void put(const Rows &m, char *row, int col, int d, char *scratch, int lane, const Oct &v) {
    if (!wide_of(kWide, m)) {
        const F2 a = of_two(v.v[0]), b = of_two(v.v[1]), c = of_two(v.v[2]), e = of_two(v.v[3]);
        const uint4 w = make_uint4(pack2(a.x, a.y), pack2(b.x, b.y), pack2(c.x, c.y), pack2(e.x, e.y));
        if (kVec || m.vec) {
            if (col + 8 * lane < d) *reinterpret_cast<uint4 *>(row + 2 * (col + 8 * lane)) = w;
            return;
        }
        __syncwarp();
        *reinterpret_cast<uint4 *>(scratch + 16 * lane) = w;
    } else {
        if (kDirect && (kVec || m.vec)) {
            if (col + 8 * lane < d) {
                ulonglong2 *q = reinterpret_cast<ulonglong2 *>(row + 4 * (col + 8 * lane));
                q[0] = make_ulonglong2(v.v[0], v.v[1]);
                q[1] = make_ulonglong2(v.v[2], v.v[3]);
            }
            return;
        }
        __syncwarp();
        keep(scratch, lane, v);
        if (kVec || m.vec) {
            __syncwarp();
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const int j = lane + 32 * i;
                if (col + 4 * j < d)
                    *reinterpret_cast<float4 *>(row + 4 * (col + 4 * j)) = *reinterpret_cast<const float4 *>(scratch + piece_at(j));
            }
            return;
        }
    }
    if constexpr (!kVec) {
        __syncwarp();
        put_values(m.wide, row, col, d, scratch, lane);
    }
}

// Eight values of a vector [d] from memory (1 where there is none, 0 beyond d).
__device__ __forceinline__ Oct vector8(const Vec &m, int at, int d) {
    Oct r;
    if (m.p != nullptr && m.vec && at + 8 <= d) {
        if (!m.wide) return unpacked(static_cast<const uint4 *>(m.p)[at / 8]);
        const ulonglong2 a = static_cast<const ulonglong2 *>(m.p)[at / 4], b = static_cast<const ulonglong2 *>(m.p)[at / 4 + 1];
        r.v[0] = a.x; r.v[1] = a.y; r.v[2] = b.x; r.v[3] = b.y;
        return r;
    }
    float v[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        v[e] = 0.f;
        if (at + e < d)
            v[e] = m.p == nullptr ? 1.f : m.wide ? static_cast<const float *>(m.p)[at + e]
                                                 : to_f32(static_cast<const bf16 *>(m.p)[at + e]);
    }
    MOSA_OCT r.v[e] = two(v[2 * e], v[2 * e + 1]);
    return r;
}

__device__ __forceinline__ void row_barrier(int W, int group) {
    asm volatile("bar.sync %0, %1;" ::"r"(group + 1), "r"(W * 32) : "memory");
}
// Sums over the threads of a row's W warps (16 at most), in every thread and in an order that is always the
// same.  `red` holds the warps' sums; each lane reads one of them.
__device__ __forceinline__ float row_sum(float v, float4 *red, int W, int w, int lane, int group) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    if (W == 1) return v;
    if (lane == 0) red[w].x = v;
    row_barrier(W, group);
    v = (lane & 15) < W ? red[lane & 15].x : 0.f;
#pragma unroll
    for (int o = 8; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}
// Of three values: lanes first share out which of them they add up (a quarter of the warp each).
__device__ __forceinline__ float4 row_sums(float a, float b, float c, float4 *red, int W, int w, int lane, int group) {
    const bool upper = lane & 16, odd = lane & 8;
    float u = (upper ? c : a) + __shfl_xor_sync(0xffffffffu, upper ? a : c, 16);
    float v = (upper ? 0.f : b) + __shfl_xor_sync(0xffffffffu, upper ? b : 0.f, 16);
    u = (odd ? v : u) + __shfl_xor_sync(0xffffffffu, odd ? u : v, 8);
#pragma unroll
    for (int o = 4; o > 0; o >>= 1) u += __shfl_xor_sync(0xffffffffu, u, o);
    if (W > 1) {
        const int which = lane >> 3, from = lane & 7;
        if (from == 0) reinterpret_cast<float *>(red + w)[which] = u;
        row_barrier(W, group);
        u = from < W ? reinterpret_cast<const float *>(red + from)[which] : 0.f;
        if (from + 8 < W) u += reinterpret_cast<const float *>(red + from + 8)[which];
#pragma unroll
        for (int o = 4; o > 0; o >>= 1) u += __shfl_xor_sync(0xffffffffu, u, o);
    }
    return make_float4(__shfl_sync(0xffffffffu, u, 0), __shfl_sync(0xffffffffu, u, 8), __shfl_sync(0xffffffffu, u, 16), 0.f);
}
__device__ __forceinline__ float sum_of(Pair p) {
    const F2 f = of_two(p);
    return f.x + f.y;
}

// 1 / (1 + e^-x): a power and a reciprocal of the hardware's, off by 7 2^-24 relative, and below 0 by |x| 1.3 2^-24 more
// (the exponent's rounding).
__device__ __forceinline__ float power_of(float x) { return pow2(x * -1.4426950408889634f); }   // e^-x
__device__ __forceinline__ float inverse(float x) {
    float y;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ float logistic(float x) { return inverse(1.f + power_of(x)); }
__device__ __forceinline__ Oct logistic(const Oct &x) {
    Oct r;
    MOSA_OCT {
        const F2 f = of_two(x.v[e]);
        r.v[e] = two(logistic(f.x), logistic(f.y));
    }
    return r;
}
// Its slope g (1 - g) = e / (1 + e)^2 with e = e^-|x|, in which nothing cancels: off by (12 + 1.3 |x|) 2^-24 relative, where
// g - g^2 has nothing left at x = 17.
__device__ __forceinline__ Oct logistic_slope(const Oct &x) {
    Oct r;
    MOSA_OCT {
        const F2 f = of_two(x.v[e]);
        const float p = power_of(fabsf(f.x)), q = power_of(fabsf(f.y));
        const Pair i = two(inverse(1.f + p), inverse(1.f + q));
        r.v[e] = mul2(mul2(two(p, q), i), i);
    }
    return r;
}


// What a warp knows of its place: W warps share a row.
struct Place {
    int W, warp, lane, group, w, nwarps;
    int d, col0;                  // columns of a warp: col0 on, 256 C
    char *ring, *scratch, *held;  // shared memory; held: gamma_post, gamma_pre, gate
    int ring_bytes;
    uint32_t ring32;              // the ring's shared address
    float4 *red;                  // two sets of a group's sums, taken in turn: one barrier a round
    uint32_t rows, step;
    __device__ __forceinline__ Place(const Args &p, char *smem, int C) {
        W = p.warps;
        warp = threadIdx.x >> 5;
        lane = threadIdx.x & 31;
        group = warp / W;
        w = warp - group * W;
        nwarps = W * p.groups;
        d = p.r.d;
        col0 = w * 256 * C;
        ring_bytes = p.stages * p.stage_bytes;
        ring = smem + warp * ring_bytes;
        ring32 = smem_at(ring);
        scratch = smem + nwarps * ring_bytes + warp * kScratch;
        red = reinterpret_cast<float4 *>(smem + nwarps * (ring_bytes + kScratch)) + group * 2 * W;
        held = smem + nwarps * (ring_bytes + kScratch + 2 * 16);
        rows = (uint32_t)p.r.B * (uint32_t)p.r.T;
        step = gridDim.x * p.groups;
    }
    __device__ __forceinline__ int column(int c) const { return col0 + 256 * c + 8 * lane; }   // the lane's eight
};

// Start of a row.
__device__ __forceinline__ char *row_at(const Args &p, const Rows &m, uint32_t row) {
    if (p.flat) return m.p + (uint64_t)row * (uint32_t)m.t;
    const uint32_t b = row / (uint32_t)p.r.T;
    return m.at((int)b, (int)(row - b * (uint32_t)p.r.T));
}

// With near strides: a row's start, and how many sequences end between a group's row and its next.
__device__ __forceinline__ char *near_at(const Args &p, const Rows &m, uint32_t row) {
    return m.p + (uint64_t)row * (uint32_t)m.t + (p.flat ? 0LL : (long long)(row / (uint32_t)p.r.T) * m.jump);
}
__device__ __forceinline__ int ends_between(const Args &p, const Place &l, uint32_t row) {
    return (int)((row + l.step) / (uint32_t)p.r.T - row / (uint32_t)p.r.T);
}

// One tensor's rows on their way to the ring.  Of known types: from pointers that move on from row to row, or (kCounts)
// counted from the row, which takes instructions (3% of the backward's time) but no registers: the forward with 24 or
// 32 columns a thread, which spills else (4096 fp32 rows of 8192: 112 -> 88 us).
template <int C, bool kFast, int kWide, bool kCounts = false>
struct Arrival {
    const char *next;   // this lane's place in the next row
    __device__ __forceinline__ void init(const Args &p, const Place &l, const Rows &m, uint32_t row) {
        if (kFast && !kCounts) next = near_at(p, m, row) + (kWide ? 4 * l.col0 : 2 * l.col0) + 16 * l.lane;
    }
    __device__ __forceinline__ void jump(const Rows &m, int ends) { next += (long long)ends * m.jump; }
    // To the shared address `to`.
    __device__ __forceinline__ void issue(const Args &p, const Place &l, const Rows &m, uint32_t row, uint32_t to) {
        if (kFast) {
            if (kCounts) next = near_at(p, m, row) + ((kWide ? 4 * l.col0 : 2 * l.col0) + 16 * l.lane);
            const uint32_t dst = to + (kWide ? piece_at(l.lane) : 16 * l.lane);
#pragma unroll
            for (int i = 0; i < (kWide ? 2 * C : C); ++i)
                if (l.col0 + (kWide ? 128 * i + 4 * l.lane : 256 * i + 8 * l.lane) < l.d) copy16(dst + 512 * i, next + 512 * i);
            if (!kCounts) next += (uint64_t)l.step * (uint32_t)m.t;
            return;
        }
        // The 16-byte pieces in which the columns lie (device memory is allocated in larger ones, so the bytes
        // before the first column are there to be read), up to the row's end; the others hold 0.
        const char *src = row_at(p, m, row), *end = src + (m.wide ? 4 : 2) * l.d;
        src += (m.wide ? 4 : 2) * l.col0;
        src -= reinterpret_cast<uintptr_t>(src) & 15;
        const int pieces = (m.wide ? 64 : 32) * C + (m.vec ? 0 : 1);
#pragma unroll 1
        for (int j = l.lane; j < pieces; j += 32) {
            const long long left = end - (src + 16 * j);
            copy16(to + (m.wide ? piece_at(j) : 16 * j), left > 0 ? src + 16 * j : src, (int)max(0LL, min(left, 16LL)));
        }
    }
    // How far into the first piece the warp's columns of a row begin (-1: pieces are whole).
    __device__ __forceinline__ int shift(const Args &p, const Place &l, const Rows &m, uint32_t row) const {
        if (kFast || m.vec) return -1;
        return (int)(reinterpret_cast<uintptr_t>(row_at(p, m, row) + (m.wide ? 4 : 2) * l.col0) & 15);
    }
};
// The lane's eight columns, c times 256 on, of what has arrived at `from`.
template <bool kFast>
__device__ __forceinline__ Oct arrived(const char *from, int wide, const Place &l, int c, int shift) {
    return kFast || shift < 0 ? take(from + bytes_of(wide, c), wide, l.lane) : take_shifted(from, wide, l.lane, c, shift);
}

// Rows of one tensor that leave.
template <int C, bool kFast, int kWide, bool kDirect = false, bool kCounts = false>
struct Departure {
    char *at;   // the row
    __device__ __forceinline__ void init(const Args &p, const Place &l, const Rows &m, uint32_t row) {
        if (kFast && !kCounts) at = near_at(p, m, row);
    }
    __device__ __forceinline__ void jump(const Rows &m, int ends) { at += (long long)ends * m.jump; }
    __device__ __forceinline__ void begin(const Args &p, const Rows &m, uint32_t row) {
        if (!kFast) at = row_at(p, m, row);
        else if (kCounts) at = near_at(p, m, row);
    }
    __device__ __forceinline__ void put_row(const Place &l, const Rows &m, int c, const Oct &v) {
        put<kFast, kWide, kDirect>(m, at, l.col0 + 256 * c, l.d, l.scratch, l.lane, v);
    }
    __device__ __forceinline__ void end(const Place &l, const Rows &m) {
        if (kFast && !kCounts) at += (uint64_t)l.step * (uint32_t)m.t;
    }
};

// The ring's places that no copy reaches hold 0: columns beyond d, and tensors that are not there.
__device__ __forceinline__ void clear_ring(const Place &l) {
    for (int i = l.lane; i < l.ring_bytes / 16; i += 32) reinterpret_cast<uint4 *>(l.ring)[i] = make_uint4(0, 0, 0, 0);
    __syncwarp();
}

// Eight columns of one of the vectors: 0 gamma_post, 1 gamma_pre, 2 the channels' gate times c (1 times c where there
// is none, which is not kept); the forward's 0 is the product of 0 and 2.
template <bool kForward>
__device__ __forceinline__ Oct vector_of(const Residual &r, int which, int col, float unit) {
    Oct v = vector8(which == 0 ? r.gpost : which == 1 ? r.gpre : r.gch, col, r.d);
    if (which == 1) return v;
    if (which == 0 && !kForward) return v;
    Oct k = which == 0 ? vector8(r.gch, col, r.d) : v;
    if (r.sigmoid && r.gate == MOSA_GATE_CHANNEL) k = logistic(k);
    k = times(k, unit);
    return which == 0 ? times(v, k) : k;
}

// How many vectors a block keeps.
__host__ __device__ __forceinline__ int vectors_of(const Residual &r, bool backward) {
    return backward && r.gate == MOSA_GATE_CHANNEL ? 3 : 2;
}

// All vectors to shared memory, the warps sharing the work.
template <int C, bool kForward>
__device__ __forceinline__ void hold(const Args &p, const Place &l, float unit) {
    const int n = C * l.W;   // 256 columns each
    for (int i = l.warp; i < vectors_of(p.r, !kForward) * n; i += l.nwarps) {
        const int which = i / n, k = i - which * n;
        keep(l.held + i * 1024, l.lane, vector_of<kForward>(p.r, which, k * 256 + 8 * l.lane, unit));
    }
    __syncthreads();
}
template <int C, bool kForward, class Ty>
__device__ __forceinline__ Oct vector_at(const Args &p, const Place &l, int which, int c, float unit) {
    if (Ty::kHeld || (!Ty::kLies && p.held)) return take(l.held + (which * l.W + l.w) * C * 1024 + c * 1024, 1, l.lane);
    return vector_of<kForward>(p.r, which, l.column(c), unit);
}

#undef MOSA_OCT

// Eights of columns of a thread: as many as registers hold, since what a row costs beside its values is
// shared by them, but enough warps for all SMs first.  The forward takes four (two with a gate per
// token); the backward, which keeps two sums of each column and what its second round needs, two in blocks
// of 8 warps (256 registers a thread) where a group has some rows, four (what the second round needs computed again) where a row
// is too wide for 16 warps of one, else one in blocks of 16.  us of the backward with one / two: B4 T4096 d1024 55.5 / 53.7,
// B2 T8192 d4096 267 / 251, fp32 B4 T1000 d768 21.2 / 22.5 (two in blocks of 16, which spill: 74, 537 and 29);
// 8192 rows of 8192 with two in blocks of 16 / four in blocks of 8: 211 / 168.
inline int times_of(const Residual &r, bool backward, int *most) {
    const long long rows = (long long)r.B * r.T;
    auto warps = [&](int times) { return (r.d + 256 * times - 1) / (256 * times); };
    *most = kWarps;
    if (backward) {
        // (how much of a block's threads and of their columns a row's width leaves at work)
        auto used = [&](int times, int of) {
            const int W = warps(times), G = of / W;
            return G == 0 ? 0.0 : (double)r.d / (256 * times * W) * (G * W) / of;
        };
        if (warps(1) > kWarps) {
            *most = kWarps / 2;
            return 4;
        }
        if (r.d > 256 && warps(2) <= kWarps / 2 && rows * warps(2) >= kSms * 8 * 16 && used(2, kWarps / 2) >= 0.95 * used(1, kWarps)) {
            *most = kWarps / 2;
            return 2;
        }
        return 1;
    }
    int times = r.gate == MOSA_GATE_TOKEN ? 2 : 4;
    while (times > 1 && rows * warps(times) < kSms * kWarps) times /= 2;
    while (warps(times) > kWarps) times *= 2;
    return times;
}

// Sizes of a block: W warps a row, G rows, the ring's stages.
inline void shape(Args &p, bool backward, int *blocks, int *times, int *bytes) {
    Residual &r = p.r;
    const long long rows = (long long)r.B * r.T;
    Rows *all[] = {&r.x, &r.y, &r.g, &r.xo, &r.h, &r.dxo, &r.dh, &r.dx, &r.dy, &r.dg};
    if (r.dh.p == nullptr) r.dh.wide = r.storage_wide;   // (zeros stand for it, of the type that most kernels know)
    p.flat = 1;
    for (Rows *m : all) {
        if (r.d % 8 != 0) m->vec = 0;   // (a piece would reach into the next row)
        if (m->p == nullptr) continue;
        if (r.T == 1) m->t = m->b;      // (rows are the sequences)
        else if (r.B > 1 && m->b != m->t * r.T) p.flat = 0;
        if (m->t >= 1LL << 32) p.flat = 0;
    }
    p.near = p.flat;
    if (!p.flat && r.B > 1 && r.T > 1) {
        p.near = 1;
        for (Rows *m : all) {
            if (m->p == nullptr) continue;
            const long long jump = m->b - m->t * r.T;
            if (m->t >= 1LL << 32 || jump >= 1LL << 31 || jump < -(1LL << 31)) p.near = 0;
            else m->jump = (int)jump;
        }
    }
    if (r.T == 1 && !p.flat)
        for (Rows *m : all) m->t = 0;
    const int each = times_of(r, backward, &p.most);
    p.warps = (r.d + 256 * each - 1) / (256 * each);
    *times = (r.d + 256 * p.warps - 1) / (256 * p.warps);   // (no more than the width asks for)
    // (a piece more where one may be cut by a row's beginning)
    bool vec = true;
    for (const Rows *m : all) vec = vec && (m->p == nullptr || m->vec);
    const int slack = vec ? 0 : 16;
    const Rows *in[kIn] = {&r.x, &r.y, &r.dxo, &r.dh, &r.g};
    p.stage_bytes = 0;
    for (int i = 0; i < kIn; ++i) {
        // (in the backward, zeros stand for a gradient that is not there: dx_out's like x)
        const int wide = i == 2 ? r.x.wide : in[i]->wide;
        p.off[i] = p.stage_bytes;
        if (in[i]->p != nullptr || (backward && (i == 2 || i == 3))) p.stage_bytes += bytes_of(wide, *times) + slack;
    }
    // As many rows as the block has warps for, but blocks for all SMs first, and two stages at least.
    const int vectors = vectors_of(r, backward) * *times * p.warps * 1024;
    p.groups = (int)std::min<long long>(p.most / p.warps, std::max(1LL, rows / kSms));
    for (;; --p.groups) {
        const int nwarps = p.warps * p.groups, fixed = nwarps * (kScratch + 2 * 16);
        p.held = fixed + nwarps * p.stage_bytes + vectors <= kSmem;
        const int room = kSmem - fixed - (p.held ? vectors : 0);
        p.stages = std::min(kMaxStages, room / (nwarps * p.stage_bytes));
        *bytes = nwarps * p.stages * p.stage_bytes + fixed + (p.held ? vectors : 0);
        if (p.stages >= 2 || p.groups == 1) break;
    }
    if (backward && p.groups > 1) *bytes = std::max(*bytes, p.groups * 3 * p.warps * 256 * *times * 4);
    *blocks = (int)std::min<long long>((rows + p.groups - 1) / p.groups, kSms);
}

// Whether a kernel of known types takes the call's places and strides.
inline bool fast(const Args &p) {
    const Residual &r = p.r;
    bool vec = p.near;
    for (const Rows *m : {&r.x, &r.y, &r.g, &r.xo, &r.h, &r.dxo, &r.dh, &r.dx, &r.dy, &r.dg})
        vec = vec && (m->p == nullptr || m->vec);
    return vec;
}

}  // namespace blk
}  // namespace mosa
