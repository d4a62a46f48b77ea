// Log probabilities of given tokens with entropy and top alternatives, one pass over the logits, and
// the logits' gradient, one pass more.  With a = scale z and everything in powers of two (c = scale log2 e):
//     forward   running maximum m, s = sum 2^(c (z - m)), t = sum 2^(c (z - m)) c (z - m)
//               lse = scale m + ln s,  entropy = ln s - ln 2 t / s
// (the differences first: the largest entry's power is exactly 1, so that s >= 1, t <= 0 and no rounding
// makes a log probability positive)
//     backward  b = (scale z - lse) log2 e,  dz = 2^b (A + B b) at all places, with the row's
//               A = scale (dlse - G - dentropy entropy), B = -scale ln 2 dentropy; then the few places
//               with a gradient of their own (the target and the alternatives) once more.  (scale z
//               is rounded as in lse, so that b of a row's only large entry is 0 however large it is.)
//               Where the caller keeps m and s, b = c (z - m), with 1/s and ln s in A and B: p's error does not
//               grow with |lse| then, as it does through lse, one rounded number (|lse| 2^-24).
// A warp takes a row, or 2, 4 or 8 of a block share one where rows are fewer, or some blocks, whose
// results a second kernel joins.  Rows move in 16-byte pieces wherever they start: a row is cut at the
// addresses' multiples of 16, its first and last pieces are read value by value.
// us and share of the copy rate, bf16: 16384 rows of 32768 forward 170 (93%), backward 312 (all of it; from m and s 318); 4096 rows of 50001
// forward 70 (86%), with 5 alternatives 76.5 (79%: 7.7 instructions a value, and each warp's end a chain); fp32, 1000 rows
// of 32003 with 8: 27.5 and 44 (68%, 86%); 8 rows of 131072 with 20: 8.6, two launches.
//
// Alternatives: the pass over the row only notes, for each lane, the largest values of its three best steps (32 bf16
// or 16 fp32 values a step) and that of the fourth.  A value T that the largest of `top` steps of lanes reach is
// one that `top` entries reach at least, so that the wanted ones lie in the few steps of lanes whose largest reaches it:
// those are read once more.  (Where a lane's fourth best reaches T as well, all steps of that lane are; where that is
// so for many lanes, as with equal values, the warp looks through its part of the row again.)  The best 32 entries are kept one a lane, in falling order, as 64-bit keys:
// the value's bits in an order of integers, then the index, low ones first.
#include <algorithm>
#include <cmath>

#include "block.h"
#include "launch.h"
#include "pairs.cuh"
#include "profile.h"

namespace mosa {
namespace blk {
namespace {

constexpr int kWarps = 8, kThreads = kWarps * 32, kSms = 152;
constexpr int kFewWarps = 4;                    // of a block where rows are many, and of the backward's
constexpr int kVecs = 4;                        // 16-byte pieces that a lane has under way
constexpr float kLeast = -0x1p90f;              // this and less is ruled out
constexpr float kLn2 = 0.69314718055994531f, kLog2e = 1.4426950408889634f;

// Columns of one step of a warp.
template <bool kWide>
constexpr int step_columns() { return 32 * kVecs * (kWide ? 4 : 8); }

struct Part {
    float m, s, t, pad;
};

struct Args {
    LogProb l;
    float c;            // scale log2 e
    int share;          // forward: warps of a row in a block (1, 2, 4, 8)
    int segments;       // forward: blocks of a row (share = 8)
    Part *parts;        // [rows][segments]
    unsigned long long *tops;   // [rows][segments][32]
    int units;          // backward: warps of a row
};

// The larger one; a NaN stays.
__device__ __forceinline__ float max_nan(float a, float b) {
    float y;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(y) : "f"(a), "f"(b));
    return y;
}
__device__ __forceinline__ uint32_t max2(uint32_t a, uint32_t b) {   // of bf16 pairs; a NaN gives way
    uint32_t y;
    asm("max.bf16x2 %0, %1, %2;" : "=r"(y) : "r"(a), "r"(b));
    return y;
}
__device__ __forceinline__ uint32_t max2_nan(uint32_t a, uint32_t b) {
    uint32_t y;
    asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(y) : "r"(a), "r"(b));
    return y;
}
// 16 bytes of a row: eight bf16 or four fp32 values.
struct Piece {
    uint32_t w[4];
};

// A row of values cut at multiples of 16 bytes: piece i holds the columns from first + i E on.
template <bool kWide>
struct Row {
    static constexpr int E = kWide ? 4 : 8;
    char *p;
    int V, first;   // first: 0 .. -(E - 1)
    __device__ __forceinline__ Row(char *row, int V_) : p(row), V(V_) {
        first = -(int)((reinterpret_cast<uintptr_t>(row) & 15) / (kWide ? 4 : 2));
    }
    __device__ __forceinline__ int steps() const { return (V - first + step_columns<kWide>() - 1) / step_columns<kWide>(); }
    __device__ __forceinline__ int column(int step, int u, int lane) const {
        return first + step * step_columns<kWide>() + (u * 32 + lane) * E;
    }
    // The piece from column col on; -infinity where there is no column.
    __device__ __forceinline__ void load(int col, Piece &v) const {
        if (col >= 0 && col + E <= V) {
            const uint4 x = *reinterpret_cast<const uint4 *>(p + (long long)col * (kWide ? 4 : 2));
            v.w[0] = x.x; v.w[1] = x.y; v.w[2] = x.z; v.w[3] = x.w;
            return;
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) v.w[i] = kWide ? 0xFF800000u : 0xFF80FF80u;
        if (col + E <= 0 || col >= V) return;
#pragma unroll
        for (int i = 0; i < 4; ++i) {   // (the first or the last piece of the row)
            if (kWide) {
                v.w[i] = col + i >= 0 && col + i < V ? reinterpret_cast<const uint32_t *>(p)[col + i] : 0xFF800000u;
            } else {
                const int a = col + 2 * i;
                const unsigned short *q = reinterpret_cast<const unsigned short *>(p);
                v.w[i] = (a >= 0 && a < V ? (uint32_t)q[a] : 0xFF80u) |
                         (a + 1 >= 0 && a + 1 < V ? (uint32_t)q[a + 1] : 0xFF80u) << 16;
            }
        }
    }
    // A step's pieces of this lane.
    __device__ __forceinline__ void load_step(int step, int lane, Piece (&v)[kVecs]) const {
        const int col = first + step * step_columns<kWide>();
        if (col >= 0 && col + step_columns<kWide>() <= V) {   // (most steps: no piece is cut)
            const uint4 *q = reinterpret_cast<const uint4 *>(p + (long long)col * (kWide ? 4 : 2)) + lane;
#pragma unroll
            for (int u = 0; u < kVecs; ++u) {
                const uint4 x = q[32 * u];
                v[u].w[0] = x.x; v[u].w[1] = x.y; v[u].w[2] = x.z; v[u].w[3] = x.w;
            }
            return;
        }
#pragma unroll
        for (int u = 0; u < kVecs; ++u) load(column(step, u, lane), v[u]);
    }
    __device__ __forceinline__ float value(int col) const {
        return kWide ? reinterpret_cast<const float *>(p)[col] : to_f32(reinterpret_cast<const bf16 *>(p)[col]);
    }
};

template <bool kWide>
__device__ __forceinline__ float value_of(const Piece &v, int e) {
    return kWide ? __uint_as_float(v.w[e]) : e & 1 ? high(v.w[e / 2]) : low(v.w[e / 2]);
}

// Largest value of a piece (a NaN gives way).
template <bool kWide>
__device__ __forceinline__ float largest(const Piece &v) {
    if constexpr (kWide)
        return fmaxf(fmaxf(__uint_as_float(v.w[0]), __uint_as_float(v.w[1])),
                     fmaxf(__uint_as_float(v.w[2]), __uint_as_float(v.w[3])));
    const uint32_t m = max2(max2(v.w[0], v.w[1]), max2(v.w[2], v.w[3]));
    return fmaxf(low(m), high(m));
}

template <bool kWide>
__device__ __forceinline__ float largest(const Piece (&v)[kVecs]) {
    if constexpr (kWide) {
        return fmaxf(fmaxf(largest<true>(v[0]), largest<true>(v[1])), fmaxf(largest<true>(v[2]), largest<true>(v[3])));
    } else {
        uint32_t m[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) m[i] = max2(max2(v[0].w[i], v[1].w[i]), max2(v[2].w[i], v[3].w[i]));
        m[0] = max2(max2(m[0], m[1]), max2(m[2], m[3]));
        return fmaxf(low(m[0]), high(m[0]));
    }
}

__device__ __forceinline__ int row_split(const LogProb &l, long long row, int *t) {
    const int b = (uint32_t)row / (uint32_t)l.T;
    *t = (int)((uint32_t)row - (uint32_t)b * (uint32_t)l.T);
    return b;
}

// -------------------------------------------------------------- alternatives

using Key = unsigned long long;

__device__ __forceinline__ uint32_t order_of(float v) {   // rises with v; -0 counts as 0
    const uint32_t b = __float_as_uint(v + 0.f);
    return b ^ (b >> 31 ? 0xFFFFFFFFu : 0x80000000u);
}
__device__ __forceinline__ float of_order(uint32_t o) {
    return __uint_as_float(o ^ (o >> 31 ? 0x80000000u : 0xFFFFFFFFu));
}

template <class K>
__device__ __forceinline__ K pick(K a, K b, bool larger) { return (a > b) == larger ? a : b; }

// Falling order over the lanes.
template <class K>
__device__ __forceinline__ K sorted(K k, int lane) {
#pragma unroll
    for (int n = 2; n <= 32; n *= 2)
#pragma unroll
        for (int o = n / 2; o > 0; o /= 2)
            k = pick(k, __shfl_xor_sync(0xffffffffu, k, o), ((lane & o) == 0) == ((lane & n) == 0));
    return k;
}
// The 32 largest of two lists in falling order.
template <class K>
__device__ __forceinline__ K merged(K a, K b, int lane) {
    K k = pick(a, __shfl_sync(0xffffffffu, b, 31 - lane), true);
#pragma unroll
    for (int o = 16; o > 0; o /= 2) k = pick(k, __shfl_xor_sync(0xffffffffu, k, o), (lane & o) == 0);
    return k;
}

// Puts lanes' keys (0: none; `who` has one) into the list: one at a time, or sorted and merged where they are many.
__device__ __forceinline__ Key put_in(Key list, Key k, uint32_t who, int lane) {
    if (__popc(who) > 8) return merged(list, sorted(k, lane), lane);
#pragma unroll 1
    for (; who != 0; who &= who - 1) {
        const Key one = __shfl_sync(0xffffffffu, k, __ffs(who) - 1);
        const int before = __popc(__ballot_sync(0xffffffffu, list > one));
        const Key up = __shfl_up_sync(0xffffffffu, list, 1);
        list = lane < before ? list : lane == before ? one : up;
    }
    return list;
}
__device__ __forceinline__ Key key_of(float v, int col) { return (Key)order_of(v) << 32 | (0xFFFFFFFFu - (uint32_t)col); }

// The best of a warp's part of a row, looked through once more: what reaches `bar` (low: whatever there is).
template <bool kWide>
__device__ __noinline__ Key look_again(const Row<kWide> z, int from, int to, float bar, bool low, int top) {
    constexpr int E = kWide ? 4 : 8;
    const int lane = threadIdx.x & 31;
    Key list = 0;
    bool full = false;   // the list holds `top` entries: what comes later has to be above the last of them
    Piece v[kVecs], next[kVecs];
    z.load_step(from, lane, v);
#pragma unroll 1
    for (int i = from; i < to; ++i) {
        if (i + 1 < to) z.load_step(i + 1, lane, next);
        const float here = largest<kWide>(v);
        if (__any_sync(0xffffffffu, low || (full ? here > bar : here >= bar))) {
#pragma unroll 1
            for (int u = 0; u < kVecs; ++u) {
                const Piece x = v[0];
#pragma unroll
                for (int j = 0; j + 1 < kVecs; ++j) v[j] = v[j + 1];
                const int col = z.column(i, u, lane);
                uint32_t on = 0;   // a bit for each value (the bar stays within a piece: lanes' values do not come by index)
#pragma unroll
                for (int e = 0; e < E; ++e) {
                    const float y = value_of<kWide>(x, e);
                    const bool in = col + e >= 0 && col + e < z.V;
                    on |= in && (low || (full ? y > bar : y >= bar)) ? 1u << e : 0u;
                }
#pragma unroll 1
                for (uint32_t who; (who = __ballot_sync(0xffffffffu, on != 0)) != 0;) {
                    const int e = __ffs(on) - 1;
                    float y = value_of<kWide>(x, 0);
#pragma unroll
                    for (int j = 1; j < E; ++j) y = e == j ? value_of<kWide>(x, j) : y;
                    list = put_in(list, on != 0 ? key_of(y, col + e) : 0, who, lane);
                    on &= on - 1;
                }
                const uint32_t last = (uint32_t)(__shfl_sync(0xffffffffu, list, top - 1) >> 32);
                if (last != 0) {
                    full = true;
                    low = false;
                    bar = of_order(last);
                }
            }
        }
#pragma unroll
        for (int u = 0; u < kVecs; ++u) v[u] = next[u];
    }
    return list;
}

// What a lane has seen: the largest values of its three best steps, and that of the fourth.  The lower 16 bits of each
// say which step it was, so that one minimum and maximum move both.
constexpr float kLowest = -0x1p127f;   // (less counts as this: with a step's bits no infinity becomes a NaN)
struct Peaks {
    float a, b, c, d;
};
__device__ __forceinline__ float peak_of(float v, int step) {   // (the sum: -0 counts as 0)
    return __uint_as_float((__float_as_uint(fmaxf(v, kLowest) + 0.f) & 0xFFFF0000u) | (step & 0xFFFF));
}
// The least value whose peak has the same upper half.
__device__ __forceinline__ float floor_of(float peak) {
    const uint32_t b = __float_as_uint(peak);
    return __uint_as_float((b & 0xFFFF0000u) | (b >> 31 ? 0xFFFFu : 0u));
}

// The 32 best of the lists that `share` warps (2, 4 or 8) left in shared memory.
template <class K>
__device__ __noinline__ K best_of(const K (*room)[32], int share, int lane) {
    K a = room[0][lane], b = room[1][lane];
#pragma unroll 1
    for (int i = 2; i < share; i += 2) {   // (two chains side by side)
        a = merged(a, room[i][lane], lane);
        b = merged(b, room[i + 1][lane], lane);
    }
    return merged(a, b, lane);
}

// Lanes whose steps are all read again, rather than every lane's (16384 rows of 32768, 20 alternatives: 302 us when that was
// done for any, 232; a tenth of the rows has some).
constexpr int kAgain = 8;
constexpr int kBatch = 4;   // steps read again at once (8: 88.5 us for 86.8, 4096 rows of 50001, 5 alternatives; 16: 92)

// The 32 best of a warp's part of a row, those that reach T at least (all threads of the block call it).
template <bool kWide>
__device__ __forceinline__ Key alternatives(const Row<kWide> z, const Peaks q, int from, int to, int share, int top,
                                         uint32_t (*room)[32]) {
    constexpr int E = kWide ? 4 : 8;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    uint32_t best = sorted(order_of(q.a), lane);
    // (few lanes for many entries: the others of a lane's steps count, which makes T larger)
    if (top > 8 * share) best = merged(merged(best, sorted(order_of(q.b), lane), lane), sorted(order_of(q.c), lane), lane);
    if (share > 1) {
        room[warp][lane] = best;
        __syncthreads();
        best = best_of(room + (warp & ~(share - 1)), share, lane);
    }
    const uint32_t order = __shfl_sync(0xffffffffu, best, top - 1);
    const float T = floor_of(of_order(order));
    const bool low = !(T > kLowest);
    if (from >= to) return 0;
    uint32_t again = __ballot_sync(0xffffffffu, floor_of(q.d) >= T);
    // (steps that 16 bits do not count are looked through as well)
    if (low || __popc(again) > kAgain || to - from > 65536) return look_again(z, from, to, T, low, top);
    Key list = 0;
    // The steps to be read: of each lane's three, then all those of a lane that had more, 32 at a time.
    const uint32_t once = ~again;
    uint32_t m0 = __ballot_sync(0xffffffffu, floor_of(q.a) >= T) & once, m1 = __ballot_sync(0xffffffffu, floor_of(q.b) >= T) & once;
    uint32_t m2 = __ballot_sync(0xffffffffu, floor_of(q.c) >= T) & once;
    int step0 = from + (int)(__float_as_uint(q.a) & 0xFFFF), of = -1, at = from;   // of: the lane of all steps; -1: each its own
    const int step1 = from + (int)(__float_as_uint(q.b) & 0xFFFF), step2 = from + (int)(__float_as_uint(q.c) & 0xFFFF);
#pragma unroll 1
    for (;;) {
        if ((m0 | m1 | m2) == 0) {
            if (again == 0) break;
            of = __ffs(again) - 1;
            step0 = at + lane;
            float here = __int_as_float(0xFF800000);
            if (step0 < to) {
#pragma unroll
                for (int u = 0; u < kVecs; ++u) {
                    Piece v;
                    z.load(z.column(step0, u, of), v);
                    here = fmaxf(here, largest<kWide>(v));
                }
            }
            m0 = __ballot_sync(0xffffffffu, here >= T);
            at += 32;
            if (at >= to) {
                at = from;
                again &= again - 1;
            }
        }
        // (some steps' values at once: a lane reads one of each, as many as a lane's step has)
        float v[kBatch];
        int col[kBatch];
        uint32_t hits = 0;
#pragma unroll
        for (int j = 0; j < kBatch; ++j) {
            const uint32_t m = m0 != 0 ? m0 : m1 != 0 ? m1 : m2;
            const int src = __ffs(m) - 1;
            const int step = __shfl_sync(0xffffffffu, m0 != 0 ? step0 : m1 != 0 ? step1 : step2, max(src, 0));
            if (m0 != 0) m0 &= m0 - 1;
            else if (m1 != 0) m1 &= m1 - 1;
            else m2 &= m2 - 1;
            col[j] = z.column(step, lane / E, of < 0 ? src : of) + lane % E;
            v[j] = __int_as_float(0xFF800000);
            if (src >= 0 && lane < kVecs * E && col[j] >= 0 && col[j] < z.V) v[j] = z.value(col[j]);
        }
#pragma unroll
        for (int j = 0; j < kBatch; ++j) hits |= v[j] >= T ? 1u << j : 0u;
#pragma unroll 1
        for (uint32_t who; (who = __ballot_sync(0xffffffffu, hits != 0)) != 0;) {
            const int j = __ffs(hits) - 1;
            float y = v[0];
            int at_col = col[0];
#pragma unroll
            for (int i = 1; i < kBatch; ++i) {
                y = j == i ? v[i] : y;
                at_col = j == i ? col[i] : at_col;
            }
            list = put_in(list, hits != 0 ? key_of(y, at_col) : 0, who, lane);
            hits &= hits - 1;
        }
    }
    return list;
}

// ------------------------------------------------------------------- forward

// (m, s, t) of the lanes together: every lane gets them.
__device__ __forceinline__ Part join(Part a, float c) {
    float m = a.m;
#pragma unroll
    for (int o = 16; o > 0; o /= 2) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
    // (a lane that saw nothing has the least m: its factor is 0)
    const float by = fmaxf((a.m - m) * c, -1000.f), f = pow2(by);
    a.t = f * fmaf(a.s, by, a.t);
    a.s *= f;
#pragma unroll
    for (int o = 16; o > 0; o /= 2) {
        a.s += __shfl_xor_sync(0xffffffffu, a.s, o);
        a.t += __shfl_xor_sync(0xffffffffu, a.t, o);
    }
    a.m = m;
    return a;
}

// A row's target and what the row holds there.
struct Target {
    long long at;
    float z;
};
template <bool kWide>
__device__ __forceinline__ Target target_of(const LogProb &l, long long row) {
    Target t{-1, 0.f};
    if (l.logp == nullptr) return t;
    t.at = l.target64 ? static_cast<const int64_t *>(l.targets)[row] : (long long)static_cast<const int32_t *>(l.targets)[row];
    if (t.at >= 0 && t.at < l.V) {
        int it;
        const int ib = row_split(l, row, &it);
        t.z = Row<kWide>(l.z.at(ib, it), l.V).value((int)t.at);
    }
    return t;
}

// One warp writes a row's results.
template <bool kTop>
__device__ __forceinline__ void finish(const Args &p, long long row, const Part &a, const Target &t, Key list, int lane) {
    const LogProb &l = p.l;
    const bool none = a.m <= kLeast, bad = a.m > -kLeast;
    const float lg = logf(a.s), inf = __int_as_float(0x7F800000), nan = __int_as_float(0x7FC00000);
    const float lse = bad ? nan : none && a.s == a.s ? -inf : __fadd_rn(__fmul_rn(a.m, l.scale), lg);
    if (lane == 0) {
        if (l.lse != nullptr) {
            l.lse[row] = lse;
            if (l.stats) {
                const long long rows = (long long)l.B * l.T;
                l.lse[rows + row] = a.m;
                l.lse[2 * rows + row] = a.s;
            }
        }
        if (l.entropy != nullptr)
            l.entropy[row] = bad ? nan : none && a.s == a.s ? 0.f : fmaf(-kLn2, a.t / a.s, lg);
        if (l.logp != nullptr)
            l.logp[row] = t.at < 0 ? 0.f : t.at >= l.V || lse != lse ? nan : t.z <= kLeast ? -inf : fmaf(t.z - a.m, l.scale, -lg);
    }
    if (kTop && lane < l.top) {
        const float v = of_order((uint32_t)(list >> 32));
        l.top_index[row * l.top + lane] = list == 0 ? 0 : (int32_t)(0xFFFFFFFFu - (uint32_t)list);
        l.top_logp[row * l.top + lane] = lse != lse ? nan : v <= kLeast || none ? -inf : fmaf(v - a.m, l.scale, -lg);
    }
}

// `share` warps of a block take a row together, or all of them a segment of one.
// (kOf: warps of a block)
template <bool kWide, bool kTop, int kOf>
__global__ void __launch_bounds__(kOf * 32, 32 / kOf) logprob_kernel(const __grid_constant__ Args p) {
    asm volatile("griddepcontrol.wait;" ::: "memory");
    constexpr int E = kWide ? 4 : 8;
    __shared__ uint32_t bars[kTop ? kOf : 1][32];
    __shared__ Key room[kTop ? kOf : 1][32];
    __shared__ Part part[kOf];
    __shared__ Target targets[kTop ? kOf : 1];
    const LogProb &l = p.l;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, mine = warp & (p.share - 1);
    const long long rows = (long long)l.B * l.T;
    const long long row = p.segments > 1 ? blockIdx.x / p.segments : (long long)blockIdx.x * (kOf / p.share) + warp / p.share;
    const int segment = p.segments > 1 ? (int)(blockIdx.x - row * p.segments) : 0;
    if (p.share == 1 && row >= rows) return;   // (else to the block's barriers, with nothing)
    int t;
    const int b = row_split(l, row < rows ? row : 0, &t);
    const Row<kWide> z(l.z.at(b, t), l.V);
    const int steps = row < rows ? z.steps() : 0, at = segment * p.share + mine, shares = p.segments * p.share;
    const int from = (int)((long long)steps * at / shares), to = (int)((long long)steps * (at + 1) / shares);
    Target target{-1, 0.f};
    if (mine == 0 && p.segments == 1 && row < rows) target = target_of<kWide>(l, row);

    float m = kLeast;
    Pair s = 0, sum_t = 0;   // pairs of sums
    Peaks q{kLowest, kLowest, kLowest, kLowest};
    const Pair c2 = both(p.c);
    Piece cur[kVecs];
    if (from < to) z.load_step(from, lane, cur);
    for (int i = from; i < to; ++i) {
        Piece next[kVecs];
        if (i + 1 < to) z.load_step(i + 1, lane, next);
        const float here = largest<kWide>(cur);
        if (kTop) {
            float k = peak_of(here, i - from), less;
            less = fminf(q.a, k);
            q.a = fmaxf(q.a, k);
            k = fminf(q.b, less);
            q.b = fmaxf(q.b, less);
            less = fminf(q.c, k);
            q.c = fmaxf(q.c, k);
            q.d = fmaxf(q.d, less);
        }
        if (here > m) {   // (false for a NaN)
            const float by = fmaxf((m - here) * p.c, -1000.f), f = pow2(by);
            m = here;
            sum_t = mul2(both(f), fma2(s, both(by), sum_t));
            s = mul2(both(f), s);
        }
        const Pair minus = both(-m);
#pragma unroll
        for (int u = 0; u < kVecs; ++u) {
#pragma unroll
            for (int e = 0; e < E; e += 2) {
                Pair a;
                if (kWide) {
                    a = two(max_nan(__uint_as_float(cur[u].w[e]), kLeast), max_nan(__uint_as_float(cur[u].w[e + 1]), kLeast));
                } else {
                    const uint32_t w = max2_nan(cur[u].w[e / 2], 0xEC80EC80u);   // -2^90 twice
                    a = two(low(w), high(w));
                }
                a = mul2(add2(a, minus), c2);
                const F2 x = of_two(a);
                const Pair ex = two(pow2(x.x), pow2(x.y));
                s = add2(s, ex);
                sum_t = fma2(ex, a, sum_t);
            }
        }
#pragma unroll
        for (int u = 0; u < kVecs; ++u) cur[u] = next[u];
    }
    const F2 s2 = of_two(s), t2 = of_two(sum_t);
    Part a = join(Part{m, s2.x + s2.y, t2.x + t2.y, 0.f}, p.c);
    Key list = 0;
    if (lane == 0) part[warp] = a;
    if (kTop) {   // (what is wanted after it lies in shared memory: registers that a call saves are memory traffic)
        if (lane == 0) targets[warp] = target;
        list = alternatives<kWide>(z, q, from, to, p.share, l.top, bars);
        __syncwarp();
        a = part[warp];
        target = targets[warp];
    }
    if (p.share > 1) {
        if (kTop) room[warp][lane] = list;
        __syncthreads();
        if (mine != 0 || row >= rows) return;
        if (kTop) list = best_of(room + warp, p.share, lane);
        a = join(lane < p.share ? part[warp + lane] : Part{kLeast, 0.f, 0.f, 0.f}, p.c);
        if (p.segments > 1) {
            if (lane == 0) p.parts[blockIdx.x] = a;
            if (kTop) p.tops[(long long)blockIdx.x * 32 + lane] = list;
            return;
        }
    }
    finish<kTop>(p, row, a, target, list, lane);
}

// The segments of a row together: a block a row.
template <bool kWide, bool kTop>
__global__ void __launch_bounds__(kThreads) logprob_join_kernel(const __grid_constant__ Args p) {
    asm volatile("griddepcontrol.wait;" ::: "memory");
    __shared__ Key room[kTop ? kWarps : 1][32];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const long long row = blockIdx.x, at = row * p.segments;
    Target target{-1, 0.f};
    if (warp == 0) target = target_of<kWide>(p.l, row);
    Key list = 0;
    if (kTop) {
#pragma unroll 1
        for (int i = warp; i < p.segments; i += kWarps) list = merged(list, (Key)p.tops[(at + i) * 32 + lane], lane);
        room[warp][lane] = list;
        __syncthreads();
    }
    if (warp != 0) return;
    if (kTop) list = best_of(room, kWarps, lane);
    const Part none{kLeast, 0.f, 0.f, 0.f};
    const Part a = join(lane < p.segments ? p.parts[at + lane] : none, p.c);
    finish<kTop>(p, row, a, target, list, lane);
}

// ------------------------------------------------------------------ backward

__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
    for (int o = 16; o > 0; o /= 2) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}

// A warp takes one of the `units` shares of a row.  kStats: the caller has kept m and s.
template <bool kWide, bool kStats>
__global__ void __launch_bounds__(kFewWarps * 32) logprob_bwd_kernel(const __grid_constant__ Args p) {
    asm volatile("griddepcontrol.wait;" ::: "memory");
    constexpr int E = kWide ? 4 : 8;
    const LogProb &l = p.l;
    const int lane = threadIdx.x & 31;
    const long long all = (long long)l.B * l.T * p.units, warps = (long long)gridDim.x * kFewWarps;
    for (long long unit = (long long)blockIdx.x * kFewWarps + (threadIdx.x >> 5); unit < all; unit += warps) {
        const long long row = unit / p.units;
        const int share = (int)(unit - row * p.units);
        int it;
        const int ib = row_split(l, row, &it);
        const Row<kWide> z(l.z.at(ib, it), l.V);
        char *out = l.dz.at(ib, it);
        const int steps = z.steps();
        const int from = (int)((long long)steps * share / p.units), to = (int)((long long)steps * (share + 1) / p.units);
        const int col0 = max(z.first + from * step_columns<kWide>(), 0);
        const int col1 = min(z.first + to * step_columns<kWide>(), l.V);

        Piece cur[kVecs];   // (under way while the row's gradients arrive)
        if (from < to) z.load_step(from, lane, cur);

        // The row's gradients.
        long long target = -1;
        float gt = 0.f, own = 0.f;   // of the target; of this lane's alternative
        int alt = -1;
        if (l.dlogp != nullptr) {
            target = l.target64 ? static_cast<const int64_t *>(l.targets)[row]
                                : (long long)static_cast<const int32_t *>(l.targets)[row];
            if (target >= 0 && target < l.V) gt = l.dlogp[row];
            else target = -1;
        }
        if (l.dtop != nullptr && lane < l.top) {
            alt = l.top_index[row * l.top + lane];
            if (alt < 0 || alt >= l.V) alt = -1;
            else own = l.dtop[row * l.top + lane];
        }
        const float dH = l.dentropy != nullptr ? l.dentropy[row] : 0.f;
        const float dL = l.dlse != nullptr ? l.dlse[row] : 0.f;
        const float lse = l.lse[row], inf = __int_as_float(0x7F800000);
        const bool zero = lse == -inf || (gt == 0.f && dH == 0.f && dL == 0.f && __all_sync(0xffffffffu, own == 0.f));
        float A = l.scale * (dL - (gt + warp_sum(own)));
        if (dH != 0.f) A -= l.scale * (dH * l.entropy[row]);
        float B = -l.scale * kLn2 * dH;
        if (zero) A = B = 0.f;
        float ref = zero ? 0.f : lse, off = ref;   // scale z where weights are near 1; what is taken off (stats: of z, else of scale z)
        if (kStats && !zero) {
            const long long rows = (long long)l.B * l.T;
            const float s = l.lse[2 * rows + row], by = 1.f / s;
            off = l.lse[rows + row];
            ref = off * l.scale;
            A = lse == lse ? fmaf(l.scale * dH, logf(s), A) * by : lse;   // (a row that is no number stays so)
            B *= by;
        }
        // Values that are clamped to this have weight 0, and no infinity meets it.  (Far enough below a large lse that
        // no rounding brings it back there.)
        const float least = fmaxf((ref - 208.f - fabsf(ref) * 0x1p-6f) / l.scale, kLeast);
        const uint32_t least2 = 0x10001u * (uint32_t)__bfloat16_as_ushort(__float2bfloat16_rd(least));
        const float leastw = __bfloat162float(__float2bfloat16_rd(least));

        // What the few places with a gradient of their own hold, before they are overwritten.
        const bool mine = alt >= col0 && alt < col1, here = target >= col0 && target < col1;
        const float z_alt = mine ? z.value(alt) : 0.f, z_target = here ? z.value((int)target) : 0.f;
        __syncwarp();

        auto weight = [&](float v) {   // 2^b and its gradient without the place's own
            v = max_nan(v, leastw);
            const float b = kStats ? (v - off) * p.c : __fsub_rn(__fmul_rn(v, l.scale), off) * kLog2e;
            return pow2(b) * fmaf(B, b, A);
        };
        const bool same = ((reinterpret_cast<uintptr_t>(out) ^ reinterpret_cast<uintptr_t>(z.p)) & 15) == 0;
        const Pair scale2 = both(l.scale), minus = both(-off), to2 = both(kStats ? p.c : kLog2e);
        const Pair A2 = both(A), B2 = both(B);
        for (int i = from; i < to; ++i) {
            Piece next[kVecs];
            if (i + 1 < to && !zero) z.load_step(i + 1, lane, next);
#pragma unroll
            for (int u = 0; u < kVecs; ++u) {
                uint32_t w[4] = {0u, 0u, 0u, 0u};
                if (!zero) {
#pragma unroll
                    for (int e = 0; e < E; e += 2) {
                        Pair a;
                        if (kWide) {
                            a = two(max_nan(__uint_as_float(cur[u].w[e]), leastw), max_nan(__uint_as_float(cur[u].w[e + 1]), leastw));
                        } else {
                            const uint32_t v = max2_nan(cur[u].w[e / 2], least2);
                            a = two(low(v), high(v));
                        }
                        a = mul2(add2(kStats ? a : mul2(a, scale2), minus), to2);
                        const F2 x = of_two(a);
                        const F2 g = of_two(mul2(two(pow2(x.x), pow2(x.y)), fma2(B2, a, A2)));
                        if (kWide) {
                            w[e] = __float_as_uint(g.x);
                            w[e + 1] = __float_as_uint(g.y);
                        } else {
                            w[e / 2] = pack2(g.x, g.y);
                        }
                    }
                }
                const int col = z.column(i, u, lane);
                if (same && col >= 0 && col + E <= l.V) {
                    *reinterpret_cast<uint4 *>(out + (long long)col * (kWide ? 4 : 2)) = make_uint4(w[0], w[1], w[2], w[3]);
                } else {
#pragma unroll
                    for (int e = 0; e < E; ++e) {
                        if (col + e < 0 || col + e >= l.V) continue;
                        if (kWide) reinterpret_cast<uint32_t *>(out)[col + e] = w[e];
                        else reinterpret_cast<unsigned short *>(out)[col + e] = (unsigned short)(w[e / 2] >> 16 * (e & 1));
                    }
                }
            }
#pragma unroll
            for (int u = 0; u < kVecs; ++u) cur[u] = next[u];
        }
        if (zero || !(here || __any_sync(0xffffffffu, mine))) continue;
        __syncwarp();
        auto place = [&](int col, float v, float g) {
            const float x = v <= kLeast && lse == lse ? 0.f : fmaf(l.scale, g, weight(v));   // (a row with a NaN is one)
            if (kWide) reinterpret_cast<float *>(out)[col] = x;
            else reinterpret_cast<bf16 *>(out)[col] = from_f32<bf16>(x);
        };
        // The same index twice: its gradients together, by the first lane that has it.
        float g = 0.f;
        bool leads = mine, listed = false;
        for (int j = 0; j < l.top; ++j) {
            const int other = __shfl_sync(0xffffffffu, alt, j);
            const float og = __shfl_sync(0xffffffffu, own, j);
            if (other == alt) g += og;
            if (other == alt && j < lane) leads = false;
            listed = listed || (other >= 0 && other == target);
        }
        if (mine && alt == target) g += gt;
        if (leads) place(alt, z_alt, g);
        if (here && !listed && lane == 0) place((int)target, z_target, gt);
    }
}

int steps_of(const LogProb &l) {   // (as if a row started at a multiple of 16 bytes)
    const int K = l.z.wide ? step_columns<true>() : step_columns<false>();
    return (int)(((long long)l.V + K - 1) / K);
}

// Forward: warps of a block, how many of them share a row, and how many blocks do.  What a choice costs is counted in steps of a
// warp while all SMs' warps are at work (1.6 us): a round of all of them takes a row's steps, one of a share x of them 0.41 + 0.59 x
// of that (fewer warps wait less for memory, which they leave idle), and each round its beginning and its end.
// us with 1 / 2 / 4 / 8 / 16 warps of a row (bf16; 16: two blocks and the second kernel), the choice in brackets:
//     4096 rows of 32003   [48] / 50 / 51 / 57        5 alternatives   [54] / 57 / 61 / 76
//     1000 of 32003        29 / 19 / [15] / 18 / 19                    32 / 22 / [18] / 23 / 31
//     300 of 32003         27 / 16 / 10 / [8] / 9                      30 / 18 / 12 / [11] / 14
//     300 of 131072        94 / 49 / 28 / 19 / [18]                    99 / 53 / 31 / 22 / [23]
struct Split {
    int of, share, segments;
};
Split split(const LogProb &l) {
    const long long rows = (long long)l.B * l.T, all = 32LL * kSms, steps = steps_of(l);
    const double end = l.top > 0 ? 3.2 + 0.17 * l.top : 1.6, join = l.top > 0 ? 2.8 : 1.3;
    auto cost = [&](long long warps) {   // of a row
        const long long w = rows * warps, full = w / all;
        const double x = (double)(w % all) / all, part = x > 0 ? 1 : 0;
        return (double)((steps + warps - 1) / warps) * (full + part * (0.41 + 0.59 * x)) + (full + part) * end;
    };
    Split p{kFewWarps, 1, 1};
    double best = cost(1);
    for (int share = 2; share <= kWarps && share <= steps; share *= 2)
        if (const double c = cost(share); c < best) {
            best = c;
            p = Split{share == kWarps ? kWarps : kFewWarps, share, 1};
        }
    for (int n = 2; n <= 32 && n * kWarps <= steps; ++n)
        if (const double c = cost(n * kWarps) + join; c < best) {
            best = c;
            p = Split{kWarps, kWarps, n};
        }
    return p;
}

template <bool kWide, bool kTop>
cudaError_t launch(const Args &p, int of, cudaStream_t s) {
    const long long rows = (long long)p.l.B * p.l.T, per = of / p.share;
    const unsigned blocks = (unsigned)(p.segments > 1 ? rows * p.segments : (rows + per - 1) / per);
    note_launches(1);
    cudaError_t e = of == kWarps
                        ? launch_pdl(logprob_kernel<kWide, kTop, kWarps>, dim3(blocks), dim3(kThreads), 0, s, p)
                        : launch_pdl(logprob_kernel<kWide, kTop, kFewWarps>, dim3(blocks), dim3(kFewWarps * 32), 0, s, p);
    if (e != cudaSuccess || p.segments == 1) return e;
    note_launches(1);
    return launch_pdl(logprob_join_kernel<kWide, kTop>, dim3((unsigned)rows), dim3(kThreads), 0, s, p);
}

Args args_of(const LogProb &l) {
    Args p{};
    p.l = l;
    p.c = (float)((double)l.scale * 1.4426950408889634073599);
    return p;
}

}  // namespace

size_t logprob_workspace(const LogProb &l) {
    const int segments = split(l).segments;
    const size_t n = segments > 1 ? (size_t)l.B * l.T * segments : 0;
    return 256 + (n + 15) / 16 * 256 + (l.top > 0 ? n * 32 * sizeof(Key) : 0);
}

cudaError_t launch_logprob(const LogProb &l, void *ws, cudaStream_t s) {
    Args p = args_of(l);
    const Split by = split(l);
    p.share = by.share;
    p.segments = by.segments;
    const size_t n = (size_t)l.B * l.T * p.segments;
    p.parts = reinterpret_cast<Part *>(static_cast<char *>(ws) + 256);
    p.tops = reinterpret_cast<Key *>(static_cast<char *>(ws) + 256 + (n + 15) / 16 * 256);
    if (l.z.wide) return l.top > 0 ? launch<true, true>(p, by.of, s) : launch<true, false>(p, by.of, s);
    return l.top > 0 ? launch<false, true>(p, by.of, s) : launch<false, false>(p, by.of, s);
}

cudaError_t launch_logprob_bwd(const LogProb &l, cudaStream_t s) {
    Args p = args_of(l);
    // (eight steps a warp, as far as they go: 313 us for 16384 rows of 32768 bf16, 322 with four, 329 with four in
    // blocks of 8 warps)
    p.units = std::max(1, steps_of(l) / 8);
    const long long units = (long long)l.B * l.T * p.units;
    const unsigned blocks = (unsigned)std::min<long long>((units + kFewWarps - 1) / kFewWarps, 1 << 20);
    note_launches(1);
    const auto kernel = l.z.wide ? l.stats ? logprob_bwd_kernel<true, true> : logprob_bwd_kernel<true, false>
                                 : l.stats ? logprob_bwd_kernel<false, true> : logprob_bwd_kernel<false, false>;
    return launch_pdl(kernel, dim3(blocks), dim3(kFewWarps * 32), 0, s, p);
}

}  // namespace blk
}  // namespace mosa
