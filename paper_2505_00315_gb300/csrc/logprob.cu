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
// A warp takes a row, or the warps of a block share one where rows are few, or some blocks, whose
// results a second kernel joins.  Rows move in 16-byte pieces wherever they start: a row is cut at the
// addresses' multiples of 16, its first and last pieces are read value by value.
//
// Alternatives: a warp keeps its 32 best entries, one a lane, as 64-bit keys in falling order (the
// value's bits in an order of integers, then the index, low ones first).  Values above the last
// one wanted are rare after the first pieces; they gather in shared memory and are sorted and merged 32
// at a time.  The first piece's bar is the top-th largest of its lanes' maxima.
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
    int segments;       // forward: blocks of a row
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
        for (int i = 0; i < 4; ++i) {
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
    if (kWide)
        return fmaxf(fmaxf(__uint_as_float(v.w[0]), __uint_as_float(v.w[1])),
                     fmaxf(__uint_as_float(v.w[2]), __uint_as_float(v.w[3])));
    const uint32_t m = max2(max2(v.w[0], v.w[1]), max2(v.w[2], v.w[3]));
    return fmaxf(low(m), high(m));
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

__device__ __forceinline__ Key pick(Key a, Key b, bool larger) { return (a > b) == larger ? a : b; }

// Falling order over the lanes.
__device__ __forceinline__ Key sorted(Key k, int lane) {
#pragma unroll
    for (int n = 2; n <= 32; n *= 2)
#pragma unroll
        for (int o = n / 2; o > 0; o /= 2)
            k = pick(k, __shfl_xor_sync(0xffffffffu, k, o), ((lane & o) == 0) == ((lane & n) == 0));
    return k;
}
// The 32 largest of two lists in falling order.
__device__ __forceinline__ Key merged(Key a, Key b, int lane) {
    Key k = pick(a, __shfl_sync(0xffffffffu, b, 31 - lane), true);
#pragma unroll
    for (int o = 16; o > 0; o /= 2) k = pick(k, __shfl_xor_sync(0xffffffffu, k, o), (lane & o) == 0);
    return k;
}

struct Best {
    Key list = 0;          // this lane's entry (0: none)
    float bar = 0.f;       // the last entry wanted
    bool all = true;       // there is no bar yet
    int waiting = 0;       // candidates in shared memory
};

// Merges the first 32 candidates (those there are).
__device__ __forceinline__ void take_in(Best &b, Key *wait, int top, int lane) {
    __syncwarp();
    Key k = lane < b.waiting ? wait[lane] : 0;
    const Key rest = 32 + lane < b.waiting ? wait[32 + lane] : 0;
    __syncwarp();
    wait[lane] = rest;
    b.waiting = max(b.waiting - 32, 0);
    b.list = merged(b.list, sorted(k, lane), lane);
    const uint32_t last = (uint32_t)(__shfl_sync(0xffffffffu, b.list, top - 1) >> 32);
    b.all = last == 0;
    b.bar = of_order(last);
    __syncwarp();
}

// The 32 best of all warps' lists, in warp 0.
__device__ __forceinline__ Key best_of_block(Key list, Key (*room)[32], int warp, int lane) {
#pragma unroll
    for (int o = kWarps / 2; o > 0; o /= 2) {
        __syncthreads();
        if (warp >= o && warp < 2 * o) room[warp - o][lane] = list;
        __syncthreads();
        if (warp < o) list = merged(list, room[warp][lane], lane);
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

// One warp writes a row's results.
template <bool kWide, bool kTop>
__device__ __forceinline__ void finish(const Args &p, long long row, const Part &a, Key list, int lane) {
    const LogProb &l = p.l;
    const bool none = a.m <= kLeast, bad = a.m > -kLeast;
    const float lg = logf(a.s), inf = __int_as_float(0x7F800000), nan = __int_as_float(0x7FC00000);
    const float lse = bad ? nan : none && a.s == a.s ? -inf : __fadd_rn(__fmul_rn(a.m, l.scale), lg);
    if (lane == 0) {
        if (l.lse != nullptr) l.lse[row] = lse;
        if (l.entropy != nullptr)
            l.entropy[row] = bad ? nan : none && a.s == a.s ? 0.f : fmaf(-kLn2, a.t / a.s, lg);
        if (l.logp != nullptr) {
            const long long t = l.target64 ? static_cast<const int64_t *>(l.targets)[row]
                                           : (long long)static_cast<const int32_t *>(l.targets)[row];
            float lp = 0.f;
            if (t >= l.V) {
                lp = nan;
            } else if (t >= 0) {
                int it;
                const int ib = row_split(l, row, &it);
                const float z = Row<kWide>(l.z.at(ib, it), l.V).value((int)t);
                lp = lse != lse ? nan : z <= kLeast ? -inf : fmaf(z - a.m, l.scale, -lg);
            }
            l.logp[row] = lp;
        }
    }
    if (kTop && lane < l.top) {
        const float v = of_order((uint32_t)(list >> 32));
        l.top_index[row * l.top + lane] = list == 0 ? 0 : (int32_t)(0xFFFFFFFFu - (uint32_t)list);
        l.top_logp[row * l.top + lane] = lse != lse ? nan : v <= kLeast || none ? -inf : fmaf(v - a.m, l.scale, -lg);
    }
}

// kShared: the warps of a block share a row (segment blockIdx.x % segments of it); else a row each.
template <bool kWide, bool kTop, bool kShared>
__global__ void __launch_bounds__(kThreads, 3) logprob_kernel(const __grid_constant__ Args p) {
    asm volatile("griddepcontrol.wait;" ::: "memory");
    constexpr int E = kWide ? 4 : 8;
    __shared__ Key waiting[kTop ? kWarps : 1][64];
    __shared__ Key room[kTop && kShared ? kWarps / 2 : 1][32];
    __shared__ Part part[kShared ? kWarps : 1];
    const LogProb &l = p.l;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const long long rows = (long long)l.B * l.T;
    long long row = kShared ? blockIdx.x / p.segments : (long long)blockIdx.x * kWarps + warp;
    const int segment = kShared ? (int)(blockIdx.x - row * p.segments) : 0;
    if (row >= rows) return;   // (kShared: no block)
    int t;
    const int b = row_split(l, row, &t);
    const Row<kWide> z(l.z.at(b, t), l.V);
    const int steps = z.steps();
    const int share = kShared ? segment * kWarps + warp : 0, shares = kShared ? p.segments * kWarps : 1;
    const int from = (int)((long long)steps * share / shares), to = (int)((long long)steps * (share + 1) / shares);

    float m = kLeast;
    Pair s = 0, sum_t = 0;   // pairs of sums
    Best best;
    const Pair c2 = both(p.c);
    Piece cur[kVecs];
#pragma unroll
    for (int u = 0; u < kVecs; ++u)
        if (from < to) z.load(z.column(from, u, lane), cur[u]);
    for (int i = from; i < to; ++i) {
        Piece next[kVecs];
#pragma unroll
        for (int u = 0; u < kVecs; ++u)
            if (i + 1 < to) z.load(z.column(i + 1, u, lane), next[u]);
        float most[kVecs], here;
#pragma unroll
        for (int u = 0; u < kVecs; ++u) most[u] = largest<kWide>(cur[u]);
        here = fmaxf(fmaxf(most[0], most[1]), fmaxf(most[2], most[3]));
        if (kTop && __any_sync(0xffffffffu, best.all || here > best.bar)) {
            float bar = best.bar;
            bool all = best.all;
            const bool first = i == from;
            if (first) {
                // as many lanes as entries are wanted hold one of at least this value
                const Key k = sorted((Key)order_of(here) << 32, lane);
                bar = of_order((uint32_t)(__shfl_sync(0xffffffffu, k, l.top - 1) >> 32));
                all = false;
            }
#pragma unroll
            for (int u = 0; u < kVecs; ++u) {
                if (!__any_sync(0xffffffffu, all || most[u] > bar || (first && most[u] == bar))) continue;
                const int col = z.column(i, u, lane);
#pragma unroll
                for (int e = 0; e < E; ++e) {
                    const float v = value_of<kWide>(cur[u], e);
                    const bool on = (all || v > bar || (first && v == bar)) && col + e >= 0 && col + e < l.V;
                    const uint32_t who = __ballot_sync(0xffffffffu, on);
                    if (who == 0) continue;
                    if (on)
                        waiting[warp][best.waiting + __popc(who & ((1u << lane) - 1))] =
                            (Key)order_of(v) << 32 | (0xFFFFFFFFu - (uint32_t)(col + e));
                    best.waiting += __popc(who);
                    if (best.waiting >= 32) take_in(best, waiting[warp], l.top, lane);
                }
            }
            // Those of the first step are at least `top`: what comes later has to be above their bar.
            if (first && best.all) {
                best.bar = bar;
                best.all = bar != bar;
            }
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
    if (kTop)
        while (best.waiting > 0) take_in(best, waiting[warp], l.top, lane);
    const F2 s2 = of_two(s), t2 = of_two(sum_t);
    Part a = join(Part{m, s2.x + s2.y, t2.x + t2.y, 0.f}, p.c);
    if (!kShared) {
        finish<kWide, kTop>(p, row, a, best.list, lane);
        return;
    }
    if (lane == 0) part[warp] = a;
    if (kTop) best.list = best_of_block(best.list, room, warp, lane);
    __syncthreads();
    if (warp != 0) return;
    a = join(lane < kWarps ? part[lane] : Part{kLeast, 0.f, 0.f, 0.f}, p.c);
    if (p.segments == 1) {
        finish<kWide, kTop>(p, row, a, best.list, lane);
        return;
    }
    if (lane == 0) p.parts[blockIdx.x] = a;
    if (kTop) p.tops[(long long)blockIdx.x * 32 + lane] = best.list;
}

// The segments of a row together: a block a row.
template <bool kWide, bool kTop>
__global__ void __launch_bounds__(kThreads) logprob_join_kernel(const __grid_constant__ Args p) {
    asm volatile("griddepcontrol.wait;" ::: "memory");
    __shared__ Key room[kTop ? kWarps / 2 : 1][32];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const long long row = blockIdx.x, at = row * p.segments;
    Key list = 0;
    if (kTop) {
        for (int i = warp; i < p.segments; i += kWarps) list = merged(list, p.tops[(at + i) * 32 + lane], lane);
        list = best_of_block(list, room, warp, lane);
    }
    if (warp != 0) return;
    const Part none{kLeast, 0.f, 0.f, 0.f};
    const Part a = join(lane < p.segments ? p.parts[at + lane] : none, p.c);
    finish<kWide, kTop>(p, row, a, list, lane);
}

// ------------------------------------------------------------------ backward

__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
    for (int o = 16; o > 0; o /= 2) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}

// A warp takes one of the `units` shares of a row.
template <bool kWide>
__global__ void __launch_bounds__(kThreads) logprob_bwd_kernel(const __grid_constant__ Args p) {
    asm volatile("griddepcontrol.wait;" ::: "memory");
    constexpr int E = kWide ? 4 : 8;
    const LogProb &l = p.l;
    const int lane = threadIdx.x & 31;
    const long long all = (long long)l.B * l.T * p.units, warps = (long long)gridDim.x * kWarps;
    for (long long unit = (long long)blockIdx.x * kWarps + (threadIdx.x >> 5); unit < all; unit += warps) {
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
        const float ref = zero ? 0.f : lse;
        // Values that are clamped to this have weight 0, and no infinity meets it.  (Rounded down, so
        // that no larger one is met.)
        const float least = fmaxf((ref - 208.f) / l.scale, kLeast);
        const uint32_t least2 = 0x10001u * (uint32_t)__bfloat16_as_ushort(__float2bfloat16_rd(least));
        const float leastw = __bfloat162float(__float2bfloat16_rd(least));

        // What the few places with a gradient of their own hold, before they are overwritten.
        const bool mine = alt >= col0 && alt < col1, here = target >= col0 && target < col1;
        const float z_alt = mine ? z.value(alt) : 0.f, z_target = here ? z.value((int)target) : 0.f;
        __syncwarp();

        auto weight = [&](float v) {   // 2^b and its gradient without the place's own
            v = max_nan(v, leastw);
            const float b = __fsub_rn(__fmul_rn(v, l.scale), ref) * kLog2e;
            return pow2(b) * fmaf(B, b, A);
        };
        const bool same = ((reinterpret_cast<uintptr_t>(out) ^ reinterpret_cast<uintptr_t>(z.p)) & 15) == 0;
        const Pair scale2 = both(l.scale), minus = both(-ref), to2 = both(kLog2e);
        const Pair A2 = both(A), B2 = both(B);
        Piece cur[kVecs];
#pragma unroll
        for (int u = 0; u < kVecs; ++u)
            if (from < to && !zero) z.load(z.column(from, u, lane), cur[u]);
        for (int i = from; i < to; ++i) {
            Piece next[kVecs];
#pragma unroll
            for (int u = 0; u < kVecs; ++u)
                if (i + 1 < to && !zero) z.load(z.column(i + 1, u, lane), next[u]);
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
                        a = mul2(add2(mul2(a, scale2), minus), to2);
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
            const float x = v <= kLeast ? 0.f : fmaf(l.scale, g, weight(v));
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

// Forward: a row is a warp's where rows are many or short; else a block's, or that of as many
// blocks as let two SMs of three have two.
int segments_of(const LogProb &l) {   // 0: a warp a row
    const long long rows = (long long)l.B * l.T;
    // (the same for both types, so that the workspace's size does not hang on a pointer)
    const int steps = (int)(((long long)l.V + 1023) / 1024);
    if (rows >= 2432 || steps < 4) return 0;
    const long long most = std::max(1, steps / kWarps);
    return (int)std::min<long long>(std::min<long long>(most, 32), std::max(1LL, 2 * kSms / rows));
}

template <bool kWide, bool kTop>
cudaError_t launch(const Args &p, cudaStream_t s) {
    const long long rows = (long long)p.l.B * p.l.T;
    cudaError_t e;
    note_launches(1);
    if (p.segments == 0) {
        const long long blocks = (rows + kWarps - 1) / kWarps;
        return launch_pdl(logprob_kernel<kWide, kTop, false>, dim3((unsigned)blocks), dim3(kThreads), 0, s, p);
    }
    e = launch_pdl(logprob_kernel<kWide, kTop, true>, dim3((unsigned)(rows * p.segments)), dim3(kThreads), 0, s, p);
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
    const size_t n = (size_t)l.B * l.T * std::max(segments_of(l), 0);
    return 256 + (n + 15) / 16 * 256 + (l.top > 0 ? n * 32 * sizeof(Key) : 0);
}

cudaError_t launch_logprob(const LogProb &l, void *ws, cudaStream_t s) {
    Args p = args_of(l);
    p.segments = segments_of(l);
    const size_t n = (size_t)l.B * l.T * p.segments;
    p.parts = reinterpret_cast<Part *>(static_cast<char *>(ws) + 256);
    p.tops = reinterpret_cast<Key *>(static_cast<char *>(ws) + 256 + (n + 15) / 16 * 256);
    if (l.z.wide) return l.top > 0 ? launch<true, true>(p, s) : launch<true, false>(p, s);
    return l.top > 0 ? launch<false, true>(p, s) : launch<false, false>(p, s);
}

cudaError_t launch_logprob_bwd(const LogProb &l, cudaStream_t s) {
    Args p = args_of(l);
    p.units = std::max(1, steps_of(l) / 4);
    const long long units = (long long)l.B * l.T * p.units;
    const long long blocks = std::min<long long>((units + kWarps - 1) / kWarps, 1 << 20);
    note_launches(1);
    if (l.z.wide)
        return launch_pdl(logprob_bwd_kernel<true>, dim3((unsigned)blocks), dim3(kThreads), 0, s, p);
    return launch_pdl(logprob_bwd_kernel<false>, dim3((unsigned)blocks), dim3(kThreads), 0, s, p);
}

}  // namespace blk
}  // namespace mosa
