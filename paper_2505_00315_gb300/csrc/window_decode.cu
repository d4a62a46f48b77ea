// One decoding step over a ring cache (mosa_window_decode): the new token's norm and
// rotation, its append and the attention over the visible slots in one kernel, and
// where a sequence's slots are split over several CTAs a second one that joins
// their partial softmaxes.
//
// For each query head, over the visible tokens u (the new one last)
//     s_u = scale q . k_u,  m = max s,  l = sum exp(s - m),  O = sum exp(s - m) v_u / l
// in one pass: running m, l and O, joined over warps and splits by
//     (m, l, O) + (m', l', O') = (M, l e^(m-M) + l' e^(m'-M), O e^(m-M) + O' e^(m'-M)).
// Bound by the cache's bytes, each read once for up to eight query heads of a group.
//   bf16   warp-wide matrix products (m16n8k16) take 16 tokens a step, with rows of K and V
//          loaded straight into fragments, 16 bytes a lane: a product's order of summation
//          is free, so a lane's eight neighbouring values may be any eight of it.  The 16
//          rows of the other operand are the eight heads twice, what bf16 holds of q (and of the weights)
//          and what its rounding leaves, so that nothing but the cache itself is rounded.
//          tcgen05 would want 128 rows and its operands in shared memory; the products are
//          a tenth of the time that the bytes take.
//   fp32, hp = 16, unaligned rows   CUDA cores: hp/8 lanes hold a row, eight values a lane.
// B48, up to 4100 tokens, 32 + 8 heads of 128, bf16: 122 us, 5.3 TB/s, 78% of the copy rate (on CUDA
// cores 539: each row's products with four heads are more instructions than its bytes have
// time for); fp32, all of them whole, 362 us, 4.4 TB/s, 66%.  B1, 1028 tokens, 16 + 4 heads: 6.4 us and 3.3 for the join, latency: the norm, the
// rotation, one trip for K, one for V, the warps' and the splits' sums in turn.
#include "head_rows.cuh"
#include "launch.h"
#include "profile.h"
#include "window.h"

namespace mosa {
namespace win {
namespace {

constexpr int kMaxSplits = 64;
constexpr float kLog2e = 1.4426950408889634f;

struct DecodeArgs {
    Decode d;
    const void *q, *k, *v, *gq, *gk;
    void *kc, *vc, *o;
    const int32_t *lens;
    int splits, chunks;
    float *po;      // [B][H][splits][hp] partial sums, relative to
    float2 *pml;    // [B][H][splits] (m, l), m in log2 units
};

__device__ __forceinline__ float merge_scale(float m, float M) {
    return m == -INFINITY ? 0.f : exp2f(m - M);
}

// The tokens of one split of one sequence: numbers lo .. hi-1 of its visible tokens, of which the
// first nS are sinks (in their slots) and the others, up to the new one, follow one another
// in the ring from slot s0 on.
struct Seen {
    int lo, hi, nS, s0, C, ring;
    __device__ __forceinline__ int slot(int u) const {
        const int s = u < nS ? u : s0 + (u - nS);
        return s >= C ? s - ring : s;   // (a window is no longer than the ring)
    }
};

// What every CTA does first: the query heads g0 .. g0+heads-1 of the group, normalised, turned
// and scaled (log2 units) into sq, and in the CTAs whose split holds the new token the
// token's rows into the caches.  False where the sequence is skipped.
template <class T, int HD, int GT, int THREADS>
__device__ __forceinline__ bool decode_prologue(const DecodeArgs &p, const Turns &tab, int split,
                                                int hk, int b, int g0, int heads, float (*sq)[HD],
                                                Seen *seen) {
    constexpr int LG = HD / 8;
    asm volatile("griddepcontrol.wait;" ::: "memory");
    __shared__ __align__(16) float2 cs[64];
    const Decode &d = p.d;
    const int G = d.H / d.Hkv, len = p.lens[b], at = len - 1;
    if (len <= 0) {   // skipped: the output is zero, the cache stays
        if (split == 0)
            for (int e = threadIdx.x; e < heads * HD; e += THREADS)
                static_cast<T *>(p.o)[d.o.at(b, 0, hk * G + g0 + e / HD) + e % HD] = from_f32<T>(0.f);
        return false;
    }
    const int ring = d.C - d.sinks, nS = min(d.sinks, len);
    const int wlo = max(d.sinks, at - d.window + 1), n = nS + max(at + 1 - wlo, 0);
    const int per = (n + p.splits - 1) / p.splits;
    *seen = Seen{min(split * per, n), min((split + 1) * per, n), nS,
                 at >= wlo ? d.sinks + (wlo - d.sinks) % ring : 0, d.C, ring};
    const bool newest = seen->lo < n && seen->hi == n;   // this split holds the new token
    for (int e = threadIdx.x; e < d.rotary / 2; e += THREADS) cs[angle_at<8, LG>(e)] = angle_of(tab.phi[e], at);
    __syncthreads();
    const int grp = threadIdx.x / LG, li = threadIdx.x % LG;
    const Part<8> part(li, d.rotary, d.halves);
    for (int u0 = 0; u0 < GT + 1; u0 += THREADS / LG) {   // (all lanes together: the sums are shuffles)
        const int u = u0 + grp;
        const bool key = u == GT, on = u < heads || (key && newest);
        float x[8], gm[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = 0.f, gm[e] = 1.f;
        if (on) {
            load_part<T, false, 8>(key ? (const T *)p.k + d.k.at(b, 0, hk)
                                : (const T *)p.q + d.q.at(b, 0, hk * G + g0 + u), part, x);
            const T *gamma = (const T *)(key ? p.gk : p.gq);
            if (d.norm && gamma != nullptr) load_part<T, false, 8>(gamma, part, gm);
        }
        if (d.norm) {
            float ss = 0.f;
#pragma unroll
            for (int e = 0; e < 8; ++e) ss = fmaf(x[e], x[e], ss);
            const float r = rsqrtf(fmaf(group_sum(ss, LG), 1.f / HD, d.eps));
#pragma unroll
            for (int e = 0; e < 8; ++e) x[e] *= r * gm[e];
        }
        turn<8, LG>(x, li, d.rotary, d.halves, cs, 1.f);
        if (on && key) {
            const int slot = seen->slot(n - 1);
            store_part<T, false, 8>((T *)p.kc + d.kc.at(b, slot, hk), part, x);
            const T *v = (const T *)p.v + d.v.at(b, 0, hk);
            T *o = (T *)p.vc + d.vc.at(b, slot, hk);
#pragma unroll
            for (int e = 0; e < 8; ++e) o[8 * li + e] = v[8 * li + e];
        } else if (u < GT) {
            const float f = d.scale * kLog2e;
#pragma unroll
            for (int e = 0; e < 8; ++e) sq[u][part.at(e)] = x[e] * f;
        }
    }
    __syncthreads();
    return true;
}

// The warps' partial softmaxes (m, l and O of each head in shared memory) joined and written.
template <class T, int HD, int GT, int WARPS>
__device__ __forceinline__ void decode_epilogue(const DecodeArgs &p, int split, int hk, int b, int g0,
                                                int heads, const float (*sm_m)[GT],
                                                const float (*sm_l)[GT], const float (*sm_o)[GT][HD]) {
    const Decode &d = p.d;
    __syncthreads();
    for (int e = threadIdx.x; e < heads * HD; e += WARPS * 32) {
        const int g = e / HD, x = e % HD, h = hk * (d.H / d.Hkv) + g0 + g;
        float M = -INFINITY, L = 0.f, o = 0.f;
#pragma unroll
        for (int w = 0; w < WARPS; ++w) M = fmaxf(M, sm_m[w][g]);
#pragma unroll
        for (int w = 0; w < WARPS; ++w) {
            const float f = merge_scale(sm_m[w][g], M);
            L += sm_l[w][g] * f;
            o += sm_o[w][g][x] * f;
        }
        if (p.splits == 1) {
            static_cast<T *>(p.o)[d.o.at(b, 0, h) + x] = from_f32<T>(o / L);
        } else {
            const long long row = ((long long)b * d.H + h) * p.splits + split;
            p.po[row * HD + x] = o;
            if (x == 0) p.pml[row] = make_float2(M, L);
        }
    }
}

// ------------------------------------------------------------- CUDA cores

constexpr int kThreads = 256;
constexpr int kWarps = kThreads / 32;
constexpr int kKeys = 4;        // rows a lane group takes at once

template <class T, bool VEC, int HD, int GT>
__global__ void __launch_bounds__(kThreads) window_decode_kernel(const __grid_constant__ DecodeArgs p,
                                                                 const __grid_constant__ Turns tab) {
    constexpr int LK = HD / 8, kRows = 32 / LK;          // lanes a row, rows a warp
    const Decode &d = p.d;
    const int split = blockIdx.x / p.chunks, g0 = blockIdx.x % p.chunks * GT;
    const int hk = blockIdx.y, b = blockIdx.z, heads = min(GT, d.H / d.Hkv - g0);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, c = (threadIdx.x % LK) * 8;
    __shared__ __align__(16) float sq[GT][HD];
    __shared__ float sm_m[kWarps][GT], sm_l[kWarps][GT];
    __shared__ __align__(16) float sm_o[kWarps][GT][HD];
    Seen seen;
    if (!decode_prologue<T, HD, GT, kThreads>(p, tab, split, hk, b, g0, heads, sq, &seen)) return;
    const Part<8> part(threadIdx.x % LK, 0, 0);
    const T *Kb = (const T *)p.kc + d.kc.at(b, 0, hk), *Vb = (const T *)p.vc + d.vc.at(b, 0, hk);
    float q[GT][8], acc[GT][8], m[GT], l[GT];
#pragma unroll
    for (int g = 0; g < GT; ++g) {
        m[g] = -INFINITY;
        l[g] = 0.f;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            q[g][e] = g < heads ? sq[g][c + e] : 0.f;
            acc[g][e] = 0.f;
        }
    }
    for (int u0 = seen.lo + warp * kRows * kKeys; u0 < seen.hi; u0 += kWarps * kRows * kKeys) {
        float kx[kKeys][8], vx[kKeys][8];
        bool on[kKeys];
#pragma unroll
        for (int j = 0; j < kKeys; ++j) {
            const int u = u0 + j * kRows + lane / LK, slot = seen.slot(u);
            on[j] = u < seen.hi;
            if (on[j]) {
                load_part<T, VEC, 8>(Kb + (long long)slot * d.kc.t, part, kx[j]);
                load_part<T, VEC, 8>(Vb + (long long)slot * d.vc.t, part, vx[j]);
            } else {
#pragma unroll
                for (int e = 0; e < 8; ++e) kx[j][e] = vx[j][e] = 0.f;
            }
        }
#pragma unroll
        for (int g = 0; g < GT; ++g) {
            float s[kKeys], mx = m[g];
#pragma unroll
            for (int j = 0; j < kKeys; ++j) {
                s[j] = 0.f;
#pragma unroll
                for (int e = 0; e < 8; ++e) s[j] = fmaf(q[g][e], kx[j][e], s[j]);
#pragma unroll
                for (int o = LK / 2; o > 0; o >>= 1) s[j] += __shfl_xor_sync(0xffffffffu, s[j], o);
                if (!on[j]) s[j] = -INFINITY;
                mx = fmaxf(mx, s[j]);
            }
            const float base = mx == -INFINITY ? 0.f : mx;
            const float corr = exp2f(m[g] - base);
            m[g] = mx;
            l[g] *= corr;
#pragma unroll
            for (int e = 0; e < 8; ++e) acc[g][e] *= corr;
#pragma unroll
            for (int j = 0; j < kKeys; ++j) {
                const float w = exp2f(s[j] - base);
                l[g] += w;
#pragma unroll
                for (int e = 0; e < 8; ++e) acc[g][e] = fmaf(w, vx[j][e], acc[g][e]);
            }
        }
    }
    // join the rows of a warp
#pragma unroll
    for (int g = 0; g < GT; ++g) {
#pragma unroll
        for (int o = LK; o < 32; o <<= 1) {
            const float mo = __shfl_xor_sync(0xffffffffu, m[g], o), lo_ = __shfl_xor_sync(0xffffffffu, l[g], o);
            const float M = fmaxf(m[g], mo), f0 = merge_scale(m[g], M), f1 = merge_scale(mo, M);
            m[g] = M;
            l[g] = l[g] * f0 + lo_ * f1;
#pragma unroll
            for (int e = 0; e < 8; ++e)
                acc[g][e] = acc[g][e] * f0 + __shfl_xor_sync(0xffffffffu, acc[g][e], o) * f1;
        }
        if (lane < LK) {
#pragma unroll
            for (int e = 0; e < 8; ++e) sm_o[warp][g][c + e] = acc[g][e];
            if (lane == 0) sm_m[warp][g] = m[g], sm_l[warp][g] = l[g];
        }
    }
    decode_epilogue<T, HD, GT, kWarps>(p, split, hk, b, g0, heads, sm_m, sm_l, sm_o);
}

// ------------------------------------------------------- matrix products

constexpr int kMmaWarps = 4, kMmaHeads = 8, kMmaTokens = 16;

// D += A B: A 16 x 16, B 16 x 8, bf16; D fp32.
__device__ __forceinline__ void mma16816(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    asm volatile(
        "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, "
        "{%8, %9}, {%0, %1, %2, %3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

// Two values as bf16 (hi) and what their rounding left, as bf16 (lo).
__device__ __forceinline__ void halves_of(float a, float b, uint32_t &hi, uint32_t &lo) {
    hi = two_bf16(a, b);
    lo = two_bf16(a - __uint_as_float(hi << 16), b - __uint_as_float(hi & 0xFFFF0000u));
}

// Lane (g, t) = (lane / 4, lane % 4).  Scores of 8 tokens: A = the heads' q (rows g: hi, g + 8: lo),
// B = the tokens' rows of K, token g on lane (g, .), whose 16-byte pieces t, t + 4, .. serve two
// 16-wide steps each.  O: A = the weights (hi and lo rows again) of 16 tokens, in the places where
// the scores' results lie; B = V, tokens 2t, 2t+1, 8+2t, 9+2t on lane (g, t), its piece g (and g + 8) of
// the row: value j of a piece is column g of output tile j.
template <int HD>
__global__ void __launch_bounds__(kMmaWarps * 32, 3) window_decode_mma_kernel(
    const __grid_constant__ DecodeArgs p, const __grid_constant__ Turns tab) {
    constexpr int kPieces = HD / 32;                 // 16-byte pieces of K a lane
    constexpr int VP = HD >= 64 ? HD / 64 : 1;       // pieces of V a lane, of
    constexpr int VE = HD >= 64 ? 8 : HD / 8;        // so many values
    const Decode &d = p.d;
    const int split = blockIdx.x / p.chunks, g0 = blockIdx.x % p.chunks * kMmaHeads;
    const int hk = blockIdx.y, b = blockIdx.z, heads = min(kMmaHeads, d.H / d.Hkv - g0);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    __shared__ __align__(16) float sq[kMmaHeads][HD];
    __shared__ float sm_m[kMmaWarps][kMmaHeads], sm_l[kMmaWarps][kMmaHeads];
    __shared__ __align__(16) float sm_o[kMmaWarps][kMmaHeads][HD];
    __shared__ uint4 sm_q[2 * kPieces][32];
    Seen seen;
    if (!decode_prologue<bf16, HD, kMmaHeads, kMmaWarps * 32>(p, tab, split, hk, b, g0, heads, sq, &seen))
        return;
    // the heads' operand, the same for every warp: in shared memory, where registers would cost a third of
    // the warps in flight
    if (warp == 0) {
#pragma unroll
        for (int i = 0; i < 2 * kPieces; ++i) {
            const float *x = &sq[g][8 * (t + 4 * (i >> 1)) + 4 * (i & 1)];
            uint4 w;
            halves_of(x[0], x[1], w.x, w.y);
            halves_of(x[2], x[3], w.z, w.w);
            sm_q[i][lane] = w;
        }
    }
    __syncthreads();
    const bf16 *Kb = (const bf16 *)p.kc + d.kc.at(b, 0, hk) + 8 * t;
    const bf16 *Vb = (const bf16 *)p.vc + d.vc.at(b, 0, hk) + VE * g;
    float acc[VP * VE][4], m = -INFINITY, l = 0.f;
#pragma unroll
    for (int j = 0; j < VP * VE; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[j][e] = 0.f;
    uint4 kx[2][kPieces];
    uint32_t vx[4][VP][VE / 2];
    auto load_k = [&](int u0) {
#pragma unroll
        for (int r = 0; r < 2; ++r) {
            const int u = u0 + 8 * r + g;
            const bf16 *row = Kb + (long long)seen.slot(u) * d.kc.t;
#pragma unroll
            for (int i = 0; i < kPieces; ++i)
                kx[r][i] = u < seen.hi ? *reinterpret_cast<const uint4 *>(row + 32 * i) : make_uint4(0, 0, 0, 0);
        }
    };
    auto load_v = [&](int u0) {
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const int u = u0 + 8 * (r >> 1) + 2 * t + (r & 1);
            const bf16 *row = Vb + (long long)seen.slot(u) * d.vc.t;
#pragma unroll
            for (int i = 0; i < VP; ++i) {
                if constexpr (VE == 8) {
                    const uint4 w = u < seen.hi ? *reinterpret_cast<const uint4 *>(row + 64 * i) : make_uint4(0, 0, 0, 0);
                    vx[r][i][0] = w.x; vx[r][i][1] = w.y; vx[r][i][2] = w.z; vx[r][i][3] = w.w;
                } else {
                    const uint2 w = u < seen.hi ? *reinterpret_cast<const uint2 *>(row) : make_uint2(0, 0);
                    vx[r][i][0] = w.x; vx[r][i][1] = w.y;
                }
            }
        }
    };
    // loads are always under way: the next tokens' K from the last use of these tokens' on, V from
    // the step's beginning
    load_k(seen.lo + warp * kMmaTokens);
    for (int u0 = seen.lo + warp * kMmaTokens; u0 < seen.hi; u0 += kMmaWarps * kMmaTokens) {
        load_v(u0);
        float s[2][4];
#pragma unroll
        for (int e = 0; e < 4; ++e) s[0][e] = s[1][e] = 0.f;
#pragma unroll
        for (int i = 0; i < kPieces; ++i) {
            const uint4 x = sm_q[2 * i][lane], y = sm_q[2 * i + 1][lane];
            const uint32_t qx[4] = {x.x, x.y, x.z, x.w}, qy[4] = {y.x, y.y, y.z, y.w};
#pragma unroll
            for (int r = 0; r < 2; ++r) {
                mma16816(s[r], qx, kx[r][i].x, kx[r][i].y);
                mma16816(s[r], qy, kx[r][i].z, kx[r][i].w);
            }
        }
        load_k(u0 + kMmaWarps * kMmaTokens);
        // this lane: head g, tokens 8 r + 2 t + e; hi and lo rows added up
        float w[4], mx = m;
#pragma unroll
        for (int x = 0; x < 4; ++x) {
            w[x] = s[x >> 1][x & 1] + s[x >> 1][2 + (x & 1)];
            if (u0 + 8 * (x >> 1) + 2 * t + (x & 1) >= seen.hi) w[x] = -INFINITY;
            mx = fmaxf(mx, w[x]);
        }
        mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 1));
        mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 2));
        const float base = mx == -INFINITY ? 0.f : mx;
        if (__any_sync(0xffffffffu, mx > m)) {
            const float corr = exp2f(m - base);
            l *= corr;
#pragma unroll
            for (int j = 0; j < VP * VE; ++j)
#pragma unroll
                for (int e = 0; e < 4; ++e) acc[j][e] *= corr;
            m = mx;
        }
#pragma unroll
        for (int x = 0; x < 4; ++x) {
            w[x] = exp2f(w[x] - base);
            l += w[x];
        }
        uint32_t pa[4];
        halves_of(w[0], w[1], pa[0], pa[1]);
        halves_of(w[2], w[3], pa[2], pa[3]);
#pragma unroll
        for (int i = 0; i < VP; ++i)
#pragma unroll
            for (int j = 0; j < VE; ++j) {
                const uint32_t sel = j & 1 ? 0x7632 : 0x5410;
                mma16816(acc[i * VE + j], pa, __byte_perm(vx[0][i][j >> 1], vx[1][i][j >> 1], sel),
                         __byte_perm(vx[2][i][j >> 1], vx[3][i][j >> 1], sel));
            }
    }
    l += __shfl_xor_sync(0xffffffffu, l, 1);
    l += __shfl_xor_sync(0xffffffffu, l, 2);
    if (t == 0) sm_m[warp][g] = m, sm_l[warp][g] = l;
#pragma unroll
    for (int i = 0; i < VP; ++i)
#pragma unroll
        for (int j = 0; j < VE; ++j)
#pragma unroll
            for (int e = 0; e < 2; ++e)   // output columns 2t, 2t+1 of the tile are pieces 2t, 2t+1
                sm_o[warp][g][64 * i + VE * (2 * t + e) + j] = acc[i * VE + j][e] + acc[i * VE + j][2 + e];
    decode_epilogue<bf16, HD, kMmaHeads, kMmaWarps>(p, split, hk, b, g0, heads, sm_m, sm_l, sm_o);
}

// O of one head: the splits' partial softmaxes joined.
template <class T>
__global__ void __launch_bounds__(128) decode_join_kernel(const __grid_constant__ DecodeArgs p) {
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const Decode &d = p.d;
    const int h = blockIdx.x, b = blockIdx.y, x = threadIdx.x;
    if (p.lens[b] <= 0) return;   // written by the first kernel
    const long long row = ((long long)b * d.H + h) * p.splits;
    float M = -INFINITY, L = 0.f, o = 0.f;
    for (int s = 0; s < p.splits; ++s) M = fmaxf(M, p.pml[row + s].x);
    for (int s = 0; s < p.splits; ++s) {
        const float2 ml = p.pml[row + s];
        const float f = merge_scale(ml.x, M);
        L += ml.y * f;
        o += p.po[(row + s) * d.hp + x] * f;
    }
    static_cast<T *>(p.o)[d.o.at(b, 0, h) + x] = from_f32<T>(o / L);
}

// Whether the step runs on matrix products (the workspace does not depend on it).
bool use_mma(const Decode &d, const void *Kc, const void *Vc) {
    return d.bf16 && d.hp >= 32 && rows16(Kc, d.kc, true) && rows16(Vc, d.vc, true);
}

int heads_of(const Decode &d, bool mma) {   // query heads a CTA takes
    const int G = d.H / d.Hkv;
    return mma ? kMmaHeads : G == 1 ? 1 : G == 2 ? 2 : G <= 4 ? 4 : 8;
}

// Splits of a sequence: four CTAs an SM in all, of at least 128 tokens each.  (At 8, 16 and 32 CTAs an SM
// the 48 sequences above took 147, 157 and 183 us against 150, with the loads as they were then.)
int splits_of(const Decode &d) {
    const int G = d.H / d.Hkv, chunks = (G + kMmaHeads - 1) / kMmaHeads;
    const long long ctas = (long long)d.B * d.Hkv * chunks;
    const long long seen = (long long)d.sinks + d.window;
    const long long want = (4 * 152 + ctas - 1) / ctas, most = (seen + 127) / 128;
    long long s = want < most ? want : most;
    return (int)(s < 1 ? 1 : s > kMaxSplits ? kMaxSplits : s);
}

cudaError_t join(const DecodeArgs &p, cudaStream_t s) {
    if (p.splits == 1) return cudaSuccess;
    const dim3 grid(p.d.H, p.d.B);
    const cudaError_t e = p.d.bf16 ? launch_pdl(decode_join_kernel<bf16>, grid, dim3(p.d.hp), 0, s, p)
                 : launch_pdl(decode_join_kernel<float>, grid, dim3(p.d.hp), 0, s, p);
    note_launches(1);
    return e;
}

template <class T, bool VEC, int HD>
cudaError_t launch_hd(const DecodeArgs &p, const Turns &tab, cudaStream_t s) {
    const dim3 grid(p.splits * p.chunks, p.d.Hkv, p.d.B);
    cudaError_t e;
    switch (heads_of(p.d, false)) {
        case 1: e = launch_pdl(window_decode_kernel<T, VEC, HD, 1>, grid, dim3(kThreads), 0, s, p, tab); break;
        case 2: e = launch_pdl(window_decode_kernel<T, VEC, HD, 2>, grid, dim3(kThreads), 0, s, p, tab); break;
        case 4: e = launch_pdl(window_decode_kernel<T, VEC, HD, 4>, grid, dim3(kThreads), 0, s, p, tab); break;
        default: e = launch_pdl(window_decode_kernel<T, VEC, HD, 8>, grid, dim3(kThreads), 0, s, p, tab); break;
    }
    note_launches(1);
    return e != cudaSuccess ? e : join(p, s);
}

template <class T, bool VEC>
cudaError_t launch_of(const DecodeArgs &p, const Turns &tab, cudaStream_t s) {
    switch (p.d.hp) {
        case 16: return launch_hd<T, VEC, 16>(p, tab, s);
        case 32: return launch_hd<T, VEC, 32>(p, tab, s);
        case 64: return launch_hd<T, VEC, 64>(p, tab, s);
        default: return launch_hd<T, VEC, 128>(p, tab, s);
    }
}

cudaError_t launch_mma(const DecodeArgs &p, const Turns &tab, cudaStream_t s) {
    const dim3 grid(p.splits * p.chunks, p.d.Hkv, p.d.B);
    cudaError_t e;
    switch (p.d.hp) {
        case 32: e = launch_pdl(window_decode_mma_kernel<32>, grid, dim3(kMmaWarps * 32), 0, s, p, tab); break;
        case 64: e = launch_pdl(window_decode_mma_kernel<64>, grid, dim3(kMmaWarps * 32), 0, s, p, tab); break;
        default: e = launch_pdl(window_decode_mma_kernel<128>, grid, dim3(kMmaWarps * 32), 0, s, p, tab); break;
    }
    note_launches(1);
    return e != cudaSuccess ? e : join(p, s);
}

size_t partial_bytes(const Decode &d, int splits) {
    return ((size_t)d.B * d.H * splits * d.hp * 4 + 255) / 256 * 256;
}

}  // namespace

size_t decode_workspace(const Decode &d) {
    const int s = splits_of(d);
    return s == 1 ? 256 : partial_bytes(d, s) + (size_t)d.B * d.H * s * sizeof(float2);
}

cudaError_t launch_decode(const Decode &d, const void *q, const void *k, const void *v,
                          const void *gq, const void *gk, const int32_t *lens, void *Kc, void *Vc,
                          void *O, void *ws, cudaStream_t s) {
    const bool mma = use_split() && use_mma(d, Kc, Vc);
    const int splits = splits_of(d), GT = heads_of(d, mma), G = d.H / d.Hkv;
    DecodeArgs p{d, q, k, v, gq, gk, Kc, Vc, O, lens, splits, (G + GT - 1) / GT, (float *)ws,
                 (float2 *)((char *)ws + partial_bytes(d, splits))};
    const Turns tab = make_turns(d.rotary, d.theta);
    if (mma) return launch_mma(p, tab, s);
    const bool vec = rows16(Kc, d.kc, d.bf16) && rows16(Vc, d.vc, d.bf16);
    if (d.bf16) return vec ? launch_of<bf16, true>(p, tab, s) : launch_of<bf16, false>(p, tab, s);
    return vec ? launch_of<float, true>(p, tab, s) : launch_of<float, false>(p, tab, s);
}

}  // namespace win
}  // namespace mosa
