// One decoding step over a ring cache (mosa_window_decode): the new token's norm and
// rotation, its append and the attention over the visible slots in one kernel, and
// where a sequence's slots are split over several CTAs a second one that joins
// their partial softmaxes.
//
// For each query head, over the visible tokens u and the new one,
//     s_u = scale q . k_u,  m = max s,  l = sum exp(s - m),  O = sum exp(s - m) v_u / l
// in one pass: running m, l and O, joined over lanes, warps and splits by
//     (m, l, O) + (m', l', O') = (M, l e^(m-M) + l' e^(m'-M), O e^(m-M) + O' e^(m'-M)).
// Bound by the cache's bytes, each read once: hp/8 lanes hold a row, eight values a
// lane, and up to eight query heads of a group meet a row while it is in registers.
#include "head_rows.cuh"
#include "launch.h"
#include "profile.h"
#include "window.h"

namespace mosa {
namespace win {
namespace {

constexpr int kThreads = 256;
constexpr int kWarps = kThreads / 32;
constexpr int kKeys = 4;        // rows a lane group takes at once
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

template <class T, bool VEC, int HD, int GT>
__global__ void __launch_bounds__(kThreads) window_decode_kernel(const __grid_constant__ DecodeArgs p,
                                                                 const __grid_constant__ Turns tab) {
    constexpr int LK = HD / 8, kRows = 32 / LK;          // lanes a row, rows a warp
    const Decode &d = p.d;
    const int G = d.H / d.Hkv;
    const int split = blockIdx.x / p.chunks, chunk = blockIdx.x % p.chunks;
    const int hk = blockIdx.y, b = blockIdx.z;
    const int g0 = chunk * GT, heads = min(GT, G - g0);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int grp = threadIdx.x / LK, c = (threadIdx.x % LK) * 8;
    __shared__ float2 cs[64];
    __shared__ __align__(16) float sq[GT][HD];
    __shared__ __align__(16) float sk[HD];
    __shared__ float sm_m[kWarps][GT], sm_l[kWarps][GT];
    __shared__ __align__(16) float sm_o[kWarps][GT][HD];

    const int len = p.lens[b], at = len - 1;
    if (len <= 0) {   // skipped: the output is zero, the cache stays
        if (split == 0)
            for (int e = threadIdx.x; e < heads * HD; e += kThreads)
                static_cast<T *>(p.o)[d.o.at(b, 0, hk * G + g0 + e / HD) + e % HD] = from_f32<T>(0.f);
        return;
    }
    for (int e = threadIdx.x; e < d.rotary / 2; e += kThreads) cs[e] = angle_of(tab.phi[e], at);
    __syncthreads();
    // the new token's q heads, and in the first split its k
    for (int u0 = 0; u0 < GT + 1; u0 += kThreads / LK) {
        const int u = u0 + grp;
        const bool key = u == GT, on = u < heads || (key && split == 0);
        float x[8], gm[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = 0.f, gm[e] = 1.f;
        if (on) {
            load8<T, false>((key ? (const T *)p.k + d.k.at(b, 0, hk)
                                 : (const T *)p.q + d.q.at(b, 0, hk * G + g0 + u)) + c, x);
            const T *gamma = (const T *)(key ? p.gk : p.gq);
            if (d.norm && gamma != nullptr) load8<T, false>(gamma + c, gm);
        }
        if (d.norm) {
            float ss = 0.f;
#pragma unroll
            for (int e = 0; e < 8; ++e) ss = fmaf(x[e], x[e], ss);
            const float r = rsqrtf(group_sum(ss, LK) / (float)HD + d.eps);
#pragma unroll
            for (int e = 0; e < 8; ++e) x[e] *= r * gm[e];
        }
        turn8(x, c, d.rotary, d.halves, cs, 1.f, lane);
        if (on) {
            float *dst = key ? sk + c : sq[u < GT ? u : 0] + c;
#pragma unroll
            for (int e = 0; e < 8; ++e) dst[e] = key ? to_f32(from_f32<T>(x[e])) : x[e];
        }
    }
    __syncthreads();
    const int ring = d.C - d.sinks;
    if (split == 0 && chunk == 0 && threadIdx.x < HD) {   // append
        const int slot = at < d.sinks ? at : d.sinks + (at - d.sinks) % ring;
        const int e = threadIdx.x;
        static_cast<T *>(p.kc)[d.kc.at(b, slot, hk) + e] = from_f32<T>(sk[e]);
        static_cast<T *>(p.vc)[d.vc.at(b, slot, hk) + e] = static_cast<const T *>(p.v)[d.v.at(b, 0, hk) + e];
    }
    // the older tokens it sees: sinks 0 .. nS-1, then wlo .. at-1, which may wrap in the ring once
    const int nS = min(d.sinks, at), wlo = max(d.sinks, at - d.window + 1);
    const int nW = max(at - wlo, 0), n = nS + nW;
    const int s0 = nW > 0 ? d.sinks + (wlo - d.sinks) % ring : 0;
    const int per = (n + p.splits - 1) / p.splits;
    const int lo = min(split * per, n), hi = min(lo + per, n);
    const T *Kb = (const T *)p.kc + d.kc.at(b, 0, hk) + c, *Vb = (const T *)p.vc + d.vc.at(b, 0, hk) + c;
    const float sl2 = d.scale * kLog2e;

    float q[GT][8], acc[GT][8], m[GT], l[GT];
#pragma unroll
    for (int g = 0; g < GT; ++g) {
        m[g] = -INFINITY;
        l[g] = 0.f;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            q[g][e] = g < heads ? sq[g][c + e] * sl2 : 0.f;
            acc[g][e] = 0.f;
        }
    }
    if (split == 0 && grp == 0) {   // the new token itself
        float v[8];
        load8<T, false>((const T *)p.v + d.v.at(b, 0, hk) + c, v);
#pragma unroll
        for (int g = 0; g < GT; ++g) {
            float s = 0.f;
#pragma unroll
            for (int e = 0; e < 8; ++e) s = fmaf(q[g][e], sk[c + e], s);
#pragma unroll
            for (int o = LK / 2; o > 0; o >>= 1)
                s += __shfl_xor_sync((LK == 32 ? 0xffffffffu : (1u << LK) - 1u), s, o);
            m[g] = s;
            l[g] = 1.f;
#pragma unroll
            for (int e = 0; e < 8; ++e) acc[g][e] = v[e];
        }
    }
    __syncwarp();
    for (int u0 = lo + warp * kRows * kKeys; u0 < hi; u0 += kWarps * kRows * kKeys) {
        float kx[kKeys][8], vx[kKeys][8];
        bool on[kKeys];
#pragma unroll
        for (int j = 0; j < kKeys; ++j) {
            const int u = u0 + j * kRows + lane / LK;
            on[j] = u < hi;
            int slot = u < nS ? u : s0 + (u - nS);
            if (slot >= d.C) slot -= ring;
            if (on[j]) {
                load8<T, VEC>(Kb + (long long)slot * d.kc.t, kx[j]);
                load8<T, VEC>(Vb + (long long)slot * d.vc.t, vx[j]);
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
    // join the rows of a warp, then the warps
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
    __syncthreads();
    for (int e = threadIdx.x; e < heads * HD; e += kThreads) {
        const int g = e / HD, x = e % HD, h = hk * G + g0 + g;
        float M = -INFINITY, L = 0.f, o = 0.f;
#pragma unroll
        for (int w = 0; w < kWarps; ++w) M = fmaxf(M, sm_m[w][g]);
#pragma unroll
        for (int w = 0; w < kWarps; ++w) {
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

int heads_of(const Decode &d) {   // query heads a CTA takes
    const int G = d.H / d.Hkv;
    return G == 1 ? 1 : G == 2 ? 2 : G <= 4 ? 4 : 8;
}

int splits_of(const Decode &d) {
    const int G = d.H / d.Hkv, GT = heads_of(d), chunks = (G + GT - 1) / GT;
    const long long ctas = (long long)d.B * d.Hkv * chunks;
    const long long seen = (long long)d.sinks + d.window;
    const long long want = (2 * 152 + ctas - 1) / ctas, most = (seen + 127) / 128;
    long long s = want < most ? want : most;
    return (int)(s < 1 ? 1 : s > kMaxSplits ? kMaxSplits : s);
}

template <class T, bool VEC, int HD>
cudaError_t launch_hd(const DecodeArgs &p, const Turns &tab, cudaStream_t s) {
    const dim3 grid(p.splits * p.chunks, p.d.Hkv, p.d.B);
    switch (heads_of(p.d)) {
        case 1: window_decode_kernel<T, VEC, HD, 1><<<grid, kThreads, 0, s>>>(p, tab); break;
        case 2: window_decode_kernel<T, VEC, HD, 2><<<grid, kThreads, 0, s>>>(p, tab); break;
        case 4: window_decode_kernel<T, VEC, HD, 4><<<grid, kThreads, 0, s>>>(p, tab); break;
        default: window_decode_kernel<T, VEC, HD, 8><<<grid, kThreads, 0, s>>>(p, tab); break;
    }
    note_launches(1);
    cudaError_t e = cudaGetLastError();
    if (e != cudaSuccess || p.splits == 1) return e;
    e = launch_pdl(decode_join_kernel<T>, dim3(p.d.H, p.d.B), dim3(HD), 0, s, p);
    note_launches(1);
    return e;
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
    const int splits = splits_of(d), GT = heads_of(d), G = d.H / d.Hkv;
    DecodeArgs p{d, q, k, v, gq, gk, Kc, Vc, O, lens, splits, (G + GT - 1) / GT, (float *)ws,
                 (float2 *)((char *)ws + partial_bytes(d, splits))};
    const Turns tab = make_turns(d.rotary, d.theta);
    const bool vec = rows16(Kc, d.kc, d.bf16) && rows16(Vc, d.vc, d.bf16);
    if (d.bf16) return vec ? launch_of<bf16, true>(p, tab, s) : launch_of<bf16, false>(p, tab, s);
    return vec ? launch_of<float, true>(p, tab, s) : launch_of<float, false>(p, tab, s);
}

}  // namespace win
}  // namespace mosa
