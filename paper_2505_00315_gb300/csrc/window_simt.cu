// Window attention on CUDA cores: fp32 storage, and any strides or alignment
// that the tensor-core kernels do not take.
//
// For a query at position p over its visible tokens t (window_tiles.cuh)
//     S = scale q k_t,  P = softmax(S),  O = sum P v,  lse = log sum exp S
// and backward, with D = sum(dO o O) and P recomputed from lse,
//     dP = dO v,  dS = P (dP - D),  dq = scale sum dS k,
//     dk = scale sum dS q,  dv = sum P dO      (over queries and the heads of a group).
// One CTA of 256 threads per 64-row tile: 64 x 64 scores a step, four by four a
// thread, operands as fp32 in shared memory, the softmax's running maximum and
// sum in registers.  The backward takes one kernel by key tiles (dk, dv) and one by
// query tiles (dq), so that every sum runs in one thread in a fixed order.
// B2 T1000, 12 heads of 64, window 125, fp32: ragged lengths: forward 43 us, dk and dv 85, dq 57; the
// FMA pipe is busy 36 to 42% of the time, shared memory 54 to 65%, the issue slots 55 to 61%.  What bounds them:
// operands from shared memory (a 16-byte load for every eight FMAs of a thread), 16 warps an
// SM whose tiles are loaded between barriers, and 384 CTAs for 304 places.  Packed FMAs changed nothing, three CTAs an SM at
// 80 registers took a third longer.
#include <algorithm>

#include "launch.h"
#include "profile.h"
#include "window_tiles.cuh"

namespace mosa {
namespace win {
namespace {

constexpr int kT = 64;         // rows of a tile, queries and keys
constexpr int kThreads = 256;
constexpr int kPS = kT + 4;    // stride of a tile of scores
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.69314718055994531f;

template <class T>
struct Ptrs {
    const T *q, *k, *v, *dO;
    T *o, *dq, *dk, *dv;
    float *partial;
    SinkSplit sinks;
    const int32_t *lens;
    float *lse;
    bf16 *rest;
    const float *lse_in, *delta;
    bool vec;   // rows of every input start at a multiple of 16 bytes
};

// Rows t0 .. t0+63 of one head into dst [64][HD + 4]; rows outside [lo, hi) are zeros.
template <int HD, class T>
__device__ __forceinline__ void load_tile(float *dst, const T *src, long long st, int t0, int lo,
                                          int hi, bool vec) {
    constexpr int E = 16 / sizeof(T), U = HD / E;
    for (int e = threadIdx.x; e < kT * U; e += kThreads) {
        const int r = e / U, u = e % U, t = t0 + r;
        float *d = dst + r * (HD + 4) + u * E;
        if (t < lo || t >= hi) {
#pragma unroll
            for (int x = 0; x < E; ++x) d[x] = 0.f;
            continue;
        }
        const T *s = src + (long long)t * st + u * E;
        if (vec) {
            alignas(16) T w[E];
            *reinterpret_cast<uint4 *>(w) = *reinterpret_cast<const uint4 *>(s);
#pragma unroll
            for (int x = 0; x < E; ++x) d[x] = to_f32(w[x]);
        } else {
#pragma unroll
            for (int x = 0; x < E; ++x) d[x] = to_f32(s[x]);
        }
    }
}

// acc[i][j] = <row ty*4+i of A, row tx+16j of B> over HD columns.
template <int HD>
__device__ __forceinline__ void dot_tiles(const float *A, const float *B, int ty, int tx,
                                          float (&acc)[4][4]) {
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[i][j] = 0.f;
#pragma unroll 2
    for (int d = 0; d < HD; d += 4) {
        float4 a[4], b[4];
#pragma unroll
        for (int i = 0; i < 4; ++i)
            a[i] = *reinterpret_cast<const float4 *>(A + (ty * 4 + i) * (HD + 4) + d);
#pragma unroll
        for (int j = 0; j < 4; ++j)
            b[j] = *reinterpret_cast<const float4 *>(B + (tx + 16 * j) * (HD + 4) + d);
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                acc[i][j] = fmaf(a[i].x, b[j].x, acc[i][j]);
                acc[i][j] = fmaf(a[i].y, b[j].y, acc[i][j]);
                acc[i][j] = fmaf(a[i].z, b[j].z, acc[i][j]);
                acc[i][j] = fmaf(a[i].w, b[j].w, acc[i][j]);
            }
    }
}

// The HD/16 columns of thread tx: runs of up to four, 16 runs side by side.
template <int HD>
__device__ __forceinline__ int col_of(int tx, int c) {
    constexpr int CW = HD / 16;
    return CW <= 4 ? tx * CW + c : (c >> 2) * 64 + tx * 4 + (c & 3);
}

// A hidden place's weight in a tile of scores.  What a query sees has +0 where it underflows, times
// whose row a NaN or an infinity is NaN.
constexpr float kHidden = -0.f;
__device__ __forceinline__ bool hidden(float w) { return __float_as_uint(w) == 0x80000000u; }

// acc[i][c] += sum_j W[ty*4+i][j] X[j][col_of(c)].  With `skip` a hidden place adds
// nothing whatever X holds (it may hold NaN).
template <int HD, bool kRowsFirst>
__device__ __forceinline__ void add_weighted(const float *W, const float *X, int ty, int tx,
                                             bool skip, float (&acc)[4][HD / 16]) {
    constexpr int CW = HD / 16;
#pragma unroll 2
    for (int j = 0; j < kT; j += 4) {
        float w[4][4];   // [row][step]
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float4 t = *reinterpret_cast<const float4 *>(
                kRowsFirst ? W + (ty * 4 + i) * kPS + j : W + (j + i) * kPS + ty * 4);
            if (kRowsFirst) {
                w[i][0] = t.x; w[i][1] = t.y; w[i][2] = t.z; w[i][3] = t.w;
            } else {
                w[0][i] = t.x; w[1][i] = t.y; w[2][i] = t.z; w[3][i] = t.w;
            }
        }
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            float x[CW];
            const float *row = X + (j + u) * (HD + 4);
            if constexpr (CW >= 4) {
#pragma unroll
                for (int c = 0; c < CW; c += 4) {
                    const float4 t = *reinterpret_cast<const float4 *>(row + (c >> 2) * 64 + tx * 4);
                    x[c] = t.x; x[c + 1] = t.y; x[c + 2] = t.z; x[c + 3] = t.w;
                }
            } else if constexpr (CW == 2) {
                const float2 t = *reinterpret_cast<const float2 *>(row + tx * 2);
                x[0] = t.x; x[1] = t.y;
            } else {
                x[0] = row[tx];
            }
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (!skip || !hidden(w[i][u])) {
#pragma unroll
                    for (int c = 0; c < CW; ++c) acc[i][c] = fmaf(w[i][u], x[c], acc[i][c]);
                }
        }
    }
}

template <int HD, class T>
__device__ __forceinline__ void store_row(T *dst, int tx, const float (&v)[HD / 16], float f) {
#pragma unroll
    for (int c = 0; c < HD / 16; ++c) dst[col_of<HD>(tx, c)] = from_f32<T>(v[c] * f);
}

__device__ __forceinline__ float max16(float x) {
#pragma unroll
    for (int o = 8; o > 0; o >>= 1) x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, o));
    return x;
}
__device__ __forceinline__ float sum16(float x) {
#pragma unroll
    for (int o = 8; o > 0; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
    return x;
}

template <int HD>
constexpr int tile_floats() { return kT * (HD + 4); }

template <int HD, class T>
__global__ void __launch_bounds__(kThreads, 2) window_fwd_simt_kernel(Attn a, Ptrs<T> p) {
    asm volatile("griddepcontrol.wait;" ::: "memory");
    extern __shared__ float sm[];
    float *sQ = sm, *sK = sQ + tile_floats<HD>(), *sV = sK + tile_floats<HD>(),
          *sP = sV + tile_floats<HD>();
    const Place at(blockIdx.x, a.H, a.B);
    const int h = at.h, b = at.b, hk = h / a.G();
    const int i0 = ((a.Tq + kT - 1) / kT - 1 - at.tile) * kT, off = a.Tk - a.Tq;
    const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
    const int len = seq_len(p.lens, b, a.Tk);
    const int pf = off + i0, pl = min(off + min(i0 + kT, a.Tq), len) - 1;
    float acc[4][HD / 16], m[4], l[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        m[i] = -INFINITY;
        l[i] = 0.f;
#pragma unroll
        for (int c = 0; c < HD / 16; ++c) acc[i][c] = 0.f;
    }
    if (pl >= pf) {
        load_tile<HD>(sQ, p.q + a.q.at(b, 0, h), a.q.t, i0, 0, pl - off + 1, p.vec);
        const KeyBlocks<kT> kb(pf, pl, a.window, a.sinks);
        const float sl2 = a.scale * kLog2e;
        for (int j = 0; j < kb.count(); ++j) {
            const int ks = kb.start(j);
            __syncthreads();
            load_tile<HD>(sK, p.k + a.k.at(b, 0, hk), a.k.t, ks, 0, len, p.vec);
            load_tile<HD>(sV, p.v + a.v.at(b, 0, hk), a.v.t, ks, 0, len, p.vec);
            __syncthreads();
            float s[4][4];
            dot_tiles<HD>(sQ, sK, ty, tx, s);
            const bool whole = kb.whole(j, pf, pl, a.window) && pl - pf == kT - 1;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int pos = pf + ty * 4 + i;
                float mb = -INFINITY;
                bool on[4];
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    on[c] = whole || (pos <= pl && kb.sees(j, ks, tx + 16 * c, pos, a.window, a.sinks));
                    s[i][c] = on[c] ? s[i][c] * sl2 : -INFINITY;
                    mb = fmaxf(mb, s[i][c]);
                }
                // (fmax drops a NaN; the exponentials keep it)
                const float mn = fmaxf(m[i], max16(mb));
                const float base = mn == -INFINITY ? 0.f : mn;
                const float corr = exp2f(m[i] - base);
                float sum = 0.f;
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    const float e = exp2f(s[i][c] - base);
                    sum += e;
                    sP[(ty * 4 + i) * kPS + tx + 16 * c] = on[c] ? e : kHidden;
                }
                l[i] = l[i] * corr + sum16(sum);
                m[i] = mn;
#pragma unroll
                for (int c = 0; c < HD / 16; ++c) acc[i][c] *= corr;
            }
            __syncwarp();   // a row of sP is written and read by the 16 lanes of one half warp
            add_weighted<HD, true>(sP, sV, ty, tx, !whole, acc);
        }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int r = i0 + ty * 4 + i;
        if (r >= a.Tq) continue;
        // (l = 0 where all that a query sees has a score of -inf: 0 / 0 there)
        const bool seen = off + r <= pl;
        const float inv = seen ? 1.f / l[i] : 0.f;
        store_row<HD>(p.o + a.o.at(b, r, h), tx, acc[i], inv);
        if (p.rest != nullptr) {
#pragma unroll
            for (int c = 0; c < HD / 16; ++c) {
                const float o = acc[i][c] * inv;
                p.rest[a.packed().at(b, r, h) + col_of<HD>(tx, c)] =
                    from_f32<bf16>(o - to_f32(from_f32<T>(o)));
            }
        }
        if (p.lse != nullptr && tx == 0)
            p.lse[((long long)b * a.H + h) * a.Tq + r] =
                seen ? (m[i] + log2f(l[i])) * kLn2 : -INFINITY;
    }
}

// P (into sP, [query][key]) and dS (into sS) of one pair of tiles: queries at
// positions pq .. pq+63 (rows past `last` see nothing), keys ks .. ks+63.  What is seen never is
// kHidden: P is not negative, and dS has +0 added (a query that sees one token: 0 times dS, which
// stays NaN where that is).
template <int HD, class Sees>
__device__ __forceinline__ void grad_scores(const float *sQ, const float *sG, const float *sK,
                                            const float *sV, const float *sL, const float *sD,
                                            float sl2, bool whole, Sees sees, float *sP, float *sS,
                                            int ty, int tx, int pq, int window, int sinks) {
    float s[4][4], dp[4][4];
    dot_tiles<HD>(sQ, sK, ty, tx, s);
    dot_tiles<HD>(sG, sV, ty, tx, dp);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int r = ty * 4 + i;
        const float lse2 = sL[r], D = sD[r];
        const bool one = sees_one(pq + r, window, sinks);
#pragma unroll
        for (int c = 0; c < 4; ++c) {
            const bool on = whole || sees(r, tx + 16 * c);
            const float e = on ? exp2f(fmaf(s[i][c], sl2, -lse2)) : kHidden;
            if (sP != nullptr) sP[r * kPS + tx + 16 * c] = e;
            sS[r * kPS + tx + 16 * c] = on ? fmaf(e * (dp[i][c] - D), one ? 0.f : 1.f, 0.f) : kHidden;
        }
    }
}

// lse (in log2 units) and D of the queries i0 .. i0+63; rows outside [0, n) see nothing.
template <class T>
__device__ __forceinline__ void load_rows(float *sL, float *sD, const Ptrs<T> &p, long long row0,
                                          int i0, int n) {
    if (threadIdx.x < kT) {
        const int i = i0 + threadIdx.x;
        const bool ok = i >= 0 && i < n;
        sL[threadIdx.x] = ok ? p.lse_in[row0 + i] * kLog2e : 0.f;
        sD[threadIdx.x] = ok ? p.delta[row0 + i] : 0.f;
    }
}

// dq of one 64-query tile.
template <int HD, class T>
__global__ void __launch_bounds__(kThreads, HD <= 64 ? 2 : 1) window_dq_simt_kernel(Attn a, Ptrs<T> p) {
    asm volatile("griddepcontrol.wait;" ::: "memory");
    extern __shared__ float sm[];
    float *sQ = sm, *sG = sQ + tile_floats<HD>(), *sK = sG + tile_floats<HD>(),
          *sV = sK + tile_floats<HD>(), *sS = sV + tile_floats<HD>(), *sL = sS + kT * kPS,
          *sD = sL + kT;
    const Place at(blockIdx.x, a.H, a.B);
    const int h = at.h, b = at.b, hk = h / a.G();
    const int i0 = ((a.Tq + kT - 1) / kT - 1 - at.tile) * kT, off = a.Tk - a.Tq;
    const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
    const int len = seq_len(p.lens, b, a.Tk);
    const int pf = off + i0, pl = min(off + min(i0 + kT, a.Tq), len) - 1;
    float acc[4][HD / 16];
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int c = 0; c < HD / 16; ++c) acc[i][c] = 0.f;
    if (pl >= pf) {
        const long long row0 = ((long long)b * a.H + h) * a.Tq;
        load_tile<HD>(sQ, p.q + a.q.at(b, 0, h), a.q.t, i0, 0, pl - off + 1, p.vec);
        load_tile<HD>(sG, p.dO + a.go.at(b, 0, h), a.go.t, i0, 0, pl - off + 1, p.vec);
        load_rows(sL, sD, p, row0, i0, pl - off + 1);
        const KeyBlocks<kT> kb(pf, pl, a.window, a.sinks);
        for (int j = 0; j < kb.count(); ++j) {
            const int ks = kb.start(j);
            __syncthreads();
            load_tile<HD>(sK, p.k + a.k.at(b, 0, hk), a.k.t, ks, 0, len, p.vec);
            load_tile<HD>(sV, p.v + a.v.at(b, 0, hk), a.v.t, ks, 0, len, p.vec);
            __syncthreads();
            const bool whole = kb.whole(j, pf, pl, a.window) && pl - pf == kT - 1;
            grad_scores<HD>(
                sQ, sG, sK, sV, sL, sD, a.scale * kLog2e, whole,
                [&](int r, int c) {
                    return pf + r <= pl && kb.sees(j, ks, c, pf + r, a.window, a.sinks);
                },
                (float *)nullptr, sS, ty, tx, pf, a.window, a.sinks);
            __syncwarp();
            add_weighted<HD, true>(sS, sK, ty, tx, !whole, acc);
        }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int r = i0 + ty * 4 + i;
        if (r < a.Tq) store_row<HD>(p.dq + a.dq.at(b, r, h), tx, acc[i], a.scale);
    }
}

// dk and dv of one 64-key tile, over the queries that see it and the group's heads; the sinks'
// far queries in CTAs of their own (SinkSplit).
template <int HD, class T>
__global__ void __launch_bounds__(kThreads, HD <= 64 ? 2 : 1) window_dkv_simt_kernel(Attn a, Ptrs<T> p) {
    asm volatile("griddepcontrol.wait;" ::: "memory");
    extern __shared__ float sm[];
    float *sQ = sm, *sG = sQ + tile_floats<HD>(), *sK = sG + tile_floats<HD>(),
          *sV = sK + tile_floats<HD>(), *sS = sV + tile_floats<HD>(), *sP = sS + kT * kPS,
          *sL = sP + kT * kPS, *sD = sL + kT;
    const Place at(blockIdx.x, a.Hkv, a.B);
    const int hk = at.h, b = at.b, G = a.G(), off = a.Tk - a.Tq;
    const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
    const int len = seq_len(p.lens, b, a.Tk);
    const KeyTile<kT> kt(at.tile, a, p.sinks, len);
    const int k0 = kt.k0;
    float dk[4][HD / 16], dv[4][HD / 16];
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int c = 0; c < HD / 16; ++c) dk[i][c] = dv[i][c] = 0.f;
    if (k0 < len && kt.first <= kt.last) {
        load_tile<HD>(sK, p.k + a.k.at(b, 0, hk), a.k.t, k0, 0, len, p.vec);
        load_tile<HD>(sV, p.v + a.v.at(b, 0, hk), a.v.t, k0, 0, len, p.vec);
        for (int g = 0; g < G; ++g) {
            const int h = hk * G + g;
            const long long row0 = ((long long)b * a.H + h) * a.Tq;
            for (int pq = kt.first; pq <= kt.last; pq += kT) {
                const int i0 = pq - off, n = kt.last + 1 - off;
                __syncthreads();
                load_tile<HD>(sQ, p.q + a.q.at(b, 0, h), a.q.t, i0, 0, n, p.vec);
                load_tile<HD>(sG, p.dO + a.go.at(b, 0, h), a.go.t, i0, 0, n, p.vec);
                load_rows(sL, sD, p, row0, i0, n);
                __syncthreads();
                const bool whole = pq >= k0 + kT - 1 && pq + kT - 1 - k0 < a.window &&
                                   pq + kT - 1 <= kt.last && k0 + kT <= len;
                grad_scores<HD>(
                    sQ, sG, sK, sV, sL, sD, a.scale * kLog2e, whole,
                    [&](int r, int c) {
                        const int pos = pq + r, t = k0 + c;
                        return pos <= kt.last && t <= pos && (pos - t < a.window || t < a.sinks);
                    },
                    sP, sS, ty, tx, pq, a.window, a.sinks);
                __syncthreads();
                add_weighted<HD, false>(sP, sG, ty, tx, !whole, dv);
                add_weighted<HD, false>(sS, sQ, ty, tx, !whole, dk);
            }
        }
    }
    float *sums = p.partial + kt.partial_at(b, hk, a);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int t = k0 + ty * 4 + i;
        if (t >= a.Tk) continue;
        if (kt.has_sinks && t < a.sinks) {
#pragma unroll
            for (int c = 0; c < HD / 16; ++c) {
                sums[(long long)t * 2 * HD + col_of<HD>(tx, c)] = dk[i][c] * a.scale;
                sums[(long long)t * 2 * HD + HD + col_of<HD>(tx, c)] = dv[i][c];
            }
        } else if (kt.part == 0) {
            store_row<HD>(p.dk + a.dk.at(b, t, hk), tx, dk[i], a.scale);
            store_row<HD>(p.dv + a.dv.at(b, t, hk), tx, dv[i], 1.f);
        }
    }
}

// dk and dv of the sink rows: the tile's own sum and the other CTAs', in order.
template <class T>
__global__ void __launch_bounds__(256) window_sink_rows_kernel(Attn a, const float *partial, int extra,
                                                               T *dk, T *dv) {
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const int b = blockIdx.z, hk = blockIdx.y, t = blockIdx.x;
    const long long slot = (long long)a.sinks * 2 * a.hp;
    for (int e = threadIdx.x; e < 2 * a.hp; e += blockDim.x) {
        const float *s = partial + ((long long)b * a.Hkv + hk) * (extra + 1) * slot + (long long)t * 2 * a.hp + e;
        float sum = 0.f;
        for (int x = 0; x <= extra; ++x) sum += s[x * slot];
        if (e < a.hp) dk[a.dk.at(b, t, hk) + e] = from_f32<T>(sum);
        else dv[a.dv.at(b, t, hk) + e - a.hp] = from_f32<T>(sum);
    }
}

// D: eight values a lane, hp/8 lanes a row (a power of two), four such items a thread in flight.
// Reads O, dO and what O's rounding left once: memory bound.
constexpr int kDeltaItems = 4;

template <class T>
__global__ void __launch_bounds__(256) window_delta_kernel(Attn a, const T *O, const T *dO,
                                                           const bf16 *rest, float *delta, bool vec) {
    asm volatile("griddepcontrol.wait;" ::: "memory");
    constexpr int V = 8 * sizeof(T) / 16;
    const int lg = 31 - __clz(a.hp >> 3), U = a.H << lg;   // items of one token
    const long long all = (long long)a.B * a.Tq * U, base = (long long)blockIdx.x * (256 * kDeltaItems);
    const long long tok0 = base / U;
    const int rem0 = (int)(base - tok0 * U), b0 = (int)(tok0 / a.Tq), t0 = (int)(tok0 - (long long)b0 * a.Tq);
    const Str pk = a.packed();
    uint4 u[kDeltaItems][V], w[kDeltaItems][V], e[kDeltaItems];
    int bb[kDeltaItems], tt[kDeltaItems], hc[kDeltaItems];
#pragma unroll
    for (int i = 0; i < kDeltaItems; ++i) {
        const int x = rem0 + threadIdx.x + 256 * i, tok = x / U, r = x - tok * U;
        const int over = (t0 + tok) / a.Tq, b = b0 + over, t = t0 + tok - over * a.Tq;
        const int h = r >> lg, c = (r & ((1 << lg) - 1)) << 3;
        bb[i] = b;
        tt[i] = t;
        hc[i] = h;
        e[i] = make_uint4(0, 0, 0, 0);
        if (base + threadIdx.x + 256 * i >= all) {
            bb[i] = -1;
#pragma unroll
            for (int k = 0; k < V; ++k) u[i][k] = w[i][k] = make_uint4(0, 0, 0, 0);
            continue;
        }
        const T *po = O + a.o.at(b, t, h) + c, *pg = dO + a.go.at(b, t, h) + c;
        if (vec) {
#pragma unroll
            for (int k = 0; k < V; ++k) {
                u[i][k] = reinterpret_cast<const uint4 *>(po)[k];
                w[i][k] = reinterpret_cast<const uint4 *>(pg)[k];
            }
        } else {
            alignas(16) T x8[8], y8[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) x8[k] = po[k], y8[k] = pg[k];
#pragma unroll
            for (int k = 0; k < V; ++k) {
                u[i][k] = reinterpret_cast<const uint4 *>(x8)[k];
                w[i][k] = reinterpret_cast<const uint4 *>(y8)[k];
            }
        }
        if (rest != nullptr) e[i] = *reinterpret_cast<const uint4 *>(rest + pk.at(b, t, h) + c);
    }
#pragma unroll
    for (int i = 0; i < kDeltaItems; ++i) {
        float sum = 0.f;
        if constexpr (sizeof(T) == 4) {
#pragma unroll
            for (int k = 0; k < V; ++k) {
                sum = fmaf(__uint_as_float(u[i][k].x), __uint_as_float(w[i][k].x), sum);
                sum = fmaf(__uint_as_float(u[i][k].y), __uint_as_float(w[i][k].y), sum);
                sum = fmaf(__uint_as_float(u[i][k].z), __uint_as_float(w[i][k].z), sum);
                sum = fmaf(__uint_as_float(u[i][k].w), __uint_as_float(w[i][k].w), sum);
            }
        } else {
            const uint32_t ou[4] = {u[i][0].x, u[i][0].y, u[i][0].z, u[i][0].w};
            const uint32_t gu[4] = {w[i][0].x, w[i][0].y, w[i][0].z, w[i][0].w};
            const uint32_t eu[4] = {e[i].x, e[i].y, e[i].z, e[i].w};
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                sum = fmaf(__uint_as_float(ou[k] << 16) + __uint_as_float(eu[k] << 16),
                           __uint_as_float(gu[k] << 16), sum);
                sum = fmaf(__uint_as_float(ou[k] & 0xFFFF0000u) + __uint_as_float(eu[k] & 0xFFFF0000u),
                           __uint_as_float(gu[k] & 0xFFFF0000u), sum);
            }
        }
        for (int o = 1 << lg >> 1; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
        if (bb[i] >= 0 && (threadIdx.x & ((1 << lg) - 1)) == 0)
            delta[((long long)bb[i] * a.H + hc[i]) * a.Tq + tt[i]] = sum;
    }
}

template <int HD>
constexpr int fwd_smem() { return 4 * (3 * tile_floats<HD>() + kT * kPS); }
template <int HD>
constexpr int dq_smem() { return 4 * (4 * tile_floats<HD>() + kT * kPS + 2 * kT); }
template <int HD>
constexpr int dkv_smem() { return 4 * (4 * tile_floats<HD>() + 2 * kT * kPS + 2 * kT); }

template <class Kernel, class T>
cudaError_t go(Kernel kernel, dim3 grid, int smem, const Attn &a, const Ptrs<T> &p, cudaStream_t s) {
    cudaError_t e = allow_smem((const void *)kernel, smem);
    if (e != cudaSuccess) return e;
    e = launch_pdl(kernel, grid, dim3(kThreads), smem, s, a, p);
    note_launches(1);
    return e;
}

template <class T>
cudaError_t fwd(const Attn &a, const Ptrs<T> &p, cudaStream_t s) {
    const dim3 grid = grid_of((a.Tq + kT - 1) / kT, a.H, a.B);
    switch (a.hp) {
        case 16: return go(window_fwd_simt_kernel<16, T>, grid, fwd_smem<16>(), a, p, s);
        case 32: return go(window_fwd_simt_kernel<32, T>, grid, fwd_smem<32>(), a, p, s);
        case 64: return go(window_fwd_simt_kernel<64, T>, grid, fwd_smem<64>(), a, p, s);
        default: return go(window_fwd_simt_kernel<128, T>, grid, fwd_smem<128>(), a, p, s);
    }
}

template <int HD, class T>
cudaError_t bwd_hd(const Attn &a, const Ptrs<T> &p, cudaStream_t s) {
    const dim3 gk = grid_of(p.sinks.ctas(a, kT), a.Hkv, a.B), gq = grid_of((a.Tq + kT - 1) / kT, a.H, a.B);
    cudaError_t e = go(window_dkv_simt_kernel<HD, T>, gk, dkv_smem<HD>(), a, p, s);
    if (e == cudaSuccess) e = go(window_dq_simt_kernel<HD, T>, gq, dq_smem<HD>(), a, p, s);
    return e != cudaSuccess ? e : add_sink_rows(a, p.partial, p.sinks.extra, p.dk, p.dv, s);
}

template <class T>
cudaError_t bwd(const Attn &a, const Ptrs<T> &p, cudaStream_t s) {
    switch (a.hp) {
        case 16: return bwd_hd<16>(a, p, s);
        case 32: return bwd_hd<32>(a, p, s);
        case 64: return bwd_hd<64>(a, p, s);
        default: return bwd_hd<128>(a, p, s);
    }
}

template <class T>
Ptrs<T> ptrs(const Attn &a, const void *q, const void *k, const void *v, const int32_t *lens) {
    Ptrs<T> p{};
    p.q = (const T *)q;
    p.k = (const T *)k;
    p.v = (const T *)v;
    p.lens = lens;
    p.vec = rows16(q, a.q, a.bf16) && rows16(k, a.k, a.bf16) && rows16(v, a.v, a.bf16);
    return p;
}

template <class T>
cudaError_t fwd_of(const Attn &a, const void *q, const void *k, const void *v, const int32_t *lens,
                   void *O, float *lse, bf16 *rest, cudaStream_t s) {
    Ptrs<T> p = ptrs<T>(a, q, k, v, lens);
    p.o = (T *)O;
    p.lse = lse;
    p.rest = rest;
    return fwd<T>(a, p, s);
}

template <class T>
cudaError_t bwd_of(const Attn &a, const void *q, const void *k, const void *v, const int32_t *lens,
                   const float *lse, const void *dO, const float *delta, void *dq, void *dk,
                   void *dv, float *partial, cudaStream_t s) {
    Ptrs<T> p = ptrs<T>(a, q, k, v, lens);
    p.partial = partial;
    p.sinks = SinkSplit(a, kT);
    p.vec = p.vec && rows16(dO, a.go, a.bf16);
    p.dO = (const T *)dO;
    p.lse_in = lse;
    p.delta = delta;
    p.dq = (T *)dq;
    p.dk = (T *)dk;
    p.dv = (T *)dv;
    return bwd<T>(a, p, s);
}

}  // namespace

cudaError_t simt_window_fwd(const Attn &a, const void *q, const void *k, const void *v,
                            const int32_t *lens, void *O, float *lse, bf16 *rest, cudaStream_t s) {
    return a.bf16 ? fwd_of<bf16>(a, q, k, v, lens, O, lse, rest, s)
                  : fwd_of<float>(a, q, k, v, lens, O, lse, nullptr, s);
}

cudaError_t simt_window_bwd(const Attn &a, const void *q, const void *k, const void *v,
                            const int32_t *lens, const float *lse, const void *dO,
                            const float *delta, void *dq, void *dk, void *dv, float *partial,
                            cudaStream_t s) {
    return a.bf16 ? bwd_of<bf16>(a, q, k, v, lens, lse, dO, delta, dq, dk, dv, partial, s)
                  : bwd_of<float>(a, q, k, v, lens, lse, dO, delta, dq, dk, dv, partial, s);
}

cudaError_t add_sink_rows(const Attn &a, const float *partial, int extra, void *dk, void *dv,
                          cudaStream_t s) {
    if (extra == 0) return cudaSuccess;
    const dim3 grid(a.sinks, a.Hkv, a.B);
    const cudaError_t e =
        a.bf16 ? launch_pdl(window_sink_rows_kernel<bf16>, grid, dim3(256), 0, s, a, partial, extra, (bf16 *)dk, (bf16 *)dv)
               : launch_pdl(window_sink_rows_kernel<float>, grid, dim3(256), 0, s, a, partial, extra, (float *)dk, (float *)dv);
    note_launches(1);
    return e;
}

// The larger of both kernels' tiles: which one runs hangs on the tensors' places.
size_t window_bwd_bytes(const Attn &a) {
    const size_t x = SinkSplit(a, kT).bytes(a);
    return a.bf16 ? std::max(x, SinkSplit(a, kTcTile).bytes(a)) : x;
}

cudaError_t window_delta(const Attn &a, const void *O, const bf16 *rest, const void *dO, float *delta,
                         cudaStream_t s) {
    const long long n = (long long)a.B * a.Tq * a.H * (a.hp / 8);
    const bool vec = rows16(O, a.o, a.bf16) && rows16(dO, a.go, a.bf16);
    const dim3 grid((unsigned)((n + 256 * kDeltaItems - 1) / (256 * kDeltaItems)));
    const cudaError_t e =
        a.bf16 ? launch_pdl(window_delta_kernel<bf16>, grid, dim3(256), 0, s, a, (const bf16 *)O, (const bf16 *)dO, rest, delta, vec)
               : launch_pdl(window_delta_kernel<float>, grid, dim3(256), 0, s, a, (const float *)O, (const float *)dO,
                            (const bf16 *)nullptr, delta, vec);
    note_launches(1);
    return e;
}

}  // namespace win
}  // namespace mosa
