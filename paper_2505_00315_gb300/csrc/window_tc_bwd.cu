// Sliding-window attention with sinks on the tensor cores, backward (bf16).
//
// P is computed again from the forward's lse; with D = sum(dO o O) per query
//     S = Q K^T,  P = exp(scale S - lse),  dP = dO V^T,  dS = P (dP - D)
//     dV = P^T dO,  dK = scale dS^T Q,  dQ = scale dS K
// in two parts, so that every sum runs in one accumulator in a fixed order:
//   dK, dV  one CTA per (128-key tile, key / value head, sequence), or one an SM for some of them, over
//           the 128-query blocks of the group's heads that see it.  Scores are taken transposed
//           (S^T = K Q^T), so that P^T and dS^T, bf16 in TMEM in the place of the
//           scores, are the A operands of dV and dK with no pass through shared memory.
//   dQ      one CTA an SM, for some (128-query tile, head, sequence) each, over the key blocks they meet.
//           dS goes into two products, what bf16 holds of it and what that leaves: a query's dS are
//           differences that cancel in its sum, and one rounding of them was 1.5 times the error of
//           a form that rounds only what it stores.  (dK and dV sum over many queries, whose
//           roundings are independent: 1.4 times; in two parts where few tokens are seen.)  Costs 512 of 2048 + 512 cycles of MMAs a block.
// CTAs of both are one grid, dQ's first (see window_grad_tc_kernel).
// One part with five products instead of the eight here would have to add dQ up
// from several CTAs: 64 KB of fp32 reductions per pair of tiles against 2560
// cycles of MMAs (hp = 128), in an order that changes from run to run, and a pass to zero
// and one to round it.
// B4 T4096, 16 + 4 heads of 128, window 1024: 373 us, of which dQ about a half (the tensor pipe is busy 67% of
// them; the rest is the chain scores -> weights -> product within a block and, with one CTA an
// SM, its beginning and end).  B2 T8192, 4 heads of 64, window 512: 66 us, where MMAs take a third of
// the cycles and the elementwise work of a block is what counts.
// Keys that are sinks are seen by every later query: those queries beyond the
// tile's window go to CTAs of their own, some blocks each, whose fp32 sums for the
// sink rows a last small kernel adds up in order (else the first tile's CTA would
// outlast the others by Tk / window).
//
// Sixteen warps compute (four per TMEM lane quadrant, each a quarter of the columns), one
// loads by TMA, one issues the MMAs, one more (dK, dV) brings lse and D.  While MMAs
// of one block run, the workers turn the other scores: the queue of MMAs is
//   dK, dV:  dV_i S_i+1 | dK_i dP_i+1        dQ:  dP_j+1 dQ_j S_j+2
// so that products always cover the elementwise work of the next scores.
//
// Where a pair of tiles is seen in part, the masked places have P = dS = 0; a NaN or
// infinity in an operand row that meets them would still make a NaN of them.  dK, dV:
// query rows whose lse or D is not finite are zeroed in shared memory (their P is NaN where it
// is seen).  dQ: a CTA whose results are not all finite runs a second time with such rows of
// K zeroed (a query that sees one has lse NaN).
#include <algorithm>

#include "launch.h"
#include "profile.h"
#include "window_tc.cuh"

namespace mosa {
namespace win {
namespace {

constexpr int kTile = kTcTile;
constexpr int kWarps = 16, kWorkers = 32 * kWarps;   // the workers'
constexpr int kCols = 128 / (kWarps / 4);            // score columns of one worker thread

struct BwdArgs {
    Map q, k, v, go;
    const int32_t *lens;
    const float *lse, *delta;           // [B, H, Tq]
    bf16 *dQ, *dK, *dV;
    Str sdq, sdk, sdv;
    int wide_dq, wide_dk, wide_dv;      // rows of these start at a multiple of 32 bytes
    float *partial;                     // [B, Hkv, slots, sinks, 2, hp] fp32: dk, dv of the sink rows
    uint32_t *status;
    uint32_t wait_ns;
    Attn a;
    SinkSplit split;
    int Tq, Tk, H, Hkv, G, hp, window, sinks;
    float scale, scale_log2;
    uint32_t q_ctas, q_tiles, kv_tiles;  // CTAs and tiles of dQ, tiles of dK, dV
};

// Which of a part's CTAs this is: it takes tiles x, x + ctas, x + 2 ctas ..
struct Share {
    uint32_t x, ctas;
};

// Threads of a CTA: the workers, the loader, the issuer and (dK, dV) one warp for lse and D.
constexpr int kThreads = kWorkers + 96;

// 32 values as bf16 into the 16 TMEM columns at taddr.
__device__ __forceinline__ void put_weights(uint32_t taddr, const float (&v)[32]) {
    uint32_t w[16];
#pragma unroll
    for (int e = 0; e < 16; ++e) w[e] = pack_bf16x2(v[2 * e], v[2 * e + 1]);
    tmem_st16_async(taddr, w);
    tmem_stored();
    tc_fence_before();
}

// The same in two parts: what bf16 holds of them, and 16 columns on what their rounding leaves.
__device__ __forceinline__ void put_weights_split(uint32_t taddr, const float (&v)[32]) {
    uint32_t w[16], y[16];
#pragma unroll
    for (int e = 0; e < 16; ++e) {
        w[e] = pack_bf16x2(v[2 * e], v[2 * e + 1]);
        y[e] = pack_bf16x2(v[2 * e] - __uint_as_float(w[e] << 16),
                           v[2 * e + 1] - __uint_as_float(w[e] & 0xFFFF0000u));
    }
    tmem_st16_async(taddr, w);
    tmem_st16_async(taddr + 16, y);
    tmem_stored();
    tc_fence_before();
}

// ------------------------------------------------------------------ dK, dV

template <int HD>
struct KvSm {
    static constexpr int NB = HD / 64;
    uint8_t k[NB][kBlk], v[NB][kBlk];
    uint8_t q[3][NB][kBlk], go[2][NB][kBlk];
    float lse[2][kTile], delta[2][kTile];      // of a block's queries (lse in log2 units)
    uint64_t kv_full, kv_empty, q_full[3], q_empty[3], g_full[2], g_empty[2], st_full[2], st_empty[2];
    uint64_t s_full, dp_full, p_ready, ds_ready, done, drained;
    uint32_t odd[2][4];                        // queries of the block with lse or D not finite
    uint32_t tmem;
    int abort;
};

// The x-th key tile of all and the (head of the group, block) pairs that see it, heads outermost.
struct KeyWork {
    int b, hk, len, blocks, n;
    KeyTile<kTile> kt;
    __device__ __forceinline__ KeyWork(const BwdArgs &p, const Place &at)
        : b(at.b), hk(at.h), len(seq_len(p.lens, at.b, p.Tk)), kt(at.tile, p.a, p.split, len) {
        blocks = kt.first <= kt.last && kt.k0 < len ? (kt.last - kt.first) / kTile + 1 : 0;
        n = blocks * p.G;
    }
    __device__ __forceinline__ KeyWork(const BwdArgs &p, uint32_t x) : KeyWork(p, Place(x, p.Hkv, p.a.B)) {}
};

// kSplit (few_terms, as in the forward): what P and dS lose by their rounding goes into second
// products.
template <int HD, bool kSplit>
__device__ __forceinline__ void key_grads(const BwdArgs &p, uint8_t *smem, const Share cta) {
    using Sm = KvSm<HD>;
    constexpr int NB = Sm::NB;
    Sm &sm = *reinterpret_cast<Sm *>(smem);
    const uint32_t all = p.kv_tiles;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int off = p.Tk - p.Tq;
    if (threadIdx.x == 0) {
        mbar_init(smem_u32(&sm.kv_full), 1);
        mbar_init(smem_u32(&sm.kv_empty), 1);
        for (int s = 0; s < 3; ++s) {
            mbar_init(smem_u32(&sm.q_full[s]), 1);
            mbar_init(smem_u32(&sm.q_empty[s]), 1);
        }
        for (int s = 0; s < 2; ++s) {
            mbar_init(smem_u32(&sm.g_full[s]), 1);
            mbar_init(smem_u32(&sm.g_empty[s]), 1);
            mbar_init(smem_u32(&sm.st_full[s]), 1);
            mbar_init(smem_u32(&sm.st_empty[s]), kWarps);
        }
        mbar_init(smem_u32(&sm.s_full), 1);
        mbar_init(smem_u32(&sm.dp_full), 1);
        mbar_init(smem_u32(&sm.p_ready), kWarps);
        mbar_init(smem_u32(&sm.ds_ready), kWarps);
        mbar_init(smem_u32(&sm.done), 1);
        mbar_init(smem_u32(&sm.drained), 1);
        sm.abort = 0;
        fence_barrier_init();
    }
    if (warp == kWarps) {
        tmem_alloc(smem_u32(&sm.tmem), 512);
        tmem_relinquish();
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tS = sm.tmem, tG = tS + 128, tdV = tS + 256, tdK = tS + 384;
    auto wait = [&](uint64_t &bar, uint32_t parity) {
        return wait_or_abort(bar, parity, &sm.abort, p.status, p.wait_ns);
    };

    // Tiles with something to see and their blocks are numbered on (it, g).
    int it = 0, g = 0;
    bool ok = true;
    if (warp == kWarps) {
        if (lane == 0) {
            int nq = 0, ng = 0;
            for (uint32_t x = cta.x; x < all && ok; x += cta.ctas) {
                const KeyWork w(p, x);
                if (w.n == 0) continue;
                if (!(ok = wait(sm.kv_empty, (it & 1) ^ 1))) break;
                ++it;
                const uint32_t kvb = smem_u32(&sm.kv_full);
                mbar_expect_tx(kvb, 2 * NB * kBlk);
                for (int c = 0; c < NB; ++c) {
                    load_box(smem_u32(sm.k[c]), p.k, kvb, 64 * c, w.kt.k0, w.hk, w.b);
                    load_box(smem_u32(sm.v[c]), p.v, kvb, 64 * c, w.kt.k0, w.hk, w.b);
                }
                for (int i = 0; i < w.n; ++i, ++g) {
                    const int h = w.hk * p.G + i / w.blocks, i0 = w.kt.first - off + kTile * (i % w.blocks);
                    if (!(ok = wait(sm.q_empty[g % 3], ((g / 3) & 1) ^ 1))) break;
                    mbar_expect_tx(smem_u32(&sm.q_full[g % 3]), NB * kBlk);
                    for (int c = 0; c < NB; ++c)
                        load_box(smem_u32(sm.q[g % 3][c]), p.q, smem_u32(&sm.q_full[g % 3]), 64 * c, i0, h, w.b);
                    nq = g + 1;
                    if (!(ok = wait(sm.g_empty[g & 1], ((g >> 1) & 1) ^ 1))) break;
                    mbar_expect_tx(smem_u32(&sm.g_full[g & 1]), NB * kBlk);
                    for (int c = 0; c < NB; ++c)
                        load_box(smem_u32(sm.go[g & 1][c]), p.go, smem_u32(&sm.g_full[g & 1]), 64 * c, i0, h, w.b);
                    ng = g + 1;
                }
            }
            // what was loaded has landed
            if (it > 0) drain_phase(smem_u32(&sm.kv_full), (it - 1) & 1);
            for (int t = max(0, nq - 3); t < nq; ++t) drain_phase(smem_u32(&sm.q_full[t % 3]), (t / 3) & 1);
            for (int t = max(0, ng - 2); t < ng; ++t) drain_phase(smem_u32(&sm.g_full[t & 1]), (t >> 1) & 1);
        }
    } else if (warp == kWarps + 1) {
        if (elect_one()) {
            constexpr uint32_t idS = idesc_bf16(128, 128, false, false);
            constexpr uint32_t idG = idesc_bf16(128, HD, false, true);
            const uint64_t dk = k_major(sm.k), dv = k_major(sm.v);
            auto s_of = [&](int g) {
                ok = ok && wait(sm.q_full[g % 3], (g / 3) & 1);
                if (!ok) return;
                tc_fence_after();
                mma_scores<NB>(tS, dk, k_major(sm.q[g % 3]), idS);
                mma_commit(smem_u32(&sm.s_full));
            };
            // (`free`: the last product of the tile that reads K and V)
            auto dp_of = [&](int g, bool free) {
                ok = ok && wait(sm.g_full[g & 1], (g >> 1) & 1);
                if (!ok) return;
                tc_fence_after();
                mma_scores<NB>(tG, dv, k_major(sm.go[g & 1]), idS);
                mma_commit(smem_u32(&sm.dp_full));
                if (free) mma_commit(smem_u32(&sm.kv_empty));
            };
            auto next_of = [&](uint32_t x, int &n) {   // the next tile with something to see
                for (n = 0; x < all; x += cta.ctas)
                    if ((n = KeyWork(p, x).n) > 0) break;
                return x;
            };
            int n, n_next;
            uint32_t x = next_of(cta.x, n);
            if (x < all) {
                ok = wait(sm.kv_full, 0);
                s_of(0);
                dp_of(0, n == 1);
            }
            while (x < all && ok) {
                const uint32_t x_next = next_of(x + cta.ctas, n_next);
                for (int i = 0; i < n && ok; ++i, ++g) {
                    const bool last = i + 1 == n, more = !last || x_next < all;
                    ok = wait(sm.p_ready, g & 1);
                    if (!ok) break;
                    tc_fence_after();
                    mma_weights<5>(tdV, tS, mn_major(sm.go[g & 1]), idG, i > 0);
                    if (kSplit) mma_weights<5>(tdV, tS + 16, mn_major(sm.go[g & 1]), idG, true);
                    mma_commit(smem_u32(&sm.g_empty[g & 1]));
                    if (!last) s_of(g + 1);
                    ok = ok && wait(sm.ds_ready, g & 1);
                    if (!ok) break;
                    tc_fence_after();
                    mma_weights<5>(tdK, tG, mn_major(sm.q[g % 3]), idG, i > 0);
                    if (kSplit) mma_weights<5>(tdK, tG + 16, mn_major(sm.q[g % 3]), idG, true);
                    mma_commit(smem_u32(&sm.q_empty[g % 3]));
                    if (last) mma_commit(smem_u32(&sm.done));
                    if (last && more) {
                        ok = wait(sm.kv_full, (it + 1) & 1);
                        s_of(g + 1);
                    }
                    if (more) dp_of(g + 1, last ? n_next == 1 : i + 2 == n);
                }
                ++it;
                x = x_next;
                n = n_next;
            }
            if (!ok) {
                mma_commit(smem_u32(&sm.done));
                mma_commit(smem_u32(&sm.s_full));
                mma_commit(smem_u32(&sm.dp_full));
            }
            drain_mmas(smem_u32(&sm.drained));
        }
    } else if (warp == kWarps + 2) {
        for (uint32_t x = cta.x; x < all && ok; x += cta.ctas) {
            const KeyWork w(p, x);
            for (int i = 0; i < w.n; ++i, ++g) {
                const int u = g & 1;
                if (!(ok = __all_sync(0xffffffffu, wait(sm.st_empty[u], ((g >> 1) & 1) ^ 1)))) break;
                const int pq = w.kt.first + kTile * (i % w.blocks);
                const long long row = ((long long)w.b * p.H + w.hk * p.G + i / w.blocks) * p.Tq + pq - off;
#pragma unroll
                for (int y = 0; y < 4; ++y) {
                    const int c = 32 * y + lane;
                    const bool on = pq + c < w.len;   // (len <= Tk)
                    float L = on ? p.lse[row + c] * kLog2e : 0.f, D = on ? p.delta[row + c] : 0.f;
                    const bool odd = !(fabsf(L) < INFINITY) || !(fabsf(D) < INFINITY);
                    if (odd) L = NAN;
                    sm.lse[u][c] = L;
                    sm.delta[u][c] = D;
                    // rows past the length are hidden from every key, whatever they hold (past Tk
                    // they were read as zeros)
                    const uint32_t m = __ballot_sync(0xffffffffu, on ? odd : pq + c < p.Tk);
                    if (lane == 0) sm.odd[u][y] = m;
                }
                warp_arrive(sm.st_full[u], lane);
            }
        }
    } else {
        const int c0 = kCols * (warp >> 2), r = (warp & 3) * 32 + lane;
        const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16, at = lanes + c0;
        const int d0 = (warp >> 2) * (HD / 4);   // this thread's quarter of the columns of dK and dV
        const float2 sl2 = make_float2(p.scale_log2, p.scale_log2);
        for (uint32_t x = cta.x; x < all && !giving_up(&sm.abort); x += cta.ctas) {
            const KeyWork w(p, x);
            const int k0 = w.kt.k0, last = w.kt.last, t = k0 + r;
            int pq = w.kt.first, i_blk = 0;
#pragma unroll 1
            for (int i = 0; i < w.n; ++i, ++g) {
                const int u = g & 1;
                const bool whole = pq >= k0 + kTile - 1 && pq + kTile - 1 - k0 < p.window &&
                                   pq + kTile - 1 <= last;
                uint32_t seen = ~0u;   // which of this thread's queries see its key
                if (!whole)
                    seen = bits(t - pq - c0, min(last, t < p.sinks ? last : t + p.window - 1) - pq - c0);
                const float *L = sm.lse[u] + c0, *D = sm.delta[u] + c0;
                wait(sm.st_full[u], (g >> 1) & 1);
                wait(sm.s_full, g & 1);
                tc_fence_after();
                float raw[32];
                tmem_get32(tS + at, raw);
                float P[32];
#pragma unroll
                for (int c = 0; c < 32; c += 4) {
                    const float4 l4 = *reinterpret_cast<const float4 *>(L + c);
                    const float2 x = fma2(make_float2(raw[c], raw[c + 1]), sl2,
                                          make_float2(-l4.x, -l4.y));
                    const float2 y = fma2(make_float2(raw[c + 2], raw[c + 3]),
                                          sl2, make_float2(-l4.z, -l4.w));
                    P[c] = exp2_fast(x.x);
                    P[c + 1] = exp2_fast(x.y);
                    P[c + 2] = exp2_fast(y.x);
                    P[c + 3] = exp2_fast(y.y);
                }
                if (!whole) {
                    hide(P, seen, 0.f);
                    if ((sm.odd[u][0] | sm.odd[u][1] | sm.odd[u][2] | sm.odd[u][3]) != 0) {
                        // zero those queries' rows, once S and dP have been taken from them
                        wait(sm.dp_full, g & 1);
                        const int row = threadIdx.x & 127;
                        if (threadIdx.x < 256 && ((sm.odd[u][row >> 5] >> (row & 31)) & 1u) != 0) {
                            uint8_t *x = threadIdx.x < 128 ? sm.q[g % 3][0] : sm.go[g & 1][0];
#pragma unroll 1
                            for (int e = 0; e < 8 * NB; ++e)
                                *reinterpret_cast<uint4 *>(x + (e >> 3) * kBlk + row * 128 + (e & 7) * 16) =
                                    make_uint4(0, 0, 0, 0);
                        }
                        fence_proxy_async();
                    }
                }
                kSplit ? put_weights_split(tS + at, P) : put_weights(tS + at, P);
                warp_arrive(sm.p_ready, lane);

                wait(sm.dp_full, g & 1);
                tc_fence_after();
                tmem_get32(tG + at, raw);
#pragma unroll
                for (int c = 0; c < 32; c += 4) {
                    const float4 d4 = *reinterpret_cast<const float4 *>(D + c);
                    const float2 x = mul2(make_float2(P[c], P[c + 1]),
                                          add2(make_float2(raw[c], raw[c + 1]),
                                               make_float2(-d4.x, -d4.y)));
                    const float2 y = mul2(make_float2(P[c + 2], P[c + 3]),
                                          add2(make_float2(raw[c + 2], raw[c + 3]),
                                               make_float2(-d4.z, -d4.w)));
                    P[c] = x.x;
                    P[c + 1] = x.y;
                    P[c + 2] = y.x;
                    P[c + 3] = y.y;
                }
                if (!whole) {
                    // (again: dP may be NaN where P is 0; and a query that sees one token only has
                    // no gradient, but NaN where it meets one)
                    if (p.window == 1 && p.sinks == 0)
#pragma unroll
                        for (int c = 0; c < 32; ++c) P[c] *= 0.f;
                    if (pq == 0 && c0 == 0) P[0] *= 0.f;
                    hide(P, seen, 0.f);
                }
                kSplit ? put_weights_split(tG + at, P) : put_weights(tG + at, P);
                warp_arrive(sm.ds_ready, lane);
                if (lane == 0) mbar_arrive(smem_u32(&sm.st_empty[u]));
                pq += kTile;
                if (++i_blk == w.blocks) i_blk = 0, pq = w.kt.first;
            }
            float dv[HD / 64][16], dk[HD / 64][16];
            if (w.n > 0) {
                wait(sm.done, it & 1);
                ++it;
                tc_fence_after();
#pragma unroll
                for (int c = 0; c < HD / 64; ++c) {
                    tmem_ld16(tdV + lanes + d0 + 16 * c, dv[c]);
                    tmem_ld16(tdK + lanes + d0 + 16 * c, dk[c]);
                }
                tc_fence_before();   // (before the arrival for the next tile's first P)
            } else {   // no query sees the tile: zeros
#pragma unroll
                for (int c = 0; c < HD / 64; ++c)
#pragma unroll
                    for (int e = 0; e < 16; ++e) dv[c][e] = dk[c][e] = 0.f;
            }
            const bool sink = w.kt.has_sinks && t < p.sinks;
            const bool stores = t < p.Tk && (sink || w.kt.part == 0) && *(volatile int *)&sm.abort == 0;
#pragma unroll
            for (int c = 0; c < HD / 64; ++c) {
                const int d = d0 + 16 * c;
                if (!stores || d >= p.hp) break;
                if (sink) {
                    float *o = p.partial + w.kt.partial_at(w.b, w.hk, p.a) + (long long)t * 2 * p.hp + d;
#pragma unroll
                    for (int e = 0; e < 16; ++e) {
                        o[e] = dk[c][e] * p.scale;
                        o[p.hp + e] = dv[c][e];
                    }
                } else {
                    uint32_t wk[8], wv[8];
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        wk[e] = pack_bf16x2(dk[c][2 * e] * p.scale, dk[c][2 * e + 1] * p.scale);
                        wv[e] = pack_bf16x2(dv[c][2 * e], dv[c][2 * e + 1]);
                    }
                    store32(p.dK + p.sdk.at(w.b, t, w.hk) + d, wk, p.wide_dk);
                    store32(p.dV + p.sdv.at(w.b, t, w.hk) + d, wv, p.wide_dv);
                }
            }
            __syncwarp();
        }
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    if (warp == kWarps) tmem_dealloc(sm.tmem, 512);
}

// ---------------------------------------------------------------------- dQ

// CTAs stay for several tiles (one CTA an SM), so that a tile's loads and first scores run beside the
// end of the tile before: Q and dO are free once the last dP is done, and dQ is read out while the
// next scores are computed.
constexpr int kMaxTiles = 64;   // of one CTA

template <int HD>
struct QSm {
    static constexpr int NB = HD / 64;
    uint8_t q[NB][kBlk], go[NB][kBlk];
    uint8_t k[3][NB][kBlk], v[2][NB][kBlk];
    uint64_t q_full, q_empty, k_full[3], k_empty[3], v_full[2], v_empty[2];
    uint64_t s_full[2], dp_full, ds_ready, dq_full, dq_empty, drained;
    uint32_t tmem;
    int abort, redo;
    uint8_t again[kMaxTiles];   // tiles whose results are not all finite
};

// The x-th query tile of all, the heaviest first.
struct QueryTile {
    int b, h, i0, pf, pl;
    __device__ __forceinline__ QueryTile(const BwdArgs &p, uint32_t x, int tiles) {
        const Place at(x, p.H, p.a.B);
        i0 = (tiles - 1 - at.tile) * kTile;
        b = at.b;
        h = at.h;
        pf = p.Tk - p.Tq + i0;
        pl = min(p.Tk - p.Tq + min(i0 + kTile, p.Tq), seq_len(p.lens, b, p.Tk)) - 1;
    }
    __device__ __forceinline__ bool empty() const { return pl < pf; }
};

template <int HD>
__device__ __forceinline__ void query_grads(const BwdArgs &p, uint8_t *smem, const Share cta) {
    using Sm = QSm<HD>;
    constexpr int NB = Sm::NB;
    Sm &sm = *reinterpret_cast<Sm *>(smem);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, tiles = (p.Tq + kTile - 1) / kTile;
    const uint32_t all = p.q_tiles;
    if (threadIdx.x == 0) {
        mbar_init(smem_u32(&sm.q_full), 1);
        mbar_init(smem_u32(&sm.q_empty), 1);
        for (int s = 0; s < 3; ++s) {
            mbar_init(smem_u32(&sm.k_full[s]), 1);
            mbar_init(smem_u32(&sm.k_empty[s]), 1);
        }
        for (int s = 0; s < 2; ++s) {
            mbar_init(smem_u32(&sm.v_full[s]), 1);
            mbar_init(smem_u32(&sm.v_empty[s]), 1);
            mbar_init(smem_u32(&sm.s_full[s]), 1);
        }
        mbar_init(smem_u32(&sm.dp_full), 1);
        mbar_init(smem_u32(&sm.ds_ready), kWarps);
        mbar_init(smem_u32(&sm.dq_full), 1);
        mbar_init(smem_u32(&sm.dq_empty), kWarps);
        mbar_init(smem_u32(&sm.drained), 1);
        sm.abort = sm.redo = 0;
        for (int x = 0; x < kMaxTiles; ++x) sm.again[x] = 0;
        fence_barrier_init();
    }
    if (warp == kWarps) {
        tmem_alloc(smem_u32(&sm.tmem), 512);
        tmem_relinquish();
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tS = sm.tmem, tG = tS + 256, tdQ = tS + 384;   // S buffers at tS, tS + 128
    auto wait = [&](uint64_t &bar, uint32_t parity) {
        return wait_or_abort(bar, parity, &sm.abort, p.status, p.wait_ns);
    };
    // Tiles and key blocks of both passes are numbered on (it, g); the S of block g lies in buffer
    // g & 1.  The second pass takes the tiles marked in `again`.
    bool ok = true;
    int it = 0, g = 0;
    for (int pass = 0; pass < 2; ++pass) {
        if (warp == kWarps) {
            if (lane == 0) {
                int nq = it, nk = g, nv = g;
                for (int t = 0; ok; ++t) {
                    const uint32_t x = cta.x + (uint32_t)t * cta.ctas;
                    if (x >= all) break;
                    if (pass == 1 && sm.again[t] == 0) continue;
                    const QueryTile w(p, x, tiles);
                    if (w.empty()) continue;
                    const KeyBlocks<kTile> kb(w.pf, w.pl, p.window, p.sinks);
                    const int hk = w.h / p.G;
                    if (!(ok = wait(sm.q_empty, (it & 1) ^ 1))) break;
                    mbar_expect_tx(smem_u32(&sm.q_full), 2 * NB * kBlk);
                    for (int c = 0; c < NB; ++c) {
                        load_box(smem_u32(sm.q[c]), p.q, smem_u32(&sm.q_full), 64 * c, w.i0, w.h, w.b);
                        load_box(smem_u32(sm.go[c]), p.go, smem_u32(&sm.q_full), 64 * c, w.i0, w.h, w.b);
                    }
                    nq = ++it;
                    for (int j = 0; j < kb.count(); ++j, ++g) {
                        const int ks = kb.start(j);
                        if (!(ok = wait(sm.k_empty[g % 3], ((g / 3) & 1) ^ 1))) break;
                        mbar_expect_tx(smem_u32(&sm.k_full[g % 3]), NB * kBlk);
                        for (int c = 0; c < NB; ++c)
                            load_box(smem_u32(sm.k[g % 3][c]), p.k, smem_u32(&sm.k_full[g % 3]), 64 * c, ks, hk, w.b);
                        nk = g + 1;
                        if (!(ok = wait(sm.v_empty[g & 1], ((g >> 1) & 1) ^ 1))) break;
                        mbar_expect_tx(smem_u32(&sm.v_full[g & 1]), NB * kBlk);
                        for (int c = 0; c < NB; ++c)
                            load_box(smem_u32(sm.v[g & 1][c]), p.v, smem_u32(&sm.v_full[g & 1]), 64 * c, ks, hk, w.b);
                        nv = g + 1;
                    }
                }
                // what was loaded has landed
                if (nq > 0) drain_phase(smem_u32(&sm.q_full), (nq - 1) & 1);
                for (int t = max(0, nk - 3); t < nk; ++t) drain_phase(smem_u32(&sm.k_full[t % 3]), (t / 3) & 1);
                for (int t = max(0, nv - 2); t < nv; ++t) drain_phase(smem_u32(&sm.v_full[t & 1]), (t >> 1) & 1);
            }
            __syncwarp();
        } else if (warp == kWarps + 1) {
            if (elect_one()) {
                constexpr uint32_t idS = idesc_bf16(128, 128, false, false);
                constexpr uint32_t idG = idesc_bf16(128, HD, false, true);
                const uint64_t dq = k_major(sm.q), dg = k_major(sm.go);
                auto s_of = [&](int g) {
                    ok = ok && wait(sm.k_full[g % 3], (g / 3) & 1);
                    if (!ok) return;
                    tc_fence_after();
                    mma_scores<NB>(tS + 128 * (g & 1), dq, k_major(sm.k[g % 3]), idS);
                    mma_commit(smem_u32(&sm.s_full[g & 1]));
                };
                auto dp_of = [&](int g, bool last) {
                    ok = ok && wait(sm.v_full[g & 1], (g >> 1) & 1);
                    if (!ok) return;
                    tc_fence_after();
                    mma_scores<NB>(tG, dg, k_major(sm.v[g & 1]), idS);
                    mma_commit(smem_u32(&sm.dp_full));
                    mma_commit(smem_u32(&sm.v_empty[g & 1]));
                    if (last) mma_commit(smem_u32(&sm.q_empty));   // (the last scores came before)
                };
                for (int t = 0; ok; ++t) {
                    const uint32_t x = cta.x + (uint32_t)t * cta.ctas;
                    if (x >= all) break;
                    if (pass == 1 && sm.again[t] == 0) continue;
                    const QueryTile w(p, x, tiles);
                    if (w.empty()) continue;
                    const int n = KeyBlocks<kTile>(w.pf, w.pl, p.window, p.sinks).count();
                    ok = wait(sm.q_full, it & 1);
                    s_of(g);
                    // (the last tile's dP has been read: its last dS was waited for)
                    dp_of(g, n == 1);
                    if (n > 1) s_of(g + 1);
                    for (int j = 0; j < n && ok; ++j, ++g) {
                        ok = wait(sm.ds_ready, g & 1);
                        if (!ok) break;
                        if (j + 1 < n) dp_of(g + 1, j + 2 == n);   // first: the workers' next step waits for it
                        if (j == 0) ok = ok && wait(sm.dq_empty, (it & 1) ^ 1);
                        if (!ok) break;
                        tc_fence_after();
                        const uint64_t dk = mn_major(sm.k[g % 3]);   // dQ += dS K_j
                        mma_weights<5>(tdQ, tS + 128 * (g & 1), dk, idG, j > 0);
                        mma_weights<5>(tdQ, tS + 128 * (g & 1) + 16, dk, idG, true);
                        mma_commit(smem_u32(&sm.k_empty[g % 3]));
                        if (j + 2 < n) s_of(g + 2);
                    }
                    mma_commit(smem_u32(&sm.dq_full));
                    ++it;
                }
                if (!ok) {
                    mma_commit(smem_u32(&sm.s_full[0]));
                    mma_commit(smem_u32(&sm.s_full[1]));
                    mma_commit(smem_u32(&sm.dp_full));
                }
            }
            __syncwarp();
        } else if (warp < kWarps) {
            const int c0 = kCols * (warp >> 2), r = (warp & 3) * 32 + lane;
            const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16;
            const int d0 = (warp >> 2) * (HD / 4);   // this thread's quarter of the columns of dQ
            const float2 sl2 = make_float2(p.scale_log2, p.scale_log2);
            // This thread's row of a tile; the next tile's is fetched while the last dQ is summed.
            struct Row {
                QueryTile w;
                float L, D;
            };
            auto row_of = [&](uint32_t x) {
                Row y{QueryTile(p, x, tiles), 0.f, 0.f};
                const int pos = y.w.pf + r;
                if (pos <= y.w.pl) {
                    const long long row = ((long long)y.w.b * p.H + y.w.h) * p.Tq + y.w.i0 + r;
                    y.L = p.lse[row] * kLog2e;
                    y.D = p.delta[row];
                    // a query that sees one token only has no gradient: P = 0
                    if (sees_one(pos, p.window, p.sinks)) y.L = INFINITY;
                }
                return y;
            };
            auto next_of = [&](int t) {   // the next tile of this pass from t on
                while (pass == 1 && cta.x + (uint32_t)t * cta.ctas < all && sm.again[t] == 0) ++t;
                return t;
            };
            int t = next_of(0);
            uint32_t x = cta.x + (uint32_t)t * cta.ctas;
            Row row = row_of(min(x, all - 1));
            while (x < all && !giving_up(&sm.abort)) {
                const QueryTile w = row.w;
                const int pos = w.pf + r, tile_no = t;
                const bool valid = pos <= w.pl;
                const float2 nL = make_float2(-row.L, -row.L), nD = make_float2(-row.D, -row.D);
                bf16 *out = p.dQ + p.sdq.at(w.b, w.i0 + r, w.h) + d0;
                t = next_of(t + 1);
                x = cta.x + (uint32_t)t * cta.ctas;
                if (w.empty()) {
                    if (w.i0 + r < p.Tq)
#pragma unroll
                        for (int c = 0; c < HD / 4; c += 8)
                            if (d0 + c < p.hp) *reinterpret_cast<uint4 *>(out + c) = make_uint4(0, 0, 0, 0);
                    row = row_of(min(x, all - 1));
                    continue;
                }
                const KeyBlocks<kTile> kb(w.pf, w.pl, p.window, p.sinks);
                const WholeBlocks wb(kb, w.pf, w.pl, p.window);
                const int n = kb.count();
#pragma unroll 1
                for (int j = 0; j < n; ++j, ++g) {
                    const uint32_t tSj = tS + 128 * (g & 1) + lanes + c0;
                    const bool whole = wb.has(j);
                    uint32_t seen = ~0u;
                    if (!whole) seen = seen_bits(kb, j, kb.start(j), c0, pos, p.window, p.sinks);
                    wait(sm.s_full[g & 1], (g >> 1) & 1);
                    tc_fence_after();
                    float raw[32];
                    tmem_get32(tSj, raw);
                    float P[32];
#pragma unroll
                    for (int c = 0; c < 32; c += 2) {
                        const float2 y = fma2(make_float2(raw[c], raw[c + 1]), sl2, nL);
                        P[c] = exp2_fast(y.x);
                        P[c + 1] = exp2_fast(y.y);
                    }
                    wait(sm.dp_full, g & 1);
                    tc_fence_after();
                    tmem_get32(tG + lanes + c0, raw);
#pragma unroll
                    for (int c = 0; c < 32; c += 2) {
                        const float2 y = mul2(make_float2(P[c], P[c + 1]), add2(make_float2(raw[c], raw[c + 1]), nD));
                        P[c] = y.x;
                        P[c + 1] = y.y;
                    }
                    if (!whole) {
                        hide(P, seen, 0.f);
                        if (pass == 1) {
                            if (c0 == 0) clean_row<NB>(sm.k[g % 3][0], r);
                            fence_proxy_async();
                        }
                    }
                    put_weights_split(tSj, P);
                    warp_arrive(sm.ds_ready, lane);
                }
                row = row_of(min(x, all - 1));
                wait(sm.dq_full, it & 1);
                ++it;
                tc_fence_after();
                float dq[HD / 64][16];
                float odd = 0.f;
#pragma unroll
                for (int c = 0; c < HD / 64; ++c) tmem_ld16(tdQ + lanes + d0 + 16 * c, dq[c]);
                tc_fence_before();
                warp_arrive(sm.dq_empty, lane);
#pragma unroll
                for (int c = 0; c < HD / 64; ++c)
#pragma unroll
                    for (int e = 0; e < 16; ++e) odd = fmaf(dq[c][e], 0.f, odd);
                if (pass == 0 && valid && !(odd == 0.f)) sm.again[tile_no] = 1, sm.redo = 1;
                if (w.i0 + r < p.Tq && *(volatile int *)&sm.abort == 0) {
#pragma unroll
                    for (int c = 0; c < HD / 64; ++c) {
                        uint32_t o[8];
#pragma unroll
                        for (int e = 0; e < 8; ++e)
                            o[e] = valid ? pack_bf16x2(dq[c][2 * e] * p.scale, dq[c][2 * e + 1] * p.scale) : 0u;
                        if (d0 + 16 * c < p.hp) store32(out + 16 * c, o, p.wide_dq);
                    }
                }
            }
        }
        tc_fence_before();
        __syncthreads();
        tc_fence_after();
        if (*(volatile int *)&sm.redo == 0 || *(volatile int *)&sm.abort != 0) break;
    }
    if (warp == kWarps + 1 && elect_one()) drain_mmas(smem_u32(&sm.drained));
    __syncthreads();
    if (warp == kWarps) tmem_dealloc(sm.tmem, 512);
}

// Both parts in one grid: dQ's CTAs first, which all end at about the same time; then dK's and dV's, which fill
// the SMs as they come free.  All of them wait for D, which the kernel before computes.
template <int HD, bool kSplit>
__global__ void __launch_bounds__(kThreads, 1) window_grad_tc_kernel(const __grid_constant__ BwdArgs p) {
    extern __shared__ __align__(1024) uint8_t smem_raw[];
    pdl_wait();
    if (blockIdx.x < p.q_ctas)
        query_grads<HD>(p, smem_raw, Share{blockIdx.x, p.q_ctas});
    else
        key_grads<HD, kSplit>(p, smem_raw, Share{blockIdx.x - p.q_ctas, gridDim.x - p.q_ctas});
}

template <int HD>
cudaError_t launch(BwdArgs p, int B, cudaStream_t s) {
    constexpr int smem = (int)std::max(sizeof(KvSm<HD>), sizeof(QSm<HD>));
    static_assert(smem <= 227 * 1024, "shared memory");
    const auto kernel = few_terms(p.a) ? window_grad_tc_kernel<HD, true> : window_grad_tc_kernel<HD, false>;
    cudaError_t e = allow_smem((const void *)kernel, smem);
    if (e != cudaSuccess) return e;
    const long long all = (long long)((p.Tq + kTile - 1) / kTile) * p.H * B;
    p.q_ctas = (uint32_t)std::max(std::min(all, 152LL), (all + kMaxTiles - 1) / kMaxTiles);
    p.q_tiles = (uint32_t)all;
    // dK, dV: CTAs that stay where a tile meets few blocks, whose loads and first scores then run beside
    // the end of the tile before; where it meets many, one tile a CTA, which leaves it to the GPU which SM takes the
    // next.  Backward, us, staying / not: B2 T8192, 4 heads of 64, window 512 (5 blocks a tile)
    // 76.7 / 81.7; B4 T4096, 16 heads of 128, window 1024 (9) 438 / 475, 1408 (12) 505 / 536, 16 + 8 heads (18) 447 /
    // 450; B2 T8192, 8 + 4 heads of 64, window 1024 (18) 183 / 196; B4 T4096, 16 + 4 heads of 128, window 1024 (36)
    // 414 / 412, of 64 335 / 332.  (Also where sink tiles that meet many more are not split: 970 / 1078, B8
    // T4096, 32 heads of 64, window 512, 4 sinks.)
    const long long keys = (long long)p.split.ctas(p.a, kTile) * p.Hkv * B;
    const long long met = (long long)p.G * ((p.window + kTile - 1) / kTile + 1);
    const long long kv_ctas = met < 24 ? std::min(keys, 152LL) : keys;
    p.kv_tiles = (uint32_t)keys;
    e = launch_pdl(kernel, dim3((unsigned)(p.q_ctas + kv_ctas)), dim3(kThreads), smem, s, p);
    note_launches(1);
    if (e != cudaSuccess) return e;
    return add_sink_rows(p.a, p.partial, p.split.extra, p.dK, p.dV, s);
}

}  // namespace

bool tc_window_bwd(const Attn &a, const void *q, const void *k, const void *v, const int32_t *lens,
                   const float *lse, const void *dO, const float *delta, void *dq, void *dk, void *dv,
                   float *partial, uint32_t *status, cudaStream_t s, cudaError_t *err) {
    if (!a.bf16) return false;
    BwdArgs p;
    if (!make_map(&p.q, q, a.q, a.B, a.Tq, a.H, a.hp) || !make_map(&p.k, k, a.k, a.B, a.Tk, a.Hkv, a.hp) ||
        !make_map(&p.v, v, a.v, a.B, a.Tk, a.Hkv, a.hp) || !make_map(&p.go, dO, a.go, a.B, a.Tq, a.H, a.hp) ||
        !rows16(dq, a.dq, true) || !rows16(dk, a.dk, true) || !rows16(dv, a.dv, true))
        return false;
    p.lens = lens;
    p.lse = lse;
    p.delta = delta;
    p.dQ = (bf16 *)dq;
    p.dK = (bf16 *)dk;
    p.dV = (bf16 *)dv;
    p.sdq = a.dq;
    auto wide = [](const void *x, const Str &st) {
        return (reinterpret_cast<uintptr_t>(x) & 31) == 0 && ((st.b | st.t | st.h) & 15) == 0;
    };
    p.wide_dq = wide(dq, a.dq);
    p.wide_dk = wide(dk, a.dk);
    p.wide_dv = wide(dv, a.dv);
    p.sdk = a.dk;
    p.sdv = a.dv;
    p.partial = partial;
    p.status = status;
    p.wait_ns = wait_limit();
    p.Tq = a.Tq;
    p.Tk = a.Tk;
    p.H = a.H;
    p.Hkv = a.Hkv;
    p.G = a.G();
    p.hp = a.hp;
    p.window = a.window;
    p.sinks = a.sinks;
    p.a = a;
    p.split = SinkSplit(a, kTile);
    p.scale = a.scale;
    p.scale_log2 = a.scale * kLog2e;
    *err = a.hp <= 64 ? launch<64>(p, a.B, s) : launch<128>(p, a.B, s);
    return true;
}

}  // namespace win
}  // namespace mosa
