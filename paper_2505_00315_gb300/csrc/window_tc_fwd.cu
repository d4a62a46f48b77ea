// Sliding-window attention with sinks on the tensor cores, forward (bf16).
//
// One CTA per (128-query tile, head, sequence).  For each 128-key block that the tile
// meets (window_tiles.cuh: the sinks, then the window up to the tile's own positions)
//     S = Q K^T                    tcgen05, fp32 in TMEM
//     P = 2^(S scale log2(e) - m)  one thread a row: running maximum m, sum l
//     O += P V                     P as bf16 in TMEM in the place of S, V from shared memory
// and O / l, lse = (m + log2 l) ln 2 at the end.  m rises only when a block's maximum
// exceeds it by more than 2^8 (O and l are then rescaled); P stays within the bf16
// range at the same relative precision.  P is rounded to bf16, the type of the V it
// meets (8 bits, as the output has); l sums the unrounded values.
//
// Warps 0-3 compute (one per TMEM lane quadrant, one thread a row), warp 4 loads by
// TMA, warp 5 issues the MMAs.  Two CTAs share an SM (256 of 512 TMEM columns, half
// the shared memory each): while one's softmax runs the other's MMAs do, so a CTA's own
// chain S -> P -> O may be plain.
//
// A masked key has P = 0, but 0 times a NaN or infinity of its V row is NaN: a CTA whose
// results are not all finite runs its blocks a second time with such V rows zeroed in
// the blocks that it sees in part, and rows that do see one set to NaN.
#include "launch.h"
#include "profile.h"
#include "window_tc.cuh"

namespace mosa {
namespace win {
namespace {

constexpr int kThreads = 192;
constexpr int kQ = 128, kN = 128;             // queries and keys of a tile
constexpr int kBlk = 128 * 64 * 2;            // 128 rows of 64 columns
constexpr float kRescaleLog2 = 8.f;

struct FwdArgs {
    Map q, k, v, o, rest;
    const int32_t *lens;
    bf16 *O;
    float *lse;
    uint32_t *status;
    Str so;
    int keep_rest;               // what O loses by its rounding goes to `rest`
    int Tq, Tk, H, G, hp, window, sinks;
    float scale_log2;
};

template <int HD>
struct FwdSm {
    static constexpr int NB = HD / 64, NS = HD == 128 ? 5 : 6;   // 112 KB with Q
    uint8_t q[NB][kBlk];
    uint8_t kv[NS][kBlk];        // 64-column blocks: K_0, V_0, K_1, V_1, ..
    uint64_t q_full, kv_full[NS], kv_empty[NS], s_full, p_ready, o_done, drained;
    uint32_t tmem;
    uint32_t odd[4];             // second pass: keys of the block whose V row was zeroed
    int abort, redo;
};

template <int HD>
__global__ void __launch_bounds__(kThreads, 2) window_fwd_tc_kernel(const __grid_constant__ FwdArgs p) {
    extern __shared__ __align__(1024) uint8_t smem_raw[];
    using Sm = FwdSm<HD>;
    constexpr int NB = Sm::NB, NS = Sm::NS;
    Sm &sm = *reinterpret_cast<Sm *>(smem_raw);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int b = blockIdx.z, h = blockIdx.y, hk = h / p.G;
    const int i0 = ((int)gridDim.x - 1 - (int)blockIdx.x) * kQ, off = p.Tk - p.Tq;
    const int len = seq_len(p.lens, b, p.Tk);
    const int pf = off + i0, pl = min(off + min(i0 + kQ, p.Tq), len) - 1;
    float *lse = p.lse == nullptr ? nullptr : p.lse + ((long long)b * p.H + h) * p.Tq;

    if (pl < pf) {   // nothing to see: zeros
        const int rows = min(kQ, p.Tq - i0), units = p.hp / 8;
        for (int e = threadIdx.x; e < rows * units; e += kThreads)
            *reinterpret_cast<uint4 *>(p.O + p.so.at(b, i0 + e / units, h) + e % units * 8) =
                make_uint4(0, 0, 0, 0);
        for (int r = threadIdx.x; lse != nullptr && r < rows; r += kThreads) lse[i0 + r] = -INFINITY;
        return;
    }
    if (threadIdx.x == 0) {
        mbar_init(smem_u32(&sm.q_full), 1);
        for (int s = 0; s < NS; ++s) {
            mbar_init(smem_u32(&sm.kv_full[s]), 1);
            mbar_init(smem_u32(&sm.kv_empty[s]), 1);
        }
        mbar_init(smem_u32(&sm.s_full), 1);
        mbar_init(smem_u32(&sm.p_ready), 128);
        mbar_init(smem_u32(&sm.o_done), 1);
        mbar_init(smem_u32(&sm.drained), 1);
        sm.abort = sm.redo = 0;
        fence_barrier_init();
    }
    if (warp == 4) {
        tmem_alloc(smem_u32(&sm.tmem), 256);
        tmem_relinquish();
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tS = sm.tmem, tP = tS, tO = tS + 128;
    const KeyBlocks<kN> kb(pf, pl, p.window, p.sinks);
    const int n = kb.count();

    int item = 0, phase = 0;   // K/V boxes and key blocks of both passes so far
    bool ok = true;
    for (int pass = 0; pass < 2; ++pass) {
        if (warp == 4) {
            if (lane == 0) {
                if (pass == 0) {
                    mbar_expect_tx(smem_u32(&sm.q_full), NB * kBlk);
                    for (int c = 0; c < NB; ++c)
                        load_box(smem_u32(sm.q[c]), p.q, smem_u32(&sm.q_full), 64 * c, i0, h, b);
                }
                for (int x = 0; x < 2 * NB * n && ok; ++x) {
                    const int s = item % NS, j = x / (2 * NB), u = x % (2 * NB);
                    ok = wait_or_abort(sm.kv_empty[s], ((item / NS) & 1) ^ 1, &sm.abort, p.status);
                    if (!ok) break;
                    const uint32_t bar = smem_u32(&sm.kv_full[s]);
                    mbar_expect_tx(bar, kBlk);
                    load_box(smem_u32(sm.kv[s]), u < NB ? p.k : p.v, bar, 64 * (u % NB), kb.start(j),
                             hk, b);
                    ++item;
                }
                // what was loaded has landed
                drain_phase(smem_u32(&sm.q_full), 0);
                for (int t = max(0, item - NS); t < item; ++t)
                    drain_phase(smem_u32(&sm.kv_full[t % NS]), (t / NS) & 1);
            }
            __syncwarp();
        } else if (warp == 5) {
            if (elect_one()) {
                constexpr uint32_t idS = idesc_bf16(128, kN, false, false);
                constexpr uint32_t idO = idesc_bf16(128, 64, false, true);
                ok = ok && wait_or_abort(sm.q_full, 0, &sm.abort, p.status);
                auto scores = [&]() {   // S = Q K_j^T
                    for (int c = 0; c < NB && ok; ++c, ++item) {
                        const int s = item % NS;
                        ok = wait_or_abort(sm.kv_full[s], (item / NS) & 1, &sm.abort, p.status);
                        if (!ok) break;
                        tc_fence_after();
#pragma unroll
                        for (int kk = 0; kk < 4; ++kk)
                            mma_bf16(tS, smem_desc_sw128(smem_u32(sm.q[c]) + kk * 32, 16, 1024),
                                     smem_desc_sw128(smem_u32(sm.kv[s]) + kk * 32, 16, 1024), idS,
                                     (c > 0 || kk > 0) ? 1u : 0u);
                        mma_commit(smem_u32(&sm.kv_empty[s]));
                    }
                    mma_commit(smem_u32(&sm.s_full));
                };
                scores();
                for (int j = 0; j < n && ok; ++j, ++phase) {
                    ok = wait_or_abort(sm.p_ready, phase & 1, &sm.abort, p.status);
                    tc_fence_after();
                    for (int c = 0; c < NB && ok; ++c, ++item) {   // O += P V_j
                        const int s = item % NS;
                        ok = wait_or_abort(sm.kv_full[s], (item / NS) & 1, &sm.abort, p.status);
                        if (!ok) break;
                        tc_fence_after();
#pragma unroll
                        for (int kk = 0; kk < 8; ++kk)
                            mma_bf16_ts(tO + 64 * c, tP + 8 * kk,
                                        smem_desc_sw128(smem_u32(sm.kv[s]) + kk * 2048, kBlk, 1024),
                                        idO, (j > 0 || kk > 0) ? 1u : 0u);
                        mma_commit(smem_u32(&sm.kv_empty[s]));
                    }
                    // (the next scores overwrite P: MMAs run in the order of issue)
                    if (ok && j + 1 < n) scores();
                }
                mma_commit(smem_u32(&sm.o_done));
                if (!ok) mma_commit(smem_u32(&sm.s_full));
            }
            __syncwarp();
        } else {
            const int r = threadIdx.x, pos = pf + r;
            const uint32_t lanes = (uint32_t)(warp * 32) << 16;
            float m = -INFINITY, l = 0.f;
            for (int j = 0; j < n; ++j, ++phase) {
                ok = wait_or_abort(sm.s_full, phase & 1, &sm.abort, p.status) && ok;
                tc_fence_after();
                uint32_t raw[4][32];
#pragma unroll
                for (int u = 0; u < 4; ++u) tmem_ld32_async(tS + lanes + 32 * u, raw[u]);
#pragma unroll
                for (int u = 0; u < 4; ++u) tmem_ready(raw[u]);
                float s[kN];
#pragma unroll
                for (int c = 0; c < kN; ++c) s[c] = __uint_as_float(raw[c >> 5][c & 31]);
                const bool whole = kb.whole(j, pf, pl, p.window);
                const int ks = kb.start(j);
                // columns first .. last of the block, and those below `sink`, are seen
                int first = 0, last = kN - 1, sink = 0;
                if (!whole) {
                    if (!kb.is_far(j)) {
                        first = max(pos - p.window + 1, 0) - ks;
                        last = min(pos - ks, kN - 1);
                        sink = min(p.sinks - ks, last + 1);
                    } else {
                        last = kb.slim - ks - 1;
                    }
                    const int low = max(-ks, 0);
#pragma unroll
                    for (int c = 0; c < kN; ++c)
                        if (!(c <= last && c >= low && (c >= first || c < sink))) s[c] = -INFINITY;
                }
                float mx[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
                for (int c = 0; c < kN; ++c) mx[c & 3] = fmaxf(mx[c & 3], s[c]);
                const float mb = fmaxf(fmaxf(mx[0], mx[1]), fmaxf(mx[2], mx[3])) * p.scale_log2;
                const bool grow = mb > m + kRescaleLog2;
                const float m_new = grow ? mb : m;
                const float corr = grow ? exp2_fast(m - m_new) : 1.f;   // 0 on the first block
                const float base = m_new == -INFINITY ? 0.f : m_new;
                float sum[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int c = 0; c < kN; ++c) {
                    s[c] = exp2_fast(fmaf(s[c], p.scale_log2, -base));
                    sum[c & 3] += s[c];
                }
                l = l * corr + ((sum[0] + sum[1]) + (sum[2] + sum[3]));
                m = m_new;
                if (j > 0 && __any_sync(0xffffffffu, grow)) {
                    // (S_j was issued after P_{j-1} V_{j-1}, so O is complete)
#pragma unroll
                    for (int c = 0; c < HD; c += 16) {
                        float o[16];
                        uint32_t w[16];
                        tmem_ld16(tO + lanes + c, o);
#pragma unroll
                        for (int e = 0; e < 16; ++e) w[e] = __float_as_uint(o[e] * corr);
                        tmem_st16_async(tO + lanes + c, w);
                    }
                    tmem_stored();
                }
                if (pass == 1 && !whole) {
                    // V rows with NaN or infinities: zeroed, and NaN for the rows that see them
                    const int at = item + 2 * NB * j + NB;
                    uint8_t *blk[NB];
                    for (int c = 0; c < NB; ++c) {
                        const int t = at + c;
                        ok = wait_or_abort(sm.kv_full[t % NS], (t / NS) & 1, &sm.abort, p.status) && ok;
                        blk[c] = sm.kv[t % NS];
                    }
                    const uint32_t odd = __ballot_sync(0xffffffffu, clean_row<NB>(blk, r));
                    if (lane == 0) sm.odd[warp] = odd;
                    fence_proxy_async();
                    named_barrier(1, 128);
                    const uint32_t any = sm.odd[0] | sm.odd[1] | sm.odd[2] | sm.odd[3];
                    bool sees_odd = false;
#pragma unroll 1
                    for (int c = max(-ks, 0); any != 0 && c <= last; ++c)
                        sees_odd = sees_odd || ((c >= first || c < sink) &&
                                                ((sm.odd[c >> 5] >> (c & 31)) & 1u) != 0);
                    if (sees_odd) s[0] = NAN;   // times the row of block column 0, whatever it holds
                    named_barrier(1, 128);
                }
#pragma unroll
                for (int u = 0; u < 4; ++u) {
                    uint32_t w[16];
#pragma unroll
                    for (int e = 0; e < 16; ++e) w[e] = pack_bf16x2(s[32 * u + 2 * e], s[32 * u + 2 * e + 1]);
                    tmem_st16_async(tP + lanes + 16 * u, w);
                }
                tmem_stored();
                tc_fence_before();
                mbar_arrive(smem_u32(&sm.p_ready));
            }
            item += 2 * NB * n;
            ok = wait_or_abort(sm.o_done, pass, &sm.abort, p.status) && ok;
            tc_fence_after();
            uint32_t raw[HD / 32][32];
#pragma unroll
            for (int u = 0; u < HD / 32; ++u) tmem_ld32_async(tO + lanes + 32 * u, raw[u]);
#pragma unroll
            for (int u = 0; u < HD / 32; ++u) tmem_ready(raw[u]);
            const bool valid = pos <= pl;
            float odd = 0.f;
#pragma unroll
            for (int u = 0; u < HD / 32; ++u)
#pragma unroll
                for (int e = 0; e < 32; ++e) odd = fmaf(__uint_as_float(raw[u][e]), 0.f, odd);
            if (pass == 0 && valid && !(odd == 0.f)) sm.redo = 1;
            named_barrier(1, 128);
            const bool live = *(volatile int *)&sm.abort == 0;
            if (live && (pass == 1 || *(volatile int *)&sm.redo == 0)) {
                const float inv = valid ? 1.f / l : 0.f;
#pragma unroll
                for (int u = 0; u < HD / 8; ++u) {
                    uint32_t w[4], y[4];
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const int c = 8 * u + 2 * e;
                        const float x0 = __uint_as_float(raw[c >> 5][c & 31]) * inv;
                        const float x1 = __uint_as_float(raw[c >> 5][(c & 31) + 1]) * inv;
                        w[e] = valid ? pack_bf16x2(x0, x1) : 0u;
                        y[e] = valid ? pack_bf16x2(x0 - __uint_as_float(w[e] << 16),
                                                   x1 - __uint_as_float(w[e] & 0xFFFF0000u)) : 0u;
                    }
                    *reinterpret_cast<uint4 *>(sm.q[u >> 3] + xoff128(r, u & 7)) =
                        make_uint4(w[0], w[1], w[2], w[3]);
                    if (p.keep_rest)
                        *reinterpret_cast<uint4 *>(sm.kv[u >> 3] + xoff128(r, u & 7)) =
                            make_uint4(y[0], y[1], y[2], y[3]);
                }
                if (lse != nullptr && i0 + r < p.Tq)
                    lse[i0 + r] = valid ? (m + log2f(l)) * kLn2 : -INFINITY;
                fence_proxy_async();
                named_barrier(1, 128);
                if (threadIdx.x == 0) {
                    for (int c = 0; c < NB; ++c) {
                        store_box(p.o, smem_u32(sm.q[c]), 64 * c, i0, h, b);
                        if (p.keep_rest) store_box(p.rest, smem_u32(sm.kv[c]), 64 * c, i0, h, b);
                    }
                    bulk_commit();
                    bulk_wait_read0();
                }
            }
        }
        tc_fence_before();
        __syncthreads();
        tc_fence_after();
        if (*(volatile int *)&sm.redo == 0 || *(volatile int *)&sm.abort != 0) break;
    }
    if (warp == 5 && elect_one()) drain_mmas(smem_u32(&sm.drained));
    __syncthreads();
    if (warp == 4) tmem_dealloc(sm.tmem, 256);
}

template <int HD>
cudaError_t launch(const FwdArgs &p, dim3 grid, cudaStream_t s) {
    constexpr int bytes = (int)sizeof(FwdSm<HD>);
    static_assert(bytes <= 115712, "two CTAs an SM");
    auto kernel = window_fwd_tc_kernel<HD>;
    cudaError_t e = allow_smem((const void *)kernel, bytes);
    if (e != cudaSuccess) return e;
    kernel<<<grid, kThreads, bytes, s>>>(p);
    note_launches(1);
    return cudaGetLastError();
}

}  // namespace

bool tc_window_fwd(const Attn &a, const void *q, const void *k, const void *v, const int32_t *lens,
                   void *O, float *lse, bf16 *rest, uint32_t *status, cudaStream_t s, cudaError_t *err) {
    if (!a.bf16) return false;
    FwdArgs p;
    if (!make_map(&p.q, q, a.q, a.B, a.Tq, a.H, a.hp) || !make_map(&p.k, k, a.k, a.B, a.Tk, a.Hkv, a.hp) ||
        !make_map(&p.v, v, a.v, a.B, a.Tk, a.Hkv, a.hp) || !make_map(&p.o, O, a.o, a.B, a.Tq, a.H, a.hp))
        return false;
    p.keep_rest = rest != nullptr;
    p.rest = p.o;
    if (rest != nullptr && !make_map(&p.rest, rest, a.packed(), a.B, a.Tq, a.H, a.hp)) return false;
    p.lens = lens;
    p.O = (bf16 *)O;
    p.lse = lse;
    p.status = status;
    p.so = a.o;
    p.Tq = a.Tq;
    p.Tk = a.Tk;
    p.H = a.H;
    p.G = a.G();
    p.hp = a.hp;
    p.window = a.window;
    p.sinks = a.sinks;
    p.scale_log2 = a.scale * kLog2e;
    const dim3 grid((a.Tq + kQ - 1) / kQ, a.H, a.B);
    *err = a.hp <= 64 ? launch<64>(p, grid, s) : launch<128>(p, grid, s);
    return true;
}

}  // namespace win
}  // namespace mosa
