// Sliding-window attention with sinks on the tensor cores, forward (bf16).
//
// One CTA per (128-query tile, head, sequence).  For each 128-key block that the tile
// meets (window_tiles.cuh: the sinks, then the window up to the tile's own positions)
//     S = Q K^T                    tcgen05, fp32 in TMEM
//     P = 2^(S scale log2(e) - m)  per row: running maximum m, sum l
//     O += P V                     P as bf16 in TMEM in the place of S, V from shared memory
// and O / l, lse = (m + log2 l) ln 2 at the end.  m rises only when a block's maximum
// exceeds it by more than 2^8 (O and l are then rescaled); P stays within the bf16
// range at the same relative precision.  P is rounded to bf16, the type of the V it
// meets (8 bits, as the output has), in two parts where few tokens are seen; l sums the unrounded values.
//
// Sixteen warps compute (four per TMEM lane quadrant, each a quarter of the keys: four threads a
// row), one loads by TMA, one issues the MMAs.  Two CTAs share an SM (256 of 512 TMEM columns, half
// the shared memory each): while one's softmax runs the other's MMAs do.  With hp = 128, S and
// O fill a CTA's columns and P takes the place of S, so its chain is S -> P -> O -> S.
// With hp <= 64 P has columns of its own, and the next scores are computed as soon as
// the warps have read the last ones (unless P is taken in two parts).
//
// B1 T16384, 32 + 8 heads of 128, window 2048: 482 us back to back (502 with the call around it and nothing of it in
// L2), 1.07 PFLOP/s of the pairs that are seen.  With hp = 128 that is bound by issue and by each CTA's chain: a thread's 32 scores take 220 instructions, 96 of
// which are maxima, scaling, exponentials, sums and packing, the others the waits, fences and exchange of
// a block; issue slots are busy 50 to 55% of the time, the tensor pipe 45%.  (Eight worker warps with 64
// columns a thread: 606 us against 531 then.)  hp = 64, B2 T8192, 4 heads, window 512: 29 us, of
// which 512 CTAs' beginnings and ends are a third; early scores took it from 33 to 31 there.
//
// A masked key has P = 0, but 0 times a NaN or infinity of its V row is NaN: a CTA whose
// results are not all finite runs its blocks a second time with such V rows zeroed in
// the blocks that it sees in part, and rows that do see one set to NaN.
#include <type_traits>

#include "launch.h"
#include "profile.h"
#include "window_tc.cuh"

namespace mosa {
namespace win {
namespace {

constexpr int kWarps = 16, kWorkers = 32 * kWarps, kThreads = kWorkers + 64;
constexpr int kQ = 128, kN = 128;             // queries and keys of a tile
constexpr float kRescaleLog2 = 8.f;

struct FwdArgs {
    Map q, k, v, o, rest;
    const int32_t *lens;
    bf16 *O;
    float *lse;
    uint32_t *status;
    uint32_t wait_ns;
    Str so;
    int keep_rest;               // what O loses by its rounding goes to `rest`
    int B, Tq, Tk, H, G, hp, window, sinks;
    float scale_log2;
};

template <int HD>
struct FwdSm {
    static constexpr int NB = HD / 64, NS = HD == 128 ? 2 : 4;
    uint8_t q[NB][kBlk];
    uint8_t kv[NS][NB][kBlk];    // the tiles of K and V in the order of kv_tile
    uint64_t q_full, kv_full[NS], kv_empty[NS], s_full, s_free, p_ready, pv_done, o_done, drained;
    float part[2][4][kQ];        // [parity][quarter]: block maxima, final sums
    uint32_t tmem;
    uint32_t odd[4];             // second pass: keys of the block whose V row was zeroed
    int abort, redo;
};

// The K and V tiles of n blocks in the order in which the MMAs take them: K_0 V_0 K_1 V_1 .., or
// where the next scores come early K_0 K_1 V_0 K_2 V_1 ..  Tile x is V's or K's of block j;
// V's of block j is tile v_tile.
template <bool kEarly>
__device__ __forceinline__ bool kv_tile(int x, int n, int &j) {
    if (!kEarly || x == 0 || x == 2 * n - 1) {
        j = x >> 1;
        return (x & 1) != 0;
    }
    j = x >> 1;   // x = 2j - 1: K_j; x = 2j + 2: V_j
    if ((x & 1) != 0) {
        ++j;
        return false;
    }
    --j;
    return true;
}
template <bool kEarly>
__device__ __forceinline__ int v_tile(int j, int n) {
    return !kEarly || j == n - 1 ? 2 * j + 1 : 2 * j + 2;
}

// kSplit (few_terms): P's rounding is given back by a second product with what it left, in columns of S
// that nothing uses any more, so that no scores come early.  (In the kernel for many terms the
// branch alone, never taken, cost a fifth.)
template <int HD, bool kSplit>
__global__ void __launch_bounds__(kThreads, 2) window_fwd_tc_kernel(const __grid_constant__ FwdArgs p) {
    extern __shared__ __align__(1024) uint8_t smem_raw[];
    using Sm = FwdSm<HD>;
    constexpr int NB = Sm::NB, NS = Sm::NS;
    constexpr bool kEarly = HD == 64 && !kSplit;
    Sm &sm = *reinterpret_cast<Sm *>(smem_raw);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    pdl_wait();
    const Place at(blockIdx.x, p.H, p.B);
    const int b = at.b, h = at.h, hk = h / p.G;
    const int i0 = ((p.Tq + kQ - 1) / kQ - 1 - at.tile) * kQ, off = p.Tk - p.Tq;
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
        mbar_init(smem_u32(&sm.s_free), kWarps);
        mbar_init(smem_u32(&sm.p_ready), kWarps);
        mbar_init(smem_u32(&sm.pv_done), 1);
        mbar_init(smem_u32(&sm.o_done), 1);
        mbar_init(smem_u32(&sm.drained), 1);
        sm.abort = sm.redo = 0;
        fence_barrier_init();
    }
    if (warp == kWarps) {
        tmem_alloc(smem_u32(&sm.tmem), 256);
        tmem_relinquish();
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    // P: columns of its own, or the first half of each quarter of S
    const uint32_t tS = sm.tmem, tO = tS + 128, tP = kEarly ? tS + 192 : tS;
    const KeyBlocks<kN> kb(pf, pl, p.window, p.sinks);
    const int n = kb.count();

    int item = 0, phase = 0;   // K/V tiles and key blocks of both passes so far
    bool ok = true;
    for (int pass = 0; pass < 2; ++pass) {
        if (warp == kWarps) {
            if (lane == 0) {
                if (pass == 0) {
                    mbar_expect_tx(smem_u32(&sm.q_full), NB * kBlk);
                    for (int c = 0; c < NB; ++c)
                        load_box(smem_u32(sm.q[c]), p.q, smem_u32(&sm.q_full), 64 * c, i0, h, b);
                }
                for (int x = 0; x < 2 * n && ok; ++x) {
                    int j;
                    const bool is_v = kv_tile<kEarly>(x, n, j);
                    const int s = item % NS;
                    ok = wait_or_abort(sm.kv_empty[s], ((item / NS) & 1) ^ 1, &sm.abort, p.status, p.wait_ns);
                    if (!ok) break;
                    const uint32_t bar = smem_u32(&sm.kv_full[s]);
                    mbar_expect_tx(bar, NB * kBlk);
                    for (int c = 0; c < NB; ++c)
                        load_box(smem_u32(sm.kv[s][c]), is_v ? p.v : p.k, bar, 64 * c, kb.start(j), hk, b);
                    ++item;
                }
                // what was loaded has landed
                drain_phase(smem_u32(&sm.q_full), 0);
                for (int t = max(0, item - NS); t < item; ++t)
                    drain_phase(smem_u32(&sm.kv_full[t % NS]), (t / NS) & 1);
            }
            __syncwarp();
        } else if (warp == kWarps + 1) {
            if (elect_one()) {
                constexpr uint32_t idS = idesc_bf16(128, kN, false, false);
                constexpr uint32_t idO = idesc_bf16(128, HD, false, true);
                const uint64_t dq = k_major(sm.q);
                ok = ok && wait_or_abort(sm.q_full, 0, &sm.abort, p.status, p.wait_ns);
                auto next = [&]() -> int {   // slot of the next tile, or -1
                    const int s = item % NS;
                    ok = ok && wait_or_abort(sm.kv_full[s], (item / NS) & 1, &sm.abort, p.status, p.wait_ns);
                    ++item;
                    tc_fence_after();
                    return ok ? s : -1;
                };
                auto scores = [&]() {        // S = Q K_j^T
                    const int s = next();
                    if (s >= 0) {
                        mma_scores<NB>(tS, dq, k_major(sm.kv[s]), idS);
                        mma_commit(smem_u32(&sm.s_full));
                        mma_commit(smem_u32(&sm.kv_empty[s]));
                    }
                };
                scores();
                for (int j = 0; j < n && ok; ++j, ++phase) {
                    if (kEarly && j + 1 < n) {
                        ok = wait_or_abort(sm.s_free, phase & 1, &sm.abort, p.status, p.wait_ns);
                        scores();
                    }
                    ok = ok && wait_or_abort(sm.p_ready, phase & 1, &sm.abort, p.status, p.wait_ns);
                    const int s = next();
                    if (s < 0) break;
                    const uint64_t dv = mn_major(sm.kv[s]);
                    mma_weights<kEarly ? 7 : 5>(tO, tP, dv, idO, j > 0);   // O += P V_j
                    if (kSplit) mma_weights<5>(tO, tS + 16, dv, idO, true);
                    mma_commit(smem_u32(&sm.kv_empty[s]));
                    if (kEarly) mma_commit(smem_u32(&sm.pv_done));
                    // (else the next scores overwrite P: MMAs run in the order of issue)
                    else if (j + 1 < n) scores();
                }
                mma_commit(smem_u32(&sm.o_done));
                if (!ok) {
                    mma_commit(smem_u32(&sm.s_full));
                    mma_commit(smem_u32(&sm.pv_done));
                }
            }
            __syncwarp();
        } else {
            const int cq = warp >> 2, q = warp & 3, r = q * 32 + lane, pos = pf + r;
            const uint32_t lanes = (uint32_t)(q * 32) << 16, tmy = tS + lanes + 32 * cq;
            const float2 sl2 = make_float2(p.scale_log2, p.scale_log2);
            const WholeBlocks wb(kb, pf, pl, p.window);
            float *const part0 = &sm.part[0][0][r];
            float m = -1e38f, l = 0.f;   // (m: below every score, and finite)
            // (the second pass's loop is one of its own: its code, never run, costs the first one's 5%)
            auto weigh = [&](auto second) {
                constexpr bool kSecond = decltype(second)::value;
#pragma unroll 1
                for (int j = 0; j < n; ++j, ++phase) {
                    const bool whole = wb.has(j);
                    uint32_t seen = ~0u;
                    if (!whole) seen = seen_bits(kb, j, kb.start(j), 32 * cq, pos, p.window, p.sinks);
                    wait_or_abort(sm.s_full, phase & 1, &sm.abort, p.status, p.wait_ns);
                    tc_fence_after();
                    float s[32];
                    tmem_get32(tmy, s);
                    if (kEarly) {   // S_{j+1} may be written
                        tc_fence_before();
                        warp_arrive(sm.s_free, lane);
                    }
                    if (!whole) hide(s, seen, -INFINITY);
                    float mx[2] = {fmaxf(s[0], s[1]), fmaxf(s[2], s[3])};
#pragma unroll
                    for (int c = 4; c < 32; c += 4) {
                        mx[0] = max3(mx[0], s[c], s[c + 1]);
                        mx[1] = max3(mx[1], s[c + 2], s[c + 3]);
                    }
                    // (the buffer of this parity was last read before the last block's barrier)
                    float *const part = part0 + (phase & 1) * (4 * kQ);
                    part[cq * kQ] = fmaxf(mx[0], mx[1]);
                    named_barrier(1 + q, 128);
                    const float mb = fmaxf(max3(part[0], part[kQ], part[2 * kQ]), part[3 * kQ]) * p.scale_log2;
                    const bool grow = mb > m + kRescaleLog2;   // the same in all four threads of the row
                    const float corr = grow ? exp2_fast(m - mb) : 1.f;   // 0 on a row's first block
                    if (grow) m = mb;
                    const float2 neg = make_float2(-m, -m);
                    float2 sum = make_float2(0.f, 0.f);
#pragma unroll
                    for (int c = 0; c < 32; c += 2) {
                        const float2 x = fma2(make_float2(s[c], s[c + 1]), sl2, neg);
                        s[c] = exp2_fast(x.x);
                        s[c + 1] = exp2_fast(x.y);
                        sum = add2(sum, make_float2(s[c], s[c + 1]));
                    }
                    l = l * corr + (sum.x + sum.y);
                    if (kSecond && !whole) {
                        // V rows with NaN or infinities: zeroed, and NaN for the rows that see them
                        const int t = item + v_tile<kEarly>(j, n);
                        wait_or_abort(sm.kv_full[t % NS], (t / NS) & 1, &sm.abort, p.status, p.wait_ns);
                        if (cq == 0) {
                            const uint32_t odd = __ballot_sync(0xffffffffu, clean_row<NB>(sm.kv[t % NS][0], r));
                            if (lane == 0) sm.odd[q] = odd;
                            fence_proxy_async();
                        }
                        named_barrier(5, kWorkers);
                        if ((sm.odd[cq] & seen) != 0) s[0] = NAN;   // times the row of that key, whatever it holds
                        named_barrier(5, kWorkers);
                    }
                    uint32_t w[16];
#pragma unroll
                    for (int e = 0; e < 16; ++e) w[e] = pack_bf16x2(s[2 * e], s[2 * e + 1]);
                    if (kEarly && j > 0) {   // P and O may be written: P_{j-1} V_{j-1} is done
                        wait_or_abort(sm.pv_done, (phase & 1) ^ 1, &sm.abort, p.status, p.wait_ns);
                        tc_fence_after();
                    }
                    tmem_st16_async(kEarly ? tP + lanes + 16 * cq : tmy, w);
                    if (kSplit) {
#pragma unroll
                        for (int e = 0; e < 16; ++e)
                            w[e] = pack_bf16x2(s[2 * e] - __uint_as_float(w[e] << 16),
                                               s[2 * e + 1] - __uint_as_float(w[e] & 0xFFFF0000u));
                        tmem_st16_async(tmy + 16, w);
                    }
                    if (j > 0 && __any_sync(0xffffffffu, grow)) {
                        // (not early: S_j was issued after P_{j-1} V_{j-1})
#pragma unroll
                        for (int c = 0; c < HD / 4; c += 16) {
                            float o[16];
                            tmem_ld16(tO + lanes + cq * (HD / 4) + c, o);
#pragma unroll
                            for (int e = 0; e < 16; ++e) w[e] = __float_as_uint(o[e] * corr);
                            tmem_st16_async(tO + lanes + cq * (HD / 4) + c, w);
                        }
                    }
                    tmem_stored();
                    tc_fence_before();
                    warp_arrive(sm.p_ready, lane);
                }
            };
            pass == 0 ? weigh(std::false_type()) : weigh(std::true_type());
            item += 2 * n;
            wait_or_abort(sm.o_done, pass, &sm.abort, p.status, p.wait_ns);
            tc_fence_after();
            float o[HD / 64][16];   // this thread's quarter of the columns
            float odd = 0.f;
            const bool valid = pos <= pl;
#pragma unroll
            for (int u = 0; u < HD / 64; ++u) {
                tmem_ld16(tO + lanes + cq * (HD / 4) + 16 * u, o[u]);
#pragma unroll
                for (int e = 0; e < 16; ++e) odd = fmaf(o[u][e], 0.f, odd);
            }
            if (pass == 0 && valid && !(odd == 0.f)) sm.redo = 1;
            float (*part)[kQ] = sm.part[phase & 1];
            part[cq][r] = l;
            const bool live = !giving_up_at(5, kWorkers, &sm.abort);
            l = (part[0][r] + part[1][r]) + (part[2][r] + part[3][r]);
            if (live && (pass == 1 || *(volatile int *)&sm.redo == 0)) {
                const float inv = valid ? 1.f / l : 0.f;
#pragma unroll
                for (int u = 0; u < HD / 32; ++u) {
                    uint32_t w[4], y[4];
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const int c = 8 * (u & 1) + 2 * e;
                        const float x0 = o[u >> 1][c] * inv, x1 = o[u >> 1][c + 1] * inv;
                        w[e] = valid ? pack_bf16x2(x0, x1) : 0u;
                        y[e] = valid ? pack_bf16x2(x0 - __uint_as_float(w[e] << 16),
                                                   x1 - __uint_as_float(w[e] & 0xFFFF0000u)) : 0u;
                    }
                    const int unit = cq * (HD / 32) + u;
                    *reinterpret_cast<uint4 *>(sm.q[unit >> 3] + xoff128(r, unit & 7)) =
                        make_uint4(w[0], w[1], w[2], w[3]);
                    if (p.keep_rest)
                        *reinterpret_cast<uint4 *>(sm.kv[0][unit >> 3] + xoff128(r, unit & 7)) =
                            make_uint4(y[0], y[1], y[2], y[3]);
                }
                if (lse != nullptr && cq == 0 && i0 + r < p.Tq)
                    lse[i0 + r] = valid ? (m + log2f(l)) * kLn2 : -INFINITY;
                fence_proxy_async();
                named_barrier(5, kWorkers);
                if (threadIdx.x == 0) {
                    for (int c = 0; c < NB; ++c) {
                        store_box(p.o, smem_u32(sm.q[c]), 64 * c, i0, h, b);
                        if (p.keep_rest) store_box(p.rest, smem_u32(sm.kv[0][c]), 64 * c, i0, h, b);
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
    if (warp == kWarps + 1 && elect_one()) drain_mmas(smem_u32(&sm.drained));
    __syncthreads();
    if (warp == kWarps) tmem_dealloc(sm.tmem, 256);
}

template <int HD, bool kSplit>
cudaError_t launch(const FwdArgs &p, dim3 grid, cudaStream_t s) {
    constexpr int bytes = (int)sizeof(FwdSm<HD>);
    static_assert(bytes <= 115712, "two CTAs an SM");
    auto kernel = window_fwd_tc_kernel<HD, kSplit>;
    cudaError_t e = allow_smem((const void *)kernel, bytes);
    if (e != cudaSuccess) return e;
    e = launch_pdl(kernel, grid, dim3(kThreads), bytes, s, p);
    note_launches(1);
    return e;
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
    p.wait_ns = wait_limit();
    p.so = a.o;
    p.Tq = a.Tq;
    p.Tk = a.Tk;
    p.B = a.B;
    p.H = a.H;
    p.G = a.G();
    p.hp = a.hp;
    p.window = a.window;
    p.sinks = a.sinks;
    p.scale_log2 = a.scale * kLog2e;
    const dim3 grid = grid_of((a.Tq + kQ - 1) / kQ, a.H, a.B);
    const bool split = few_terms(a);
    *err = a.hp <= 64 ? (split ? launch<64, true>(p, grid, s) : launch<64, false>(p, grid, s))
                      : (split ? launch<128, true>(p, grid, s) : launch<128, false>(p, grid, s));
    return true;
}

}  // namespace win
}  // namespace mosa
