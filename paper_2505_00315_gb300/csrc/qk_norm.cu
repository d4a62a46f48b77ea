// Norm and rotation of queries and keys, one pass over each (Sec. 2.2, positional
// encodings, after an RMS norm per head):
//     r = 1/sqrt(mean(x^2) + eps),  n = r x gamma,  y = R(t) n
// and backward, with g = R(t)^T dy (the rotation's transpose turns back),
//     dgamma = sum g r x,  u = g gamma,  dx = r (u - r x mean(u r x)).
// Memory bound: x and y move once, forward; x, dy and dx backward (r is computed
// again from x, which is read anyway).  A head's hp values lie on hp/W lanes, W = 16 a
// lane where the rows' places allow it (32 bytes of bf16), else 8, so that the mean is a few
// shuffles and nothing is staged; a block takes some tokens with all their heads and
// computes each token's sines and cosines once for all of them, in shared memory.  Loads of the
// next item are under way while one is worked on.  What bounds it is how many bytes the
// registers keep in flight: B4 T4096, 32 + 8 heads of 128, bf16: forward 61 us (5.5 TB/s, 81% of
// the copy rate), backward 107 (4.7 TB/s, 69%); fp32 113 (6.0 TB/s, 88%) and 180 (5.6 TB/s, 82%).  One new token of eight sequences: 3 us, a
// launch and one trip to memory.
#include <cmath>

#include "head_rows.cuh"
#include "launch.h"
#include "profile.h"
#include "window.h"

namespace mosa {
namespace win {

Turns make_turns(int rotary, double theta) {
    Turns t{};
    const double two_pi = 6.283185307179586476925286766559;
    for (int p = 0; p < rotary / 2 && p < 64; ++p) {
        const double turns = std::pow(theta, -2.0 * p / rotary) / two_pi;   // <= 0.16
        t.phi[p] = (uint64_t)(turns * 18446744073709551616.0);
    }
    return t;
}

namespace {

constexpr int kThreads = 256;
// Tokens of one item: 64 bytes of loads that a lane keeps in flight while it works on the last.
constexpr int batch_of(int lane_bytes, bool backward) { return (backward ? 32 : 64) / lane_bytes; }
constexpr int kMaxTokens = 8;   // tokens of one block's step

struct NormArgs {
    Norm n;
    const void *q, *k, *gq, *gk, *dyq, *dyk;
    void *oq, *ok;          // forward: y; backward: dx
    const int32_t *pos;
    float *partial;         // backward: [blocks][2][hp] partial sums of dgamma
    int step, batch;        // tokens of a step, and of an item
};

// What a block keeps of a step's tokens: cosines and sines, and where each token's rows start in
// the input, the output (backward: its gradient) and the input's gradient.
struct StepTokens {
    alignas(16) float2 cs[kMaxTokens][64];
    long long in[2][kMaxTokens], y[2][kMaxTokens], d[2][kMaxTokens];   // [queries, keys]
};

template <class T, bool VEC, bool kBackward, int W, int LG>
__global__ void __launch_bounds__(kThreads, kBackward ? 2 : 3) qk_norm_rope_kernel(const __grid_constant__ NormArgs p,
                                                                const __grid_constant__ Turns tab) {
    constexpr int groups = kThreads / LG, hp = W * LG;
    constexpr int kBatch = batch_of(W * sizeof(T), kBackward);
    asm volatile("griddepcontrol.wait;" ::: "memory");
    // Three steps' tokens: the next ones are filled in while a slower warp may still be at the last.
    __shared__ StepTokens buf[3];
    __shared__ __align__(16) float gamma[2][hp];
    extern __shared__ float red[];   // backward: [groups][2][hp]
    const Norm &n = p.n;
    const int grp = threadIdx.x / LG, li = threadIdx.x % LG;
    const Part<W> at(li, n.rotary, n.halves);
    const long long N = (long long)n.B * n.T;
    for (int e = threadIdx.x; e < 2 * hp; e += kThreads) {
        const T *g = static_cast<const T *>(e < hp ? p.gq : p.gk);
        gamma[e / hp][e % hp] = g == nullptr ? 1.f : to_f32(g[e % hp]);
    }
    float acc[2][W];   // backward: this lane's sums of g r x, of queries and keys
#pragma unroll
    for (int e = 0; e < W; ++e) acc[0][e] = acc[1][e] = 0.f;
    const int HH = n.H + n.Hkv;   // heads 0 .. H-1 are queries, the others keys
    const int pairs = n.rotary >> 1;
    struct Step {
        const StepTokens *st;
        int tokens, items;
    };
    // Fills in the step of tokens from tok0 on.
    auto fill = [&](StepTokens &st, long long tok0) {
        const int tokens = (int)min((long long)p.step, N - tok0);
        const int b0 = (int)(tok0 / n.T), t0 = (int)(tok0 - (long long)b0 * n.T);
        if (threadIdx.x < tokens) {
            const int over = (t0 + (int)threadIdx.x) / n.T, b = b0 + over, t = t0 + threadIdx.x - over * n.T;
            st.in[0][threadIdx.x] = n.q.at(b, t, 0);
            st.in[1][threadIdx.x] = n.k.at(b, t, 0);
            st.y[0][threadIdx.x] = n.yq.at(b, t, 0);
            st.y[1][threadIdx.x] = n.yk.at(b, t, 0);
            st.d[0][threadIdx.x] = n.dq.at(b, t, 0);
            st.d[1][threadIdx.x] = n.dk.at(b, t, 0);
        }
        for (int e = threadIdx.x; e < tokens * pairs; e += kThreads) {
            const int i = e / pairs, a = e - i * pairs;
            const int t = p.pos != nullptr ? p.pos[tok0 + i] : (t0 + i) % n.T;
            st.cs[i][angle_at<W, LG>(a)] = angle_of(tab.phi[a], t);
        }
        return Step{&st, tokens, (tokens + p.batch - 1) / p.batch * HH};
    };
    // An item: `batch` tokens of one head, on one lane group.
    struct Item {
        const StepTokens *st;
        int key, h, i0, count;
    };
    auto item = [&](const Step &s, int it) {
        const int bat = it / HH, hh = it - bat * HH, i0 = bat * p.batch;
        const int key = hh >= n.H;
        return Item{s.st, key, key ? hh - n.H : hh, i0, it < s.items ? min(p.batch, s.tokens - i0) : 0};
    };
    auto load = [&](const Item &w, Raw<T, W> (&xr)[kBatch], Raw<T, W> (&yr)[kBackward ? kBatch : 1]) {
        const T *in = static_cast<const T *>(w.key ? p.k : p.q) + w.h * (w.key ? n.k.h : n.q.h);
        const T *gr = static_cast<const T *>(w.key ? p.dyk : p.dyq) + w.h * (w.key ? n.yk.h : n.yq.h);
#pragma unroll
        for (int u = 0; u < kBatch; ++u) {
            if (u < w.count) {
                load_raw<T, VEC, W>(in + w.st->in[w.key][w.i0 + u], at, xr[u]);
                if (kBackward) load_raw<T, VEC, W>(gr + w.st->y[w.key][w.i0 + u], at, yr[kBackward ? u : 0]);
            }
        }
    };
    auto work = [&](const Item &w, Raw<T, W> (&xr)[kBatch], Raw<T, W> (&yr)[kBackward ? kBatch : 1]) {
        T *out = static_cast<T *>(w.key ? p.ok : p.oq) +
                 w.h * (kBackward ? (w.key ? n.dk.h : n.dq.h) : (w.key ? n.yk.h : n.yq.h));
        float gm[W];
#pragma unroll
        for (int e = 0; e < W; e += 4) {
            const float4 g4 = *reinterpret_cast<const float4 *>(&gamma[w.key][at.at(e)]);
            gm[e] = g4.x; gm[e + 1] = g4.y; gm[e + 2] = g4.z; gm[e + 3] = g4.w;
        }
#pragma unroll
        for (int u = 0; u < kBatch; ++u) {
            if (u >= p.batch) break;
            const bool on = u < w.count;
            const float2 *cs = w.st->cs[on ? w.i0 + u : 0];
            float v[W], ss = 0.f;
            unpack<T, W>(xr[u], v);
#pragma unroll
            for (int e = 0; e < W; ++e) ss = fmaf(v[e], v[e], ss);
            const float r = rsqrtf(fmaf(group_sum(ss, LG), 1.f / hp, n.eps));
            if (!kBackward) {
#pragma unroll
                for (int e = 0; e < W; ++e) v[e] *= r * gm[e];
                turn<W, LG>(v, li, n.rotary, n.halves, cs, 1.f);
                if (on) store_part<T, VEC, W>(out + w.st->y[w.key][w.i0 + u], at, v);
            } else {
                float g[W], dot = 0.f;
                unpack<T, W>(yr[kBackward ? u : 0], g);
                turn<W, LG>(g, li, n.rotary, n.halves, cs, -1.f);
#pragma unroll
                for (int e = 0; e < W; ++e) {
                    v[e] *= r;
                    // (chosen, not multiplied by 0 or 1: a NaN of a key reaches no query's sum)
                    const float d = on ? g[e] * v[e] : 0.f;
                    acc[0][e] += w.key ? 0.f : d;
                    acc[1][e] += w.key ? d : 0.f;
                    g[e] *= gm[e];
                    dot = fmaf(g[e], v[e], dot);
                }
                dot = group_sum(dot, LG) * (1.f / hp);
#pragma unroll
                for (int e = 0; e < W; ++e) g[e] = r * fmaf(-v[e], dot, g[e]);
                if (on) store_part<T, VEC, W>(out + w.st->d[w.key][w.i0 + u], at, g);
            }
        }
    };
    // The next item's loads are under way while one is worked on, across steps too.
    const long long stride = (long long)gridDim.x * p.step;
    long long tok0 = (long long)blockIdx.x * p.step;   // (below N: no block is without a step)
    Step cur_step = fill(buf[0], tok0);
    __syncthreads();
    Raw<T, W> x[kBatch], dy[kBackward ? kBatch : 1];
    Item cur = item(cur_step, grp);
    load(cur, x, dy);
    for (int no = 1;; no = no == 2 ? 0 : no + 1) {
        tok0 += stride;
        const bool more = tok0 < N;
        Step next_step{};
        if (more) next_step = fill(buf[no], tok0);
        __syncthreads();
        for (int it0 = 0; it0 < cur_step.items; it0 += groups) {   // (all lanes together: the sums are shuffles)
            const bool last = it0 + groups >= cur_step.items;
            Item next{cur.st, 0, 0, 0, 0};
            if (!last) next = item(cur_step, it0 + groups + grp);
            else if (more) next = item(next_step, grp);
            Raw<T, W> nx[kBatch], ndy[kBackward ? kBatch : 1];
            load(next, nx, ndy);
            work(cur, x, dy);
            cur = next;
#pragma unroll
            for (int u = 0; u < kBatch; ++u) {
                x[u] = nx[u];
                if (kBackward) dy[kBackward ? u : 0] = ndy[kBackward ? u : 0];
            }
        }
        if (!more) break;
        cur_step = next_step;
    }
    if (kBackward && p.partial != nullptr) {
#pragma unroll
        for (int e = 0; e < W; ++e) {
            const int c = at.at(e);
            red[(grp * 2 + 0) * hp + c] = acc[0][e];
            red[(grp * 2 + 1) * hp + c] = acc[1][e];
        }
        __syncthreads();
        for (int o = threadIdx.x; o < 2 * hp; o += kThreads) {
            float sum = 0.f;
            for (int u = 0; u < groups; ++u) sum += red[u * 2 * hp + o];
            p.partial[(long long)blockIdx.x * 2 * hp + o] = sum;
        }
    }
}

// dgamma = the blocks' partial sums: 32 columns a block, 32 runs of rows each,
// added up in a fixed order.
__global__ void __launch_bounds__(1024) qk_dgamma_kernel(const float *partial, int blocks, int hp,
                                                         float *dgq, float *dgk) {
    asm volatile("griddepcontrol.wait;" ::: "memory");
    __shared__ float red[32][33];
    const int cc = threadIdx.x & 31, run = threadIdx.x >> 5;
    const int col = blockIdx.x * 32 + cc;
    float sum = 0.f;
    for (int r = run; r < blocks; r += 32) sum += partial[(long long)r * 2 * hp + col];
    red[run][cc] = sum;
    __syncthreads();
    if (run == 0) {
        float t = 0.f;
        for (int u = 0; u < 32; ++u) t += red[u][cc];
        float *out = col < hp ? dgq : dgk;
        if (out != nullptr) out[col < hp ? col : col - hp] = t;
    }
}

// A block stays for several steps: three blocks an SM (a fourth would have to spill), two in the
// backward, whose blocks also keep their dgamma to the end.
constexpr int kMaxBlocks = 152 * 2, kMaxForwardBlocks = 152 * 3;

// Tokens of a step: as many as leave three of four SMs a block.  More tokens of a step are more
// loads in flight and angles at work; with fewer, more SMs take part.  us, forward / backward, 16 + 4
// heads of 64, steps of 1, 2, 4, 8 tokens:
//      128 tokens   2.9 / 6.1    3.3 / 6.1    3.1 / 6.8    4.4 / 7.5
//      512          4.7 / 10.6   3.7 / 8.3    3.2 / 7.0    4.4 / 7.9
//     2048         10.8 / 19.9   8.2 / 14.3   5.7 / 13.2   5.4 / 11.0
int tokens_of_step(const Norm &n) {
    const long long N = (long long)n.B * n.T;
    int t = kMaxTokens;
    while (t > 1 && 4 * N < 3LL * 152 * t) t /= 2;
    return t;
}

int bwd_blocks(const Norm &n) {
    const long long N = (long long)n.B * n.T, t = tokens_of_step(n), steps = (N + t - 1) / t;
    return (int)(steps < kMaxBlocks ? steps : kMaxBlocks);
}

// Values of a lane: 16 where rows are whole 16-byte pieces of bf16 and rotated halves split into
// eights.  B4 T4096 H32 + 8 of 128, forward: 79 us at 16 a lane, 88 at 8 (before blocks stayed for
// several steps).
bool wide(const Norm &n, bool vec) { return n.bf16 && vec && (!n.halves || n.rotary % 16 == 0); }

template <bool kBackward, class T, bool VEC, int W>
cudaError_t launch_of(const NormArgs &p, unsigned blocks, cudaStream_t s) {
    const Turns tab = make_turns(p.n.rotary, p.n.theta);
    const int smem = kBackward ? kThreads * W * 2 * 4 : 0;   // 16 or 32 KB
    auto go = [&](auto kernel) { return launch_pdl(kernel, dim3(blocks), dim3(kThreads), smem, s, p, tab); };
    note_launches(1);
    switch (p.n.hp) {
        case 16: return go(qk_norm_rope_kernel<T, VEC, kBackward, W, 16 / W>);
        case 32: return go(qk_norm_rope_kernel<T, VEC, kBackward, W, 32 / W>);
        case 64: return go(qk_norm_rope_kernel<T, VEC, kBackward, W, 64 / W>);
        default: return go(qk_norm_rope_kernel<T, VEC, kBackward, W, 128 / W>);
    }
}

template <bool kBackward>
cudaError_t launch(NormArgs p, bool vec, unsigned blocks, cudaStream_t s) {
    const bool w16 = wide(p.n, vec);
    if (p.step > 1) p.batch = batch_of((w16 ? 16 : 8) * (p.n.bf16 ? 2 : 4), kBackward);
    if (w16) return launch_of<kBackward, bf16, true, 16>(p, blocks, s);
    if (p.n.bf16)
        return vec ? launch_of<kBackward, bf16, true, 8>(p, blocks, s) : launch_of<kBackward, bf16, false, 8>(p, blocks, s);
    return vec ? launch_of<kBackward, float, true, 8>(p, blocks, s) : launch_of<kBackward, float, false, 8>(p, blocks, s);
}

}  // namespace

size_t norm_workspace(const Norm &n) { return (size_t)bwd_blocks(n) * 2 * n.hp * sizeof(float); }

cudaError_t launch_norm(const Norm &n, const void *q, const void *k, const void *gq, const void *gk,
                        const int32_t *pos, void *yq, void *yk, cudaStream_t s) {
    NormArgs p{n, q, k, gq, gk, nullptr, nullptr, yq, yk, pos, nullptr, tokens_of_step(n), 1};
    const bool vec = rows16(q, n.q, n.bf16) && rows16(k, n.k, n.bf16) && rows16(yq, n.yq, n.bf16) &&
                     rows16(yk, n.yk, n.bf16);
    const long long N = (long long)n.B * n.T;
    const long long steps = (N + p.step - 1) / p.step;
    return launch<false>(p, vec, (unsigned)(steps < kMaxForwardBlocks ? steps : kMaxForwardBlocks), s);
}

cudaError_t launch_norm_bwd(const Norm &n, const void *q, const void *k, const void *gq,
                            const void *gk, const int32_t *pos, const void *dyq, const void *dyk,
                            void *dq, void *dk, float *dgq, float *dgk, void *ws, cudaStream_t s) {
    const bool sums = dgq != nullptr || dgk != nullptr;
    NormArgs p{n, q, k, gq, gk, dyq, dyk, dq, dk, pos, sums ? (float *)ws : nullptr,
               tokens_of_step(n), 1};
    const bool vec = rows16(q, n.q, n.bf16) && rows16(k, n.k, n.bf16) &&
                     rows16(dyq, n.yq, n.bf16) && rows16(dyk, n.yk, n.bf16) &&
                     rows16(dq, n.dq, n.bf16) && rows16(dk, n.dk, n.bf16);
    const int blocks = bwd_blocks(n);
    cudaError_t e = launch<true>(p, vec, (unsigned)blocks, s);
    if (e != cudaSuccess || !sums) return e;
    e = launch_pdl(qk_dgamma_kernel, dim3(2 * n.hp / 32), dim3(1024), 0, s, (const float *)p.partial,
                   blocks, n.hp, dgq, dgk);
    note_launches(1);
    return e;
}

}  // namespace win
}  // namespace mosa
