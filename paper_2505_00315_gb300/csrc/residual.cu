// The residual step between two blocks, one pass over its tensors, and its backward.  For each token
//     n = r_y y gamma_post,  u = keep/(1-p) g n,  x' = x + scale u,  h = r_x x' gamma_pre
// and, with e = dh gamma_pre, xh = r_x x', yh = r_y y, c = scale keep/(1-p),
//     t = dx' + r_x (e - xh mean(e xh)),  dx = t,  dgamma_pre = sum dh xh
//     w = c g gamma_post t,  dy = r_y (w - yh mean(w yh)),  dgamma_post = sum c g t yh,  dg = c t n.
// x' is computed again from x and y in the backward (the bytes are those of x' itself, and no
// rounding of x' comes in), the mask from its counters.  Both means are known from one round of
// sums: mean(w yh) = mean(q b) - r_x mean(e xh) mean(q xh), with q = c g gamma_post yh and b = dx' + r_x e.
//
// A row lies on W warps, eight neighbouring columns (C times) on a thread; a block has G such
// groups, each with its own rows.  Rows arrive by asynchronous copies, a few ahead, in a ring of
// the warp's own in shared memory, so that no registers hold what is under way.  Sums over tokens
// stay in registers and leave once a block; a second kernel adds the blocks' up in order.
#include <algorithm>

#include "block.h"
#include "launch.h"
#include "profile.h"

namespace mosa {
namespace blk {
namespace {

constexpr int kThreads = 512, kSms = 152;
constexpr int kIn = 5;              // tensors that may arrive: x, y, gate, dx_out, dh
constexpr int kMaxStages = 4;
constexpr int kSmem = 200 * 1024;   // of a block that has an SM to itself
constexpr int kScratch = 1024;      // bytes of a warp: 256 columns on their way out

struct Args {
    Residual r;
    float *partial;     // backward: [blocks][3][d] sums over tokens, of gamma_post, gamma_pre, gate
    int warps, groups;  // W, G
    int stages, stage_bytes;
    int off[kIn];       // of each tensor within a warp's stage
};

__device__ __forceinline__ uint32_t smem_at(const void *p) { return (uint32_t)__cvta_generic_to_shared(p); }

// 16 bytes on their way to shared memory, `bytes` of them from src (the others are 0).
__device__ __forceinline__ void copy16(uint32_t dst, const void *src, int bytes) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(bytes) : "memory");
}
__device__ __forceinline__ void copies_end() { asm volatile("cp.async.commit_group;" ::: "memory"); }
// All but the last n rounds of copies have arrived.
__device__ __forceinline__ void copies_wait(int n) {
    if (n == 3) asm volatile("cp.async.wait_group 3;" ::: "memory");
    else if (n == 2) asm volatile("cp.async.wait_group 2;" ::: "memory");
    else if (n == 1) asm volatile("cp.async.wait_group 1;" ::: "memory");
    else asm volatile("cp.async.wait_group 0;" ::: "memory");
}

// 256 columns of a warp in shared memory: 16-byte pieces in order, those of fp32 with every second run
// of eight swapped in pairs, so that lanes that read two neighbouring pieces each meet no bank twice.
__device__ __forceinline__ int piece_at(int j) { return 16 * (j ^ ((j >> 3) & 1)); }

// The columns [col, col + 256) of a row, as far as there are any (0 beyond d), to `to`.
__device__ __forceinline__ void fetch(const Rows &m, const char *row, int col, int d, char *to, int lane) {
    if (m.vec) {
        if (m.wide) {
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const int j = lane + 32 * i, at = col + 4 * j, n = min(max((d - at) * 4, 0), 16);
                copy16(smem_at(to + piece_at(j)), n > 0 ? row + at * 4 : row, n);
            }
        } else {
            const int at = col + 8 * lane, n = min(max((d - at) * 2, 0), 16);
            copy16(smem_at(to + 16 * lane), n > 0 ? row + at * 2 : row, n);
        }
    } else if (m.wide) {
        float v[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int at = col + 32 * i + lane;
            v[i] = at < d ? reinterpret_cast<const float *>(row)[at] : 0.f;
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int e = 32 * i + lane;
            *reinterpret_cast<float *>(to + piece_at(e >> 2) + 4 * (e & 3)) = v[i];
        }
    } else {
        unsigned short v[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int at = col + 32 * i + lane;
            v[i] = at < d ? reinterpret_cast<const unsigned short *>(row)[at] : (unsigned short)0;
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) *reinterpret_cast<unsigned short *>(to + 2 * (32 * i + lane)) = v[i];
    }
}

__device__ __forceinline__ void unpack2(uint32_t w, float &a, float &b) {
    a = __uint_as_float(w << 16);
    b = __uint_as_float(w & 0xFFFF0000u);
}

// The lane's eight columns of what fetch brought.
__device__ __forceinline__ void take(const char *from, int wide, int lane, float (&v)[8]) {
    if (wide) {
        const float4 a = *reinterpret_cast<const float4 *>(from + piece_at(2 * lane));
        const float4 b = *reinterpret_cast<const float4 *>(from + piece_at(2 * lane + 1));
        v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w;
        v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
    } else {
        const uint4 a = *reinterpret_cast<const uint4 *>(from + 16 * lane);
        unpack2(a.x, v[0], v[1]);
        unpack2(a.y, v[2], v[3]);
        unpack2(a.z, v[4], v[5]);
        unpack2(a.w, v[6], v[7]);
    }
}

__device__ __forceinline__ uint32_t pack2(float a, float b) {
    uint32_t w;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(w) : "f"(b), "f"(a));
    return w;
}

// The warp's 256 columns from `col` on to a row, through its scratch where lanes' own eight columns
// are not the pieces that leave together.
__device__ __forceinline__ void put(const Rows &m, char *row, int col, int d, char *scratch, int lane,
                                    const float (&v)[8]) {
    if (!m.wide) {
        const uint4 w = make_uint4(pack2(v[0], v[1]), pack2(v[2], v[3]), pack2(v[4], v[5]), pack2(v[6], v[7]));
        const int at = col + 8 * lane;
        if (m.vec && col + 256 <= d) {
            *reinterpret_cast<uint4 *>(row + 2 * at) = w;
            return;
        }
        __syncwarp();
        *reinterpret_cast<uint4 *>(scratch + 16 * lane) = w;
        __syncwarp();
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int e = 32 * i + lane;
            if (col + e < d)
                reinterpret_cast<unsigned short *>(row)[col + e] = *reinterpret_cast<unsigned short *>(scratch + 2 * e);
        }
        return;
    }
    __syncwarp();
    *reinterpret_cast<float4 *>(scratch + piece_at(2 * lane)) = make_float4(v[0], v[1], v[2], v[3]);
    *reinterpret_cast<float4 *>(scratch + piece_at(2 * lane + 1)) = make_float4(v[4], v[5], v[6], v[7]);
    __syncwarp();
    if (m.vec && col + 256 <= d) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int j = lane + 32 * i;
            reinterpret_cast<float4 *>(row)[col / 4 + j] = *reinterpret_cast<const float4 *>(scratch + piece_at(j));
        }
        return;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int e = 32 * i + lane;
        if (col + e < d)
            reinterpret_cast<float *>(row)[col + e] =
                *reinterpret_cast<const float *>(scratch + piece_at(e >> 2) + 4 * (e & 3));
    }
}

// Eight values of a vector [d] (1 where there is none, 0 beyond d).
__device__ __forceinline__ void vector8(const Vec &m, int at, int d, float (&v)[8]) {
    if (m.p == nullptr) {
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = 1.f;
    } else if (m.vec && at + 8 <= d) {
        if (m.wide) {
            const float4 a = static_cast<const float4 *>(m.p)[at / 4], b = static_cast<const float4 *>(m.p)[at / 4 + 1];
            v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w;
            v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
        } else {
            const uint4 a = static_cast<const uint4 *>(m.p)[at / 8];
            unpack2(a.x, v[0], v[1]);
            unpack2(a.y, v[2], v[3]);
            unpack2(a.z, v[4], v[5]);
            unpack2(a.w, v[6], v[7]);
        }
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            v[e] = 0.f;
            if (at + e < d)
                v[e] = m.wide ? static_cast<const float *>(m.p)[at + e] : to_f32(static_cast<const bf16 *>(m.p)[at + e]);
        }
    }
}

// Sums of N values over the threads of a row's warps, in every thread, in an order that is always the same.
template <int N>
__device__ __forceinline__ void row_sums(float (&v)[N], float4 *red, int W, int w, int lane, int group) {
#pragma unroll
    for (int i = 0; i < N; ++i)
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) v[i] += __shfl_xor_sync(0xffffffffu, v[i], o);
    if (W == 1) return;
    if (lane == 0) red[w] = make_float4(v[0], N > 1 ? v[1 % N] : 0.f, N > 2 ? v[2 % N] : 0.f, 0.f);
    asm volatile("bar.sync %0, %1;" ::"r"(group + 1), "r"(W * 32) : "memory");
    const float4 s = red[lane & (W - 1)];
    v[0] = s.x;
    if (N > 1) v[1 % N] = s.y;
    if (N > 2) v[2 % N] = s.z;
    for (int o = W >> 1; o > 0; o >>= 1)
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] += __shfl_xor_sync(0xffffffffu, v[i], o);
}

__device__ __forceinline__ float logistic(float x) { return 1.f / (1.f + __expf(-x)); }

template <int C, bool kBackward>
__global__ void __launch_bounds__(kThreads, !kBackward && C == 1 ? 2 : 1) residual_kernel(const __grid_constant__ Args p) {
    asm volatile("griddepcontrol.wait;" ::: "memory");
    extern __shared__ __align__(16) char smem[];
    const Residual &r = p.r;
    const int W = p.warps, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int group = warp / W, w = warp - group * W, nwarps = W * p.groups;
    char *ring = smem + warp * p.stages * p.stage_bytes;
    char *scratch = smem + nwarps * p.stages * p.stage_bytes + warp * kScratch;
    // two sets of a group's sums, taken in turn: one barrier a round
    float4 *red = reinterpret_cast<float4 *>(smem + nwarps * (p.stages * p.stage_bytes + kScratch)) + group * 2 * W;
    const int d = r.d, span = W * 256;
    const long long rows = (long long)r.B * r.T, step = (long long)gridDim.x * p.groups;
    const float inv_d = 1.f / d;
    const DropKey key = drop_key(r.drop);
    const bool drops = r.drop.rng != nullptr;
    const float unit = r.scale * (drops ? r.drop.scale : 1.f);   // c of a kept value

    auto issue = [&](long long row, int slot) {
        if (row < rows) {
            const int b = (uint32_t)row / (uint32_t)r.T, t = (int)((uint32_t)row - (uint32_t)b * (uint32_t)r.T);
            const Rows *in[kIn] = {&r.x, &r.y, &r.g, &r.dxo, &r.dh};
#pragma unroll
            for (int i = 0; i < (kBackward ? kIn : 3); ++i) {
                if (in[i]->p == nullptr) continue;
                const char *at = in[i]->at(b, t);
#pragma unroll
                for (int c = 0; c < C; ++c)
                    fetch(*in[i], at, c * span + w * 256, d,
                          ring + slot * p.stage_bytes + p.off[i] + c * (in[i]->wide ? 1024 : 512), lane);
            }
        }
        copies_end();
    };

    long long row = (long long)blockIdx.x * p.groups + group;
    const int ahead = p.stages - 1;
    for (int i = 0; i < ahead; ++i) issue(row + i * step, i);
    int slot = 0, turn = 0;
    float acc[3][C][8];
#pragma unroll
    for (int i = 0; i < 3; ++i)
#pragma unroll
        for (int c = 0; c < C; ++c)
#pragma unroll
            for (int e = 0; e < 8; ++e) acc[i][c][e] = 0.f;
    float ry = 1.f, rx = 1.f, next_ry = 1.f, next_rx = 1.f;
    if (kBackward && row < rows) {
        next_ry = r.stats[row];
        next_rx = r.stats[rows + row];
    }
    for (; row < rows; row += step) {
        const int b = (uint32_t)row / (uint32_t)r.T, t = (int)((uint32_t)row - (uint32_t)b * (uint32_t)r.T);
        __syncwarp();   // (the slot that is filled next has been read by all lanes)
        issue(row + ahead * step, slot == 0 ? ahead : slot - 1);
        copies_wait(ahead);
        __syncwarp();
        const char *in = ring + slot * p.stage_bytes;
        slot = slot == ahead ? 0 : slot + 1;
        auto at = [&](int i, const Rows &m, int c, float (&v)[8]) {
            take(in + p.off[i] + c * (m.wide ? 1024 : 512), m.wide, lane, v);
        };
        uint32_t kept[C];
#pragma unroll
        for (int c = 0; c < C; ++c)
            kept[c] = drops ? kept8(r.drop, key, (uint32_t)row, (uint32_t)(c * span / 8 + w * 32 + lane)) : 0xFFu;
        // The gate of eight columns: its value, and with `slope` what its gradient is multiplied by.
        auto gate8 = [&](int c, float (&g)[8]) {
            if (r.gate == MOSA_GATE_TOKEN) at(2, r.g, c, g);
            else vector8(r.gch, c * span + w * 256 + 8 * lane, d, g);
            if (r.sigmoid && r.gate != MOSA_GATE_NONE) {
#pragma unroll
                for (int e = 0; e < 8; ++e) g[e] = logistic(g[e]);
            }
        };
        if (kBackward) {
            ry = next_ry;
            rx = next_rx;
            if (row + step < rows) {
                next_ry = r.stats[row + step];
                next_rx = r.stats[rows + row + step];
            }
            if (!r.post) ry = 1.f;
        } else if (r.post) {
            float s[1] = {0.f};
#pragma unroll
            for (int c = 0; c < C; ++c) {
                float y[8];
                at(1, r.y, c, y);
#pragma unroll
                for (int e = 0; e < 8; ++e) s[0] = fmaf(y[e], y[e], s[0]);
            }
            row_sums<1>(s, red + turn * W, W, w, lane, group);
            turn ^= 1;
            ry = rsqrtf(fmaf(s[0], inv_d, r.eps));
        }
        // yh, gate and x' of eight columns
        auto forward8 = [&](int c, float (&yh)[8], float (&gm)[8], float (&g)[8], float (&x)[8]) {
            at(1, r.y, c, yh);
            at(0, r.x, c, x);
            gate8(c, g);
            vector8(r.gpost, c * span + w * 256 + 8 * lane, d, gm);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                yh[e] *= ry;
                // (a dropped value is chosen away, whatever it holds)
                const float u = unit * (g[e] * (yh[e] * gm[e]));
                x[e] += kept[c] >> e & 1 ? u : 0.f;
            }
        };
        if constexpr (!kBackward) {
            float x[C][8], s[1] = {0.f};
            char *xo = r.xo.at(b, t);
#pragma unroll
            for (int c = 0; c < C; ++c) {
                float yh[8], gm[8], g[8];
                forward8(c, yh, gm, g, x[c]);
                put(r.xo, xo, c * span + w * 256, d, scratch, lane, x[c]);
                const int n = d - (c * span + w * 256 + 8 * lane);   // columns there are
#pragma unroll
                for (int e = 0; e < 8; ++e) s[0] = fmaf(e < n ? x[c][e] : 0.f, x[c][e], s[0]);
            }
            if (r.pre) {
                row_sums<1>(s, red + turn * W, W, w, lane, group);
                turn ^= 1;
                rx = rsqrtf(fmaf(s[0], inv_d, r.eps));
                char *h = r.h.at(b, t);
#pragma unroll
                for (int c = 0; c < C; ++c) {
                    float gm[8];
                    vector8(r.gpre, c * span + w * 256 + 8 * lane, d, gm);
#pragma unroll
                    for (int e = 0; e < 8; ++e) x[c][e] *= rx * gm[e];
                    put(r.h, h, c * span + w * 256, d, scratch, lane, x[c]);
                }
            }
            if (r.stats != nullptr && w == 0 && lane == 0) {
                r.stats[row] = ry;
                r.stats[rows + row] = rx;
            }
        } else {
            float base[C][8], s[3] = {0.f, 0.f, 0.f};
            // xh, yh, gate and n of eight columns (0 beyond d), from what the ring holds
            auto values = [&](int c, float (&xh)[8], float (&yh)[8], float (&gm)[8], float (&g)[8]) {
                forward8(c, yh, gm, g, xh);
#pragma unroll
                for (int e = 0; e < 8; ++e) xh[e] *= rx;
            };
#pragma unroll
            for (int c = 0; c < C; ++c) {
                float xh[8], yh[8], gm[8], g[8], dh[8], gp[8];
                values(c, xh, yh, gm, g);
#pragma unroll
                for (int e = 0; e < 8; ++e) base[c][e] = 0.f;
                if (r.dxo.p != nullptr) at(3, r.dxo, c, base[c]);
                if (r.dh.p != nullptr) {
                    at(4, r.dh, c, dh);
                    vector8(r.gpre, c * span + w * 256 + 8 * lane, d, gp);
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        acc[1][c][e] = fmaf(dh[e], xh[e], acc[1][c][e]);
                        const float q = dh[e] * gp[e];
                        s[0] = fmaf(q, xh[e], s[0]);
                        base[c][e] = fmaf(rx, q, base[c][e]);
                    }
                }
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const float q = kept[c] >> e & 1 ? unit * g[e] * gm[e] * yh[e] : 0.f;
                    s[1] = fmaf(q, base[c][e], s[1]);
                    s[2] = fmaf(q, xh[e], s[2]);
                }
            }
            row_sums<3>(s, red + turn * W, W, w, lane, group);
            turn ^= 1;
            const float m1 = r.dh.p != nullptr ? rx * s[0] * inv_d : 0.f;   // r_x mean(e xh)
            const float m2 = r.post ? (s[1] - m1 * s[2]) * inv_d : 0.f;     // mean(w yh)
#pragma unroll
            for (int c = 0; c < C; ++c) {
                const int col = c * span + w * 256;
                float xh[8], yh[8], gm[8], g[8], dg[8];
                values(c, xh, yh, gm, g);
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    base[c][e] = fmaf(-m1, xh[e], base[c][e]);
                    const bool on = kept[c] >> e & 1;
                    const float ct = unit * base[c][e], f = on ? ct * g[e] : 0.f;
                    dg[e] = on ? ct * (yh[e] * gm[e]) : 0.f;
                    if (r.sigmoid) dg[e] *= g[e] * (1.f - g[e]);
                    acc[0][c][e] = fmaf(f, yh[e], acc[0][c][e]);
                    acc[2][c][e] += dg[e];
                    yh[e] = r.post ? ry * fmaf(-yh[e], m2, f * gm[e]) : f;
                }
                put(r.dx, r.dx.at(b, t), col, d, scratch, lane, base[c]);
                put(r.dy, r.dy.at(b, t), col, d, scratch, lane, yh);
                if (r.dg.p != nullptr) put(r.dg, r.dg.at(b, t), col, d, scratch, lane, dg);
            }
        }
    }
    if (kBackward && p.partial != nullptr) {
        copies_wait(0);
        __syncthreads();
        float *sums = p.groups > 1 ? reinterpret_cast<float *>(smem) : p.partial + (long long)blockIdx.x * 3 * d;
        const int width = p.groups > 1 ? span * C : d;
#pragma unroll
        for (int i = 0; i < 3; ++i)
#pragma unroll
            for (int c = 0; c < C; ++c)
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const int col = c * span + w * 256 + 8 * lane + e;
                    if (col < d) sums[(group * 3 + i) * width + col] = acc[i][c][e];
                }
        if (p.groups > 1) {
            __syncthreads();
            for (int o = threadIdx.x; o < 3 * d; o += blockDim.x) {
                const int i = o / d, col = o - i * d;
                float sum = 0.f;
                for (int g = 0; g < p.groups; ++g) sum += sums[(g * 3 + i) * width + col];
                p.partial[(long long)blockIdx.x * 3 * d + o] = sum;
            }
        }
    }
}

// The sums over tokens from the blocks': 32 columns a block, 32 runs of blocks each, in a fixed order.
__global__ void __launch_bounds__(1024) residual_sums_kernel(const float *partial, int blocks, int d,
                                                             float *dgpost, float *dgpre, float *dgate) {
    asm volatile("griddepcontrol.wait;" ::: "memory");
    __shared__ float red[32][33];
    const int cc = threadIdx.x & 31, run = threadIdx.x >> 5, col = blockIdx.x * 32 + cc;
    float sum = 0.f;
    if (col < 3 * d)
        for (int b = run; b < blocks; b += 32) sum += partial[(long long)b * 3 * d + col];
    red[run][cc] = sum;
    __syncthreads();
    if (run == 0 && col < 3 * d) {
        float t = 0.f;
        for (int u = 0; u < 32; ++u) t += red[u][cc];
        const int i = col / d;
        float *out = i == 0 ? dgpost : i == 1 ? dgpre : dgate;
        if (out != nullptr) out[col - i * d] = t;
    }
}

// Warps of a row (eight columns a thread, up to 16 warps), and how often eight columns (rows of more
// than 8192 are refused: five fp32 rows of that width fill a block's shared memory).
int warps_of(int d) {
    int W = 1;
    while (W < kThreads / 32 && W * 256 < d) W *= 2;
    return W;
}
int times_of(int d) {
    const int W = warps_of(d);
    return d <= W * 256 ? 1 : 2;
}

// Groups of a block: as many as there are threads for, but blocks for all SMs first.
int groups_of(const Residual &r) {
    const long long rows = (long long)r.B * r.T, most = kThreads / 32 / warps_of(r.d);
    return (int)std::min(most, std::max(1LL, rows / kSms));
}

int blocks_of(const Residual &r, int per_sm) {
    const long long rows = (long long)r.B * r.T, G = groups_of(r);
    return (int)std::min<long long>((rows + G - 1) / G, kSms * per_sm);
}

template <int C, bool kBackward>
cudaError_t launch_as(Args &p, int blocks, int limit, cudaStream_t s) {
    const Residual &r = p.r;
    const Rows *in[kIn] = {&r.x, &r.y, &r.g, &r.dxo, &r.dh};
    p.stage_bytes = 0;
    for (int i = 0; i < kIn; ++i) {
        p.off[i] = p.stage_bytes;
        if (in[i]->p != nullptr) p.stage_bytes += C * (in[i]->wide ? 1024 : 512);
    }
    const int nwarps = p.warps * p.groups, fixed = nwarps * (kScratch + 2 * 16);
    p.stages = std::min(kMaxStages, (limit - fixed) / (nwarps * p.stage_bytes));
    int bytes = nwarps * p.stages * p.stage_bytes + fixed;
    if (kBackward && p.groups > 1) bytes = std::max(bytes, p.groups * 3 * p.warps * 256 * C * 4);
    cudaError_t e = allow_smem((const void *)residual_kernel<C, kBackward>, kSmem);
    if (e != cudaSuccess) return e;
    e = launch_pdl(residual_kernel<C, kBackward>, dim3(blocks), dim3(nwarps * 32), bytes, s, p);
    note_launches(1);
    return e;
}

template <bool kBackward>
cudaError_t launch(Args &p, cudaStream_t s) {
    const int C = times_of(p.r.d);
    p.warps = warps_of(p.r.d);
    p.groups = groups_of(p.r);
    if (C == 1) return launch_as<1, kBackward>(p, blocks_of(p.r, kBackward ? 1 : 2), kBackward ? kSmem : kSmem / 2, s);
    return launch_as<2, kBackward>(p, blocks_of(p.r, 1), kSmem, s);
}

}  // namespace

size_t residual_workspace(const Residual &r) { return (size_t)blocks_of(r, 1) * 3 * r.d * sizeof(float); }

cudaError_t launch_residual(const Residual &r, cudaStream_t s) {
    Args p{};
    p.r = r;
    return launch<false>(p, s);
}

cudaError_t launch_residual_bwd(const Residual &r, float *partial, cudaStream_t s) {
    Args p{};
    p.r = r;
    const bool sums = r.dgpost != nullptr || r.dgpre != nullptr || r.dgate != nullptr;
    p.partial = sums ? partial : nullptr;
    cudaError_t e = launch<true>(p, s);
    if (e != cudaSuccess || !sums) return e;
    e = launch_pdl(residual_sums_kernel, dim3((3 * r.d + 31) / 32), dim3(1024), 0, s, (const float *)partial,
                   blocks_of(r, 1), r.d, r.dgpost, r.dgpre, r.dgate);
    note_launches(1);
    return e;
}

}  // namespace blk
}  // namespace mosa
