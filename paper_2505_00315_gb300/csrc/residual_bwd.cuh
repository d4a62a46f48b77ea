// The residual step's backward, one pass over its tensors.  With yh = r_y y, xh = r_x x', e = dh gamma_pre and
// c = scale keep/(1-p),
//     t = dx' + r_x (e - xh mean(e xh)),  dx = t,  dgamma_pre = sum dh xh
//     w = c g gamma_post t,  dy = r_y (w - yh mean(w yh)),  dgamma_post = sum c g t yh,  dg = c t n.
// x' is computed again from x and y (the bytes are those of x' itself, and no rounding of x' comes in),
// the mask from its counters.  Both means are known from one round of sums: with u = c g gamma_post yh and
// b = dx' + r_x e, mean(w yh) = mean(u b) - r_x mean(e xh) mean(u xh).  Sums over tokens stay in
// registers and leave once a block; a second kernel adds the blocks' up in order.
// x, y, dx', dh (and a gate per token) come in, dx, dy (and the gate's gradient) go out, once.  What bounds it at bf16 is the chain of
// a row (arrival, sums over the warps, second round: 2 us) on the few warps that 250 registers a thread leave; at fp32 and
// at wide rows the bytes.  us and share of the copy rate, the second kernel's 5 us among them: B4 T4096 d1024, fp32 y and dh, gate
// per channel, dropout 54 (74%); B2 T8192 d4096, fp32 stream, gate per token, dropout 244 (89%); fp32, 16384 rows of
// 2048, 128 (92%).  A spill of two registers cost a fifth (16384 rows of 768, fp32 stream, y and dh: 66 us, 56 without); the kernels of
// 16 warps that still have some (4 to 24 bytes) were not seen to gain from less.
#pragma once

#include "residual.cuh"

namespace mosa {
namespace blk {

// kMost: warps of a block at most.  kCut: sequences lie apart; kernels of their own, since the jumps between them cost
// registers (B2 T8192 d4096: 248 us in one kernel with the others, 242).  kSecond: the second norm has a gradient (dh).
// Without one, dx is dx_out whatever x and y hold, so nothing of xh is computed, since 0 times an infinity of it would
// count; kernels of their own for it, since a choice in each row moves registers (8192 rows of 8192: 170 -> 178 us).
template <int C, int kMost, class Ty, bool kCut, bool kSecond>
__global__ void __launch_bounds__(kMost * 32, 1) residual_bwd_kernel(const __grid_constant__ Args p) {
    asm volatile("griddepcontrol.wait;" ::: "memory");
    constexpr bool kFast = Ty::kFast;
    extern __shared__ __align__(16) char smem[];
    const Residual &r = p.r;
    const Place l(p, smem, C);
    const DropKey key = drop_key(r.drop);
    const bool drops = r.drop.rng != nullptr, token = r.gate == MOSA_GATE_TOKEN;
    const bool has_dxo = r.dxo.p != nullptr;
    const float unit = r.scale * (drops ? r.drop.scale : 1.f), inv_d = 1.f / l.d;   // unit: c of a kept value
    if (l.d < 256 * C * l.W || !has_dxo) clear_ring(l);
    uint32_t row = blockIdx.x * p.groups + l.group;   // (row + kMaxStages step fits 32 bits)
    Arrival<C, kFast, Ty::x> x_in, dxo_in;
    Arrival<C, kFast, Ty::y> y_in;
    Arrival<C, kFast, Ty::dh> dh_in;
    Arrival<C, kFast, Ty::storage> g_in;
    x_in.init(p, l, r.x, row);
    y_in.init(p, l, r.y, row);
    dxo_in.init(p, l, r.dxo, row);
    dh_in.init(p, l, r.dh, row);
    g_in.init(p, l, r.g, row);
    Departure<C, kFast, Ty::x, Ty::storage == 0> dx_out;
    Departure<C, kFast, Ty::storage> dy_out, dg_out;
    dx_out.init(p, l, r.dx, row);
    dy_out.init(p, l, r.dy, row);
    dg_out.init(p, l, r.dg, row);
    // Where the tensors' columns lie in a stage.
    const int y_off = kFast ? bytes_of(Ty::x, C) : p.off[1], dxo_off = kFast ? y_off + bytes_of(Ty::y, C) : p.off[2];
    const int dh_off = kFast ? dxo_off + bytes_of(Ty::x, C) : p.off[3];
    const int g_off = kFast ? dh_off + bytes_of(Ty::dh, C) : p.off[4];
    auto fill = [&](uint32_t at, int slot) {
        const uint32_t to = l.ring32 + slot * p.stage_bytes;
        if (kSecond) x_in.issue(p, l, r.x, at, to);
        y_in.issue(p, l, r.y, at, to + y_off);
        if (has_dxo) dxo_in.issue(p, l, r.dxo, at, to + dxo_off);
        if (kSecond) dh_in.issue(p, l, r.dh, at, to + dh_off);
        if (token) g_in.issue(p, l, r.g, at, to + g_off);
    };
    auto jump = [&](uint32_t at) {   // (after fill)
        const int ends = ends_between(p, l, at);
        if (kSecond) x_in.jump(r.x, ends);
        y_in.jump(r.y, ends);
        dxo_in.jump(r.dxo, ends);
        if (kSecond) dh_in.jump(r.dh, ends);
        g_in.jump(r.g, ends);
    };
    const int ahead = p.stages - 1;
    for (int i = 0; i < ahead; ++i) {
        if (row + i * l.step < l.rows) fill(row + i * l.step, i);
        if (kCut) jump(row + i * l.step);
        copies_end();
    }
    if (Ty::kHeld || (!Ty::kLies && p.held)) hold<C, false>(p, l, unit);

    int slot = 0, turn = 0;
    // Sums over tokens: 0 of gamma_post over c g, which the gate of a channel shares (each has a factor of
    // the column's own), with a gate per token of gamma_post itself; 1 of gamma_pre.
    Oct acc[2][C];
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int c = 0; c < C; ++c) acc[i][c] = zeros();
    float next_ry = 1.f, next_rx = 1.f;
    if (row < l.rows) {
        next_ry = r.stats[row];
        if (kSecond) next_rx = r.stats[(uint64_t)l.rows + row];
    }
    for (; row < l.rows; row += l.step) {
        __syncwarp();   // (the slot that is filled next has been read by all lanes)
        if (row + ahead * l.step < l.rows) fill(row + ahead * l.step, slot == 0 ? ahead : slot - 1);
        copies_end();
        const float ry = r.post ? next_ry : 1.f, rx = next_rx;
        if (row + l.step < l.rows) {
            next_ry = r.stats[row + l.step];
            if (kSecond) next_rx = r.stats[(uint64_t)l.rows + row + l.step];
        }
        uint32_t bits[C];
#pragma unroll
        for (int c = 0; c < C; ++c) bits[c] = 0xFFu;
        if (drops) {
#pragma unroll
            for (int c = 0; c < C; ++c) bits[c] = kept8(r.drop, key, row, (uint32_t)l.column(c) >> 3);
        }
        copies_wait(ahead);
        __syncwarp();
        const char *in = l.ring + slot * p.stage_bytes;
        slot = slot == ahead ? 0 : slot + 1;
        const int xw = wide_of(Ty::x, r.x), yw = wide_of(Ty::y, r.y), hw = wide_of(Ty::dh, r.dh);
        const int gw = wide_of(Ty::storage, r.g);
        const int xs = x_in.shift(p, l, r.x, row), ys = y_in.shift(p, l, r.y, row), gs = token ? g_in.shift(p, l, r.g, row) : -1;
        const int dxos = has_dxo ? dxo_in.shift(p, l, r.dxo, row) : -1, dhs = kSecond ? dh_in.shift(p, l, r.dh, row) : -1;
        auto token_gate = [&](int c, bool slope) {
            const Oct g = arrived<kFast>(in + g_off, gw, l, c, gs);
            return !r.sigmoid ? g : slope ? logistic_slope(g) : logistic(g);
        };
        // What both rounds need, from what the ring holds.  kEarly: all of it is fetched first (us, first / when needed: B2 T8192
        // d4096 243.7 / 246.3, 4096 rows of 8192 with a gate per channel and dropout 140 / 144; with 8 columns a thread, which
        // spills sooner, 16384 rows of 768 in fp32 71.6 / 70.4).
        constexpr bool kEarly = C > 1;
        struct Values {
            Oct yh, xh, cg, base;   // cg: c g (0 where dropped); base: dx' + r_x e
        };
        auto values = [&](int c, Oct &u, Oct &dh, Oct &e) {
            Values v;
            const Oct y = arrived<kFast>(in + y_off, yw, l, c, ys);
            Oct x = zeros();
            if (kSecond && kEarly) x = arrived<kFast>(in, xw, l, c, xs);
            const Oct dxo = arrived<kFast>(in + dxo_off, xw, l, c, dxos);
            if (kSecond && kEarly) dh = arrived<kFast>(in + dh_off, hw, l, c, dhs);
            v.cg = token ? times(token_gate(c, false), unit)
                   : r.gate == MOSA_GATE_NONE ? all_of(unit) : vector_at<C, false, Ty>(p, l, 2, c, unit);
            v.yh = times(y, ry);
            if (drops) {
                v.cg = chosen(v.cg, bits[c]);
                // (with a norm, a NaN is one in its whole row; an infinity makes r_y 0, and counts only where it is kept)
                if (!r.post || ry == 0.f) v.yh = chosen(v.yh, bits[c]);
            }
            u = times(times(v.yh, vector_at<C, false, Ty>(p, l, 0, c, unit)), v.cg);
            if (kSecond) {
                if (!kEarly) {
                    x = arrived<kFast>(in, xw, l, c, xs);
                    dh = arrived<kFast>(in + dh_off, hw, l, c, dhs);
                }
                v.xh = times(plus(x, u), rx);
                e = times(dh, vector_at<C, false, Ty>(p, l, 1, c, unit));
                v.base = fused(e, rx, dxo);
            } else {
                v.base = dxo;
            }
            return v;
        };
        // (they stay in registers from one round to the other where those suffice)
        constexpr bool kStay = C <= 2;
        Values stay[C];
        Pair s0 = 0, s1 = 0, s2 = 0;
#pragma unroll
        for (int c = 0; c < C; ++c) {
            Oct u, dh, e;
            const Values v = values(c, u, dh, e);
            if (kStay) stay[c] = v;
            if (kSecond) {
                acc[1][c] = fused(dh, v.xh, acc[1][c]);
                add_products(s0, e, v.xh);
            }
            add_products(s1, u, v.base);
            if (kSecond) add_products(s2, u, v.xh);
        }
        const float4 s = row_sums(sum_of(s0), sum_of(s1), sum_of(s2), l.red + turn * l.W, l.W, l.w, l.lane, l.group);
        turn ^= 1;
        const float m1 = rx * s.x * inv_d;                      // r_x mean(e xh)
        const float m2 = r.post ? (s.y - m1 * s.z) * inv_d : 0.f;   // mean(w yh)
        dx_out.begin(p, r.dx, row);
        dy_out.begin(p, r.dy, row);
        if (r.dg.p != nullptr) dg_out.begin(p, r.dg, row);
#pragma unroll
        for (int c = 0; c < C; ++c) {
            Oct u, dh, e;
            Values v = stay[c];
            if (!kStay) v = values(c, u, dh, e);
            const Oct gamma = vector_at<C, false, Ty>(p, l, 0, c, unit);
            const Oct t = kSecond ? fused(v.xh, -m1, v.base) : v.base, f = times(t, v.cg);
            dx_out.put_row(l, r.dx, c, t);
            if (token) {
                acc[0][c] = fused(f, v.yh, acc[0][c]);
                if (r.dg.p != nullptr) {
                    Oct g = times(times(t, unit), times(v.yh, gamma));
                    if (r.sigmoid) g = times(g, token_gate(c, true));
                    if (drops) g = chosen(g, bits[c]);
                    dg_out.put_row(l, r.dg, c, g);
                }
            } else {
                acc[0][c] = fused(drops ? chosen(t, bits[c]) : t, v.yh, acc[0][c]);
            }
            // (without a norm of y dy does not see it, and an infinity may not meet m2 = 0; with the second norm its
            // row is lost anyhow)
            const Oct w = times(f, gamma);
            dy_out.put_row(l, r.dy, c, kSecond || r.post ? times(fused(v.yh, -m2, w), ry) : w);
        }
        dx_out.end(l, r.dx);
        dy_out.end(l, r.dy);
        dg_out.end(l, r.dg);
        if (kCut) {
            jump(row + ahead * l.step);
            const int ends = ends_between(p, l, row);
            dx_out.jump(r.dx, ends);
            dy_out.jump(r.dy, ends);
            dg_out.jump(r.dg, ends);
        }
    }
    if (p.partial != nullptr) {
        copies_wait(0);
        __syncthreads();
        float *sums = p.groups > 1 ? reinterpret_cast<float *>(smem) : p.partial + (long long)blockIdx.x * 3 * l.d;
        const int width = p.groups > 1 ? 256 * C * l.W : l.d;
#pragma unroll
        for (int c = 0; c < C; ++c) {
            Oct of[3] = {acc[0][c], acc[1][c], zeros()};   // of gamma_post, gamma_pre, gate
            if (!token) {
                const Oct own = acc[0][c];
                of[0] = times(own, vector_of<false>(r, 2, l.column(c), unit));
                if (r.gate == MOSA_GATE_CHANNEL) {
                    of[2] = times(times(own, unit), vector_of<false>(r, 0, l.column(c), unit));
                    if (r.sigmoid) of[2] = times(of[2], logistic_slope(vector8(r.gch, l.column(c), l.d)));
                }
            }
#pragma unroll
            for (int i = 0; i < 3; ++i)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int col = l.column(c) + 2 * e;
                    const F2 f = of_two(of[i].v[e]);
                    if (col < l.d) sums[(l.group * 3 + i) * width + col] = f.x;
                    if (col + 1 < l.d) sums[(l.group * 3 + i) * width + col + 1] = f.y;
                }
        }
        if (p.groups > 1) {
            __syncthreads();
            for (int o = threadIdx.x; o < 3 * l.d; o += blockDim.x) {
                const int i = o / l.d, col = o - i * l.d;
                float sum = 0.f;
                for (int g = 0; g < p.groups; ++g) sum += sums[(g * 3 + i) * width + col];
                p.partial[(long long)blockIdx.x * 3 * l.d + o] = sum;
            }
        }
    }
}

// The kernel for a call's types.
template <int C, int kMost, class Ty, bool kCut, bool kSecond>
cudaError_t go(const Args &p, int blocks, int bytes, cudaStream_t s) {
    const auto kernel = residual_bwd_kernel<C, kMost, Ty, kCut, kSecond>;
    cudaError_t e = allow_smem((const void *)kernel, kSmem);
    if (e != cudaSuccess) return e;
    note_launches(1);
    return launch_pdl(kernel, dim3(blocks), dim3(p.warps * p.groups * 32), bytes, s, p);
}
template <int C, int kMost, bool kCut, bool kSecond>
cudaError_t go_by_types(const Args &p, int blocks, int bytes, cudaStream_t s) {
    const Residual &r = p.r;
    const int x = r.x.wide, y = r.y.wide, dh = r.dh.wide, st = r.storage_wide;
    if constexpr (C == 4)
        if (!p.held) return go<C, kMost, Types<1, 1, 1, 1, 0>, kCut, kSecond>(p, blocks, bytes, s);
    if (st) return go<C, kMost, Types<1, 1, 1, 1>, kCut, kSecond>(p, blocks, bytes, s);
    if constexpr (kSecond)   // (else dh counts as of the storage type)
        if (dh) switch (2 * x + y) {
            case 0: return go<C, kMost, Types<0, 0, 1, 0>, kCut, true>(p, blocks, bytes, s);
            case 1: return go<C, kMost, Types<0, 1, 1, 0>, kCut, true>(p, blocks, bytes, s);
            case 2: return go<C, kMost, Types<1, 0, 1, 0>, kCut, true>(p, blocks, bytes, s);
            default: return go<C, kMost, Types<1, 1, 1, 0>, kCut, true>(p, blocks, bytes, s);
        }
    switch (2 * x + y) {
        case 0: return go<C, kMost, Types<0, 0, 0, 0>, kCut, kSecond>(p, blocks, bytes, s);
        case 1: return go<C, kMost, Types<0, 1, 0, 0>, kCut, kSecond>(p, blocks, bytes, s);
        case 2: return go<C, kMost, Types<1, 0, 0, 0>, kCut, kSecond>(p, blocks, bytes, s);
        default: return go<C, kMost, Types<1, 1, 0, 0>, kCut, kSecond>(p, blocks, bytes, s);
    }
}

// Sequences that lie apart, `times` eights of columns a thread; blocks of 8 warps with two and with four; calls without dh
// (files of their own for the compiler's time).
cudaError_t residual_bwd_cut(const Args &p, int times, int blocks, int bytes, cudaStream_t s);
cudaError_t residual_bwd_16_cut(const Args &p, int blocks, int bytes, cudaStream_t s);
cudaError_t residual_bwd_16(const Args &p, int blocks, int bytes, cudaStream_t s);
cudaError_t residual_bwd_32(const Args &p, int blocks, int bytes, cudaStream_t s);
cudaError_t residual_bwd_alone(const Args &p, int times, int blocks, int bytes, cudaStream_t s);
cudaError_t residual_bwd_alone_cut(const Args &p, int times, int blocks, int bytes, cudaStream_t s);

// The kernel for a call: of its types, where its places, strides and types have one.
template <int C, int kMost, bool kSecond>
cudaError_t go_by_places(const Args &p, int blocks, int bytes, cudaStream_t s) {
    const Residual &r = p.r;
    const int st = r.storage_wide;
    if (!fast(p) || (st && !(r.x.wide && r.y.wide && r.dh.wide)) || (!p.held && !(C == 4 && st)))
        return go<C, kMost, Types<-1, -1, -1, -1>, false, kSecond>(p, blocks, bytes, s);
    if (p.flat) return go_by_types<C, kMost, false, kSecond>(p, blocks, bytes, s);
    return kSecond ? residual_bwd_cut(p, C, blocks, bytes, s) : residual_bwd_alone_cut(p, C, blocks, bytes, s);
}

}  // namespace blk
}  // namespace mosa
