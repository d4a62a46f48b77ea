// The residual step between two blocks, one pass over its tensors: for each token
//     n = r_y y gamma_post,  u = keep/(1-p) g n,  x' = x + scale u,  h = r_x x' gamma_pre
// with r = 1/sqrt(mean of squares + eps).  Layout and tools: residual.cuh.
// Memory bound: x, y (and a gate per token) come in, x' and h go out, once; a row's squares are summed twice, of y and of
// x', which is the chain of a row.  us and share of the copy rate: B4 T4096 d1024 with fp32 y 28.7 (86%), with dropout 30
// (83%: the random words are 11 of its 29 instructions a value); B2 T8192 d4096, fp32 stream, gate per token, dropout 151
// (91%); eight tokens of 1024: 2.9.
#include "residual.cuh"

namespace mosa {
namespace blk {
namespace {

template <int C, class Ty>
__global__ void __launch_bounds__(kThreads, 1) residual_kernel(const __grid_constant__ Args p) {
    asm volatile("griddepcontrol.wait;" ::: "memory");
    constexpr bool kFast = Ty::kFast, kCounts = kFast && C > 2;
    extern __shared__ __align__(16) char smem[];
    const Residual &r = p.r;
    const Place l(p, smem, C);
    const DropKey key = drop_key(r.drop);
    const bool drops = r.drop.rng != nullptr, token = r.gate == MOSA_GATE_TOKEN;
    const float unit = r.scale * (drops ? r.drop.scale : 1.f), inv_d = 1.f / l.d;
    if (l.d < 256 * C * l.W) clear_ring(l);
    uint32_t row = blockIdx.x * p.groups + l.group;   // (row + kMaxStages step fits 32 bits)
    Arrival<C, kFast, Ty::x, kCounts> x_in;
    Arrival<C, kFast, Ty::y, kCounts> y_in;
    Arrival<C, kFast, Ty::storage, kCounts> g_in;
    x_in.init(p, l, r.x, row);
    y_in.init(p, l, r.y, row);
    g_in.init(p, l, r.g, row);
    Departure<C, kFast, Ty::x, false, kCounts> x_out;
    Departure<C, kFast, Ty::storage, false, kCounts> h_out;
    x_out.init(p, l, r.xo, row);
    h_out.init(p, l, r.h, row);
    // Where the tensors' columns lie in a stage.
    const int y_off = kFast ? bytes_of(Ty::x, C) : p.off[1], g_off = kFast ? y_off + bytes_of(Ty::y, C) : p.off[4];
    auto fill = [&](uint32_t at, int slot) {
        const uint32_t to = l.ring32 + slot * p.stage_bytes;
        x_in.issue(p, l, r.x, at, to);
        y_in.issue(p, l, r.y, at, to + y_off);
        if (token) g_in.issue(p, l, r.g, at, to + g_off);
    };
    auto jump = [&](uint32_t at) {   // (after fill)
        const int ends = ends_between(p, l, at);
        x_in.jump(r.x, ends);
        y_in.jump(r.y, ends);
        g_in.jump(r.g, ends);
    };
    const int ahead = p.stages - 1;
    for (int i = 0; i < ahead; ++i) {
        if (row + i * l.step < l.rows) fill(row + i * l.step, i);
        if (kFast && !kCounts && !p.flat) jump(row + i * l.step);
        copies_end();
    }
    if (Ty::kHeld || (!Ty::kLies && p.held)) hold<C, true>(p, l, unit);

    int slot = 0, turn = 0;
    for (; row < l.rows; row += l.step) {
        __syncwarp();   // (the slot that is filled next has been read by all lanes)
        if (row + ahead * l.step < l.rows) fill(row + ahead * l.step, slot == 0 ? ahead : slot - 1);
        copies_end();
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
        const int xw = wide_of(Ty::x, r.x), yw = wide_of(Ty::y, r.y);
        const int xs = x_in.shift(p, l, r.x, row), ys = y_in.shift(p, l, r.y, row), gs = token ? g_in.shift(p, l, r.g, row) : -1;
        auto y_at = [&](int c) { return arrived<kFast>(in + y_off, yw, l, c, ys); };
        float ry = 1.f, rx = 1.f;
        if (r.post) {
            Pair s = 0;
#pragma unroll
            for (int c = 0; c < C; ++c) {
                const Oct y = y_at(c);
                add_products(s, y, y);
            }
            ry = rsqrtf(fmaf(row_sum(sum_of(s), l.red + turn * l.W, l.W, l.w, l.lane, l.group), inv_d, r.eps));
            turn ^= 1;
        }
        Oct x[C];
        Pair s = 0;
        if (token || drops) {
#pragma unroll
            for (int c = 0; c < C; ++c) {
                Oct u = times(y_at(c), times(vector_at<C, true, Ty>(p, l, 0, c, unit), ry));
                if (token) {
                    const int gw = wide_of(Ty::storage, r.g);
                    const Oct g = arrived<kFast>(in + g_off, gw, l, c, gs);
                    u = times(u, r.sigmoid ? logistic(g) : g);
                }
                x[c] = plus(arrived<kFast>(in, xw, l, c, xs), chosen(u, bits[c]));
                add_products(s, x[c], x[c]);
            }
        } else {
#pragma unroll
            for (int c = 0; c < C; ++c) {
                x[c] = fused(y_at(c), times(vector_at<C, true, Ty>(p, l, 0, c, unit), ry),
                             arrived<kFast>(in, xw, l, c, xs));
                add_products(s, x[c], x[c]);
            }
        }
        x_out.begin(p, r.xo, row);
#pragma unroll
        for (int c = 0; c < C; ++c) x_out.put_row(l, r.xo, c, x[c]);
        x_out.end(l, r.xo);
        if (r.pre) {
            rx = rsqrtf(fmaf(row_sum(sum_of(s), l.red + turn * l.W, l.W, l.w, l.lane, l.group), inv_d, r.eps));
            turn ^= 1;
            h_out.begin(p, r.h, row);
#pragma unroll
            for (int c = 0; c < C; ++c)
                h_out.put_row(l, r.h, c, times(x[c], times(vector_at<C, true, Ty>(p, l, 1, c, unit), rx)));
            h_out.end(l, r.h);
        }
        if (r.stats != nullptr && l.w == 0 && l.lane == 0) {
            r.stats[row] = ry;
            r.stats[(uint64_t)l.rows + row] = rx;
        }
        if (kFast && !kCounts && !p.flat) {
            jump(row + ahead * l.step);
            const int ends = ends_between(p, l, row);
            x_out.jump(r.xo, ends);
            h_out.jump(r.h, ends);
        }
    }
}

template <class Ty>
cudaError_t go(const Args &p, int blocks, int times, int bytes, cudaStream_t s) {
    const auto kernel = times == 1 ? residual_kernel<1, Ty> : times == 2 ? residual_kernel<2, Ty>
                        : times == 3 ? residual_kernel<3, Ty> : residual_kernel<4, Ty>;
    cudaError_t e = allow_smem((const void *)kernel, kSmem);
    if (e != cudaSuccess) return e;
    note_launches(1);
    return launch_pdl(kernel, dim3(blocks), dim3(p.warps * p.groups * 32), bytes, s, p);
}

}  // namespace

cudaError_t launch_residual(const Residual &r, cudaStream_t s) {
    Args p{};
    p.r = r;
    int blocks, times, bytes;
    shape(p, false, &blocks, &times, &bytes);
    if (fast(p) && p.held) {
        const int x = r.x.wide, y = r.y.wide, st = r.storage_wide;
        if (!st && !x && !y) return go<Types<0, 0, 0, 0>>(p, blocks, times, bytes, s);
        if (!st && !x && y) return go<Types<0, 1, 0, 0>>(p, blocks, times, bytes, s);
        if (!st && x && !y) return go<Types<1, 0, 0, 0>>(p, blocks, times, bytes, s);
        if (!st && x && y) return go<Types<1, 1, 0, 0>>(p, blocks, times, bytes, s);
        if (st && x && y) return go<Types<1, 1, 0, 1>>(p, blocks, times, bytes, s);
    }
    return go<Types<-1, -1, -1, -1>>(p, blocks, times, bytes, s);
}

}  // namespace blk
}  // namespace mosa
