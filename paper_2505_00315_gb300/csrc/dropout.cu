// Dropout without a stored mask: y = keep/(1-p) x, the words of a token's columns from their counters
// (philox.cuh).  Memory bound: x and y move once; two counters for eight columns are some ten
// instructions a value.
#include <algorithm>

#include "block.h"
#include "launch.h"
#include "profile.h"

namespace mosa {
namespace blk {
namespace {

constexpr int kThreads = 256, kTimes = 4;   // eights of columns that a lane has under way

struct Args {
    int B, T, d;
    Rows x, y;
    Drop drop;
    int lanes;          // of a row: a power of two, 32 where a row has 256 columns or more
    long long units;    // of a warp: kTimes times 32 / lanes rows, or kTimes * 256 columns of one row
    int row_units;      // units of one row (lanes = 32)
};

struct Eight {
    uint4 a, b;   // bf16: a alone
};

__device__ __forceinline__ void load8(const Rows &m, const char *row, int col, int n, Eight &v) {
    if (m.vec && n >= 8) {
        const uint4 *p = reinterpret_cast<const uint4 *>(row + (long long)col * (m.wide ? 4 : 2));
        v.a = p[0];
        if (m.wide) v.b = p[1];
        return;
    }
    uint32_t w[8];
    if (m.wide) {
#pragma unroll
        for (int e = 0; e < 8; ++e) w[e] = e < n ? reinterpret_cast<const uint32_t *>(row)[col + e] : 0u;
        v.b = make_uint4(w[4], w[5], w[6], w[7]);
    } else {
        const unsigned short *p = reinterpret_cast<const unsigned short *>(row) + col;
#pragma unroll
        for (int e = 0; e < 4; ++e)
            w[e] = (2 * e < n ? (uint32_t)p[2 * e] : 0u) | (2 * e + 1 < n ? (uint32_t)p[2 * e + 1] << 16 : 0u);
    }
    v.a = make_uint4(w[0], w[1], w[2], w[3]);
}

// Zero bits where a value is dropped, else the value times `scale`.
__device__ __forceinline__ uint32_t narrow2(uint32_t w, uint32_t bits, float scale) {
    const float lo = bits & 1 ? __uint_as_float(w << 16) * scale : 0.f;
    const float hi = bits & 2 ? __uint_as_float(w & 0xFFFF0000u) * scale : 0.f;
    uint32_t r;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}
__device__ __forceinline__ uint32_t wide1(uint32_t w, uint32_t bit, float scale) {
    return bit ? __float_as_uint(__uint_as_float(w) * scale) : 0u;
}

__global__ void __launch_bounds__(kThreads) dropout_kernel(const __grid_constant__ Args p) {
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const DropKey key = drop_key(p.drop);
    const int lane = threadIdx.x & 31, per = 32 / p.lanes;
    const long long rows = (long long)p.B * p.T, warps = (long long)gridDim.x * (kThreads / 32);
    for (long long u = (long long)blockIdx.x * (kThreads / 32) + (threadIdx.x >> 5); u < p.units; u += warps) {
        const long long u_row = p.lanes == 32 ? u / p.row_units : 0;
        long long row[kTimes];
        int col[kTimes], n[kTimes];
        Eight v[kTimes];
#pragma unroll
        for (int i = 0; i < kTimes; ++i) {
            if (p.lanes == 32) {
                const long long at = ((u - u_row * p.row_units) * kTimes + i) * 256 + 8 * lane;
                row[i] = u_row;
                col[i] = (int)min(at, (long long)p.d);
            } else {
                row[i] = (u * kTimes + i) * per + lane / p.lanes;
                col[i] = 8 * (lane % p.lanes);
            }
            n[i] = row[i] < rows ? p.d - col[i] : 0;
            if (n[i] <= 0) continue;
            const int b = (uint32_t)row[i] / (uint32_t)p.T, t = (int)((uint32_t)row[i] - (uint32_t)b * (uint32_t)p.T);
            load8(p.x, p.x.at(b, t), col[i], n[i], v[i]);
        }
#pragma unroll
        for (int i = 0; i < kTimes; ++i) {
            if (n[i] <= 0) continue;
            const int b = (uint32_t)row[i] / (uint32_t)p.T, t = (int)((uint32_t)row[i] - (uint32_t)b * (uint32_t)p.T);
            char *out = p.y.at(b, t);
            const uint32_t bits = p.drop.rng != nullptr ? kept8(p.drop, key, (uint32_t)row[i], (uint32_t)(col[i] >> 3)) : 0xFFu;
            const float s = p.drop.scale;
            uint32_t w[8] = {v[i].a.x, v[i].a.y, v[i].a.z, v[i].a.w, v[i].b.x, v[i].b.y, v[i].b.z, v[i].b.w};
            if (p.y.wide) {
#pragma unroll
                for (int e = 0; e < 8; ++e) w[e] = wide1(w[e], bits >> e & 1, s);
            } else {
#pragma unroll
                for (int e = 0; e < 4; ++e) w[e] = narrow2(w[e], bits >> 2 * e, s);
            }
            if (p.y.vec && n[i] >= 8) {
                uint4 *q = reinterpret_cast<uint4 *>(out + (long long)col[i] * (p.y.wide ? 4 : 2));
                q[0] = make_uint4(w[0], w[1], w[2], w[3]);
                if (p.y.wide) q[1] = make_uint4(w[4], w[5], w[6], w[7]);
            } else if (p.y.wide) {
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    if (e < n[i]) reinterpret_cast<uint32_t *>(out)[col[i] + e] = w[e];
            } else {
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    if (e < n[i])
                        reinterpret_cast<unsigned short *>(out)[col[i] + e] = (unsigned short)(w[e / 2] >> 16 * (e & 1));
            }
        }
    }
}

}  // namespace

cudaError_t launch_dropout(int B, int T, int d, const Rows &x, const Rows &y, const Drop &drop,
                           cudaStream_t s) {
    Args p{B, T, d, x, y, drop, 1, 0, 1};
    while (p.lanes < 32 && p.lanes * 8 < d) p.lanes *= 2;
    const long long rows = (long long)B * T, per = 32 / p.lanes;
    if (p.lanes == 32) {
        p.row_units = (int)((d + kTimes * 256LL - 1) / (kTimes * 256));
        p.units = rows * p.row_units;
    } else {
        p.units = (rows + per * kTimes - 1) / (per * kTimes);
    }
    const int warps = kThreads / 32;
    const long long blocks = std::min<long long>((p.units + warps - 1) / warps, 152 * 8);
    cudaError_t e = launch_pdl(dropout_kernel, dim3((unsigned)blocks), dim3(kThreads), 0, s, p);
    note_launches(1);
    return e;
}

}  // namespace blk
}  // namespace mosa
