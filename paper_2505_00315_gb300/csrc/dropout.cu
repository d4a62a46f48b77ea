// Dropout without a stored mask: y = keep/(1-p) x, the words of a token's columns from their counters
// (philox.cuh).  Memory bound in fp32: x and y move once; two counters for eight columns are some ten
// instructions of 25 a value (bf16 23).  A warp takes a few runs of 256 columns (or of some whole rows, where those are
// short), one after another in memory, all loads first.  fp32 B4 T4096 d1024 22.3 us (6.0 TB/s, 89% of the copy rate;
// runs of whole units of 1024 columns a warp 29.7); B8 T1024 d512 bf16 6.8 (10.8), one wave.
// bf16 B4 T4096 d1024 18.0, 55% of the copy rate: as many instructions for half the bytes, with 59% of the issue slots busy.
// Rows that are not whole pieces go value by value: 16384 of 1001 fp32 49, bf16 43.
#include <algorithm>

#include "block.h"
#include "launch.h"
#include "pairs.cuh"
#include "profile.h"

namespace mosa {
namespace blk {
namespace {

constexpr int kThreads = 256, kSms = 152;
constexpr int times_of(bool wide) { return wide ? 2 : 4; }   // runs that a warp has under way: 64 bytes a lane

struct Args {
    int T, d;
    uint32_t rows;
    Rows x, y;
    Drop drop;
    int flat;           // rows lie one stride apart, sequences too
    int lanes;          // of a row: a power of two, 32 where a row has more than 128 columns
    uint32_t runs, per_row;   // runs in all, and of one row
};

// Eight columns: bf16 in the first four words, fp32.
template <bool kWide>
struct Eight {
    uint32_t w[kWide ? 8 : 4];
};

// n: how many of the eight columns there are.
template <bool kWide>
__device__ __forceinline__ void load8(const char *p, bool vec, int n, Eight<kWide> &v) {
    if (vec && n >= 8) {
#pragma unroll
        for (int i = 0; i < (kWide ? 2 : 1); ++i) {
            const uint4 a = reinterpret_cast<const uint4 *>(p)[i];
            v.w[4 * i] = a.x; v.w[4 * i + 1] = a.y; v.w[4 * i + 2] = a.z; v.w[4 * i + 3] = a.w;
        }
        return;
    }
#pragma unroll
    for (int e = 0; e < (kWide ? 8 : 4); ++e) {
        if (kWide) {
            v.w[e] = e < n ? reinterpret_cast<const uint32_t *>(p)[e] : 0u;
        } else {
            const unsigned short *q = reinterpret_cast<const unsigned short *>(p);
            v.w[e] = (2 * e < n ? (uint32_t)q[2 * e] : 0u) | (2 * e + 1 < n ? (uint32_t)q[2 * e + 1] << 16 : 0u);
        }
    }
}
template <bool kWide>
__device__ __forceinline__ void store8(char *p, bool vec, int n, const Eight<kWide> &v) {
    if (vec && n >= 8) {
#pragma unroll
        for (int i = 0; i < (kWide ? 2 : 1); ++i)
            reinterpret_cast<uint4 *>(p)[i] = make_uint4(v.w[4 * i], v.w[4 * i + 1], v.w[4 * i + 2], v.w[4 * i + 3]);
        return;
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        if (e >= n) continue;
        if (kWide) reinterpret_cast<uint32_t *>(p)[e] = v.w[kWide ? e : 0];
        else reinterpret_cast<unsigned short *>(p)[e] = (unsigned short)(v.w[e / 2] >> 16 * (e & 1));
    }
}

template <bool kWide>
__global__ void __launch_bounds__(kThreads, 4) dropout_kernel(const __grid_constant__ Args p) {
    asm volatile("griddepcontrol.wait;" ::: "memory");
    constexpr int kTimes = times_of(kWide), kSize = kWide ? 4 : 2;
    const DropKey key = drop_key(p.drop);
    const uint32_t lane = threadIdx.x & 31, per = 32 / p.lanes, step = gridDim.x * (kThreads / 32) * kTimes;
    for (uint32_t run = (blockIdx.x * (kThreads / 32) + (threadIdx.x >> 5)) * kTimes; run < p.runs; run += step) {
        uint32_t row[kTimes], col[kTimes];
        int n[kTimes];
        Eight<kWide> v[kTimes];
        uint32_t r = run / p.per_row, part = run - r * p.per_row;
#pragma unroll
        for (int i = 0; i < kTimes; ++i) {
            row[i] = per == 1 ? r : r * per + lane / p.lanes;
            col[i] = per == 1 ? part * 256 + 8 * lane : 8 * (lane & (p.lanes - 1));
            n[i] = run + i < p.runs && row[i] < p.rows ? p.d - (int)col[i] : 0;
            if (++part == p.per_row) {
                part = 0;
                ++r;
            }
            if (n[i] <= 0) continue;
            const uint32_t b = p.flat ? 0 : row[i] / (uint32_t)p.T, t = p.flat ? row[i] : row[i] - b * (uint32_t)p.T;
            load8<kWide>(p.x.p + (long long)b * p.x.b + (long long)t * p.x.t + (long long)col[i] * kSize, p.x.vec, n[i], v[i]);
        }
#pragma unroll
        for (int i = 0; i < kTimes; ++i) {
            if (n[i] <= 0) continue;
            const uint32_t bits = p.drop.rng != nullptr ? kept8(p.drop, key, row[i], col[i] >> 3) : 0xFFu;
            const float s = p.drop.scale;
#pragma unroll
            for (int e = 0; e < (kWide ? 8 : 4); ++e) {   // (a dropped value is chosen away, whatever it holds)
                if (kWide) {
                    v[i].w[e] = bits >> e & 1 ? __float_as_uint(__uint_as_float(v[i].w[e]) * s) : 0u;
                } else {
                    v[i].w[e] = pack2(bits >> 2 * e & 1 ? low(v[i].w[e]) * s : 0.f,
                                      bits >> (2 * e + 1) & 1 ? high(v[i].w[e]) * s : 0.f);
                }
            }
            const uint32_t b = p.flat ? 0 : row[i] / (uint32_t)p.T, t = p.flat ? row[i] : row[i] - b * (uint32_t)p.T;
            store8<kWide>(p.y.p + (long long)b * p.y.b + (long long)t * p.y.t + (long long)col[i] * kSize, p.y.vec, n[i], v[i]);
        }
    }
}

}  // namespace

cudaError_t launch_dropout(int B, int T, int d, const Rows &x, const Rows &y, const Drop &drop,
                           cudaStream_t s) {
    const long long rows = (long long)B * T;
    Args p{T, d, (uint32_t)rows, x, y, drop, 0, 1, 0, 1};
    if (T == 1) {   // (rows are the sequences)
        p.x.t = x.b;
        p.y.t = y.b;
        p.flat = 1;
    } else {
        p.flat = B == 1 || (x.b == x.t * T && y.b == y.t * T);
    }
    while (p.lanes < 32 && p.lanes * 8 < d) p.lanes *= 2;
    const long long per = 32 / p.lanes, per_row = per == 1 ? (d + 255LL) / 256 : 1, runs = (rows + per - 1) / per * per_row;
    p.runs = (uint32_t)runs;
    p.per_row = (uint32_t)per_row;
    const long long each = kThreads / 32 * times_of(x.wide), blocks = std::min<long long>((runs + each - 1) / each, kSms * 8);
    note_launches(1);
    return x.wide ? launch_pdl(dropout_kernel<true>, dim3((unsigned)blocks), dim3(kThreads), 0, s, p)
                  : launch_pdl(dropout_kernel<false>, dim3((unsigned)blocks), dim3(kThreads), 0, s, p);
}

}  // namespace blk
}  // namespace mosa
