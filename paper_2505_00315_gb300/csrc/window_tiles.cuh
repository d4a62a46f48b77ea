// Window heads: which keys a tile of queries meets, and which queries a tile of
// keys, shared by the CUDA-core and the tensor-core kernels.
//
// Query positions p (of the Tk tokens) see tokens t <= p with p - t < window or
// t < sinks, both below the sequence's length.
#pragma once

#include <algorithm>

#include "window.h"

namespace mosa {
namespace win {

__device__ __forceinline__ int seq_len(const int32_t *lens, int b, int Tk) {
    return lens == nullptr ? Tk : min(max(lens[b], 0), Tk);
}

// Key blocks of NK tokens for the queries at positions pf .. pl (pf <= pl < len), in the
// order of their tokens: blocks 0 .. far-1 hold the sinks below the window, from token 0 up,
// the others lead up to the last query's own position, the end of the last block, so
// that window + tile tokens take as few blocks as can be wherever the tile starts.
// Sinks come first because weight often lies on them: a softmax whose running
// maximum starts there seldom has to be rescaled, and their weights are powers of two then,
// which a rounding to bf16 leaves as they are.
template <int NK>
struct KeyBlocks {
    int top, near, far, slim;   // slim: sinks [0, slim) are left to the far blocks
    __device__ __forceinline__ KeyBlocks(int pf, int pl, int window, int sinks) {
        const int lo = pf >= window ? pf - window + 1 : 0;
        top = pl + 1;
        near = (top - lo + NK - 1) / NK;
        slim = min(sinks, max(top - NK * near, 0));
        far = (slim + NK - 1) / NK;
    }
    __device__ __forceinline__ int count() const { return near + far; }
    __device__ __forceinline__ bool is_far(int j) const { return j < far; }
    __device__ __forceinline__ int start(int j) const {
        return is_far(j) ? NK * j : top - NK * (far + near - j);
    }
    // Every query pf .. pl sees every key of block j.
    __device__ __forceinline__ bool whole(int j, int pf, int pl, int window) const {
        const int ks = start(j);
        if (is_far(j)) return ks + NK <= slim;
        return ks >= 0 && ks + NK - 1 <= pf && pl - ks < window;
    }
    // Whether position p (in pf .. pl) sees column c of block j, which starts at ks.
    __device__ __forceinline__ bool sees(int j, int ks, int c, int p, int window, int sinks) const {
        const int t = ks + c;
        if (is_far(j)) return t < slim;
        return t >= 0 && t <= p && (p - t < window || t < sinks);
    }
};

// A CTA's tile, head and sequence.  Tiles count slowest, so that those with less to do, which are
// the last of every head, are the last of all: no heavy one is left to start when
// the others end, and CTAs that run together work on the same part of all the texts.
struct Place {
    int tile, h, b;
    __device__ __forceinline__ Place(uint32_t x, int H, int B) {
        const uint32_t all = (uint32_t)H * (uint32_t)B, t = x / all, rest = x - t * all;
        tile = (int)t;
        b = (int)(rest / (uint32_t)H);
        h = (int)rest - b * H;
    }
};

inline dim3 grid_of(int tiles, int H, int B) { return dim3((unsigned)((long long)tiles * H * B)); }

// dk and dv are summed by one CTA per key tile, over the queries that see it: window + tile of them,
// but for sinks all later ones, Tk / window times as many.  Those beyond a sink tile's window go
// to `extra` CTAs of their own, `chunk` tiles of queries each (as many as other tiles have, and more
// where that would take over kMostExtra CTAs, or over kMostBytes for their sums), which leave fp32 sums of the
// sink rows; add_sink_rows adds them up in order.  Where the sink tiles of all heads and sequences are as
// many as SMs they fill the GPU by themselves and nothing is split (so kMostBytes has room for three sums
// at least).  Backward, us, split / not: B1 T16384, 8 heads on 1 of 64, window 512, 513 sinks (5 tiles) 202 / 1437;
// B8 T4096, 8 heads of 64, window 256, 512 sinks (256 tiles) 400 / 279; B8 T4096, 32 heads of 64,
// window 512, 4 sinks (256 tiles) 1011 / 970; B16 T4096, 16 heads of 64, window 256, 1 sink (256 tiles) 842 / 870.
struct SinkSplit {
    static constexpr int kMostExtra = 64;
    static constexpr long long kMostBytes = 64 << 20;
    int extra = 0, chunk = 1;
    SinkSplit() = default;
    SinkSplit(const Attn &a, int tile) {
        const long long beyond = ((long long)a.Tk - (tile - 1 + (long long)a.window) + tile - 1) / tile;   // tiles
        const long long tiles = (long long)((a.sinks + tile - 1) / tile) * a.Hkv * a.B;
        if (tiles == 0 || tiles >= 152 || beyond <= 0) return;
        const long long most = std::min<long long>(kMostExtra, kMostBytes / sum_bytes(a) - 1);
        chunk = std::max((a.window + tile - 2) / tile + 1, (int)((beyond + most - 1) / most));
        extra = (int)((beyond + chunk - 1) / chunk);
    }
    __host__ __device__ int extras(const Attn &a, int tile) const { return (a.sinks + tile - 1) / tile * extra; }
    // CTAs of one key head of one sequence: the extra ones first.
    int ctas(const Attn &a, int tile) const { return extras(a, tile) + (a.Tk + tile - 1) / tile; }
    // Of one sum of all sink rows' dk and dv, and of all of them.
    static long long sum_bytes(const Attn &a) { return (long long)a.B * a.Hkv * a.sinks * 2 * a.hp * (long long)sizeof(float); }
    size_t bytes(const Attn &a) const { return extra == 0 ? 0 : (size_t)(extra + 1) * sum_bytes(a); }
};

// One of those CTAs: its key tile from k0 on and its query positions first .. last.
template <int N>
struct KeyTile {
    int k0, part, first, last, extra;
    bool has_sinks;   // rows below the number of sinks go to the partial sums
    __host__ __device__ __forceinline__ KeyTile(int x, const Attn &a, const SinkSplit &sp, int len) {
        const int extras = sp.extras(a, N), off = a.Tk - a.Tq;
        extra = sp.extra;
        part = x < extras ? 1 + x % extra : 0;
        k0 = (x < extras ? x / extra : x - extras) * N;
        has_sinks = k0 < a.sinks && extra > 0;
        if (part == 0) {
            first = max(k0, off);
            last = k0 < a.sinks && extra == 0 ? len - 1 : min(k0 + N - 1 + a.window - 1, len - 1);
        } else {
            first = max(k0 + N - 1 + a.window, off) + (part - 1) * sp.chunk * N;
            last = min(first + sp.chunk * N, len) - 1;
        }
    }
    // Where this CTA's sums start in the partial sums [B, Hkv, extra + 1, sinks, 2, hp].
    __device__ __forceinline__ long long partial_at(int b, int hk, const Attn &a) const {
        return (((long long)b * a.Hkv + hk) * (extra + 1) + part) * a.sinks * 2 * a.hp;
    }
};

// A query that sees one token only has P = 1: its scores have no gradient.  Set to
// exactly zero there, where rounding would leave a remainder of dP - D.
__device__ __forceinline__ bool sees_one(int p, int window, int sinks) {
    return p == 0 || (window == 1 && sinks == 0);
}

}  // namespace win
}  // namespace mosa
