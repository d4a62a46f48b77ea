// Which queries the CTAs of dk and dv take (window_tiles.cuh), on the host: every visible pair of a query and
// a key once, no sum of positions past 32 bits, sink rows' far queries spread out and their sums in 64 MB.  Prints the first mistake and returns 1.
#include <algorithm>
#include <cstdio>
#include <cstdlib>
#include <vector>

#include "window_tiles.cuh"

using namespace mosa::win;

static Attn shape(int Tq, int Tk, int window, int sinks) {
    Attn a{};
    a.B = a.H = a.Hkv = 1;
    a.hp = 16;
    a.Tq = Tq;
    a.Tk = Tk;
    a.window = window == 0 || window > Tk ? Tk : window;
    a.sinks = sinks < Tk ? sinks : Tk;
    return a;
}

// Small shapes, pair by pair.
template <int N>
static bool pairs(const Attn &a, int len) {
    const SinkSplit sp(a, N);
    std::vector<int> count((size_t)a.Tk * a.Tk, 0);
    for (int x = 0; x < sp.ctas(a, N); ++x) {
        const KeyTile<N> t(x, a, sp, len);
        for (int p = t.first; p <= t.last; ++p)
            for (int k = t.k0; k < t.k0 + N && k < a.Tk; ++k)
                if (k <= p && (p - k < a.window || k < a.sinks)) ++count[(size_t)p * a.Tk + k];
    }
    for (int p = 0; p < a.Tk; ++p)
        for (int k = 0; k < a.Tk; ++k) {
            const bool sees = p >= a.Tk - a.Tq && p < len && k <= p && (p - k < a.window || k < a.sinks);
            if (count[(size_t)p * a.Tk + k] != sees) {
                printf("N %d Tq %d Tk %d window %d sinks %d len %d: query %d key %d taken %d times\n", N, a.Tq, a.Tk,
                       a.window, a.sinks, len, p, k, count[(size_t)p * a.Tk + k]);
                return false;
            }
        }
    return true;
}

// Large shapes: where a tile's queries begin and end, in 64 bits.
template <int N>
static bool ends(const Attn &a, int len) {
    const SinkSplit sp(a, N);
    const long long off = (long long)a.Tk - a.Tq;
    const int ctas = sp.ctas(a, N);
    for (int i = 0; i < 300; ++i) {
        const int x = i < 100 ? i : i < 200 ? ctas - 1 - (i - 100) : (int)((long long)rand() * 31 % ctas);
        if (x < 0 || x >= ctas) continue;
        const KeyTile<N> t(x, a, sp, len);
        const long long k0 = t.k0, beyond = k0 + N - 1 + a.window;
        long long first = std::max<long long>(k0, off), last = std::min<long long>(beyond, len) - 1;
        if (t.part == 0 && k0 < a.sinks && sp.extra == 0) last = len - 1;
        if (t.part > 0) {
            first = std::max(beyond, off) + (t.part - 1LL) * sp.chunk * N;
            last = std::min<long long>(first + (long long)sp.chunk * N, len) - 1;
        }
        const bool any = first <= last;
        if (any != (t.first <= t.last) || (any && (t.first != first || t.last != last))) {
            printf("N %d Tq %d Tk %d window %d sinks %d len %d CTA %d: queries %d .. %d for %lld .. %lld\n", N, a.Tq,
                   a.Tk, a.window, a.sinks, len, x, t.first, t.last, first, last);
            return false;
        }
    }
    return true;
}

// The sums' room, and that a few sink tiles' far queries do not all fall to the CTAs of those tiles.
template <int N>
static bool split(int B, int Tk, int Hkv, int hp, int window, int sinks) {
    Attn a = shape(Tk, Tk, window, sinks);
    a.B = B;
    a.H = a.Hkv = Hkv;
    a.hp = hp;
    const SinkSplit sp(a, N);
    const long long tiles = (a.sinks + N - 1LL) / N * Hkv * B, blocks = (Tk + N - 1LL) / N;
    long long most = 0;   // blocks of queries that a CTA meets
    for (int x = 0; x < sp.ctas(a, N); ++x) {
        const KeyTile<N> t(x, a, sp, Tk);
        if (t.first <= t.last) most = std::max(most, (t.last - t.first) / N + 1LL);
    }
    const bool fair = tiles >= 152 || most <= std::max({(window + N - 1LL) / N + 2, (blocks + 63) / 64 + 1,
                                                       (blocks * SinkSplit::sum_bytes(a) + (1 << 25)) / (1 << 25)});
    if (sp.bytes(a) > 64 << 20 || !fair) {
        printf("N %d B %d Tk %d heads %d of %d window %d sinks %d: %zu bytes, up to %lld of %lld blocks a CTA\n", N, B,
               Tk, Hkv, hp, window, sinks, sp.bytes(a), most, blocks);
        return false;
    }
    return true;
}

int main() {
    srand(1);
    for (int n = 0; n < 400; ++n) {
        const int Tk = 1 + rand() % 700, Tq = rand() % 2 ? Tk : 1 + rand() % Tk;
        const Attn a = shape(Tq, Tk, rand() % 3 == 0 ? rand() % 8 : rand() % (Tk + 1), rand() % 3 ? rand() % 9 : rand() % 300);
        const int len = rand() % 2 ? Tk : rand() % (Tk + 1);
        if (!pairs<64>(a, len) || !pairs<128>(a, len)) return 1;
    }
    for (int B : {1, 2, 8, 64})
        for (int Hkv : {1, 4, 8, 32})
            for (int hp : {16, 64, 128})
                for (int sinks : {1, 4, 130, 512, 513, 2000})
                    for (int window : {1, 64, 512})
                        for (int Tk : {1000, 16384})
                            if (!split<64>(B, Tk, Hkv, hp, window, sinks) || !split<128>(B, Tk, Hkv, hp, window, sinks))
                                return 1;
    const int most = (1 << 30) - 1;   // the most tokens that a call takes
    for (int Tk : {most, most - 1, most - 62, most - 2000, 1 << 29})
        for (int Tq : {1, 1000, Tk})
            for (int window : {0, 1, 2, 1000, Tk / 2, Tk - 1})
                for (int sinks : {0, 1, 512, 513})
                    for (int len : {Tk, Tk - 1, Tk / 2}) {
                        const Attn a = shape(Tq, Tk, window, sinks);
                        if (!ends<64>(a, len) || !ends<128>(a, len)) return 1;
                    }
    printf("ok\n");
    return 0;
}
