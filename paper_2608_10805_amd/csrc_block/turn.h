// Turning tiles between planes and rows.
//
// In planes a thread reads V adjacent pixels of a channel, in rows G = 16 bytes
// of adjacent channels of a pixel. A thread that holds V pixels of G channels
// can write or read either side in whole vectors; the two sides meet in LDS, in
// units of 16 bytes, pixel by pixel: unit u of pixel p lies at p * U + (u ^
// f(p)), U a multiple of 8, so that eight lanes side by side, of different
// pixels on the planes' side and of different units on the rows' side, touch
// all 32 banks.
#pragma once

#include "norm_device.h"

namespace wtc {

// TH threads: LP lanes of V pixels side by side, NS slots of K * G channels.
// WHOLE: C is a multiple of G.
template <typename T, int TH_, int V_, int LP_, int K_, bool WHOLE>
struct Tile {
    using Type = T;
    static constexpr int TH = TH_, V = V_, LP = LP_, K = K_, G = 16 / (int)sizeof(T);
    static constexpr bool kWhole = WHOLE;
    static constexpr int P = LP * V, NS = TH / LP, NW = TH / 64;
    static constexpr int kChannels = NS * G;       // channels of one step k
    static constexpr int kMaxC = kChannels * K;
    static_assert(NW * 64 == TH && NS * LP == TH && (LP & (LP - 1)) == 0 && (V & (V - 1)) == 0, "whole wavefronts");
};

#define ALWAYS __attribute__((always_inline))  // (of lambdas: their arrays stay in registers)

constexpr int kTurnBytes = 32 * 1024;  // LDS for it: leaves room for four workgroups a CU and more

template <typename Ti>
constexpr int turn_units(int steps) { return (steps * Ti::NS + 7) / 8 * 8; }

// Steps k that are turned at once.
template <typename Ti>
constexpr int turn_steps()
{
    int n = Ti::K;
    while (n > 1 && Ti::P * turn_units<Ti>(n) * 16 > kTurnBytes) --n;
    return n;
}

template <typename Ti>
struct Turn {
    using T = typename Ti::Type;
    static constexpr int kSteps = turn_steps<Ti>(), U = turn_units<Ti>(kSteps), kWidth = kSteps * Ti::kChannels;
    static constexpr int kSize = Ti::P * U;

    static DEV int at(int p, int u) { return p * U + turned(p / Ti::V, u); }
    // The place of unit u in every pixel of lane px.
    static DEV int turned(int px, int u)
    {
        constexpr int spread = Ti::LP >= 8 ? 1 : 8 / Ti::LP;
        return u ^ (px * spread & 7);
    }

    // The planes' side: unit u (channels (slot + k * NS) * G and on) of the V
    // pixels of lane px.
    static DEV void put(uint4* lds, int px, int u, const float (&f)[Ti::V][Ti::G])
    {
        uint4* first = lds + px * Ti::V * U + turned(px, u);
#pragma unroll
        for (int i = 0; i < Ti::V; ++i) {
            Pack<T, Ti::G> q;
#pragma unroll
            for (int g = 0; g < Ti::G; ++g) q.v[g] = from_f32<T>(f[i][g]);
            first[i * U] = __builtin_bit_cast(uint4, q);
        }
    }
    static DEV void get(const uint4* lds, int px, int u, float (&f)[Ti::V][Ti::G])
    {
        const uint4* first = lds + px * Ti::V * U + turned(px, u);
#pragma unroll
        for (int i = 0; i < Ti::V; ++i) {
            const auto q = __builtin_bit_cast(Pack<T, Ti::G>, first[i * U]);
#pragma unroll
            for (int g = 0; g < Ti::G; ++g) f[i][g] = to_f32(q.v[g]);
        }
    }

    // The rows' side: `rows` rows of `width` channels, `pitch` elements apart, to
    // or from memory. Whole units where they are aligned; else elements, two at
    // once where 16-bit rows follow each other without a gap.
    template <bool OUT>
    static DEV void copy(std::conditional_t<OUT, T, const T>* mem, int64_t pitch, uint4* lds, int rows, int width)
    {
        if (width % Ti::G == 0 && pitch % Ti::G == 0 && (uintptr_t)mem % 16 == 0) {
            using M = std::conditional_t<OUT, uint4, const uint4>;
            const int per = width / Ti::G, n = rows * per;
            const uint32_t magic = divider(per);
            const int dr = divide(Ti::TH, per, magic), du = Ti::TH - dr * per;
            int r = divide(threadIdx.x, per, magic), u = threadIdx.x - r * per;
            const bool dense = pitch == width;
#pragma unroll 4
            for (int i = threadIdx.x; i < n; i += Ti::TH) {
                M* m = dense ? reinterpret_cast<M*>(mem) + i : reinterpret_cast<M*>(mem + r * pitch) + u;
                if constexpr (OUT)
                    *m = lds[at(r, u)];
                else
                    lds[at(r, u)] = *m;
                r += dr;
                u += du;
                if (u >= per) {
                    u -= per;
                    ++r;
                }
            }
            return;
        }
        T* elements = reinterpret_cast<T*>(lds);
        auto element = [&](int r, int c) -> T& { return elements[at(r, c / Ti::G) * Ti::G + c % Ti::G]; };
        const uint32_t magic = divider(width);
        const int n = rows * width;
        if (sizeof(T) == 2 && (pitch == width || rows == 1) && (uintptr_t)mem % 4 == 0) {
            for (int i = threadIdx.x * 2; i < n; i += Ti::TH * 2) {
                const int r = divide(i, width, magic), c = i - r * width;
                const bool last = i + 1 == n;
                const int r2 = c + 1 == width ? r + 1 : r, c2 = c + 1 == width ? 0 : c + 1;
                if constexpr (OUT) {
                    const T v = element(r, c);
                    if (last)
                        mem[i] = v;
                    else
                        *reinterpret_cast<Pack<T, 2>*>(mem + i) = {{v, element(r2, c2)}};
                } else if (last) {
                    element(r, c) = mem[i];
                } else {
                    const auto q = *reinterpret_cast<const Pack<T, 2>*>(mem + i);
                    element(r, c) = q.v[0];
                    element(r2, c2) = q.v[1];
                }
            }
            return;
        }
        for (int i = threadIdx.x; i < n; i += Ti::TH) {
            const int r = divide(i, width, magic), c = i - r * width;
            if constexpr (OUT)
                mem[r * pitch + c] = element(r, c);
            else
                element(r, c) = mem[r * pitch + c];
        }
    }

    // i / per for i * per < 2^32, per > 0
    static DEV uint32_t divider(int per) { return 0xffffffffu / (uint32_t)per + 1u; }
    static DEV int divide(int i, int per, uint32_t magic) { return per == 1 ? i : (int)__umulhi((uint32_t)i, magic); }
};

// Where a thread's pixels and channels lie in planes: bytes from the first
// image of its tile on, as 32 bits from an address that is the same for the
// whole workgroup (the host checks that they suffice), so that the loads of all
// channels share one register of addresses.
struct Pixels {
    int64_t S;       // pixels of an image
    uint64_t magic;  // ceil(2^shift / S): q / S for q < 2^31
    int shift;
    int C;

    DEV uint32_t image(uint32_t q) const { return (uint32_t)((q * magic) >> shift); }
};

template <typename Ti>
bool pixels_fit(int64_t N, int64_t S, int C)
{
    return N < (int64_t)1 << 31 && ((int64_t)Ti::P + 2 * S) * C + (int64_t)Ti::kChannels * S <
                                       ((int64_t)1 << 32) / (int64_t)sizeof(typename Ti::Type);
}

inline Pixels pixels_of(int64_t S, int C)
{
    Pixels p;
    p.S = S;
    p.C = C;
    p.shift = 31;
    while (((int64_t)1 << (p.shift - 31)) < S && p.shift < 62) ++p.shift;
    p.magic = S > 0 ? (((uint64_t)1 << p.shift) + S - 1) / S : 0;
    return p;
}

template <typename Ti>
struct Place {
    int64_t base;   // first element of the tile's first image, the same for all threads
    uint32_t bytes; // from there to channel slot * G of this thread's first pixel

    DEV Place(const Pixels& p, uint32_t q0, uint32_t q, int slot)
    {
        using T = typename Ti::Type;
        const uint32_t b0 = p.image(q0), b = p.image(q);
        base = (int64_t)b0 * p.C * p.S;
        bytes = ((b - b0) * (uint32_t)p.C * (uint32_t)p.S + (q - b * (uint32_t)p.S) +
                 (uint32_t)slot * Ti::G * (uint32_t)p.S) * (uint32_t)sizeof(T);
    }
    // The thread's pixels in channel (k * NS + slot) * G + g.
    template <typename U>
    DEV U* at(U* p, int64_t S, int k, int g) const
    {
        using B = std::conditional_t<std::is_const_v<U>, const char, char>;
        B* first = reinterpret_cast<B*>(p + base + (k * Ti::kChannels + g) * S);
        return reinterpret_cast<U*>(first + bytes);
    }
};

// Calls f(g) for each of the thread's channels of a step that there are, `left`
// of them from its first on. Where C is a multiple of G a unit is whole or not
// there, and one test is enough.
template <typename Ti, typename F>
DEV void over_channels(int left, F&& f)
{
    if constexpr (Ti::kWhole) {
        if (left > 0) {
#pragma unroll
            for (int g = 0; g < Ti::G; ++g) f(g);
        }
    } else {
#pragma unroll
        for (int g = 0; g < Ti::G; ++g)
            if (g < left) f(g);
    }
}

// The thread's V pixels of its G channels of step k; what is past C is not
// written.
template <typename Ti, typename T = typename Ti::Type>
DEV void load_pixels(const T* p, const Place<Ti>& at, const Pixels& px, int left, int k, float (&f)[Ti::V][Ti::G])
{
    over_channels<Ti>(left, [&](int g) ALWAYS {
        float v[Ti::V];
        load_pack<Ti::V>(at.at(p, px.S, k, g), v);
#pragma unroll
        for (int i = 0; i < Ti::V; ++i) f[i][g] = v[i];
    });
}

template <typename Ti, typename T = typename Ti::Type>
DEV void store_pixels(T* p, const Place<Ti>& at, const Pixels& px, int left, int k, const float (&f)[Ti::V][Ti::G])
{
    over_channels<Ti>(left, [&](int g) ALWAYS {
        float v[Ti::V];
#pragma unroll
        for (int i = 0; i < Ti::V; ++i) v[i] = f[i][g];
        store_pack<Ti::V>(at.at(p, px.S, k, g), v);
    });
}

}  // namespace wtc
