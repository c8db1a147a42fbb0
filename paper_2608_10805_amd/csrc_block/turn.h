// Tiles of pixels and channels, turned between planes and rows.
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
// REGULAR: C is a multiple of G and S one of V, so that no unit and no vector is
// incomplete.
template <typename T, int TH_, int V_, int LP_, int K_, bool REGULAR>
struct Tile {
    using Type = T;
    static constexpr int TH = TH_, V = V_, LP = LP_, K = K_, G = 16 / (int)sizeof(T);
    static constexpr bool kRegular = REGULAR;
    // Tiles run over all images' pixels where no vector crosses from one image to
    // the next, else over each image's by itself.
    static constexpr bool kFlat = REGULAR || V == 1;
    static constexpr int P = LP * V, NS = TH / LP, NW = TH / 64;
    // Tiles side by side share lines of 128 bytes.
    static constexpr bool kShared = !REGULAR || P * sizeof(T) < 128;
    static constexpr int kChannels = NS * G;       // channels of one step k
    static constexpr int kMaxC = kChannels * K;
    static_assert(NW * 64 == TH && NS * LP == TH && (LP & (LP - 1)) == 0 && (V & (V - 1)) == 0, "whole wavefronts");
};

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

// i / per for i * per < 2^32, per > 0
struct Divider {
    int per;
    uint32_t magic;
    DEV explicit Divider(int n) : per(n), magic(0xffffffffu / (uint32_t)n + 1u) {}
    DEV int operator()(int i) const { return per == 1 ? i : (int)__umulhi((uint32_t)i, magic); }
};

template <typename Ti>
struct Turn {
    using T = typename Ti::Type;
    using Unit = Pack<T, Ti::G>;
    static constexpr int kSteps = turn_steps<Ti>(), U = turn_units<Ti>(kSteps), kWidth = kSteps * Ti::kChannels;
    static constexpr int kSize = Ti::P * U;

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
            Unit q;
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
            const auto q = __builtin_bit_cast(Unit, first[i * U]);
#pragma unroll
            for (int g = 0; g < Ti::G; ++g) f[i][g] = to_f32(q.v[g]);
        }
    }

    // The rows' side: `rows` rows of `width` channels, `pitch` elements apart, to
    // or from memory. What comes in is followed by rows of zeros up to P.
    template <bool OUT>
    static DEV void copy(std::conditional_t<OUT, T, const T>* mem, int64_t pitch, uint4* lds, int rows, int width)
    {
        const int per = (width + Ti::G - 1) / Ti::G, n = rows * per, tail = width - (per - 1) * Ti::G;
        const Divider over(per);
        const int dr = over(Ti::TH), du = Ti::TH - dr * per;
        int r = over(threadIdx.x), u = threadIdx.x - r * per;
        const bool dense = Ti::kRegular && pitch == width;
#pragma unroll 4
        for (int i = threadIdx.x; i < n; i += Ti::TH) {
            auto* m = dense ? mem + i * Ti::G : mem + r * pitch + u * Ti::G;
            uint4* t = lds + r * U + turned(r / Ti::V, u);
            const int count = Ti::kRegular || u + 1 < per ? Ti::G : tail;
            if constexpr (OUT)
                store_upto<Ti::G>(m, count, __builtin_bit_cast(Unit, *t));
            else
                *t = __builtin_bit_cast(uint4, load_upto<Ti::G>(m, count));
            r += dr;
            u += du;
            if (u >= per) {
                u -= per;
                ++r;
            }
        }
        if (!OUT && rows < Ti::P)
            for (int i = rows * U + threadIdx.x; i < Ti::P * U; i += Ti::TH) lds[i] = uint4{0, 0, 0, 0};
    }

    // The rows' side from memory without registers between: `rows` rows (up to P)
    // of `per` whole units, all addresses multiples of 16 bytes. What is not there
    // stays as it was. Lane l of a wavefront writes the l-th unit of 64 adjacent
    // ones, so that it is the lane that finds the unit that belongs there.
    static constexpr bool kDirect = Ti::kRegular && kSteps == Ti::K;
    static DEV void fetch(const T* mem, int64_t pitch, uint4* lds, uint32_t rows, int per)
    {
        static_assert(kSize % 64 == 0, "whole wavefronts");
        const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
#pragma unroll
        for (int n = 0; n < (kSize + Ti::TH - 1) / Ti::TH; ++n) {
            const int i0 = n * Ti::TH + w * 64;
            if (kSize % Ti::TH && i0 >= kSize) break;
            const int i = i0 + lane, r = i / U, u = turned(r / Ti::V, i % U);
            if ((uint32_t)r < rows && u < per)
                __builtin_amdgcn_global_load_lds((__attribute__((address_space(1))) void*)(mem + r * pitch + u * Ti::G),
                                                 (__attribute__((address_space(3))) void*)(lds + i0), 16, 0, 0);
        }
    }
    // Waits for this wavefront's part of it.
    static DEV void fetched() { asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); }
};

// The planes that tiles run over, and n / d for n < 2^31 as (n * magic) >> shift.
struct Pixels {
    int64_t S;       // pixels of an image
    uint64_t magic;  // of S in flat tiles, of an image's tiles in others
    int shift;
    int C;
    uint32_t N;      // pixels of all images
    uint32_t tiles, per_image;

    DEV uint32_t quotient(uint32_t n) const { return (uint32_t)((n * magic) >> shift); }
};

// The tiles of B images of S pixels; false where 32 bits do not hold the bytes
// of a tile from its first image on, or the pixels' numbers.
template <typename Ti>
bool pixels_of(int64_t B, int64_t S, int C, Pixels& p)
{
    const int64_t N = B * S, e = sizeof(typename Ti::Type), bytes = (int64_t)1 << 32;
    if (N < 1 || N >= (int64_t)1 << 31) return false;
    if (((Ti::kFlat ? (Ti::P + 2 * S) * C : Ti::P) + (int64_t)Ti::kChannels * S) * e >= bytes) return false;
    p.S = S;
    p.C = C;
    p.N = (uint32_t)N;
    p.per_image = (uint32_t)((S + Ti::P - 1) / Ti::P);
    p.tiles = Ti::kFlat ? (uint32_t)((N + Ti::P - 1) / Ti::P) : (uint32_t)B * p.per_image;
    const int64_t d = Ti::kFlat ? S : p.per_image;
    p.shift = 31;
    while (((int64_t)1 << (p.shift - 31)) < d) ++p.shift;
    p.magic = (((uint64_t)1 << p.shift) + d - 1) / d;
    return true;
}

// Where a tile and a thread's pixels and channels lie. Planes are addressed by
// bytes from an element that is the same for the whole workgroup, so that the
// loads of all channels share one register of addresses.
template <typename Ti>
struct Place {
    using T = typename Ti::Type;
    uint32_t q0;    // the tile's first pixel, and its number of pixels
    int rows;
    uint32_t q;     // the thread's first pixel, and its number of pixels, up to V
    int count;
    uint32_t image; // of the thread's pixels
    int64_t base;   // element of the planes
    uint32_t bytes; // from there to channel slot * G of the thread's first pixel

    DEV Place(const Pixels& p, uint32_t tile, int px, int slot)
    {
        const uint32_t S = (uint32_t)p.S;
        if constexpr (Ti::kFlat) {
            q0 = tile * Ti::P;
            q = q0 + px * Ti::V;
            rows = p.N - q0 < Ti::P ? (int)(p.N - q0) : Ti::P;
            count = q < p.N ? Ti::V : 0;
            const uint32_t b0 = p.quotient(q0);
            image = count ? p.quotient(q) : b0;
            base = (int64_t)b0 * p.C * p.S;
            bytes = count ? (image - b0) * (uint32_t)p.C * S + (q - image * S) : 0;
        } else {
            image = p.quotient(tile);
            const uint32_t s0 = (tile - image * p.per_image) * Ti::P;
            q0 = image * S + s0;
            q = q0 + px * Ti::V;
            rows = S - s0 < Ti::P ? (int)(S - s0) : Ti::P;
            const int n = rows - px * Ti::V;
            count = n < 0 ? 0 : n < Ti::V ? n : Ti::V;
            base = (int64_t)image * p.C * p.S + s0;
            bytes = px * Ti::V;
        }
        bytes = (bytes + (uint32_t)(slot * Ti::G) * S) * (uint32_t)sizeof(T);
    }
    // Channels of the thread's unit of step k that there are, of C; more than G
    // where others follow, none or less where there is no unit.
    DEV int left(int C, int slot, int k) const { return count ? C - (k * Ti::NS + slot) * Ti::G : 0; }

    // The thread's pixels in channel (k * NS + slot) * G + g.
    template <typename E>
    DEV E* at(E* p, int64_t S, int k, int g) const
    {
        using B = std::conditional_t<std::is_const_v<E>, const char, char>;
        B* first = reinterpret_cast<B*>(p + base + (k * Ti::kChannels + g) * S);
        return reinterpret_cast<E*>(first + bytes);
    }
};

// Keeps the compiler from joining the common end of two branches into one that
// goes over arrays by an index (which puts them into memory).
#define APART asm volatile("")

// Whether a wavefront's units are all whole, or not there: one test for all of
// their channels then.
template <typename Ti>
DEV bool all_whole(int left) { return Ti::kRegular || !__any(left > 0 && left < Ti::G); }

// The thread's pixels of its unit of step k, if there is one; zeros for pixels
// and for channels that are not there.
template <typename Ti, typename T = typename Ti::Type>
DEV void load_pixels(const T* p, const Place<Ti>& at, int64_t S, int left, int k, float (&f)[Ti::V][Ti::G])
{
    const auto load = [&](int g, bool there) ALWAYS {
        Pack<T, Ti::V> q;
        if (Ti::kFlat || at.rows == Ti::P) {
#pragma unroll
            for (int i = 0; i < Ti::V; ++i) q.v[i] = T(0);
            if (there) q = load_pack<Ti::V>(at.at(p, S, k, g));
        } else {
            q = load_upto<Ti::V>(at.at(p, S, k, g), there ? at.count : 0);
            APART;
        }
#pragma unroll
        for (int i = 0; i < Ti::V; ++i) f[i][g] = to_f32(q.v[i]);
    };
    if (all_whole<Ti>(left)) {
        if (left > 0) {
#pragma unroll
            for (int g = 0; g < Ti::G; ++g) load(g, true);
        }
    } else {
#pragma unroll
        for (int g = 0; g < Ti::G; ++g) load(g, g < left);
        APART;
    }
}

template <typename Ti, typename T = typename Ti::Type>
DEV void store_pixels(T* p, const Place<Ti>& at, int64_t S, int left, int k, const float (&f)[Ti::V][Ti::G])
{
    const auto store = [&](int g) ALWAYS {
        Pack<T, Ti::V> q;
#pragma unroll
        for (int i = 0; i < Ti::V; ++i) q.v[i] = from_f32<T>(f[i][g]);
        if (Ti::kFlat || at.rows == Ti::P) {
            store_pack<Ti::V>(at.at(p, S, k, g), q);
        } else {
            store_upto<Ti::V>(at.at(p, S, k, g), at.count, q);
            APART;
        }
    };
    if (all_whole<Ti>(left)) {
        if (left > 0) {
#pragma unroll
            for (int g = 0; g < Ti::G; ++g) store(g);
        }
    } else {
#pragma unroll
        for (int g = 0; g < Ti::G; ++g)
            if (g < left) store(g);
        APART;
    }
}

}  // namespace wtc
