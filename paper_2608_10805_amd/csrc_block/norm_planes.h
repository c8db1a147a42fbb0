// Layer norm of planes with the channels of a tile of pixels in registers.
//
// A workgroup takes P pixels and all C channels. LP lanes side by side hold V
// adjacent pixels each (P = LP * V), so that every load is a run of P pixels of
// one channel; slot s = thread / LP holds the channels s, s + NS, ... of them,
// at most K. Each value is read once. The sums over the channels go lane by
// lane over the K values, across the slots of a wavefront, and across the
// wavefronts through LDS. Rows (the output of the forward pass, dy of the
// backward pass) are turned in LDS, `chunk` channels at a time, with rows an
// odd number of words apart so that neither side meets its own banks.
#pragma once

#include "norm_device.h"

namespace wtc {

template <int TH_, int V_, int LP_, int K_>
struct PlanesShape {
    static constexpr int TH = TH_, V = V_, LP = LP_, K = K_;
    static constexpr int P = LP * V, NS = TH / LP, NW = TH / 64;
    static constexpr int kMaxC = NS * K;
};

constexpr int kTurnBytes = 32 * 1024;  // LDS that turns rows: leaves room for four workgroups a CU and more

// Elements between two rows in LDS: an odd number of words, at least `width` elements.
template <typename T>
__host__ __device__ constexpr int turn_stride(int width)
{
    constexpr int per = 4 / sizeof(T);
    const int words = (width + per - 1) / per;
    return (words | 1) * per;
}

// Slots' values that are turned at once: chunk channels = slots * (this many).
template <typename T, typename Sh>
__host__ __device__ constexpr int turn_steps()
{
    int n = Sh::K;
    while (n > 1 && Sh::P * turn_stride<T>(n * Sh::NS) * (int)sizeof(T) > kTurnBytes) --n;
    return n;
}

template <typename T, typename Sh>
constexpr int turn_elements()
{
    return Sh::P * turn_stride<T>(turn_steps<T, Sh>() * Sh::NS);
}

// The sum of s over all slots, for this lane's pixels.
template <typename Sh>
DEV void slot_sum(float (&s)[Sh::V], float (*red)[Sh::P])
{
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, px = threadIdx.x % Sh::LP;
#pragma unroll
    for (int v = 0; v < Sh::V; ++v)
#pragma unroll
        for (int o = Sh::LP; o < 64; o <<= 1) s[v] += __shfl_xor(s[v], o);
    if (lane < Sh::LP)
#pragma unroll
        for (int v = 0; v < Sh::V; ++v) red[w][px * Sh::V + v] = s[v];
    __syncthreads();
#pragma unroll
    for (int v = 0; v < Sh::V; ++v) {
        s[v] = 0.f;
#pragma unroll
        for (int i = 0; i < Sh::NW; ++i) s[v] += red[i][px * Sh::V + v];
    }
}

// Calls f(row, column, element of the tile) for the count x width elements of
// consecutive rows, two adjacent columns at once for 16-bit types if `pairs`.
template <int TH, int STEP, typename F>
DEV void over_rows(int count, int width, F&& f)
{
    const int per = width / STEP;
    const uint32_t magic = 0xffffffffu / (uint32_t)per + 1u;  // exact for products below 2^32 / width
    for (int i = threadIdx.x; i < count * per; i += TH) {
        const int r = per == 1 ? i : (int)__umulhi((uint32_t)i, magic);
        f(r, (i - r * per) * STEP);
    }
}

// Copies `count` rows of `width` channels from c0 on between memory (rows
// `pitch` apart) and LDS (rows `stride` apart).
template <bool OUT, int TH, typename T, typename U>
DEV void turn_rows(U* mem, int64_t pitch, T* turn, int stride, int count, int width, int c0, bool pairs)
{
    if (sizeof(T) == 2 && pairs) {
        over_rows<TH, 2>(count, width, [&](int r, int c) {
            auto* m = reinterpret_cast<std::conditional_t<OUT, uint32_t, const uint32_t>*>(mem + r * pitch + c0 + c);
            auto* t = reinterpret_cast<uint32_t*>(turn + r * stride + c);
            if constexpr (OUT)
                *m = *t;
            else
                *t = *m;
        });
    } else {
        over_rows<TH, 1>(count, width, [&](int r, int c) {
            if constexpr (OUT)
                mem[r * pitch + c0 + c] = turn[r * stride + c];
            else
                turn[r * stride + c] = mem[r * pitch + c0 + c];
        });
    }
}

// First element of pixel q of planes.
DEV int64_t pixel_at(const NormArgs& a, int64_t q)
{
    const int64_t b = q / a.S;
    return b * a.C * a.S + (q - b * a.S);
}

// The shapes by number of channels, smallest tile of values first; a shape is
// chosen by pick_planes().
template <int V, typename F>
bool planes_shape(int index, F&& f)
{
    if constexpr (V == 4) {
        switch (index) {
            case 0: f(PlanesShape<256, 4, 16, 6>{}); return true;
            case 1: f(PlanesShape<256, 4, 16, 12>{}); return true;
            case 2: f(PlanesShape<256, 4, 8, 6>{}); return true;
            case 3: f(PlanesShape<256, 4, 8, 12>{}); return true;
            case 4: f(PlanesShape<256, 4, 4, 6>{}); return true;
            case 5: f(PlanesShape<256, 4, 4, 12>{}); return true;
            case 6: f(PlanesShape<512, 4, 4, 16>{}); return true;
        }
    } else {
        switch (index) {
            case 0: f(PlanesShape<256, 1, 64, 12>{}); return true;
            case 1: f(PlanesShape<256, 1, 64, 24>{}); return true;
            case 2: f(PlanesShape<256, 1, 32, 12>{}); return true;
            case 3: f(PlanesShape<256, 1, 32, 24>{}); return true;
            case 4: f(PlanesShape<256, 1, 16, 12>{}); return true;
            case 5: f(PlanesShape<256, 1, 16, 24>{}); return true;
            case 6: f(PlanesShape<512, 1, 16, 24>{}); return true;
            case 7: f(PlanesShape<512, 1, 8, 32>{}); return true;
        }
    }
    return false;
}

// The shape for C channels and N pixels, or -1 where none holds them: the
// longest runs of pixels that still leave four tiles a CU, else the shortest.
template <int V>
int pick_planes(int C, int64_t N)
{
    int best = -1, best_pixels = 0, most = 0, pixels = 0;
    for (int i = 0; planes_shape<V>(i, [&](auto sh) { most = decltype(sh)::kMaxC; pixels = decltype(sh)::P; }); ++i) {
        if (C > most || (best >= 0 && C * 4 < most)) continue;  // (too few channels for so many slots)
        if (N >= (int64_t)pixels * 1024) return i;
        if (best < 0 || pixels < best_pixels) {
            best = i;
            best_pixels = pixels;
        }
    }
    return best;
}

// Pixels that are loaded at once: four where every image's planes begin and end
// at a whole vector.
inline int planes_vector(const NormArgs& a, size_t element, const void* other)
{
    const uintptr_t all = (uintptr_t)a.x | (uintptr_t)a.out | (uintptr_t)other;
    return a.S % 4 == 0 && all % (4 * element) == 0 ? 4 : 1;
}

}  // namespace wtc
