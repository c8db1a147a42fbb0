// Layer norm of planes with the channels of a tile of pixels in registers: one
// read and one write of every element.
//
// A workgroup takes P pixels and all C channels. LP lanes side by side hold V
// adjacent pixels each (P = LP * V), so that every load is a run of P pixels of
// one channel; slot s = thread / LP holds the channels (k * NS + s) * G to + G
// for k < K. The sums over the channels go over a lane's values, across the
// slots of a wavefront, and across the wavefronts through LDS. Rows (the output
// of the forward pass, dy of the backward pass) are turned in LDS (turn.h). The
// backward pass keeps the weight's and bias's gradients of its channels in
// registers over all of its workgroup's tiles.
//
// Bound by memory where runs of pixels and units of channels are whole: 64
// images of 96 channels, 56 x 56, float32, planes to rows, forward 31.7 us (4.9
// TB/s of x and y), backward 41 to 45 us (5.1 to 5.6 TB/s of x, dy and dx; a large
// copy reaches 5.3); 16 images of 64 channels, 224 x 224, planes to planes, 74.5 us
// (5.5 TB/s) and 137 us (4.5). In 16 bits 128 images of 96 channels, 56 x 56, take
// 31 us (5.0 TB/s) and 51 us (4.5), the backward pass with three wavefronts a SIMD
// by its registers. Odd channels and odd images cost up to twice the regular ones
// (32 images of 95 channels, 63 x 95, bfloat16: 32 and 61 us, 2.3 and 1.9 TB/s; of
// 96 channels, 64 x 96: 18 and 31 us).
#pragma once

#include "turn.h"

namespace wtc {

// The sum of s over all slots, for this lane's pixels.
template <typename Ti>
DEV void slot_sum(float (&s)[Ti::V], float (*red)[Ti::P])
{
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, px = threadIdx.x % Ti::LP;
#pragma unroll
    for (int v = 0; v < Ti::V; ++v) s[v] = sum_beyond<Ti::LP>(s[v]);
    if (lane < Ti::LP)
#pragma unroll
        for (int v = 0; v < Ti::V; ++v) red[w][px * Ti::V + v] = s[v];
    __syncthreads();
#pragma unroll
    for (int v = 0; v < Ti::V; ++v) {
        s[v] = 0.f;
#pragma unroll
        for (int i = 0; i < Ti::NW; ++i) s[v] += red[i][px * Ti::V + v];
    }
}

// f[g] = p[c + g], or `none` without p or past C.
template <int G>
DEV void load_channels(const float* p, int c, int C, float none, float (&f)[G])
{
    struct Quad { float v[4]; };
    if (p && c + G <= C) {
#pragma unroll
        for (int g = 0; g < G; g += 4) {
            const Quad q = *reinterpret_cast<const Quad*>(p + c + g);
#pragma unroll
            for (int i = 0; i < 4; ++i) f[g + i] = q.v[i];
        }
    } else {
#pragma unroll
        for (int g = 0; g < G; ++g) f[g] = p && c + g < C ? p[c + g] : none;
    }
}

template <typename Ti, bool OUT_PLANES>
__global__ void __launch_bounds__(Ti::TH) planes_forward(const NormArgs a, const Pixels ps)
{
    using T = typename Ti::Type;
    using Tu = Turn<Ti>;
    constexpr int V = Ti::V, NS = Ti::NS, K = Ti::K, G = Ti::G;
    __shared__ float red[2][Ti::NW][Ti::P];
    __shared__ uint4 turn[OUT_PLANES ? 1 : Tu::kSize];
    const int px = threadIdx.x % Ti::LP, slot = threadIdx.x / Ti::LP;
    const uint32_t tile = Ti::kShared ? follow(blockIdx.x, gridDim.x) : blockIdx.x;
    if (tile >= ps.tiles) return;
    const Place<Ti> at(ps, tile, px, slot);
    float v[K][V][G], w[K][G], b[K][G], s[V] = {}, mean[V], rstd[V];
    int left[K];
#pragma unroll
    for (int k = 0; k < K; ++k) {
        left[k] = at.left(a.C, slot, k);
        load_pixels<Ti>((const T*)a.x, at, a.S, left[k], k, v[k]);
    }
    // on their way behind x, and here before the sums need them
#pragma unroll
    for (int k = 0; k < K; ++k) {
        load_channels<G>(a.w, (k * NS + slot) * G, a.C, 1.0f, w[k]);
        load_channels<G>(a.b, (k * NS + slot) * G, a.C, 0.0f, b[k]);
    }
#pragma unroll
    for (int k = 0; k < K; ++k)
        if (left[k] > 0) {
#pragma unroll
            for (int i = 0; i < V; ++i)
#pragma unroll
                for (int g = 0; g < G; ++g) s[i] += v[k][i][g];
        }
    slot_sum<Ti>(s, red[0]);
    const float per = 1.0f / a.C;
#pragma unroll
    for (int i = 0; i < V; ++i) {
        mean[i] = divided(s[i], (float)a.C, per);
        s[i] = 0.f;
    }
    // the variance from the centred values, which are at hand: no cancellation
#pragma unroll
    for (int k = 0; k < K; ++k)
        if (left[k] > 0) {
#pragma unroll
            for (int i = 0; i < V; ++i)
#pragma unroll
                for (int g = 0; g < G; ++g) {
                    v[k][i][g] = Ti::kRegular || g < left[k] ? v[k][i][g] - mean[i] : 0.f;
                    s[i] += v[k][i][g] * v[k][i][g];
                }
        }
    slot_sum<Ti>(s, red[1]);
#pragma unroll
    for (int i = 0; i < V; ++i) rstd[i] = inverse_root(s[i] * per + a.eps);
    if (a.mean && slot == 0) {
        store_upto<V>(a.mean + at.q, at.count, __builtin_bit_cast(Pack<float, V>, mean));
        store_upto<V>(a.rstd + at.q, at.count, __builtin_bit_cast(Pack<float, V>, rstd));
    }
#pragma unroll
    for (int k = 0; k < K; ++k) {
        if (left[k] <= 0) continue;
#pragma unroll
        for (int i = 0; i < V; ++i)
#pragma unroll
            for (int g = 0; g < G; ++g) v[k][i][g] = v[k][i][g] * rstd[i] * w[k][g] + b[k][g];
        if (OUT_PLANES) store_pixels<Ti>((T*)a.out, at, a.S, left[k], k, v[k]);
    }
    if constexpr (!OUT_PLANES) {
#pragma unroll
        for (int k0 = 0; k0 < K; k0 += Tu::kSteps) {
            const int c0 = k0 * Ti::kChannels;
            if (c0 >= a.C) break;
            if (k0) __syncthreads();
#pragma unroll
            for (int k = k0; k < k0 + Tu::kSteps && k < K; ++k)
                if (left[k] > 0) Tu::put(turn, px, (k - k0) * NS + slot, v[k]);
            __syncthreads();
            Tu::template copy<true>((T*)a.out + (int64_t)at.q0 * a.C + c0, a.C, turn, at.rows,
                                    a.C - c0 < Tu::kWidth ? a.C - c0 : Tu::kWidth);
        }
    }
}

// DIRECT: dy's rows go from memory into LDS, the next tile's as soon as all have
// read this one's, instead of through registers after x has come. Planes to rows
// without and with it: bfloat16, 128 images of 96 channels, 56 x 56, 57.2 and 51.4
// us, 64 of 768, 14 x 14, 36.3 and 30.8; float32, 64 of 96, 56 x 56, 49.2 and 45.2.
// (x read ahead as well cost a wavefront a SIMD: 64 of 64 bfloat16 channels, 112 x
// 112, with the last sums 72.4 and 87.0 us.) It needs rows that begin at multiples
// of 16 bytes and units that are whole.
template <typename Ti, bool OUT_PLANES, bool DIRECT>
__global__ void __launch_bounds__(Ti::TH) planes_backward(const NormArgs a, const Pixels ps)
{
    using T = typename Ti::Type;
    using Tu = Turn<Ti>;
    constexpr int V = Ti::V, NS = Ti::NS, K = Ti::K, G = Ti::G;
    __shared__ float red[2][Ti::NW][Ti::P];
    __shared__ uint4 turn[OUT_PLANES ? 1 : Tu::kSize];
    const int px = threadIdx.x % Ti::LP, slot = threadIdx.x / Ti::LP;
    const float per = 1.0f / a.C;
    float sw[K][G] = {}, sb[K][G] = {};
    const uint32_t first = !Ti::kShared || gridDim.x % 8 ? blockIdx.x : follow(blockIdx.x, gridDim.x);
    const auto fetch = [&](uint32_t tile) ALWAYS {
        if constexpr (DIRECT)
            if (tile < ps.tiles) {
                const uint32_t q0 = tile * Ti::P;
                Tu::fetch((const T*)a.dy + q0 * a.dy_stride, a.dy_stride, turn, ps.N - q0, a.C / G);
            }
    };
    fetch(first);
    for (uint32_t tile = first; tile < ps.tiles; tile += gridDim.x) {
        const Place<Ti> at(ps, tile, px, slot);
        float xhat[K][V][G], g[K][V][G], s1[V] = {}, s2[V] = {}, mean[V], rstd[V];
        int left[K];
#pragma unroll
        for (int k = 0; k < K; ++k) {
            left[k] = at.left(a.C, slot, k);
            load_pixels<Ti>((const T*)a.x, at, a.S, left[k], k, xhat[k]);
            if (OUT_PLANES) load_pixels<Ti>((const T*)a.dy, at, a.S, left[k], k, g[k]);
        }
        // (a pixel that is not there: zeros, which add nothing to the sums)
        const auto m = load_upto<V>(a.mean + at.q, at.count), r = load_upto<V>(a.rstd + at.q, at.count);
#pragma unroll
        for (int i = 0; i < V; ++i) {
            mean[i] = m.v[i];
            rstd[i] = r.v[i];
        }
        if constexpr (DIRECT) {
            Tu::fetched();
            __syncthreads();
#pragma unroll
            for (int k = 0; k < K; ++k)
                if (left[k] > 0) Tu::get(turn, px, k * NS + slot, g[k]);
        } else if constexpr (!OUT_PLANES) {
#pragma unroll
            for (int k0 = 0; k0 < K; k0 += Tu::kSteps) {
                const int c0 = k0 * Ti::kChannels;
                if (c0 >= a.C) break;
                __syncthreads();
                Tu::template copy<false>((const T*)a.dy + at.q0 * a.dy_stride + c0, a.dy_stride, turn, at.rows,
                                         a.C - c0 < Tu::kWidth ? a.C - c0 : Tu::kWidth);
                __syncthreads();
#pragma unroll
                for (int k = k0; k < k0 + Tu::kSteps && k < K; ++k)
                    if (left[k] > 0) Tu::get(turn, px, (k - k0) * NS + slot, g[k]);
            }
        }
#pragma unroll
        for (int k = 0; k < K; ++k) {
            // (a channel that is not there has dy = 0: it adds nothing to any sum)
            if (left[k] <= 0) continue;
            float w[G];
            load_channels<G>(a.w, (k * NS + slot) * G, a.C, 1.0f, w);
#pragma unroll
            for (int j = 0; j < G; ++j)
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    xhat[k][i][j] = (xhat[k][i][j] - mean[i]) * rstd[i];
                    sw[k][j] += g[k][i][j] * xhat[k][i][j];
                    sb[k][j] += g[k][i][j];
                    g[k][i][j] *= w[j];
                    s1[i] += g[k][i][j];
                    s2[i] += g[k][i][j] * xhat[k][i][j];
                }
        }
        if (!a.out) {
            if constexpr (DIRECT) __syncthreads();
            fetch(tile + gridDim.x);
            continue;
        }
        if constexpr (!DIRECT) __syncthreads();  // the last tile's sums have been read
        slot_sum<Ti>(s1, red[0]);
        fetch(tile + gridDim.x);
        slot_sum<Ti>(s2, red[1]);
#pragma unroll
        for (int i = 0; i < V; ++i) {
            s1[i] *= per * rstd[i];
            s2[i] *= per * rstd[i];
        }
#pragma unroll
        for (int k = 0; k < K; ++k) {
            if (left[k] > 0) {
#pragma unroll
                for (int i = 0; i < V; ++i)
#pragma unroll
                    for (int j = 0; j < G; ++j)
                        g[k][i][j] = rstd[i] * g[k][i][j] - s1[i] - xhat[k][i][j] * s2[i];
            }
            store_pixels<Ti>((T*)a.out, at, a.S, left[k], k, g[k]);
        }
    }
    if (!a.part) return;
    float* part = a.part + (int64_t)blockIdx.x * 2 * a.C;
#pragma unroll
    for (int k = 0; k < K; ++k)
#pragma unroll
        for (int j = 0; j < G; ++j) {
            const int c = (k * NS + slot) * G + j;
#pragma unroll
            for (int o = Ti::LP >> 1; o; o >>= 1) {
                sw[k][j] += __shfl_xor(sw[k][j], o);
                sb[k][j] += __shfl_xor(sb[k][j], o);
            }
            if (px == 0 && c < a.C) {
                part[c] = sw[k][j];
                part[a.C + c] = sb[k][j];
            }
        }
}

// The tiles of a type and vector, by index.
template <typename T, int V, bool REGULAR, typename F>
bool planes_tile(int index, F&& f)
{
#define WTC_TILE(i, TH, LP, K) \
    case i: f(Tile<T, TH, V, LP, K, REGULAR>{}); return true
    if constexpr (sizeof(T) == 4 && V == 4) {
        switch (index) {
            WTC_TILE(0, 192, 16, 2);
            WTC_TILE(1, 256, 16, 2);
            WTC_TILE(2, 192, 8, 1);
            WTC_TILE(3, 192, 8, 2);
            WTC_TILE(4, 256, 8, 3);
            WTC_TILE(5, 192, 4, 1);
            WTC_TILE(6, 192, 4, 2);
            WTC_TILE(7, 256, 4, 3);
            WTC_TILE(8, 512, 4, 3);
            WTC_TILE(9, 512, 2, 2);
            WTC_TILE(10, 64, 16, 2);
            WTC_TILE(11, 128, 16, 2);
        }
    } else if constexpr (V == 4) {
        switch (index) {
            WTC_TILE(0, 192, 16, 1);
            WTC_TILE(1, 256, 16, 1);
            WTC_TILE(2, 192, 8, 1);
            WTC_TILE(3, 256, 8, 1);
            WTC_TILE(4, 192, 4, 1);
            WTC_TILE(5, 256, 4, 1);
            WTC_TILE(6, 384, 4, 1);
            WTC_TILE(7, 384, 8, 1);
            WTC_TILE(8, 512, 8, 2);
            WTC_TILE(9, 512, 4, 1);
            WTC_TILE(10, 512, 2, 1);
            WTC_TILE(11, 64, 16, 1);
            WTC_TILE(12, 128, 16, 1);
        }
    } else {
        constexpr int E = 4 / sizeof(T);  // twice the channels a unit, half the steps
        switch (index) {
            WTC_TILE(0, 256, 64, E == 1 ? 6 : 3);
            WTC_TILE(1, 256, 32, E == 1 ? 6 : 3);
            WTC_TILE(2, 256, 16, E == 1 ? 6 : 3);
            WTC_TILE(3, 512, 16, E == 1 ? 6 : 3);
            WTC_TILE(4, 512, 8, E == 1 ? 8 : 4);
        }
    }
#undef WTC_TILE
    return false;
}

// The tile for B images of S pixels and C channels, or -1 where none holds the
// channels: by the share of lanes that have channels and pixels, the length of
// the runs of pixels (whole lines of 128 bytes are best), and whether there are
// two tiles a CU.
template <typename T, int V, bool REGULAR>
int pick_tile(int64_t B, int64_t S, int C, double& best_score)
{
    int best = -1, most = 0, pixels = 0, step = 1;
    bool flat = false;
    best_score = 0;
    for (int i = 0; planes_tile<T, V, REGULAR>(i, [&](auto t) {
             using Ti = decltype(t);
             most = Ti::kMaxC;
             pixels = Ti::P;
             step = Ti::kChannels;
             flat = Ti::kFlat;
         });
         ++i) {
        if (C > most) continue;
        const double tiles = flat ? (double)(B * S + pixels - 1) / pixels : (double)B * ((S + pixels - 1) / pixels);
        const double lanes = (double)C / ((C + step - 1) / step * step) * ((double)(B * S) / (tiles * pixels));
        const int run = pixels * (int)sizeof(T);
        // (shorter runs meet in the XCD's L2; off alignment each has two ends in lines of others)
        const double lines = run >= 128 ? 1.0 : run >= 64 || REGULAR ? 0.9 : 0.7;
        const double score = lanes * lines * (tiles >= 512 ? 1.0 : tiles / 512);
        if (score > best_score) {
            best_score = score;
            best = i;
        }
    }
    return best;
}

// Calls f with the tile for these planes, false where there is none: vectors of
// four pixels, but for images so small that too many of them would be incomplete
// (single pixels then run over all images). 128 channels, forward and backward,
// single pixels against fours. float32, whose single pixels are slower: images of
// 9 pixels 13.3 + 40.0 and 13.7 + 28.0 us (of the tiles' scores the ratio is 0.34),
// of 3 12.9 + 29.3 and 15.9 + 32.1. bfloat16: of 35 9.7 + 25.8 and 11.4 + 29.1 (ratio
// 0.61), of 81 11.0 + 32.5 and 11.3 + 28.8 (0.70).
template <typename T, typename F>
bool with_tile(int64_t B, int64_t S, int C, F&& f)
{
    double fours = 0, ones = 0;
    if (S % 4 == 0 && C % (16 / (int)sizeof(T)) == 0) return planes_tile<T, 4, true>(pick_tile<T, 4, true>(B, S, C, fours), f);
    const int i = pick_tile<T, 4, false>(B, S, C, fours), j = pick_tile<T, 1, false>(B, S, C, ones);
    return fours >= (sizeof(T) == 4 ? 0.3 : 0.65) * ones ? planes_tile<T, 4, false>(i, f) : planes_tile<T, 1, false>(j, f);
}

// Workgroups of the backward pass: as many as are resident by the registers that
// their threads' values take, no more than there are tiles. What each adds is 2 C
// sums to write and to read again, so that many channels get four a CU at most.
// Measured on 384 bfloat16 channels, 14 x 14, B128: tiles of 192 threads 48.2,
// 35.6, 34.8 us with 256, 512, 1024 workgroups, tiles of 512 threads 44.0, 46.5,
// 55.6 us.
template <typename T>
int64_t planes_parts(int64_t B, int64_t S, int C)
{
    int64_t n = 0;
    with_tile<T>(B, S, C, [&](auto t) {
        using Ti = decltype(t);
        Pixels ps;
        if (!pixels_of<Ti>(B, S, C, ps)) return;
        const int resident = 24576 / (Ti::TH * Ti::K * Ti::V * Ti::G), few = C <= 32 ? 12 : C <= 64 ? 6 : 4;
        n = at_most(ps.tiles, 256 * (resident < 1 ? 1 : resident < few ? resident : few));
    });
    return n;
}

// x and dx are planes, and y or dy if `out_planes`.
template <typename T>
bool planes_launch(bool forward, bool out_planes, const NormArgs& a, hipStream_t s)
{
    bool done = false;
    with_tile<T>(a.B, a.S, a.C, [&](auto t) {
        using Ti = decltype(t);
        Pixels ps;
        if (!pixels_of<Ti>(a.B, a.S, a.C, ps)) return;
        if (forward && ((int64_t)ps.tiles + 7) / 8 * 8 * Ti::TH >= kMaxThreads) return;
        done = true;
        const dim3 grid(forward ? (ps.tiles + 7) / 8 * 8 : (unsigned)a.nparts), block(Ti::TH);
        if (forward && out_planes)
            hipLaunchKernelGGL((planes_forward<Ti, true>), grid, block, 0, s, a, ps);
        else if (forward)
            hipLaunchKernelGGL((planes_forward<Ti, false>), grid, block, 0, s, a, ps);
        else if (out_planes)
            hipLaunchKernelGGL((planes_backward<Ti, true, false>), grid, block, 0, s, a, ps);
        else if constexpr (Turn<Ti>::kDirect) {
            if (((uintptr_t)a.dy | (uintptr_t)a.dy_stride * sizeof(T)) % 16 == 0)
                hipLaunchKernelGGL((planes_backward<Ti, false, true>), grid, block, 0, s, a, ps);
            else
                hipLaunchKernelGGL((planes_backward<Ti, false, false>), grid, block, 0, s, a, ps);
        } else
            hipLaunchKernelGGL((planes_backward<Ti, false, false>), grid, block, 0, s, a, ps);
    });
    return done;
}

}  // namespace wtc
