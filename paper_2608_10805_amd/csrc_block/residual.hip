// Scaled residual between planes and rows, forward and backward: one read of
// every input, one write of every output. Bound by memory: 128 images of 96
// bfloat16 channels, 56 x 56, 48 us forward (4.8 TB/s of x, z and y) and 59 us
// backward with d_gamma's sums (3.9); 64 images of 192 float32 channels, 28 x
// 28, 26 to 30 and 27 us (3.9 to 4.4 and 4.3 TB/s), of which the one round of
// workgroups that such a tensor makes spends a fifth with loads or stores alone;
// 32 images of 128 bfloat16 channels, 63 x 95 off alignment, 33 to 37 and 44 us
// (4.0 to 4.4 and 3.4 TB/s).
//
// A workgroup takes tiles of P pixels by a block of channels; rows are turned in
// LDS (turn.h), where a thread's own units are its own on both ways, so that z
// comes in and dz goes out through the same place without a barrier between.
// The backward pass keeps its channels' part of d_gamma in registers over all of
// its tiles.
#include "turn.h"

namespace wtc {
namespace {

constexpr int kThreads = 256, kTile = 64;  // tiles of 64 pixels by 64 channels, turned in LDS

DEV float wave_sum(float v)
{
#pragma unroll
    for (int o = 32; o; o >>= 1) v += __shfl_xor(v, o);
    return v;
}

// ----------------------------------------------------------------------------
// tensors whose offsets pass 32 bits within a tile, or with more tiles than one launch takes
// ----------------------------------------------------------------------------

// Workgroup: 64 channels (blockIdx.y), one tile of 64 pixels after another.
template <typename T>
__global__ void __launch_bounds__(kThreads) residual_forward_any(const ResidualArgs a)
{
    __shared__ T turn[kTile][kTile + 1];
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, c0 = blockIdx.y * kTile;
    const int cn = a.C - c0 < kTile ? a.C - c0 : kTile;
    const T *x = (const T*)a.x, *z = (const T*)a.z;
    for (int64_t q0 = (int64_t)blockIdx.x * kTile; q0 < a.N; q0 += (int64_t)gridDim.x * kTile) {
        for (int p = w; p < kTile && q0 + p < a.N; p += 4)
            if (lane < cn) turn[p][lane] = z[(q0 + p) * a.C + c0 + lane];
        __syncthreads();
        const int64_t q = q0 + lane;
        if (q < a.N) {
            const int64_t b = q / a.S, at = (b * a.C + c0) * a.S + (q - b * a.S);
            const float keep = a.keep ? a.keep[b] : 1.0f;
            for (int c = w; c < cn; c += 4) {
                const float scale = (a.gamma ? a.gamma[c0 + c] : 1.0f) * keep;
                ((T*)a.out)[at + c * a.S] = from_f32<T>(to_f32(x[at + c * a.S]) + scale * to_f32(turn[lane][c]));
            }
        }
        __syncthreads();
    }
}

// dz, and the partial sums for d_gamma of one of nparts runs of tiles (blockIdx.x).
template <typename T>
__global__ void __launch_bounds__(kThreads) residual_backward_any(const ResidualArgs a)
{
    __shared__ T turn[kTile][kTile + 1], back[kTile][kTile + 1];
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, c0 = blockIdx.y * kTile;
    const int cn = a.C - c0 < kTile ? a.C - c0 : kTile;
    const T *dy = (const T*)a.x, *z = (const T*)a.z;
    const int64_t tiles = (a.N + kTile - 1) / kTile, run = (tiles + a.nparts - 1) / a.nparts;
    float sum[kTile / 4] = {};
    for (int64_t t = blockIdx.x * run; t < (blockIdx.x + 1) * run && t < tiles; ++t) {
        const int64_t q0 = t * kTile;
        if (a.part)
            for (int p = w; p < kTile && q0 + p < a.N; p += 4)
                if (lane < cn) turn[p][lane] = z[(q0 + p) * a.C + c0 + lane];
        __syncthreads();
        const int64_t q = q0 + lane;
        if (q < a.N) {
            const int64_t b = q / a.S, at = (b * a.C + c0) * a.S + (q - b * a.S);
            const float keep = a.keep ? a.keep[b] : 1.0f;
#pragma unroll
            for (int i = 0; i < kTile / 4; ++i) {
                const int c = w + 4 * i;
                if (c >= cn) break;
                const float d = to_f32(dy[at + c * a.S]);
                if (a.part) sum[i] += d * to_f32(turn[lane][c]) * keep;
                back[lane][c] = from_f32<T>((a.gamma ? a.gamma[c0 + c] : 1.0f) * keep * d);
            }
        }
        __syncthreads();
        if (a.out)
            for (int p = w; p < kTile && q0 + p < a.N; p += 4)
                if (lane < cn) ((T*)a.out)[(q0 + p) * a.C + c0 + lane] = back[p][lane];
        __syncthreads();
    }
    if (!a.part) return;
#pragma unroll
    for (int i = 0; i < kTile / 4; ++i) {
        const float u = wave_sum(sum[i]);
        const int c = w + 4 * i;
        if (c < cn && lane == 0) a.part[(int64_t)blockIdx.x * a.C + c0 + c] = u;
    }
}

// ----------------------------------------------------------------------------
// the others
// ----------------------------------------------------------------------------

DEV float factor(const float* p, int64_t i) { return p ? p[i] : 1.0f; }

// f[g] = scale[c + g], ones without it or past C.
template <int G>
DEV void channel_factors(const float* p, int c, int left, float (&f)[G])
{
#pragma unroll
    for (int g = 0; g < G; ++g) f[g] = p && g < left ? p[c + g] : 1.0f;
}

template <typename Ti>
__global__ void __launch_bounds__(Ti::TH) residual_forward(const ResidualArgs a, const Pixels ps)
{
    using T = typename Ti::Type;
    using Tu = Turn<Ti>;
    constexpr int V = Ti::V, NS = Ti::NS, K = Ti::K, G = Ti::G;
    static_assert(Tu::kSteps == K, "a block of channels is turned at once");
    __shared__ uint4 turn[Tu::kSize];
    const int px = threadIdx.x % Ti::LP, slot = threadIdx.x / Ti::LP, c0 = blockIdx.y * Ti::kMaxC;
    const uint32_t tile = Ti::kShared ? follow(blockIdx.x, gridDim.x) : blockIdx.x;
    if (tile >= ps.tiles) return;
    const Place<Ti> at(ps, tile, px, slot);
    const T* x = (const T*)a.x + c0 * a.S;
    T* y = (T*)a.out + c0 * a.S;
    float v[K][V][G];
    int left[K];
#pragma unroll
    for (int k = 0; k < K; ++k) {
        left[k] = at.left(a.C - c0, slot, k);
        load_pixels<Ti>(x, at, a.S, left[k], k, v[k]);
    }
    Tu::template copy<false>((const T*)a.z + (int64_t)at.q0 * a.C + c0, a.C, turn, at.rows,
                             a.C - c0 < Tu::kWidth ? a.C - c0 : Tu::kWidth);
    const float keep = factor(a.keep, at.image);
    __syncthreads();
#pragma unroll
    for (int k = 0; k < K; ++k) {
        if (left[k] <= 0) continue;
        float z[V][G], scale[G];
        Tu::get(turn, px, k * NS + slot, z);
        channel_factors<G>(a.gamma, c0 + (k * NS + slot) * G, left[k], scale);
#pragma unroll
        for (int g = 0; g < G; ++g)
#pragma unroll
            for (int i = 0; i < V; ++i) v[k][i][g] += scale[g] * keep * z[i][g];
        store_pixels<Ti>(y, at, a.S, left[k], k, v[k]);
    }
}

template <typename Ti>
__global__ void __launch_bounds__(Ti::TH) residual_backward(const ResidualArgs a, const Pixels ps)
{
    using T = typename Ti::Type;
    using Tu = Turn<Ti>;
    constexpr int V = Ti::V, NS = Ti::NS, K = Ti::K, G = Ti::G;
    static_assert(Tu::kSteps == K, "a block of channels is turned at once");
    __shared__ uint4 turn[Tu::kSize];
    const int px = threadIdx.x % Ti::LP, slot = threadIdx.x / Ti::LP, c0 = blockIdx.y * Ti::kMaxC;
    const int width = a.C - c0 < Tu::kWidth ? a.C - c0 : Tu::kWidth;
    const T* dy = (const T*)a.x + c0 * a.S;
    float sum[K][G] = {};
    const uint32_t first = !Ti::kShared || gridDim.x % 8 ? blockIdx.x : follow(blockIdx.x, gridDim.x);
    for (uint32_t tile = first; tile < ps.tiles; tile += gridDim.x) {
        const Place<Ti> at(ps, tile, px, slot);
        float d[K][V][G];
        int left[K];
#pragma unroll
        for (int k = 0; k < K; ++k) {
            left[k] = at.left(a.C - c0, slot, k);
            load_pixels<Ti>(dy, at, a.S, left[k], k, d[k]);
        }
        const float keep = factor(a.keep, at.image);
        if (a.part) {
            Tu::template copy<false>((const T*)a.z + (int64_t)at.q0 * a.C + c0, a.C, turn, at.rows, width);
            __syncthreads();
        }
#pragma unroll
        for (int k = 0; k < K; ++k) {
            if (left[k] <= 0) continue;
            float z[V][G], scale[G];
            if (a.part) Tu::get(turn, px, k * NS + slot, z);
            channel_factors<G>(a.gamma, c0 + (k * NS + slot) * G, left[k], scale);
#pragma unroll
            for (int g = 0; g < G; ++g)
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    if (a.part) sum[k][g] += d[k][i][g] * z[i][g] * keep;  // (both zero past the end)
                    d[k][i][g] *= scale[g] * keep;
                }
            if (a.out) Tu::put(turn, px, k * NS + slot, d[k]);
        }
        __syncthreads();
        if (a.out) {
            Tu::template copy<true>((T*)a.out + (int64_t)at.q0 * a.C + c0, a.C, turn, at.rows, width);
            __syncthreads();
        }
    }
    if (!a.part) return;
#pragma unroll
    for (int k = 0; k < K; ++k)
#pragma unroll
        for (int g = 0; g < G; ++g) {
            const int c = c0 + (k * NS + slot) * G + g;
#pragma unroll
            for (int o = Ti::LP >> 1; o; o >>= 1) sum[k][g] += __shfl_xor(sum[k][g], o);
            if (px == 0 && c < a.C) a.part[(int64_t)blockIdx.x * a.C + c] = sum[k][g];
        }
}

// Channels of a block: the widest of those that leave the fewest lanes idle in
// the last one (32 and 64 where there are no more).
int block_channels(int C)
{
    if (C <= 32) return 32;
    if (C <= 64) return 64;
    return (C + 95) / 96 * 96 < (C + 127) / 128 * 128 ? 96 : 128;
}

template <typename Ti>
bool launch(bool forward, const ResidualArgs& a, hipStream_t s)
{
    Pixels ps;
    if (!pixels_of<Ti>(a.B, a.S, a.C, ps)) return false;
    if (forward && ((int64_t)ps.tiles + 7) / 8 * 8 * Ti::TH >= kMaxThreads) return false;
    const unsigned blocks = (unsigned)((a.C + Ti::kMaxC - 1) / Ti::kMaxC);
    if (forward)
        hipLaunchKernelGGL(residual_forward<Ti>, dim3((ps.tiles + 7) / 8 * 8, blocks), dim3(Ti::TH), 0, s, a, ps);
    else
        hipLaunchKernelGGL(residual_backward<Ti>, dim3(a.nparts, blocks), dim3(Ti::TH), 0, s, a, ps);
    return true;
}

template <typename T, int V, bool REGULAR>
bool launch_tile(bool forward, const ResidualArgs& a, hipStream_t s)
{
    constexpr int E = sizeof(T) / 2;  // 16-byte units of float32 hold half the channels: twice the steps
    constexpr int LP = V == 4 ? 16 : 64, K = V == 4 ? E : 4 * E;
    switch (block_channels(a.C)) {
        case 32: return launch<Tile<T, 64, V, LP, K, REGULAR>>(forward, a, s);
        case 64: return launch<Tile<T, 128, V, LP, K, REGULAR>>(forward, a, s);
        case 96:  // (float32, 192 channels: 33.2 and 40.3 us with 192 threads, 28.8 and 39.6 with 384)
            return launch<Tile<T, V == 4 ? 192 * E : 192, V, LP, V == 4 ? 1 : K, REGULAR>>(forward, a, s);
        default: return launch<Tile<T, 256, V, LP, K, REGULAR>>(forward, a, s);
    }
}

// Vectors of four pixels, but for images so small that too much of a tile of 64
// pixels would be empty: single pixels then run over all images. 128 channels,
// forward and backward, single pixels against fours. float32: images of 25 pixels
// 17.8 + 29.4 and 17.3 + 32.8 us, of 35 18.0 + 29.9 and 16.6 + 26.3. bfloat16: of 49
// 12.3 + 24.0 and 14.9 + 26.6, of 65 14.2 + 23.6 and 11.0 + 20.4.
template <typename T>
hipError_t launch_t(bool forward, const ResidualArgs& a, hipStream_t s)
{
    bool done;
    if (a.S % 4 == 0 && a.C % (16 / (int)sizeof(T)) == 0)
        done = launch_tile<T, 4, true>(forward, a, s);
    else if (a.S >= (sizeof(T) == 4 ? 32 : 64) && launch_tile<T, 4, false>(forward, a, s))
        done = true;
    else
        done = launch_tile<T, 1, false>(forward, a, s);
    if (!done) {
        const unsigned blocks = (unsigned)((a.C + kTile - 1) / kTile);
        if (forward)
            hipLaunchKernelGGL(residual_forward_any<T>, dim3(at_most((a.N + kTile - 1) / kTile, 1 << 16), blocks),
                               dim3(kThreads), 0, s, a);
        else
            hipLaunchKernelGGL(residual_backward_any<T>, dim3(a.nparts, blocks), dim3(kThreads), 0, s, a);
    }
    return hipGetLastError();
}

hipError_t launch_type(wtconv_dtype dt, bool forward, const ResidualArgs& a, hipStream_t s)
{
    switch (dt) {
        case WTCONV_F32: return launch_t<float>(forward, a, s);
        case WTCONV_BF16: return launch_t<uint16_t>(forward, a, s);
        case WTCONV_F16: return launch_t<_Float16>(forward, a, s);
    }
    return hipErrorInvalidValue;
}

}  // namespace

// 16 wavefronts a CU over all blocks of channels.
int64_t residual_parts(const wtconv_residual_desc& d)
{
    const int64_t width = block_channels(d.C), blocks = (d.C + width - 1) / width, parts = 4096 / (width / 32) / blocks;
    return at_most((d.B * d.S + kTile - 1) / kTile, parts < 64 ? 64 : parts);
}

hipError_t launch_residual_forward(wtconv_dtype dt, const ResidualArgs& a, hipStream_t s)
{
    return launch_type(dt, true, a, s);
}

hipError_t launch_residual_backward(wtconv_dtype dt, ResidualArgs a, float* dgamma, hipStream_t s)
{
    const hipError_t e = launch_type(dt, false, a, s);
    if (e != hipSuccess || !a.part) return e;
    return launch_sum_parts(a.part, a.nparts, a.C, a.C, dgamma, nullptr, s);
}

}  // namespace wtc
