// Scaled residual between planes and rows, forward and backward.
#include "block_internal.h"
#include "wtconv_device.h"

namespace wtc {
namespace {

constexpr int kThreads = 256, kTile = 64;  // tiles of 64 pixels by 64 channels, turned in LDS

DEV float wave_sum(float v)
{
#pragma unroll
    for (int o = 32; o; o >>= 1) v += __shfl_xor(v, o);
    return v;
}

// Workgroup: 64 channels (blockIdx.y), one tile of 64 pixels after another.
template <typename T>
__global__ void __launch_bounds__(kThreads) residual_forward(const ResidualArgs a)
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
__global__ void __launch_bounds__(kThreads) residual_backward(const ResidualArgs a)
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

int grid_for(int64_t items, int64_t most) { return (int)(items < most ? (items > 1 ? items : 1) : most); }

template <typename T>
hipError_t forward_t(const ResidualArgs& a, hipStream_t s)
{
    const dim3 grid(grid_for((a.N + kTile - 1) / kTile, 1 << 16), (a.C + kTile - 1) / kTile);
    hipLaunchKernelGGL(residual_forward<T>, grid, dim3(kThreads), 0, s, a);
    return hipGetLastError();
}

template <typename T>
hipError_t backward_t(const ResidualArgs& a, hipStream_t s)
{
    hipLaunchKernelGGL(residual_backward<T>, dim3(a.nparts, (a.C + kTile - 1) / kTile), dim3(kThreads), 0, s, a);
    return hipGetLastError();
}

}  // namespace

int64_t residual_parts(const wtconv_residual_desc& d) { return grid_for((d.B * d.S + kTile - 1) / kTile, 512); }

hipError_t launch_residual_forward(wtconv_dtype dt, const ResidualArgs& a, hipStream_t s)
{
    switch (dt) {
        case WTCONV_F32: return forward_t<float>(a, s);
        case WTCONV_BF16: return forward_t<uint16_t>(a, s);
        case WTCONV_F16: return forward_t<_Float16>(a, s);
    }
    return hipErrorInvalidValue;
}

hipError_t launch_residual_backward(wtconv_dtype dt, ResidualArgs a, float* dgamma, hipStream_t s)
{
    hipError_t e = hipErrorInvalidValue;
    switch (dt) {
        case WTCONV_F32: e = backward_t<float>(a, s); break;
        case WTCONV_BF16: e = backward_t<uint16_t>(a, s); break;
        case WTCONV_F16: e = backward_t<_Float16>(a, s); break;
    }
    if (e != hipSuccess || !a.part) return e;
    return launch_sum_parts(a.part, a.nparts, a.C, a.C, dgamma, nullptr, s);
}

}  // namespace wtc
