// Layer norm over the channels of each pixel, forward and backward: the
// kernels for any number of channels, the sum of the workgroups' partial sums,
// and which kernels run.
#include "norm_device.h"

namespace wtc {
namespace {

constexpr int kThreads = 256, kTile = 64;  // a tile: 64 pixels or 64 channels, one a lane

DEV float wave_sum(float v)
{
#pragma unroll
    for (int o = 32; o; o >>= 1) v += __shfl_xor(v, o);
    return v;
}

// Sum over the four wavefronts, for each lane.
DEV float tile_sum(float v, float (*red)[kTile])
{
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    __syncthreads();
    red[w][lane] = v;
    __syncthreads();
    return (red[0][lane] + red[1][lane]) + (red[2][lane] + red[3][lane]);
}

// First element of pixel q of planes.
DEV int64_t plane_at(const NormArgs& a, int64_t q)
{
    const int64_t b = q / a.S;
    return b * a.C * a.S + (q - b * a.S);
}

DEV float weight(const NormArgs& a, int c) { return a.w ? a.w[c] : 1.0f; }
DEV float bias(const NormArgs& a, int c) { return a.b ? a.b[c] : 0.0f; }

// ----------------------------------------------------------------------------
// any number of channels, and planes whose offsets pass 32 bits within a tile:
// the input is swept again for each statistic (three and two sweeps from cache
// for one from memory; 8 images of 1600 float32 channels, 49 x 49, took 460 and
// 975 us, a third of the tiles' rate)
// ----------------------------------------------------------------------------

// One row a wavefront.
template <typename T>
__global__ void __launch_bounds__(kThreads) rows_forward_any(const NormArgs a)
{
    const int lane = threadIdx.x & 63;
    for (int64_t q = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6); q < a.N; q += (int64_t)gridDim.x * 4) {
        const T* x = (const T*)a.x + q * a.x_stride;
        T* y = (T*)a.out + q * a.C;
        float s = 0.f;
        for (int c = lane; c < a.C; c += 64) s += to_f32(x[c]);
        const float mean = wave_sum(s) / a.C;
        s = 0.f;
        for (int c = lane; c < a.C; c += 64) {
            const float d = to_f32(x[c]) - mean;
            s += d * d;
        }
        const float rstd = 1.0f / sqrtf(wave_sum(s) / a.C + a.eps);
        for (int c = lane; c < a.C; c += 64)
            y[c] = from_f32<T>((to_f32(x[c]) - mean) * rstd * weight(a, c) + bias(a, c));
        if (a.mean && lane == 0) {
            a.mean[q] = mean;
            a.rstd[q] = rstd;
        }
    }
}

// One tile of 64 pixels a workgroup, each wavefront every fourth channel; rows
// go out through LDS, 64 channels at a time.
template <typename T, bool OUT_PLANES>
__global__ void __launch_bounds__(kThreads) planes_forward_any(const NormArgs a)
{
    __shared__ float red[4][kTile];
    __shared__ T turn[kTile][kTile + 1];
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    for (int64_t q0 = (int64_t)blockIdx.x * kTile; q0 < a.N; q0 += (int64_t)gridDim.x * kTile) {
        const int64_t q = q0 + lane;
        const bool in = q < a.N;
        const int64_t at = in ? plane_at(a, q) : 0;
        const T* x = (const T*)a.x + at;
        float s = 0.f;
        if (in)
            for (int c = w; c < a.C; c += 4) s += to_f32(x[c * a.S]);
        const float mean = tile_sum(s, red) / a.C;
        s = 0.f;
        if (in)
            for (int c = w; c < a.C; c += 4) {
                const float d = to_f32(x[c * a.S]) - mean;
                s += d * d;
            }
        const float rstd = 1.0f / sqrtf(tile_sum(s, red) / a.C + a.eps);
        if (a.mean && in && w == 0) {
            a.mean[q] = mean;
            a.rstd[q] = rstd;
        }
        for (int c0 = 0; c0 < a.C; c0 += kTile) {
            const int cn = a.C - c0 < kTile ? a.C - c0 : kTile;
            for (int c = w; c < cn; c += 4) {
                if (!in) break;
                const T y = from_f32<T>((to_f32(x[(c0 + c) * a.S]) - mean) * rstd * weight(a, c0 + c) + bias(a, c0 + c));
                if (OUT_PLANES)
                    ((T*)a.out)[at + (c0 + c) * a.S] = y;
                else
                    turn[c][lane] = y;
            }
            if (!OUT_PLANES) {
                __syncthreads();
                for (int p = w; p < kTile && q0 + p < a.N; p += 4)
                    if (lane < cn) ((T*)a.out)[(q0 + p) * a.C + c0 + lane] = turn[lane][p];
                __syncthreads();
            }
        }
    }
}

// dx, one row a wavefront.
template <typename T>
__global__ void __launch_bounds__(kThreads) rows_backward_any(const NormArgs a)
{
    const int lane = threadIdx.x & 63;
    for (int64_t q = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6); q < a.N; q += (int64_t)gridDim.x * 4) {
        const T* x = (const T*)a.x + q * a.x_stride;
        const T* dy = (const T*)a.dy + q * a.dy_stride;
        T* dx = (T*)a.out + q * a.C;
        const float mean = a.mean[q], rstd = a.rstd[q];
        float s1 = 0.f, s2 = 0.f;
        for (int c = lane; c < a.C; c += 64) {
            const float g = to_f32(dy[c]) * weight(a, c);
            s1 += g;
            s2 += g * ((to_f32(x[c]) - mean) * rstd);
        }
        s1 = wave_sum(s1) / a.C;
        s2 = wave_sum(s2) / a.C;
        for (int c = lane; c < a.C; c += 64)
            dx[c] = from_f32<T>(rstd * (to_f32(dy[c]) * weight(a, c) - s1 - (to_f32(x[c]) - mean) * rstd * s2));
    }
}

// dx of one tile of 64 pixels a workgroup; dy that is rows comes in through LDS.
template <typename T, bool OUT_PLANES>
__global__ void __launch_bounds__(kThreads) planes_backward_any(const NormArgs a)
{
    __shared__ float red[4][kTile];
    __shared__ T turn[kTile][kTile + 1];
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    for (int64_t q0 = (int64_t)blockIdx.x * kTile; q0 < a.N; q0 += (int64_t)gridDim.x * kTile) {
        const int64_t q = q0 + lane;
        const bool in = q < a.N;
        const int64_t at = in ? plane_at(a, q) : 0;
        const T* x = (const T*)a.x + at;
        const T* dy = (const T*)a.dy;
        const float mean = in ? a.mean[q] : 0.f, rstd = in ? a.rstd[q] : 0.f;
        float s1 = 0.f, s2 = 0.f;
        for (int pass = 0; pass < 2; ++pass) {
            for (int c0 = 0; c0 < a.C; c0 += kTile) {
                const int cn = a.C - c0 < kTile ? a.C - c0 : kTile;
                if (!OUT_PLANES) {
                    __syncthreads();
                    for (int p = w; p < kTile && q0 + p < a.N; p += 4)
                        if (lane < cn) turn[p][lane] = dy[(q0 + p) * a.dy_stride + c0 + lane];
                    __syncthreads();
                }
                for (int c = w; c < cn; c += 4) {
                    if (!in) break;
                    const float d = to_f32(OUT_PLANES ? dy[at + (c0 + c) * a.S] : turn[lane][c]);
                    const float g = d * weight(a, c0 + c);
                    const float xhat = (to_f32(x[(c0 + c) * a.S]) - mean) * rstd;
                    if (pass == 0) {
                        s1 += g;
                        s2 += g * xhat;
                    } else {
                        ((T*)a.out)[at + (c0 + c) * a.S] = from_f32<T>(rstd * (g - s1 - xhat * s2));
                    }
                }
            }
            if (pass == 0) {
                s1 = tile_sum(s1, red) / a.C;
                s2 = tile_sum(s2, red) / a.C;
            }
        }
    }
}

// Sums over pixels of dy * xhat and dy for 64 channels (blockIdx.x) and one of
// nparts runs of tiles (blockIdx.y).
template <typename T>
__global__ void __launch_bounds__(kThreads) rows_sums_any(const NormArgs a)
{
    __shared__ float red[4][kTile];
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, c = blockIdx.x * kTile + lane;
    const int64_t run = (a.N + a.nparts - 1) / a.nparts, q1 = blockIdx.y * run, q2 = q1 + run < a.N ? q1 + run : a.N;
    float sw = 0.f, sb = 0.f;
    if (c < a.C)
        for (int64_t q = q1 + w; q < q2; q += 4) {
            const float d = to_f32(((const T*)a.dy)[q * a.dy_stride + c]);
            sw += d * ((to_f32(((const T*)a.x)[q * a.x_stride + c]) - a.mean[q]) * a.rstd[q]);
            sb += d;
        }
    sw = tile_sum(sw, red);
    sb = tile_sum(sb, red);
    if (w == 0 && c < a.C) {
        float* part = a.part + (int64_t)blockIdx.y * 2 * a.C;
        part[c] = sw;
        part[a.C + c] = sb;
    }
}

template <typename T, bool OUT_PLANES>
__global__ void __launch_bounds__(kThreads) planes_sums_any(const NormArgs a)
{
    __shared__ T turn[kTile][kTile + 1];
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, c0 = blockIdx.x * kTile;
    const int cn = a.C - c0 < kTile ? a.C - c0 : kTile;
    const int64_t tiles = (a.N + kTile - 1) / kTile, run = (tiles + a.nparts - 1) / a.nparts;
    const T* dy = (const T*)a.dy;
    float sw[kTile / 4] = {}, sb[kTile / 4] = {};
    for (int64_t t = blockIdx.y * run; t < (blockIdx.y + 1) * run && t < tiles; ++t) {
        const int64_t q0 = t * kTile, q = q0 + lane;
        if (!OUT_PLANES) {
            __syncthreads();
            for (int p = w; p < kTile && q0 + p < a.N; p += 4)
                if (lane < cn) turn[p][lane] = dy[(q0 + p) * a.dy_stride + c0 + lane];
            __syncthreads();
        }
        if (q >= a.N) continue;
        const int64_t at = plane_at(a, q) + c0 * a.S;
        const float mean = a.mean[q], rstd = a.rstd[q];
#pragma unroll
        for (int i = 0; i < kTile / 4; ++i) {
            const int c = w + 4 * i;
            if (c >= cn) break;
            const float d = to_f32(OUT_PLANES ? dy[at + c * a.S] : turn[lane][c]);
            sw[i] += d * ((to_f32(((const T*)a.x)[at + c * a.S]) - mean) * rstd);
            sb[i] += d;
        }
    }
#pragma unroll
    for (int i = 0; i < kTile / 4; ++i) {
        const int c = w + 4 * i;
        const float u = wave_sum(sw[i]), v = wave_sum(sb[i]);
        if (c >= cn || lane) continue;
        float* part = a.part + (int64_t)blockIdx.y * 2 * a.C;
        part[c0 + c] = u;
        part[a.C + c0 + c] = v;
    }
}

// The sums of the rows of partial sums, in a fixed order: 16 columns a
// workgroup, every 16th row a thread, several rows on their way at once. 4 us,
// bound by latency (1024 rows of 192 sums).
constexpr int kColumns = 16, kRows = kThreads / kColumns;

__global__ void __launch_bounds__(kThreads)
sum_parts_kernel(const float* part, int64_t rows, int width, int half, float* out, float* out2)
{
    __shared__ float red[kRows][kColumns + 1];
    const int col = threadIdx.x % kColumns, row = threadIdx.x / kColumns, i = blockIdx.x * kColumns + col;
    float s = 0.f;
    if (i < width) {
#pragma unroll 8
        for (int64_t r = row; r < rows; r += kRows) s += part[r * width + i];
    }
    red[row][col] = s;
    __syncthreads();
    if (row || i >= width) return;
    s = 0.f;
#pragma unroll
    for (int r = 0; r < kRows; ++r) s += red[r][col];
    if (i < half) {
        if (out) out[i] = s;
    } else if (out2) {
        out2[i - half] = s;
    }
}

template <typename T>
hipError_t forward_t(const wtconv_norm_desc& d, const NormArgs& a, hipStream_t s)
{
    if (d.in == WTCONV_ROWS) {
        hipLaunchKernelGGL(rows_forward_any<T>, dim3(at_most((a.N + 3) / 4, 1 << 16)), dim3(kThreads), 0, s, a);
    } else {
        const dim3 grid(at_most((a.N + kTile - 1) / kTile, 1 << 16));
        if (d.out == WTCONV_PLANES)
            hipLaunchKernelGGL((planes_forward_any<T, true>), grid, dim3(kThreads), 0, s, a);
        else
            hipLaunchKernelGGL((planes_forward_any<T, false>), grid, dim3(kThreads), 0, s, a);
    }
    return hipGetLastError();
}

template <typename T>
hipError_t backward_t(const wtconv_norm_desc& d, const NormArgs& a, hipStream_t s)
{
    const dim3 sums((a.C + kTile - 1) / kTile, a.nparts);
    if (d.in == WTCONV_ROWS) {
        if (a.out)
            hipLaunchKernelGGL(rows_backward_any<T>, dim3(at_most((a.N + 3) / 4, 1 << 16)), dim3(kThreads), 0, s, a);
        if (a.part) hipLaunchKernelGGL(rows_sums_any<T>, sums, dim3(kThreads), 0, s, a);
    } else {
        const dim3 grid(at_most((a.N + kTile - 1) / kTile, 1 << 16));
        if (d.out == WTCONV_PLANES) {
            if (a.out) hipLaunchKernelGGL((planes_backward_any<T, true>), grid, dim3(kThreads), 0, s, a);
            if (a.part) hipLaunchKernelGGL((planes_sums_any<T, true>), sums, dim3(kThreads), 0, s, a);
        } else {
            if (a.out) hipLaunchKernelGGL((planes_backward_any<T, false>), grid, dim3(kThreads), 0, s, a);
            if (a.part) hipLaunchKernelGGL((planes_sums_any<T, false>), sums, dim3(kThreads), 0, s, a);
        }
    }
    return hipGetLastError();
}

bool launch_planes(bool forward, const wtconv_norm_desc& d, const NormArgs& a, hipStream_t s)
{
    const bool out_planes = d.out == WTCONV_PLANES;
    switch (d.dtype) {
        case WTCONV_F32: return launch_planes_f32(forward, out_planes, a, s);
        case WTCONV_BF16: return launch_planes_bf16(forward, out_planes, a, s);
        case WTCONV_F16: return launch_planes_f16(forward, out_planes, a, s);
    }
    return false;
}

}  // namespace

// Of rows, and of planes that the kernels here take: four workgroups a CU, half
// of that where their sums are long (2047 bfloat16 channels, 4096 rows: 61.0 us
// with 1024, 42.8 with 512), and no more than there are 16 rows.
int64_t norm_parts(const wtconv_norm_desc& d)
{
    int64_t parts = 0;
    if (d.in == WTCONV_PLANES && d.B && d.S)
        parts = (d.dtype == WTCONV_F32 ? parts_planes_f32 : parts_planes_16)(d.B, d.S, d.C);
    return parts ? parts : at_most((d.B * d.S + 15) / 16, d.C > 1024 ? 512 : 1024);
}

hipError_t launch_sum_parts(const float* part, int64_t rows, int width, int half, float* out, float* out2,
                            hipStream_t s)
{
    hipLaunchKernelGGL(sum_parts_kernel, dim3((width + kColumns - 1) / kColumns), dim3(kThreads), 0, s, part, rows, width,
                       half, out, out2);
    return hipGetLastError();
}

hipError_t launch_norm_forward(const wtconv_norm_desc& d, const NormArgs& a, hipStream_t s)
{
    if (d.in == WTCONV_ROWS ? launch_rows_forward(d.dtype, a, s) : launch_planes(true, d, a, s))
        return hipGetLastError();
    // More pixels than one launch takes (at most 256 threads a pixel): in two halves.
    const bool rows = d.in == WTCONV_ROWS;
    if (a.N >= kMaxThreads / 256 && (rows || a.B > 1)) {
        NormArgs half = a;
        half.B = a.B / 2;  // (of no concern to rows)
        half.N = rows ? a.N / 2 : half.B * a.S;
        const hipError_t e = launch_norm_forward(d, half, s);
        if (e != hipSuccess) return e;
        const int64_t size = d.dtype == WTCONV_F32 ? 4 : 2;
        half.x = (const char*)a.x + half.N * (rows ? a.x_stride : a.C) * size;
        half.out = (char*)a.out + half.N * a.C * size;
        half.mean = a.mean ? a.mean + half.N : nullptr;
        half.rstd = a.rstd ? a.rstd + half.N : nullptr;
        half.N = a.N - half.N;
        half.B = a.B - half.B;
        return launch_norm_forward(d, half, s);
    }
    switch (d.dtype) {
        case WTCONV_F32: return forward_t<float>(d, a, s);
        case WTCONV_BF16: return forward_t<uint16_t>(d, a, s);
        case WTCONV_F16: return forward_t<_Float16>(d, a, s);
    }
    return hipErrorInvalidValue;
}

hipError_t launch_norm_backward(const wtconv_norm_desc& d, NormArgs a, float* dw, float* db, hipStream_t s)
{
    hipError_t e = hipErrorInvalidValue;
    if (d.in == WTCONV_ROWS ? launch_rows_backward(d.dtype, a, s) : launch_planes(false, d, a, s)) {
        e = hipGetLastError();
    } else {
        switch (d.dtype) {
            case WTCONV_F32: e = backward_t<float>(d, a, s); break;
            case WTCONV_BF16: e = backward_t<uint16_t>(d, a, s); break;
            case WTCONV_F16: e = backward_t<_Float16>(d, a, s); break;
        }
    }
    if (e != hipSuccess || !a.part) return e;
    return launch_sum_parts(a.part, a.nparts, 2 * a.C, a.C, dw, db, s);
}

}  // namespace wtc
