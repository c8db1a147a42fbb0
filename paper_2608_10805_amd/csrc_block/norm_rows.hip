// Layer norm of rows with a row in the registers of a group of lanes, forward
// and backward: one read of every input, one write of every output.
//
// GL lanes (a power of two, up to a wavefront) hold a row: lane l the vectors
// l, l + GL, ... of V elements, at most R of them. 64 / GL rows a wavefront.
#include "norm_device.h"

namespace wtc {
namespace {

constexpr int kThreads = 256;

template <typename T, int V, int R>
__global__ void __launch_bounds__(kThreads) rows_forward(const NormArgs a, int gl)
{
    const int lane = threadIdx.x & (gl - 1);
    const int64_t q = (int64_t)blockIdx.x * (kThreads / gl) + threadIdx.x / gl;
    if (q >= a.N) return;  // (whole groups)
    const T* x = (const T*)a.x + q * a.x_stride;
    float v[R][V], s = 0.f;
#pragma unroll
    for (int r = 0; r < R; ++r) {
        const int c = (r * gl + lane) * V;
        if (c < a.C) {
            load_pack<V>(x + c, v[r]);
        } else {
#pragma unroll
            for (int i = 0; i < V; ++i) v[r][i] = 0.f;
        }
    }
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
        for (int i = 0; i < V; ++i) s += v[r][i];
    const float per = 1.0f / a.C, mean = sum_within(s, gl) * per;
    s = 0.f;
    // the variance from the centred values, which are at hand: no cancellation
#pragma unroll
    for (int r = 0; r < R; ++r)
        if ((r * gl + lane) * V < a.C)
#pragma unroll
            for (int i = 0; i < V; ++i) {
                v[r][i] -= mean;
                s += v[r][i] * v[r][i];
            }
    const float rstd = 1.0f / sqrtf(sum_within(s, gl) * per + a.eps);
    if (a.mean && lane == 0) {
        a.mean[q] = mean;
        a.rstd[q] = rstd;
    }
    T* y = (T*)a.out + q * a.C;
#pragma unroll
    for (int r = 0; r < R; ++r) {
        const int c = (r * gl + lane) * V;
        if (c < a.C) {
#pragma unroll
            for (int i = 0; i < V; ++i)
                v[r][i] = v[r][i] * rstd * (a.w ? a.w[c + i] : 1.0f) + (a.b ? a.b[c + i] : 0.0f);
            store_pack<V>(y + c, v[r]);
        }
    }
}

// A workgroup takes rows in steps of all workgroups' rows; each lane sums the
// gradients of its own columns, the groups and wavefronts join at the end.
template <typename T, int V, int R>
__global__ void __launch_bounds__(kThreads) rows_backward(const NormArgs a, int gl)
{
    extern __shared__ float sums[];  // 2 C
    const int lane = threadIdx.x & (gl - 1), groups = kThreads / gl;
    const float per = 1.0f / a.C;
    float sw[R][V] = {}, sb[R][V] = {};
    for (int64_t q = (int64_t)blockIdx.x * groups + threadIdx.x / gl; q < a.N; q += (int64_t)gridDim.x * groups) {
        const T* x = (const T*)a.x + q * a.x_stride;
        const T* dy = (const T*)a.dy + q * a.dy_stride;
        float xhat[R][V], g[R][V], s1 = 0.f, s2 = 0.f;
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const int c = (r * gl + lane) * V;
            if (c < a.C) {
                load_pack<V>(x + c, xhat[r]);
                load_pack<V>(dy + c, g[r]);
            }
        }
        const float mean = a.mean[q], rstd = a.rstd[q];
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const int c = (r * gl + lane) * V;
            if (c < a.C)
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    xhat[r][i] = (xhat[r][i] - mean) * rstd;
                    sw[r][i] += g[r][i] * xhat[r][i];
                    sb[r][i] += g[r][i];
                    g[r][i] *= a.w ? a.w[c + i] : 1.0f;
                    s1 += g[r][i];
                    s2 += g[r][i] * xhat[r][i];
                }
        }
        if (!a.out) continue;
        s1 = sum_within(s1, gl) * per;
        s2 = sum_within(s2, gl) * per;
        T* dx = (T*)a.out + q * a.C;
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const int c = (r * gl + lane) * V;
            if (c < a.C) {
#pragma unroll
                for (int i = 0; i < V; ++i) g[r][i] = rstd * (g[r][i] - s1 - xhat[r][i] * s2);
                store_pack<V>(dx + c, g[r]);
            }
        }
    }
    if (!a.part) return;
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
        for (int i = 0; i < V; ++i)
            for (int o = gl; o < 64; o <<= 1) {
                sw[r][i] += __shfl_xor(sw[r][i], o);
                sb[r][i] += __shfl_xor(sb[r][i], o);
            }
    for (int w = 0; w < kThreads / 64; ++w) {  // one wavefront after the other, in their order
        if ((int)(threadIdx.x >> 6) == w && (threadIdx.x & 63) < gl)
#pragma unroll
            for (int r = 0; r < R; ++r)
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    const int c = (r * gl + lane) * V + i;
                    if (c < a.C) {
                        sums[c] = (w ? sums[c] : 0.f) + sw[r][i];
                        sums[a.C + c] = (w ? sums[a.C + c] : 0.f) + sb[r][i];
                    }
                }
        __syncthreads();
    }
    float* part = a.part + (int64_t)blockIdx.x * 2 * a.C;
    for (int i = threadIdx.x; i < 2 * a.C; i += kThreads) part[i] = sums[i];
}

// Lanes a row and vectors a lane for n vectors: the fewest idle lanes, of those
// the most vectors a lane (more bytes on their way, fewer steps of the sums).
bool layout(int n, int most, int& gl, int& r)
{
    int best = 0;
    for (int t = 1; t <= most; t = t < 4 ? t + 1 : t * 2) {
        int lanes = 1;
        while (lanes * t < n) lanes *= 2;
        if (lanes > 64) continue;
        const int used = n * 1024 / (lanes * t);
        if (used < best) continue;
        if (t > 4 && best) break;
        best = used;
        gl = lanes;
        r = t;
    }
    return best != 0;
}

template <typename T, int V, int R>
void launch_r(bool forward, const NormArgs& a, int gl, hipStream_t s)
{
    const int groups = kThreads / gl;
    if (forward)
        hipLaunchKernelGGL((rows_forward<T, V, R>), dim3((unsigned)((a.N + groups - 1) / groups)), dim3(kThreads), 0, s,
                           a, gl);
    else
        hipLaunchKernelGGL((rows_backward<T, V, R>), dim3(a.nparts), dim3(kThreads), (size_t)a.C * 8, s, a, gl);
}

template <typename T, int V>
bool launch_v(bool forward, const NormArgs& a, hipStream_t s)
{
    int gl = 0, r = 0;
    if (a.C % V || !layout(a.C / V, V == 1 ? 32 : 16 / sizeof(T) == V ? 8 : 16, gl, r)) return false;
    switch (r) {
        case 1: launch_r<T, V, 1>(forward, a, gl, s); return true;
        case 2: launch_r<T, V, 2>(forward, a, gl, s); return true;
        case 3: launch_r<T, V, 3>(forward, a, gl, s); return true;
        case 4: launch_r<T, V, 4>(forward, a, gl, s); return true;
        case 8: launch_r<T, V, 8>(forward, a, gl, s); return true;
        case 16:
            if constexpr (V == 1) launch_r<T, V, 16>(forward, a, gl, s);
            return V == 1;
        case 32:
            if constexpr (V == 1) launch_r<T, V, 32>(forward, a, gl, s);
            return V == 1;
    }
    return false;
}

template <typename T>
bool launch_t(bool forward, const NormArgs& a, hipStream_t s)
{
    constexpr int W = 16 / sizeof(T);
    const uintptr_t all = (uintptr_t)a.x | (uintptr_t)a.out | (uintptr_t)a.dy;
    if (all % 16 == 0 && a.x_stride % W == 0 && (forward || a.dy_stride % W == 0) && launch_v<T, W>(forward, a, s))
        return true;
    return launch_v<T, 1>(forward, a, s);
}

bool launch(wtconv_dtype dt, bool forward, const NormArgs& a, hipStream_t s)
{
    if (a.N > (int64_t)1 << 30) return false;  // workgroups of one launch
    switch (dt) {
        case WTCONV_F32: return launch_t<float>(forward, a, s);
        case WTCONV_BF16: return launch_t<uint16_t>(forward, a, s);
        case WTCONV_F16: return launch_t<_Float16>(forward, a, s);
    }
    return false;
}

}  // namespace

bool launch_rows_forward(wtconv_dtype dt, const NormArgs& a, hipStream_t s) { return launch(dt, true, a, s); }
bool launch_rows_backward(wtconv_dtype dt, const NormArgs& a, hipStream_t s) { return launch(dt, false, a, s); }

}  // namespace wtc
