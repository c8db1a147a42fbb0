// Layer norm of planes, backward: one read of x and dy, one write of dx, and
// the weight's and bias's gradients in registers over all of a workgroup's
// tiles.
#include "norm_planes.h"

namespace wtc {
namespace {

template <typename T, typename Sh, bool OUT_PLANES>
__global__ void __launch_bounds__(Sh::TH) planes_backward(const NormArgs a)
{
    constexpr int V = Sh::V, NS = Sh::NS, K = Sh::K, P = Sh::P;
    __shared__ float red[2][Sh::NW][P];
    __shared__ alignas(16) T turn[OUT_PLANES ? 1 : turn_elements<T, Sh>()];
    const int px = threadIdx.x % Sh::LP, slot = threadIdx.x / Sh::LP;
    const float per = 1.0f / a.C;
    float sw[K] = {}, sb[K] = {};
    for (int64_t q0 = (int64_t)blockIdx.x * P; q0 < a.N; q0 += (int64_t)gridDim.x * P) {
        const int64_t q = q0 + px * V;
        const bool in = q < a.N;
        const int64_t at = in ? pixel_at(a, q) : 0;
        const T* x = (const T*)a.x + at;
        float xhat[K][V], g[K][V], s1[V] = {}, s2[V] = {}, rstd[V];
#pragma unroll
        for (int k = 0; k < K; ++k) {
            const int c = slot + k * NS;
            if (in && c < a.C) {
                load_pack<V>(x + c * a.S, xhat[k]);
                if (OUT_PLANES) load_pack<V>((const T*)a.dy + at + c * a.S, g[k]);
            } else {
#pragma unroll
                for (int i = 0; i < V; ++i) xhat[k][i] = g[k][i] = 0.f;
            }
        }
        if constexpr (!OUT_PLANES) {
            constexpr int STEPS = turn_steps<T, Sh>(), ST = turn_stride<T>(STEPS * NS);
            const int rows = a.N - q0 < P ? (int)(a.N - q0) : P;
            const T* dy = (const T*)a.dy + q0 * a.dy_stride;
            const bool pairs = a.C % 2 == 0 && a.dy_stride % 2 == 0 && (uintptr_t)dy % 4 == 0;
#pragma unroll
            for (int k0 = 0; k0 < K; k0 += STEPS) {
                if (k0 * NS >= a.C) break;
                const int left = a.C - k0 * NS, width = left < STEPS * NS ? left : STEPS * NS;
                __syncthreads();
                turn_rows<false, Sh::TH>(dy, a.dy_stride, turn, ST, rows, width, k0 * NS, pairs);
                __syncthreads();
#pragma unroll
                for (int k = k0; k < k0 + STEPS && k < K; ++k) {
                    const int c = slot + k * NS;
                    if (in && c < a.C)
#pragma unroll
                        for (int i = 0; i < V; ++i) g[k][i] = to_f32(turn[(px * V + i) * ST + c - k0 * NS]);
                }
            }
        }
        if (in) {
            float mean[V];
#pragma unroll
            for (int i = 0; i < V; ++i) {
                mean[i] = a.mean[q + i];
                rstd[i] = a.rstd[q + i];
            }
#pragma unroll
            for (int k = 0; k < K; ++k) {
                const int c = slot + k * NS;
                if (c < a.C) {
                    const float w = a.w ? a.w[c] : 1.0f;
#pragma unroll
                    for (int i = 0; i < V; ++i) {
                        xhat[k][i] = (xhat[k][i] - mean[i]) * rstd[i];
                        sw[k] += g[k][i] * xhat[k][i];
                        sb[k] += g[k][i];
                        g[k][i] *= w;
                        s1[i] += g[k][i];
                        s2[i] += g[k][i] * xhat[k][i];
                    }
                }
            }
        }
        if (!a.out) continue;
        __syncthreads();  // the last tile's sums have been read
        slot_sum<Sh>(s1, red[0]);
        slot_sum<Sh>(s2, red[1]);
        if (in)
#pragma unroll
            for (int k = 0; k < K; ++k) {
                const int c = slot + k * NS;
                if (c < a.C) {
#pragma unroll
                    for (int i = 0; i < V; ++i) g[k][i] = rstd[i] * (g[k][i] - s1[i] * per - xhat[k][i] * (s2[i] * per));
                    store_pack<V>((T*)a.out + at + c * a.S, g[k]);
                }
            }
    }
    if (!a.part) return;
    float* part = a.part + (int64_t)blockIdx.x * 2 * a.C;
#pragma unroll
    for (int k = 0; k < K; ++k) {
        const int c = slot + k * NS;
#pragma unroll
        for (int o = Sh::LP >> 1; o; o >>= 1) {
            sw[k] += __shfl_xor(sw[k], o);
            sb[k] += __shfl_xor(sb[k], o);
        }
        if (px == 0 && c < a.C) {
            part[c] = sw[k];
            part[a.C + c] = sb[k];
        }
    }
}

template <typename T, int V>
bool launch_v(const wtconv_norm_desc& d, const NormArgs& a, hipStream_t s)
{
    const int i = pick_planes<V>(a.C, a.N);
    if (i < 0) return false;
    planes_shape<V>(i, [&](auto sh) {
        using Sh = decltype(sh);
        const dim3 grid(a.nparts);
        if (d.out == WTCONV_PLANES)
            hipLaunchKernelGGL((planes_backward<T, Sh, true>), grid, dim3(Sh::TH), 0, s, a);
        else
            hipLaunchKernelGGL((planes_backward<T, Sh, false>), grid, dim3(Sh::TH), 0, s, a);
    });
    return true;
}

template <typename T>
bool launch_t(const wtconv_norm_desc& d, const NormArgs& a, hipStream_t s)
{
    const void* dy = d.out == WTCONV_PLANES ? a.dy : nullptr;
    return planes_vector(a, sizeof(T), dy) == 4 ? launch_v<T, 4>(d, a, s) : launch_v<T, 1>(d, a, s);
}

}  // namespace

bool launch_planes_backward(const wtconv_norm_desc& d, const NormArgs& a, hipStream_t s)
{
    switch (d.dtype) {
        case WTCONV_F32: return launch_t<float>(d, a, s);
        case WTCONV_BF16: return launch_t<uint16_t>(d, a, s);
        case WTCONV_F16: return launch_t<_Float16>(d, a, s);
    }
    return false;
}

}  // namespace wtc
