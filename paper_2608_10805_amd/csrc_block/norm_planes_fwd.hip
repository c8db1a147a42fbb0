// Layer norm of planes, forward: one read and one write of every element.
#include "norm_planes.h"

namespace wtc {
namespace {

template <typename T, typename Sh, bool OUT_PLANES>
__global__ void __launch_bounds__(Sh::TH) planes_forward(const NormArgs a)
{
    constexpr int V = Sh::V, NS = Sh::NS, K = Sh::K, P = Sh::P;
    __shared__ float red[2][Sh::NW][P];
    __shared__ alignas(16) T turn[OUT_PLANES ? 1 : turn_elements<T, Sh>()];
    const int px = threadIdx.x % Sh::LP, slot = threadIdx.x / Sh::LP;
    const int64_t q0 = (int64_t)blockIdx.x * P, q = q0 + px * V;
    const bool in = q < a.N;  // (a vector lies within one image)
    const int64_t at = in ? pixel_at(a, q) : 0;
    const T* x = (const T*)a.x + at;
    float v[K][V], s[V] = {}, mean[V], rstd[V];
#pragma unroll
    for (int k = 0; k < K; ++k) {
        const int c = slot + k * NS;
        if (in && c < a.C) {
            load_pack<V>(x + c * a.S, v[k]);
        } else {
#pragma unroll
            for (int i = 0; i < V; ++i) v[k][i] = 0.f;
        }
    }
#pragma unroll
    for (int k = 0; k < K; ++k)
#pragma unroll
        for (int i = 0; i < V; ++i) s[i] += v[k][i];
    slot_sum<Sh>(s, red[0]);
    const float per = 1.0f / a.C;
#pragma unroll
    for (int i = 0; i < V; ++i) {
        mean[i] = s[i] * per;
        s[i] = 0.f;
    }
    // the variance from the centred values, which are at hand: no cancellation
#pragma unroll
    for (int k = 0; k < K; ++k)
        if (slot + k * NS < a.C)
#pragma unroll
            for (int i = 0; i < V; ++i) {
                v[k][i] -= mean[i];
                s[i] += v[k][i] * v[k][i];
            }
    slot_sum<Sh>(s, red[1]);
#pragma unroll
    for (int i = 0; i < V; ++i) rstd[i] = 1.0f / sqrtf(s[i] * per + a.eps);
    if (a.mean && in && slot == 0)
#pragma unroll
        for (int i = 0; i < V; ++i) {
            a.mean[q + i] = mean[i];
            a.rstd[q + i] = rstd[i];
        }
#pragma unroll
    for (int k = 0; k < K; ++k) {
        const int c = slot + k * NS;
        if (c < a.C) {
            const float w = a.w ? a.w[c] : 1.0f, b = a.b ? a.b[c] : 0.0f;
#pragma unroll
            for (int i = 0; i < V; ++i) v[k][i] = v[k][i] * rstd[i] * w + b;
        }
    }
    if constexpr (OUT_PLANES) {
        if (in)
#pragma unroll
            for (int k = 0; k < K; ++k) {
                const int c = slot + k * NS;
                if (c < a.C) store_pack<V>((T*)a.out + at + c * a.S, v[k]);
            }
    } else {
        constexpr int STEPS = turn_steps<T, Sh>(), ST = turn_stride<T>(STEPS * NS);
        const int rows = a.N - q0 < P ? (int)(a.N - q0) : P;
        T* y = (T*)a.out + q0 * a.C;
        const bool pairs = a.C % 2 == 0 && (uintptr_t)y % 4 == 0;
#pragma unroll
        for (int k0 = 0; k0 < K; k0 += STEPS) {
            if (k0 * NS >= a.C) break;
            if (k0) __syncthreads();
#pragma unroll
            for (int k = k0; k < k0 + STEPS && k < K; ++k) {
                const int c = slot + k * NS;
                if (in && c < a.C)
#pragma unroll
                    for (int i = 0; i < V; ++i) turn[(px * V + i) * ST + c - k0 * NS] = from_f32<T>(v[k][i]);
            }
            __syncthreads();
            const int left = a.C - k0 * NS, width = left < STEPS * NS ? left : STEPS * NS;
            turn_rows<true, Sh::TH>(y, a.C, turn, ST, rows, width, k0 * NS, pairs);
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
        const dim3 grid((unsigned)((a.N + Sh::P - 1) / Sh::P));
        if (d.out == WTCONV_PLANES)
            hipLaunchKernelGGL((planes_forward<T, Sh, true>), grid, dim3(Sh::TH), 0, s, a);
        else
            hipLaunchKernelGGL((planes_forward<T, Sh, false>), grid, dim3(Sh::TH), 0, s, a);
    });
    return true;
}

template <typename T>
bool launch_t(const wtconv_norm_desc& d, const NormArgs& a, hipStream_t s)
{
    // (y that is rows needs no alignment to vectors of pixels)
    NormArgs b = a;
    if (d.out == WTCONV_ROWS) b.out = nullptr;
    return planes_vector(b, sizeof(T), nullptr) == 4 ? launch_v<T, 4>(d, a, s) : launch_v<T, 1>(d, a, s);
}

}  // namespace

bool launch_planes_forward(const wtconv_norm_desc& d, const NormArgs& a, hipStream_t s)
{
    if (a.N > (int64_t)1 << 33) return false;  // workgroups of one launch
    switch (d.dtype) {
        case WTCONV_F32: return launch_t<float>(d, a, s);
        case WTCONV_BF16: return launch_t<uint16_t>(d, a, s);
        case WTCONV_F16: return launch_t<_Float16>(d, a, s);
    }
    return false;
}

}  // namespace wtc
