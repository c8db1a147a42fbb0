// Layer norm of rows with a row in the registers of a group of lanes, forward
// and backward: one read of every input, one write of every output.
//
// GL lanes (a power of two, up to a wavefront) hold a row: lane l the vectors
// l, l + GL, ... of V elements (16 bytes), at most R of them. 64 / GL rows a
// wavefront. WHOLE: C is a multiple of V; else the last vector is incomplete,
// and rows may begin at any element.
//
// Bound by memory where many rows are on their way (191520 rows of 96 float32
// channels: forward 34 us, 4.3 TB/s, backward 49 us, 4.5 TB/s). In 16 bits the
// latency of a row shows: a group of the forward pass takes one row, loads the
// weight and the bias after its sums and has nothing on its way meanwhile, and
// the sums over lanes and the conversions are as many as for twice the bytes (the
// same rows in bfloat16 23.7 us, 3.1 TB/s, and 37 us, 3.0 TB/s; 47880 rows of 127
// float16 channels 10.4 and 15.2 us, 2.3 TB/s, with incomplete vectors besides).
#include "norm_device.h"

namespace wtc {
namespace {

constexpr int kThreads = 256;

// The elements of a vector that there are: all of WHOLE rows' vectors up to C.
template <int V, bool WHOLE>
DEV int count_of(int c, int C) { return WHOLE ? (c < C ? V : 0) : C - c; }

template <int V>
DEV void load_columns(const float* p, int c, int n, float none, float (&f)[V])
{
#pragma unroll
    for (int i = 0; i < V; ++i) f[i] = none;
    if (!p) return;
    const Pack<float, V> q = load_upto<V>(p + c, n);
#pragma unroll
    for (int i = 0; i < V; ++i) f[i] = q.v[i];
}

template <typename T, int R, bool WHOLE>
__global__ void __launch_bounds__(kThreads) rows_forward(const NormArgs a, int gl)
{
    constexpr int V = 16 / sizeof(T);
    const int lane = threadIdx.x & (gl - 1);
    const int64_t q = (int64_t)blockIdx.x * (kThreads / gl) + threadIdx.x / gl;
    if (q >= a.N) return;  // (whole groups)
    const T* x = (const T*)a.x + q * a.x_stride;
    float v[R][V], s = 0.f;
#pragma unroll
    for (int r = 0; r < R; ++r) {
        const int c = (r * gl + lane) * V;
        const auto p = load_upto<V>(x + c, count_of<V, WHOLE>(c, a.C));
#pragma unroll
        for (int i = 0; i < V; ++i) v[r][i] = to_f32(p.v[i]);
    }
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
        for (int i = 0; i < V; ++i) s += v[r][i];
    const float per = 1.0f / a.C, mean = divided(sum_within(s, gl), (float)a.C, per);
    s = 0.f;
    // the variance from the centred values, which are at hand: no cancellation
#pragma unroll
    for (int r = 0; r < R; ++r) {
        const int n = count_of<V, WHOLE>((r * gl + lane) * V, a.C);
#pragma unroll
        for (int i = 0; i < V; ++i) {
            v[r][i] = i < n ? v[r][i] - mean : 0.f;
            s += v[r][i] * v[r][i];
        }
    }
    const float rstd = inverse_root(sum_within(s, gl) * per + a.eps);
    if (a.mean && lane == 0) {
        a.mean[q] = mean;
        a.rstd[q] = rstd;
    }
    T* y = (T*)a.out + q * a.C;
#pragma unroll
    for (int r = 0; r < R; ++r) {
        const int c = (r * gl + lane) * V, n = count_of<V, WHOLE>(c, a.C);
        float w[V], b[V];
        load_columns<V>(a.w, c, n, 1.0f, w);
        load_columns<V>(a.b, c, n, 0.0f, b);
        Pack<T, V> p;
#pragma unroll
        for (int i = 0; i < V; ++i) p.v[i] = from_f32<T>(v[r][i] * rstd * w[i] + b[i]);
        store_upto<V>(y + c, n, p);
    }
}

// A workgroup takes rows in steps of all workgroups' rows; each lane sums the
// gradients of its own columns, the groups and wavefronts join at the end.
template <typename T, int R, bool WHOLE>
__global__ void __launch_bounds__(kThreads) rows_backward(const NormArgs a, int gl)
{
    constexpr int V = 16 / sizeof(T);
    extern __shared__ float sums[];  // 2 C
    const int lane = threadIdx.x & (gl - 1), groups = kThreads / gl;
    const float per = 1.0f / a.C;
    float sw[R][V] = {}, sb[R][V] = {}, w[R][V];
#pragma unroll
    for (int r = 0; r < R; ++r) {
        const int c = (r * gl + lane) * V;
        load_columns<V>(a.w, c, count_of<V, WHOLE>(c, a.C), 1.0f, w[r]);
    }
    for (int64_t q = (int64_t)blockIdx.x * groups + threadIdx.x / gl; q < a.N; q += (int64_t)gridDim.x * groups) {
        const T* x = (const T*)a.x + q * a.x_stride;
        const T* dy = (const T*)a.dy + q * a.dy_stride;
        float xhat[R][V], g[R][V], s1 = 0.f, s2 = 0.f;
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const int c = (r * gl + lane) * V, n = count_of<V, WHOLE>(c, a.C);
            const auto px = load_upto<V>(x + c, n), pd = load_upto<V>(dy + c, n);
#pragma unroll
            for (int i = 0; i < V; ++i) {
                xhat[r][i] = to_f32(px.v[i]);
                g[r][i] = to_f32(pd.v[i]);  // (zero past C: nothing in any sum)
            }
        }
        const float mean = a.mean[q], rstd = a.rstd[q];
#pragma unroll
        for (int r = 0; r < R; ++r)
#pragma unroll
            for (int i = 0; i < V; ++i) {
                xhat[r][i] = (xhat[r][i] - mean) * rstd;
                sw[r][i] += g[r][i] * xhat[r][i];
                sb[r][i] += g[r][i];
                g[r][i] *= w[r][i];
                s1 += g[r][i];
                s2 += g[r][i] * xhat[r][i];
            }
        if (!a.out) continue;
        s1 = sum_within(s1, gl) * per * rstd;
        s2 = sum_within(s2, gl) * per * rstd;
        T* dx = (T*)a.out + q * a.C;
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const int c = (r * gl + lane) * V;
            Pack<T, V> p;
#pragma unroll
            for (int i = 0; i < V; ++i) p.v[i] = from_f32<T>(rstd * g[r][i] - s1 - xhat[r][i] * s2);
            store_upto<V>(dx + c, count_of<V, WHOLE>(c, a.C), p);
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

// Lanes a row and vectors a lane for n vectors. Forward: the fewest idle lanes,
// of those layouts the one with the most lanes (384 bfloat16 channels, 25088
// rows: 16 lanes of 3 vectors 13.0 us, 64 of 1, a quarter idle, 15.3). Backward:
// the most lanes, since every vector a lane holds has 2 V sums to join at the
// end (the same rows: 46.8 us with 3 vectors a lane, 26.8 with 1).
bool layout(int n, bool forward, int& gl, int& r)
{
    int best = 0;
    for (int t : {1, 2, 3, 4, 8}) {
        int lanes = 1;
        while (lanes * t < n) lanes *= 2;
        if (lanes > 64 || (best && (t > 4 || !forward))) continue;
        const int used = n * 1024 / (lanes * t);
        if (used <= best) continue;
        best = used;
        gl = lanes;
        r = t;
    }
    return best != 0;
}

template <typename T, int R, bool WHOLE>
bool launch_r(bool forward, const NormArgs& a, int gl, hipStream_t s)
{
    const int groups = kThreads / gl;
    if (forward && (a.N + groups - 1) / groups * kThreads >= kMaxThreads) return false;
    if (forward)
        hipLaunchKernelGGL((rows_forward<T, R, WHOLE>), dim3((unsigned)((a.N + groups - 1) / groups)), dim3(kThreads),
                           0, s, a, gl);
    else
        hipLaunchKernelGGL((rows_backward<T, R, WHOLE>), dim3(a.nparts), dim3(kThreads), (size_t)a.C * 8, s, a, gl);
    return true;
}

template <typename T, bool WHOLE>
bool launch_v(bool forward, const NormArgs& a, hipStream_t s)
{
    constexpr int V = 16 / sizeof(T);
    int gl = 0, r = 0;
    if (!layout((a.C + V - 1) / V, forward, gl, r)) return false;
    switch (r) {
        case 1: return launch_r<T, 1, WHOLE>(forward, a, gl, s);
        case 2: return launch_r<T, 2, WHOLE>(forward, a, gl, s);
        case 3: return launch_r<T, 3, WHOLE>(forward, a, gl, s);
        case 4: return launch_r<T, 4, WHOLE>(forward, a, gl, s);
        case 8: return launch_r<T, 8, WHOLE>(forward, a, gl, s);
    }
    return false;
}

template <typename T>
bool launch_t(bool forward, const NormArgs& a, hipStream_t s)
{
    return a.C % (16 / (int)sizeof(T)) == 0 ? launch_v<T, true>(forward, a, s) : launch_v<T, false>(forward, a, s);
}

bool launch(wtconv_dtype dt, bool forward, const NormArgs& a, hipStream_t s)
{
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
