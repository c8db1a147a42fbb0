// C entry points of the operators around the convolution: argument checks on
// the host, then the launches. Nothing is allocated and nothing is kept.
#include <cmath>
#include <cstdint>
#include <utility>

#include "block_internal.h"

namespace wtc {
namespace {

constexpr int64_t kMaxElements = (int64_t)1 << 46;  // far below where byte offsets pass 63 bits

size_t element_size(wtconv_dtype dt) { return dt == WTCONV_F32 ? 4 : 2; }

bool known(wtconv_dtype dt) { return dt == WTCONV_F32 || dt == WTCONV_BF16 || dt == WTCONV_F16; }

struct Range {
    uintptr_t begin, end;
    Range(const void* p, size_t bytes) : begin((uintptr_t)p), end(p ? (uintptr_t)p + bytes : (uintptr_t)p) {}
    bool meets(const Range& o) const { return begin < o.end && o.begin < end; }
};

template <size_t NOut, size_t NIn>
bool overlap(const Range (&out)[NOut], const Range (&in)[NIn])
{
    for (size_t i = 0; i < NOut; ++i) {
        for (const Range& r : in)
            if (out[i].meets(r)) return true;
        for (size_t j = i + 1; j < NOut; ++j)
            if (out[i].meets(out[j])) return true;
    }
    return false;
}

bool misaligned(const void* p, size_t a) { return (uintptr_t)p % a != 0; }

wtconv_status of(hipError_t e) { return e == hipSuccess ? WTCONV_OK : WTCONV_ERR_HIP; }

wtconv_status check_size(long long B, long long S, int C, wtconv_dtype dt)
{
    if (B < 0 || S < 0 || C < 1 || C > WTCONV_MAX_CHANNELS) return WTCONV_ERR_SHAPE;
    if (B && S > kMaxElements / B) return WTCONV_ERR_SHAPE;
    if (B * S > kMaxElements / C) return WTCONV_ERR_SHAPE;
    if (S > kMaxElements / C) return WTCONV_ERR_SHAPE;
    return known(dt) ? WTCONV_OK : WTCONV_ERR_DTYPE;
}

wtconv_status check(const wtconv_norm_desc* d)
{
    if (!d) return WTCONV_ERR_NULL;
    const wtconv_status st = check_size(d->B, d->S, d->C, d->dtype);
    if (st != WTCONV_OK) return st;
    const bool in_rows = d->in == WTCONV_ROWS, out_rows = d->out == WTCONV_ROWS;
    if ((!in_rows && d->in != WTCONV_PLANES) || (!out_rows && d->out != WTCONV_PLANES) || (in_rows && !out_rows))
        return WTCONV_ERR_UNSUPPORTED;
    for (const auto& [stride, rows] : {std::pair<long long, bool>{d->x_stride, in_rows}, {d->dy_stride, out_rows}}) {
        if (stride == 0) continue;
        if (!rows || stride < d->C) return WTCONV_ERR_SHAPE;
        if (d->B * d->S && stride > kMaxElements / (d->B * d->S)) return WTCONV_ERR_SHAPE;
    }
    if (!(d->eps >= 0) || !std::isfinite(d->eps)) return WTCONV_ERR_UNSUPPORTED;
    return WTCONV_OK;
}

wtconv_status check(const wtconv_residual_desc* d)
{
    return d ? check_size(d->B, d->S, d->C, d->dtype) : WTCONV_ERR_NULL;
}

// Bytes from the first element of N rows to the last's end.
size_t span(int64_t N, int C, long long stride, size_t e)
{
    return N ? ((size_t)(N - 1) * (stride ? stride : C) + C) * e : 0;
}

NormArgs norm_args(const wtconv_norm_desc& d)
{
    NormArgs a = {};
    a.B = d.B;
    a.S = d.S;
    a.N = d.B * d.S;
    a.C = d.C;
    a.x_stride = d.x_stride ? d.x_stride : d.C;
    a.dy_stride = d.dy_stride ? d.dy_stride : d.C;
    a.eps = (float)d.eps;
    return a;
}

}  // namespace
}  // namespace wtc

using namespace wtc;

extern "C" {

wtconv_status wtconv_layer_norm_forward(const wtconv_norm_desc* desc, const void* x, const float* weight,
                                        const float* bias, void* y, float* mean, float* rstd, hipStream_t stream)
{
    const wtconv_status st = check(desc);
    if (st != WTCONV_OK) return st;
    const int64_t N = desc->B * desc->S;
    if (N == 0) return WTCONV_OK;
    if (!x || !y || !mean != !rstd) return WTCONV_ERR_NULL;
    const size_t e = element_size(desc->dtype), c4 = (size_t)desc->C * 4, n4 = (size_t)N * 4;
    if (misaligned(x, e) || misaligned(y, e) || misaligned(weight, 4) || misaligned(bias, 4) ||
        misaligned(mean, 4) || misaligned(rstd, 4))
        return WTCONV_ERR_SHAPE;
    const Range in[] = {{x, span(N, desc->C, desc->x_stride, e)}, {weight, c4}, {bias, c4}};
    const Range out[] = {{y, span(N, desc->C, 0, e)}, {mean, n4}, {rstd, n4}};
    if (overlap(out, in)) return WTCONV_ERR_ALIAS;
    NormArgs a = norm_args(*desc);
    a.x = x;
    a.w = weight;
    a.b = bias;
    a.out = y;
    a.mean = mean;
    a.rstd = rstd;
    return of(launch_norm_forward(*desc, a, stream));
}

size_t wtconv_layer_norm_backward_workspace_bytes(const wtconv_norm_desc* desc)
{
    if (check(desc) != WTCONV_OK) return 0;
    return ((size_t)norm_parts(*desc) * 2 * desc->C * 4 + 255) & ~(size_t)255;
}

wtconv_status wtconv_layer_norm_backward(const wtconv_norm_desc* desc, const void* dy, const void* x,
                                         const float* mean, const float* rstd, const float* weight, void* dx,
                                         float* d_weight, float* d_bias, void* workspace, size_t workspace_bytes,
                                         hipStream_t stream)
{
    const wtconv_status st = check(desc);
    if (st != WTCONV_OK) return st;
    const int64_t N = desc->B * desc->S;
    const bool sums = d_weight || d_bias;
    if (!sums && (!dx || N == 0)) return WTCONV_OK;
    const size_t e = element_size(desc->dtype), c4 = (size_t)desc->C * 4, n4 = (size_t)N * 4;
    if (N && (!dy || !x || !mean || !rstd)) return WTCONV_ERR_NULL;
    if (misaligned(x, e) || misaligned(dy, e) || misaligned(dx, e) || misaligned(weight, 4) ||
        misaligned(mean, 4) || misaligned(rstd, 4) || misaligned(d_weight, 4) || misaligned(d_bias, 4))
        return WTCONV_ERR_SHAPE;
    const size_t need = sums ? wtconv_layer_norm_backward_workspace_bytes(desc) : 0;
    if (need && (!workspace || workspace_bytes < need || misaligned(workspace, 16))) return WTCONV_ERR_WORKSPACE;
    const Range in[] = {{x, span(N, desc->C, desc->x_stride, e)},
                        {dy, span(N, desc->C, desc->dy_stride, e)},
                        {mean, n4},
                        {rstd, n4},
                        {weight, c4}};
    const Range out[] = {{dx, span(N, desc->C, 0, e)}, {d_weight, c4}, {d_bias, c4}, {need ? workspace : nullptr, need}};
    if (overlap(out, in)) return WTCONV_ERR_ALIAS;
    NormArgs a = norm_args(*desc);
    a.x = x;
    a.dy = dy;
    a.w = weight;
    a.mean = const_cast<float*>(mean);
    a.rstd = const_cast<float*>(rstd);
    a.out = N ? dx : nullptr;
    a.part = need ? (float*)workspace : nullptr;
    a.nparts = (int)norm_parts(*desc);
    return of(launch_norm_backward(*desc, a, d_weight, d_bias, stream));
}

wtconv_status wtconv_scaled_residual_forward(const wtconv_residual_desc* desc, const void* x, const void* z,
                                             const float* gamma, const float* sample_scale, void* y,
                                             hipStream_t stream)
{
    const wtconv_status st = check(desc);
    if (st != WTCONV_OK) return st;
    const int64_t N = desc->B * desc->S;
    if (N == 0) return WTCONV_OK;
    if (!x || !z || !y) return WTCONV_ERR_NULL;
    const size_t e = element_size(desc->dtype), bytes = (size_t)N * desc->C * e;
    if (misaligned(x, e) || misaligned(z, e) || misaligned(y, e) || misaligned(gamma, 4) || misaligned(sample_scale, 4))
        return WTCONV_ERR_SHAPE;
    const Range in[] = {{x, bytes}, {z, bytes}, {gamma, (size_t)desc->C * 4}, {sample_scale, (size_t)desc->B * 4}};
    const Range out[] = {{y, bytes}};
    if (overlap(out, in)) return WTCONV_ERR_ALIAS;
    ResidualArgs a = {};
    a.x = x;
    a.z = z;
    a.gamma = gamma;
    a.keep = sample_scale;
    a.out = y;
    a.B = desc->B;
    a.S = desc->S;
    a.N = N;
    a.C = desc->C;
    return of(launch_residual_forward(desc->dtype, a, stream));
}

size_t wtconv_scaled_residual_backward_workspace_bytes(const wtconv_residual_desc* desc)
{
    if (check(desc) != WTCONV_OK) return 0;
    return ((size_t)residual_parts(*desc) * desc->C * 4 + 255) & ~(size_t)255;
}

wtconv_status wtconv_scaled_residual_backward(const wtconv_residual_desc* desc, const void* dy, const void* z,
                                              const float* gamma, const float* sample_scale, void* dz,
                                              float* d_gamma, void* workspace, size_t workspace_bytes,
                                              hipStream_t stream)
{
    const wtconv_status st = check(desc);
    if (st != WTCONV_OK) return st;
    const int64_t N = desc->B * desc->S;
    if (!d_gamma && (!dz || N == 0)) return WTCONV_OK;
    if (N && (!dy || (d_gamma && !z))) return WTCONV_ERR_NULL;
    const size_t e = element_size(desc->dtype), bytes = (size_t)N * desc->C * e, c4 = (size_t)desc->C * 4;
    if (misaligned(dy, e) || misaligned(z, e) || misaligned(dz, e) || misaligned(gamma, 4) ||
        misaligned(sample_scale, 4) || misaligned(d_gamma, 4))
        return WTCONV_ERR_SHAPE;
    const size_t need = d_gamma ? wtconv_scaled_residual_backward_workspace_bytes(desc) : 0;
    if (need && (!workspace || workspace_bytes < need || misaligned(workspace, 16))) return WTCONV_ERR_WORKSPACE;
    const Range in[] = {{dy, bytes}, {d_gamma ? z : nullptr, bytes}, {gamma, c4}, {sample_scale, (size_t)desc->B * 4}};
    const Range out[] = {{dz, bytes}, {d_gamma, c4}, {need ? workspace : nullptr, need}};
    if (overlap(out, in)) return WTCONV_ERR_ALIAS;
    ResidualArgs a = {};
    a.x = dy;
    a.z = z;
    a.gamma = gamma;
    a.keep = sample_scale;
    a.out = N ? dz : nullptr;
    a.part = need ? (float*)workspace : nullptr;
    a.B = desc->B;
    a.S = desc->S;
    a.N = N;
    a.C = desc->C;
    a.nparts = (int)residual_parts(*desc);
    return of(launch_residual_backward(desc->dtype, a, d_gamma, stream));
}

wtconv_status wtconv_adamw_step(int n_groups, const wtconv_adamw_group* groups, int n_tensors,
                                const wtconv_adamw_tensor* tensors, wtconv_dtype dtype, int state_bits,
                                const float* grad_scale, hipStream_t stream)
{
    if (n_groups < 0 || n_tensors < 0) return WTCONV_ERR_SHAPE;
    if (!known(dtype)) return WTCONV_ERR_DTYPE;
    if (state_bits != 8 && state_bits != 32) return WTCONV_ERR_UNSUPPORTED;
    if (n_tensors == 0) return WTCONV_OK;
    if (!groups || !tensors) return WTCONV_ERR_NULL;
    if (misaligned(grad_scale, 4)) return WTCONV_ERR_SHAPE;
    const bool coded = state_bits == 8;
    for (int i = 0; i < n_groups; ++i) {
        const wtconv_adamw_group& g = groups[i];
        if (!(g.lr >= 0) || !(g.eps >= 0) || !(g.weight_decay >= 0) || !(g.beta1 >= 0 && g.beta1 < 1) ||
            !(g.beta2 >= 0 && g.beta2 < 1) || !std::isfinite(g.lr) || !std::isfinite(g.eps) ||
            !std::isfinite(g.weight_decay) || g.step < 1)
            return WTCONV_ERR_UNSUPPORTED;
        if (!g.exp_avg || !g.exp_avg_sq || (coded && (!g.exp_avg_scale || !g.exp_avg_sq_scale)))
            return WTCONV_ERR_NULL;
        if (misaligned(g.exp_avg, 16) || misaligned(g.exp_avg_sq, 16)) return WTCONV_ERR_SHAPE;
    }
    const size_t e = element_size(dtype);
    const int64_t chunk = adam_chunk_elements(), most = adam_most_chunks();
    for (int i = 0; i < n_tensors; ++i) {
        const wtconv_adamw_tensor& t = tensors[i];
        if (t.numel < 0 || t.numel > kMaxElements || t.offset < 0 || t.offset > kMaxElements || t.offset % 64 ||
            t.group < 0 || t.group >= n_groups)
            return WTCONV_ERR_SHAPE;
        if (!t.numel) continue;
        if (!t.param || !t.grad) return WTCONV_ERR_NULL;
        if (misaligned(t.param, e) || misaligned(t.grad, e)) return WTCONV_ERR_SHAPE;
        if (Range(t.param, t.numel * e).meets(Range(t.grad, t.numel * e))) return WTCONV_ERR_ALIAS;
    }

    AdamArgs a;
    a.scale = grad_scale;
    int loaded[kAdamGroups];  // the group in each place of a.group
    int places = 0;
    a.count = 0;
    a.chunks = 0;
    auto flush = [&]() {
        const hipError_t err = a.count ? launch_adamw(dtype, state_bits, a, stream) : hipSuccess;
        a.count = places = 0;
        a.chunks = 0;
        return err;
    };
    for (int i = 0; i < n_tensors; ++i) {
        const wtconv_adamw_tensor& t = tensors[i];
        if (!t.numel) continue;
        // (a tensor of more chunks than one launch takes goes in pieces of whole chunks)
        for (int64_t done = 0; done < t.numel; done += most * chunk) {
            const int64_t numel = t.numel - done < most * chunk ? t.numel - done : most * chunk;
            const int64_t chunks = (numel + chunk - 1) / chunk;
            int place = 0;
            while (place < places && loaded[place] != t.group) ++place;
            if (a.count == kAdamTensors || place == kAdamGroups || a.chunks + chunks > most) {
                const hipError_t err = flush();
                if (err != hipSuccess) return WTCONV_ERR_HIP;
                place = 0;
            }
            if (place == places) {
                const wtconv_adamw_group& g = groups[t.group];
                AdamGroup& o = a.group[place];
                o.m = g.exp_avg;
                o.v = g.exp_avg_sq;
                o.ms = g.exp_avg_scale;
                o.vs = g.exp_avg_sq_scale;
                o.b1 = (float)g.beta1;
                o.omb1 = (float)(1 - g.beta1);
                o.b2 = (float)g.beta2;
                o.omb2 = (float)(1 - g.beta2);
                o.rcorr2 = (float)(1 / std::sqrt(1 - std::pow(g.beta2, (double)g.step)));
                o.eps = (float)g.eps;
                o.keep = (float)(1 - g.lr * g.weight_decay);
                o.rate = (float)(g.lr / (1 - std::pow(g.beta1, (double)g.step)));
                o.key = g.key;
                loaded[places++] = t.group;
            }
            a.p[a.count] = (char*)t.param + done * e;
            a.g[a.count] = (const char*)t.grad + done * e;
            a.n[a.count] = numel;
            a.at[a.count] = t.offset + done;
            a.first[a.count] = a.chunks;
            a.of[a.count] = (uint8_t)place;
            a.chunks += (uint32_t)chunks;
            ++a.count;
        }
    }
    return of(flush());
}

wtconv_status wtconv_adamw_moments(long long n, const unsigned char* exp_avg, const unsigned char* exp_avg_scale,
                                   const unsigned char* exp_avg_sq, const unsigned char* exp_avg_sq_scale, void* m,
                                   void* v, wtconv_dtype dtype, hipStream_t stream)
{
    if (n < 0 || n > kMaxElements || n % 64) return WTCONV_ERR_SHAPE;
    if (!known(dtype)) return WTCONV_ERR_DTYPE;
    if (n == 0) return WTCONV_OK;
    if (!exp_avg || !exp_avg_scale || !exp_avg_sq || !exp_avg_sq_scale || !m || !v) return WTCONV_ERR_NULL;
    if (misaligned(exp_avg, 16) || misaligned(exp_avg_sq, 16) || misaligned(m, 16) || misaligned(v, 16))
        return WTCONV_ERR_SHAPE;
    const size_t e = element_size(dtype);
    const Range in[] = {{exp_avg, (size_t)n}, {exp_avg_scale, (size_t)n / 64}, {exp_avg_sq, (size_t)n},
                        {exp_avg_sq_scale, (size_t)n / 64}};
    const Range out[] = {{m, n * e}, {v, n * e}};
    if (overlap(out, in)) return WTCONV_ERR_ALIAS;
    return of(launch_adamw_moments(dtype, n, exp_avg, exp_avg_scale, exp_avg_sq, exp_avg_sq_scale, m, v, stream));
}

}  // extern "C"
