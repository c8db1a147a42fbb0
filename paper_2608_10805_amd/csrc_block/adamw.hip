// AdamW over many tensors, with moments in 32 or 8 bits.
#include "block_internal.h"
#include "wtconv_device.h"

namespace wtc {
namespace {

constexpr int kThreads = 256, kVec = 4;
constexpr int kChunk = 8 * kThreads * kVec;  // elements of one workgroup
constexpr int kMTop = 14, kVTop = 30;        // exponent field of a block's largest moment

// 32 random bits for an element's place under a key.
DEV uint32_t random_bits(uint32_t place, uint32_t key)
{
    uint32_t x = place * 0x9E3779B1u + key;
    x = (x ^ (x >> 15)) * 0x85EBCA6Bu;
    x = (x ^ (x >> 13)) * 0xC2B2AE35u;
    return x ^ (x >> 16);
}

// The largest of the 16 lanes that hold a block of 64 elements.
DEV uint32_t block_max(uint32_t v)
{
#pragma unroll
    for (int o = 8; o; o >>= 1) {
        const uint32_t u = __shfl_xor(v, o);
        v = u > v ? u : v;
    }
    return v;
}

// The value that a code's low bits stand for under its block's scale.
DEV float decode(uint32_t code, int scale, int top)
{
    const float v = __builtin_ldexpf(__uint_as_float(code << 20), scale - top);
    return scale == 255 ? __uint_as_float(0x7fc00000u) : v;
}

// The code's low bits of a magnitude under its block's scale.
DEV uint32_t encode(float mag, int scale, int top, uint32_t rest)
{
    return (__float_as_uint(__builtin_ldexpf(mag, top - scale)) + rest) >> 20;
}

template <typename T>
DEV void load_vec(const T* p, int64_t left, bool whole, float (&v)[kVec])
{
    if (whole) {
        struct alignas(sizeof(T) * kVec) Pack { T v[kVec]; };
        const Pack q = *reinterpret_cast<const Pack*>(p);
#pragma unroll
        for (int i = 0; i < kVec; ++i) v[i] = to_f32(q.v[i]);
    } else {
#pragma unroll
        for (int i = 0; i < kVec; ++i) v[i] = i < left ? to_f32(p[i]) : 0.f;
    }
}

template <typename T>
DEV void store_vec(T* p, int64_t left, bool whole, const float (&v)[kVec])
{
    if (whole) {
        struct alignas(sizeof(T) * kVec) Pack { T v[kVec]; } q;
#pragma unroll
        for (int i = 0; i < kVec; ++i) q.v[i] = from_f32<T>(v[i]);
        *reinterpret_cast<Pack*>(p) = q;
    } else {
#pragma unroll
        for (int i = 0; i < kVec; ++i)
            if (i < left) p[i] = from_f32<T>(v[i]);
    }
}

template <typename T, bool CODED>
__global__ void __launch_bounds__(kThreads) adamw_kernel(const AdamArgs a)
{
    int t = 0;
    for (int lo = 1, hi = a.count; lo < hi;) {  // the last tensor whose first chunk is not after this one
        const int mid = (lo + hi) >> 1;
        if (a.first[mid] <= blockIdx.x) {
            t = mid;
            lo = mid + 1;
        } else {
            hi = mid;
        }
    }
    const AdamGroup& h = a.group[a.of[t]];
    const int64_t n = a.n[t], e0 = (int64_t)(blockIdx.x - a.first[t]) * kChunk;
    T* p = (T*)a.p[t];
    const T* g = (const T*)a.g[t];
    const float gscale = a.scale ? *a.scale : 1.0f;
    const bool aligned = ((uintptr_t)p | (uintptr_t)g) % (sizeof(T) * kVec) == 0;
    for (int64_t e = e0 + threadIdx.x * kVec; e < e0 + kChunk && (e & ~(int64_t)63) < n; e += kThreads * kVec) {
        const int64_t left = n - e, at = a.at[t] + e;
        const bool whole = aligned && left >= kVec;
        float pv[kVec], gv[kVec], m[kVec], v[kVec];
        load_vec(p + e, left, whole, pv);
        load_vec(g + e, left, whole, gv);
        if (CODED) {
            const uint32_t mc = *(const uint32_t*)((const uint8_t*)h.m + at);
            const uint32_t vc = *(const uint32_t*)((const uint8_t*)h.v + at);
            const int ms = h.ms[at >> 6], vs = h.vs[at >> 6];
#pragma unroll
            for (int i = 0; i < kVec; ++i) {
                const uint32_t c = (mc >> (8 * i)) & 0xff;
                const float d = decode(c & 0x7f, ms, kMTop);
                m[i] = i < left ? (c & 0x80 ? -d : d) : 0.f;
                v[i] = i < left ? decode((vc >> (8 * i)) & 0xff, vs, kVTop) : 0.f;
            }
        } else {
            load_vec((const float*)h.m + at, left, left >= kVec, m);
            load_vec((const float*)h.v + at, left, left >= kVec, v);
        }
#pragma unroll
        for (int i = 0; i < kVec; ++i) {
            // each product and sum rounded by itself, so that a moment's rounding to a code is reproducible
#pragma clang fp contract(off)
            const float gr = gv[i] * gscale;
            m[i] = m[i] * h.b1 + gr * h.omb1;
            v[i] = v[i] * h.b2 + gr * gr * h.omb2;
            pv[i] = pv[i] * h.keep - m[i] / (sqrtf(v[i]) * h.rcorr2 + h.eps) * h.rate;
        }
        store_vec(p + e, left, whole, pv);
        if (CODED) {
            uint32_t bm = 0, bv = 0;
#pragma unroll
            for (int i = 0; i < kVec; ++i) {
                const uint32_t um = __float_as_uint(m[i]) & 0x7fffffffu, uv = __float_as_uint(v[i]) & 0x7fffffffu;
                bm = um > bm ? um : bm;
                bv = uv > bv ? uv : bv;
            }
            const int ms = block_max(bm) >> 23, vs = block_max(bv) >> 23;
            uint32_t mc = 0, vc = 0;
            const uint32_t key = h.key + (uint32_t)((uint64_t)at >> 32) * 0x9E3779B1u;
#pragma unroll
            for (int i = 0; i < kVec; ++i) {
                const uint32_t r = random_bits((uint32_t)at + i, key);
                uint32_t c = encode(fabsf(m[i]), ms, kMTop, (r & 0xffffu) << 4 | 8) | (__float_as_uint(m[i]) >> 31) << 7;
                mc |= (ms == 255 ? 0 : c) << (8 * i);
                c = encode(v[i], vs, kVTop, (r >> 16) << 4 | 8);
                vc |= (vs == 255 ? 0 : c) << (8 * i);
            }
            *(uint32_t*)((uint8_t*)h.m + at) = mc;
            *(uint32_t*)((uint8_t*)h.v + at) = vc;
            if ((threadIdx.x & 15) == 0) {
                h.ms[at >> 6] = (uint8_t)ms;
                h.vs[at >> 6] = (uint8_t)vs;
            }
        } else {
            store_vec((float*)h.m + at, left, left >= kVec, m);
            store_vec((float*)h.v + at, left, left >= kVec, v);
        }
    }
}

template <typename T>
__global__ void __launch_bounds__(kThreads)
moments_kernel(int64_t n, const uint8_t* m, const uint8_t* ms, const uint8_t* v, const uint8_t* vs, T* om, T* ov)
{
    for (int64_t e = ((int64_t)blockIdx.x * kThreads + threadIdx.x) * kVec; e < n;
         e += (int64_t)gridDim.x * kThreads * kVec) {
        const uint32_t mc = *(const uint32_t*)(m + e), vc = *(const uint32_t*)(v + e);
        const int sm = ms[e >> 6], sv = vs[e >> 6];
        float dm[kVec], dv[kVec];
#pragma unroll
        for (int i = 0; i < kVec; ++i) {
            const uint32_t c = (mc >> (8 * i)) & 0xff;
            const float d = decode(c & 0x7f, sm, kMTop);
            dm[i] = c & 0x80 ? -d : d;
            dv[i] = decode((vc >> (8 * i)) & 0xff, sv, kVTop);
        }
        store_vec(om + e, kVec, true, dm);
        store_vec(ov + e, kVec, true, dv);
    }
}

template <typename T>
hipError_t step_t(int bits, const AdamArgs& a, hipStream_t s)
{
    if (bits == 8)
        hipLaunchKernelGGL((adamw_kernel<T, true>), dim3(a.chunks), dim3(kThreads), 0, s, a);
    else
        hipLaunchKernelGGL((adamw_kernel<T, false>), dim3(a.chunks), dim3(kThreads), 0, s, a);
    return hipGetLastError();
}

template <typename T>
hipError_t moments_t(int64_t n, const uint8_t* m, const uint8_t* ms, const uint8_t* v, const uint8_t* vs, void* om,
                     void* ov, hipStream_t s)
{
    const int64_t blocks = (n / kVec + kThreads - 1) / kThreads;
    const int grid = (int)(blocks < (1 << 20) ? blocks : (1 << 20));
    hipLaunchKernelGGL(moments_kernel<T>, dim3(grid), dim3(kThreads), 0, s, n, m, ms, v, vs, (T*)om, (T*)ov);
    return hipGetLastError();
}

}  // namespace

int64_t adam_chunk_elements() { return kChunk; }

hipError_t launch_adamw(wtconv_dtype dt, int bits, const AdamArgs& a, hipStream_t s)
{
    switch (dt) {
        case WTCONV_F32: return step_t<float>(bits, a, s);
        case WTCONV_BF16: return step_t<uint16_t>(bits, a, s);
        case WTCONV_F16: return step_t<_Float16>(bits, a, s);
    }
    return hipErrorInvalidValue;
}

hipError_t launch_adamw_moments(wtconv_dtype dt, int64_t n, const uint8_t* m, const uint8_t* ms, const uint8_t* v,
                                const uint8_t* vs, void* om, void* ov, hipStream_t s)
{
    switch (dt) {
        case WTCONV_F32: return moments_t<float>(n, m, ms, v, vs, om, ov, s);
        case WTCONV_BF16: return moments_t<uint16_t>(n, m, ms, v, vs, om, ov, s);
        case WTCONV_F16: return moments_t<_Float16>(n, m, ms, v, vs, om, ov, s);
    }
    return hipErrorInvalidValue;
}

}  // namespace wtc
