// AdamW over many tensors, with moments in 32 or 8 bits: one read and one write
// of every parameter and moment, one read of every gradient.
//
// A workgroup takes one chunk of one tensor; which, its wavefronts find among
// the launch's tensors with one load and a vote (a search by halves cost seven
// loads one after the other: launches of small tensors 7.5 us, now 5.4). Chunks
// of 2048 elements: with 8192, 20 million elements gave some CUs five workgroups
// and others four.
//
// Bound by memory with 32-bit moments: 39 million float32 elements 206 us, 5.3
// TB/s of 28 bytes an element, what a large copy reaches; 20 million bfloat16 ones
// 90 us, 4.9 TB/s of 22 bytes. With 8-bit moments (16.06 bytes) 20 million float32
// elements take 64 us, 5.0 TB/s; bfloat16 parameters (10.06 bytes) 51 to 59 us, 3.4
// to 3.9 TB/s, bound by the arithmetic of the codes (303 vector instructions in the
// loop over four elements, the branches that few take among them).
#include "norm_device.h"

namespace wtc {
namespace {

constexpr int kThreads = 256, kVec = 4;
constexpr int kChunk = 2 * kThreads * kVec;  // elements of one workgroup
constexpr int kMTop = 14, kVTop = 30;        // exponent field of a block's largest moment

// 32 random bits for an element's place under a key: a golden-ratio step from
// place to place (2^32 / 1.618, as a prime), then the shifts and multipliers of
// a published 32-bit hash's last mixing (A. Appleby, public domain).
DEV uint32_t random_bits(uint32_t place, uint32_t key)
{
    uint32_t x = place * 0x9E3779B1u + key;
    x = (x ^ (x >> 15)) * 0x85EBCA6Bu;
    x = (x ^ (x >> 13)) * 0xC2B2AE35u;
    return x ^ (x >> 16);
}

// The values that four codes stand for under their block's scale: the float that
// has a code's exponent and mantissa bits below its sign, times 2^(scale - top);
// NaN under scale 255.
template <bool SIGNED>
DEV void decode(uint32_t codes, int scale, float (&f)[kVec])
{
    const uint32_t nan = scale == 255 ? 0x7fc00000u : 0u;
#pragma unroll
    for (int i = 0; i < kVec; ++i) {
        // (a signed code is extended to all bits above it and loses what lies between)
        const uint32_t bits = SIGNED ? ((uint32_t)(int8_t)(codes >> (8 * i)) << 20 & 0x87f00000u) | nan
                                     : ((codes >> (8 * i)) & 0xffu) << 20 | nan;
        f[i] = __builtin_ldexpf(__uint_as_float(bits), scale - (SIGNED ? kMTop : kVTop));
    }
}

// The codes of four values under their block's scale: 20 mantissa bits are
// dropped after `rest` was added to them. Zero under scale 255. A second moment
// that is not zero gets at least the first code: rounded to zero beside a first
// moment that was rounded up, the next step would divide by the root of nearly
// nothing (gradients of five decades in a block: updates of 700 times the rate,
// now at most 1.8 times). The first code's root is the smallest step of m, in
// units of their largest.
template <bool SIGNED>
DEV uint32_t encode(const float (&f)[kVec], int scale, const uint32_t (&rest)[kVec])
{
    uint32_t c[kVec];
#pragma unroll
    for (int i = 0; i < kVec; ++i) {
        c[i] = (__float_as_uint(__builtin_ldexpf(f[i], (SIGNED ? kMTop : kVTop) - scale)) + rest[i]) >> 20;
        if (SIGNED) {
            c[i] |= c[i] >> 4 & 0x80u;  // the sign, 11 bits up
        } else {
            const uint32_t least = f[i] > 0.f;
            c[i] = c[i] > least ? c[i] : least;
        }
    }
    // the lowest bytes
    const uint32_t low = __builtin_amdgcn_perm(c[1], c[0], 0x0c0c0400u), high = __builtin_amdgcn_perm(c[3], c[2], 0x04000c0cu);
    return scale == 255 ? 0u : low | high;
}

// The biased exponent of the largest magnitude of the 16 lanes' (64 values'), 255
// if one is not finite.
template <bool SIGNED>
DEV int block_scale(const float (&f)[kVec])
{
    uint32_t v = 0;
    const auto larger = [&v](uint32_t u) ALWAYS { v = u > v ? u : v; };
#pragma unroll
    for (int i = 0; i < kVec; ++i) larger(__float_as_uint(f[i]) & (SIGNED ? 0x7fffffffu : 0xffffffffu));
    larger(__float_as_uint(from_lane<0x128>(__uint_as_float(v))));
    larger(__float_as_uint(from_lane<0x124>(__uint_as_float(v))));
    larger(__float_as_uint(from_lane<0x122>(__uint_as_float(v))));
    larger(__float_as_uint(from_lane<0x121>(__uint_as_float(v))));
    return (int)(v >> 23 & 0xffu);  // (a NaN's sign is no part of it)
}

// The tensor that this workgroup's chunk is of.
DEV int find_tensor(const AdamArgs& a)
{
    const int lane = threadIdx.x & 63;
    int t = -1;
#pragma unroll
    for (int i = 0; i < (kAdamTensors + 63) / 64; ++i) {
        const int j = i * 64 + lane;
        t += __popcll(__ballot(j < a.count && a.first[j < kAdamTensors ? j : 0] <= blockIdx.x));
    }
    return __builtin_amdgcn_readfirstlane(t);
}

// An address for every lane as bytes from one for the workgroup.
template <typename E>
DEV E* at_bytes(E* p, uint32_t bytes)
{
    using B = std::conditional_t<std::is_const_v<E>, const char, char>;
    return reinterpret_cast<E*>(reinterpret_cast<B*>(p) + bytes);
}

template <typename T, bool CODED>
__global__ void __launch_bounds__(kThreads) adamw_kernel(const AdamArgs a)
{
    const int t = find_tensor(a);
    const AdamGroup& h = a.group[a.of[t]];
    const int64_t n = a.n[t], e0 = (int64_t)(blockIdx.x - a.first[t]) * kChunk, at0 = a.at[t] + e0;
    T* p = (T*)a.p[t] + e0;
    const T* g = (const T*)a.g[t] + e0;
    using M = std::conditional_t<CODED, uint8_t, float>;
    M *hm = (M*)h.m + at0, *hv = (M*)h.v + at0;
    uint8_t *hms = h.ms + (at0 >> 6), *hvs = h.vs + (at0 >> 6);
    const float gscale = a.scale ? *a.scale : 1.0f;
    const int end = n - e0 < kChunk ? (int)(n - e0) : kChunk;
    // (lanes of one block of 64 elements go on or stop together; past a tensor's
    // end its last block has zeros, which stay zeros)
    const uint32_t stop = CODED ? (end + 63) & ~63 : end;
    for (uint32_t c = threadIdx.x * kVec; c < stop; c += kThreads * kVec) {
        const int left = end - (int)c;
        auto pp = load_upto<kVec>(at_bytes(p, c * sizeof(T)), left);
        const auto pg = load_upto<kVec>(at_bytes(g, c * sizeof(T)), left);
        float m[kVec], v[kVec];
        if constexpr (CODED) {
            const uint32_t mc = *(const uint32_t*)at_bytes(hm, c), vc = *(const uint32_t*)at_bytes(hv, c);
            decode<true>(mc, *at_bytes(hms, c >> 6), m);
            decode<false>(vc, *at_bytes(hvs, c >> 6), v);
        } else {
            const auto pm = load_upto<kVec>(at_bytes(hm, c * 4), left), pv = load_upto<kVec>(at_bytes(hv, c * 4), left);
#pragma unroll
            for (int i = 0; i < kVec; ++i) {
                m[i] = pm.v[i];
                v[i] = pv.v[i];
            }
        }
#pragma unroll
        for (int i = 0; i < kVec; ++i) {
            const float gr = to_f32(pg.v[i]) * gscale;
            {
                // each product and sum rounded by itself, so that a moment's rounding to a code is reproducible
#pragma clang fp contract(off)
                m[i] = m[i] * h.b1 + gr * h.omb1;
                v[i] = v[i] * h.b2 + gr * gr * h.omb2;
            }
        }
        // square root and reciprocal to one unit in the last place: the update is far below the parameter
        float root[kVec];
        // the hardware's root of a subnormal is zero; what it should be, up to 2^-63, is less than a rounding beside
        // all but the smallest eps
        if (h.eps < 0x1p-38f * h.rcorr2) {
            asm volatile("");  // (keeps this a branch: else both sides are computed)
#pragma unroll
            for (int i = 0; i < kVec; ++i)
                root[i] = v[i] < 0x1p-96f ? __builtin_amdgcn_sqrtf(v[i] * 0x1p64f) * 0x1p-32f : __builtin_amdgcn_sqrtf(v[i]);
        } else {
#pragma unroll
            for (int i = 0; i < kVec; ++i) root[i] = __builtin_amdgcn_sqrtf(v[i]);
        }
#pragma unroll
        for (int i = 0; i < kVec; ++i) {
            const float denom = root[i] * h.rcorr2 + h.eps;
            pp.v[i] = from_f32<T>(to_f32(pp.v[i]) * h.keep - m[i] * __builtin_amdgcn_rcpf(denom) * h.rate);
        }
        store_upto<kVec>(at_bytes(p, c * sizeof(T)), left, pp);
        if constexpr (CODED) {
            const int ms = block_scale<true>(m), vs = block_scale<false>(v);
            uint32_t rm[kVec], rv[kVec];
            // from the 2^32nd place on, which four places side by side do not cross, under a key of their own
            const uint64_t place = (uint64_t)at0 + c;
            const uint32_t high = (uint32_t)(place >> 32), key = high ? random_bits(high, h.key) : h.key;
#pragma unroll
            for (int i = 0; i < kVec; ++i) {
                const uint32_t r = random_bits((uint32_t)place + i, key);
                rm[i] = (r << 4 & 0xffff0u) | 8;
                rv[i] = (r >> 12 & 0xffff0u) | 8;
            }
            *(uint32_t*)at_bytes(hm, c) = encode<true>(m, ms, rm);
            *(uint32_t*)at_bytes(hv, c) = encode<false>(v, vs, rv);
            if ((threadIdx.x & 15) == 0) {
                *at_bytes(hms, c >> 6) = (uint8_t)ms;
                *at_bytes(hvs, c >> 6) = (uint8_t)vs;
            }
        } else {
            store_upto<kVec>(at_bytes(hm, c * 4), left, Pack<float, kVec>{{m[0], m[1], m[2], m[3]}});
            store_upto<kVec>(at_bytes(hv, c * 4), left, Pack<float, kVec>{{v[0], v[1], v[2], v[3]}});
        }
    }
}

template <typename T>
__global__ void __launch_bounds__(kThreads)
moments_kernel(int64_t n, const uint8_t* m, const uint8_t* ms, const uint8_t* v, const uint8_t* vs, T* om, T* ov)
{
    for (int64_t e = ((int64_t)blockIdx.x * kThreads + threadIdx.x) * kVec; e < n;
         e += (int64_t)gridDim.x * kThreads * kVec) {
        float dm[kVec], dv[kVec];
        decode<true>(*(const uint32_t*)(m + e), ms[e >> 6], dm);
        decode<false>(*(const uint32_t*)(v + e), vs[e >> 6], dv);
        Pack<T, kVec> pm, pv;
#pragma unroll
        for (int i = 0; i < kVec; ++i) {
            pm.v[i] = from_f32<T>(dm[i]);
            pv.v[i] = from_f32<T>(dv[i]);
        }
        store_pack<kVec>(om + e, pm);
        store_pack<kVec>(ov + e, pv);
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
int64_t adam_most_chunks() { return kMaxThreads / kThreads - 1; }

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
