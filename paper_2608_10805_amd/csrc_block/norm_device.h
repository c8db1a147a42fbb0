// What the kernels share: vectors of the storage types and sums over lanes.
#pragma once

#include "block_internal.h"
#include "wtconv_device.h"

namespace wtc {

#define ALWAYS __attribute__((always_inline))  // (of lambdas: what they capture stays in registers)

// V elements. In memory they need no more than an element's alignment: the
// copies below become whole vector loads and stores, which the hardware takes
// from any address.
template <typename T, int V>
struct alignas(sizeof(T) * V) Pack {
    T v[V];
};

template <int V, typename T>
DEV Pack<T, V> load_pack(const T* p)
{
    Pack<T, V> q;
    __builtin_memcpy(&q, p, sizeof(q));
    return q;
}

template <int V, typename T>
DEV void store_pack(T* p, const Pack<T, V>& q) { __builtin_memcpy(p, &q, sizeof(q)); }

// The first n elements alone, zeros after them.
template <int V, typename T>
DEV Pack<T, V> load_upto(const T* p, int n)
{
    Pack<T, V> q;
    if (n >= V) {
        q = load_pack<V>(p);
    } else {
#pragma unroll
        for (int i = 0; i < V; ++i) q.v[i] = i < n ? p[i] : T(0);
    }
    return q;
}

template <int V, typename T>
DEV void store_upto(T* p, int n, const Pack<T, V>& q)
{
    if (n >= V) {
        store_pack<V>(p, q);
    } else {
#pragma unroll
        for (int i = 0; i < V; ++i)
            if (i < n) p[i] = q.v[i];
    }
}

// Value of the lane that the DPP control names (within 16 lanes).
template <int CTRL>
DEV float from_lane(float v)
{
    return __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(v), CTRL, 0xf, 0xf, false));
}

// v plus its value 16 or 32 lanes away (the lanes' number with that bit turned).
DEV float add_16(float v)
{
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}
DEV float add_32(float v)
{
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

// Sum over the lanes whose number is the same modulo LP, in each of them: by
// rotations within 16 lanes (each step's values repeat at the last one's
// distance), then across the rows of 16.
template <int LP>
DEV float sum_beyond(float v)
{
    if constexpr (LP <= 8) v += from_lane<0x128>(v);
    if constexpr (LP <= 4) v += from_lane<0x124>(v);
    if constexpr (LP <= 2) v += from_lane<0x122>(v);
    if constexpr (LP <= 1) v += from_lane<0x121>(v);
    if constexpr (LP <= 16) v = add_16(v);
    if constexpr (LP <= 32) v = add_32(v);
    return v;
}

// Sum over each group of `n` lanes side by side, a power of two, in each of them.
DEV float sum_within(float v, int n)
{
    if (n > 1) v += from_lane<0xb1>(v);   // quad_perm 1 0 3 2
    if (n > 2) v += from_lane<0x4e>(v);   // quad_perm 2 3 0 1
    if (n > 4) v += from_lane<0x141>(v);  // row_half_mirror
    if (n > 8) v += from_lane<0x140>(v);  // row_mirror
    if (n > 16) v = add_16(v);
    if (n > 32) v = add_32(v);
    return v;
}

// Workgroups go round the 8 XCDs, each with an L2 of its own: the number of this
// workgroup among `n` (a multiple of 8) such that the ones on an XCD follow each
// other, and tiles that share lines of memory share an L2.
DEV uint32_t follow(uint32_t block, uint32_t n) { return (block & 7) * (n >> 3) + (block >> 3); }

// s / n for a whole n with 1 / n at hand: correctly rounded but for rare cases of
// half a unit (a constant row's mean is its value).
DEV float divided(float s, float n, float per)
{
    const float q = s * per;
    return __builtin_fmaf(__builtin_fmaf(-q, n, s), per, q);
}

// 1 / sqrt(v), the hardware's approximation and one Newton step. Every lane of a
// pixel computes it, so the library's exact steps would cost more than the sums.
// The hardware takes a subnormal v for zero, so small ones are scaled first; at
// zero and infinity (a variance that overflowed) the approximation is exact and
// the step would make it NaN.
DEV float inverse_root(float v)
{
    const bool small = v < 0x1p-96f;
    const float u = small ? v * 0x1p64f : v;
    const float r = __builtin_amdgcn_rsqf(u);
    const float n = __builtin_fmaf(0.5f * __builtin_fmaf(-u * r, r, 1.0f), r, r);
    const float root = u > 0.f && u < __builtin_inff() ? n : r;
    return small ? root * 0x1p32f : root;
}

inline int at_most(int64_t items, int64_t most) { return (int)(items < most ? (items > 1 ? items : 1) : most); }

}  // namespace wtc
