// What the layer norm kernels share: vectors of the storage types and sums over
// lanes.
#pragma once

#include "block_internal.h"
#include "wtconv_device.h"

namespace wtc {

template <typename T, int V>
struct alignas(sizeof(T) * V) Pack {
    T v[V];
};

template <int V, typename T>
DEV void load_pack(const T* p, float (&f)[V])
{
    const Pack<T, V> q = *reinterpret_cast<const Pack<T, V>*>(p);
#pragma unroll
    for (int i = 0; i < V; ++i) f[i] = to_f32(q.v[i]);
}

template <int V, typename T>
DEV void store_pack(T* p, const float (&f)[V])
{
    Pack<T, V> q;
#pragma unroll
    for (int i = 0; i < V; ++i) q.v[i] = from_f32<T>(f[i]);
    *reinterpret_cast<Pack<T, V>*>(p) = q;
}

inline int at_most(int64_t items, int64_t most) { return (int)(items < most ? (items > 1 ? items : 1) : most); }

}  // namespace wtc
