// Host-only dump of an optimizer step's launches (no GPU, no kernels): includes
// the library's host source with the launchers stubbed out, and for each element
// count on stdin (bfloat16 tensors, 64 million elements apart) prints its
// entries in the launches, one line each:
//   <launch> <first chunk> <byte offset of param> <of grad> <element of moments> <elements>
// with chunks of 2048 elements and 5 of them in a launch. Built and run by
// tests/test_block_host.py.
#include "block_api.cpp"

#include <stdio.h>

#include <vector>

namespace wtc {
static int launches = 0;
int64_t norm_parts(const wtconv_norm_desc&) { return 1; }
int64_t residual_parts(const wtconv_residual_desc&) { return 1; }
hipError_t launch_norm_forward(const wtconv_norm_desc&, const NormArgs&, hipStream_t) { return hipSuccess; }
hipError_t launch_norm_backward(const wtconv_norm_desc&, NormArgs, float*, float*, hipStream_t) { return hipSuccess; }
hipError_t launch_residual_forward(wtconv_dtype, const ResidualArgs&, hipStream_t) { return hipSuccess; }
hipError_t launch_residual_backward(wtconv_dtype, ResidualArgs, float*, hipStream_t) { return hipSuccess; }
hipError_t launch_adamw_moments(wtconv_dtype, int64_t, const uint8_t*, const uint8_t*, const uint8_t*, const uint8_t*,
                                void*, void*, hipStream_t)
{
    return hipSuccess;
}
int64_t adam_chunk_elements() { return 2048; }
int64_t adam_most_chunks() { return 5; }
hipError_t launch_adamw(wtconv_dtype, int, const AdamArgs& a, hipStream_t)
{
    for (int i = 0; i < a.count; ++i)
        printf("%d %u %llu %llu %lld %lld\n", launches, a.first[i], (unsigned long long)(uintptr_t)a.p[i],
               (unsigned long long)(uintptr_t)a.g[i], (long long)a.at[i], (long long)a.n[i]);
    ++launches;
    return hipSuccess;
}
}  // namespace wtc

int main()
{
    const uintptr_t param = (uintptr_t)1 << 40, grad = (uintptr_t)1 << 41;
    std::vector<wtconv_adamw_tensor> tensors;
    long long n;
    while (scanf("%lld", &n) == 1) {
        const long long at = 1000000ll * 64 * (long long)tensors.size();
        tensors.push_back({(void*)(param + at * 2), (const void*)(grad + at * 2), n, at, 0});
    }
    wtconv_adamw_group g = {};
    g.lr = 1e-3;
    g.step = 1;
    g.exp_avg = g.exp_avg_sq = (void*)4096;
    return wtconv_adamw_step(1, &g, (int)tensors.size(), tensors.data(), WTCONV_BF16, 32, nullptr, nullptr);
}
