// Layer norm of planes in bfloat16.
#include "norm_planes.h"

namespace wtc {

bool launch_planes_bf16(bool forward, bool out_planes, const NormArgs& a, hipStream_t s)
{
    return planes_launch<uint16_t>(forward, out_planes, a, s);
}

int64_t parts_planes_16(int64_t B, int64_t S, int C) { return planes_parts<uint16_t>(B, S, C); }

}  // namespace wtc
