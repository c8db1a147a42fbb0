// Layer norm of planes in float32.
#include "norm_planes.h"

namespace wtc {

bool launch_planes_f32(bool forward, bool out_planes, const NormArgs& a, hipStream_t s)
{
    return planes_launch<float>(forward, out_planes, a, s);
}

int64_t parts_planes_f32(int64_t B, int64_t S, int C) { return planes_parts<float>(B, S, C); }

}  // namespace wtc
