// Layer norm of planes in bfloat16.
#include "norm_planes.h"

namespace wtc {

bool launch_planes_bf16(bool forward, bool out_planes, const NormArgs& a, hipStream_t s)
{
    return planes_launch<uint16_t>(forward, out_planes, a, s);
}

}  // namespace wtc
