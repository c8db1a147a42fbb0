// Layer norm of planes in float16.
#include "norm_planes.h"

namespace wtc {

bool launch_planes_f16(bool forward, bool out_planes, const NormArgs& a, hipStream_t s)
{
    return planes_launch<_Float16>(forward, out_planes, a, s);
}

}  // namespace wtc
