// Block norms, stream of float and branch of float (net_norm.hpp).
#include "net_norm.hpp"

namespace kannet {

hipError_t launch_norm_f32(const NormCall &a, bool layer, bool backward, bool grouped, int blocks, hipStream_t st)
{
    return layer ? launch_norm_types<float, float, true>(a, backward, grouped, blocks, st)
                 : launch_norm_types<float, float, false>(a, backward, grouped, blocks, st);
}

}  // namespace kannet
