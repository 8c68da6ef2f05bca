// Block norms, stream of bf16 and branch of float (net_norm.hpp).
#include "net_norm.hpp"

namespace kannet {

hipError_t launch_norm_bf16_f32(const NormCall &a, bool layer, bool backward, bool grouped, int blocks, hipStream_t st)
{
    return layer ? launch_norm_types<bf16, float, true>(a, backward, grouped, blocks, st)
                 : launch_norm_types<bf16, float, false>(a, backward, grouped, blocks, st);
}

}  // namespace kannet
