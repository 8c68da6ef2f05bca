// Block norms, stream of bf16 and branch of bf16 (net_norm.hpp).
#include "net_norm.hpp"

namespace kannet {

hipError_t launch_norm_bf16(const NormCall &a, bool layer, bool backward, bool grouped, int blocks, hipStream_t st)
{
    return layer ? launch_norm_types<bf16, bf16, true>(a, backward, grouped, blocks, st)
                 : launch_norm_types<bf16, bf16, false>(a, backward, grouped, blocks, st);
}

}  // namespace kannet
