// Block norms, stream of bf16 and branch of float (net_norm.hpp).
#include "net_norm.hpp"

namespace kannet {

hipError_t launch_norm_bf16_f32(const NormCall &a, const NormPick &p, hipStream_t st)
{
    return p.layer ? launch_norm_types<bf16, float, true>(a, p, st) : launch_norm_types<bf16, float, false>(a, p, st);
}

}  // namespace kannet
