// Block norms, stream of float and branch of float (net_norm.hpp).
#include "net_norm.hpp"

namespace kannet {

hipError_t launch_norm_f32(const NormCall &a, const NormPick &p, hipStream_t st)
{
    return p.layer ? launch_norm_types<float, float, true>(a, p, st) : launch_norm_types<float, float, false>(a, p, st);
}

}  // namespace kannet
