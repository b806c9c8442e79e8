// The register-resident routing kernels for float logits.
#include <algorithm>

#include "route_fast.cuh"

namespace gshard {

template bool launch_route_fwd_fast<float>(const RouteArgs&, int, float*, cudaStream_t);
template bool launch_route_bwd_fast<float>(const RouteGradArgs&, cudaStream_t);

}  // namespace gshard
