// The register-resident routing kernels for __nv_bfloat16 logits.
#include <algorithm>

#include "route_fast.cuh"

namespace gshard {

template bool launch_route_fwd_fast<__nv_bfloat16>(const RouteArgs&, int, float*, cudaStream_t);
template bool launch_route_bwd_fast<__nv_bfloat16>(const RouteGradArgs&, cudaStream_t);

}  // namespace gshard
