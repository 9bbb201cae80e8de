// The router whose selection is limited to the best groups of experts: the kernel of route_kernels.h with a stage for the groups.
#include "route_kernels.h"

namespace tacg {

void start_route_groups(const RouteArgs& a, int32_t dtype, bool bal, dim3 grid, hipStream_t stream) {
  start_rows<true>(a, dtype, bal, grid, stream);
}

}  // namespace tacg
