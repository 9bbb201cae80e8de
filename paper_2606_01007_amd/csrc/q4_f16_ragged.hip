// The experts' 4-bit products in float16, columns that are no whole number of groups or less than a step.
#include "q4_kernels.h"

namespace tacg {
template void q4_start<_Float16, true>(const Q4Args& a, hipStream_t stream);
}  // namespace tacg
