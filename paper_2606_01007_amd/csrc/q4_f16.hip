// The experts' 4-bit products in float16.
#include "q4_kernels.h"

namespace tacg {
template void q4_start<_Float16, false>(const Q4Args& a, hipStream_t stream);
}  // namespace tacg
