// The experts' 4-bit products in bfloat16.
#include "q4_kernels.h"

namespace tacg {
template void q4_start<__bf16, false>(const Q4Args& a, hipStream_t stream);
}  // namespace tacg
