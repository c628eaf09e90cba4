// Norms and ends of blocks for bf16 streams and branches.
#include "block_forward.h"
#include "block_grad.h"

namespace dedloc {
template void launch_forward<__bf16, __bf16>(const ResidualArgs &, hipStream_t);
template void launch_grad<__bf16, __bf16>(const ResidualGradArgs &, hipStream_t);
}  // namespace dedloc
