// Norms and ends of blocks for fp16 streams and branches.
#include "block_forward.h"
#include "block_grad.h"

namespace dedloc {
template void launch_forward<_Float16, _Float16>(const ResidualArgs &, hipStream_t);
template void launch_grad<_Float16, _Float16>(const ResidualGradArgs &, hipStream_t);
}  // namespace dedloc
