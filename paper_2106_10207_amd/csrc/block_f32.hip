// Norms and ends of blocks for fp32 streams and branches.
#include "block_forward.h"
#include "block_grad.h"

namespace dedloc {
template void launch_forward<float, float>(const ResidualArgs &, hipStream_t);
template void launch_grad<float, float>(const ResidualGradArgs &, hipStream_t);
}  // namespace dedloc
