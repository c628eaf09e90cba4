// Norms and ends of blocks for fp32 streams and fp16 branches.
#include "block_forward.h"
#include "block_grad.h"

namespace dedloc {
template void launch_forward<float, _Float16>(const ResidualArgs &, hipStream_t);
template void launch_grad<float, _Float16>(const ResidualGradArgs &, hipStream_t);
}  // namespace dedloc
