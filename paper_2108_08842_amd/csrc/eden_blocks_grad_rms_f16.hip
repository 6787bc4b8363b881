// The gradients of the join, type f16, an rms norm behind the branch.
#include "eden_blocks_grad.h"

namespace eden_layers {
template hipError_t launch_block_grad<EDEN_F16, 1>(const GradArgs &, hipStream_t);
}  // namespace eden_layers
