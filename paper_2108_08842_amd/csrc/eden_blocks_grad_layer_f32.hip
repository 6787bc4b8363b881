// The gradients of the join, type f32, a layer norm behind the branch.
#include "eden_blocks_grad.h"

namespace eden_layers {
template hipError_t launch_block_grad<EDEN_F32, 2>(const GradArgs &, hipStream_t);
}  // namespace eden_layers
