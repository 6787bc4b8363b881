// The gradients of the join, type bf16, no norm behind the branch.
#include "eden_blocks_grad.h"

namespace eden_layers {
template hipError_t launch_block_grad<EDEN_BF16, 0>(const GradArgs &, hipStream_t);
}  // namespace eden_layers
