// The tiled backward pass of the group norm on bf16 activations.
#include "norm_backward.h"

namespace kavg {

template hipError_t tiled_backward<__bf16>(const NormCall&, const NormTiles&, void*, hipStream_t);

}  // namespace kavg
