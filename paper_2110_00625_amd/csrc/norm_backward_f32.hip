// The tiled backward pass of the group norm on fp32 activations.
#include "norm_backward.h"

namespace kavg {

template hipError_t tiled_backward<float>(const NormCall&, const NormTiles&, void*, hipStream_t);

}  // namespace kavg
