// The tiled forward pass of the group norm on fp32 activations.
#include "norm_forward.h"

namespace kavg {

template hipError_t tiled_forward<float>(const NormCall&, const NormTiles&, void*, hipStream_t);

}  // namespace kavg
