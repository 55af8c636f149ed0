// The tiled forward pass of the group norm on bf16 activations.
#include "norm_forward.h"

namespace kavg {

template hipError_t tiled_forward<__bf16>(const NormCall&, const NormTiles&, void*, hipStream_t);

}  // namespace kavg
