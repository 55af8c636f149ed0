// Tiles of the products of bf16 operands, both turned (linear_tile.h).
#include "linear_tile.h"

namespace kavg {

hipError_t start_bf16_gradient(int tile, bool direct, const ProductArgs& a, hipStream_t st) { return start_kind<__bf16, true, true>(tile, direct, a, st); }

}  // namespace kavg
