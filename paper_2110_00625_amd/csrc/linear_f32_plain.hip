// Tiles of the products of f32 operands, neither of them turned (linear_tile.h).
#include "linear_tile.h"

namespace kavg {

hipError_t start_f32_plain(int tile, bool direct, const ProductArgs& a, hipStream_t st) { return start_kind<float, false, false>(tile, direct, a, st); }

}  // namespace kavg
