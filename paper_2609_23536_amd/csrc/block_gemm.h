// Launch of a block-scaled product with a given tile, for operands of formats FA and FB.
#pragma once

#include "kernels.h"

namespace qe {

constexpr int kFewRowsTile = 0;  // in place of a GemmTile

template <int FA, int FB>
hipError_t launch_block_tile(int tile, const BlockGemmParams &p, hipStream_t s);

}  // namespace qe
