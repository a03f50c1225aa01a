// Block-scaled products of E4M3 by E4M3.
#include "block_gemm_tiles.h"

namespace qe {

template hipError_t launch_block_tile<0, 0>(int, const BlockGemmParams &, hipStream_t);

}  // namespace qe
