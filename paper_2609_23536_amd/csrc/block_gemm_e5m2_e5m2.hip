// Block-scaled products of E5M2 by E5M2.
#include "block_gemm_tiles.h"

namespace qe {

template hipError_t launch_block_tile<1, 1>(int, const BlockGemmParams &, hipStream_t);

}  // namespace qe
