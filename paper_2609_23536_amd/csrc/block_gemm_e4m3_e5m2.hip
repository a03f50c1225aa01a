// Block-scaled products of E4M3 by E5M2.
#include "block_gemm_tiles.h"

namespace qe {

template hipError_t launch_block_tile<0, 1>(int, const BlockGemmParams &, hipStream_t);

}  // namespace qe
