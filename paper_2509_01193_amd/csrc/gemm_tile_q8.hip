// The tiled kernel on a base in 8-bit integers (gemm_tile.hip).
#define LOBRA_GT_Q8 1
#define LOBRA_GT_KERNEL gemm_tile_q8_kernel
#define LOBRA_GT_BESIDE gemm_tile_beside_q8_kernel
#include "gemm_tile.hip"
