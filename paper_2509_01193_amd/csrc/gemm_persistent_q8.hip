// The persistent kernel on a base in 8-bit integers (gemm_persistent.hip).  16384 x 4096 x 11008 with four tasks of rank 16 572 to 684 us (2.2 to 2.6 Pop/s; bound: the matrix
// cores at the clock the power limit leaves, the library's product alone, without scales and adapters, takes 652), 8190 x 4096 x 4096 115 to 122, 777 x 4096 x 11008, whose
// 172 tiles are less than one for each compute unit, 54.
#define LOBRA_GP_Q8 1
#define LOBRA_GP_KTAIL 0
#define LOBRA_GP_KERNEL gemm_persistent_q8_kernel
#define LOBRA_GP_HOST gemm_persistent_q8
#include "gemm_persistent.hip"
