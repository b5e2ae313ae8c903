// The persistent kernel on a base in 8-bit integers (gemm_persistent.hip).
#define LOBRA_GP_Q8 1
#define LOBRA_GP_KTAIL 0
#define LOBRA_GP_KERNEL gemm_persistent_q8_kernel
#define LOBRA_GP_HOST gemm_persistent_q8
#include "gemm_persistent.hip"
