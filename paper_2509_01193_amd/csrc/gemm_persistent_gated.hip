// The forward product of a gated feed-forward block: gemm_persistent.hip once more, with tiles of gate and up columns and the activation in
// the epilogue (see GATED there).
#define LOBRA_GP_KTAIL 0
#define LOBRA_GP_GATED 1
#define LOBRA_GP_KERNEL gemm_persistent_gated_kernel
#define LOBRA_GP_HOST gemm_persistent_gated
#include "gemm_persistent.hip"
