// gemm_fused.hip -- the GEMM kernels of gemm.hip with bias, activation and residual
// in their epilogue (qg::fused::launch, for qg_gemm_fused): the same source, compiled
// again beside it, so that the plain linears' kernels stay what they are.
#define QG_EPILOGUE 1
#include "gemm.hip"
