// gemm_gated.hip -- the GEMM kernels of gemm.hip with an activated gate times its up projection
// in their epilogue (qg::gated::launch, for qg_gemm_fused): the same source, compiled
// again beside it, so that the plain linears' kernels stay what they are.
#define QG_EPILOGUE 2
#include "gemm.hip"
