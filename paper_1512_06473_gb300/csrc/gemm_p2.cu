// gemm_p2.cu -- the tensor-core products (gemm_kernel.cuh) of orthogonalize.cu: operands in
// two planes, and the symmetric ones of three.
#define QCNN_UNIT_RECORDS
#include "gemm_kernel.cuh"

namespace qcnn {

using GemmLaunch = qcnn_status (*)(const void *, int, size_t, cudaStream_t);
GemmLaunch gemm_launch_p2(int kind, int cg) {
    if (kind == GEMM_SYM)
        return cg == 1 ? GemmKernel<2, GEMM_SYM, 1, false>::launch : GemmKernel<2, GEMM_SYM, 2, false>::launch;
    return cg == 1 ? GemmKernel<2, GEMM_OUT, 1, false>::launch : GemmKernel<2, GEMM_OUT, 2, false>::launch;
}
GemmLaunch gemm_launch_p3_sym(int cg) {
    return cg == 1 ? GemmKernel<3, GEMM_SYM, 1, false>::launch : GemmKernel<3, GEMM_SYM, 2, false>::launch;
}

}  // namespace qcnn
