// gemm_p2.cu -- the tensor-core products (gemm_kernel.cuh) of orthogonalize.cu: operands and
// results in two planes or three.
#define QCNN_UNIT_RECORDS
#include "gemm_kernel.cuh"

namespace qcnn {

using GemmLaunch = qcnn_status (*)(const void *, int, size_t, cudaStream_t);
template <int P>
static GemmLaunch of_kind(int kind, int cg) {
    if (kind == GEMM_SYM)
        return cg == 1 ? GemmKernel<P, GEMM_SYM, 1, false>::launch : GemmKernel<P, GEMM_SYM, 2, false>::launch;
    return cg == 1 ? GemmKernel<P, GEMM_PLANES, 1, false>::launch : GemmKernel<P, GEMM_PLANES, 2, false>::launch;
}
GemmLaunch gemm_launch_planes(int planes, int kind, int cg) {
    if (planes == 3) return of_kind<3>(kind, cg);
    if (kind == GEMM_OUT)
        return cg == 1 ? GemmKernel<2, GEMM_OUT, 1, false>::launch : GemmKernel<2, GEMM_OUT, 2, false>::launch;
    return of_kind<2>(kind, cg);
}

}  // namespace qcnn
