// gemm_p1.cu -- the tensor-core product (gemm_kernel.cuh) of operands in 1 plane.
#define QCNN_UNIT_RECORDS
#include "gemm_kernel.cuh"

namespace qcnn {

using GemmLaunch = qcnn_status (*)(const void *, int, size_t, cudaStream_t);
// (a kernel of the products, to ask how many clusters of such CTAs are resident at once)
const void *gemm_kernel_address() {
    return reinterpret_cast<const void *>(gemm_kernel<1, GEMM_OUT, 1, false>);
}
GemmLaunch gemm_launch_p1(int kind, int cg) {
    switch (kind) {
        case GEMM_STATS:
            return cg == 1 ? GemmKernel<1, GEMM_STATS, 1, false>::launch : GemmKernel<1, GEMM_STATS, 2, false>::launch;
        case GEMM_DLOGITS:
            return cg == 1 ? GemmKernel<1, GEMM_DLOGITS, 1, false>::launch : GemmKernel<1, GEMM_DLOGITS, 2, false>::launch;
        default:
            return cg == 1 ? GemmKernel<1, GEMM_OUT, 1, false>::launch : GemmKernel<1, GEMM_OUT, 2, false>::launch;
    }
}

}  // namespace qcnn
