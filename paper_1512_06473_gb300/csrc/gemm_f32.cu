// gemm_f32.cu -- the tensor-core product (gemm_kernel.cuh) of fp32 operands that are split
// on their way to tensor memory.
#define QCNN_UNIT_RECORDS
#include "gemm_kernel.cuh"

namespace qcnn {

using GemmLaunch = qcnn_status (*)(const void *, int, size_t, cudaStream_t);
GemmLaunch gemm_launch_f32() { return GemmKernel<3, GEMM_OUT, 1, true>::launch; }

}  // namespace qcnn
