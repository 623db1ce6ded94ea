// ortho_small.cuh -- Newton-Schulz steps of a small matrix in one launch
// (orthogonalize_small.cu).
#pragma once

#include "gemm.cuh"

namespace qcnn {

struct OrthoSmall {
    int cluster = 0;  // CTAs; 0: not taken
    int qs = 0;       // columns (of the larger side) per CTA
    double score = 0;
};
// products: the estimated SM clocks of the steps as products on the tensor cores.
OrthoSmall ortho_small_plan(int m, int n, int steps, double products);
qcnn_status launch_ortho_small(const OrthoSmall &o, const void *G, long long ldg, int m, int n, int steps,
                               const float *coeffs, float eps, void *out, long long ldo, int bf16,
                               cudaStream_t st);

}  // namespace qcnn
