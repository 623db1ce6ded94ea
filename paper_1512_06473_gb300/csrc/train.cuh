// train.cuh -- what the entry points of dense.cu, xent.cu and orthogonalize.cu share.
#pragma once

#include "gemm.cuh"

#include <algorithm>
#include <climits>

namespace qcnn {

inline bool dtype_ok(int t) { return t == QCNN_F32 || t == QCNN_BF16; }
inline size_t type_bytes(int dtype) { return dtype == QCNN_F32 ? 4 : 2; }
// A matrix of rows x cols: a pointer where there are elements, aligned to them, rows that
// do not overlap.
inline bool matrix_ok(const void *p, long long ld, long long rows, long long cols, int dtype) {
    return ld >= cols && (rows == 0 || p) && reinterpret_cast<uintptr_t>(p) % type_bytes(dtype) == 0;
}
// Rows that TMA can read.
inline bool tma_ok(const void *p, long long ld, int dtype) {
    return reinterpret_cast<uintptr_t>(p) % 16 == 0 && ld * type_bytes(dtype) % 16 == 0;
}

// Weights that a product reads without a pass over them: fp32 of any row distance.
inline bool weights_ok(const void *p, long long ld, int dtype) {
    return dtype == QCNN_BF16 ? tma_ok(p, ld, dtype) : reinterpret_cast<uintptr_t>(p) % 16 == 0;
}

// A workspace, carved in order.  With no base it only counts.
struct Carver {
    uint8_t *base;
    size_t used = 0;
    void *take(size_t bytes) {
        void *p = base ? base + used : nullptr;
        used += align_up(bytes, kWsAlign);
        return p;
    }
    template <typename T>
    T *array(size_t n) {
        return static_cast<T *>(take(n * sizeof(T)));
    }
};
inline qcnn_status workspace_ok(const void *ws, size_t have, size_t need) {
    if (need && (!ws || have < need || reinterpret_cast<uintptr_t>(ws) % kWsAlign)) return QCNN_ERR_WORKSPACE;
    return QCNN_OK;
}

// SM clocks that a pass over `bytes` costs a call beside its products (the memory's
// rate at the SMs' clock, and a launch).
inline double pass_clocks(double bytes) { return bytes / 3200.0 + 4000.0; }

// y = x W^T of few rows (dense.cu).
constexpr int kFewRows = 8;
// In SM clocks: up to four rows the weights' bytes, with eight the multiply-adds (0.75 and 1
// million elements of W per us).
inline double few_rows_clocks(int N, int Cs, int Ct, bool bf16) {
    const double elements = (double)Cs * Ct;
    return 5000.0 + (N <= 4 ? elements * (bf16 ? 2.0 : 4.0) / 3400.0 : elements / (bf16 ? 540.0 : 400.0));
}
// Whether that is sooner done than the product g.  Up to four rows it always is (4 x 4096 ->
// 19456 in fp32 51 us and the product 57), and where a product cannot read W as it is (8 x 4097 ->
// 19456, fp32 off 16 bytes 72 and 104, bf16 69 and 112).  With eight it depends on the size of
// the weights: 8 x 4096 -> 1000 in fp32 8.3 us and the product 14.4, in bf16 6.9 and 9.4; -> 4096
// 24.6 and 21.2, 19.4 and 11.5; -> 19456 83 and 58, 50 and 29.  (7000: the product's launches.)
inline bool few_rows_sooner(int N, int Cs, int Ct, bool bf16, bool w_direct, const GemmPlan &g) {
    if (N <= 4 || N > kFewRows || !w_direct) return N <= kFewRows;
    const double bytes = (double)Cs * Ct * (bf16 ? 2.0 : 4.0);
    return few_rows_clocks(N, Cs, Ct, bf16) < std::max(g.score, bytes / 3400.0) + 7000.0;
}
struct FewRows {
    const void *x, *W;
    long long ldx, ldw;
    int N, Cs, Ct, bf16;
    GemmEpi e;  // bias, act, add (beta 1), pre, out; n = row, m = output
};
qcnn_status launch_few_rows(const FewRows &f, cudaStream_t st);

// Column sums of partial rows: dst[c] = sum over r < rows of part[r][ld] (in order), times
// *scale (null: 1).
qcnn_status launch_column_join(const float *part, int rows, long long ld, int cols, const float *scale,
                               float *dst, cudaStream_t st);

}  // namespace qcnn
