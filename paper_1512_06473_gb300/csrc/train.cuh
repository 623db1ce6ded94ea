// train.cuh -- what the entry points of dense.cu, xent.cu and orthogonalize.cu share.
#pragma once

#include "gemm.cuh"

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
inline bool tma_ok(const void *p, long long ld) {
    return reinterpret_cast<uintptr_t>(p) % 16 == 0 && ld % 8 == 0;
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

// y = x W^T of few rows (dense.cu): N <= kFewRows.
constexpr int kFewRows = 8;
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
