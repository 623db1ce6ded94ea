// int8_gemm.cuh -- the product of codes on the tensor cores (int8_gemm.cu) for int8.cu: its plan and its
// launch.
#pragma once

#include "gemm.cuh"

namespace qcnn {

// y[n][m] = epilogue of xscale[n] wscale[m] sum_k x[n][k] W[m][k].
struct Int8Problem {
    const void *x;       // fp16 [n][k], rows of 16-byte multiples, 16-byte aligned
    long long ldx;
    const int8_t *W;     // [m][k], 16-byte aligned rows
    long long ldw;
    bool w_late = false; // W comes from a kernel of this call
    const float *xscale, *wscale;
    const int *sums = nullptr;  // of the magnitudes of x's codes, [n][segs]: of 1024 terms each (int8_sums)
    int segs = 0;
    int m, n, k;
    GemmEpi e;  // bias, act, add (beta 1), out
};
struct Int8Plan {
    int cg = 1, bn = 0;
    int splits = 1, kb_per_split = 0;  // shares of a tile's terms, a CTA of a cluster each
    double score = 0;                  // estimated SM clocks
};
Int8Plan plan_int8(int m, int n, int k);
// Terms of a segment whose sum is exact whatever the codes are, and whether a plan of k terms goes by the
// sums of magnitudes.
constexpr int kInt8Segment = 1024;
constexpr int kInt8MaxTerms = 131071;  // whose sum of products fits 32 bits
// A row's scale from which on a sum takes the output's first: a sum below 2^31 times less stays finite.
constexpr float kLargeScale = 0x1p96f;
inline bool int8_sums(const Int8Plan &p, int k) { return p.bn > 128 && k > kInt8Segment; }
qcnn_status launch_int8(const Int8Plan &plan, const Int8Problem &p, cudaStream_t st);

}  // namespace qcnn
