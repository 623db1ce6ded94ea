// gemm.cuh -- matrix products on the tensor cores for the operators that train
// dense layers (dense.cu, xent.cu, orthogonalize.cu): what a product is made of,
// its plan and its launch.  The kernel is in gemm_kernel.cuh.
//
// A product is C[n][m] = sum_k A[m][k] B[n][k], with m the index that is contiguous
// in the result.  Operands are bf16 "planes": one for bf16 data; two or three whose
// sum is the value where more bits are needed (split2, split3).  Either operand may
// lie with k or with its row index contiguous, so no operand is ever transposed in
// memory: x W^T, dz W and dz^T x are the same kernel.
#pragma once

#include "qcnn_internal.cuh"

#include <cuda.h>

namespace qcnn {

// An operand: planes of bf16, `plane` elements apart, rows of `ld` elements (16-byte
// multiples); mn: [k][row], else [row][k].  A of the fp32 kernel (GEMM_F32): fp32, any
// ld and alignment.
struct GemmOperand {
    const void *p = nullptr;
    long long ld = 0, plane = 0;
    int mn = 0;
};

enum GemmType { GEMM_T_F32 = 0, GEMM_T_BF16 = 1 };

// What becomes of a sum.  OUT: v = alpha * sum + bias[m] (alpha: *alpha_ptr where set); pre =
// v; v = act(v); v += beta * add[n][m]; out[n][m] = v (products of three planes: all fp32).
// PLANES: v = alpha * sum + beta * add, + diagonal where n == m; out and add are planes of the
// product's number, whose matrices have room for whole tiles (rows and columns up to the next
// multiple of 256).  SYM: PLANES of a symmetric product (A and B the same matrix): only m >= n
// is computed, and stored at both places.  STATS: m are rows, n classes: the maximum and the
// sum of exp over a tile's classes of v = sum + bias[n], and the value at the row's target.
// DLOGITS: m are classes, n rows: out = g_n (row_share(v) - [target_n == m]), in planes of the
// product's number whose rows have room for one more.
struct GemmEpi {
    float alpha = 1.f, beta = 0.f, diagonal = 0.f;
    const float *alpha_ptr = nullptr;  // in device memory
    const float *bias = nullptr;
    void *out = nullptr;
    long long ldo = 0, out_plane = 0;
    int out_type = GEMM_T_F32;  // (OUT)
    void *pre = nullptr;  // same type as out
    long long ldp = 0;
    const void *add = nullptr;
    long long lda = 0, add_plane = 0;
    int add_type = GEMM_T_F32;  // (OUT)
    int act = 0;
    int pair = 0;  // (launch_gemm) bits: out, pre, add go in pairs of elements
    // STATS, DLOGITS
    float2 *stats = nullptr;           // [tile along n][half][m]
    const long long *targets = nullptr;
    float *target_logit = nullptr;     // [m]
    const float4 *rows = nullptr;      // [n]: maximum, g, target (bits), log2 of the sum of exp
    int class0 = 0;                    // first class of this piece
    float *col_part = nullptr;         // DLOGITS: sums over a tile's rows, [tile along n][half][ld_col]
    long long ld_col = 0;
};

enum GemmKind { GEMM_OUT = 0, GEMM_SYM = 1, GEMM_STATS = 2, GEMM_DLOGITS = 3, GEMM_PLANES = 4 };

struct GemmProblem {
    GemmOperand a, b;
    int m = 0, n = 0, k = 0;
    GemmEpi e;
};

// planes: 1, 2, 3, or GEMM_F32 (A in fp32, split on its way to the tensor cores; B in
// three planes).
constexpr int GEMM_F32 = 0;
// Terms of a block: 64 of one plane; GEMM_F32: 32 of B's three planes.
constexpr int gemm_block_k(int planes) { return planes == GEMM_F32 ? 32 : 64; }

struct GemmPlan {
    int planes = 1, kind = 0, cg = 1;
    int bn = 0;       // tile columns
    // Shares of a tile's terms, of a CTA each in a cluster of that many (1, 2, 4, 8).  (Partial
    // sums through memory and a launch that joined them took 7 us more per product, and 19
    // of them added up by a tile's last CTA 28 us.)
    int splits = 1, kb_per_split = 0;
    int groups = 1;   // or shares whose sums stay apart: out is [groups][n][m], fp32, nothing else
    double score = 0;  // estimated SM clocks
    int n_tiles = 0;
};
// max_groups > 1: the caller adds up groups.
GemmPlan plan_gemm(int planes, int kind, int m, int n, int k, int max_groups = 1);

// Whether two products of one tile shape and kind, a's first, are sooner done in one launch than
// in two (their tiles are dealt out in turn).
bool gemm_together(const GemmPlan &a, int m_a, int n_a, int k_a, const GemmPlan &b, int m_b, int n_b, int k_b);

// One launch of one or two products of the same kind and planes (the second fills
// the SMs that the first one's last tiles leave idle); both with `plan`'s tile, unsplit
// if there are two.  A plan with shares is of the product's own k: one that has shares without
// terms is refused.
qcnn_status launch_gemm(const GemmPlan &plan, const GemmProblem *p, int count, cudaStream_t st);

// Smallest multiple of 8 elements: rows of 16-byte multiples.
inline long long pad8(long long v) { return (v + 7) / 8 * 8; }
// Of a matrix with room for whole tiles.
inline long long pad256(long long v) { return (v + 255) / 256 * 256; }

// src [rows][cols] (fp32 or bf16, row stride ld) -> bf16 planes [planes][rows][pad8(cols)],
// rows * pad8(cols) elements apart, to dst (null: not) and to kept (null: not), there with
// zeros in the rows whose class index in `classes` is outside [0, Ct).
struct PlanesJob {
    const void *src = nullptr;
    unsigned short *dst = nullptr, *kept = nullptr;
    const long long *classes = nullptr;
    long long all = 0, ld = 0, plane = 0;  // all: pieces of rows, per_row of them each
    int per_row = 0, cols = 0, planes = 0, Ct = 0, vec = 0;
    int blocks = 0;  // CTAs of 256 threads; 0: nothing to do
};
PlanesJob planes_job(const void *src, int bf16, long long rows, int cols, long long ld, int planes, void *dst,
                     void *kept = nullptr, const long long *classes = nullptr, int Ct = 0);
constexpr int kPieceCols = 1024;
// One launch of two of them, of one type.
qcnn_status launch_planes(const PlanesJob &a, const PlanesJob &b, int bf16, cudaStream_t st);

}  // namespace qcnn

#ifdef __CUDACC__
namespace qcnn {

// v = b0 + b1 (+ b2), bf16 pieces of two values each (low half: the first).  b0 is
// rounded to nearest (above bf16's largest finite value: to that; an infinity leaves an infinite b1,
// so that no result of it is finite), the differences are exact; of three pieces b1 is cut off and b2
// the rest, which has at most 8 bits: the sum is v, exactly, down to 2^-133 (bf16's
// last bit).  Of two, b1 is rounded: 16 to 17 bits of v.
__device__ __forceinline__ unsigned pack_bf16x2_finite(float lo, float hi) {
    unsigned r;
    asm("cvt.rn.satfinite.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}
__device__ __forceinline__ float2 bf16_rest(float v0, float v1, unsigned p) {
    return __ffma2_rn(make_float2(__uint_as_float(p << 16), __uint_as_float(p & 0xffff0000u)),
                      make_float2(-1.f, -1.f), make_float2(v0, v1));
}
__device__ __forceinline__ void planes3(float v0, float v1, unsigned &p0, unsigned &p1, unsigned &p2) {
    p0 = pack_bf16x2_finite(v0, v1);
    const float2 r = bf16_rest(v0, v1, p0);
    const unsigned rx = __float_as_uint(r.x), ry = __float_as_uint(r.y);
    p1 = __byte_perm(rx, ry, 0x7632);
    const float2 s = bf16_rest(r.x, r.y, p1);
    p2 = __byte_perm(__float_as_uint(s.x), __float_as_uint(s.y), 0x7632);
}
__device__ __forceinline__ void planes2(float v0, float v1, unsigned &p0, unsigned &p1) {
    p0 = pack_bf16x2_finite(v0, v1);
    const float2 r = bf16_rest(v0, v1, p0);
    p1 = pack_bf16x2(r.x, r.y);
}
// Two values in the pieces of a call's type: three in fp32 calls, one (a rounding) in bf16 calls.
template <bool F32>
__device__ __forceinline__ void planes_of(float v0, float v1, unsigned &p0, unsigned &p1, unsigned &p2) {
    if constexpr (F32) planes3(v0, v1, p0, p1, p2);
    else p0 = pack_bf16x2(v0, v1), p1 = p2 = 0;
}

// Activations and their derivatives (include/qcnn.h, qcnn_activation).
__device__ __forceinline__ float act_apply(float z, int act) {
    switch (act) {
        case QCNN_ACT_RELU: return z < 0.f ? 0.f : z;  // (NaN stays)
        case QCNN_ACT_GELU: return 0.5f * z * (1.f + erff(z * 0.70710678118654752f));
        case QCNN_ACT_SILU: return z / (1.f + expf(-z));
        default: return z;
    }
}
__device__ __forceinline__ float act_slope(float z, int act) {
    switch (act) {
        case QCNN_ACT_RELU: return z > 0.f ? 1.f : z != z ? z : 0.f;
        case QCNN_ACT_GELU:
            return 0.5f * (1.f + erff(z * 0.70710678118654752f)) +
                   z * 0.39894228040143268f * expf(-0.5f * z * z);
        case QCNN_ACT_SILU: {
            const float s = 1.f / (1.f + expf(-z));
            return s * (1.f + z * (1.f - s));
        }
        default: return 1.f;
    }
}

constexpr float kLog2e = 1.4426950408889634f;
// 2^x to 2 ulp; results below 2^-126 are zero.
__device__ __forceinline__ float ex2(float x) {
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}
// The softmax of a logit of a row (GemmEpi's rows).
__device__ __forceinline__ float row_share(float logit, const float4 &row) {
    return ex2(fmaf(logit - row.x, kLog2e, -row.w));
}

__device__ __forceinline__ float bf16_to_float(unsigned short v) {
    return __uint_as_float((unsigned)v << 16);
}
__device__ __forceinline__ unsigned short float_to_bf16(float v) {
    return (unsigned short)(pack_bf16x2(v, 0.f) & 0xffffu);
}
// One value of a matrix of `type`, element offset o.
__device__ __forceinline__ float load_as(const void *p, int type, long long o) {
    return type == GEMM_T_F32 ? static_cast<const float *>(p)[o]
                              : bf16_to_float(static_cast<const unsigned short *>(p)[o]);
}

// CTA `block` of a job.  A warp takes pieces of rows, a lane eight columns at a time: two 16-byte
// loads (or eight of an element), a 16-byte store per plane.
template <typename T>
__device__ __forceinline__ void planes_part(const PlanesJob &j, int block) {
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, cols = j.cols;
    const long long pitch = (cols + 7) / 8 * 8;
    for (long long i = (long long)block * 8 + warp; i < j.all; i += (long long)j.blocks * 8) {
        const long long r = i / j.per_row;
        const int first = (int)(i - r * j.per_row) * kPieceCols, end = min(cols, first + kPieceCols);
        const bool in = !j.kept || (unsigned long long)j.classes[r] < (unsigned long long)j.Ct;
        const T *s = static_cast<const T *>(j.src) + r * j.ld;
#pragma unroll 2
        for (int c = first + lane * 8; c < end; c += 256) {
            float v[8];
            if (j.vec && c + 8 <= cols) {
                if constexpr (sizeof(T) == 4) {
                    const float4 a = *reinterpret_cast<const float4 *>(s + c);
                    const float4 b = *reinterpret_cast<const float4 *>(s + c + 4);
                    v[0] = a.x, v[1] = a.y, v[2] = a.z, v[3] = a.w, v[4] = b.x, v[5] = b.y, v[6] = b.z, v[7] = b.w;
                } else {
                    const uint4 a = *reinterpret_cast<const uint4 *>(s + c);
                    const unsigned w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        v[2 * k] = __uint_as_float(w[k] << 16);
                        v[2 * k + 1] = __uint_as_float(w[k] & 0xffff0000u);
                    }
                }
            } else {
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    v[k] = 0.f;
                    if (c + k < cols) {
                        if constexpr (sizeof(T) == 4) v[k] = s[c + k];
                        else v[k] = bf16_to_float(s[c + k]);
                    }
                }
            }
            unsigned w[3][4];
#pragma unroll
            for (int k = 0; k < 4; ++k) planes_of<sizeof(T) == 4>(v[2 * k], v[2 * k + 1], w[0][k], w[1][k], w[2][k]);
#pragma unroll
            for (int p = 0; p < 3; ++p) {
                if (p >= j.planes) break;
                const uint4 q = make_uint4(w[p][0], w[p][1], w[p][2], w[p][3]);
                const long long o = p * j.plane + r * pitch + c;
                if (j.dst) *reinterpret_cast<uint4 *>(j.dst + o) = q;
                if (j.kept) *reinterpret_cast<uint4 *>(j.kept + o) = in ? q : make_uint4(0, 0, 0, 0);
            }
        }
    }
}

}  // namespace qcnn
#endif
