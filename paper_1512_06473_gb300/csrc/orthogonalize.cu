// orthogonalize.cu -- qcnn_orthogonalize: Newton-Schulz products.
//
//   X = G / (||G||_F + eps); steps times: A = X X^T, B = a I + b A + c A A, X = B X
//
// of the smaller side p (q the larger; G with more rows than columns from the right, by
// reading X with its rows contiguous: nothing is transposed).  Three products a step, of
// 2 p^2 q, 2 p^3 and 2 p^2 q operations; A and B are symmetric, so of the first two the
// tiles on one side of the diagonal are computed and stored twice.  (a X + (B - a I) X
// instead of B X read X again in the third product's epilogue, 12 us a step of 1000 x 4096.)
// X, A and B live as bf16 planes that the epilogues write and TMA reads: two in bf16 calls (in
// one, each step's rounding of X and B would be that of the result), three in fp32 calls.
// 4096 x 9216 in bf16, five steps: 4.5 ms, 1,770 TFLOP/s of its three products (tensor cores; at the
// power limit 4.7); 1000 x 4096 in fp32 391 us, half of that rate: 15 products of 36 to 256
// tiles one after another.
// Matrices whose smaller side is 64 or less are done in one launch where that is sooner done
// (orthogonalize_small.cu).
#include "ortho_small.cuh"
#include "train.cuh"

#include <algorithm>

namespace qcnn {
namespace {

constexpr int kNormBlocks = 608;

// The eight (or fewer) columns from c of a row in fp32, zeros past the last; vec: 16-byte
// loads are possible.
template <typename T>
__device__ __forceinline__ void row8(const T *row, int c, int cols, bool vec, float (&v)[8]) {
    if (vec && c + 8 <= cols) {
        if constexpr (sizeof(T) == 4) {
            const float4 a = *reinterpret_cast<const float4 *>(row + c), b = *reinterpret_cast<const float4 *>(row + c + 4);
            v[0] = a.x, v[1] = a.y, v[2] = a.z, v[3] = a.w, v[4] = b.x, v[5] = b.y, v[6] = b.z, v[7] = b.w;
        } else {
            const uint4 a = *reinterpret_cast<const uint4 *>(row + c);
            const unsigned w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                v[2 * j] = __uint_as_float(w[j] << 16);
                v[2 * j + 1] = __uint_as_float(w[j] & 0xffff0000u);
            }
        }
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            float x = 0.f;
            if (c + j < cols) {
                if constexpr (sizeof(T) == 4) x = row[c + j];
                else x = bf16_to_float(row[c + j]);
            }
            v[j] = x;
        }
    }
}

// Both passes over G: a warp takes pieces of rows (of at most kNormCols columns), a lane
// eight columns at a time.
constexpr int kNormCols = 2048;
struct Pieces {
    long long rows, all;  // rows, and rows x pieces of a row
    int cols, per_row;
};

// Sums of squares by CTA, in fp64; a lane's run of up to 64 squares in fp32.  A run whose largest value
// is above 2^48 or below 2^-40 is taken again, scaled by 2^-64 or 2^96: no square overflows, and none
// vanishes or loses bits that the run's sum has (with eps 0 a matrix of subnormal values has its own
// norm).  (With sums for the three ranges side by side 1000 x 4096 in fp32 is normalized in 35 us, 28.)
constexpr float kLarge = 0x1p48f, kSmall = 0x1p-40f;
__device__ __forceinline__ double add_lanes(double v) {
#pragma unroll
    for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}
template <typename T>
__global__ void __launch_bounds__(256) norm_kernel(const T *g, long long ldg, Pieces q, int vec, double *part) {
    __shared__ double red[8];
    grid_dep_sync();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    double s = 0.;
    for (long long i = (long long)blockIdx.x * 8 + warp; i < q.all; i += (long long)gridDim.x * 8) {
        const long long r = i / q.per_row;
        const int first = (int)(i - r * q.per_row) * kNormCols, end = min(q.cols, first + kNormCols);
        const T *row = g + r * ldg;
        float sum = 0.f, top = 0.f;
#pragma unroll 4
        for (int c = first + lane * 8; c < end; c += 256) {
            float v[8];
            row8(row, c, end, vec, v);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                sum = fmaf(v[j], v[j], sum);
                top = fmaxf(top, fabsf(v[j]));
            }
        }
        const bool large = top > kLarge;
        if (large || (top < kSmall && top > 0.f)) {
            const float scale = large ? 0x1p-64f : 0x1p96f;
            sum = 0.f;
#pragma unroll 1
            for (int c = first + lane * 8; c < end; c += 256) {
                float v[8];
                row8(row, c, end, vec, v);
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const float x = v[j] * scale;
                    sum = fmaf(x, x, sum);
                }
            }
            s = fma((double)sum, large ? 0x1p128 : 0x1p-192, s);
        } else {
            s += sum;
        }
    }
    s = add_lanes(s);
    if (lane == 0) red[warp] = s;
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int i = 1; i < 8; ++i) s += red[i];
        part[blockIdx.x] = s;
    }
}

// X = G / (norm + eps) in planes, rows of pitch elements (or, planes 0, as the result);
// every CTA adds the sums up in the same order.
template <typename T>
__global__ void __launch_bounds__(256) scale_kernel(const T *g, long long ldg, Pieces q, int vec,
                                                    const double *part, int parts, float eps, int planes,
                                                    unsigned short *dst, long long pitch, long long plane, T *out,
                                                    long long ldo) {
    __shared__ double red[8];
    grid_dep_sync();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    double s = 0.;
    for (int i = threadIdx.x; i < parts; i += 256) s += part[i];
    s = add_lanes(s);
    if (lane == 0) red[warp] = s;
    __syncthreads();
    s = red[0];
    for (int i = 1; i < 8; ++i) s += red[i];
    const double norm = sqrt(s) + (double)eps;
    // (a norm of zero with eps zero: the matrix is zero; a factor above fp32's range, of tiny
    // matrices with a tiny eps, is taken in two: f2 is 1 otherwise)
    const double f = norm > 0. || norm != norm ? 1.0 / norm : 0.;
    const float f2 = f > 1e30 ? 1e30f : 1.f, f1 = (float)(f > 1e30 ? f / 1e30f : f);
    for (long long i = (long long)blockIdx.x * 8 + warp; i < q.all; i += (long long)gridDim.x * 8) {
        const long long r = i / q.per_row;
        const int first = (int)(i - r * q.per_row) * kNormCols, end = min(q.cols, first + kNormCols);
        const T *row = g + r * ldg;
#pragma unroll 2
        for (int c = first + lane * 8; c < end; c += 256) {
            float v[8];
            row8(row, c, end, vec, v);
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] = v[j] * f1 * f2;
            if (planes == 0) {
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    if (c + j < end) {
                        if constexpr (sizeof(T) == 4) out[r * ldo + c + j] = v[j];
                        else out[r * ldo + c + j] = float_to_bf16(v[j]);
                    }
                continue;
            }
            unsigned w[3][4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                if (planes == 3) planes3(v[2 * j], v[2 * j + 1], w[0][j], w[1][j], w[2][j]);
                else planes2(v[2 * j], v[2 * j + 1], w[0][j], w[1][j]);
            }
#pragma unroll
            for (int p = 0; p < 3; ++p)
                if (p < planes)
                    *reinterpret_cast<uint4 *>(dst + p * plane + r * pitch + c) =
                        make_uint4(w[p][0], w[p][1], w[p][2], w[p][3]);
        }
    }
}

struct OrthoPlan {
    int P, p, q;  // planes; smaller and larger side
    GemmPlan gram, poly, apply;
    // of all steps as products, in SM clocks (2,500 more per product than its plan says: the
    // launch)
    double score(int steps) const { return 12000.0 + steps * (gram.score + poly.score + apply.score + 3 * 2500.0); }
};
OrthoPlan plan_ortho(int m, int n, int dtype) {
    OrthoPlan o;
    o.P = dtype == QCNN_F32 ? 3 : 2;
    o.p = std::min(m, n);
    o.q = std::max(m, n);
    // (one side of the diagonal, or both in smaller tiles where that is sooner done)
    const auto sym = [&](int k) {
        const GemmPlan s = plan_gemm(o.P, GEMM_SYM, o.p, o.p, k), f = plan_gemm(o.P, GEMM_PLANES, o.p, o.p, k);
        return f.score < s.score ? f : s;
    };
    o.gram = sym(o.q);
    o.poly = sym(o.p);
    o.apply = m <= n ? plan_gemm(o.P, GEMM_PLANES, o.q, o.p, o.p) : plan_gemm(o.P, GEMM_PLANES, o.p, o.q, o.p);
    return o;
}
struct OrthoSpace {
    double *norm;
    unsigned short *x[2], *a, *b;
    size_t bytes;
};
OrthoSpace carve_ortho(const OrthoPlan &o, int m, int n, void *ws) {
    Carver c{static_cast<uint8_t *>(ws)};
    OrthoSpace s;
    const size_t xs = (size_t)o.P * pad256(m) * pad256(n), as = (size_t)o.P * pad256(o.p) * pad256(o.p);
    s.norm = c.array<double>(kNormBlocks);
    s.x[0] = c.array<unsigned short>(xs);
    s.x[1] = c.array<unsigned short>(xs);
    s.a = c.array<unsigned short>(as);
    s.b = c.array<unsigned short>(as);
    s.bytes = c.used;
    return s;
}

template <typename T>
qcnn_status run_ortho(const T *G, long long ldg, int m, int n, int steps, const float *k, float eps, T *out,
                      long long ldo, const OrthoPlan &o, const OrthoSpace &s, cudaStream_t st) {
    PdlScope pdl;
    const bool wide = m <= n;
    const Pieces q{m, (long long)m * cdiv(n, kNormCols), n, cdiv(n, kNormCols)};
    const int blocks = (int)std::min<long long>(kNormBlocks, (q.all + 7) / 8);
    const int vec = tma_ok(G, ldg, sizeof(T) == 4 ? QCNN_F32 : QCNN_BF16);
    qcnn_status rc = launch_pdl(norm_kernel<T>, dim3(blocks), dim3(256), 0, st, G, ldg, q, vec, s.norm);
    if (rc != QCNN_OK) return rc;
    const long long px = pad256(n), xplane = pad256(m) * px, pa = pad256(o.p), aplane = pa * pa;
    const int grid = (int)std::min<long long>(2 * kNormBlocks, (q.all + 7) / 8);
    rc = launch_pdl(scale_kernel<T>, dim3(grid), dim3(256), 0, st, G, ldg, q, vec, s.norm, blocks, eps,
                    steps ? o.P : 0, s.x[0], px, xplane, out, ldo);
    for (int i = 0; i < steps && rc == QCNN_OK; ++i) {
        const GemmOperand x{s.x[i & 1], px, xplane, 0}, a{s.a, pa, aplane, 0}, b{s.b, pa, aplane, 0};
        GemmProblem g;
        g.a = g.b = x;
        g.a.mn = g.b.mn = wide ? 0 : 1;
        g.m = g.n = o.p;
        g.k = o.q;
        g.e.out = s.a;
        g.e.ldo = pa;
        g.e.out_plane = aplane;
        if ((rc = launch_gemm(o.gram, &g, 1, st)) != QCNN_OK) break;
        g.a = g.b = a;
        g.k = o.p;
        g.e.alpha = k[2];
        g.e.beta = k[1];
        g.e.add = s.a;
        g.e.lda = pa;
        g.e.add_plane = aplane;
        g.e.diagonal = k[0];
        g.e.out = s.b;
        if ((rc = launch_gemm(o.poly, &g, 1, st)) != QCNN_OK) break;
        GemmProblem u;
        u.k = o.p;
        if (wide) {  // X' [p][q] = B X
            u.m = o.q;
            u.n = o.p;
            u.a = x;
            u.a.mn = 1;
            u.b = b;
        } else {  // X' [q][p] = X B
            u.m = o.p;
            u.n = o.q;
            u.a = b;
            u.b = x;
        }
        GemmPlan apply = o.apply;
        if (i + 1 < steps) {
            u.e.out = s.x[(i + 1) & 1];
            u.e.ldo = px;
            u.e.out_plane = xplane;
        } else {
            apply.kind = GEMM_OUT;
            u.e.out = out;
            u.e.ldo = ldo;
            u.e.out_type = sizeof(T) == 4 ? GEMM_T_F32 : GEMM_T_BF16;
        }
        rc = launch_gemm(apply, &u, 1, st);
    }
    return rc;
}

}  // namespace
}  // namespace qcnn

using namespace qcnn;

extern "C" {

qcnn_status qcnn_orthogonalize_workspace_size(int m, int n, int dtype, size_t *bytes) {
    if (!bytes || m <= 0 || n <= 0 || !dtype_ok(dtype)) return QCNN_ERR_INVALID_ARG;
    *bytes = carve_ortho(plan_ortho(m, n, dtype), m, n, nullptr).bytes;
    return QCNN_OK;
}

qcnn_status qcnn_orthogonalize(const void *G, long long ldg, int m, int n, int steps, const float *coeffs,
                               float eps, void *out, long long ldo, int dtype, void *workspace,
                               size_t workspace_bytes, void *stream) {
    if (m <= 0 || n <= 0 || !dtype_ok(dtype) || steps < 0 || steps > 100 || !(eps >= 0.f) ||
        !matrix_ok(G, ldg, m, n, dtype) || !matrix_ok(out, ldo, m, n, dtype))
        return QCNN_ERR_INVALID_ARG;
    static const float muon[3] = {3.4445f, -4.7750f, 2.0315f};
    const float *k = coeffs ? coeffs : muon;
    const cudaStream_t st = static_cast<cudaStream_t>(stream);
    const OrthoPlan o = plan_ortho(m, n, dtype);
    const OrthoSpace s = carve_ortho(o, m, n, workspace);
    const qcnn_status rc = workspace_ok(workspace, workspace_bytes, s.bytes);
    if (rc != QCNN_OK) return rc;
    const OrthoSmall small = ortho_small_plan(m, n, steps, o.score(steps));
    if (small.cluster)
        return launch_ortho_small(small, G, ldg, m, n, steps, k, eps, out, ldo, dtype == QCNN_BF16, st);
    if (dtype == QCNN_F32)
        return run_ortho(static_cast<const float *>(G), ldg, m, n, steps, k, eps, static_cast<float *>(out), ldo, o, s, st);
    return run_ortho(static_cast<const unsigned short *>(G), ldg, m, n, steps, k, eps,
                     static_cast<unsigned short *>(out), ldo, o, s, st);
}

}  // extern "C"
