// orthogonalize.cu -- qcnn_orthogonalize: Newton-Schulz products.
//
//   X = G / (||G||_F + eps); steps times: A = X X^T, B = b A + c A A, X = a X + B X
//
// of the smaller side p (q the larger; G with more rows than columns from the right, by
// reading X with its rows contiguous: nothing is transposed).  Three products a step, of
// 2 p^2 q, 2 p^3 and 2 p^2 q operations; A and B are symmetric, so of the first two the
// tiles on one side of the diagonal are computed and stored twice.  X, A and B live as bf16
// planes that the epilogues write and TMA reads: two in bf16 calls (in one, each step's
// rounding of X and B would be that of the result), three in fp32 calls.
#include "train.cuh"

#include <algorithm>

namespace qcnn {
namespace {

constexpr int kNormBlocks = 304;

template <typename T>
__device__ __forceinline__ float value(const T *p) {
    if constexpr (sizeof(T) == 4) return *p;
    else return bf16_to_float(*p);
}

// Sums of squares by CTA: of values above 2^48 scaled by 2^-64, and of the others (whose
// squares neither overflow nor, where they count beside eps, vanish).
constexpr float kLarge = 281474976710656.f, kLargeScale = 5.421010862427522e-20f;
template <typename T>
__global__ void __launch_bounds__(256) norm_kernel(const T *g, long long ldg, long long rows, int cols, int vec,
                                                   double2 *part) {
    __shared__ double2 red[8];
    grid_dep_sync();
    float small = 0.f, large = 0.f;
    double dsmall = 0., dlarge = 0.;
    const int c4 = (cols + 3) / 4;
    const long long all = rows * c4;
    int n = 0;
    for (long long i = (long long)blockIdx.x * 256 + threadIdx.x; i < all; i += (long long)gridDim.x * 256) {
        const long long r = i / c4;
        const int c = (int)(i - r * c4) * 4;
        const T *s = g + r * ldg + c;
        float v[4];
        if (vec && c + 4 <= cols) {
            if constexpr (sizeof(T) == 4) {
                const float4 a = *reinterpret_cast<const float4 *>(s);
                v[0] = a.x, v[1] = a.y, v[2] = a.z, v[3] = a.w;
            } else {
                const uint2 a = *reinterpret_cast<const uint2 *>(s);
                v[0] = __uint_as_float(a.x << 16), v[1] = __uint_as_float(a.x & 0xffff0000u);
                v[2] = __uint_as_float(a.y << 16), v[3] = __uint_as_float(a.y & 0xffff0000u);
            }
        } else {
#pragma unroll
            for (int j = 0; j < 4; ++j) v[j] = c + j < cols ? value(s + j) : 0.f;
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const bool big = fabsf(v[j]) > kLarge;
            const float w = big ? v[j] * kLargeScale : v[j];
            if (big) large = fmaf(w, w, large);
            else small = fmaf(w, w, small);  // (NaN too)
        }
        if (++n == 16) {  // (runs of 64 squares in fp32)
            dsmall += small;
            dlarge += large;
            small = large = 0.f;
            n = 0;
        }
    }
    dsmall += small;
    dlarge += large;
#pragma unroll
    for (int o = 16; o; o >>= 1) {
        dsmall += __shfl_xor_sync(0xffffffffu, dsmall, o);
        dlarge += __shfl_xor_sync(0xffffffffu, dlarge, o);
    }
    if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = make_double2(dsmall, dlarge);
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int i = 1; i < 8; ++i) {
            dsmall += red[i].x;
            dlarge += red[i].y;
        }
        part[blockIdx.x] = make_double2(dsmall, dlarge);
    }
}

// X = G / (norm + eps) in planes (or, planes 0, as the result); every CTA adds the sums up
// in the same order.
template <typename T>
__global__ void __launch_bounds__(256) scale_kernel(const T *g, long long ldg, long long rows, int cols,
                                                    const double2 *part, int parts, float eps, int planes,
                                                    unsigned short *dst, long long plane, T *out, long long ldo) {
    __shared__ double2 red[256];
    grid_dep_sync();
    double2 s = make_double2(0., 0.);
    for (int i = threadIdx.x; i < parts; i += 256) {
        s.x += part[i].x;
        s.y += part[i].y;
    }
    red[threadIdx.x] = s;
    __syncthreads();
    for (int o = 128; o; o >>= 1) {
        if ((int)threadIdx.x < o) {
            red[threadIdx.x].x += red[threadIdx.x + o].x;
            red[threadIdx.x].y += red[threadIdx.x + o].y;
        }
        __syncthreads();
    }
    const double norm = sqrt(red[0].x + red[0].y * 340282366920938463463374607431768211456.0) + (double)eps;
    // (a norm of zero with eps zero: the matrix is zero; a factor above fp32's range is
    // taken in two)
    const double f = norm > 0. || norm != norm ? 1.0 / norm : 0.;
    const int c8 = (cols + 7) / 8;
    const long long pitch = (long long)c8 * 8, all = rows * c8;
    for (long long i = (long long)blockIdx.x * 256 + threadIdx.x; i < all; i += (long long)gridDim.x * 256) {
        const long long r = i / c8;
        const int c = (int)(i - r * c8) * 8;
        float v[8];
        const float ff = (float)f;
        const bool plain = ff < 3e38f;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const float x = c + j < cols ? value(g + r * ldg + c + j) : 0.f;
            v[j] = plain ? x * ff : (float)(x * f);
        }
        if (planes == 0) {
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (c + j < cols) {
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

struct OrthoPlan {
    int P, p, q;  // planes; smaller and larger side
    Product gram, poly, apply;
};
OrthoPlan plan_ortho(int m, int n, int dtype) {
    OrthoPlan o;
    o.P = dtype == QCNN_F32 ? 3 : 2;
    o.p = std::min(m, n);
    o.q = std::max(m, n);
    o.gram.plan = plan_gemm(o.P, GEMM_SYM, o.p, o.p, o.q, 1);
    o.poly.plan = plan_gemm(o.P, GEMM_SYM, o.p, o.p, o.p, 1);
    o.apply.plan = m <= n ? plan_gemm(o.P, GEMM_OUT, o.q, o.p, o.p, 64) : plan_gemm(o.P, GEMM_OUT, o.p, o.q, o.p, 64);
    return o;
}
struct OrthoSpace {
    double2 *norm;
    unsigned short *x[2], *a, *b;
    void *partial;
    size_t bytes;
};
OrthoSpace carve_ortho(const OrthoPlan &o, int m, int n, void *ws) {
    Carver c{static_cast<uint8_t *>(ws)};
    OrthoSpace s;
    const size_t xs = (size_t)o.P * m * pad8(n), as = (size_t)o.P * o.p * pad8(o.p);
    s.norm = c.array<double2>(kNormBlocks);
    s.x[0] = c.array<unsigned short>(xs);
    s.x[1] = c.array<unsigned short>(xs);
    s.a = c.array<unsigned short>(as);
    s.b = c.array<unsigned short>(as);
    s.partial = c.take(o.apply.scratch());
    s.bytes = c.used;
    return s;
}

template <typename T>
qcnn_status run_ortho(const T *G, long long ldg, int m, int n, int steps, const float *k, float eps, T *out,
                      long long ldo, const OrthoPlan &o, const OrthoSpace &s, cudaStream_t st) {
    PdlScope pdl;
    const bool wide = m <= n;
    const long long all = (long long)m * cdiv(n, 4);
    const int blocks = (int)std::min<long long>(kNormBlocks, (all + 255) / 256);
    const int vec = reinterpret_cast<uintptr_t>(G) % (4 * sizeof(T)) == 0 && ldg % 4 == 0;
    qcnn_status rc = launch_pdl(norm_kernel<T>, dim3(blocks), dim3(256), 0, st, G, ldg, (long long)m, n, vec, s.norm);
    if (rc != QCNN_OK) return rc;
    const long long px = pad8(n), xplane = m * px, pa = pad8(o.p), aplane = o.p * pa;
    const int grid = (int)std::min<long long>(((long long)m * cdiv(n, 8) + 255) / 256, (long long)num_sms() * 8);
    rc = launch_pdl(scale_kernel<T>, dim3(grid), dim3(256), 0, st, G, ldg, (long long)m, n, s.norm, blocks, eps,
                    steps ? o.P : 0, s.x[0], xplane, out, ldo);
    for (int i = 0; i < steps && rc == QCNN_OK; ++i) {
        const GemmOperand x{s.x[i & 1], px, xplane, 0}, a{s.a, pa, aplane, 0}, b{s.b, pa, aplane, 0};
        const int type = o.P;  // GEMM_T_PLANES2, GEMM_T_PLANES3
        GemmProblem g;
        g.a = g.b = x;
        g.a.mn = g.b.mn = wide ? 0 : 1;
        g.m = g.n = o.p;
        g.k = o.q;
        g.e.out = s.a;
        g.e.ldo = pa;
        g.e.out_plane = aplane;
        g.e.out_type = type;
        if ((rc = launch_gemm(o.gram.plan, &g, 1, st)) != QCNN_OK) break;
        g.a = g.b = a;
        g.k = o.p;
        g.e.alpha = k[2];
        g.e.beta = k[1];
        g.e.add = s.a;
        g.e.lda = pa;
        g.e.add_plane = aplane;
        g.e.add_type = type;
        g.e.out = s.b;
        if ((rc = launch_gemm(o.poly.plan, &g, 1, st)) != QCNN_OK) break;
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
        u.e.beta = k[0];
        u.e.add = s.x[i & 1];
        u.e.lda = px;
        u.e.add_plane = xplane;
        u.e.add_type = type;
        if (i + 1 < steps) {
            u.e.out = s.x[i + 1 & 1];
            u.e.ldo = px;
            u.e.out_plane = xplane;
            u.e.out_type = type;
        } else {
            u.e.out = out;
            u.e.ldo = ldo;
            u.e.out_type = sizeof(T) == 4 ? GEMM_T_F32 : GEMM_T_BF16;
        }
        rc = o.apply.run(u, s.partial, st);
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
    const OrthoPlan o = plan_ortho(m, n, dtype);
    const OrthoSpace s = carve_ortho(o, m, n, workspace);
    const qcnn_status rc = workspace_ok(workspace, workspace_bytes, s.bytes);
    if (rc != QCNN_OK) return rc;
    static const float muon[3] = {3.4445f, -4.7750f, 2.0315f};
    const float *k = coeffs ? coeffs : muon;
    const cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (dtype == QCNN_F32)
        return run_ortho(static_cast<const float *>(G), ldg, m, n, steps, k, eps, static_cast<float *>(out), ldo, o, s, st);
    return run_ortho(static_cast<const unsigned short *>(G), ldg, m, n, steps, k, eps,
                     static_cast<unsigned short *>(out), ldo, o, s, st);
}

}  // extern "C"
