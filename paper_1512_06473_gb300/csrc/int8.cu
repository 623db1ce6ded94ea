// int8.cu -- qcnn_int8_quantize and qcnn_int8_dense_forward: rows in 8-bit integers with a scale each,
// and a dense layer of such weights.
//
//   scale = max(max |x| / 127, 2^-126), q = rint(x / scale);
//   y = act(xscale[n] wscale[m] sum_k q[n][k] W[m][k] + bias[m]) + r
#include "train.cuh"

namespace qcnn {
namespace {

constexpr float kInv127 = 1.f / 127.f;
constexpr int kMaxTerms = 131071;  // whose sum of products fits 32 bits

template <typename T>
__device__ __forceinline__ float to_float(T v) {
    if constexpr (sizeof(T) == 4) return v;
    else return bf16_to_float(v);
}

// --------------------------------------------------------------- quantizer
// A CTA per row: its largest magnitude (as bits, whose order is that of the values, infinities and
// NaN above all), then its codes.
template <typename T>
__global__ void __launch_bounds__(256) quantize_kernel(const T *x, long long ldx, int cols, int8_t *codes,
                                                       long long ldc, int padded, float *scale) {
    __shared__ unsigned red[8];
    grid_dep_sync();
    const T *row = x + (long long)blockIdx.x * ldx;
    int8_t *out = codes + (long long)blockIdx.x * ldc;
    unsigned top = 0;
    for (int c = threadIdx.x; c < cols; c += 256) top = max(top, __float_as_uint(to_float(row[c])) & 0x7fffffffu);
    top = __reduce_max_sync(0xffffffffu, top);
    if (threadIdx.x % 32 == 0) red[threadIdx.x / 32] = top;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 8; ++i) top = max(top, red[i]);
    const bool finite = top < 0x7f800000u;
    const float t = __fmul_rn(__uint_as_float(top), kInv127), s = t < 1.17549435e-38f ? 1.17549435e-38f : t;
    const float inverse = __frcp_rn(s);
    for (int c = threadIdx.x; c < padded; c += 256) {
        int q = 0;
        if (finite && c < cols) q = __float2int_rn(__fmul_rn(to_float(row[c]), inverse));
        out[c] = (int8_t)max(-127, min(127, q));
    }
    if (threadIdx.x == 0) scale[blockIdx.x] = s;
}

// ------------------------------------------------------------------ product
struct Int8Product {
    const int8_t *x, *W;
    long long ldx, ldw;
    const float *xscale, *wscale;
    int N, Cs, Ct;
    GemmEpi e;  // bias, act, add (beta 1), out; n = row, m = output
};

// A warp sums four outputs x NB rows, four products at a time (dp4a).
template <int NB, bool VEC>
__global__ void __launch_bounds__(256) few_rows_kernel(Int8Product f) {
    constexpr int OUT = 4;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int c0 = (blockIdx.x * 8 + warp) * OUT, n0 = blockIdx.y * NB;
    grid_dep_sync();
    if (c0 >= f.Ct) return;
    const int8_t *w[OUT], *x[NB];
#pragma unroll
    for (int i = 0; i < OUT; ++i) w[i] = f.W + (long long)min(c0 + i, f.Ct - 1) * f.ldw;
#pragma unroll
    for (int n = 0; n < NB; ++n) x[n] = f.x + (long long)min(n0 + n, f.N - 1) * f.ldx;
    int acc[OUT][NB] = {};
    const int whole = VEC ? f.Cs / 16 * 16 : 0;
    for (int k = lane * 16; k < whole; k += 512) {
        uint4 v[OUT];
#pragma unroll
        for (int i = 0; i < OUT; ++i) v[i] = *reinterpret_cast<const uint4 *>(w[i] + k);
#pragma unroll
        for (int n = 0; n < NB; ++n) {
            const uint4 u = *reinterpret_cast<const uint4 *>(x[n] + k);
#pragma unroll
            for (int i = 0; i < OUT; ++i) {
                acc[i][n] = __dp4a((int)v[i].x, (int)u.x, acc[i][n]);
                acc[i][n] = __dp4a((int)v[i].y, (int)u.y, acc[i][n]);
                acc[i][n] = __dp4a((int)v[i].z, (int)u.z, acc[i][n]);
                acc[i][n] = __dp4a((int)v[i].w, (int)u.w, acc[i][n]);
            }
        }
    }
    for (int k = whole + lane; k < f.Cs; k += 32) {
        int v[OUT];
#pragma unroll
        for (int i = 0; i < OUT; ++i) v[i] = w[i][k];
#pragma unroll
        for (int n = 0; n < NB; ++n)
#pragma unroll
            for (int i = 0; i < OUT; ++i) acc[i][n] += v[i] * x[n][k];
    }
#pragma unroll
    for (int i = 0; i < OUT; ++i)
#pragma unroll
        for (int n = 0; n < NB; ++n) {
            const int sum = __reduce_add_sync(0xffffffffu, acc[i][n]);
            const int m = c0 + i, r = n0 + n;
            if (lane != (i * NB + n) % 32 || m >= f.Ct || r >= f.N) continue;
            const GemmEpi &e = f.e;
            float v = (float)sum * f.xscale[r] * f.wscale[m];
            if (e.bias) v += e.bias[m];
            v = act_apply(v, e.act);
            if (e.add) v += load_as(e.add, e.add_type, (long long)r * e.lda + m);
            if (e.out_type == GEMM_T_F32) static_cast<float *>(e.out)[(long long)r * e.ldo + m] = v;
            else static_cast<unsigned short *>(e.out)[(long long)r * e.ldo + m] = float_to_bf16(v);
        }
}

// ------------------------------------------------------------------- space
struct Space {
    int8_t *codes = nullptr;
    float *scale = nullptr;
    size_t bytes = 0;
};
long long pad16(long long v) { return (v + 15) / 16 * 16; }
Space carve(int N, int Cs, bool x_codes, void *ws) {
    Carver c{static_cast<uint8_t *>(ws)};
    Space s;
    if (!x_codes) {
        s.codes = c.array<int8_t>((size_t)N * pad16(Cs));
        s.scale = c.array<float>(N);
    }
    s.bytes = c.used;
    return s;
}
bool rows16(const void *p, long long ld) { return reinterpret_cast<uintptr_t>(p) % 16 == 0 && ld % 16 == 0; }
bool codes_ok(const void *p, long long ld, long long rows, long long cols) { return ld >= cols && (rows == 0 || p); }

qcnn_status launch_quantize(const void *x, long long ldx, int rows, int cols, int8_t *codes, long long ldc,
                            int padded, float *scale, int dtype, cudaStream_t st) {
    if (dtype == QCNN_BF16)
        return launch_pdl(quantize_kernel<unsigned short>, dim3(rows), dim3(256), 0, st,
                          static_cast<const unsigned short *>(x), ldx, cols, codes, ldc, padded, scale);
    return launch_pdl(quantize_kernel<float>, dim3(rows), dim3(256), 0, st, static_cast<const float *>(x), ldx, cols,
                      codes, ldc, padded, scale);
}

}  // namespace
}  // namespace qcnn

using namespace qcnn;

extern "C" {

qcnn_status qcnn_int8_quantize(const void *x, long long ldx, int N, int C, int8_t *codes, long long ldc,
                               float *scale, int dtype, void *stream) {
    if (N < 0 || C <= 0 || !dtype_ok(dtype) || !matrix_ok(x, ldx, N, C, dtype) || !codes_ok(codes, ldc, N, C) ||
        (N && !scale) || reinterpret_cast<uintptr_t>(scale) % 4)
        return QCNN_ERR_INVALID_ARG;
    if (N == 0) return QCNN_OK;
    return launch_quantize(x, ldx, N, C, codes, ldc, C, scale, dtype, static_cast<cudaStream_t>(stream));
}

qcnn_status qcnn_int8_dense_workspace_size(int N, int Cs, int Ct, int x_codes, int aligned, size_t *bytes) {
    if (!bytes || N < 0 || Cs <= 0 || Cs > kMaxTerms || Ct <= 0) return QCNN_ERR_INVALID_ARG;
    (void)aligned;
    *bytes = N ? carve(N, Cs, x_codes, nullptr).bytes : 0;
    return QCNN_OK;
}

qcnn_status qcnn_int8_dense_forward(const void *x, long long ldx, const float *xscale, int N, int Cs,
                                    const int8_t *W, long long ldw, const float *wscale, int Ct, const float *bias,
                                    int act, const void *residual, long long ldr, void *y, long long ldy, int dtype,
                                    void *workspace, size_t workspace_bytes, void *stream) {
    if (N < 0 || Cs <= 0 || Cs > kMaxTerms || Ct <= 0 || !dtype_ok(dtype) || act < QCNN_ACT_NONE ||
        act > QCNN_ACT_SILU)
        return QCNN_ERR_INVALID_ARG;
    if (!(xscale ? codes_ok(x, ldx, N, Cs) : matrix_ok(x, ldx, N, Cs, dtype)) || !codes_ok(W, ldw, Ct, Cs) ||
        !wscale || !matrix_ok(y, ldy, N, Ct, dtype) || (residual && !matrix_ok(residual, ldr, N, Ct, dtype)) ||
        reinterpret_cast<uintptr_t>(bias) % 4 || reinterpret_cast<uintptr_t>(wscale) % 4 ||
        reinterpret_cast<uintptr_t>(xscale) % 4)
        return QCNN_ERR_INVALID_ARG;
    if (N == 0) return QCNN_OK;
    const Space s = carve(N, Cs, xscale != nullptr, workspace);
    qcnn_status rc = workspace_ok(workspace, workspace_bytes, s.bytes);
    if (rc != QCNN_OK) return rc;
    const cudaStream_t st = static_cast<cudaStream_t>(stream);
    PdlScope pdl;
    Int8Product f;
    f.x = static_cast<const int8_t *>(x);
    f.ldx = ldx;
    f.xscale = xscale;
    if (!xscale) {
        rc = launch_quantize(x, ldx, N, Cs, s.codes, pad16(Cs), (int)pad16(Cs), s.scale, dtype, st);
        if (rc != QCNN_OK) return rc;
        f.x = s.codes;
        f.ldx = pad16(Cs);
        f.xscale = s.scale;
    }
    f.W = W;
    f.ldw = ldw;
    f.wscale = wscale;
    f.N = N;
    f.Cs = Cs;
    f.Ct = Ct;
    const int type = dtype == QCNN_BF16 ? GEMM_T_BF16 : GEMM_T_F32;
    f.e.bias = bias;
    f.e.act = act;
    f.e.add = residual;
    f.e.lda = ldr;
    f.e.add_type = type;
    f.e.out = y;
    f.e.ldo = ldy;
    f.e.out_type = type;
    const bool vec = rows16(f.x, f.ldx) && rows16(W, ldw);
    const dim3 grid(cdiv(Ct, 32), cdiv(N, N > 4 ? 8 : N));
    if (grid.y > 65535) return QCNN_ERR_UNSUPPORTED;
    const auto launch = [&](auto k) { return launch_pdl(k, grid, dim3(256), 0, st, f); };
    if (N == 1) return launch(vec ? few_rows_kernel<1, true> : few_rows_kernel<1, false>);
    if (N == 2) return launch(vec ? few_rows_kernel<2, true> : few_rows_kernel<2, false>);
    if (N <= 4) return launch(vec ? few_rows_kernel<4, true> : few_rows_kernel<4, false>);
    return launch(vec ? few_rows_kernel<8, true> : few_rows_kernel<8, false>);
}

}  // extern "C"
