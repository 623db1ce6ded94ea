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

// --------------------------------------------------------------- quantizer
// The largest magnitude of a row goes by its bits, whose order is that of the values, infinities and
// NaN above all.  |x| / scale <= 127 (1 + 2^-21), so no code is clamped.
struct RowScale {
    float scale, inverse;
    bool finite;
};
__device__ __forceinline__ RowScale row_scale(unsigned top) {
    const float t = __fmul_rn(__uint_as_float(top), kInv127), s = t < 1.17549435e-38f ? 1.17549435e-38f : t;
    const bool finite = top < 0x7f800000u;
    return {s, finite ? __frcp_rn(s) : 0.f, finite};
}
// x / scale to the nearest integer, ties to even: in the low bits of a float around 1.5 2^23.
constexpr float kRound = 12582912.f;
__device__ __forceinline__ float rounded(float x, float inverse) { return __fadd_rn(__fmul_rn(x, inverse), kRound); }

__device__ __forceinline__ unsigned pack_codes(float a, float b, float c, float d) {
    return __byte_perm(__byte_perm(__float_as_uint(a), __float_as_uint(b), 0x0040),
                       __byte_perm(__float_as_uint(c), __float_as_uint(d), 0x0040), 0x5410);
}

struct QuantizeArgs {
    const void *x;
    long long ldx;
    int rows, cols, padded;  // (codes from cols to padded are 0)
    int8_t *codes;
    long long ldc;
    float *scale;
    int wide;  // codes go several at a time
};

// G threads a row (a warp, several or the CTA), which keep up to H vectors of V elements each between
// the two steps; what a row has beyond that is read again.  V: 16 bytes, or (rows off 16 bytes) one
// element.
template <typename T, int G, int H, bool VEC>
__global__ void __launch_bounds__(G > 256 ? G : 256) quantize_kernel(QuantizeArgs a) {
    constexpr int V = VEC ? 16 / (int)sizeof(T) : 1, BLOCK = G > 256 ? G : 256, ROWS = BLOCK / G;
    constexpr int W = VEC ? 4 : 1;  // words of a vector
    __shared__ unsigned red[BLOCK / 32];
    grid_dep_sync();
    const int t = threadIdx.x % G, group = threadIdx.x / G;
    const long long row = (long long)blockIdx.x * ROWS + group;
    const bool is = row < a.rows;
    const T *const x = static_cast<const T *>(a.x) + (is ? row : 0) * a.ldx;
    int8_t *const out = a.codes + (is ? row : 0) * a.ldc;
    const int vectors = is ? a.cols / V : 0;
    struct Vec {
        unsigned w[W];
    };
    auto load = [&](unsigned v) {
        Vec r;
        if constexpr (VEC) {
            const uint4 q = *reinterpret_cast<const uint4 *>(x + (long long)v * V);
            r.w[0] = q.x, r.w[1] = q.y, r.w[2] = q.z, r.w[3] = q.w;
        } else if constexpr (sizeof(T) == 4) {
            r.w[0] = __float_as_uint(x[v]);
        } else {
            r.w[0] = (unsigned)x[v] << 16;
        }
        return r;
    };
    unsigned top = 0;
    auto look = [&](const Vec &r) {
#pragma unroll
        for (int i = 0; i < W; ++i) {
            if constexpr (VEC && sizeof(T) == 2) top = max(top, r.w[i] << 16 & 0x7fff0000u);
            top = max(top, r.w[i] & (VEC && sizeof(T) == 2 ? 0x7fff0000u : 0x7fffffffu));
        }
    };
    Vec kept[H];
#pragma unroll
    for (int h = 0; h < H; ++h)
        if (t + h * G < vectors) kept[h] = load(t + h * G);
#pragma unroll
    for (int h = 0; h < H; ++h)
        if (t + h * G < vectors) look(kept[h]);
#pragma unroll 4
    for (unsigned v = t + H * G; v < (unsigned)vectors; v += G) look(load(v));
    const int rest = VEC && is ? a.cols % V : 0;
    unsigned last = 0;  // (an element of the rest)
    if (t < rest) {
        const T v = x[(long long)vectors * V + t];
        if constexpr (sizeof(T) == 4) last = __float_as_uint(v);
        else last = (unsigned)v << 16;
        top = max(top, last & 0x7fffffffu);
    }
    top = __reduce_max_sync(0xffffffffu, top);
    if constexpr (G > 32) {
        if (threadIdx.x % 32 == 0) red[threadIdx.x / 32] = top;
        __syncthreads();
#pragma unroll
        for (int i = 0; i < G / 32; ++i) top = max(top, red[group * (G / 32) + i]);
    }
    if (!is) return;
    const RowScale s = row_scale(top);
    if (t == 0) a.scale[row] = s.scale;
    auto code = [&](unsigned w) { return rounded(s.finite ? __uint_as_float(w) : 0.f, s.inverse); };
    auto put = [&](unsigned v, const Vec &r) {
        int8_t *const o = out + (long long)v * V;
        if constexpr (!VEC) {
            *o = (int8_t)__float_as_uint(code(r.w[0]));
        } else {
            constexpr int N = V / 4;  // words of codes
            unsigned c[N];
#pragma unroll
            for (int i = 0; i < N; ++i) {
                if constexpr (sizeof(T) == 4)
                    c[i] = pack_codes(code(r.w[0]), code(r.w[1]), code(r.w[2]), code(r.w[3]));
                else
                    c[i] = pack_codes(code(r.w[2 * i] << 16), code(r.w[2 * i] & 0xffff0000u),
                                      code(r.w[2 * i + 1] << 16), code(r.w[2 * i + 1] & 0xffff0000u));
            }
            if (a.wide) {
                if constexpr (N == 1) *reinterpret_cast<unsigned *>(o) = c[0];
                else *reinterpret_cast<uint2 *>(o) = make_uint2(c[0], c[1]);
            } else {
#pragma unroll
                for (int i = 0; i < V; ++i) o[i] = (int8_t)(c[i / 4] >> i % 4 * 8);
            }
        }
    };
#pragma unroll
    for (int h = 0; h < H; ++h)
        if (t + h * G < vectors) put(t + h * G, kept[h]);
#pragma unroll 4
    for (unsigned v = t + H * G; v < (unsigned)vectors; v += G) put(v, load(v));
    if (t < rest) out[(long long)vectors * V + t] = (int8_t)__float_as_uint(code(last));
    for (unsigned c = (unsigned)a.cols + t; c < (unsigned)a.padded; c += G) out[c] = 0;
}

template <typename T>
qcnn_status launch_quantize_of(const QuantizeArgs &a, cudaStream_t st) {
    constexpr int V = 16 / (int)sizeof(T);
    const auto launch = [&](auto k, int G) {
        const int rows = G > 256 ? 1 : 256 / G;
        return launch_pdl(k, dim3((unsigned)((a.rows + (long long)rows - 1) / rows)), dim3(G > 256 ? G : 256), 0, st, a);
    };
    if (reinterpret_cast<uintptr_t>(a.x) % 16 == 0 && (a.ldx % V == 0 || a.rows == 1)) {
        const int vectors = a.cols / V;
        if (vectors <= 128) return launch(quantize_kernel<T, 32, 4, true>, 32);
        if (vectors <= 512) return launch(quantize_kernel<T, 128, 4, true>, 128);
        if (vectors <= 1024) return launch(quantize_kernel<T, 256, 4, true>, 256);
        return launch(quantize_kernel<T, 512, 8, true>, 512);
    }
    if (a.cols <= 256) return launch(quantize_kernel<T, 32, 8, false>, 32);
    if (a.cols <= 2048) return launch(quantize_kernel<T, 128, 16, false>, 128);
    return launch(quantize_kernel<T, 512, 16, false>, 512);
}
qcnn_status launch_quantize(const void *x, long long ldx, int rows, int cols, int8_t *codes, long long ldc,
                            int padded, float *scale, int dtype, cudaStream_t st) {
    const int V = dtype == QCNN_BF16 ? 8 : 4;
    const int wide = reinterpret_cast<uintptr_t>(codes) % V == 0 && (ldc % V == 0 || rows == 1);
    const QuantizeArgs a{x, ldx, rows, cols, padded, codes, ldc, scale, wide};
    return dtype == QCNN_BF16 ? launch_quantize_of<unsigned short>(a, st) : launch_quantize_of<float>(a, st);
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
