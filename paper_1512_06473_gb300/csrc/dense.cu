// dense.cu -- qcnn_dense_forward and qcnn_dense_backward: a dense layer with its epilogue,
// and its gradients.
//
//   z = x W^T + b, y = act(z) + r;   dz = dy * act'(z), dx = dz W, dW = dz^T x, db = sum dz
//
// Each product is gemm.cuh's, with the layer's outputs (dx, dW: its inputs) as the
// contiguous index m.  Three ways, by the estimated time of each:
//   few rows (forward, N <= 4, or 8 where few_rows_sooner says so): no tensor cores; the
//     weights are streamed once through fp32 multiply-adds;
//   fp32 weights split on their way to the tensor cores: no pass over them, so it has the
//     products that their bytes bound (the other operand's planes are small then): 128 x 9216
//     -> 4096 56 us, 127 with planes; backward of 128 x 4096 -> 4096 70 and 101;
//   all operands as planes in the workspace (fp32), or the bf16 operands themselves.
#include "train.cuh"

#include <algorithm>
#include <type_traits>
#include <utility>

namespace qcnn {
namespace {

// ------------------------------------------------------------- few rows
// A warp sums kFewOut outputs x NB rows over its part of the inputs: lanes take
// neighbouring 16 bytes (VEC) or elements.  kw warps share an output's inputs and add up
// through shared memory; 8 / kw groups of kFewOut outputs per CTA.  The rows x are
// read from L1/L2 once per kFewOut weights rows.
constexpr int kFewOut = 4;

template <typename T>
__device__ __forceinline__ float as_float(T v) {
    if constexpr (sizeof(T) == 4) return v;
    else return bf16_to_float(v);
}
// V neighbouring elements (16 bytes)
template <typename T, int V>
__device__ __forceinline__ void load_vec(const T *p, float (&v)[V]) {
    if constexpr (sizeof(T) == 4) {
        const float4 a = *reinterpret_cast<const float4 *>(p);
        v[0] = a.x, v[1] = a.y, v[2] = a.z, v[3] = a.w;
    } else {
        const uint4 a = *reinterpret_cast<const uint4 *>(p);
        const unsigned w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            v[2 * j] = __uint_as_float(w[j] << 16);
            v[2 * j + 1] = __uint_as_float(w[j] & 0xffff0000u);
        }
    }
}

// (Eight rows: two CTAs per SM for loads in flight; with one, 8 rows of 4096 -> 19456 in fp32
// took 111 us, with two 83.  One row takes 47, 6.8 TB/s, four 51.)
template <typename T, int NB, bool VEC>
__global__ void __launch_bounds__(256, NB == 8 ? 2 : 1) few_rows_kernel(FewRows f, int kw) {
    constexpr int V = VEC ? 16 / (int)sizeof(T) : 4;
    __shared__ float red[8][kFewOut * NB];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int group = warp / kw, part = warp - group * kw;
    const int c0 = (blockIdx.x * (8 / kw) + group) * kFewOut;
    grid_dep_sync();
    const T *x = static_cast<const T *>(f.x), *w = static_cast<const T *>(f.W);
    float acc[kFewOut][NB] = {};
    const T *wr[kFewOut];
#pragma unroll
    for (int i = 0; i < kFewOut; ++i) wr[i] = w + (long long)min(c0 + i, f.Ct - 1) * f.ldw;
    const T *xr[NB];
#pragma unroll
    for (int n = 0; n < NB; ++n) xr[n] = x + (long long)min(n, f.N - 1) * f.ldx;
    const int step = kw * 32 * V;
    // (VEC: Cs is a multiple of V)
    if constexpr (VEC) {
#pragma unroll(NB * V <= 8 ? 4 : 2)
        for (int k = (part * 32 + lane) * V; k < f.Cs; k += step) {
            float wv[kFewOut][V];
#pragma unroll
            for (int i = 0; i < kFewOut; ++i) load_vec<T, V>(wr[i] + k, wv[i]);
#pragma unroll
            for (int n = 0; n < NB; ++n) {
                float xv[V];
                load_vec<T, V>(xr[n] + k, xv);
#pragma unroll
                for (int i = 0; i < kFewOut; ++i)
#pragma unroll
                    for (int j = 0; j < V; ++j) acc[i][n] = fmaf(wv[i][j], xv[j], acc[i][n]);
            }
        }
    } else {
        for (int k0 = part * 32 * V + lane; k0 < f.Cs; k0 += step) {
            float wv[kFewOut][V];
#pragma unroll
            for (int i = 0; i < kFewOut; ++i)
#pragma unroll
                for (int j = 0; j < V; ++j) wv[i][j] = k0 + j * 32 < f.Cs ? as_float<T>(wr[i][k0 + j * 32]) : 0.f;
#pragma unroll
            for (int n = 0; n < NB; ++n)
#pragma unroll
                for (int j = 0; j < V; ++j) {
                    const float xv = k0 + j * 32 < f.Cs ? as_float<T>(xr[n][k0 + j * 32]) : 0.f;
#pragma unroll
                    for (int i = 0; i < kFewOut; ++i) acc[i][n] = fmaf(wv[i][j], xv, acc[i][n]);
                }
        }
    }
#pragma unroll
    for (int i = 0; i < kFewOut; ++i)
#pragma unroll
        for (int n = 0; n < NB; ++n) {
            float v = acc[i][n];
#pragma unroll
            for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
            if (lane == 0) red[warp][i * NB + n] = v;
        }
    __syncthreads();
    // one thread per output of the CTA
    const int per = kFewOut * NB, t = threadIdx.x;
    if (t >= (8 / kw) * per) return;
    const int g = t / per, o = t - g * per;
    // (neighbouring threads: neighbouring outputs of a row)
    const int i = o % kFewOut, n = o / kFewOut;
    const int m = (blockIdx.x * (8 / kw) + g) * kFewOut + i;
    if (m >= f.Ct || n >= f.N) return;
    float v = 0.f;
    for (int p = 0; p < kw; ++p) v += red[g * kw + p][i * NB + n];
    const GemmEpi &e = f.e;
    if (e.bias) v += e.bias[m];
    auto put = [&](void *p, long long ld, float r) {
        if (e.out_type == GEMM_T_F32) static_cast<float *>(p)[(long long)n * ld + m] = r;
        else static_cast<unsigned short *>(p)[(long long)n * ld + m] = float_to_bf16(r);
    };
    if (e.pre) put(e.pre, e.ldp, v);
    v = act_apply(v, e.act);
    if (e.add) v += load_as(e.add, e.add_type, (long long)n * e.lda + m);
    put(e.out, e.ldo, v);
}

template <typename T, bool VEC>
qcnn_status few_rows_of(const FewRows &f, cudaStream_t st) {
    constexpr int V = VEC ? 16 / (int)sizeof(T) : 4;
    // as many warps to an output as have inputs, and fewer where outputs alone fill the SMs
    int kw = 8;
    while (kw > 1 && (f.Cs <= kw / 2 * 32 * V || cdiv(f.Ct, kFewOut * 8 / (kw / 2)) >= num_sms() * 4)) kw /= 2;
    const dim3 grid(cdiv(f.Ct, kFewOut * 8 / kw));
    if (f.N == 1) return launch_pdl(few_rows_kernel<T, 1, VEC>, grid, dim3(256), 0, st, f, kw);
    if (f.N == 2) return launch_pdl(few_rows_kernel<T, 2, VEC>, grid, dim3(256), 0, st, f, kw);
    if (f.N <= 4) return launch_pdl(few_rows_kernel<T, 4, VEC>, grid, dim3(256), 0, st, f, kw);
    return launch_pdl(few_rows_kernel<T, 8, VEC>, grid, dim3(256), 0, st, f, kw);
}

// ------------------------------------------------- gradient of z, bias
// dz = dy * act'(z) in planes (out null: only sums) and sums over a slab of rows:
// part[slab][cols].  A CTA takes 128 columns x a slab: a warp a row, a lane four
// columns: neighbours (VEC), or 32 apart, so that rows off the 8- or 16-byte alignment are
// read and written by neighbouring lanes too (3001 x 5003 in bf16 41 us with the lane's four
// next to each other).  JOBS: CTAs past dz's copy the other operands that need it, a launch less
// (backward of 128 x 4096 -> 4096 in fp32 69 us, 71 apart; with the copies' code in it, dz of 3001
// x 5003 alone takes 10 us more).
template <typename T, bool VEC, bool JOBS>
__global__ void __launch_bounds__(256) dz_kernel(const T *dy, long long lddy, const T *pre, long long ldp,
                                                 int N, int Ct, int act, unsigned short *out, int planes,
                                                 long long ldo, long long plane, float *part, int slab, int slabs,
                                                 PlanesJob j0, PlanesJob j1) {
    __shared__ float red[8][128];
    grid_dep_sync();
    int slab_at = blockIdx.y, tile = blockIdx.x;
    if constexpr (JOBS) {
        const int tiles = (Ct + 127) / 128, other = (int)blockIdx.x - tiles * slabs;
        if (other >= 0) {
            if (other < j0.blocks) planes_part<T>(j0, other);
            else planes_part<T>(j1, other - j0.blocks);
            return;
        }
        slab_at = (int)blockIdx.x / tiles;
        tile = (int)blockIdx.x - slab_at * tiles;
    }
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    constexpr int GAP = VEC ? 1 : 32;
    const int own = VEC ? lane * 4 : lane, c = tile * 128 + own;
    const int r1 = min(N, (slab_at + 1) * slab);
    float sum[4] = {};
    auto load4 = [&](const T *p, float (&v)[4]) {
        if (VEC && c + 4 <= Ct) {
            if constexpr (sizeof(T) == 4) {
                const float4 a = *reinterpret_cast<const float4 *>(p);
                v[0] = a.x, v[1] = a.y, v[2] = a.z, v[3] = a.w;
            } else {
                const uint2 a = *reinterpret_cast<const uint2 *>(p);
                v[0] = __uint_as_float(a.x << 16), v[1] = __uint_as_float(a.x & 0xffff0000u);
                v[2] = __uint_as_float(a.y << 16), v[3] = __uint_as_float(a.y & 0xffff0000u);
            }
        } else {
#pragma unroll
            for (int j = 0; j < 4; ++j) v[j] = c + j * GAP < Ct ? as_float<T>(p[j * GAP]) : 0.f;
        }
    };
    if (c < Ct) {
#pragma unroll 4
        for (int r = slab_at * slab + warp; r < r1; r += 8) {
            float v[4];
            load4(dy + (long long)r * lddy + c, v);
            if (act != QCNN_ACT_NONE) {
                float z[4];
                load4(pre + (long long)r * ldp + c, z);
#pragma unroll
                for (int j = 0; j < 4; ++j) v[j] *= act_slope(z[j], act);
            }
#pragma unroll
            for (int j = 0; j < 4; ++j) sum[j] += v[j];
            if (out) {  // (its rows are ours: multiples of 8 elements, 16-byte aligned)
                unsigned w[3][2];
                unsigned short *d = out + (long long)r * ldo + c;
#pragma unroll
                for (int j = 0; j < 2; ++j)
                    planes_of<sizeof(T) == 4>(v[2 * j], v[2 * j + 1], w[0][j], w[1][j], w[2][j]);
#pragma unroll
                for (int i = 0; i < 3; ++i, d += plane) {
                    if (i >= planes) break;
                    if constexpr (VEC) {
                        *reinterpret_cast<uint2 *>(d) = make_uint2(w[i][0], w[i][1]);
                    } else {
#pragma unroll
                        for (int j = 0; j < 4; ++j)
                            if (c + j * GAP < Ct) d[j * GAP] = (unsigned short)(w[i][j / 2] >> (j & 1) * 16);
                    }
                }
            }
        }
    }
    if (!part) return;
#pragma unroll
    for (int j = 0; j < 4; ++j) red[warp][own + j * GAP] = sum[j];
    __syncthreads();
    const int t = threadIdx.x, col = tile * 128 + t;
    if (t < 128 && col < Ct) {
        float v = 0.f;
#pragma unroll
        for (int w = 0; w < 8; ++w) v += red[w][t];
        part[(long long)slab_at * Ct + col] = v;
    }
}

// A CTA takes 32 columns; eight warps an eighth of the rows each, added up in their order.
__global__ void __launch_bounds__(256) column_join_kernel(const float *part, int rows, long long ld, int cols,
                                                          const float *scale, float *dst) {
    __shared__ float red[8][32];
    grid_dep_sync();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, c = blockIdx.x * 32 + lane;
    const int per = (rows + 7) / 8, r0 = min(rows, warp * per), r1 = min(rows, r0 + per);
    red[warp][lane] = c < cols ? add_groups<true>(part + (long long)r0 * ld + c, r1 - r0, ld) : 0.f;
    __syncthreads();
    if (warp == 0 && c < cols) {
        float v = red[0][lane];
#pragma unroll
        for (int w = 1; w < 8; ++w) v += red[w][lane];
        dst[c] = v * (scale ? *scale : 1.f);
    }
}

// Rows per CTA of dz_kernel: enough CTAs to fill the SMs twice, 32 rows at least.
int dz_slab(int N, int Ct) {
    const int want = std::max(1, 4 * num_sms() / cdiv(Ct, 128));
    return std::max(32, cdiv(cdiv(N, want), 8) * 8);
}

// ---------------------------------------------------------------- plans
// fp32: rows (x, dz) always as planes; wplanes: the weights too.  bf16: copies of what
// TMA cannot read.
struct ForwardPlan {
    bool few = false, wplanes = false;
    GemmPlan g;
};
ForwardPlan plan_forward(int N, int Cs, int Ct, int dtype, bool wa) {
    ForwardPlan p;
    if (dtype == QCNN_BF16) {
        p.g = plan_gemm(1, GEMM_OUT, Ct, N, Cs);
    } else {
        p.g = plan_gemm(GEMM_F32, GEMM_OUT, Ct, N, Cs);
        const GemmPlan q = plan_gemm(3, GEMM_OUT, Ct, N, Cs);
        if (q.score + pass_clocks((double)Ct * Cs * 10.0) < p.g.score) {
            p.wplanes = true;
            p.g = q;
        }
    }
    p.few = few_rows_sooner(N, Cs, Ct, dtype == QCNN_BF16, wa, p.g);
    return p;
}
struct ForwardSpace {
    unsigned short *x = nullptr, *w = nullptr;
    size_t bytes = 0;
};
ForwardSpace carve_forward(const ForwardPlan &p, int N, int Cs, int Ct, int dtype, bool xa, bool wa, void *ws) {
    Carver c{static_cast<uint8_t *>(ws)};
    ForwardSpace s;
    if (p.few) return s;
    const bool bf16 = dtype == QCNN_BF16;
    const int P = bf16 ? 1 : 3;
    const bool x_copy = !bf16 || !xa;
    if (x_copy) s.x = c.array<unsigned short>((size_t)P * N * pad8(Cs));
    if (bf16 ? !wa : p.wplanes) s.w = c.array<unsigned short>((size_t)P * Ct * pad8(Cs));
    s.bytes = c.used;
    return s;
}

struct BackwardPlan {
    bool wplanes = false;
    int slab = 0, slabs = 1;
    GemmPlan gx, gw;
};
BackwardPlan plan_backward(int N, int Cs, int Ct, int dtype) {
    BackwardPlan p;
    p.slab = dz_slab(N, Ct);
    p.slabs = cdiv(N, p.slab);
    const int P = dtype == QCNN_BF16 ? 1 : 3;
    p.gw = plan_gemm(P, GEMM_OUT, Cs, Ct, N);
    p.gx = plan_gemm(P, GEMM_OUT, Cs, N, Ct);
    p.wplanes = true;
    if (P == 3) {
        const GemmPlan q = plan_gemm(GEMM_F32, GEMM_OUT, Cs, N, Ct);
        if (q.score <= p.gx.score + pass_clocks((double)Ct * Cs * 10.0)) {
            p.wplanes = false;
            p.gx = q;
        }
    }
    return p;
}
struct BackwardSpace {
    void *dz = nullptr;
    unsigned short *x = nullptr, *w = nullptr;
    float *db = nullptr;
    size_t bytes = 0;
};
BackwardSpace carve_backward(const BackwardPlan &p, int N, int Cs, int Ct, int dtype, bool dz, bool x_copy,
                             bool w_copy, void *ws) {
    Carver c{static_cast<uint8_t *>(ws)};
    BackwardSpace s;
    const size_t P = dtype == QCNN_BF16 ? 1 : 3;
    if (dz) s.dz = c.take(P * N * pad8(Ct) * 2);
    if (x_copy) s.x = c.array<unsigned short>(P * N * pad8(Cs));
    if (w_copy) s.w = c.array<unsigned short>(P * Ct * pad8(Cs));
    if (p.slabs > 1) s.db = c.array<float>((size_t)p.slabs * Ct);
    s.bytes = c.used;
    return s;
}

}  // namespace

qcnn_status launch_few_rows(const FewRows &f, cudaStream_t st) {
    const int v = f.bf16 ? 8 : 4;
    const bool vec = reinterpret_cast<uintptr_t>(f.x) % 16 == 0 && reinterpret_cast<uintptr_t>(f.W) % 16 == 0 &&
                     f.ldx % v == 0 && f.ldw % v == 0 && f.Cs % v == 0;
    if (f.bf16) return vec ? few_rows_of<unsigned short, true>(f, st) : few_rows_of<unsigned short, false>(f, st);
    return vec ? few_rows_of<float, true>(f, st) : few_rows_of<float, false>(f, st);
}

qcnn_status launch_column_join(const float *part, int rows, long long ld, int cols, const float *scale,
                               float *dst, cudaStream_t st) {
    return launch_pdl(column_join_kernel, dim3(cdiv(cols, 32)), dim3(256), 0, st, part, rows, ld, cols, scale, dst);
}

}  // namespace qcnn

using namespace qcnn;

extern "C" {

qcnn_status qcnn_dense_forward_workspace_size(int N, int Cs, int Ct, int dtype, int aligned,
                                              size_t *bytes) {
    if (!bytes || N < 0 || Cs <= 0 || Ct <= 0 || !dtype_ok(dtype)) return QCNN_ERR_INVALID_ARG;
    *bytes = 0;
    if (N == 0) return QCNN_OK;
    for (int wa = 0; wa < 2; ++wa) {  // (of fp32 calls, `aligned` says nothing)
        if (!wa && aligned && dtype == QCNN_BF16) continue;
        const ForwardPlan p = plan_forward(N, Cs, Ct, dtype, wa);
        *bytes = std::max(*bytes, carve_forward(p, N, Cs, Ct, dtype, aligned, aligned, nullptr).bytes);
    }
    return QCNN_OK;
}

qcnn_status qcnn_dense_forward(const void *x, long long ldx, int N, int Cs, const void *W, long long ldw,
                               int Ct, const float *bias, int act, const void *residual, long long ldr,
                               void *y, long long ldy, void *pre, long long ldp, int dtype,
                               void *workspace, size_t workspace_bytes, void *stream) {
    if (N < 0 || Cs <= 0 || Ct <= 0 || !dtype_ok(dtype) || act < QCNN_ACT_NONE || act > QCNN_ACT_SILU)
        return QCNN_ERR_INVALID_ARG;
    if (!matrix_ok(x, ldx, N, Cs, dtype) || !matrix_ok(W, ldw, Ct, Cs, dtype) ||
        !matrix_ok(y, ldy, N, Ct, dtype) || (residual && !matrix_ok(residual, ldr, N, Ct, dtype)) ||
        (pre && !matrix_ok(pre, ldp, N, Ct, dtype)) || reinterpret_cast<uintptr_t>(bias) % 4)
        return QCNN_ERR_INVALID_ARG;
    if (N == 0) return QCNN_OK;
    const bool bf16 = dtype == QCNN_BF16;
    const bool xa = tma_ok(x, ldx, dtype), wa = weights_ok(W, ldw, dtype);
    const ForwardPlan p = plan_forward(N, Cs, Ct, dtype, wa);
    const ForwardSpace s = carve_forward(p, N, Cs, Ct, dtype, xa, wa, workspace);
    qcnn_status rc = workspace_ok(workspace, workspace_bytes, s.bytes);
    if (rc != QCNN_OK) return rc;
    const cudaStream_t st = static_cast<cudaStream_t>(stream);
    PdlScope pdl;
    GemmProblem g;
    const int type = bf16 ? GEMM_T_BF16 : GEMM_T_F32;
    g.e.bias = bias;
    g.e.act = act;
    g.e.beta = 1.f;
    g.e.add = residual;
    g.e.lda = ldr;
    g.e.add_type = type;
    g.e.out = y;
    g.e.ldo = ldy;
    g.e.out_type = type;
    g.e.pre = pre;
    g.e.ldp = ldp;
    if (p.few) return launch_few_rows(FewRows{x, W, ldx, ldw, N, Cs, Ct, bf16, g.e}, st);
    g.m = Ct;
    g.n = N;
    g.k = Cs;
    g.a = GemmOperand{W, ldw, 0, 0};
    g.b = GemmOperand{x, ldx, 0, 0};
    const int P = bf16 ? 1 : 3;
    const long long pitch = pad8(Cs);
    PlanesJob jobs[2];
    if (s.x) {
        jobs[0] = planes_job(x, bf16, N, Cs, ldx, P, s.x);
        g.b = GemmOperand{s.x, pitch, N * pitch, 0};
    }
    if (s.w) {
        jobs[1] = planes_job(W, bf16, Ct, Cs, ldw, P, s.w);
        g.a = GemmOperand{s.w, pitch, Ct * pitch, 0};
    }
    if ((rc = launch_planes(jobs[0], jobs[1], bf16, st)) != QCNN_OK) return rc;
    return launch_gemm(p.g, &g, 1, st);
}

qcnn_status qcnn_dense_backward_workspace_size(int N, int Cs, int Ct, int dtype, int aligned,
                                               size_t *bytes) {
    if (!bytes || N < 0 || Cs <= 0 || Ct <= 0 || !dtype_ok(dtype)) return QCNN_ERR_INVALID_ARG;
    const BackwardPlan p = plan_backward(N, Cs, Ct, dtype);
    const bool f32 = dtype == QCNN_F32;
    *bytes = N ? carve_backward(p, N, Cs, Ct, dtype, true, f32 || !aligned, f32 ? p.wplanes : !aligned, nullptr).bytes
               : 0;
    return QCNN_OK;
}

qcnn_status qcnn_dense_backward(const void *dy, long long lddy, const void *x, long long ldx, const void *W,
                                long long ldw, const void *pre, long long ldp, int N, int Cs, int Ct,
                                int act, void *dx, long long lddx, void *dW, long long lddw,
                                float *dbias, int dtype, void *workspace, size_t workspace_bytes,
                                void *stream) {
    if (N < 0 || Cs <= 0 || Ct <= 0 || !dtype_ok(dtype) || act < QCNN_ACT_NONE || act > QCNN_ACT_SILU)
        return QCNN_ERR_INVALID_ARG;
    if (!matrix_ok(dy, lddy, N, Ct, dtype) || (dW && !matrix_ok(x, ldx, N, Cs, dtype)) ||
        (dx && !matrix_ok(W, ldw, Ct, Cs, dtype)) ||
        (act != QCNN_ACT_NONE && !matrix_ok(pre, ldp, N, Ct, dtype)) ||
        (dx && !matrix_ok(dx, lddx, N, Cs, dtype)) || (dW && !matrix_ok(dW, lddw, Ct, Cs, dtype)) ||
        reinterpret_cast<uintptr_t>(dbias) % 4)
        return QCNN_ERR_INVALID_ARG;
    const cudaStream_t st = static_cast<cudaStream_t>(stream);
    const bool bf16 = dtype == QCNN_BF16;
    if (N == 0) {  // sums of nothing
        cudaError_t e = cudaSuccess;
        if (dW) e = cudaMemset2DAsync(dW, lddw * type_bytes(dtype), 0, Cs * type_bytes(dtype), Ct, st);
        if (dbias && e == cudaSuccess) e = cudaMemsetAsync(dbias, 0, (size_t)Ct * 4, st);
        return cuda_status(e);
    }
    const BackwardPlan p = plan_backward(N, Cs, Ct, dtype);
    // dy itself where it is dz in a form that the products read
    const bool products = dx || dW;
    const bool dz = products && (act != QCNN_ACT_NONE || !bf16 || !tma_ok(dy, lddy, dtype));
    const bool x_copy = dW && (!bf16 || !tma_ok(x, ldx, dtype));
    const bool w_copy = dx && (bf16 ? !tma_ok(W, ldw, dtype) : p.wplanes);
    const BackwardSpace s = carve_backward(p, N, Cs, Ct, dtype, dz, x_copy, w_copy, workspace);
    qcnn_status rc = workspace_ok(workspace, workspace_bytes, s.bytes);
    if (rc != QCNN_OK) return rc;
    PdlScope pdl;
    const long long pz = pad8(Ct), pc = pad8(Cs);
    const int P = bf16 ? 1 : 3;
    GemmOperand z{dy, lddy, 0, 0}, xo{x, ldx, 0, 1}, wo{W, ldw, 0, 1};
    PlanesJob jobs[2];
    if (x_copy) {
        jobs[0] = planes_job(x, bf16, N, Cs, ldx, P, s.x);
        xo = GemmOperand{s.x, pc, N * pc, 1};
    }
    if (w_copy) {
        jobs[1] = planes_job(W, bf16, Ct, Cs, ldw, P, s.w);
        wo = GemmOperand{s.w, pc, Ct * pc, 1};
    }
    if (dz || dbias) {
        const int copies = jobs[0].blocks + jobs[1].blocks, tiles = cdiv(Ct, 128);
        const dim3 grid = copies ? dim3(tiles * p.slabs + copies) : dim3(tiles, p.slabs);
        float *const part = !dbias ? nullptr : p.slabs > 1 ? s.db : dbias;
        const int e = bf16 ? 2 : 4;
        const auto vec_ok = [&](const void *q, long long ld) {
            return reinterpret_cast<uintptr_t>(q) % (4 * e) == 0 && ld % 4 == 0;
        };
        const bool vec = vec_ok(dy, lddy) && (act == QCNN_ACT_NONE || vec_ok(pre, ldp));
        unsigned short *const out = static_cast<unsigned short *>(s.dz);
        const auto launch = [&](auto *type) {
            using T = std::remove_pointer_t<decltype(type)>;
            const auto k = copies ? (vec ? dz_kernel<T, true, true> : dz_kernel<T, false, true>)
                                  : (vec ? dz_kernel<T, true, false> : dz_kernel<T, false, false>);
            return launch_pdl(k, grid, dim3(256), 0, st, static_cast<const T *>(dy), lddy,
                              static_cast<const T *>(pre), ldp, N, Ct, act, out, P, pz, (long long)N * pz, part,
                              p.slab, p.slabs, jobs[0], jobs[1]);
        };
        rc = bf16 ? launch(static_cast<unsigned short *>(nullptr)) : launch(static_cast<float *>(nullptr));
        if (rc != QCNN_OK) return rc;
        if (dbias && p.slabs > 1 && (rc = launch_column_join(s.db, p.slabs, Ct, Ct, nullptr, dbias, st)) != QCNN_OK)
            return rc;
        if (dz) z = GemmOperand{s.dz, pz, (long long)N * pz, 0};
    } else if ((rc = launch_planes(jobs[0], jobs[1], bf16, st)) != QCNN_OK) {
        return rc;
    }
    GemmProblem g[2];
    const int type = bf16 ? GEMM_T_BF16 : GEMM_T_F32;
    GemmProblem &x_ = g[0], &w_ = g[1];
    x_.a = wo;
    x_.b = z;
    x_.m = Cs;
    x_.n = N;
    x_.k = Ct;
    x_.e.out = dx;
    x_.e.ldo = lddx;
    x_.e.out_type = type;
    w_.a = xo;
    w_.b = z;
    w_.b.mn = 1;
    w_.m = Cs;
    w_.n = Ct;
    w_.k = N;
    w_.e.out = dW;
    w_.e.ldo = lddw;
    w_.e.out_type = type;
    if (dx && dW) {  // one launch, the longer tiles first, where that fills the SMs better
        const bool x_first = Ct >= N;
        const GemmPlan &px = p.gx, &pw = p.gw;
        if (x_first ? gemm_together(px, Cs, N, Ct, pw, Cs, Ct, N) : gemm_together(pw, Cs, Ct, N, px, Cs, N, Ct)) {
            if (!x_first) std::swap(x_, w_);
            return launch_gemm(px, g, 2, st);
        }
    }
    if (dx && (rc = launch_gemm(p.gx, &x_, 1, st)) != QCNN_OK) return rc;
    if (dW && (rc = launch_gemm(p.gw, &w_, 1, st)) != QCNN_OK) return rc;
    return QCNN_OK;
}

}  // extern "C"
