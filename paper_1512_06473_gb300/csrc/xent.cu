// xent.cu -- qcnn_xent_forward and qcnn_xent_grad: softmax cross entropy over the classes of
// a linear layer, with its gradient.
//
//   l = x W^T + b;  lse_n = log sum_c exp l_nc;  loss_n = lse_n - l_n,t(n)
//   dl = g_n (exp(l - lse_n) - [c == t(n)]);  dx = dl W;  dW = dl^T x;  db = sum_n dl
//
// lse_n = top + log(sum) is rounded where it is an output alone: loss_n is (top - l_n,t) + log(sum) and
// exp(l - lse) is 2^((l - top) log2 e - log2(sum)).  (With lse in them, rows that the layer is sure of,
// whose logits are large and whose losses small, had losses off by 2^-24 of the logit.)
//
// Two ways, by the estimated time of each (plan_xent):
//   kept (the fp32 logits fit kPiece bytes): a product, a pass per row (lse, loss), and for the
//     gradient a pass over the logits (dl, db) and two products.  It has products whose terms
//     are shared among CTAs, and fp32 weights read without a pass over them.
//   not kept: one product over all classes leaves, per tile and row, the maximum and the sum
//     of exp; joined they are lse.  The gradient then goes in pieces of the classes: the
//     piece's logits again, whose epilogue turns them into dl (bf16, or planes), dx += dl
//     W_piece (summed in fp32), dW_piece = dl^T x.
// In us, kept and not: 128 x 4096 -> 1000 in fp32 19 and 60, with the gradient 51 and 136; 2048 x
// 1024 -> 8192 in bf16 46 and 32, 133 and 127; 2048 x 256 -> 8192 36 and 24, 93 and 81; 1024 x
// 1024 -> 16000 in fp32 164 and 165, 481 and 599 (the fourth product costs six there).
#include "train.cuh"

#include <algorithm>

namespace qcnn {
namespace {

constexpr size_t kPiece = 128u << 20;    // bytes of kept logits at most
constexpr size_t kPieceDl = 128u << 20;  // bytes of a piece of the gradient of others
// Shares of the terms of kept logits, joined by the pass over their rows (128 rows of 4096 ->
// 1000 in fp32: 9 us with 19, 24 us with clusters of eight CTAs, which fill fewer SMs).
constexpr int kGroups = 32;

__device__ __forceinline__ int class_of(const int64_t *targets, int n, int Ct) {
    const long long t = targets[n];
    QCNN_CHECK(t < Ct, QCNN_CHECK_CODE);
    return t >= 0 && t < Ct ? (int)t : -1;
}

// 1 / (rows with a class), by one CTA.
__device__ void count_rows(const int64_t *targets, int N, int Ct, float *inv) {
    __shared__ int part[32];
    int c = 0;
    for (int n = threadIdx.x; n < N; n += blockDim.x) c += (unsigned long long)targets[n] < (unsigned long long)Ct;
#pragma unroll
    for (int o = 16; o; o >>= 1) c += __shfl_xor_sync(0xffffffffu, c, o);
    if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = c;
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int i = 1; i < (int)blockDim.x / 32; ++i) c += part[i];
        *inv = c ? 1.f / (float)c : 0.f;
    }
}

// Maximum and sum of exp, of two parts (as in the products' epilogue).
__device__ __forceinline__ void join(float &top, float &sum, float t2, float s2) {
    const float t = fmaxf(top, t2);
    if (t == -INFINITY) {
        sum += s2;
        return;
    }
    sum = sum * expf(top - t) + s2 * expf(t2 - t);
    top = t;
}
struct RowOut {
    const int64_t *targets;
    const float *dloss;
    float *loss, *lse;
    float4 *rows;  // null: no gradient
    float *inv;
    int N, Ct;
};
__device__ __forceinline__ void finish_row(const RowOut &o, int n, float top, float sum, float target_logit) {
    const int t = class_of(o.targets, n, o.Ct);
    const float log_sum = logf(sum);
    o.lse[n] = top + log_sum;
    o.loss[n] = t >= 0 ? (top - target_logit) + log_sum : 0.f;
    if (o.rows) o.rows[n] = make_float4(top, o.dloss ? o.dloss[n] : 1.f, __int_as_float(t), log2f(sum));
}

// Kept: a CTA per row of logits; one more counts the rows.  GROUPS: the logits come as
// partial sums [group][N][Ct] without bias, are added up here and (where there is a gradient)
// left in `logits`.  U classes of a thread at a time, their loads in flight together; the
// maximum of all, then the sums.  (Maximum and sum joined pair by pair, and 1024 threads for
// any row, took 86 us for 2048 rows of 8192.)
template <bool GROUPS>
__global__ void __launch_bounds__(1024) rows_kernel(const float *part, int groups, const float *bias,
                                                    float *logits, RowOut o) {
    grid_dep_sync();
    if ((int)blockIdx.x == o.N) {
        count_rows(o.targets, o.N, o.Ct, o.inv);
        return;
    }
    constexpr int U = GROUPS ? 4 : 8;
    __shared__ float tops[32], sums[32], picked;
    const int t = class_of(o.targets, blockIdx.x, o.Ct), T = blockDim.x;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const size_t row = (size_t)blockIdx.x * o.Ct, stride = (size_t)o.N * o.Ct;
    if (threadIdx.x == 0) picked = 0.f;
    __syncthreads();
    float top = -INFINITY, sum = 0.f;
    for (int c0 = threadIdx.x; c0 < o.Ct; c0 += T * U) {
        float v[U], m = top;
#pragma unroll
        for (int i = 0; i < U; ++i) {
            const int c = c0 + i * T;
            v[i] = -INFINITY;
            if (c >= o.Ct) continue;
            if constexpr (GROUPS) {
                v[i] = add_groups<true>(part + row + c, groups, stride) + (bias ? bias[c] : 0.f);
                if (o.rows) logits[row + c] = v[i];
            } else {
                v[i] = logits[row + c];
            }
        }
#pragma unroll
        for (int i = 0; i < U; ++i) {
            if (c0 + i * T == t) picked = v[i];
            m = fmaxf(m, v[i]);
        }
        if (m == -INFINITY) {  // nothing to add (or NaN)
#pragma unroll
            for (int i = 0; i < U; ++i)
                if (v[i] != v[i]) sum = v[i];
            continue;
        }
        sum = top == -INFINITY ? sum : sum * ex2((top - m) * kLog2e);
#pragma unroll
        for (int i = 0; i < U; ++i) sum += ex2((v[i] - m) * kLog2e);
        top = m;
    }
    float all = top;
#pragma unroll
    for (int s = 16; s; s >>= 1) all = fmaxf(all, __shfl_xor_sync(0xffffffffu, all, s));
    if (lane == 0) tops[warp] = all;
    __syncthreads();
    all = lane * 32 < T ? tops[lane] : -INFINITY;
#pragma unroll
    for (int s = 16; s; s >>= 1) all = fmaxf(all, __shfl_xor_sync(0xffffffffu, all, s));
    // (-inf minus -inf is left out; a sum of NaN stays)
    if (top != all) sum *= ex2((top - all) * kLog2e);
#pragma unroll
    for (int s = 16; s; s >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, s);
    if (lane == 0) sums[warp] = sum;
    __syncthreads();
    if (warp == 0) {
        sum = lane * 32 < T ? sums[lane] : 0.f;
#pragma unroll
        for (int s = 16; s; s >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, s);
        if (lane == 0) finish_row(o, blockIdx.x, all, sum, picked);
    }
}

// Not kept: the tiles' maxima and sums of 32 rows per CTA; 32 warps take the tiles in turn.
__global__ void __launch_bounds__(1024) stats_join_kernel(const float2 *stats, int parts,
                                                         const float *target_logit, RowOut o) {
    grid_dep_sync();
    if ((int)blockIdx.x * 32 >= o.N) {
        count_rows(o.targets, o.N, o.Ct, o.inv);
        return;
    }
    __shared__ float2 red[32][32];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, n = blockIdx.x * 32 + lane;
    float top = -INFINITY, sum = 0.f;
    if (n < o.N)
        for (int p = warp; p < parts; p += 128) {
            float2 v[4];
#pragma unroll
            for (int i = 0; i < 4; ++i)
                v[i] = p + 32 * i < parts ? stats[(size_t)(p + 32 * i) * o.N + n] : make_float2(-INFINITY, 0.f);
#pragma unroll
            for (int i = 0; i < 4; ++i) join(top, sum, v[i].x, v[i].y);
        }
    red[warp][lane] = make_float2(top, sum);
    __syncthreads();
    if (warp == 0 && n < o.N) {
        for (int i = 1; i < 32; ++i) join(top, sum, red[i][lane].x, red[i][lane].y);
        finish_row(o, n, top, sum, target_logit[n]);
    }
}

// Kept: the gradient of the logits and its sums over a slab of rows.  A CTA takes 128
// classes x a slab: a warp a row, a lane four classes (VEC: Ct is a multiple of 4).
template <bool VEC>
__global__ void __launch_bounds__(256) dl_kernel(const float *logits, const float4 *rows, int N, int Ct,
                                                 unsigned short *out, int planes, long long ldo, long long plane,
                                                 float *part, const float *scale, int slab) {
    __shared__ float red[8][128];
    grid_dep_sync();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int c = blockIdx.x * 128 + lane * 4;
    const int r1 = min(N, ((int)blockIdx.y + 1) * slab);
    float sum[4] = {};
    if (c < Ct) {
#pragma unroll 4
        for (int r = (int)blockIdx.y * slab + warp; r < r1; r += 8) {
            const float4 row = rows[r];
            const int target = __float_as_int(row.z);
            const float *l = logits + (size_t)r * Ct + c;
            float v[4];
            if constexpr (VEC) {
                const float4 a = *reinterpret_cast<const float4 *>(l);
                v[0] = a.x, v[1] = a.y, v[2] = a.z, v[3] = a.w;
            } else {
#pragma unroll
                for (int j = 0; j < 4; ++j) v[j] = c + j < Ct ? l[j] : -INFINITY;
            }
            const float g = row.y;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const float p = row_share(v[j], row);
                // (a row without a class is zero, whatever its logits are)
                v[j] = target >= 0 && c + j < Ct ? g * (target == c + j ? p - 1.f : p) : 0.f;
                sum[j] += v[j];
            }
            const long long o = (long long)r * ldo + c;  // (rows of multiples of 8)
            unsigned w[3][2];
            unsigned short *d = out + o;
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                if (planes == 3) planes_of<true>(v[2 * j], v[2 * j + 1], w[0][j], w[1][j], w[2][j]);
                else planes_of<false>(v[2 * j], v[2 * j + 1], w[0][j], w[1][j], w[2][j]);
            }
            *reinterpret_cast<uint2 *>(d) = make_uint2(w[0][0], w[0][1]);
            if (planes == 3) {
                *reinterpret_cast<uint2 *>(d + plane) = make_uint2(w[1][0], w[1][1]);
                *reinterpret_cast<uint2 *>(d + 2 * plane) = make_uint2(w[2][0], w[2][1]);
            }
        }
    }
    if (!part) return;
#pragma unroll
    for (int j = 0; j < 4; ++j) red[warp][lane * 4 + j] = sum[j];
    __syncthreads();
    const int t = threadIdx.x, col = blockIdx.x * 128 + t;
    if (t < 128 && col < Ct) {
        float v = 0.f;
#pragma unroll
        for (int w = 0; w < 8; ++w) v += red[w][t];
        part[(long long)blockIdx.y * Ct + col] = scale ? *scale * v : v;
    }
}

// Threads of rows_kernel: one per class where there are few rows; where the rows fill the SMs
// eight CTAs of 256 at most each.
int rows_threads(int N, int Ct) {
    if (N <= 2 * num_sms()) return std::min(1024, std::max(128, cdiv(Ct, 128) * 128));
    return Ct <= 1024 ? 128 : 256;
}

// fp32: x and dl always as planes; wplanes: the weights too.  bf16: copies of what TMA
// cannot read.
struct XentPlan {
    bool keep = false, few = false, wplanes = false;
    GemmPlan logits, stats, dl, dx, dw;
    int piece = 0;  // classes of a piece
    int slab = 0, slabs = 1;
};
XentPlan plan_kept(int N, int Cs, int Ct, bool bf16, bool wa, bool grad, double *clocks) {
    XentPlan p;
    const int P = bf16 ? 1 : 3;
    const double logits = (double)N * Ct;
    p.keep = true;
    p.piece = Ct;
    p.wplanes = true;
    p.slab = std::max(32, cdiv(cdiv(N, std::max(1, 4 * num_sms() / cdiv(Ct, 128))), 8) * 8);
    p.slabs = cdiv(N, p.slab);
    p.logits = plan_gemm(P, GEMM_OUT, Ct, N, Cs, kGroups);
    p.dx = plan_gemm(P, GEMM_OUT, Cs, N, Ct);
    p.dw = plan_gemm(P, GEMM_OUT, Cs, Ct, N);
    const GemmPlan l = bf16 ? p.logits : plan_gemm(GEMM_F32, GEMM_OUT, Ct, N, Cs, kGroups);
    p.few = few_rows_sooner(N, Cs, Ct, bf16, wa, l);
    const double few = few_rows_clocks(N, Cs, Ct, bf16);
    *clocks = (p.few ? few : p.logits.score) + (grad ? p.dx.score : 0);
    if (!bf16) {
        const GemmPlan x = plan_gemm(GEMM_F32, GEMM_OUT, Cs, N, Ct);
        const double direct = (p.few ? few : l.score) + (grad ? x.score : 0);
        *clocks += p.few && !grad ? 0 : pass_clocks((double)Ct * Cs * 10.0);
        if (direct <= *clocks) {
            p.wplanes = false;
            p.logits = l;
            p.dx = x;
            *clocks = direct;
        }
    }
    // (rows_kernel; few rows leave SMs idle)
    const double sums = 4.0 * (p.few ? 1 : p.logits.groups);
    *clocks += std::max(pass_clocks(logits * sums), 4000.0 + Ct * sums / 20.0);
    if (grad) *clocks += pass_clocks(logits * (4.0 + 2.0 * P)) + p.dw.score;
    return p;
}
XentPlan plan_xent(int N, int Cs, int Ct, int dtype, bool wa, bool grad) {
    const bool bf16 = dtype == QCNN_BF16;
    const int P = bf16 ? 1 : 3;
    XentPlan p;
    p.wplanes = true;
    p.stats = plan_gemm(P, GEMM_STATS, N, Ct, Cs);
    const long long most = (long long)(kPieceDl / ((size_t)N * 2 * P)) / 256 * 256;
    p.piece = (int)std::min<long long>(Ct, std::max<long long>(256, most));
    // (pieces of equal size)
    p.piece = std::min(Ct, cdiv(cdiv(Ct, cdiv(Ct, p.piece)), 256) * 256);
    p.dl = plan_gemm(P, GEMM_DLOGITS, p.piece, N, Cs);
    p.dx = plan_gemm(P, GEMM_OUT, Cs, N, p.piece);
    p.dw = plan_gemm(P, GEMM_OUT, Cs, p.piece, N);
    if ((size_t)N * Ct * 4 > kPiece) return p;
    double kept = 0.0, again = p.stats.score + 5000.0;
    const XentPlan q = plan_kept(N, Cs, Ct, bf16, wa, grad, &kept);
    if (!bf16) again += pass_clocks((double)Ct * Cs * 10.0);
    // (of few rows the product reads weights at 4.2 TB/s, the stream of few rows at 6.3: 1 x 4096
    // -> 31273 in bf16 47 us kept, 67 not)
    if (q.few) again = std::max(again, (double)Ct * Cs * (bf16 ? 2.0 : 4.0) / 2200.0 + 5000.0);
    if (grad) again += cdiv(Ct, p.piece) * (p.dl.score + p.dx.score + p.dw.score);
    return kept <= again ? q : p;
}
// dx += dl W of a piece of cn classes.  (The last piece has fewer terms: shares of a whole one's
// would leave CTAs of a cluster without any.)
GemmPlan plan_dx(const XentPlan &p, int N, int Cs, int cn) {
    return cn == p.piece ? p.dx : plan_gemm(p.dx.planes, GEMM_OUT, Cs, N, cn);
}
struct XentSpace {
    float *inv = nullptr, *logits = nullptr, *part = nullptr, *target_logit = nullptr, *db = nullptr, *dx = nullptr;
    float4 *rows = nullptr;
    float2 *stats = nullptr;
    unsigned short *x = nullptr, *w = nullptr, *kept = nullptr, *dl = nullptr;
    size_t bytes = 0;
};
XentSpace carve_xent(const XentPlan &p, int N, int Cs, int Ct, int dtype, bool grad, bool xa, bool wa, void *ws) {
    Carver c{static_cast<uint8_t *>(ws)};
    XentSpace s;
    const bool bf16 = dtype == QCNN_BF16;
    const size_t P = bf16 ? 1 : 3;
    const long long pc = pad8(Cs);
    s.inv = c.array<float>(1);
    if (grad) s.rows = c.array<float4>(N);
    // (few rows read the operands as they are; their gradient does not)
    const bool x_copy = !p.few && (!bf16 || !xa);
    if (x_copy) s.x = c.array<unsigned short>(P * N * pc);
    if ((!p.few || grad) && (bf16 ? !wa : p.wplanes)) s.w = c.array<unsigned short>(P * Ct * pc);
    if (p.keep) {
        s.logits = c.array<float>((size_t)N * Ct);
        if (!p.few && p.logits.groups > 1) s.part = c.array<float>((size_t)p.logits.groups * N * Ct);
    } else {
        s.stats = c.array<float2>((size_t)p.stats.n_tiles * 2 * N);
        s.target_logit = c.array<float>(N);
    }
    if (grad) {
        // rows without a class must not reach dW, not even as 0 * NaN
        s.kept = c.array<unsigned short>(P * N * pc);
        s.dl = c.array<unsigned short>(P * N * pad8(p.piece));
        if (p.keep) {
            if (p.slabs > 1) s.db = c.array<float>((size_t)p.slabs * Ct);
        } else {
            s.db = c.array<float>((size_t)p.dl.n_tiles * 2 * p.piece);
            if (p.piece < Ct) s.dx = c.array<float>((size_t)N * Cs);
        }
    }
    s.bytes = c.used;
    return s;
}

struct XentCall {
    const void *x, *W;
    long long ldx, ldw;
    int N, Cs, Ct, dtype;
    const float *bias;
    const int64_t *targets;
    const float *dloss;
    float *loss, *lse;
    void *dx, *dW;
    long long lddx, lddw;
    float *dbias;
    bool grad;
};

qcnn_status run_xent(const XentCall &a, void *workspace, size_t workspace_bytes, cudaStream_t st) {
    const int N = a.N, Cs = a.Cs, Ct = a.Ct;
    const bool bf16 = a.dtype == QCNN_BF16;
    const bool xa = tma_ok(a.x, a.ldx, a.dtype), wa = weights_ok(a.W, a.ldw, a.dtype);
    const XentPlan p = plan_xent(N, Cs, Ct, a.dtype, wa, a.grad);
    const XentSpace s = carve_xent(p, N, Cs, Ct, a.dtype, a.grad, xa, wa, workspace);
    qcnn_status rc = workspace_ok(workspace, workspace_bytes, s.bytes);
    if (rc != QCNN_OK) return rc;
    PdlScope pdl;
    const int P = bf16 ? 1 : 3;
    const long long pc = pad8(Cs);
    GemmOperand xo{a.x, a.ldx, 0, 0}, wo{a.W, a.ldw, 0, 0};
    PlanesJob jobs[2];
    if (s.x || s.kept) {
        jobs[0] = planes_job(a.x, bf16, N, Cs, a.ldx, P, s.x, s.kept, reinterpret_cast<const long long *>(a.targets),
                             Ct);
        if (s.x) xo = GemmOperand{s.x, pc, N * pc, 0};
    }
    if (s.w) {
        jobs[1] = planes_job(a.W, bf16, Ct, Cs, a.ldw, P, s.w);
        wo = GemmOperand{s.w, pc, Ct * pc, 0};
    }
    if ((rc = launch_planes(jobs[0], jobs[1], bf16, st)) != QCNN_OK) return rc;
    const GemmOperand xk{s.kept, pc, N * pc, 1};
    RowOut ro{a.targets, a.dloss, a.loss, a.lse, s.rows, s.inv, N, Ct};
    const int type = bf16 ? GEMM_T_BF16 : GEMM_T_F32;
    GemmProblem g;
    if (p.keep) {
        g.e.bias = a.bias;
        g.e.out = s.logits;
        g.e.ldo = Ct;
        if (p.few) {
            rc = launch_few_rows(FewRows{a.x, a.W, a.ldx, a.ldw, N, Cs, Ct, bf16, g.e}, st);
        } else {
            g.a = wo;
            g.b = xo;
            g.m = Ct;
            g.n = N;
            g.k = Cs;
            if (p.logits.groups > 1) {
                g.e.bias = nullptr;
                g.e.out = s.part;
            }
            rc = launch_gemm(p.logits, &g, 1, st);
        }
        if (rc != QCNN_OK) return rc;
        const bool groups = !p.few && p.logits.groups > 1;
        rc = launch_pdl(groups ? rows_kernel<true> : rows_kernel<false>, dim3(N + (a.grad ? 1 : 0)),
                        dim3(rows_threads(N, Ct)), 0, st, static_cast<const float *>(s.part), p.logits.groups,
                        a.bias, s.logits, ro);
    } else {
        g.a = xo;
        g.b = wo;
        g.m = N;
        g.n = Ct;
        g.k = Cs;
        g.e.bias = a.bias;
        g.e.stats = s.stats;
        g.e.targets = reinterpret_cast<const long long *>(a.targets);
        g.e.target_logit = s.target_logit;
        if ((rc = launch_gemm(p.stats, &g, 1, st)) != QCNN_OK) return rc;
        rc = launch_pdl(stats_join_kernel, dim3(cdiv(N, 32) + (a.grad ? 1 : 0)), dim3(1024), 0, st, s.stats,
                        p.stats.n_tiles * 2, s.target_logit, ro);
    }
    if (rc != QCNN_OK || !a.grad) return rc;

    // The factor 1 / rows of a mean is left out of dl and joins the sums that it is in:
    // rounded to bf16 with dl it would put the same error into every gradient (0.2%).
    const float *inv = a.dloss ? nullptr : s.inv;
    for (int c0 = 0; c0 < Ct; c0 += p.piece) {
        const int cn = std::min(p.piece, Ct - c0);
        const long long pz = pad8(cn), zplane = (long long)N * pz;
        const GemmOperand wp{static_cast<const uint8_t *>(wo.p) + c0 * wo.ld * (bf16 || s.w ? 2 : 4), wo.ld,
                             wo.plane, 1};
        if (p.keep) {
            // (of one slab the sums are db: no launch to join them)
            float *const part = a.dbias && p.slabs > 1 ? s.db : a.dbias;
            rc = launch_pdl(Ct % 4 ? dl_kernel<false> : dl_kernel<true>, dim3(cdiv(Ct, 128), p.slabs), dim3(256), 0,
                            st, s.logits, s.rows, N, Ct, s.dl, P, pz, zplane, part,
                            p.slabs > 1 ? nullptr : inv, p.slab);
            if (rc == QCNN_OK && p.slabs > 1 && a.dbias)
                rc = launch_column_join(s.db, p.slabs, Ct, Ct, inv, a.dbias, st);
        } else {
            GemmProblem d;
            d.a = wp;
            d.a.mn = 0;
            d.b = xo;
            d.m = cn;
            d.n = N;
            d.k = Cs;
            d.e.bias = a.bias ? a.bias + c0 : nullptr;
            d.e.rows = s.rows;
            d.e.class0 = c0;
            d.e.out = s.dl;
            d.e.ldo = pz;
            d.e.out_plane = zplane;
            d.e.col_part = s.db;
            d.e.ld_col = p.piece;
            rc = launch_gemm(p.dl, &d, 1, st);
            if (rc == QCNN_OK && a.dbias)
                rc = launch_column_join(s.db, p.dl.n_tiles * 2, p.piece, cn, inv, a.dbias + c0, st);
        }
        if (rc != QCNN_OK) return rc;
        GemmProblem q;
        q.a = wp;
        q.b = GemmOperand{s.dl, pz, zplane, 0};
        q.m = Cs;
        q.n = N;
        q.k = cn;
        const bool first = c0 == 0, last = c0 + cn == Ct;
        if (!first) {
            q.e.add = s.dx;
            q.e.lda = Cs;
            q.e.beta = 1.f;
        }
        q.e.alpha_ptr = inv;
        q.e.out = last ? a.dx : s.dx;
        q.e.ldo = last ? a.lddx : Cs;
        q.e.out_type = last ? type : GEMM_T_F32;
        if ((rc = launch_gemm(plan_dx(p, N, Cs, cn), &q, 1, st)) != QCNN_OK) return rc;
        GemmProblem v;
        v.a = xk;
        v.b = GemmOperand{s.dl, pz, zplane, 1};
        v.m = Cs;
        v.n = cn;
        v.k = N;
        v.e.alpha_ptr = inv;
        v.e.out = static_cast<uint8_t *>(a.dW) + c0 * a.lddw * type_bytes(a.dtype);
        v.e.ldo = a.lddw;
        v.e.out_type = type;
        if ((rc = launch_gemm(p.dw, &v, 1, st)) != QCNN_OK) return rc;
    }
    return QCNN_OK;
}

bool xent_args_ok(const XentCall &a) {
    return a.N >= 0 && a.Cs > 0 && a.Ct > 0 && dtype_ok(a.dtype) && matrix_ok(a.x, a.ldx, a.N, a.Cs, a.dtype) &&
           matrix_ok(a.W, a.ldw, a.Ct, a.Cs, a.dtype) && reinterpret_cast<uintptr_t>(a.bias) % 4 == 0 &&
           (a.N == 0 || (a.targets && a.loss && a.lse)) && reinterpret_cast<uintptr_t>(a.targets) % 8 == 0 &&
           reinterpret_cast<uintptr_t>(a.loss) % 4 == 0 && reinterpret_cast<uintptr_t>(a.lse) % 4 == 0 &&
           reinterpret_cast<uintptr_t>(a.dloss) % 4 == 0 && reinterpret_cast<uintptr_t>(a.dbias) % 4 == 0;
}

}  // namespace
}  // namespace qcnn

using namespace qcnn;

extern "C" {

qcnn_status qcnn_xent_workspace_size(int N, int Cs, int Ct, int dtype, int aligned, int grad, size_t *bytes) {
    if (!bytes || N < 0 || Cs <= 0 || Ct <= 0 || !dtype_ok(dtype)) return QCNN_ERR_INVALID_ARG;
    *bytes = 0;
    if (N == 0) return QCNN_OK;
    for (int wa = 0; wa < 2; ++wa) {  // (of fp32 calls, `aligned` says nothing)
        if (!wa && aligned && dtype == QCNN_BF16) continue;
        const XentPlan p = plan_xent(N, Cs, Ct, dtype, wa, grad != 0);
        *bytes = std::max(*bytes, carve_xent(p, N, Cs, Ct, dtype, grad != 0, aligned, aligned, nullptr).bytes);
    }
    return QCNN_OK;
}

qcnn_status qcnn_xent_route_info(int N, int Cs, int Ct, int dtype, int grad, int info[6]) {
    if (!info || N <= 0 || Cs <= 0 || Ct <= 0 || !dtype_ok(dtype)) return QCNN_ERR_INVALID_ARG;
    const XentPlan p = plan_xent(N, Cs, Ct, dtype, true, grad != 0);
    info[0] = p.keep;
    info[1] = grad ? p.piece : Ct;
    info[2] = Ct - (cdiv(Ct, info[1]) - 1) * info[1];
    info[3] = grad ? cdiv(Ct, p.piece) : 1;
    info[4] = info[5] = 0;
    if (!grad) return QCNN_OK;
    const GemmPlan last = plan_dx(p, N, Cs, info[2]);
    info[4] = last.splits;
    info[5] = last.kb_per_split * gemm_block_k(last.planes);
    return QCNN_OK;
}

qcnn_status qcnn_xent_forward(const void *x, long long ldx, int N, int Cs, const void *W, long long ldw, int Ct,
                              const float *bias, const int64_t *targets, float *loss, float *lse, int dtype,
                              void *workspace, size_t workspace_bytes, void *stream) {
    const XentCall a{x, W, ldx, ldw, N, Cs, Ct, dtype, bias, targets, nullptr, loss, lse, nullptr, nullptr, 0, 0,
                     nullptr, false};
    if (!xent_args_ok(a)) return QCNN_ERR_INVALID_ARG;
    if (N == 0) return QCNN_OK;
    return run_xent(a, workspace, workspace_bytes, static_cast<cudaStream_t>(stream));
}

qcnn_status qcnn_xent_grad(const void *x, long long ldx, int N, int Cs, const void *W, long long ldw, int Ct,
                           const float *bias, const int64_t *targets, const float *dloss, float *loss,
                           float *lse, void *dx, long long lddx, void *dW, long long lddw, float *dbias,
                           int dtype, void *workspace, size_t workspace_bytes, void *stream) {
    const XentCall a{x, W, ldx, ldw, N, Cs, Ct, dtype, bias, targets, dloss, loss, lse, dx, dW, lddx, lddw,
                     dbias, true};
    if (!xent_args_ok(a) || !matrix_ok(dx, lddx, N, Cs, dtype) || !matrix_ok(dW, lddw, Ct, Cs, dtype))
        return QCNN_ERR_INVALID_ARG;
    const cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (N == 0) {
        cudaError_t e = cudaMemset2DAsync(dW, lddw * type_bytes(dtype), 0, Cs * type_bytes(dtype), Ct, st);
        if (dbias && e == cudaSuccess) e = cudaMemsetAsync(dbias, 0, (size_t)Ct * 4, st);
        return cuda_status(e);
    }
    return run_xent(a, workspace, workspace_bytes, st);
}

}  // extern "C"
