// orthogonalize_small.cu -- Newton-Schulz steps of a small matrix in one launch.
//
// On the tensor cores a step is three dependent products of 3 us at least, whatever their
// size (first loads, a few MMAs, an epilogue, the next launch).  A matrix of few rows p (the
// smaller side) needs little arithmetic, and all of it can stay on the chip: one cluster of
// CTAs holds X, a slice of the q columns each, in shared memory in fp32, and A = X X^T and
// B = a I + b A + c A A (p x p) in every CTA.  A step is then
//   partial sums of A over the slice, 4 x 4 per thread; their sum over the cluster, a part per
//   CTA, handed to all (distributed shared memory, two barriers of the cluster);
//   B, by every CTA for itself;
//   X = B X of the slice, eight columns per warp at a time, in place;
// in fp32 multiply-adds.  It is taken where that is estimated to be sooner done than the
// products (ortho_small_plan): 18 x 36 in 26 us, 65 as products; 31 x 512 in fp32 37 and 73; 48
// x 1024 69 and 79; 62 x 326 the same.  Bound by the latency of a step's parts, 5 us.
#include "ortho_small.cuh"

#include <algorithm>

namespace qcnn {
namespace {

constexpr int kThreads = 512;
constexpr int kMaxP = 64;
constexpr size_t kSmemMax = 220 * 1024;

struct Args {
    const void *g;
    void *out;
    long long ldg, ldo;
    int m, n, p, q, p4, qs, steps, bf16;  // p4: p in multiples of 4; qs: columns per CTA
    float a, b, c, eps;
};

// X[j][i], i < p4 contiguous (zeros from p on): column j of the slice.
__device__ __forceinline__ float load_g(const Args &a, int i, int j) {
    const long long o = a.m <= a.n ? (long long)i * a.ldg + j : (long long)j * a.ldg + i;
    return a.bf16 ? bf16_to_float(static_cast<const unsigned short *>(a.g)[o]) : static_cast<const float *>(a.g)[o];
}
__device__ __forceinline__ void store_o(const Args &a, int i, int j, float v) {
    const long long o = a.m <= a.n ? (long long)i * a.ldo + j : (long long)j * a.ldo + i;
    if (a.bf16) static_cast<unsigned short *>(a.out)[o] = float_to_bf16(v);
    else static_cast<float *>(a.out)[o] = v;
}
__device__ __forceinline__ void fma4(float (&d)[4], float x, const float4 &y) {
    d[0] = fmaf(x, y.x, d[0]);
    d[1] = fmaf(x, y.y, d[1]);
    d[2] = fmaf(x, y.z, d[2]);
    d[3] = fmaf(x, y.w, d[3]);
}

__global__ void __launch_bounds__(kThreads, 1) ortho_small_kernel(const Args a) {
    namespace cg = cooperative_groups;
    extern __shared__ __align__(16) float smem_f[];
    __shared__ double2 norms[kThreads / 32 + 8];
    cg::cluster_group cluster = cg::this_cluster();
    cluster.barrier_arrive();  // (this CTA runs: its shared memory may be written to)
    grid_dep_sync();
    const int CL = (int)cluster.num_blocks(), rank = (int)cluster.block_rank();
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int p4 = a.p4, pp = p4 * p4;
    float *const X = smem_f, *const A = X + (size_t)a.qs * p4, *const B = A + pp, *const part = B + pp,
                *const sums = part + pp;  // sums: [16 per thread]
    const int j0 = rank * a.qs, cols = max(0, min(a.qs, a.q - j0));

    // G, and the sums of squares of its small and its large values (as norm_kernel's)
    double small = 0., large = 0.;
    const bool by_row = a.m <= a.n;  // (neighbours in memory: j, else i)
    for (int e = tid; e < cols * p4; e += kThreads) {
        const int j = by_row ? e % cols : e / p4, i = by_row ? e / cols : e - j * p4;
        const float v = i < a.p ? load_g(a, i, j0 + j) : 0.f;
        X[j * p4 + i] = v;
        const bool big = fabsf(v) > 281474976710656.f;
        const double w = big ? (double)v * 5.421010862427522e-20 : (double)v;
        if (big) large += w * w;
        else small += w * w;
    }
#pragma unroll
    for (int o = 16; o; o >>= 1) {
        small += __shfl_xor_sync(0xffffffffu, small, o);
        large += __shfl_xor_sync(0xffffffffu, large, o);
    }
    if (lane == 0) norms[warp] = make_double2(small, large);
    __syncthreads();
    cluster.barrier_wait();
    if (tid == 0) {
        double2 s = norms[0];
        for (int w = 1; w < kThreads / 32; ++w) {
            s.x += norms[w].x;
            s.y += norms[w].y;
        }
        for (int r = 0; r < CL; ++r) cluster.map_shared_rank(norms, r)[kThreads / 32 + rank] = s;
    }
    cluster.sync();
    small = large = 0.;
    for (int r = 0; r < CL; ++r) {
        small += norms[kThreads / 32 + r].x;
        large += norms[kThreads / 32 + r].y;
    }
    const double norm = sqrt(small + large * 340282366920938463463374607431768211456.0) + (double)a.eps;
    const double f = norm > 0. || norm != norm ? 1.0 / norm : 0.;
    const float f2 = f > 1e30 ? 1e30f : 1.f, f1 = (float)(f > 1e30 ? f / 1e30f : f);
    for (int e = tid; e < cols * p4; e += kThreads) X[e] = X[e] * f1 * f2;
    __syncthreads();

    const int t4 = p4 / 4, tiles = t4 * t4, groups = min(32, kThreads / tiles);  // (tiles <= 256)
    const int tile = tid % tiles, group = tid / tiles, ti = (tile / t4) * 4, tk = (tile % t4) * 4;
    for (int step = 0; step < a.steps; ++step) {
        // sums of this slice: a thread has 4 x 4 of A and every groups-th column
        if (group < groups) {
            float d[4][4] = {};
#pragma unroll 2
            for (int j = group; j < cols; j += groups) {
                const float4 x = *reinterpret_cast<const float4 *>(X + j * p4 + ti);
                const float4 y = *reinterpret_cast<const float4 *>(X + j * p4 + tk);
                fma4(d[0], x.x, y);
                fma4(d[1], x.y, y);
                fma4(d[2], x.z, y);
                fma4(d[3], x.w, y);
            }
#pragma unroll
            for (int r = 0; r < 4; ++r)
                *reinterpret_cast<float4 *>(sums + (size_t)group * pp + (ti + r) * p4 + tk) =
                    make_float4(d[r][0], d[r][1], d[r][2], d[r][3]);
        }
        __syncthreads();
        float *const to = CL > 1 ? part : A;
        for (int e = tid; e < pp; e += kThreads) {
            float v = 0.f;
#pragma unroll 8
            for (int g = 0; g < groups; ++g) v += sums[(size_t)g * pp + e];
            to[e] = v;
        }
        if (CL > 1) {
            cluster.sync();
            const int per = (pp + CL - 1) / CL, e1 = min(pp, (rank + 1) * per);
            for (int e = rank * per + tid; e < e1; e += kThreads) {
                float v = 0.f;
                for (int r = 0; r < CL; ++r) v += cluster.map_shared_rank(part, r)[e];
                for (int r = 0; r < CL; ++r) cluster.map_shared_rank(A, r)[e] = v;
            }
            cluster.sync();
        } else {
            __syncthreads();
        }
        // B (A is symmetric to the bit: both halves add the same products in the same order)
        for (int t = tid; t < tiles; t += kThreads) {
            const int bi = (t / t4) * 4, bk = (t % t4) * 4;
            float d[4][4] = {};
#pragma unroll 4
            for (int k = 0; k < p4; ++k) {
                const float4 x = *reinterpret_cast<const float4 *>(A + k * p4 + bi);
                const float4 y = *reinterpret_cast<const float4 *>(A + k * p4 + bk);
                fma4(d[0], x.x, y);
                fma4(d[1], x.y, y);
                fma4(d[2], x.z, y);
                fma4(d[3], x.w, y);
            }
#pragma unroll
            for (int r = 0; r < 4; ++r)
#pragma unroll
                for (int s = 0; s < 4; ++s) {
                    const int i = bi + r, k = bk + s;
                    B[i * p4 + k] = fmaf(a.c, d[r][s], a.b * A[i * p4 + k]) + (i == k ? a.a : 0.f);
                }
        }
        __syncthreads();
        // X = B X: a warp has 128 / t4 ... columns: a lane 4 rows x 4 columns
        const int lanes_i = min(32, t4), per_warp = 32 / lanes_i * 4;  // columns of a warp at a time
        const int li = lane % lanes_i, lj = lane / lanes_i;
        for (int jb = warp * per_warp; jb < cols; jb += kThreads / 32 * per_warp) {
            const int j = jb + lj * 4, i = li * 4;
            const bool in = lj < 32 / lanes_i && j < cols;
            float d[4][4] = {};  // [column][row]
            if (in) {
                const float *x = X + j * p4;
                // (columns past the last are read from the last)
                const int s1 = j + 1 < cols ? p4 : 0, s2 = j + 2 < cols ? 2 * p4 : 0, s3 = j + 3 < cols ? 3 * p4 : 0;
#pragma unroll 2
                for (int k = 0; k < p4; k += 4) {
                    const float4 x0 = *reinterpret_cast<const float4 *>(x + k);
                    const float4 x1 = *reinterpret_cast<const float4 *>(x + s1 + k);
                    const float4 x2 = *reinterpret_cast<const float4 *>(x + s2 + k);
                    const float4 x3 = *reinterpret_cast<const float4 *>(x + s3 + k);
                    const float4 b0 = *reinterpret_cast<const float4 *>(B + k * p4 + i);
                    const float4 b1 = *reinterpret_cast<const float4 *>(B + (k + 1) * p4 + i);
                    const float4 b2 = *reinterpret_cast<const float4 *>(B + (k + 2) * p4 + i);
                    const float4 b3 = *reinterpret_cast<const float4 *>(B + (k + 3) * p4 + i);
                    fma4(d[0], x0.x, b0), fma4(d[0], x0.y, b1), fma4(d[0], x0.z, b2), fma4(d[0], x0.w, b3);
                    fma4(d[1], x1.x, b0), fma4(d[1], x1.y, b1), fma4(d[1], x1.z, b2), fma4(d[1], x1.w, b3);
                    fma4(d[2], x2.x, b0), fma4(d[2], x2.y, b1), fma4(d[2], x2.z, b2), fma4(d[2], x2.w, b3);
                    fma4(d[3], x3.x, b0), fma4(d[3], x3.y, b1), fma4(d[3], x3.z, b2), fma4(d[3], x3.w, b3);
                }
            }
            __syncwarp();  // (the warp's columns have been read)
            if (in)
#pragma unroll
                for (int r = 0; r < 4; ++r)
                    if (j + r < cols)
                        *reinterpret_cast<float4 *>(X + (j + r) * p4 + i) =
                            make_float4(d[r][0], d[r][1], d[r][2], d[r][3]);
            __syncwarp();
        }
        __syncthreads();
    }
    for (int e = tid; e < cols * a.p; e += kThreads) {
        const int j = by_row ? e % cols : e / a.p, i = by_row ? e / cols : e - j * a.p;
        store_o(a, i, j0 + j, X[j * p4 + i]);
    }
    cluster.sync();  // (no CTA leaves while another may still write to it)
}

size_t smem_bytes(int p4, int qs) { return ((size_t)qs * p4 + 3 * (size_t)p4 * p4 + kThreads * 16) * sizeof(float); }

}  // namespace

OrthoSmall ortho_small_plan(int m, int n, int steps, double products) {
    OrthoSmall best;
    const int p = std::min(m, n), q = std::max(m, n), p4 = (p + 3) / 4 * 4;
    if (p > kMaxP) return best;
    for (int cl = 1; cl <= 8; cl *= 2) {
        const int qs = cdiv(cdiv(q, cl), 4) * 4;
        if (smem_bytes(p4, qs) > kSmemMax) continue;
        // Clocks: multiply-adds at 60 per clock and SM (of 128: the loads of 4 x 4 tiles), and
        // per step B and the barriers; X comes and goes once.
        const double step = 2.0 * p4 * p4 * qs / 60.0 + (double)p4 * p4 * p4 / 40.0 + (cl > 1 ? 6000.0 : 2500.0);
        const double score = 5000.0 + (double)qs * p4 / 40.0 + steps * step;
        if (score >= products || (best.cluster && score >= best.score)) continue;
        best.cluster = cl;
        best.qs = qs;
        best.score = score;
    }
    return best;
}

qcnn_status launch_ortho_small(const OrthoSmall &o, const void *G, long long ldg, int m, int n, int steps,
                               const float *k, float eps, void *out, long long ldo, int bf16, cudaStream_t st) {
    const int p = std::min(m, n), q = std::max(m, n), p4 = (p + 3) / 4 * 4;
    const Args a{G, out, ldg, ldo, m, n, p, q, p4, o.qs, steps, bf16, k[0], k[1], k[2], eps};
    qcnn_status rc = allow_smem(reinterpret_cast<const void *>(ortho_small_kernel));
    if (rc != QCNN_OK) return rc;
    return launch_k(ortho_small_kernel, dim3(o.cluster), dim3(kThreads), smem_bytes(p4, o.qs), st,
                    dim3(o.cluster, 1, 1), a);
}

}  // namespace qcnn
