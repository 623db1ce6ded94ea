// dropout.cu -- qcnn_dropout_forward and qcnn_dropout_backward: dropout whose mask is computed where
// it is needed, never stored.
//
//   y = keep ? x / (1 - p) : 0 (+ r);   keep: word i mod 4 of Philox-4x32-10(counter (i / 4, offset),
//   key seed) >= p 2^32, for element i of the matrix
//
// One pass: x (and r) read once, y written once.  Ten rounds are 20 products of 32 x 32 -> 64 bits per
// four elements, and these go at 32 lanes per clock and SM (measured), nothing else of their warps'
// quarter of the SM being issued meanwhile: 32 slots of a lane per element, of which 132 us for the 151
// million elements of 16384 x 9216.  Four bytes an element (bf16 without a residual) are bound by that
// (3001 x 5003 17 us, of which its bytes take 9), six (with a residual) by both (906 MB in 139 us, 6.5
// TB/s), eight (fp32) by the bytes (604 MB in 91 us, 6.7 TB/s).
#include "train.cuh"

#include <cmath>
#include <type_traits>

namespace qcnn {
namespace {

constexpr int kDropoutThreads = 128;
// From here on four per thread.  us, one and four: fp32 2^19 vectors 5.2 and 5.4, 2^20 9.5 and 8.2, 2^21 18.6 and
// 13.9; bf16 2^19 6.2 and 6.6 (with a residual 6.5 and 8.0), 2^20 10.6 and 11.0 (10.9 and 12.1), 2^21 19.2 and
// 19.0 (20.0 and 20.7), 2^23 69 and 62 (70 and 66).
constexpr unsigned long long kManyVectors = 1u << 19;

struct DropoutArgs {
    const void *x, *r;
    void *y;
    long long ldx, ldr, ldy;
    unsigned long long n;  // elements
    unsigned long long offset;
    const long long *offset_add;
    int cols;
    unsigned k0, k1, threshold;
    float scale;
};

// The four words of a counter: Salmon, Moraes, Dror and Shaw, "Parallel random numbers: as easy as 1,
// 2, 3" (SC 2011), Philox-4x32 with ten rounds.
__device__ __forceinline__ void philox(unsigned long long block, unsigned long long offset, unsigned k0, unsigned k1,
                                       unsigned (&c)[4]) {
    c[0] = (unsigned)block, c[1] = (unsigned)(block >> 32);
    c[2] = (unsigned)offset, c[3] = (unsigned)(offset >> 32);
#pragma unroll
    for (int i = 0; i < 10; ++i) {
        const unsigned long long a = (unsigned long long)c[0] * 0xD2511F53u, b = (unsigned long long)c[2] * 0xCD9E8D57u;
        c[0] = (unsigned)(b >> 32) ^ c[1] ^ k0;
        c[1] = (unsigned)b;
        c[2] = (unsigned)(a >> 32) ^ c[3] ^ k1;
        c[3] = (unsigned)a;
        k0 += 0x9E3779B9u;
        k1 += 0xBB67AE85u;
    }
}

template <typename T>
__device__ __forceinline__ float to_float(T v) {
    if constexpr (sizeof(T) == 4) return v;
    else return bf16_to_float(v);
}
template <typename T>
__device__ __forceinline__ T from_float(float v) {
    if constexpr (sizeof(T) == 4) return v;
    else return float_to_bf16(v);
}

// 16 bytes of elements in registers; two bf16 in a word.
template <typename T>
__device__ __forceinline__ uint4 drop_vec(const uint4 &x, const uint4 &r, bool res, const DropoutArgs &d,
                                          unsigned long long block, unsigned long long offset) {
    const unsigned xs[4] = {x.x, x.y, x.z, x.w}, rs[4] = {r.x, r.y, r.z, r.w};
    unsigned w[4], out[4];
    philox(block, offset, d.k0, d.k1, w);
    if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            float v = w[j] >= d.threshold ? __uint_as_float(xs[j]) * d.scale : 0.f;
            if (res) v += __uint_as_float(rs[j]);
            out[j] = __float_as_uint(v);
        }
    } else {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            if (j == 2) philox(block + 1, offset, d.k0, d.k1, w);
            const int k = (j & 1) * 2;
            float v0 = w[k] >= d.threshold ? __uint_as_float(xs[j] << 16) * d.scale : 0.f;
            float v1 = w[k + 1] >= d.threshold ? __uint_as_float(xs[j] & 0xffff0000u) * d.scale : 0.f;
            if (res) v0 += __uint_as_float(rs[j] << 16), v1 += __uint_as_float(rs[j] & 0xffff0000u);
            out[j] = pack_bf16x2(v0, v1);
        }
    }
    return make_uint4(out[0], out[1], out[2], out[3]);
}

// U vectors of 16 bytes per thread, all loads first.  FLAT: no gaps between rows, so that the matrix is
// one row, whatever its width (its last elements, fewer than a vector, go one by one); else rows of
// whole vectors.  LOW: counters below 2^32, so that two of an element's products are the same for all.
// (16384 x 9216 of zeros with a residual in bf16: a grid that stays and loads its next vectors ahead 152
// to 163 us, this way 132; CTAs of 256 threads 137; one vector 146; counters of 64 bits 146.)
template <typename T, int U, bool FLAT, bool LOW>
__global__ void __launch_bounds__(kDropoutThreads) dropout_vec_kernel(DropoutArgs d) {
    constexpr int V = 16 / (int)sizeof(T), B = kDropoutThreads;
    using L = unsigned long long;
    const L vectors = d.n / V, first = (L)blockIdx.x * (B * U) + threadIdx.x;
    grid_dep_sync();
    const L offset = d.offset + (d.offset_add ? *d.offset_add : 0);
    const bool res = d.r != nullptr;
    const T *const x = static_cast<const T *>(d.x), *const r = static_cast<const T *>(d.r);
    T *const y = static_cast<T *>(d.y);
    // where a vector begins
    auto at = [&](L v, long long ld) -> long long {
        if constexpr (FLAT) {
            return (long long)(v * V);
        } else {
            const unsigned per = (unsigned)d.cols / V;
            const L row = vectors <= 0xffffffffull ? (unsigned)v / per : v / per;
            return (long long)row * ld + (long long)(v - row * per) * V;
        }
    };
    uint4 a[U], b[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const L v = first + u * B;
        if (v >= vectors) continue;
        a[u] = *reinterpret_cast<const uint4 *>(x + at(v, d.ldx));
        if (res) b[u] = *reinterpret_cast<const uint4 *>(r + at(v, d.ldr));
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const L v = first + u * B, block = v * (V / 4);
        if (v >= vectors) continue;
        *reinterpret_cast<uint4 *>(y + at(v, d.ldy)) =
            drop_vec<T>(a[u], b[u], res, d, LOW ? (L)(unsigned)block : block, offset);
    }
    if constexpr (FLAT) {
        const int rest = (int)(d.n - vectors * V);
        if (blockIdx.x == 0 && (int)threadIdx.x < rest) {
            const L i = vectors * V + threadIdx.x;
            unsigned w[4];
            philox(i / 4, offset, d.k0, d.k1, w);
            const unsigned word = i & 2 ? (i & 1 ? w[3] : w[2]) : (i & 1 ? w[1] : w[0]);
            float v = word >= d.threshold ? to_float(x[i]) * d.scale : 0.f;
            if (res) v += to_float(r[i]);
            y[i] = from_float<T>(v);
        }
    }
}

// Four elements of a counter per thread, wherever their rows begin.
template <typename T>
__global__ void __launch_bounds__(256) dropout_kernel(DropoutArgs d) {
    const unsigned long long block = (unsigned long long)blockIdx.x * 256 + threadIdx.x, i0 = block * 4;
    grid_dep_sync();
    if (i0 >= d.n) return;
    unsigned w[4];
    philox(block, d.offset + (d.offset_add ? *d.offset_add : 0), d.k0, d.k1, w);
    unsigned long long row = i0 / (unsigned)d.cols;
    int col = (int)(i0 - row * (unsigned)d.cols);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        if (i0 + j < d.n) {
            float v = w[j] >= d.threshold ? to_float(static_cast<const T *>(d.x)[row * d.ldx + col]) * d.scale : 0.f;
            if (d.r) v += to_float(static_cast<const T *>(d.r)[row * d.ldr + col]);
            static_cast<T *>(d.y)[row * d.ldy + col] = from_float<T>(v);
        }
        if (++col == d.cols) col = 0, ++row;
    }
}

qcnn_status dropout(const void *x, long long ldx, int N, int C, double p, uint64_t seed, uint64_t offset,
                    const int64_t *offset_add, const void *r, long long ldr, void *y, long long ldy, int dtype,
                    void *stream) {
    if (N < 0 || C <= 0 || !dtype_ok(dtype) || !(p >= 0.0 && p < 1.0)) return QCNN_ERR_INVALID_ARG;
    if (!matrix_ok(x, ldx, N, C, dtype) || !matrix_ok(y, ldy, N, C, dtype) || (r && !matrix_ok(r, ldr, N, C, dtype)) ||
        reinterpret_cast<uintptr_t>(offset_add) % 8)
        return QCNN_ERR_INVALID_ARG;
    if (N == 0) return QCNN_OK;
    DropoutArgs d;
    d.x = x, d.r = r, d.y = y;
    d.ldx = ldx, d.ldr = ldr, d.ldy = ldy;
    d.n = (unsigned long long)N * C;
    d.offset = offset;
    d.offset_add = reinterpret_cast<const long long *>(offset_add);
    d.cols = C;
    d.k0 = (unsigned)seed, d.k1 = (unsigned)(seed >> 32);
    d.threshold = (unsigned)std::min(std::nearbyint(p * 4294967296.0), 4294967295.0);
    d.scale = (float)(1.0 / (1.0 - p));
    const cudaStream_t st = static_cast<cudaStream_t>(stream);
    const int V = dtype == QCNN_BF16 ? 8 : 4;
    const auto vec = [&](const void *q, long long ld, bool flat) {
        return reinterpret_cast<uintptr_t>(q) % 16 == 0 && (flat || ld % V == 0);
    };
    const bool flat = N == 1 || (ldx == C && ldy == C && (!r || ldr == C));
    if ((flat || C % V == 0) && vec(x, ldx, flat) && vec(y, ldy, flat) && (!r || vec(r, ldr, flat))) {
        const unsigned long long vectors = d.n / V;
        const int per = (vectors >= kManyVectors ? 4 : 1) * kDropoutThreads;
        const unsigned long long ctas = std::max(1ull, (vectors + per - 1) / per);
        if (ctas > INT_MAX) return QCNN_ERR_UNSUPPORTED;
        const bool low = vectors * (V / 4) < 1ull << 32, many = vectors >= kManyVectors;
        const auto launch = [&](auto *type) {
            using T = std::remove_pointer_t<decltype(type)>;
            auto k = many ? dropout_vec_kernel<T, 4, true, true> : dropout_vec_kernel<T, 1, true, true>;
            if (!flat) k = many ? dropout_vec_kernel<T, 4, false, true> : dropout_vec_kernel<T, 1, false, true>;
            if (!low) k = flat ? dropout_vec_kernel<T, 4, true, false> : dropout_vec_kernel<T, 4, false, false>;
            return launch_pdl(k, dim3((unsigned)ctas), dim3(kDropoutThreads), 0, st, d);
        };
        return V == 8 ? launch(static_cast<unsigned short *>(nullptr)) : launch(static_cast<float *>(nullptr));
    }
    const unsigned long long ctas = ((d.n + 3) / 4 + 255) / 256;
    if (ctas > INT_MAX) return QCNN_ERR_UNSUPPORTED;
    return launch_pdl(dtype == QCNN_BF16 ? dropout_kernel<unsigned short> : dropout_kernel<float>, dim3((unsigned)ctas),
                      dim3(256), 0, st, d);
}

}  // namespace
}  // namespace qcnn

using namespace qcnn;

extern "C" {

qcnn_status qcnn_dropout_forward(const void *x, long long ldx, int N, int C, double p, uint64_t seed,
                                 uint64_t offset, const int64_t *offset_add, const void *residual, long long ldr,
                                 void *y, long long ldy, int dtype, void *stream) {
    return dropout(x, ldx, N, C, p, seed, offset, offset_add, residual, ldr, y, ldy, dtype, stream);
}

qcnn_status qcnn_dropout_backward(const void *dy, long long lddy, int N, int C, double p, uint64_t seed,
                                  uint64_t offset, const int64_t *offset_add, void *dx, long long lddx, int dtype,
                                  void *stream) {
    return dropout(dy, lddy, N, C, p, seed, offset, offset_add, nullptr, 0, dx, lddx, dtype, stream);
}

}  // extern "C"
