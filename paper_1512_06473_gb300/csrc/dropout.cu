// dropout.cu -- qcnn_dropout_forward and qcnn_dropout_backward: dropout whose mask is computed where
// it is needed, never stored.
//
//   y = keep ? x / (1 - p) : 0 (+ r);   keep: word i mod 4 of Philox-4x32-10(counter (i / 4, offset),
//   key seed) >= p 2^32, for element i of the matrix
//
// One pass: x (and r) read once, y written once; 905 MB of 16384 x 9216 bf16 with a residual at least
// 134 us at the 6.78 TB/s of a copy.  Ten rounds are 20 multiplications of 32 x 32 -> 64 bits and as
// many three-way xors per four elements, which run while the loads are on their way.
#include "train.cuh"

#include <cmath>

namespace qcnn {
namespace {

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

// Four elements of a counter per thread, wherever their rows begin.
template <typename T>
__global__ void __launch_bounds__(256) dropout_kernel(DropoutArgs d) {
    const unsigned long long block = (unsigned long long)blockIdx.x * 256 + threadIdx.x, i0 = block * 4;
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
    const unsigned long long ctas = ((d.n + 3) / 4 + 255) / 256;
    if (ctas > INT_MAX) return QCNN_ERR_UNSUPPORTED;
    const cudaStream_t st = static_cast<cudaStream_t>(stream);
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
