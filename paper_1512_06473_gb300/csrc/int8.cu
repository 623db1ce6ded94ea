// int8.cu -- qcnn_int8_quantize and qcnn_int8_dense_forward: rows in 8-bit integers with a scale each,
// and a dense layer of such weights.
//
//   scale = max(max |x| (1 / 127), 2^-126), q = rint(x (1 / scale)), each step rounded to fp32;
//   y = act(xscale[n] wscale[m] sum_k q[n][k] W[m][k] + bias[m]) + r
#include "int8_gemm.cuh"
#include "train.cuh"

namespace qcnn {
namespace {

constexpr float kInv127 = 1.f / 127.f;

// --------------------------------------------------------------- quantizer
// A row's largest magnitude, NaN if it holds one (max.NaN).  |x| / scale <= 127 (1 + 2^-21), so no code
// is clamped.
__device__ __forceinline__ float max_nan(float a, float b) {
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
    return r;
}
struct RowScale {
    float scale, inverse;  // (inverse 0 where the scale is not finite)
};
__device__ __forceinline__ RowScale row_scale(float top) {
    const float t = __fmul_rn(top, kInv127), s = t < 1.17549435e-38f ? 1.17549435e-38f : t;
    return {s, s <= 3.402823466e38f ? __frcp_rn(s) : 0.f};
}
// x (1 / scale) to the nearest integers, ties to even: in the low bits of floats around 1.5 2^23.
// (Products one by one: a packed product and a packed sum, in intrinsics or with .rn in PTX, became one
// operation that rounds once, and ties of bf16 rows went the other way.)
constexpr float kRound = 12582912.f;
__device__ __forceinline__ float2 rounded(float x, float y, float inverse) {
    return __fadd2_rn(make_float2(__fmul_rn(x, inverse), __fmul_rn(y, inverse)), make_float2(kRound, kRound));
}
__device__ __forceinline__ unsigned pack_codes(float2 a, float2 b) {
    return __byte_perm(__byte_perm(__float_as_uint(a.x), __float_as_uint(a.y), 0x0040),
                       __byte_perm(__float_as_uint(b.x), __float_as_uint(b.y), 0x0040), 0x5410);
}
__device__ __forceinline__ unsigned pack_half(float2 a) {  // (exact)
    const float2 v = __fadd2_rn(a, make_float2(-kRound, -kRound));
    unsigned r;
    asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(v.y), "f"(v.x));
    return r;
}

struct QuantizeArgs {
    const void *x;
    long long ldx;
    int rows, cols;
    void *codes;    // int8, or (HALF) fp16 with zeros up to the next multiple of 8
    long long ldc;  // elements
    float *scale;
    int wide;   // codes go several at a time
    int *sums;  // HALF: null, or of the codes' magnitudes, [rows][segs]
    int segs;
};

// G threads a row (a warp, several or the CTA), which keep up to H vectors of 16 bytes each between
// the two steps; what a row has beyond that is read again.  Bound by the bytes (4096 x 9216 in fp32 28.8
// us, 6.6 TB/s).  SHIFT: rows begin off the 16 bytes, and a
// vector is taken out of the two aligned ones that it lies in (1000 x 4097 in bf16 8.6 us element by
// element).
template <typename T, int G, int H, bool SHIFT, bool HALF>
__global__ void __launch_bounds__(G > 256 ? G : 256) quantize_kernel(QuantizeArgs a) {
    constexpr int E = (int)sizeof(T), V = 16 / E, BLOCK = G > 256 ? G : 256, ROWS = BLOCK / G;
    // segments of 1024 codes of a row
    constexpr int SEGS = !HALF ? 1 : G == 512 ? (kInt8MaxTerms + 1) / kInt8Segment : G * H * V / kInt8Segment + 1;
    __shared__ float red[BLOCK / 32];
    [[maybe_unused]] __shared__ int seg[ROWS][SEGS];
    if constexpr (HALF) {
        for (int i = threadIdx.x; i < ROWS * SEGS; i += BLOCK) seg[i / SEGS][i % SEGS] = 0;
        if (G == 32) __syncthreads();  // (else a barrier follows)
    }
    grid_dep_sync();
    const int t = threadIdx.x % G, group = threadIdx.x / G;
    const long long row = (long long)blockIdx.x * ROWS + group;
    const bool is = row < a.rows;
    const T *const x = static_cast<const T *>(a.x) + (is ? row : 0) * a.ldx;
    const unsigned vectors = is ? a.cols / V : 0, rest = is ? a.cols % V : 0;
    struct Vec {
        unsigned w[4];
    };
    [[maybe_unused]] const uintptr_t base = reinterpret_cast<uintptr_t>(a.x),
                                     end = base + ((a.rows - 1) * a.ldx + a.cols) * E;
    auto element = [&](unsigned c) {
        if constexpr (E == 4) return __float_as_uint(x[c]);
        else return (unsigned)x[c];
    };
    auto load = [&](unsigned v) {
        Vec r;
        if constexpr (!SHIFT) {
            const uint4 q = reinterpret_cast<const uint4 *>(x)[v];
            r.w[0] = q.x, r.w[1] = q.y, r.w[2] = q.z, r.w[3] = q.w;
        } else {
            const uintptr_t at = reinterpret_cast<uintptr_t>(x) + (uintptr_t)v * 16, low = at & ~(uintptr_t)15;
            const unsigned off = (unsigned)(at - low);
            if (low >= base && low + 32 <= end) {
                const uint4 p = *reinterpret_cast<const uint4 *>(low), q = *reinterpret_cast<const uint4 *>(low + 16);
                unsigned w[8] = {p.x, p.y, p.z, p.w, q.x, q.y, q.z, q.w};
                if (off & 8) {
#pragma unroll
                    for (int i = 0; i < 6; ++i) w[i] = w[i + 2];
                }
                if (off & 4) {
#pragma unroll
                    for (int i = 0; i < 5; ++i) w[i] = w[i + 1];
                }
#pragma unroll
                for (int i = 0; i < 4; ++i) r.w[i] = E == 4 ? w[i] : __funnelshift_r(w[i], w[i + 1], off * 8 & 16);
            } else {  // (at the matrix's ends: nothing outside it is read)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    if constexpr (E == 4) r.w[i] = element(v * V + i);
                    else r.w[i] = element(v * V + 2 * i) | element(v * V + 2 * i + 1) << 16;
                }
            }
        }
        return r;
    };
    auto value = [](const Vec &r, int i) {  // element i
        if constexpr (E == 4) return __uint_as_float(r.w[i]);
        else return __uint_as_float(i & 1 ? r.w[i / 2] & 0xffff0000u : r.w[i / 2] << 16);
    };
    float top = 0.f;
    auto look = [&](const Vec &r) {
#pragma unroll
        for (int i = 0; i < V; ++i) top = max_nan(top, fabsf(value(r, i)));
    };
    Vec kept[H];
#pragma unroll
    for (int h = 0; h < H; ++h)
        if (t + h * G < vectors) kept[h] = load(t + h * G);
    Vec last = {};  // (an element of the rest, its first)
    if (t < rest) last.w[0] = element(vectors * V + t);
#pragma unroll
    for (int h = 0; h < H; ++h)
        if (t + h * G < vectors) look(kept[h]);
    if constexpr (H >= 5)
#pragma unroll 2
        for (unsigned v = t + H * G; v < vectors; v += G) look(load(v));
    top = max_nan(top, fabsf(value(last, 0)));
    // (as bits: their order is that of the values, NaN above all)
    top = __uint_as_float(__reduce_max_sync(0xffffffffu, __float_as_uint(top) & 0x7fffffffu));
    if constexpr (G > 32) {
        if (threadIdx.x % 32 == 0) red[threadIdx.x / 32] = top;
        __syncthreads();
#pragma unroll
        for (int i = 0; i < G / 32; ++i) top = max_nan(top, red[group * (G / 32) + i]);
    }
    if constexpr (!HALF)
        if (!is) return;
    const RowScale s = row_scale(top);
    if (is && t == 0) a.scale[row] = s.scale;
    const bool none = s.inverse == 0.f;
    [[maybe_unused]] int8_t *const bytes = static_cast<int8_t *>(a.codes) + row * a.ldc;
    [[maybe_unused]] unsigned short *const halves = static_cast<unsigned short *>(a.codes) + row * a.ldc;
    // the sum of the codes' magnitudes (HALF)
    auto put = [&](unsigned v, const Vec &from) {
        float magnitude = 0.f;
        Vec r = from;
        if (none) r = Vec{};
        float2 c[V / 2];
#pragma unroll
        for (int i = 0; i < V / 2; ++i) c[i] = rounded(value(r, 2 * i), value(r, 2 * i + 1), s.inverse);
        if constexpr (HALF) {
            unsigned short *const o = halves + (size_t)v * V;
#pragma unroll
            for (int i = 0; i < V / 2; ++i) magnitude += fabsf(c[i].x - kRound) + fabsf(c[i].y - kRound);
            if constexpr (V == 4) *reinterpret_cast<uint2 *>(o) = make_uint2(pack_half(c[0]), pack_half(c[1]));
            else *reinterpret_cast<uint4 *>(o) = make_uint4(pack_half(c[0]), pack_half(c[1]), pack_half(c[2]), pack_half(c[3]));
        } else {
            int8_t *const o = bytes + (size_t)v * V;
            unsigned w[V / 4];
#pragma unroll
            for (int i = 0; i < V / 4; ++i) w[i] = pack_codes(c[2 * i], c[2 * i + 1]);
            if (a.wide) {
                if constexpr (V == 4) *reinterpret_cast<unsigned *>(o) = w[0];
                else *reinterpret_cast<uint2 *>(o) = make_uint2(w[0], w[1]);
            } else {
#pragma unroll
                for (int i = 0; i < V; ++i) o[i] = (int8_t)(w[i / 4] >> i % 4 * 8);
            }
        }
        return magnitude;
    };
    // (a warp's vectors, 128 or 256 codes, lie in one segment; v0: the first of them)
    [[maybe_unused]] auto count = [&](unsigned v0, float magnitude) {
        const int sum = __reduce_add_sync(0xffffffffu, (int)magnitude);
        if (threadIdx.x % 32 == 0 && sum) atomicAdd(&seg[group][v0 * V / kInt8Segment], sum);
    };
    const unsigned t0 = t & ~31;
#pragma unroll
    for (int h = 0; h < H; ++h) {
        float magnitude = 0.f;
        if (t + h * G < vectors) magnitude = put(t + h * G, kept[h]);
        if (HALF && a.sums && t0 + h * G < vectors) count(t0 + h * G, magnitude);
    }
    if constexpr (H >= 5)
#pragma unroll 2
        for (unsigned v0 = t0 + H * G; v0 < vectors; v0 += G) {
            const unsigned v = v0 + threadIdx.x % 32;
            float magnitude = 0.f;
            if (v < vectors) magnitude = put(v, load(v));
            if (HALF && a.sums) count(v0, magnitude);
        }
    const float2 c = rounded(none ? 0.f : value(last, 0), 0.f, s.inverse);
    if constexpr (HALF) {
        const unsigned pad = (8 - a.cols % 8) % 8;
        if (t < rest) halves[(size_t)vectors * V + t] = (unsigned short)pack_half(c);
        if (is && t < pad) halves[a.cols + t] = 0;
        if (a.sums) {
            if (t < rest) atomicAdd(&seg[group][(vectors * V + t) / kInt8Segment], (int)fabsf(c.x - kRound));
            __syncthreads();
            if (is)
                for (int i = t; i < a.segs; i += G) a.sums[row * a.segs + i] = seg[group][i];
        }
    } else {
        if (t < rest) bytes[(size_t)vectors * V + t] = (int8_t)__float_as_uint(c.x);
    }
}

template <typename T, bool HALF>
qcnn_status launch_quantize_of(const QuantizeArgs &a, cudaStream_t st) {
    constexpr int V = 16 / (int)sizeof(T);
    const bool shift = reinterpret_cast<uintptr_t>(a.x) % 16 || (a.ldx % V && a.rows > 1);
    const auto launch = [&](auto k, auto ks, int G) {
        const int rows = G > 256 ? 1 : 256 / G;
        return launch_pdl(shift ? ks : k, dim3((unsigned)((a.rows + (long long)rows - 1) / rows)),
                          dim3(G > 256 ? G : 256), 0, st, a);
    };
    // (as few threads as hold the row in registers: several rows of a CTA wait for each other less)
    const int vectors = a.cols / V;
    if (vectors <= 128) return launch(quantize_kernel<T, 32, 4, false, HALF>, quantize_kernel<T, 32, 4, true, HALF>, 32);
    if (vectors <= 512) return launch(quantize_kernel<T, 128, 4, false, HALF>, quantize_kernel<T, 128, 4, true, HALF>, 128);
    if (vectors <= 1024) return launch(quantize_kernel<T, 256, 4, false, HALF>, quantize_kernel<T, 256, 4, true, HALF>, 256);
    return launch(quantize_kernel<T, 512, 5, false, HALF>, quantize_kernel<T, 512, 5, true, HALF>, 512);
}
// codes: int8, rows ldc apart; half: fp16, rows of 16-byte multiples
qcnn_status launch_quantize(const void *x, long long ldx, int rows, int cols, void *codes, long long ldc, bool half,
                            float *scale, int *sums, int dtype, cudaStream_t st) {
    const int V = dtype == QCNN_BF16 ? 8 : 4;
    const int wide = reinterpret_cast<uintptr_t>(codes) % V == 0 && (ldc % V == 0 || rows == 1);
    const QuantizeArgs a{x, ldx, rows, cols, codes, ldc, scale, wide, sums, cdiv(cols, kInt8Segment)};
    if (dtype == QCNN_BF16)
        return half ? launch_quantize_of<unsigned short, true>(a, st) : launch_quantize_of<unsigned short, false>(a, st);
    return half ? launch_quantize_of<float, true>(a, st) : launch_quantize_of<float, false>(a, st);
}

// ------------------------------------------------------------------ few rows
// No tensor cores: W is streamed once through sums of four products (dp4a, exact).
struct Int8Product {
    const void *x;        // codes, or (fused kernel) fp32 or bf16
    const int8_t *W;
    long long ldx, ldw;
    const float *xscale, *wscale;  // (xscale: of codes)
    int N, Cs, Ct;
    GemmEpi e;  // bias, act, add (beta 1), out; n = row, m = output
    int kw;     // warps that share an output's terms
};

constexpr int kOut = 4;  // outputs of a warp
__device__ __forceinline__ void finish_one(const GemmEpi &e, int r, int m, float v) {
    if (e.bias) v += e.bias[m];
    v = act_apply(v, e.act);
    if (e.add) v += load_as(e.add, e.add_type, (long long)r * e.lda + m);
    if (e.out_type == GEMM_T_F32) static_cast<float *>(e.out)[(long long)r * e.ldo + m] = v;
    else static_cast<unsigned short *>(e.out)[(long long)r * e.ldo + m] = float_to_bf16(v);
}
__device__ __forceinline__ int dot16(const uint4 &a, const uint4 &b, int c) {
    c = __dp4a((int)a.x, (int)b.x, c);
    c = __dp4a((int)a.y, (int)b.y, c);
    c = __dp4a((int)a.z, (int)b.z, c);
    return __dp4a((int)a.w, (int)b.w, c);
}

// One launch, no workspace: each CTA makes the codes of x for itself, in shared memory, while its first
// weights are on their way.  A warp sums kOut outputs x NB rows, or kw warps do, each a part of the terms.
// VEC: W's rows on 16 bytes.  T: float, bf16, or int8_t (codes).
// CTAs per SM and their threads: with more rows one, whose threads share the work on x.  (8 x 9216 -> 4096 in
// fp32 18.4 us, 22.9 with two of 256 threads; one row of 4096 -> 1000 4.0, 4.6 with one of 512.)
constexpr int few_ctas(int NB) { return NB <= 2 ? 2 : 1; }
constexpr int few_threads(int NB) { return 512 / few_ctas(NB); }
template <typename T, int NB, bool VEC>
__global__ void __launch_bounds__(few_threads(NB), few_ctas(NB)) few_rows_kernel(Int8Product f) {
    constexpr int kWarps = few_threads(NB) / 32;
    extern __shared__ __align__(16) int8_t codes[];  // [NB][pitch]
    __shared__ unsigned top[NB];
    __shared__ float scale[NB];
    __shared__ int red[kWarps][kOut * NB];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    if (blockIdx.y) {  // (more than eight rows: eight per CTA)
        const long long n = (long long)blockIdx.y * NB;
        f.x = static_cast<const T *>(f.x) + n * f.ldx;
        if (f.xscale) f.xscale += n;
        f.N -= (int)n;
        const int size = f.e.out_type == GEMM_T_F32 ? 4 : 2;
        f.e.out = static_cast<char *>(f.e.out) + n * f.e.ldo * size;
        if (f.e.add) f.e.add = static_cast<const char *>(f.e.add) + n * f.e.lda * size;
    }
    const int pitch = (f.Cs + 15) / 16 * 16, kw = f.kw;
    const int part = warp & (kw - 1), per = kWarps / kw, groups = (f.Ct + kOut - 1) / kOut;
    const int whole = VEC ? f.Cs / 16 : 0;  // vectors of 16 codes
    int group = blockIdx.x * per + warp / kw;
    grid_dep_sync();
    const int8_t *w[kOut];
    auto rows_of = [&] {
#pragma unroll
        for (int i = 0; i < kOut; ++i) w[i] = f.W + (long long)min(group * kOut + i, f.Ct - 1) * f.ldw;
    };
    constexpr int D = NB == 1 ? 4 : 1;  // steps of W that are loaded before x's codes are made
    uint4 first[D][kOut];
    const int v0 = part * 32 + lane;
    auto load_first = [&] {
        rows_of();
#pragma unroll
        for (int d = 0; d < D; ++d)
            if (VEC && v0 + d * kw * 32 < whole)
#pragma unroll
                for (int i = 0; i < kOut; ++i) first[d][i] = reinterpret_cast<const uint4 *>(w[i])[v0 + d * kw * 32];
    };
    load_first();

    // ---- the codes of x: 16 / NB warps a row
    {
        constexpr int WR = kWarps / NB;
        const int n = warp / WR, at = (warp % WR) * 32 + lane;
        int8_t *const out = codes + n * pitch;
        if (n < f.N) {
            const T *const x = static_cast<const T *>(f.x) + (long long)n * f.ldx;
            if constexpr (sizeof(T) == 1) {
                if (at == 0) scale[n] = f.xscale[n];
                if (reinterpret_cast<uintptr_t>(x) % 16 == 0) {
                    for (int v = at; v < f.Cs / 16; v += WR * 32)
                        reinterpret_cast<uint4 *>(out)[v] = reinterpret_cast<const uint4 *>(x)[v];
                    for (int c = f.Cs / 16 * 16 + at; c < f.Cs; c += WR * 32) out[c] = x[c];
                } else {
                    for (int c = at; c < f.Cs; c += WR * 32) out[c] = x[c];
                }
            }
        }
        if constexpr (sizeof(T) > 1) {
            if (threadIdx.x < NB) top[threadIdx.x] = 0;
            __syncthreads();
            constexpr int V = 16 / (int)sizeof(T), H = 4;  // vectors of x kept by a lane
            const T *const x = static_cast<const T *>(f.x) + (long long)(n < f.N ? n : 0) * f.ldx;
            const int cols = n < f.N ? f.Cs : 0;
            const bool wide = reinterpret_cast<uintptr_t>(x) % 16 == 0;
            const int vectors = wide ? cols / V : 0;
            auto value = [](const uint4 &q, int i) {
                const unsigned u[4] = {q.x, q.y, q.z, q.w};
                if constexpr (V == 4) return __uint_as_float(u[i]);
                else return __uint_as_float(i & 1 ? u[i / 2] & 0xffff0000u : u[i / 2] << 16);
            };
            auto single = [&](int c) {
                if constexpr (V == 4) return x[c];
                else return bf16_to_float(x[c]);
            };
            uint4 kept[H];
            float most = 0.f;
#pragma unroll
            for (int h = 0; h < H; ++h)
                if (at + h * WR * 32 < vectors) kept[h] = reinterpret_cast<const uint4 *>(x)[at + h * WR * 32];
#pragma unroll
            for (int h = 0; h < H; ++h)
                if (at + h * WR * 32 < vectors)
#pragma unroll
                    for (int i = 0; i < V; ++i) most = max_nan(most, fabsf(value(kept[h], i)));
            for (int v = at + H * WR * 32; v < vectors; v += WR * 32) {
                const uint4 q = reinterpret_cast<const uint4 *>(x)[v];
#pragma unroll
                for (int i = 0; i < V; ++i) most = max_nan(most, fabsf(value(q, i)));
            }
            for (int c = vectors * V + at; c < cols; c += WR * 32) most = max_nan(most, fabsf(single(c)));
            const unsigned bits = __reduce_max_sync(0xffffffffu, __float_as_uint(most) & 0x7fffffffu);
            if (lane == 0) atomicMax(&top[n], bits);
            __syncthreads();
            const RowScale s = row_scale(__uint_as_float(top[n]));
            const bool none = s.inverse == 0.f;
            if (n < f.N && at == 0) scale[n] = s.scale;
            auto put = [&](int v, uint4 q) {
                if (none) q = make_uint4(0, 0, 0, 0);
                unsigned c[V / 4];
#pragma unroll
                for (int i = 0; i < V / 4; ++i)
                    c[i] = pack_codes(rounded(value(q, 4 * i), value(q, 4 * i + 1), s.inverse),
                                      rounded(value(q, 4 * i + 2), value(q, 4 * i + 3), s.inverse));
                if constexpr (V == 4) reinterpret_cast<unsigned *>(out)[v] = c[0];
                else reinterpret_cast<uint2 *>(out)[v] = make_uint2(c[0], c[1]);
            };
#pragma unroll
            for (int h = 0; h < H; ++h)
                if (at + h * WR * 32 < vectors) put(at + h * WR * 32, kept[h]);
            for (int v = at + H * WR * 32; v < vectors; v += WR * 32) put(v, reinterpret_cast<const uint4 *>(x)[v]);
            for (int c = vectors * V + at; c < cols; c += WR * 32)
                out[c] = (int8_t)__float_as_uint(rounded(none ? 0.f : single(c), 0.f, s.inverse).x);
        }
    }
    __syncthreads();

    // ---- the sums (all warps go through as many rounds: partial sums meet in shared memory)
    const int rounds = (groups + (int)gridDim.x * per - 1) / ((int)gridDim.x * per);
    for (int round = 0; round < rounds; ++round) {
        int acc[kOut][NB] = {};
        if (group < groups) {
#pragma unroll
            for (int d = 0; d < D; ++d)
                if (VEC && v0 + d * kw * 32 < whole) {
#pragma unroll
                    for (int n = 0; n < NB; ++n) {
                        const uint4 u = reinterpret_cast<const uint4 *>(codes + n * pitch)[v0 + d * kw * 32];
#pragma unroll
                        for (int i = 0; i < kOut; ++i) acc[i][n] = dot16(first[d][i], u, acc[i][n]);
                    }
                }
#pragma unroll(NB == 1 ? 4 : NB <= 4 ? 2 : 1)
            for (int v = v0 + D * kw * 32; v < whole; v += kw * 32) {
                uint4 q[kOut];
#pragma unroll
                for (int i = 0; i < kOut; ++i) q[i] = reinterpret_cast<const uint4 *>(w[i])[v];
#pragma unroll
                for (int n = 0; n < NB; ++n) {
                    const uint4 u = reinterpret_cast<const uint4 *>(codes + n * pitch)[v];
#pragma unroll
                    for (int i = 0; i < kOut; ++i) acc[i][n] = dot16(q[i], u, acc[i][n]);
                }
            }
            for (int k = whole * 16 + v0; k < f.Cs; k += kw * 32) {
                int q[kOut];
#pragma unroll
                for (int i = 0; i < kOut; ++i) q[i] = w[i][k];
#pragma unroll
                for (int n = 0; n < NB; ++n) {
                    const int u = codes[n * pitch + k];
#pragma unroll
                    for (int i = 0; i < kOut; ++i) acc[i][n] += q[i] * u;
                }
            }
        }
        const int mine = group;
        group += gridDim.x * per;
        if (group < groups) load_first();
#pragma unroll
        for (int i = 0; i < kOut; ++i)
#pragma unroll
            for (int n = 0; n < NB; ++n) {
                const int sum = __reduce_add_sync(0xffffffffu, acc[i][n]);
                if (lane == i * NB + n) red[warp][lane] = sum;
            }
        if (kw > 1) __syncthreads();
        else __syncwarp();
        const int i = lane / NB, n = lane % NB, m = mine * kOut + i;
        if (part == 0 && lane < kOut * NB && mine < groups && m < f.Ct && n < f.N) {
            int sum = 0;
            for (int p = 0; p < kw; ++p) sum += red[warp + p][lane];
            const float xs = scale[n], ws = f.wscale[m];
            const bool swap = !(fabsf(xs) < kLargeScale);  // (as scaled16_large has it)
            finish_one(f.e, n, m, (float)sum * (swap ? ws : xs) * (swap ? xs : ws));
        }
        if (kw > 1 && round + 1 < rounds) __syncthreads();
    }
}

int few_block(int N) { return N <= 2 ? N : N <= 4 ? 4 : 8; }  // rows of a kernel, of a CTA
// Whether that is sooner done than a product on the tensor cores behind a launch that makes the codes:
// every CTA making them for itself costs more with more of them, and sums of four products, and the
// joining of each output's, more with more of those.  us from memory, few rows and tensor cores: 1 x 9216 -> 4096
// 10.9 and 15.3, 4 x 9216 -> 4096 13.4 and 15.5, 8 x 4096 -> 1000 7.3 and 10.4, -> 4096 10.5 and 11.7, -> 8192
// 14.2 and 14.5; 8 x 9216 -> 4096 17.9 and 15.5, -> 9216 27.4 and 21.8.  More rows: 64 x 1024 -> 1024 5.0 and 8.3,
// 16 x 2000 -> 2000 8.5 and 9.6, 30 x 2000 -> 2000 10.1 and 9.8, 100 x 1000 -> 1000 7.9 and 9.0; 9 x 4096 -> 4096
// 12.5 and 11.9, 57 x 78 -> 6139 12.4 and 6.5.  x as codes: 8 x 4096 -> 4096 9.0 and 11.8, 30 x 2000 -> 2000 8.0 and
// 9.8, 8 x 9216 -> 4096 14.6 and 15.5.  It goes by sizes alone, so that where it holds no workspace is asked for:
// with W off 16 bytes one row is sooner here (9216 -> 4096 28.8 and 38.1, 4096 -> 1000 6.7 and 14.0), four rows and
// more are not (4 x 9216 -> 4096 49 and 37, 8 x 4096 -> 4096 36.6 and 22.0, 64 x 1024 -> 1024 11.9 and 10.6).
bool few_rows(int N, int Cs, int Ct) {
    if ((long long)std::min(N, kFewRows) * Cs > 40960) return false;
    return N <= kFewRows || ((long long)N * Ct <= 1 << 17 && (double)N * Cs * Ct <= 1.2e8);
}

template <typename T, bool VEC>
qcnn_status launch_few_of(Int8Product f, cudaStream_t st) {
    const int NB = few_block(f.N), groups = cdiv(f.Ct, kOut), blocks = cdiv(f.N, NB);
    const int most = std::max(1, few_ctas(NB) * num_sms() / blocks);
    const int threads = few_threads(NB), warps = threads / 32;
    // as many warps to an output as have terms, while the outputs alone do not take all warps
    f.kw = 1;
    while (f.kw < warps && groups * 2ll * f.kw <= most * warps && f.Cs > f.kw * 512) f.kw *= 2;
    const dim3 grid(std::min(most, cdiv(groups, warps / f.kw)), blocks);
    const size_t smem = (size_t)NB * ((f.Cs + 15) / 16 * 16);
    const auto launch = [&](auto k) {
        const qcnn_status rc = allow_smem(reinterpret_cast<const void *>(k));
        return rc != QCNN_OK ? rc : launch_pdl(k, grid, dim3(threads), smem, st, f);
    };
    if (NB == 1) return launch(few_rows_kernel<T, 1, VEC>);
    if (NB == 2) return launch(few_rows_kernel<T, 2, VEC>);
    if (NB == 4) return launch(few_rows_kernel<T, 4, VEC>);
    return launch(few_rows_kernel<T, 8, VEC>);
}
qcnn_status launch_few(const Int8Product &f, bool codes, int dtype, bool vec, cudaStream_t st) {
    if (codes) return vec ? launch_few_of<int8_t, true>(f, st) : launch_few_of<int8_t, false>(f, st);
    if (dtype == QCNN_BF16)
        return vec ? launch_few_of<unsigned short, true>(f, st) : launch_few_of<unsigned short, false>(f, st);
    return vec ? launch_few_of<float, true>(f, st) : launch_few_of<float, false>(f, st);
}

// ------------------------------------------------------------------ copies
// What the tensor-core product cannot read as it is: codes of x as fp16, and codes of W whose rows are
// off 16 bytes.  A warp takes pieces of rows, a lane 16 neighbours at a time.
struct CopyJob {
    const int8_t *src = nullptr;
    long long ld = 0, rows = 0;
    int cols = 0, per_row = 0, vec = 0;
    void *dst = nullptr;
    long long pitch = 0;  // elements, a multiple of 16 bytes
    int *sums = nullptr;  // HALF: null, or of the codes' magnitudes, a piece of a row each
    int blocks = 0;       // CTAs of 256 threads; 0: nothing to do
};
constexpr int kCopyCols = kInt8Segment;
template <bool HALF>
__device__ __forceinline__ void copy_part(const CopyJob &j, int block) {
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const long long all = j.rows * j.per_row;
    for (long long i = (long long)block * 8 + warp; i < all; i += (long long)j.blocks * 8) {
        const long long r = i / j.per_row;
        const int first = (int)(i - r * j.per_row) * kCopyCols, end = min(j.cols, first + kCopyCols);
        const int8_t *s = j.src + r * j.ld;
        [[maybe_unused]] int magnitude = 0;
        for (int c = first + lane * 16; c < end; c += 512) {
            unsigned w[4] = {};
            if (j.vec && c + 16 <= j.cols) {
                const uint4 q = *reinterpret_cast<const uint4 *>(s + c);
                w[0] = q.x, w[1] = q.y, w[2] = q.z, w[3] = q.w;
            } else {
#pragma unroll
                for (int k = 0; k < 16; ++k)
                    if (c + k < j.cols) w[k / 4] |= (unsigned)(uint8_t)s[c + k] << k % 4 * 8;
            }
            if constexpr (!HALF) {
                *reinterpret_cast<uint4 *>(static_cast<int8_t *>(j.dst) + r * j.pitch + c) =
                    make_uint4(w[0], w[1], w[2], w[3]);
            } else {
                unsigned h[8];
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    const float2 v = make_float2((float)(int8_t)(w[k / 2] >> k % 2 * 16),
                                                 (float)(int8_t)(w[k / 2] >> (k % 2 * 16 + 8)));
                    asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(h[k]) : "f"(v.y), "f"(v.x));
                    magnitude += (int)(fabsf(v.x) + fabsf(v.y));
                }
                uint4 *d = reinterpret_cast<uint4 *>(static_cast<unsigned short *>(j.dst) + r * j.pitch + c);
                d[0] = make_uint4(h[0], h[1], h[2], h[3]);
                if (c + 8 < j.pitch) d[1] = make_uint4(h[4], h[5], h[6], h[7]);
            }
        }
        if constexpr (HALF) {
            if (j.sums) {
                magnitude = __reduce_add_sync(0xffffffffu, magnitude);
                if (lane == 0) j.sums[i] = magnitude;
            }
        }
    }
}
__global__ void __launch_bounds__(256) copy_kernel(CopyJob x, CopyJob w) {
    grid_dep_sync();
    if ((int)blockIdx.x < x.blocks) copy_part<true>(x, blockIdx.x);
    else copy_part<false>(w, blockIdx.x - x.blocks);
}

// ------------------------------------------------------------------- space
long long pad16(long long v) { return (v + 15) / 16 * 16; }
bool rows16(const void *p, long long ld) { return reinterpret_cast<uintptr_t>(p) % 16 == 0 && ld % 16 == 0; }
bool codes_ok(const void *p, long long ld, long long rows, long long cols) { return ld >= cols && (rows == 0 || p); }
// Tiles of up to 256 rows or outputs count from 0 in ints, past the last of them too.
qcnn_status dense_sizes(int N, int Cs, int Ct) {
    if (N < 0 || Cs <= 0 || Cs > kInt8MaxTerms || Ct <= 0) return QCNN_ERR_INVALID_ARG;
    return std::max(N, Ct) > INT_MAX - 256 ? QCNN_ERR_UNSUPPORTED : QCNN_OK;
}

// (few rows: none) x in fp16, its scales and sums, W's rows on 16 bytes.
struct Space {
    void *x = nullptr;
    float *scale = nullptr;
    int *sums = nullptr;
    int8_t *w = nullptr;
    size_t bytes = 0;
};
Space carve(int N, int Cs, int Ct, bool x_codes, bool w_copy, void *ws) {
    Carver c{static_cast<uint8_t *>(ws)};
    Space s;
    if (few_rows(N, Cs, Ct)) return s;
    s.x = c.take((size_t)N * pad8(Cs) * 2);
    if (!x_codes) s.scale = c.array<float>(N);
    if (int8_sums(plan_int8(Ct, N, Cs), Cs)) s.sums = c.array<int>((size_t)N * cdiv(Cs, kInt8Segment));
    if (w_copy) s.w = c.array<int8_t>((size_t)Ct * pad16(Cs));
    s.bytes = c.used;
    return s;
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
    return launch_quantize(x, ldx, N, C, codes, ldc, false, scale, nullptr, dtype, static_cast<cudaStream_t>(stream));
}

qcnn_status qcnn_int8_dense_workspace_size(int N, int Cs, int Ct, int x_codes, int aligned, size_t *bytes) {
    const qcnn_status sizes = bytes ? dense_sizes(N, Cs, Ct) : QCNN_ERR_INVALID_ARG;
    if (sizes != QCNN_OK) return sizes;
    *bytes = N ? carve(N, Cs, Ct, x_codes, !aligned, nullptr).bytes : 0;
    return QCNN_OK;
}

qcnn_status qcnn_int8_route_info(int N, int Cs, int Ct, int info[4]) {
    const qcnn_status sizes = info && N ? dense_sizes(N, Cs, Ct) : QCNN_ERR_INVALID_ARG;
    if (sizes != QCNN_OK) return sizes;
    const bool few = few_rows(N, Cs, Ct);
    const Int8Plan p = few ? Int8Plan{0, 0, 0} : plan_int8(Ct, N, Cs);
    info[0] = few;
    info[1] = p.bn;
    info[2] = p.cg;
    info[3] = p.splits;
    return QCNN_OK;
}

qcnn_status qcnn_int8_dense_forward(const void *x, long long ldx, const float *xscale, int N, int Cs,
                                    const int8_t *W, long long ldw, const float *wscale, int Ct, const float *bias,
                                    int act, const void *residual, long long ldr, void *y, long long ldy, int dtype,
                                    void *workspace, size_t workspace_bytes, void *stream) {
    const qcnn_status sizes = dense_sizes(N, Cs, Ct);
    if (sizes == QCNN_ERR_INVALID_ARG || !dtype_ok(dtype) || act < QCNN_ACT_NONE || act > QCNN_ACT_SILU)
        return QCNN_ERR_INVALID_ARG;
    if (!(xscale ? codes_ok(x, ldx, N, Cs) : matrix_ok(x, ldx, N, Cs, dtype)) || !codes_ok(W, ldw, Ct, Cs) ||
        !wscale || !matrix_ok(y, ldy, N, Ct, dtype) || (residual && !matrix_ok(residual, ldr, N, Ct, dtype)) ||
        reinterpret_cast<uintptr_t>(bias) % 4 || reinterpret_cast<uintptr_t>(wscale) % 4 ||
        reinterpret_cast<uintptr_t>(xscale) % 4)
        return QCNN_ERR_INVALID_ARG;
    if (sizes != QCNN_OK || N == 0) return sizes;
    const bool w_copy = !rows16(W, ldw);
    const Space s = carve(N, Cs, Ct, xscale != nullptr, w_copy, workspace);
    qcnn_status rc = workspace_ok(workspace, workspace_bytes, s.bytes);
    if (rc != QCNN_OK) return rc;
    const cudaStream_t st = static_cast<cudaStream_t>(stream);
    PdlScope pdl;
    GemmEpi e;
    const int type = dtype == QCNN_BF16 ? GEMM_T_BF16 : GEMM_T_F32;
    e.bias = bias;
    e.act = act;
    e.add = residual;
    e.lda = ldr;
    e.add_type = type;
    e.out = y;
    e.ldo = ldy;
    e.out_type = type;
    if (few_rows(N, Cs, Ct))
        return launch_few(Int8Product{x, W, ldx, ldw, xscale, wscale, N, Cs, Ct, e, 1}, xscale != nullptr, dtype, !w_copy, st);
    CopyJob jx, jw;
    const auto job = [&](const void *src, long long ld, long long rows, void *dst, long long pitch) {
        CopyJob j;
        j.src = static_cast<const int8_t *>(src);
        j.ld = ld;
        j.rows = rows;
        j.cols = Cs;
        j.per_row = cdiv(Cs, kCopyCols);
        j.vec = rows16(src, ld);
        j.dst = dst;
        j.pitch = pitch;
        j.blocks = (int)std::min<long long>((rows * j.per_row + 7) / 8, (long long)num_sms() * 8);
        return j;
    };
    if (!xscale) {
        rc = launch_quantize(x, ldx, N, Cs, s.x, pad8(Cs), true, s.scale, s.sums, dtype, st);
        if (rc != QCNN_OK) return rc;
    } else {
        jx = job(x, ldx, N, s.x, pad8(Cs));
        jx.sums = s.sums;
    }
    if (w_copy) jw = job(W, ldw, Ct, s.w, pad16(Cs));
    if (jx.blocks + jw.blocks &&
        (rc = launch_pdl(copy_kernel, dim3(jx.blocks + jw.blocks), dim3(256), 0, st, jx, jw)) != QCNN_OK)
        return rc;
    Int8Problem p;
    p.x = s.x;
    p.ldx = pad8(Cs);
    p.W = w_copy ? s.w : W;
    p.ldw = w_copy ? pad16(Cs) : ldw;
    p.w_late = w_copy;
    p.xscale = xscale ? xscale : s.scale;
    p.wscale = wscale;
    p.sums = s.sums;
    p.segs = cdiv(Cs, kInt8Segment);
    p.m = Ct;
    p.n = N;
    p.k = Cs;
    p.e = e;
    return launch_int8(plan_int8(Ct, N, Cs), p, st);
}

}  // extern "C"
