// int8_gemm.cu -- products of 8-bit integers on the tensor cores (int8_gemm.cuh).
//
//   y[n][m] = act(xscale[n] (wscale[m] sum_k x[n][k] W[m][k]) + bias[m]) + r
//
// GB300's tcgen05 multiplies no 8-bit integers (kind::i8 does not assemble for sm_103a), and those of mma.sync go
// at 158 TOP/s (m16n8k32 from registers, measured) where fp16 by tcgen05 has 1,880 TFLOP/s; and fp16 holds every
// code exactly: W is widened on its way, from bytes in shared memory to tensor memory, from where
// the MMAs take it as their operand A; x comes widened (fp16, of the pass that quantizes it) as B.  So W
// is read once, as bytes, and shared memory carries per 128 terms and 128 rows 16 KB of W in and out
// beside x's tile in and out.
//
// Sums.  Products of codes are integers of at most 2^14, sums of up to 1024 of them at most 2^24: fp32
// accumulators hold every one of them exactly.  Before a sum could leave that range it is drained to
// registers, and the sums that a result has more than one of are added there as integers: exact, and
// rounded to fp32 once.
//
// Tile.  As gemm_kernel.cuh's: 128 (a pair of CTAs: 256) rows of m, TMEM lanes, x bn columns of n.  160
// to 256 columns (of a pair, in steps of 32, so that the last round of tiles is a full one: 1000 x 2000 ->
// 3000 in tiles of 192 20.0 us, of 256 22.5; 1500 x 9216 -> 4096 94 and 108) are two accumulators, of 64 to
// 128 columns, that the MMAs of a block of 128 terms fill one after the other, so that draining the first
// overlaps the MMAs of the second; up to 128 columns take two accumulators in turn.  TMEM: 256 columns of
// accumulators, four stages of W (three where results are staged), 128 terms in 64 columns each.
//
// Bounds.  Large: the MMAs (4096 x 4096 -> 8192 with GELU and a residual in bf16 145 us, 1.9 PFLOP/s, the
// tensor pipe active for 75%).  Ragged: last rounds and stores of odd rows (3001 x 2047 -> 5003 in fp32 42
// us).  Tiles of 128 columns of one CTA: what passes through its shared memory for a block of 128 terms, 48 KB in
// and out, 768 of its 1,000 clocks (128 x 9216 -> 4096 16 us, tensor pipe 16%); narrower ones: the widening.
//
// Roles (20 warps, WIDE 16): 0 TMA of x, 1 MMA, 2 TMEM and TMA of W, 3 (WIDE) where sums are drained, 4-11
// drain and epilogue (two warps per TMEM lane quarter), from 12 on widen: a warp has its 32 rows of W, a lane
// a row, 128 terms at a time.
#define QCNN_UNIT_RECORDS
#include "int8_gemm.cuh"

#include "gemm_kernel.cuh"

#include <algorithm>
#include <array>
#include <map>
#include <mutex>

namespace qcnn {
namespace {

// WIDE: one group of four warps widens (the drain's registers leave no room for another).  Else two, in turn a
// block each, up to 64 columns (16 x 9216 -> 9216 22.0 us, 24.5 with one, 257 x 2047 -> 2001 13.6 and 15.1, 64 x
// 9216 -> 4096 17.9 and 19.0); of 128 columns, bound by shared memory, one (128 x 9216 -> 4096 20.6, 21.1 with
// two).
constexpr int int8_threads(bool wide) { return wide ? 512 : 640; }
constexpr int kTerms = 128;            // of a block (with half of that, its waits took a fifth of the time)
constexpr int kStages = 4;             // blocks of W in TMEM, at most
constexpr int kWCols = 64;             // TMEM columns of one
constexpr unsigned kRawBytes = 128 * kTerms;  // a copy of W: 128 rows
constexpr int kRawStagesMax = 8;
constexpr int kSumBlocks = kInt8Segment / kTerms;  // blocks whose sum is exact, whatever the codes
constexpr int kSegs = kInt8MaxTerms / kInt8Segment + 1;  // segments at most
constexpr size_t kSmem = 222 * 1024;   // dynamic, with 1 KB to align the stages
constexpr size_t kSmemFloor = 120 * 1024;  // one CTA per SM: all tensor memory is taken

struct Int8Args {
    CUtensorMap map_w, map_x;
    int m, n, kblocks, m_tiles, n_tiles, kb_per_split, group, units;
    int bn, S, R, cl, w_late;
    int wide[2];     // WIDE: columns of a tile's two accumulators
    uint32_t idesc[2];
    CUtensorMap map_x2;  // WIDE: x for the second
    int staged;      // WIDE: results (and the residual) pass through shared memory behind the stages
    CUtensorMap map_out, map_add;
    unsigned stage;  // bytes of a stage of x
    const float *xscale, *wscale;
    const int *sums;  // WIDE: of the magnitudes of x's codes, [n][segs], each of 1024 terms; null: segs 1
    int segs;
    GemmEpi e;
};
struct Int8Shared {
    uint64_t full[kStages], empty[kStages], raw_full[kRawStagesMax], raw_empty[kRawStagesMax], tfull[2], tempty[2], done;
    uint64_t plan_full[2], plan_empty[2];
    uint64_t residual[8];
    // Of two tiles: whether a sum ends with segment s.  A byte each: kept as bits of 32-bit words, whose indices
    // were in range, the kernel faulted from segment 8 on; why was not found.
    uint8_t ends[2][kSegs];
    unsigned tmem;
    int give_up;
};

struct Int8Tile {
    int mt, nt, kb0, kb1;
};
__device__ __forceinline__ Int8Tile int8_tile(const Int8Args &g, int u, int share) {
    const int per = g.group * g.n_tiles, gr = u / per, m0 = gr * g.group, w = min(g.group, g.m_tiles - m0);
    u -= gr * per;
    Int8Tile t;
    t.nt = u / w;
    t.mt = m0 + u - t.nt * w;
    t.kb0 = share * g.kb_per_split;
    t.kb1 = min(g.kblocks, t.kb0 + g.kb_per_split);
    return t;
}

__device__ __forceinline__ bool wait_for(Int8Shared &s, uint64_t *bar, unsigned parity) {
    bool ok = mbar_wait_bounded(bar, parity, 64);
    for (unsigned i = 0; i < kPolls / 64 && !ok; ++i) {
        if (*reinterpret_cast<volatile int *>(&s.give_up)) return false;
        ok = mbar_wait_bounded(bar, parity, 64);
    }
    if (!ok) {
        *reinterpret_cast<volatile int *>(&s.give_up) = 1;
        QCNN_RECORD_IF(true, QCNN_CHECK_TIMEOUT);
    }
    return ok;
}
__device__ __forceinline__ bool warp_wait_for(Int8Shared &s, uint64_t *bar, unsigned parity) {
    return __all_sync(0xffffffffu, wait_for(s, bar, parity));
}
template <int CG>
__device__ __forceinline__ void tma_box(unsigned dst, const CUtensorMap *map, int x, int y, uint64_t *bar) {
    if constexpr (CG == 1)
        tma_load_2d(dst, map, x, y, bar);
    else  // (counted on the pair's first CTA)
        asm volatile(
            "cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.tile.mbarrier::complete_tx::bytes "
            "[%0], [%1, {%2, %3}], [%4];\n" ::"r"(dst),
            "l"(map), "r"(x), "r"(y), "r"(smem_addr(bar) & 0xFEFFFFFFu)
            : "memory");
}
template <int CG>
__device__ __forceinline__ void mma_tmem(unsigned d, unsigned a, uint64_t b, uint32_t idesc, bool acc) {
    if constexpr (CG == 1)
        mma_ts(d, a, b, idesc, acc);
    else
        asm volatile(
            "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
            "tcgen05.mma.cta_group::2.kind::f16 [%0], [%1], %2, %3, p;\n\t}\n" ::"r"(d),
            "r"(a), "l"(b), "r"(idesc), "r"((unsigned)acc)
            : "memory");
}
__device__ __forceinline__ void tmem_st32(unsigned taddr, const unsigned (&v)[32]) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], "
        "{%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, "
        "%17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31, %32};\n" ::"r"(taddr),
        "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7]), "r"(v[8]), "r"(v[9]),
        "r"(v[10]), "r"(v[11]), "r"(v[12]), "r"(v[13]), "r"(v[14]), "r"(v[15]), "r"(v[16]), "r"(v[17]), "r"(v[18]),
        "r"(v[19]), "r"(v[20]), "r"(v[21]), "r"(v[22]), "r"(v[23]), "r"(v[24]), "r"(v[25]), "r"(v[26]), "r"(v[27]),
        "r"(v[28]), "r"(v[29]), "r"(v[30]), "r"(v[31])
        : "memory");
}

// An arrival on CTA 0 of the pair, of what this thread did to tensor memory: tcgen05.wait::st has completed
// its stores and the fence before it orders them with the arrival, so that the arrival itself orders nothing
// and is relaxed, at the scope of both CTAs.  (With .release.cluster, which waits for all that the thread has
// under way, a block of 64 terms took 1,700 clocks instead of 600.)
__device__ __forceinline__ void arrive_first(uint64_t *bar) {
    asm volatile(
        "{\n\t.reg .b32 a;\n\t"
        "mapa.shared::cluster.u32 a, %0, 0;\n\t"
        "mbarrier.arrive.relaxed.cluster.shared::cluster.b64 _, [a];\n\t}\n" ::"r"(smem_addr(bar))
        : "memory");
}
// 32 columns of this warp's lanes, there after tcgen05.wait::ld.
__device__ __forceinline__ void tmem_ld32_nowait(unsigned taddr, float (&a)[16], float (&b)[16]) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 "
        "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
        "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];\n"
        : "=f"(a[0]), "=f"(a[1]), "=f"(a[2]), "=f"(a[3]), "=f"(a[4]), "=f"(a[5]), "=f"(a[6]), "=f"(a[7]), "=f"(a[8]),
          "=f"(a[9]), "=f"(a[10]), "=f"(a[11]), "=f"(a[12]), "=f"(a[13]), "=f"(a[14]), "=f"(a[15]), "=f"(b[0]),
          "=f"(b[1]), "=f"(b[2]), "=f"(b[3]), "=f"(b[4]), "=f"(b[5]), "=f"(b[6]), "=f"(b[7]), "=f"(b[8]), "=f"(b[9]),
          "=f"(b[10]), "=f"(b[11]), "=f"(b[12]), "=f"(b[13]), "=f"(b[14]), "=f"(b[15])
        : "r"(taddr)
        : "memory");
}

// Four codes as fp16: a byte with its sign bit turned over is code + 128, below 0x64 in the high byte
// 1024 more; 1152 taken off leaves the code, exactly.
__device__ __forceinline__ void widen4(unsigned w, unsigned &lo, unsigned &hi) {
    const unsigned u = w ^ 0x80808080u;
    const unsigned a = __byte_perm(u, 0x64646464u, 0x4140), b = __byte_perm(u, 0x64646464u, 0x4342);
    asm("sub.rn.f16x2 %0, %1, %2;" : "=r"(lo) : "r"(a), "r"(0x64806480u));
    asm("sub.rn.f16x2 %0, %1, %2;" : "=r"(hi) : "r"(b), "r"(0x64806480u));
}

// ------------------------------------------------------------------ epilogue
// gelu(z) = max(z, 0) - |z| / 2 erfc(|z| / sqrt 2), erfc(x) = t (a1 + t (a2 + ...)) exp(-x^2), t = 1 / (1 +
// p x): Abramowitz and Stegun, Handbook of Mathematical Functions, 7.1.26, to 1.5e-7, here of |z| / 2.
// silu(z) = z / (1 + exp(-z)).  In pairs, exponentials and reciprocals by the fast units (2 and 1 ulp):
// with erff the 256 x 256 tiles of 4096 terms took longer in the epilogue than in the products.  For
// bf16 results, whose rounding is up to 2^-8 of them.
__device__ __forceinline__ float fast_rcp(float x) {
    float r;
    asm("rcp.approx.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}
__device__ __forceinline__ float2 both(float v) { return make_float2(v, v); }
__device__ __forceinline__ float above_zero(float a) {  // (NaN stays)
    float r;
    asm("max.NaN.f32 %0, %1, 0f00000000;" : "=f"(r) : "f"(a));
    return r;
}
// |a|, but of +inf the largest finite value: times erfc's 0 that is 0, and gelu(inf) = inf.
__device__ __forceinline__ float magnitude(float a) { return fmaxf(fminf(a, 3.402823466e38f), -a); }
__device__ __forceinline__ void gelu2(float &a, float &b) {
    const float2 z = make_float2(a, b);
    constexpr float kP = 0.3275911f * 0.70710678118654752f;
    const float2 t = make_float2(fast_rcp(fmaf(fabsf(a), kP, 1.f)), fast_rcp(fmaf(fabsf(b), kP, 1.f)));
    const float2 x = __fmul2_rn(__fmul2_rn(z, both(-0.5f * kLog2e)), z);
    const float2 q = make_float2(ex2(x.x), ex2(x.y));
    // (the polynomial times -1/2)
    float2 p = __ffma2_rn(t, both(-0.5f * 1.061405429f), both(0.5f * 1.453152027f));
    p = __ffma2_rn(p, t, both(-0.5f * 1.421413741f));
    p = __ffma2_rn(p, t, both(0.5f * 0.284496736f));
    p = __ffma2_rn(p, t, both(-0.5f * 0.254829592f));
    p = __fmul2_rn(__fmul2_rn(p, t), q);
    a = fmaf(magnitude(a), p.x, above_zero(a));
    b = fmaf(magnitude(b), p.y, above_zero(b));
}
// The same for fp32 results, to their last bits.
// gelu: below 1.5 z (1/2 + z R(z^2)), R a polynomial near (Phi(z) - 1/2) / z (to 2.7e-9 of it); beyond as above
// with a sixth term and coefficients for that range alone (to 6e-7 of erfc, 4e-8 of what it is taken from).
// Both fitted for the least largest error (Lawson's weights).  In fp32 2.9e-8 of the norm of normal z where
// erff has 4.8e-8.
__device__ __forceinline__ void gelu2_exact(float &a, float &b) {
    const float2 z = make_float2(a, b), u = __fmul2_rn(z, z);
    float2 r = __ffma2_rn(u, both(4.11555712e-07f), both(-8.71830202e-06f));
    r = __ffma2_rn(r, u, both(0.000114356385f));
    r = __ffma2_rn(r, u, both(-0.00118648848f));
    r = __ffma2_rn(r, u, both(0.0099732413f));
    r = __ffma2_rn(r, u, both(-0.066490335f));
    r = __ffma2_rn(r, u, both(0.398942279f));
    const float2 near = __ffma2_rn(z, __fmul2_rn(z, r), __fmul2_rn(z, both(0.5f)));
    constexpr float kP = 0.3275911f * 0.70710678118654752f;
    const float2 t = make_float2(fast_rcp(fmaf(fabsf(a), kP, 1.f)), fast_rcp(fmaf(fabsf(b), kP, 1.f)));
    const float2 x = __fmul2_rn(__fmul2_rn(z, both(-0.5f * kLog2e)), z);
    const float2 q = make_float2(ex2(x.x), ex2(x.y));
    // (times -1/2)
    float2 p = __ffma2_rn(t, both(-0.5f * 0.324728743f), both(0.5f * 0.128127106f));
    p = __ffma2_rn(p, t, both(-0.5f * 0.295275164f));
    p = __ffma2_rn(p, t, both(-0.5f * 0.132917903f));
    p = __ffma2_rn(p, t, both(-0.5f * 0.191366617f));
    p = __ffma2_rn(p, t, both(-0.5f * 0.184408403f));
    p = __fmul2_rn(__fmul2_rn(p, t), q);
    a = fabsf(a) < 1.5f ? near.x : fmaf(magnitude(a), p.x, above_zero(a));
    b = fabsf(b) < 1.5f ? near.y : fmaf(magnitude(b), p.y, above_zero(b));
}
// silu: z log2 e in two parts, the second (what rounding the first took off, and log2 e's own rest) as 1 + d ln 2
// behind the exponential.  z is held to where that is finite: beyond, exp(-z) is 0 or infinite all the same.
__device__ __forceinline__ void silu2_exact(float &a, float &b) {
    const float2 z = make_float2(fminf(fmaxf(a, -200.f), 200.f), fminf(fmaxf(b, -200.f), 200.f));
    const float2 t = __fmul2_rn(z, both(-kLog2e));
    float2 d = __ffma2_rn(z, both(kLog2e), t);
    d = __ffma2_rn(z, both((float)(1.4426950408889634074 - kLog2e)), d);
    float2 q = __fmul2_rn(make_float2(ex2(t.x), ex2(t.y)), __ffma2_rn(d, both(-0.69314718f), both(1.f)));
    q = __fadd2_rn(q, both(1.f));
    a *= fast_rcp(q.x);
    b *= fast_rcp(q.y);
}
// exact: of fp32 results
__device__ __forceinline__ void int8_act16(float (&v)[16], int act, bool exact) {
    if (act == QCNN_ACT_RELU) {
#pragma unroll
        for (int i = 0; i < 16; ++i) v[i] = act_apply(v[i], QCNN_ACT_RELU);
    } else if (exact) {
        if (act == QCNN_ACT_GELU) {
            // (four at a time, the others moving up: its instructions come four times and not sixteen, and its
            // constants, in pairs, leave the drain its registers)
#pragma unroll 1
            for (int k = 0; k < 4; ++k) {
                float t[4];
#pragma unroll
                for (int j = 0; j < 4; ++j) t[j] = v[j];
#pragma unroll
                for (int j = 0; j < 4; j += 2) gelu2_exact(t[j], t[j + 1]);
#pragma unroll
                for (int j = 0; j < 12; ++j) v[j] = v[j + 4];
#pragma unroll
                for (int j = 0; j < 4; ++j) v[12 + j] = t[j];
            }
        } else if (act == QCNN_ACT_SILU) {
#pragma unroll
            for (int i = 0; i < 16; i += 2) silu2_exact(v[i], v[i + 1]);
        }
    } else if (act == QCNN_ACT_GELU) {
#pragma unroll
        for (int i = 0; i < 16; i += 2) gelu2(v[i], v[i + 1]);
    } else if (act == QCNN_ACT_SILU) {
#pragma unroll
        for (int i = 0; i < 16; ++i) v[i] *= fast_rcp(1.f + ex2(-kLog2e * v[i]));
    }
}

// v = alpha xs v + bias of 16 columns.  xs first: sums are whole numbers below 2^31, so that neither product
// leaves fp32's range where the result does not while xs is below kLargeScale.
__device__ __forceinline__ void scaled16(float (&v)[16], const float *xs, float alpha, float bias) {
    const float2 a2 = both(alpha), b2 = both(bias);
#pragma unroll
    for (int j = 0; j < 16; j += 4) {
        const float4 s = *reinterpret_cast<const float4 *>(xs + j);
        float2 z = __ffma2_rn(a2, __fmul2_rn(make_float2(v[j], v[j + 1]), make_float2(s.x, s.y)), b2);
        v[j] = z.x, v[j + 1] = z.y;
        z = __ffma2_rn(a2, __fmul2_rn(make_float2(v[j + 2], v[j + 3]), make_float2(s.z, s.w)), b2);
        v[j + 2] = z.x, v[j + 3] = z.y;
    }
}
// The same where a scale may be larger: such columns take alpha first.  (In a place of its own, before the
// epilogue, which then has scales of one, or behind a branch around the whole of int8_finish: as a branch of
// scaled16, whose instructions come many times, 3001 x 2047 -> 5003 took 58.6 us instead of 56.8 without a
// large scale.)
__device__ __forceinline__ void scaled16_large(float (&v)[16], const float *xs, float alpha, float bias) {
#pragma unroll
    for (int j = 0; j < 16; ++j) {
        const bool swap = !(fabsf(xs[j]) < kLargeScale);
        v[j] = fmaf(swap ? xs[j] : alpha, v[j] * (swap ? alpha : xs[j]), bias);
    }
}

// WIDE, where TMA can write the result (and read the residual): a warp's 32 rows of m pass through its
// part of shared memory, [column][row], by chunks of 16 columns, the residual there before and the result after, each
// element a lane's own.  Few instructions for an element, and few copies of them, are what counts: a tile's
// epilogue is run through once, and is slower the longer its code is (see the copies' times in the kernel).
constexpr unsigned kStagedBytes = 8192;  // of a warp: 128 columns of bf16, 64 of fp32
template <typename T>
__device__ __forceinline__ void staged16(float (&v)[16], const float *xs, float alpha, float bias, int act, bool res,
                                         T *at) {
    scaled16(v, xs, alpha, bias);
    int8_act16(v, act, sizeof(T) == 4);
    if (res) {
#pragma unroll
        for (int j = 0; j < 16; j += 2) {
            if constexpr (sizeof(T) == 4) add2(v[j], v[j + 1], at[j * 32], at[j * 32 + 32]);
            else add2(v[j], v[j + 1], bf16_to_float(at[j * 32]), bf16_to_float(at[j * 32 + 32]));
        }
    }
#pragma unroll
    for (int j = 0; j < 16; j += 2) {
        if constexpr (sizeof(T) == 4) {
            at[j * 32] = v[j], at[j * 32 + 32] = v[j + 1];
        } else {
            const unsigned w = pack_bf16x2(v[j], v[j + 1]);
            at[j * 32] = (unsigned short)w, at[j * 32 + 32] = (unsigned short)(w >> 16);
        }
    }
}
__device__ __forceinline__ void tma_store(const CUtensorMap *map, int x, int y, unsigned src) {
    asm volatile("cp.async.bulk.tensor.2d.global.shared::cta.tile.bulk_group [%0, {%1, %2}], [%3];\n" ::"l"(map),
                 "r"(x), "r"(y), "r"(src)
                 : "memory");
}
// Until this thread's stores have read their shared memory.
__device__ __forceinline__ void tma_stores_read() { asm volatile("cp.async.bulk.wait_group.read 0;\n" ::: "memory"); }

// What the residual has at 16 columns of a lane from n on; count: of them that exist.
__device__ __forceinline__ void fetch_values(const GemmEpi &e, int m, int n, int count, float (&r)[16]) {
    if (e.out_type == GEMM_T_F32) {
        const float *p = static_cast<const float *>(e.add) + (long long)n * e.lda + m;
#pragma unroll
        for (int j = 0; j < 16; ++j, p += e.lda) r[j] = j < count ? *p : 0.f;
    } else {
        const unsigned short *p = static_cast<const unsigned short *>(e.add) + (long long)n * e.lda + m;
#pragma unroll
        for (int j = 0; j < 16; ++j, p += e.lda) r[j] = j < count ? bf16_to_float(*p) : 0.f;
    }
}
// 16 columns of a lane: sums v of row m, columns n to n + count - 1, to the result.  xs: the columns'
// scales; LARGE: some from kLargeScale on.  A warp's lanes are neighbours in the result; two-byte elements go
// in pairs where pairs are aligned (gemm_kernel.cuh).  The whole warp calls it.
template <bool LARGE = false>
__device__ __forceinline__ void int8_finish(const GemmEpi &e, int m, int n, int count, float alpha, float bias,
                                            const float *xs, float (&v)[16]) {
    const bool odd = m & 1;
    if constexpr (LARGE) scaled16_large(v, xs, alpha, bias);
    else scaled16(v, xs, alpha, bias);
    if (e.add) {
        float r[16];
        fetch_values(e, m, n, count, r);
        int8_act16(v, e.act, e.out_type == GEMM_T_F32);
#pragma unroll
        for (int j = 0; j < 16; j += 2) add2(v[j], v[j + 1], r[j], r[j + 1]);
    } else {
        int8_act16(v, e.act, e.out_type == GEMM_T_F32);
    }
    if (e.out_type == GEMM_T_F32) {
        float *p = static_cast<float *>(e.out) + (long long)n * e.ldo + m;
#pragma unroll
        for (int j = 0; j < 16; ++j, p += e.ldo)
            if (j < count) *p = v[j];
    } else if (e.pair & 1) {
        unsigned short *p = static_cast<unsigned short *>(e.out) + (long long)(n + odd) * e.ldo + (m - odd);
#pragma unroll
        for (int j = 0; j < 8; ++j, p += 2 * e.ldo) {
            const unsigned x = exchange(pack_bf16x2(v[2 * j], v[2 * j + 1]), odd);
            if (2 * j < count - odd) *reinterpret_cast<unsigned *>(p) = x;
        }
    } else {
        unsigned short *p = static_cast<unsigned short *>(e.out) + (long long)n * e.ldo + m;
#pragma unroll
        for (int j = 0; j < 16; ++j, p += e.ldo)
            if (j < count) *p = float_to_bf16(v[j]);
    }
}

// ------------------------------------------------------------------- kernel
// WIDE: tiles of 160 to 256 columns, by pairs of CTAs.
template <int CG, bool WIDE>
__global__ void __launch_bounds__(int8_threads(WIDE), 1) int8_kernel(const __grid_constant__ Int8Args g) {
    extern __shared__ __align__(128) unsigned char smem_raw[];
    __shared__ Int8Shared sh;
    __shared__ __align__(16) float column_scales[8][128];
    unsigned char *const smem = smem_raw + (-smem_addr(smem_raw) & 1023u);  // (swizzle atoms)
    const int tid = threadIdx.x, lane = tid & 31;
    const int warp = __shfl_sync(0xffffffffu, tid >> 5, 0);
    unsigned rank = 0;  // of the pair
    int share = 0;      // of a tile's terms
    if constexpr (CG == 2) {
        asm("mov.u32 %0, %%cluster_ctarank;\n" : "=r"(rank));
    } else if (g.cl > 1) {
        asm("mov.u32 %0, %%cluster_ctarank;\n" : "=r"(share));
    }
    const int first_unit = (int)blockIdx.x / (CG * g.cl), step = (int)gridDim.x / (CG * g.cl);
    constexpr int NH = WIDE ? 2 : 1;                 // accumulators of a tile
    // (columns that a tile has before accumulator h, and rows of x here that the first one's MMAs read)
    [[maybe_unused]] const int wide0 = WIDE ? g.wide[0] : g.bn;
    const int rows_x = wide0 / CG;
    const unsigned raw0 = smem_addr(smem) + g.S * g.stage;
    if (tid == 0) {
        for (int i = 0; i < g.S; ++i) {
            mbar_init(&sh.full[i], 1 + 4 * CG);
            mbar_init(&sh.empty[i], 1);
        }
        for (int i = 0; i < g.R; ++i) {
            mbar_init(&sh.raw_full[i], 1);
            mbar_init(&sh.raw_empty[i], 4);
        }
        for (int i = 0; i < 2; ++i) {
            mbar_init(&sh.tfull[i], 1);
            mbar_init(&sh.tempty[i], (WIDE ? 4 : 8) * CG);
            mbar_init(&sh.plan_full[i], 1);
            mbar_init(&sh.plan_empty[i], 8 + (rank == 0));  // (the epilogue's warps, the MMAs' thread)
        }
        for (int i = 0; i < 8; ++i) mbar_init(&sh.residual[i], 1);
        mbar_init(&sh.done, 1);
        sh.give_up = 0;
        asm volatile("fence.mbarrier_init.release.cluster;\n" ::: "memory");
        fence_async_smem();
    }
    if (warp == 2) tmem_alloc_cg<CG>(&sh.tmem);
    tc_fence_before_sync();
    __syncthreads();
    if constexpr (CG == 2) cluster_sync_all();
    tc_fence_after_sync();
    const unsigned tmem = sh.tmem;

    // (640 threads: 48, 2 x 144 and 2 x 72 are 480, 5 x 96; 512: 48, 2 x 192 and 80 are 512, 4 x 128)
    if (warp < 4) set_registers<48, false>();
    if (warp == 0) {
        // ----------------------------------------------------------- TMA of x
        if (elect_one()) {
            grid_dep_sync();
            int slot = 0;
            unsigned par = 0, issued = 0;
            bool ok = true;
            for (int u = first_unit; u < g.units && ok; u += step) {
                const Int8Tile t = int8_tile(g, u, share);
                const int n0 = t.nt * g.bn + (int)rank * rows_x;
                [[maybe_unused]] const int n1 = t.nt * g.bn + wide0 + (int)rank * (g.wide[1] / CG);
                for (int kb = t.kb0; kb < t.kb1; ++kb) {
                    if (!(ok = wait_for(sh, &sh.empty[slot], par ^ 1))) break;
                    uint64_t *const full = &sh.full[slot];
                    if (rank == 0) arrive_expect(full, g.stage * CG);
                    const unsigned d = smem_addr(smem) + slot * g.stage;
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        tma_box<CG>(d + i * rows_x * 128, &g.map_x, kb * kTerms + i * 64, n0, full);
                        if constexpr (WIDE)
                            tma_box<CG>(d + (2 * rows_x + i * (g.wide[1] / CG)) * 128, &g.map_x2, kb * kTerms + i * 64, n1,
                                        full);
                    }
                    ++issued;
                    if (++slot == g.S) {
                        slot = 0;
                        par ^= 1;
                    }
                }
            }
            // no copy of its own under way when the CTA leaves
            if (rank == 0 || !ok)
                for (unsigned i = issued > (unsigned)g.S ? issued - g.S : 0; i < issued; ++i)
                    mbar_wait_bounded(rank == 0 ? &sh.full[i % g.S] : &sh.empty[i % g.S], i / g.S & 1, kPolls);
        }
        __syncwarp();
    } else if (warp == 1) {
        // --------------------------------------------------------------- MMA
        if (rank == 0 && elect_one()) {
            int slot = 0;
            unsigned par = 0;
            unsigned sums = 0, tiles = 0;  // so far
            bool ok = true;
            const uint64_t desc = 1ull << 16 | (uint64_t)(1024 >> 4) << 32 | 1ull << 46 | 2ull << 61 |
                                  (uint64_t)((smem_addr(smem) >> 4) & 0x3FFFu);
            for (int u = first_unit; u < g.units && ok; u += step, ++tiles) {
                const Int8Tile t = int8_tile(g, u, share);
                const bool planned = WIDE && g.sums;
                if (planned && !(ok = wait_for(sh, &sh.plan_full[tiles & 1], tiles >> 1 & 1))) break;
                bool first = true;  // of a sum
                for (int kb = t.kb0; kb < t.kb1; ++kb) {
                    const int seg = (kb - t.kb0) / kSumBlocks;
                    const bool last = kb + 1 == t.kb1 || ((kb + 1 - t.kb0) % kSumBlocks == 0 &&
                                                          (!planned || sh.ends[tiles & 1][seg]));
                    const unsigned buf = WIDE ? 0 : sums & 1, round = WIDE ? sums : sums >> 1;
                    if (!(ok = wait_for(sh, &sh.full[slot], par))) break;
                    tc_fence_after_sync();
                    const unsigned a = tmem + 256 + slot * kWCols;
                    const uint64_t b = desc + (uint64_t)(slot * (g.stage >> 4));
#pragma unroll
                    for (int h = 0; h < NH; ++h) {
                        if (first) {
                            if (!(ok = wait_for(sh, &sh.tempty[buf + h], (round & 1) ^ 1))) break;
                            tc_fence_after_sync();
                        }
                        const unsigned d = tmem + (buf + h) * 128;
                        const uint64_t bh = b + h * (2 * rows_x * 8);
                        const unsigned half_terms = (h ? g.wide[1] / CG : rows_x) * 8;
#pragma unroll
                        for (int s = 0; s < 8; ++s)
                            mma_tmem<CG>(d, a + s * 8, bh + s / 4 * half_terms + s % 4 * 2, g.idesc[h], !first || s > 0);
                        if (last && h + 1 < NH) commit<CG>(&sh.tfull[buf + h]);
                    }
                    if (!ok) break;
                    commit<CG>(&sh.empty[slot]);
                    if (last) {
                        commit<CG>(&sh.tfull[buf + NH - 1]);
                        ++sums;
                    }
                    first = last;
                    if (++slot == g.S) {
                        slot = 0;
                        par ^= 1;
                    }
                }
                if (planned) arrive(&sh.plan_empty[tiles & 1]);
            }
            // nothing in flight when the tensor memory is freed
            commit_here<CG>(&sh.done);
            mbar_wait_bounded(&sh.done, 0, kPolls);
        }
        __syncwarp();
    } else if (warp == 2) {
        // ----------------------------------------------------------- TMA of W
        // (no wait for the kernel before, unless it made W: the weights are the caller's, complete
        // before the first kernel of this call)
        if (elect_one()) {
            if (g.w_late) grid_dep_sync();
            int slot = 0;
            unsigned par = 0, issued = 0;
            bool ok = true;
            for (int u = first_unit; u < g.units && ok; u += step) {
                const Int8Tile t = int8_tile(g, u, share);
                const int m0 = (t.mt * CG + (int)rank) * 128;
                for (int kb = t.kb0; kb < t.kb1; ++kb) {
                    if (!(ok = wait_for(sh, &sh.raw_empty[slot], par ^ 1))) break;
                    arrive_expect(&sh.raw_full[slot], kRawBytes);
                    tma_load_2d(raw0 + slot * kRawBytes, &g.map_w, kb * kTerms, m0, &sh.raw_full[slot]);
                    ++issued;
                    if (++slot == g.R) {
                        slot = 0;
                        par ^= 1;
                    }
                }
            }
            for (unsigned i = issued > (unsigned)g.R ? issued - g.R : 0; i < issued; ++i)
                mbar_wait_bounded(&sh.raw_full[i % g.R], i / g.R & 1, kPolls);
        }
        __syncwarp();
    } else if (WIDE && warp == 3) {
        // ------------------------------------------------ where sums are drained
        // A sum goes on while it is sure to stay exact: any code of W is at most 128, so while 128 times
        // the magnitudes of x's codes in it, of the tile's row that has most in a segment, stay within
        // 2^24.
        if (g.sums) {
            grid_dep_sync();
            unsigned tiles = 0;
            for (int u = first_unit; u < g.units; u += step, ++tiles) {
                const Int8Tile t = int8_tile(g, u, share);
                if (!warp_wait_for(sh, &sh.plan_empty[tiles & 1], (tiles >> 1 & 1) ^ 1)) break;
                int used = 0;
                for (int seg = 0; seg < g.segs; ++seg) {
                    int most = 0;
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        const int c = lane + 32 * i, n = t.nt * g.bn + c;
                        if (c < g.bn && n < g.n) most = max(most, g.sums[(long long)n * g.segs + seg]);
                    }
                    most = __reduce_max_sync(0xffffffffu, most);
                    const bool full = used + most > (1 << 24) / 128;  // (the one before is the last)
                    if (seg && lane == 0) sh.ends[tiles & 1][seg - 1] = full;
                    used = full ? most : used + most;
                }
                __syncwarp();
                if (lane == 0) arrive(&sh.plan_full[tiles & 1]);
            }
        }
        __syncwarp();
    } else if (warp >= 4 && warp < 12) {
        // ---------------------------------------------------- drain, epilogue
        set_registers<WIDE ? 192 : 144, true>();
        const int quarter = warp & 3, half = (warp - 4) >> 2;
        const unsigned tl = tmem + ((unsigned)(quarter * 32) << 16);
        grid_dep_sync();
        const GemmEpi &e = g.e;
        constexpr int CH = WIDE ? 8 : 4;  // chunks of 16 columns of a warp at most
        // this warp's chunk i: WIDE: of its accumulator; else every other one
        const int chunks = WIDE ? g.wide[half] / 16 : (g.bn / 16 - half + 1) / 2;
        [[maybe_unused]] const int before = half ? wide0 : 0;  // (WIDE) columns of the tile before this warp's
        auto chunk_at = [&](int i) { return WIDE ? before / 16 + i : 2 * i + half; };
        unsigned sums = 0, tiles = 0;
        bool ok = true, large = false;  // large: a scale of the tile's columns (kLargeScale)
        float acc[CH][16];
        float *const scales = column_scales[warp - 4];
        // (WIDE) this warp's part of the shared memory that results pass through
        [[maybe_unused]] unsigned char *const mine = smem + g.S * g.stage + g.R * kRawBytes + (warp - 4) * kStagedBytes;
        [[maybe_unused]] const bool f32 = e.out_type == GEMM_T_F32, lead = elect_one();
        [[maybe_unused]] uint64_t *const there = &sh.residual[warp - 4];
        [[maybe_unused]] unsigned loads = 0;  // of the residual, so far
        // the residual of chunks c0 to c1 - 1, when what was stored from there has been read
        [[maybe_unused]] auto load_residual = [&](int x, int y, int c0, int c1) {
            if (lead) {
                const unsigned bytes = f32 ? 2048 : 1024;
                tma_stores_read();
                arrive_expect(there, (c1 - c0) * bytes);
                for (int c = c0; c < c1; ++c)
                    tma_load_2d(smem_addr(mine) + (c - c0) * bytes, &g.map_add, x, y + c * 16, there);
            }
            ++loads;
        };
        auto release = [&](unsigned buf) {
            tc_fence_before_sync();
            __syncwarp();
            if (lane == 0) {
                if constexpr (CG == 1) arrive(&sh.tempty[buf]);
                else arrive_leader(&sh.tempty[buf]);
            }
        };
        for (int u = first_unit; u < g.units; u += step) {
            const Int8Tile t = int8_tile(g, u, share);
            const int m = (t.mt * CG + (int)rank) * 128 + quarter * 32 + lane, n0 = t.nt * g.bn;
            // the scales of its columns
            __syncwarp();  // (the tile before has been read)
            large = false;
#pragma unroll
            for (int i = lane; i < 128; i += 32) {
                const int n = n0 + (WIDE ? before : 0) + i;
                const float s = n < g.n ? g.xscale[n] : 0.f;
                scales[i] = s;
                large |= !(fabsf(s) < kLargeScale);
            }
            large = __any_sync(0xffffffffu, large);
            __syncwarp();
            float alpha = m < g.m ? g.wscale[m] : 0.f, bias = e.bias && m < g.m ? e.bias[m] : 0.f;
            // the residual, on its way while the products run
            const int mw = m - lane, nw = n0 + before;
            if (WIDE && g.staged && e.add) load_residual(mw, nw, 0, f32 ? 4 : chunks);
            const bool planned = WIDE && g.sums;
            if (planned && !(ok = warp_wait_for(sh, &sh.plan_full[tiles & 1], tiles >> 1 & 1))) break;
            bool first = true, whole = false;  // whole: acc holds integers
            auto to_whole = [&] {
#pragma unroll
                for (int c = 0; c < CH; ++c)
#pragma unroll
                    for (int i = 0; i < 16; ++i) acc[c][i] = __int_as_float((int)acc[c][i]);
                whole = true;
            };
            for (int k0 = t.kb0; k0 < t.kb1; k0 += kSumBlocks) {
                const int seg = (k0 - t.kb0) / kSumBlocks;
                if (planned && k0 + kSumBlocks < t.kb1 && !(sh.ends[tiles & 1][seg])) continue;
                const unsigned buf = WIDE ? half : sums & 1;
                if (!(ok = warp_wait_for(sh, &sh.tfull[buf], (WIDE ? sums : sums >> 1) & 1))) break;
                ++sums;
                tc_fence_after_sync();
                const unsigned from = tl + buf * 128;
                if (!first && !whole) to_whole();  // (from the second on they are added as integers)
                if (WIDE && first) {
#pragma unroll
                    for (int c = 0; c < CH; c += 2) tmem_ld32_nowait(from + c * 16, acc[c], acc[c + 1]);
                    asm volatile("tcgen05.wait::ld.sync.aligned;\n" ::: "memory");
#pragma unroll
                    for (int c = 0; c < CH; ++c)
#pragma unroll
                        for (int i = 0; i < 16; ++i) asm volatile("" : "+f"(acc[c][i]));  // (not used before)
                } else {
#pragma unroll
                    for (int c = 0; c < CH; ++c) {
                        if (c < chunks) {
                            float v[16];
                            tmem_ld16(from + (WIDE ? c : 2 * c + half) * 16, v);
#pragma unroll
                            for (int i = 0; i < 16; ++i)
                                acc[c][i] = first ? v[i] : __int_as_float(__float_as_int(acc[c][i]) + (int)v[i]);
                        }
                    }
                }
                first = false;
                release(buf);
            }
            if (!ok) break;
            if (planned && lane == 0) arrive(&sh.plan_empty[tiles & 1]);
            ++tiles;
            if (g.cl > 1) {
                if (!whole) to_whole();  // (the shares' sums meet as integers)
            } else if (whole) {
#pragma unroll
                for (int c = 0; c < CH; ++c)
#pragma unroll
                    for (int i = 0; i < 16; ++i) acc[c][i] = (float)__float_as_int(acc[c][i]);
            }
            if (large && g.cl == 1) {
#pragma unroll 1
                for (int c = 0; c < CH; ++c) {
                    scaled16_large(acc[0], scales + (WIDE ? c : chunk_at(c)) * 16, alpha, bias);
#pragma unroll
                    for (int i = 0; i < 16; ++i) {
                        const float t = acc[0][i];
#pragma unroll
                        for (int k = 0; k + 1 < CH; ++k) acc[k][i] = acc[k + 1][i];
                        acc[CH - 1][i] = t;
                    }
                }
                __syncwarp();
                for (int i = lane; i < 128; i += 32) scales[i] = 1.f;
                alpha = 1.f, bias = 0.f;
                __syncwarp();
            }
            // (Four chunks at a time, two by two; the sums move through their registers: all eight unrolled, the
            // epilogue's instructions would come eight times, and each move counts too.  4096 x 1024 -> 8192 in fp32
            // with GELU 90.7 us, with four copies 93.8, with one 95.8.)
            if (WIDE && g.staged) {
                const auto rounds = [&](auto *at) {  // of four chunks
                    constexpr unsigned kBytes = sizeof(*at) * 512;  // of one
#pragma unroll 1
                    for (int i = 0; i < 2; ++i) {
                        if (e.add && (i == 0 || f32)) {
                            if (!(ok = warp_wait_for(sh, there, (loads - 1) & 1))) return;
                        } else if (i == 0 || f32) {
                            if (lead) tma_stores_read();
                            __syncwarp();
                        }
#pragma unroll 1
                        for (int k = 0; k < 4; k += 2) {
#pragma unroll
                            for (int q = 0; q < 2; ++q)
                                if (4 * i + k + q < chunks)
                                    staged16(acc[q], scales + (4 * i + k + q) * 16, alpha, bias, e.act, e.add,
                                             at + (k + q) * 512);
#pragma unroll
                            for (int q = 0; q < 2; ++q)
#pragma unroll
                                for (int j = 0; j < 16; ++j) acc[q][j] = acc[q + 2][j];
                        }
                        fence_async_smem();
                        __syncwarp();
                        if (lead && mw < g.m)
                            for (int c = 4 * i; c < min(4 * i + 4, chunks) && nw + c * 16 < g.n; ++c)
                                tma_store(&g.map_out, mw, nw + c * 16, smem_addr(mine) + (f32 ? c & 3 : c) * kBytes);
                        if (lead) asm volatile("cp.async.bulk.commit_group;\n" ::: "memory");
                        if (i == 0) {
                            if (!f32) at += 2048;
                            else if (e.add) load_residual(mw, nw, 4, chunks);
#pragma unroll
                            for (int k = 0; k + 4 < CH; ++k)
#pragma unroll
                                for (int j = 0; j < 16; ++j) acc[k][j] = acc[k + 4][j];
                        }
                    }
                };
                if (f32) rounds(reinterpret_cast<float *>(mine) + lane);
                else rounds(reinterpret_cast<unsigned short *>(mine) + lane);
                if (!ok) break;
                continue;
            }
            const float *const xs = scales - (WIDE ? before : 0);
            const auto chunk = [&](int c, float (&v)[16]) {
                const int n = n0 + c * 16, left = g.n - n;
                if (g.cl > 1) {  // to the cluster
                    const unsigned d = smem_addr(smem) + (unsigned)(c * 4 + quarter) * 2048 + lane * 16;
#pragma unroll
                    for (int j = 0; j < 4; ++j)
                        asm volatile("st.shared.v4.f32 [%0], {%1, %2, %3, %4};\n" ::"r"(d + j * 512), "f"(v[4 * j]),
                                     "f"(v[4 * j + 1]), "f"(v[4 * j + 2]), "f"(v[4 * j + 3])
                                     : "memory");
                } else if (left > 0) {
                    int8_finish(e, m, n, m < g.m ? min(left, 16) : 0, alpha, bias, xs + c * 16, v);
                }
            };
            if constexpr (WIDE) {
                // (one copy of the instructions: 3001 x 2047 -> 5003 in bf16 with GELU 67.9 us, with four 80.8)
#pragma unroll 1
                for (int i = 0; i < chunks; ++i) {
                    chunk(chunk_at(i), acc[0]);
#pragma unroll
                    for (int k = 0; k < 3; ++k)
#pragma unroll
                        for (int j = 0; j < 16; ++j) acc[k][j] = acc[k + 1][j];
                    if (i == 3)
#pragma unroll
                        for (int k = 0; k < 4; ++k)
#pragma unroll
                            for (int j = 0; j < 16; ++j) acc[k][j] = acc[k + 4][j];
                }
            } else {
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    if (i >= chunks) break;
                    chunk(chunk_at(i), acc[i]);
                }
            }
        }
        if (WIDE && g.staged) {  // nothing of its own under way when the CTA leaves
            if (lead) {
                if (loads) mbar_wait_bounded(there, (loads - 1) & 1, kPolls);
                tma_stores_read();
            }
            __syncwarp();
        }
        if constexpr (CG == 1) {
            if (g.cl > 1) {
                // The sums of a tile's shares meet in shared memory, where each CTA has left its own: each
                // adds up a part of the columns and does their epilogue.
                __syncwarp();
                cluster_sync_all();
                const Int8Tile t = int8_tile(g, first_unit, share);
                const int m = t.mt * 128 + quarter * 32 + lane;
                const float alpha = m < g.m ? g.wscale[m] : 0.f, bias = e.bias && m < g.m ? e.bias[m] : 0.f;
#pragma unroll 1
                for (int c = share + half * g.cl; c < g.bn / 16; c += 2 * g.cl) {
                    const int n = t.nt * g.bn + c * 16, left = g.n - n;
                    if (left <= 0) break;
                    const int count = m < g.m ? min(left, 16) : 0;
                    const unsigned mine = smem_addr(smem) + (unsigned)(c * 4 + quarter) * 2048 + lane * 16;
                    int sum[16] = {};
#pragma unroll 4
                    for (int s = 0; s < g.cl; ++s) {
                        unsigned at;
                        asm("mapa.shared::cluster.u32 %0, %1, %2;\n" : "=r"(at) : "r"(mine), "r"(s));
                        int o[16];
#pragma unroll
                        for (int i = 0; i < 4; ++i)
                            asm volatile("ld.shared::cluster.v4.s32 {%0, %1, %2, %3}, [%4];\n"
                                         : "=r"(o[4 * i]), "=r"(o[4 * i + 1]), "=r"(o[4 * i + 2]), "=r"(o[4 * i + 3])
                                         : "r"(at + i * 512)
                                         : "memory");
#pragma unroll
                        for (int i = 0; i < 16; ++i) sum[i] += o[i];
                    }
                    float v[16];
#pragma unroll
                    for (int i = 0; i < 16; ++i) v[i] = (float)sum[i];
                    if (large) int8_finish<true>(e, m, n, count, alpha, bias, scales + c * 16, v);
                    else int8_finish(e, m, n, count, alpha, bias, scales + c * 16, v);
                }
                __syncwarp();
                cluster_sync_all();  // (no CTA leaves while another reads from it)
            }
        }
    } else if (warp >= 12) {
        // -------------------------------------------------------------- widen
        set_registers<WIDE ? 80 : 72, false>();
        const int groups = WIDE || g.bn > 64 ? 1 : 2;  // each has every second block
        const int quarter = warp & 3, group = (warp - 12) >> 2;
        const unsigned a_dst = tmem + 256 + ((unsigned)(quarter * 32) << 16);
        const unsigned own = raw0 + (quarter * 32 + lane) * 128;  // (the pieces of a row permuted: 128-byte swizzle)
        int slot = group, rslot = group;
        unsigned par = 0, rpar = 0;
        auto next = [groups](int &at, unsigned &parity, int stages) {
            if ((at += groups) >= stages) at -= stages, parity ^= 1;
        };
        bool ok = true;
        int left = -group;  // blocks from this group's first on
        for (int u = first_unit; u < g.units && group < groups; u += step) {
            const Int8Tile t = int8_tile(g, u, share);
            left += t.kb1 - t.kb0;
        }
        unsigned w[32];
        auto read = [&] {
            if (!(ok = warp_wait_for(sh, &sh.raw_full[rslot], rpar))) return;
            const unsigned from = own + rslot * kRawBytes;
#pragma unroll
            for (int i = 0; i < 8; ++i)
                asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];\n"
                             : "=r"(w[4 * i]), "=r"(w[4 * i + 1]), "=r"(w[4 * i + 2]), "=r"(w[4 * i + 3])
                             : "r"(from + ((i ^ (lane & 7)) << 4)));
        };
        if (left > 0) read();
        for (; left > 0 && ok; left -= groups) {
            if (!(ok = warp_wait_for(sh, &sh.empty[slot], par ^ 1))) break;
            tc_fence_after_sync();
#pragma unroll
            for (int s = 0; s < 2; ++s) {
                unsigned v[32];
#pragma unroll
                for (int i = 0; i < 16; ++i) widen4(w[16 * s + i], v[2 * i], v[2 * i + 1]);
                tmem_st32(a_dst + slot * kWCols + s * 32, v);
            }
            __syncwarp();  // (all have read)
            if (lane == 0) arrive(&sh.raw_empty[rslot]);
            next(rslot, rpar, g.R);
            if (left > groups) read();  // (the next, while the stores are under way)
            asm volatile("tcgen05.wait::st.sync.aligned;\n" ::: "memory");
            tc_fence_before_sync();
            __syncwarp();
            if (lane == 0) {
                if constexpr (CG == 1) arrive(&sh.full[slot]);
                else arrive_first(&sh.full[slot]);
            }
            next(slot, par, g.S);
        }
    }
    if constexpr (CG == 1) {
        if (g.cl > 1 && (warp < 4 || warp >= 12)) {  // (as the epilogue's warps)
            __syncwarp();
            cluster_sync_all();
            cluster_sync_all();
        }
    }
    tc_fence_before_sync();
    __syncthreads();
    if constexpr (CG == 2) cluster_sync_all();
    tc_fence_after_sync();
    if (warp == 2) tmem_dealloc_cg<CG>(tmem);
}

template <int CG, bool WIDE>
qcnn_status launch_of(const Int8Args &g, int ctas, size_t smem, cudaStream_t st) {
    const auto k = int8_kernel<CG, WIDE>;
    const qcnn_status rc = allow_smem(reinterpret_cast<const void *>(k));
    if (rc != QCNN_OK) return rc;
    const int cluster = CG * g.cl;
    return launch_k(k, dim3(ctas), dim3(int8_threads(WIDE)), smem, st, dim3(cluster > 1 ? cluster : 0, 1, 1), g);
}

// Whether a matrix of two-byte elements can go in pairs of neighbours along m.
bool in_pairs(const void *p, int type, long long ld, int m) {
    return type != GEMM_T_F32 && p && reinterpret_cast<uintptr_t>(p) % 4 == 0 && ld % 2 == 0 && m % 2 == 0;
}

Int8Plan plan_int8_anew(int m, int n, int k, int sms) {
    Int8Plan best;
    const int kblocks = cdiv(k, kTerms);
    static const int tiles[8] = {16, 32, 64, 128, 160, 192, 224, 256};
    for (int bn : tiles) {
        const int cg = bn > 128 ? 2 : 1;
        if (bn > 16 && bn >= 2 * n) continue;
        const int mt = cdiv(m, 128 * cg), nt = cdiv(n, bn);
        const long long units = (long long)mt * nt;
        // Clocks of a block of 128 terms: MMAs; bytes of W at the memory's rate when all SMs read, with
        // x's at TMA's; shared memory, in and out; the widening.  (Pairs as measured: 1,200 with 160
        // columns, 1,350 with 224, 1,390 with 256; of a CTA with 128 950 to 1,200.)
        const double mma = 8 * (bn / 2 + 10.0), w = kRawBytes, x = bn / cg * 256.0;
        const double per = cg == 2 ? 1000.0 + 1.5 * bn
                                   : std::max({mma, w / 23.0, (w + x) / 50.0, 2.4 * (w + x) / 128.0, 500.0});
        const double tail = 4500.0 + bn * 16.0;
        for (int cl = 1; cl <= 8; cl *= 2) {
            if (cl > 1 && (cg > 1 || cl > kblocks)) break;
            const int kps = cdiv(kblocks, cl);
            if (cdiv(kblocks, kps) != cl) continue;
            const int slots = cl == 1 ? sms / cg
                                      : std::max(1, cluster_capacity(reinterpret_cast<const void *>(int8_kernel<1, false>),
                                                                     int8_threads(false), cl, kSmem));
            const double waves = (double)((units + slots - 1) / slots);
            const double meet = cl > 1 ? 2500.0 + bn * 10.0 : 0.0, more = cl > 1 ? tail + meet : 1000.0;
            const double score = waves * kps * per + tail + meet + (waves - 1) * more;
            if (best.bn && score >= best.score) continue;
            best.cg = cg;
            best.bn = bn;
            best.splits = cl;
            best.kb_per_split = kps;
            best.score = score;
        }
    }
    return best;
}

}  // namespace

Int8Plan plan_int8(int m, int n, int k) {
    static std::mutex mu;
    static std::map<std::array<int, 4>, Int8Plan> cache;
    const std::array<int, 4> key = {m, n, k, num_sms()};
    {
        std::lock_guard<std::mutex> g(mu);
        const auto it = cache.find(key);
        if (it != cache.end()) return it->second;
    }
    const Int8Plan p = plan_int8_anew(m, n, k, key[3]);
    std::lock_guard<std::mutex> g(mu);
    if (cache.size() >= 256) cache.clear();
    cache.emplace(key, p);
    return p;
}

qcnn_status launch_int8(const Int8Plan &plan, const Int8Problem &p, cudaStream_t st) {
    Int8Args g = {};
    const int cg = plan.cg, bn = plan.bn;
    const bool wide = bn > 128;
    // (of a pair's MMAs an accumulator has a multiple of 32 columns)
    const int wide0 = bn > 192 ? 128 : 96, cols = wide ? wide0 : bn;
    if (wide ? bn % 32 || bn < 160 || bn > 256 : bn % 16) return QCNN_ERR_UNSUPPORTED;
    qcnn_status rc = tensor_map(CU_TENSOR_MAP_DATA_TYPE_UINT8, p.W, p.k, p.m, p.ldw, kTerms, 128, true, &g.map_w);
    if (rc != QCNN_OK) return rc;
    rc = tensor_map(CU_TENSOR_MAP_DATA_TYPE_FLOAT16, p.x, p.k, p.n, p.ldx * 2, 64, cols / cg, true, &g.map_x);
    if (rc == QCNN_OK && wide)
        rc = tensor_map(CU_TENSOR_MAP_DATA_TYPE_FLOAT16, p.x, p.k, p.n, p.ldx * 2, 64, (bn - wide0) / cg, true, &g.map_x2);
    if (rc != QCNN_OK) return rc;
    g.wide[0] = wide0;
    g.wide[1] = bn - wide0;
    g.m = p.m;
    g.n = p.n;
    g.kblocks = cdiv(p.k, kTerms);
    g.m_tiles = cdiv(p.m, 128 * cg);
    g.n_tiles = cdiv(p.n, bn);
    g.kb_per_split = plan.splits > 1 ? plan.kb_per_split : g.kblocks;
    // (a share without terms would never have its sum)
    if ((plan.splits - 1) * (long long)g.kb_per_split >= g.kblocks || plan.splits * (long long)g.kb_per_split < g.kblocks)
        return QCNN_ERR_UNSUPPORTED;
    g.group = std::max(1, 16 / cg);
    const long long units = (long long)g.m_tiles * g.n_tiles;
    if (units > (1 << 27)) return QCNN_ERR_UNSUPPORTED;
    g.units = (int)units;
    g.bn = bn;
    g.cl = plan.splits;
    g.w_late = p.w_late;
    g.stage = (unsigned)(bn / cg * 2 * kTerms);
    const auto tma_can = [](const void *q, long long row_bytes) {
        return reinterpret_cast<uintptr_t>(q) % 16 == 0 && row_bytes % 16 == 0;
    };
    const long long size = p.e.out_type == GEMM_T_F32 ? 4 : 2;
    // (a store writes the 16 bytes that a row of the result ends in as a whole)
    g.staged = wide && p.m * size % 16 == 0 && tma_can(p.e.out, p.e.ldo * size) &&
               (!p.e.add || tma_can(p.e.add, p.e.lda * size));
    if (g.staged) {
        const CUtensorMapDataType type = size == 4 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT32 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16;
        rc = tensor_map(type, p.e.out, p.m, p.n, p.e.ldo * size, 32, 16, false, &g.map_out);
        if (rc == QCNN_OK && p.e.add)
            rc = tensor_map(type, p.e.add, p.m, p.n, p.e.lda * size, 32, 16, false, &g.map_add);
        if (rc != QCNN_OK) return rc;
    }
    const size_t staged = g.staged ? 8 * (size_t)kStagedBytes : 0;
    g.S = g.staged ? kStages - 1 : kStages;
    g.R = (int)std::min<size_t>(kRawStagesMax, (kSmem - 1024 - staged - g.S * (size_t)g.stage) / kRawBytes);
    // fp32 sums of fp16, 128 (256) rows x the columns of an accumulator
    for (int h = 0; h < 2; ++h)
        g.idesc[h] = (1u << 4) | (uint32_t)((h ? bn - wide0 : cols) >> 3) << 17 | (uint32_t)(128 * cg >> 4) << 24;
    g.sums = wide && p.segs > 1 ? p.sums : nullptr;
    g.segs = p.segs;
    g.xscale = p.xscale;
    g.wscale = p.wscale;
    g.e = p.e;
    g.e.beta = 1.f;
    g.e.pair = in_pairs(p.e.out, p.e.out_type, p.e.ldo, p.m) ? 1 : 0;
    const size_t stash = g.cl > 1 ? (size_t)bn * 512 : 0;
    const size_t smem = std::max({kSmemFloor, g.S * (size_t)g.stage + g.R * (size_t)kRawBytes + staged + 1024, stash + 1024});
    const int ctas = g.cl > 1 ? g.units * g.cl : std::min(g.units, num_sms() / cg) * cg;
    return wide ? launch_of<2, true>(g, ctas, smem, st) : launch_of<1, false>(g, ctas, smem, st);
}

}  // namespace qcnn
