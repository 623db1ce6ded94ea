// gemm_kernel.cuh -- the tensor-core product of gemm.cuh, instantiated by gemm_*.cu.
//
// Tile.  A CTA (CG 1) or a pair of CTAs (CG 2: tcgen05.mma.cta_group::2, each CTA with
// its own 128 rows of A and half of B's columns) takes 128 (256) rows of m, TMEM lanes,
// x bn columns of n.  m is the contiguous index of the result, so a warp's 32 lanes
// store 32 neighbours whatever the row stride and alignment, bias and column sums are a
// register per lane, and few rows n (a small batch) make a narrow tile, not an empty one.
//
// Operands come by TMA, 16 to 48 KB a stage, in the 128-byte swizzle (64-byte where the
// stage is 32 terms deep and k is contiguous), with k or the row index contiguous.
//
// Planes.  One: bf16 data, 64 terms a stage, one product, the whole sum in TMEM.  Two
// (16 to 17 bits): 32 terms a stage, three products, the small ones first.  Three (all 24
// bits of fp32): the six products of order <= 2; tcgen05.mma adds without rounding to
// nearest, so a stage's sum (32 terms, small products first) is drained to fp32
// registers and added there.  Against 64 bits that is closer than a chain of fp32
// multiply-adds (K = 4096: 1.4e-7 of the result).
//
// Roles (12 warps): 0 TMA, 1 MMA, 2 TMEM, 4-11 drain and epilogue: two warps per TMEM
// lane quarter, 16 columns in turn.  GEN adds warps 12-19, which take the place of TMA: they
// copy fp32 operands of any stride and alignment (cp.async), split them and store the
// planes.  That costs no pass over the operands, so a product bound by their bytes (few
// rows) reads them once.
#pragma once

#include "gemm.cuh"

namespace qcnn {
namespace {

constexpr int kMT = 128;          // rows of a CTA's tile
constexpr int kAccCols = 256;     // TMEM columns of an accumulator, of two
constexpr int kStagesMax = 8;
constexpr int kEpiWarps = 8;
constexpr int kGenThreads = 256;  // converters
constexpr int kRawSlots = 3;      // GEN: raw copies in flight, stages
constexpr unsigned kPolls = 1u << 22;

// An operand of a problem as the kernel sees it.
struct OpArgs {
    int mn;                        // row index contiguous
    unsigned bytes, group_bytes;   // of a stage; of 64 rows (mn)
    unsigned plane, kstep;         // descriptor units (16 bytes)
    unsigned long long desc;       // descriptor without the address
    const float *src;              // GEN
    long long ld;
    int rows, vec;                 // GEN: extent, 16-byte copies possible
};
struct ProblemArgs {
    CUtensorMap map_a, map_b;
    OpArgs a, b;
    unsigned idesc;
    int m, n, k, kblocks, m_tiles, n_tiles, splits, kb_per_split, group, units;
    GemmEpi e;
};
struct GemmArgs {
    ProblemArgs p[2];
    int count, units, bn, S;
    unsigned stage, b_off;  // bytes of a stage, of A's part of it
};

struct Shared {
    uint64_t full[kStagesMax], empty[kStagesMax], tfull[2], tempty[2], done;
    unsigned tmem;
    int give_up;
};

struct Tile {
    int q;               // problem
    int mt, nt, kb0, kb1, split;
};
// Unit u of a launch.  Neighbouring units are a patch of `group` row tiles, whose
// operands the L2 then holds.  SYM: row tiles from the diagonal on.
template <int KIND, int CG>
__device__ __forceinline__ Tile tile_of(const GemmArgs &g, int u) {
    Tile t;
    t.q = g.count > 1 && u >= g.p[0].units;
    const ProblemArgs &p = g.p[t.q];
    if (t.q) u -= g.p[0].units;
    if constexpr (KIND == GEMM_SYM) {
        const int per = g.bn / (kMT * CG);  // row tiles per column tile (bn a multiple)
        int nt = 0, first = 0;
        while (u >= p.m_tiles - first) {
            u -= p.m_tiles - first;
            ++nt;
            first = nt * per;
        }
        t.nt = nt;
        t.mt = first + u;
        t.split = 0;
    } else {
        const int tiles = p.m_tiles * p.n_tiles;
        t.split = u / tiles;
        u -= t.split * tiles;
        const int per = p.group * p.n_tiles, gr = u / per, m0 = gr * p.group;
        const int w = min(p.group, p.m_tiles - m0);
        u -= gr * per;
        t.nt = u / w;
        t.mt = m0 + u - t.nt * w;
    }
    t.kb0 = t.split * p.kb_per_split;
    t.kb1 = min(p.kblocks, t.kb0 + p.kb_per_split);
    return t;
}

__device__ __forceinline__ bool wait_one(Shared &s, uint64_t *bar, unsigned parity) {
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
__device__ __forceinline__ bool wait_warp(Shared &s, uint64_t *bar, unsigned parity) {
    return __all_sync(0xffffffffu, wait_one(s, bar, parity));
}
__device__ __forceinline__ void arrive(uint64_t *bar) {
    asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];\n" ::"r"(smem_addr(bar)) : "memory");
}
// The same on CTA 0 of the cluster.
__device__ __forceinline__ void arrive_leader(uint64_t *bar) {
    asm volatile(
        "{\n\t.reg .b32 a;\n\t"
        "mapa.shared::cluster.u32 a, %0, 0;\n\t"
        "mbarrier.arrive.release.cluster.shared::cluster.b64 _, [a];\n\t}\n" ::"r"(smem_addr(bar))
        : "memory");
}
__device__ __forceinline__ void arrive_expect(uint64_t *bar, unsigned bytes) {
    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;\n" ::"r"(smem_addr(bar)),
                 "r"(bytes)
                 : "memory");
}
// A box of a tensor map to shared memory, counted on the barrier (CG 2: on the one at
// the same place in the pair's first CTA).
template <int CG>
__device__ __forceinline__ void tma_load(unsigned dst, const CUtensorMap *map, int x, int y,
                                         uint64_t *bar) {
    if constexpr (CG == 1)
        asm volatile(
            "cp.async.bulk.tensor.3d.shared::cta.global.tile.mbarrier::complete_tx::bytes "
            "[%0], [%1, {%2, %3, %4}], [%5];\n" ::"r"(dst),
            "l"(map), "r"(x), "r"(y), "r"(0), "r"(smem_addr(bar))
            : "memory");
    else
        asm volatile(
            "cp.async.bulk.tensor.3d.cta_group::2.shared::cluster.global.tile.mbarrier::complete_tx::bytes "
            "[%0], [%1, {%2, %3, %4}], [%5];\n" ::"r"(dst),
            "l"(map), "r"(x), "r"(y), "r"(0), "r"(smem_addr(bar) & 0xFEFFFFFFu)
            : "memory");
}
template <int CG>
__device__ __forceinline__ void mma_ss(unsigned d, uint64_t a, uint64_t b, uint32_t idesc, bool acc) {
    if constexpr (CG == 1)
        asm volatile(
            "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
            "tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}\n" ::"r"(d),
            "l"(a), "l"(b), "r"(idesc), "r"((unsigned)acc)
            : "memory");
    else
        asm volatile(
            "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
            "tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n\t}\n" ::"r"(d),
            "l"(a), "l"(b), "r"(idesc), "r"((unsigned)acc)
            : "memory");
}
// One arrival, on the barrier of each CTA of the pair, when the MMAs so far are done.
template <int CG>
__device__ __forceinline__ void commit(uint64_t *bar) {
    if constexpr (CG == 1)
        mma_commit(bar);
    else
        asm volatile(
            "tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 "
            "[%0], %1;\n" ::"r"(smem_addr(bar)),
            "h"((unsigned short)3)
            : "memory");
}
// The same on this CTA's alone.
template <int CG>
__device__ __forceinline__ void commit_here(uint64_t *bar) {
    if constexpr (CG == 1)
        mma_commit(bar);
    else
        asm volatile(
            "tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.b64 [%0];\n" ::"r"(
                smem_addr(bar))
            : "memory");
}
template <int CG>
__device__ __forceinline__ void tmem_alloc_cg(unsigned *dst) {
    if constexpr (CG == 1) {
        tmem_alloc(dst, 512);
    } else {
        asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], 512;\n" ::"r"(
                         smem_addr(dst))
                     : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;\n" ::: "memory");
    }
}
template <int CG>
__device__ __forceinline__ void tmem_dealloc_cg(unsigned t) {
    if constexpr (CG == 1)
        tmem_dealloc(t, 512);
    else
        asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, 512;\n" ::"r"(t) : "memory");
}
__device__ __forceinline__ bool elect_one() {
    unsigned p;
    asm volatile(
        "{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}\n"
        : "=r"(p));
    return p != 0;
}
__device__ __forceinline__ void cluster_sync_all() {
    asm volatile("barrier.cluster.arrive.release.aligned;\n" ::: "memory");
    asm volatile("barrier.cluster.wait.acquire.aligned;\n" ::: "memory");
}
// 16 columns of this warp's lanes.
__device__ __forceinline__ void tmem_ld16(unsigned taddr, float (&v)[16]) {
    unsigned r[16];
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 "
        "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];\n\t"
        "tcgen05.wait::ld.sync.aligned;\n"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]),
          "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]),
          "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
        : "r"(taddr)
        : "memory");
#pragma unroll
    for (int i = 0; i < 16; ++i) v[i] = __uint_as_float(r[i]);
}

// ------------------------------------------------------------------ epilogue
// 16 columns of a lane to out[n0 + i][m] (m in range), row by row: the warp's lanes are
// neighbours.
__device__ __forceinline__ void store16(void *out, int type, long long ld, long long plane, int m, int n0,
                                        int n_end, const float (&v)[16]) {
    long long o = (long long)n0 * ld + m;
    if (type == GEMM_T_F32) {
        float *p = static_cast<float *>(out) + o;
#pragma unroll
        for (int i = 0; i < 16; ++i, p += ld)
            if (n0 + i < n_end) *p = v[i];
        return;
    }
    unsigned short *p = static_cast<unsigned short *>(out) + o;
#pragma unroll
    for (int i = 0; i < 16; i += 2, p += 2 * ld) {
        unsigned w[3];
        if (type == GEMM_T_BF16) w[0] = pack_bf16x2(v[i], v[i + 1]);
        else if (type == GEMM_T_PLANES2) planes2(v[i], v[i + 1], w[0], w[1]);
        else planes3(v[i], v[i + 1], w[0], w[1], w[2]);
        const int np = type == GEMM_T_BF16 ? 1 : type;
#pragma unroll
        for (int j = 0; j < 3; ++j) {
            if (j >= np) break;
            if (n0 + i < n_end) p[j * plane] = (unsigned short)w[j];
            if (n0 + i + 1 < n_end) p[j * plane + ld] = (unsigned short)(w[j] >> 16);
        }
    }
}

// OUT and SYM: sums v of lane m, columns n0 .. n0 + 15.
template <int KIND>
__device__ __forceinline__ void finish_out(const GemmEpi &e, int m, int m_end, int n0, int n_end,
                                           float alpha, float bias, float (&v)[16]) {
    if (m >= m_end) return;
#pragma unroll
    for (int i = 0; i < 16; ++i) v[i] = fmaf(alpha, v[i], bias);
    if (e.pre) store16(e.pre, e.out_type, e.ldp, 0, m, n0, n_end, v);
    if (e.act != QCNN_ACT_NONE) {
#pragma unroll
        for (int i = 0; i < 16; ++i) v[i] = act_apply(v[i], e.act);
    }
    if (e.add) {
        const long long o = (long long)n0 * e.lda + m;
        float r[16];
#pragma unroll
        for (int i = 0; i < 16; ++i)
            r[i] = n0 + i < n_end ? load_as(e.add, e.add_type, o + i * e.lda, e.add_plane) : 0.f;
#pragma unroll
        for (int i = 0; i < 16; ++i) v[i] = fmaf(e.beta, r[i], v[i]);
    }
    if constexpr (KIND == GEMM_OUT) {
        store16(e.out, e.out_type, e.ldo, e.out_plane, m, n0, n_end, v);
    } else {
        // one value for both places: this tile's where m >= n
        const int end = min(n_end, m + 1);
        if (n0 >= end) return;
        store16(e.out, e.out_type, e.ldo, e.out_plane, m, n0, end, v);
        unsigned short *p = static_cast<unsigned short *>(e.out) + (long long)m * e.ldo + n0;
#pragma unroll
        for (int h = 0; h < 16; h += 8) {  // (rows of planes: 16-byte multiples)
            unsigned w[3][4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if (e.out_type == GEMM_T_PLANES2) planes2(v[h + 2 * i], v[h + 2 * i + 1], w[0][i], w[1][i]);
                else planes3(v[h + 2 * i], v[h + 2 * i + 1], w[0][i], w[1][i], w[2][i]);
            }
#pragma unroll
            for (int j = 0; j < 3; ++j) {
                if (j >= e.out_type) break;
                unsigned short *d = p + j * e.out_plane + h;
                if (n0 + h + 8 <= end) {
                    *reinterpret_cast<uint4 *>(d) = make_uint4(w[j][0], w[j][1], w[j][2], w[j][3]);
                } else {
#pragma unroll
                    for (int i = 0; i < 8; ++i)
                        if (n0 + h + i < end) d[i] = (unsigned short)(w[j][i / 2] >> (i & 1) * 16);
                }
            }
        }
    }
}

constexpr float kLog2e = 1.4426950408889634f;

// Running maximum and sum of exp of a lane.  A maximum of -inf has no sum (and adds
// nothing: exp of -inf minus -inf is left out).
struct RunningSum {
    float top = -INFINITY, sum = 0.f;
};
__device__ __forceinline__ void running_join(RunningSum &a, float top, float sum) {
    const float t = fmaxf(a.top, top);
    if (t == -INFINITY) {
        a.sum += sum;  // (NaN stays NaN)
        return;
    }
    a.sum = a.sum * exp2f((a.top - t) * kLog2e) + sum * exp2f((top - t) * kLog2e);
    a.top = t;
}
__device__ __forceinline__ void stats16(const GemmEpi &e, RunningSum &s, int n0, int n_end, int target,
                                        float *target_logit, float (&v)[16]) {
    float top = -INFINITY;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        v[i] = n0 + i < n_end ? (e.bias ? v[i] + e.bias[n0 + i] : v[i]) : -INFINITY;
        top = fmaxf(top, v[i]);
    }
    if ((unsigned)(target - n0) < 16u) {
#pragma unroll
        for (int i = 0; i < 16; ++i)
            if (target == n0 + i) *target_logit = v[i];
    }
    top = fmaxf(top, s.top);
    if (top == -INFINITY) {
        // all -inf (nothing to add) or NaN (which fmaxf passes over)
#pragma unroll
        for (int i = 0; i < 16; ++i)
            if (v[i] != v[i]) s.sum = v[i];
        return;
    }
    const float shift = top * kLog2e;
    float a0 = 0.f, a1 = 0.f;
#pragma unroll
    for (int i = 0; i < 16; i += 2) {
        a0 += exp2f(fmaf(v[i], kLog2e, -shift));
        a1 += exp2f(fmaf(v[i + 1], kLog2e, -shift));
    }
    s.sum = (s.top == -INFINITY ? s.sum : s.sum * exp2f(fmaf(s.top, kLog2e, -shift))) + (a0 + a1);
    s.top = top;
}

// Gradient of a class (lane m) for 16 rows.
__device__ __forceinline__ void dlogits16(const GemmEpi &e, int m, int m_end, int n0, int n_end, float bias,
                                          float &col, float (&v)[16]) {
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        float d = 0.f;
        if (n0 + i < n_end) {
            const float4 r = e.rows[n0 + i];
            const int target = __float_as_int(r.z);
            const float p = exp2f((v[i] + bias - r.x) * kLog2e);
            // (a row without a class is zero, whatever its logits are)
            if (target >= 0) d = r.y * (target == e.class0 + m ? p - 1.f : p);
        }
        v[i] = d;
        col += d;
    }
    if (m < m_end) store16(e.out, e.out_type, e.ldo, e.out_plane, m, n0, n_end, v);
}

// ---------------------------------------------------------------------- GEN
// A thread's copies of a stage: 8 neighbouring elements of one row (32 bytes), items
// kGenThreads apart.  Rows of k: item = row * 4 + k / 8; rows of m: item = k * (rows / 8)
// + row / 8.
struct GenItem {
    unsigned dst;     // bytes into the operand's stage part, plane 0
    int row, k;       // first element
};
__device__ __forceinline__ GenItem gen_item(const OpArgs &o, int rows8, int it) {
    GenItem r;
    if (!o.mn) {
        const int row = it >> 2, c = it & 3;
        r.row = row;
        r.k = c * 8;
        r.dst = row * 64 + ((c ^ (row >> 1 & 3)) << 4);  // 64-byte swizzle
    } else {
        const int k = it / rows8, c = it - k * rows8;
        r.row = c * 8;
        r.k = k;
        r.dst = (c >> 3) * o.group_bytes + k * 128 + (((c & 7) ^ (k & 7)) << 4);  // 128-byte swizzle
    }
    return r;
}
__device__ __forceinline__ void cp_async16_part(unsigned dst, const void *src, unsigned bytes) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;\n" ::"r"(dst), "l"(src), "r"(bytes)
                 : "memory");
}
__device__ __forceinline__ void cp_async4_part(unsigned dst, const void *src, unsigned bytes) {
    asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;\n" ::"r"(dst), "l"(src), "r"(bytes)
                 : "memory");
}
// Elements i .. of the item to raw (its two halves 16 * kGenThreads bytes apart); what is
// outside the matrix is zero.
__device__ __forceinline__ void gen_copy(const OpArgs &o, int row, int k, int k_end, unsigned raw) {
    // along the contiguous index: first element, and how many of the eight exist
    const int first = o.mn ? row : k, line = o.mn ? k : row;
    const int have = (o.mn ? o.rows : k_end) - first;
    const bool in = line < (o.mn ? k_end : o.rows) && have > 0;
    const float *s = in ? o.src + (long long)line * o.ld + first : o.src;
    const int n = in ? min(have, 8) : 0;
    if (o.vec) {
        cp_async16_part(raw, n > 0 ? s : o.src, 4 * min(n, 4));
        cp_async16_part(raw + 16 * kGenThreads, n > 4 ? s + 4 : o.src, n > 4 ? 4 * (n - 4) : 0);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            cp_async4_part(raw + (i >> 2) * 16 * kGenThreads + (i & 3) * 4, i < n ? s + i : o.src, i < n ? 4 : 0);
    }
}

// ------------------------------------------------------------------- kernel
template <int P, int KIND, int CG, bool GEN>
__global__ void __launch_bounds__(GEN ? 640 : 384, 1) gemm_kernel(const __grid_constant__ GemmArgs g) {
    constexpr int BK = P == 1 ? 64 : 32, KS = BK / 16;
    constexpr bool DRAIN = P == 3;  // a stage's sum at a time
    extern __shared__ __align__(128) unsigned char smem_raw[];
    __shared__ Shared sh;
    unsigned char *const smem = smem_raw + (-smem_addr(smem_raw) & 1023u);  // (swizzle atoms)
    const int tid = threadIdx.x, lane = tid & 31;
    const int warp = __shfl_sync(0xffffffffu, tid >> 5, 0);
    unsigned rank = 0;
    if constexpr (CG == 2) asm("mov.u32 %0, %%cluster_ctarank;\n" : "=r"(rank));
    const int first_unit = (int)blockIdx.x / CG, step = (int)gridDim.x / CG;

    if (tid == 0) {
        for (int i = 0; i < g.S; ++i) {
            mbar_init(&sh.full[i], GEN ? kGenThreads : 1);
            mbar_init(&sh.empty[i], 1);
        }
        for (int i = 0; i < 2; ++i) {
            mbar_init(&sh.tfull[i], 1);
            mbar_init(&sh.tempty[i], kEpiWarps * CG);
        }
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
    grid_dep_sync();

    if (warp == 0) {
        if constexpr (!GEN) {
            // ----------------------------------------------------------- TMA
            if (elect_one()) {
                int slot = 0, issued = 0;
                unsigned par = 0;
                bool ok = true;
                for (int u = first_unit; u < g.units && ok; u += step) {
                    const Tile t = tile_of<KIND, CG>(g, u);
                    const ProblemArgs &p = g.p[t.q];
                    const int m0 = (t.mt * CG + (int)rank) * kMT;
                    const int bn = g.bn / CG, n0 = t.nt * g.bn + (int)rank * bn;
                    const unsigned bytes = (p.a.bytes + p.b.bytes) * CG;
                    for (int kb = t.kb0; kb < t.kb1; ++kb) {
                        if (!(ok = wait_one(sh, &sh.empty[slot], par ^ 1))) break;
                        uint64_t *const full = &sh.full[slot];
                        if (rank == 0) arrive_expect(full, bytes);
                        const unsigned a = smem_addr(smem) + slot * g.stage, b = a + g.b_off;
                        const int k = kb * BK;
                        if (p.a.mn) {
                            tma_load<CG>(a, &p.map_a, m0, k, full);
                            tma_load<CG>(a + p.a.group_bytes, &p.map_a, m0 + 64, k, full);
                        } else {
                            tma_load<CG>(a, &p.map_a, k, m0, full);
                        }
                        if (p.b.mn) {
                            for (int i = 0; i < bn; i += 64)
                                tma_load<CG>(b + (i >> 6) * p.b.group_bytes, &p.map_b, n0 + i, k, full);
                        } else {
                            tma_load<CG>(b, &p.map_b, k, n0, full);
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
                    for (int i = max(0, issued - g.S); i < issued; ++i)
                        mbar_wait_bounded(rank == 0 ? &sh.full[i % g.S] : &sh.empty[i % g.S],
                                          (unsigned)(i / g.S) & 1, kPolls);
            }
        }
        __syncwarp();
    } else if (warp == 1) {
        // --------------------------------------------------------------- MMA
        if (rank == 0 && elect_one()) {
            int slot = 0;
            unsigned par = 0, use = 0;  // use: accumulators so far
            bool ok = true;
            const uint64_t base = (uint64_t)((smem_addr(smem) >> 4) & 0x3FFFu);
            for (int u = first_unit; u < g.units && ok; u += step) {
                const Tile t = tile_of<KIND, CG>(g, u);
                const ProblemArgs &p = g.p[t.q];
                const uint64_t da = p.a.desc + base, db = p.b.desc + base + (g.b_off >> 4);
                const unsigned pa = p.a.plane, pb = p.b.plane, ka = p.a.kstep, kb_ = p.b.kstep;
                const uint32_t idesc = p.idesc;
                for (int kb = t.kb0; kb < t.kb1; ++kb) {
                    const bool fresh = DRAIN || kb == t.kb0;
                    if (fresh) {
                        if (!(ok = wait_one(sh, &sh.tempty[use & 1], (use >> 1 & 1) ^ 1))) break;
                    }
                    if (!(ok = wait_one(sh, &sh.full[slot], par))) break;
                    tc_fence_after_sync();
                    const unsigned d = tmem + (use & 1) * kAccCols;
                    const uint64_t a = da + slot * (g.stage >> 4), b = db + slot * (g.stage >> 4);
                    bool acc = !fresh;
                    auto product = [&](int i, int j) {
#pragma unroll
                        for (int s = 0; s < KS; ++s) {
                            mma_ss<CG>(d, a + i * pa + s * ka, b + j * pb + s * kb_, idesc, acc);
                            acc = true;
                        }
                    };
                    if constexpr (P == 3) {
                        product(2, 0);
                        product(1, 1);
                        product(0, 2);
                    }
                    if constexpr (P >= 2) {
                        product(1, 0);
                        product(0, 1);
                    }
                    product(0, 0);
                    commit<CG>(&sh.empty[slot]);
                    if (DRAIN || kb + 1 == t.kb1) {
                        commit<CG>(&sh.tfull[use & 1]);
                        ++use;
                    }
                    if (++slot == g.S) {
                        slot = 0;
                        par ^= 1;
                    }
                }
            }
            // nothing in flight when the tensor memory is freed
            commit_here<CG>(&sh.done);
            mbar_wait_bounded(&sh.done, 0, kPolls);
        }
        __syncwarp();
    } else if (warp >= 4 && warp < 4 + kEpiWarps) {
        // ---------------------------------------------------- drain, epilogue
        const int quarter = warp & 3, half = (warp - 4) >> 2;
        const unsigned tl = tmem + ((unsigned)(quarter * 32) << 16);
        const int chunks = g.bn / 16;  // this warp's: half, half + 2, ...
        unsigned use = 0;
        bool ok = true;
        auto release = [&](unsigned buf) {
            tc_fence_before_sync();
            __syncwarp();
            if (lane == 0) {
                if constexpr (CG == 1) arrive(&sh.tempty[buf]);
                else arrive_leader(&sh.tempty[buf]);
            }
        };
        for (int u = first_unit; u < g.units; u += step) {
            const Tile t = tile_of<KIND, CG>(g, u);
            const ProblemArgs &p = g.p[t.q];
            const GemmEpi &e = p.e;
            const int m = (t.mt * CG + (int)rank) * kMT + quarter * 32 + lane, n0 = t.nt * g.bn;
            float bias = 0.f;
            RunningSum run;
            int target = -1;
            float col = 0.f;
            [[maybe_unused]] const float alpha = KIND == GEMM_OUT && e.alpha_ptr ? *e.alpha_ptr : e.alpha;
            if constexpr (KIND == GEMM_STATS) {
                if (m < p.m) {
                    const long long c = e.targets[m];
                    target = c >= 0 && c < p.n ? (int)c : -1;
                }
            } else {
                if (e.bias && m < p.m && !e.partial) bias = e.bias[m];
            }
            auto chunk = [&](int n, float (&v)[16]) {
                if constexpr (KIND == GEMM_STATS) {
                    stats16(e, run, n, p.n, target, e.target_logit + m, v);
                } else if constexpr (KIND == GEMM_DLOGITS) {
                    dlogits16(e, m, p.m, n, p.n, bias, col, v);
                } else {
                    if (KIND == GEMM_OUT && e.partial) {
                        if (m < p.m)
                            store16(e.partial + (long long)t.split * p.n * p.m, GEMM_T_F32, p.m, 0, m, n,
                                    p.n, v);
                    } else {
                        finish_out<KIND>(e, m, p.m, n, p.n, alpha, bias, v);
                    }
                }
            };
            if constexpr (DRAIN) {
                constexpr int CH = GEN ? 4 : 8;  // chunks of a warp at most
                float acc[CH][16];
#pragma unroll
                for (int c = 0; c < CH; ++c)
#pragma unroll
                    for (int i = 0; i < 16; ++i) acc[c][i] = 0.f;
                for (int kb = t.kb0; kb < t.kb1; ++kb, ++use) {
                    const unsigned buf = use & 1;
                    if (!(ok = wait_warp(sh, &sh.tfull[buf], use >> 1 & 1))) break;
                    tc_fence_after_sync();
#pragma unroll
                    for (int c = 0; c < CH; ++c) {
                        if (2 * c + half < chunks) {
                            float v[16];
                            tmem_ld16(tl + buf * kAccCols + (2 * c + half) * 16, v);
#pragma unroll
                            for (int i = 0; i < 16; i += 2)
                                add2(acc[c][i], acc[c][i + 1], v[i], v[i + 1]);
                        }
                    }
                    release(buf);
                }
                if (!ok) break;
#pragma unroll
                for (int c = 0; c < CH; ++c)
                    if (2 * c + half < chunks) chunk(n0 + (2 * c + half) * 16, acc[c]);
            } else {
                const unsigned buf = use & 1;
                if (!(ok = wait_warp(sh, &sh.tfull[buf], use >> 1 & 1))) break;
                tc_fence_after_sync();
                for (int c = half; c < chunks; c += 2) {
                    float v[16];
                    tmem_ld16(tl + buf * kAccCols + c * 16, v);
                    chunk(n0 + c * 16, v);
                }
                release(buf);
                ++use;
            }
            if constexpr (KIND == GEMM_STATS) {
                if (m < p.m) e.stats[(long long)(t.nt * 2 + half) * p.m + m] = make_float2(run.top, run.sum);
            }
            if constexpr (KIND == GEMM_DLOGITS) {
                if (m < p.m) e.col_part[(long long)(t.nt * 2 + half) * e.ld_col + m] = col;
            }
        }
    } else if (GEN && warp >= 12) {
        // ------------------------------------------ copy, split, store planes
        const int gt = tid - 384;
        unsigned char *const raw0 = smem + (size_t)g.S * g.stage + gt * 16;
        const ProblemArgs &p = g.p[0];
        const int a_items = kMT * 4, items = a_items + g.bn * 4;  // 32 terms of 128 + bn rows
        constexpr int IT = 4;                                      // a thread's at most (bn <= 128)
        const unsigned raw_slot = (unsigned)((items + kGenThreads - 1) / kGenThreads) * 32 * kGenThreads;
        // the stages of this CTA, in order: raw copies run kRawSlots - 1 ahead
        int cu = first_unit, ckb = 0;  // next to copy: unit and block
        Tile ct = {};
        bool cok = cu < g.units;
        if (cok) {
            ct = tile_of<KIND, CG>(g, cu);
            ckb = ct.kb0;
        }
        int cslot = 0;
        auto copy_next = [&]() {
            if (cok) {
                const int m0 = ct.mt * kMT, n0 = ct.nt * g.bn, k0 = ckb * BK;
                const unsigned raw = smem_addr(raw0) + cslot * raw_slot;
#pragma unroll
                for (int j = 0; j < IT; ++j) {
                    const int it = gt + j * kGenThreads;
                    if (it < items) {
                        const bool is_a = it < a_items;
                        const OpArgs &o = is_a ? p.a : p.b;
                        const GenItem x = gen_item(o, (is_a ? kMT : g.bn) / 8, is_a ? it : it - a_items);
                        gen_copy(o, (is_a ? m0 : n0) + x.row, k0 + x.k, p.k, raw + j * 32 * kGenThreads);
                    }
                }
                if (++ckb == ct.kb1) {
                    cu += step;
                    if ((cok = cu < g.units)) {
                        ct = tile_of<KIND, CG>(g, cu);
                        ckb = ct.kb0;
                    }
                }
                if (++cslot == kRawSlots) cslot = 0;
            }
            cp_async_commit();
        };
        for (int i = 0; i < kRawSlots - 1; ++i) copy_next();
        int slot = 0, rslot = 0;
        unsigned par = 0;
        bool ok = true;
        for (int u = first_unit; u < g.units && ok; u += step) {
            const Tile t = tile_of<KIND, CG>(g, u);
            for (int kb = t.kb0; kb < t.kb1; ++kb) {
                copy_next();
                cp_async_wait<kRawSlots - 1>();
                if (!(ok = wait_warp(sh, &sh.empty[slot], par ^ 1))) break;
                const unsigned char *raw = raw0 + rslot * raw_slot;
                unsigned char *const st = smem + (size_t)slot * g.stage;
#pragma unroll
                for (int j = 0; j < IT; ++j) {
                    const int it = gt + j * kGenThreads;
                    if (it < items) {
                        const bool is_a = it < a_items;
                        const OpArgs &o = is_a ? p.a : p.b;
                        const GenItem x = gen_item(o, (is_a ? kMT : g.bn) / 8, is_a ? it : it - a_items);
                        const float4 f = *reinterpret_cast<const float4 *>(raw + j * 32 * kGenThreads);
                        const float4 h = *reinterpret_cast<const float4 *>(raw + j * 32 * kGenThreads +
                                                                          16 * kGenThreads);
                        uint4 w0, w1, w2;
                        planes3(f.x, f.y, w0.x, w1.x, w2.x);
                        planes3(f.z, f.w, w0.y, w1.y, w2.y);
                        planes3(h.x, h.y, w0.z, w1.z, w2.z);
                        planes3(h.z, h.w, w0.w, w1.w, w2.w);
                        unsigned char *d = st + (is_a ? 0u : g.b_off) + x.dst;
                        *reinterpret_cast<uint4 *>(d) = w0;
                        *reinterpret_cast<uint4 *>(d + o.plane * 16) = w1;
                        *reinterpret_cast<uint4 *>(d + o.plane * 32) = w2;
                    }
                }
                fence_async_smem();
                arrive(&sh.full[slot]);
                if (++slot == g.S) {
                    slot = 0;
                    par ^= 1;
                }
                if (++rslot == kRawSlots) rslot = 0;
            }
        }
        cp_async_wait<0>();
    }
    tc_fence_before_sync();
    __syncthreads();
    if constexpr (CG == 2) cluster_sync_all();
    tc_fence_after_sync();
    if (warp == 2) tmem_dealloc_cg<CG>(tmem);
}

}  // namespace

// The kernel of a plan, by translation unit.
template <int P, int KIND, int CG, bool GEN>
struct GemmKernel {
    static qcnn_status launch(const void *args, int ctas, size_t smem, cudaStream_t st) {
        const GemmArgs &g = *static_cast<const GemmArgs *>(args);
        const auto k = gemm_kernel<P, KIND, CG, GEN>;
        qcnn_status rc = allow_smem(reinterpret_cast<const void *>(k));
        if (rc != QCNN_OK) return rc;
        return launch_k(k, dim3(ctas), dim3(GEN ? 640 : 384), smem, st, CG == 2 ? dim3(2, 1, 1) : dim3(0, 0, 0), g);
    }
};

}  // namespace qcnn
