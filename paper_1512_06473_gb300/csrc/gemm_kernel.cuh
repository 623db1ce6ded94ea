// gemm_kernel.cuh -- the tensor-core product of gemm.cuh, instantiated by gemm_*.cu.
//
// Tile.  A CTA (CG 1) or a pair of CTAs (CG 2: tcgen05.mma.cta_group::2, each CTA with
// its own 128 rows of A and half of B's columns) takes 128 (256) rows of m, TMEM lanes,
// x bn columns of n.  m is the contiguous index of the result, so a warp's 32 lanes
// store 32 neighbours whatever the row stride and alignment, bias and column sums are a
// register per lane, and few rows n (a small batch) make a narrow tile, not an empty one.
//
// Operands come by TMA, with k or the row index contiguous, in the 128-byte swizzle: a
// stage is 64 terms of one plane of A and B, 32 to 48 KB.  (Rows of 64 bytes, 32 terms of
// all planes, came at 40 bytes per clock and SM; rows of 128 come at 68.)
//
// Planes.  One: bf16 data, one product, the whole sum in TMEM.  Two (16 to 17 bits): three
// products, the small ones first.  Three (all 24 bits of fp32): the six products of order
// <= 2; tcgen05.mma adds without rounding to nearest, so the sum of 64 terms (GEN: 32;
// small products first) is drained to fp32 registers and added there.  A plane's stage is
// free again after its last product.  Against 64 bits that is closer than a chain of fp32
// multiply-adds (K = 4096: 1.4e-7 of the result).
//
// Roles (12 warps): 0 TMA, 1 (three planes: and 3) MMA, 2 TMEM, 4-11 drain and epilogue: two
// warps per TMEM lane quarter, 16 columns in turn.
//
// GEN (20 warps): A is fp32 of any stride and alignment (a layer's weights), split on its way,
// so that a product bound by A's bytes (few rows n) reads them once and writes no planes.  It
// comes to shared memory by TMA (warp 2), or where its base is off the 16-byte alignment by
// cp.async of the warps that split it, 12-19; these store the planes to TMEM as the MMAs' A
// operand.  Shared memory then carries per stage of 32 terms and 128 columns 32 KB for the
// copies, 24 KB of B's planes and 48 KB that the twelve MMAs read, 832 clocks of its bandwidth
// to the 888 of the MMAs.  (With A's planes in shared memory and B split by the same warps it
// was 1664, and the kernel took 3,500: 115 us for 128 rows of 9216 -> 4096.)
//
// Measured, of 6.67 TB/s copied and 1,946 (a long run: 1,742) TFLOP/s of bf16: 4096 x 4096 ->
// 8192 in bf16 with GELU and residual 173 us, 1,590 TFLOP/s (tensor cores; at the power limit 192);
// GEN, 8192 -> 19456: 12 rows 114 us, 5.6 TB/s (the memory and the split), 128 rows 164 us, 1,490
// TFLOP/s (six products; tensor cores); 128 x 9216 -> 4096 56 us, of which 46 are the product at
// that rate on the 128 CTAs that 32 tiles make.
#pragma once

#include "gemm.cuh"

#include <type_traits>

namespace qcnn {
namespace {

constexpr int kMT = 128;          // rows of a CTA's tile
constexpr int kAccCols = 256;     // TMEM columns of an accumulator, of two (GEN: 128)
constexpr int kStagesMax = 8;
constexpr int kEpiWarps = 8;
constexpr int kGenWarps = 4;      // that split a block's A
constexpr int kGenThreads = 640;
constexpr int kRawSlots = 3;      // GEN: blocks of raw copies, 4 KB per warp each
constexpr int kRawMax = 10;       // the same by TMA, at most
// A shifted block: [4][32 rows][36 words], or rows contiguous [4][8 terms][132 words].
constexpr unsigned kShiftedPart = 32 * 36 * 4, kShiftedPartMn = 8 * 132 * 4;
constexpr int kGenCols = 48;      // TMEM columns of a stage's A: 3 planes x 32 terms
constexpr int kGenStages = 4;     // (at most (512 - 2 * 128) / 48)
constexpr unsigned kPolls = 1u << 22;

// An operand of a problem as the kernel sees it.
struct OpArgs {
    int mn;                        // row index contiguous
    unsigned bytes, group_bytes;   // of a stage; of 64 rows (mn)
    unsigned plane, kstep;         // descriptor units (16 bytes): GEN's planes; 16 terms
    unsigned long long desc;       // descriptor without the address
    const float *src;              // GEN
    long long ld;
    int way;                       // GEN: RawWay
};
// How GEN's fp32 comes: element by element; in boxes; or, where only the base is on 16 bytes, in
// a box for every fourth row (their distance is a multiple of 16 bytes again), four words wider
// and read from the word where the row begins.
enum RawWay { RAW_WORDS = 0, RAW_BOXES = 1, RAW_SHIFTED = 2 };
struct ProblemArgs {
    CUtensorMap map_a, map_b;
    OpArgs a, b;
    unsigned idesc;
    int m, n, k, kblocks, m_tiles, n_tiles, kb_per_split, group, units;
    GemmEpi e;
};
struct GemmArgs {
    ProblemArgs p[2];
    int count, units, bn, S;
    int raw;                // GEN: stages of raw copies, of raw_bytes each
    unsigned raw_bytes;
    int shift[4];           // GEN: words that rows r mod 4 begin after a 16-byte boundary
    CUtensorMap map_raw[3];  // GEN, shifted: of rows 1, 2, 3 mod 4 (map_a: 0)
    int cl;                 // CTAs of a cluster that share a tile's terms (CG 1)
    int groups;             // shares whose sums stay apart (OUT, cl 1)
    int stay;               // three planes: a tile's sum stays in TMEM
    unsigned stage, b_off;  // bytes of a stage, of A's part of it
};

struct Shared {
    uint64_t full[kStagesMax], empty[kStagesMax], tfull[2], tempty[2], done[2];
    uint64_t raw_full[kRawMax], raw_empty[kRawMax];  // GEN, copies by TMA
    unsigned tmem;
    int give_up;
};

struct Tile {
    int q;               // problem
    int mt, nt, kb0, kb1, group;
};
// Unit u of a launch, of the terms of CTA `share` of a cluster (or of the unit's group).
// Neighbouring units are a patch of `group` row tiles, whose operands the L2 then holds.  SYM:
// row tiles from the diagonal on.
template <int KIND, int CG>
__device__ __forceinline__ Tile tile_of(const GemmArgs &g, int u, int share) {
    Tile t;
    t.q = g.count > 1 && u >= g.p[0].units;
    const ProblemArgs &p = g.p[t.q];
    if (t.q) u -= g.p[0].units;
    t.group = 0;
    if (KIND == GEMM_OUT && g.groups > 1) {
        share = t.group = u / p.units;
        u -= share * p.units;
    }
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
    } else {
        const int per = p.group * p.n_tiles, gr = u / per, m0 = gr * p.group;
        const int w = min(p.group, p.m_tiles - m0);
        u -= gr * per;
        t.nt = u / w;
        t.mt = m0 + u - t.nt * w;
    }
    t.kb0 = share * p.kb_per_split;
    t.kb1 = min(p.kblocks, t.kb0 + p.kb_per_split);
    return t;
}

// The unit of a CTA's round r.  Of two products the second round is dealt out backwards: what
// it still has of the longer tiles goes to those that the last, incomplete round passes by.
__device__ __forceinline__ int unit_at(const GemmArgs &g, int r, int first, int step) {
    return r * step + (r == 1 && g.count > 1 ? step - 1 - first : first);
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
__device__ __forceinline__ void tma_load(unsigned dst, const CUtensorMap *map, int x, int y, int z,
                                         uint64_t *bar) {
    if constexpr (CG == 1)
        asm volatile(
            "cp.async.bulk.tensor.3d.shared::cta.global.tile.mbarrier::complete_tx::bytes "
            "[%0], [%1, {%2, %3, %4}], [%5];\n" ::"r"(dst),
            "l"(map), "r"(x), "r"(y), "r"(z), "r"(smem_addr(bar))
            : "memory");
    else
        asm volatile(
            "cp.async.bulk.tensor.3d.cta_group::2.shared::cluster.global.tile.mbarrier::complete_tx::bytes "
            "[%0], [%1, {%2, %3, %4}], [%5];\n" ::"r"(dst),
            "l"(map), "r"(x), "r"(y), "r"(z), "r"(smem_addr(bar) & 0xFEFFFFFFu)
            : "memory");
}
__device__ __forceinline__ void tma_load_2d(unsigned dst, const CUtensorMap *map, int x, int y, uint64_t *bar) {
    asm volatile(
        "cp.async.bulk.tensor.2d.shared::cta.global.tile.mbarrier::complete_tx::bytes "
        "[%0], [%1, {%2, %3}], [%4];\n" ::"r"(dst),
        "l"(map), "r"(x), "r"(y), "r"(smem_addr(bar))
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
template <typename T>
__device__ __forceinline__ void swap(T &a, T &b) {
    const T t = a;
    a = b;
    b = t;
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

__device__ __forceinline__ void tmem_st16(unsigned taddr, const float (&v)[16]) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], "
        "{%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};\n" ::"r"(taddr),
        "f"(v[0]), "f"(v[1]), "f"(v[2]), "f"(v[3]), "f"(v[4]), "f"(v[5]), "f"(v[6]), "f"(v[7]), "f"(v[8]),
        "f"(v[9]), "f"(v[10]), "f"(v[11]), "f"(v[12]), "f"(v[13]), "f"(v[14]), "f"(v[15])
        : "memory");
}

// ------------------------------------------------------------------ epilogue
// The loops below are over 16 columns of a lane, unrolled, with what does not change
// decided outside them: inside, a decision per element kept each load behind the one
// before (a tile with a residual took 123 us instead of its product's 52).

// Types of two bytes go in pairs where pairs are aligned (`pair`): of columns 2 i and 2 i + 1
// an even lane takes the first for itself and its neighbour, the odd one the second, after
// (before) an exchange between the two.  Half the accesses: with one of two bytes per
// element the epilogue took 8 x 3,700 clocks for a tile of 256 columns in three planes.

// The word of this lane after the exchange: w = (column 2 i, column 2 i + 1) of its row m ->
// (even) column 2 i of rows m, m + 1, (odd) column 2 i + 1 of m - 1, m.  And back.
__device__ __forceinline__ unsigned exchange(unsigned w, bool odd) {
    const unsigned o = __shfl_xor_sync(0xffffffffu, w, 1);
    return odd ? __byte_perm(o, w, 0x7632) : __byte_perm(w, o, 0x5410);
}

// 16 columns of a lane to out[n0 + i][m], row by row: the warp's lanes are neighbours.
// m_end, left: rows m and columns that exist (of planes, a row more may be written).  FULL:
// all 16 and all 32 do, and nothing is asked per element (in three planes with an addend,
// the questions were most of 6,300 clocks per 16 columns).  The whole warp calls it.
template <bool FULL>
__device__ __forceinline__ void store_plane(unsigned short *out, long long ld, bool pair, int m_end, int m, int n0,
                                            int left, const unsigned (&w)[8]) {
    const bool odd = m & 1;
    const bool in = (pair ? m - odd : m) < m_end;
    if (pair) {
        unsigned short *p = out + (long long)(n0 + odd) * ld + (m - odd);
        if (odd) --left;
#pragma unroll
        for (int i = 0; i < 8; ++i, p += 2 * ld) {
            const unsigned x = exchange(w[i], odd);
            if (FULL || (in && 2 * i < left)) *reinterpret_cast<unsigned *>(p) = x;
        }
    } else {
        unsigned short *p = out + (long long)n0 * ld + m;
#pragma unroll
        for (int i = 0; i < 8; ++i, p += 2 * ld) {
            if (FULL || (in && 2 * i < left)) p[0] = (unsigned short)w[i];
            if (FULL || (in && 2 * i + 1 < left)) p[ld] = (unsigned short)(w[i] >> 16);
        }
    }
}
// fp32 or bf16.  (Sums of three planes go to fp32 alone, F32: what a tile's epilogue has in
// instructions it fetches once, and waits for.)
template <bool F32, bool FULL>
__device__ __forceinline__ void store16(void *out, int type, long long ld, bool pair, int m_end, int m, int n0,
                                        int left, const float (&v)[16]) {
    if (F32 || type == GEMM_T_F32) {
        const bool in = m < m_end;
        float *p = static_cast<float *>(out) + (long long)n0 * ld + m;
#pragma unroll
        for (int i = 0; i < 16; ++i, p += ld)
            if (FULL || (in && i < left)) *p = v[i];
        return;
    }
    if constexpr (!F32) {
        unsigned w[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) w[i] = pack_bf16x2(v[2 * i], v[2 * i + 1]);
        store_plane<FULL>(static_cast<unsigned short *>(out), ld, pair, m_end, m, n0, left, w);
    }
}

// 16 columns of a lane of a matrix, on their way: loaded by fetch, values by take (a chunk
// of columns later: nothing waits in between).  fp32 and single elements: 16 words; pairs:
// eight words a plane (planes always go in pairs).
struct Chunk16 {
    unsigned w[24];
};
template <int J, bool FULL>
__device__ __forceinline__ void fetch_pairs(Chunk16 &c, const unsigned short *src, long long ld, int m_end, int m,
                                            int n0, int left) {
    const bool odd = m & 1, in = m - odd < m_end;
    const unsigned short *p = src + (long long)(n0 + odd) * ld + (m - odd);
    if (odd) --left;
#pragma unroll
    for (int i = 0; i < 8; ++i, p += 2 * ld) {
        if (!FULL) c.w[8 * J + i] = 0;
        if (FULL || (in && 2 * i < left)) c.w[8 * J + i] = *reinterpret_cast<const unsigned *>(p);
    }
}
template <bool F32, bool FULL>
__device__ __forceinline__ void fetch16(Chunk16 &c, const void *src, int type, long long ld, bool pair, int m_end,
                                        int m, int n0, int left) {
    const bool in = m < m_end;
    const unsigned short *p = static_cast<const unsigned short *>(src);
    if (F32 || type == GEMM_T_F32) {
        const float *f = static_cast<const float *>(src) + (long long)n0 * ld + m;
#pragma unroll
        for (int i = 0; i < 16; ++i, f += ld) {
            if (!FULL) c.w[i] = 0;
            if (FULL || (in && i < left)) c.w[i] = __float_as_uint(*f);
        }
    } else if (!pair) {
        p += (long long)n0 * ld + m;
#pragma unroll
        for (int i = 0; i < 16; ++i, p += ld) {
            if (!FULL) c.w[i] = 0;
            if (FULL || (in && i < left)) c.w[i] = *p;
        }
    } else {
        fetch_pairs<0, FULL>(c, p, ld, m_end, m, n0, left);
    }
}
// v += scale * what was fetched: P planes in pairs (one: bf16).
template <int P>
__device__ __forceinline__ void take_pairs(const Chunk16 &c, bool odd, float scale, float (&v)[16]) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        float lo = 0.f, hi = 0.f;
#pragma unroll
        for (int j = P - 1; j >= 0; --j) {
            const unsigned x = exchange(c.w[8 * j + i], odd);
            lo += __uint_as_float(x << 16);
            hi += __uint_as_float(x & 0xffff0000u);
        }
        v[2 * i] = fmaf(scale, lo, v[2 * i]);
        v[2 * i + 1] = fmaf(scale, hi, v[2 * i + 1]);
    }
}
// fp32 or bf16.
template <bool F32>
__device__ __forceinline__ void take16(const Chunk16 &c, int type, bool pair, bool odd, float scale,
                                       float (&v)[16]) {
    if (F32 || type == GEMM_T_F32) {
#pragma unroll
        for (int i = 0; i < 16; ++i) v[i] = fmaf(scale, __uint_as_float(c.w[i]), v[i]);
    } else if (!pair) {
#pragma unroll
        for (int i = 0; i < 16; ++i) v[i] = fmaf(scale, __uint_as_float(c.w[i] << 16), v[i]);
    } else {
        take_pairs<1>(c, odd, scale, v);
    }
}
__device__ __forceinline__ void act16(float (&v)[16], int act) {
    if (act == QCNN_ACT_RELU) {
#pragma unroll
        for (int i = 0; i < 16; ++i) v[i] = act_apply(v[i], QCNN_ACT_RELU);
    } else if (act == QCNN_ACT_GELU) {
#pragma unroll
        for (int i = 0; i < 16; ++i) v[i] = act_apply(v[i], QCNN_ACT_GELU);
    } else if (act == QCNN_ACT_SILU) {
#pragma unroll
        for (int i = 0; i < 16; ++i) v[i] = act_apply(v[i], QCNN_ACT_SILU);
    }
}

// OUT: sums v of lane m, columns n0 .. n0 + left - 1; c: what add has there, which next() then
// fetches for the columns that follow.  The whole warp calls it; rows m up to m_end exist.
template <bool F32, bool FULL, typename F>
__device__ __forceinline__ void finish_out(const GemmEpi &e, int m_end, int m, int n0, int left, float alpha,
                                           float bias, float (&v)[16], const Chunk16 &c, F &&next) {
#pragma unroll
    for (int i = 0; i < 16; ++i) v[i] = fmaf(alpha, v[i], bias);
    if (e.pre) store16<F32, FULL>(e.pre, e.out_type, e.ldp, e.pair & 2, m_end, m, n0, left, v);
    act16(v, e.act);
    if (e.add) {
        take16<F32>(c, e.add_type, e.pair & 4, m & 1, e.beta, v);
        next();
    }
    store16<F32, FULL>(e.out, e.out_type, e.ldo, e.pair & 1, m_end, m, n0, left, v);
}

// 16 columns of a lane in P planes.
template <int P>
__device__ __forceinline__ void split16(const float (&v)[16], unsigned (&w)[P][8]) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        if constexpr (P == 3) planes3(v[2 * i], v[2 * i + 1], w[0][i], w[1][i], w[2][i]);
        else if constexpr (P == 2) planes2(v[2 * i], v[2 * i + 1], w[0][i], w[1][i]);
        else w[0][i] = pack_bf16x2(v[2 * i], v[2 * i + 1]);
    }
}

// PLANES and SYM: v = alpha * sum + beta * add (+ diagonal) to P planes whose matrix has room
// for whole tiles, so that nothing is asked about an element.  mirror: to the mirror image as
// well.  (Small products run this once: what counts is how few instructions there are to
// fetch; element by element at the diagonal it took 12,000 clocks.)
template <int P>
__device__ __forceinline__ void finish_planes(const GemmEpi &e, bool mirror, int m, int n0, float (&v)[16],
                                              const Chunk16 &c) {
#pragma unroll
    for (int i = 0; i < 16; ++i) v[i] *= e.alpha;
    if (e.add) take_pairs<P>(c, m & 1, e.beta, v);
    if ((unsigned)(m - n0) < 16u) {
#pragma unroll
        for (int i = 0; i < 16; ++i)
            if (m == n0 + i) v[i] += e.diagonal;
    }
    unsigned w[P][8];
    split16<P>(v, w);
    unsigned short *p = static_cast<unsigned short *>(e.out);
#pragma unroll
    for (int j = 0; j < P; ++j, p += e.out_plane) {
        store_plane<true>(p, e.ldo, true, 0, m, n0, 16, w[j]);
        if (mirror) {  // (rows of 16-byte multiples)
            uint4 *d = reinterpret_cast<uint4 *>(p + (long long)m * e.ldo + n0);
            d[0] = make_uint4(w[j][0], w[j][1], w[j][2], w[j][3]);
            d[1] = make_uint4(w[j][4], w[j][5], w[j][6], w[j][7]);
        }
    }
}

// Running maximum and sum of exp of a lane.  A maximum of -inf has no sum (and adds
// nothing: exp of -inf minus -inf is left out).
struct RunningSum {
    float top = -INFINITY, sum = 0.f;
};
// bias: of the 16 classes, -inf past the last.
__device__ __forceinline__ void stats16(RunningSum &s, int n0, int target, float *target_logit,
                                        const float *bias, float (&v)[16]) {
    float t0 = s.top, t1 = -INFINITY;
#pragma unroll
    for (int i = 0; i < 16; i += 4) {
        const float4 b = *reinterpret_cast<const float4 *>(bias + i);
        v[i] += b.x, v[i + 1] += b.y, v[i + 2] += b.z, v[i + 3] += b.w;
        t0 = fmaxf(t0, fmaxf(v[i], v[i + 1]));
        t1 = fmaxf(t1, fmaxf(v[i + 2], v[i + 3]));
    }
    if ((unsigned)(target - n0) < 16u) {
#pragma unroll
        for (int i = 0; i < 16; ++i)
            if (target == n0 + i) *target_logit = v[i];
    }
    const float top = fmaxf(t0, t1);
    if (top == -INFINITY) {
        // all -inf (nothing to add) or NaN (which fmaxf passes over)
#pragma unroll
        for (int i = 0; i < 16; ++i)
            if (v[i] != v[i]) s.sum = v[i];
        return;
    }
    // (subtracted before it is scaled: top * log2(e) overflows where a whole block is masked by the
    // lowest value, and rounded it would leave exp(0) off 1, again with each block)
    const float2 down = make_float2(-top, -top), scale = make_float2(kLog2e, kLog2e);
    float a0 = 0.f, a1 = 0.f;
#pragma unroll
    for (int i = 0; i < 16; i += 2) {
        const float2 d = __fmul2_rn(__fadd2_rn(make_float2(v[i], v[i + 1]), down), scale);
        a0 += ex2(d.x);
        a1 += ex2(d.y);
    }
    s.sum = (s.top == -INFINITY ? s.sum : s.sum * ex2((s.top - top) * kLog2e)) + (a0 + a1);
    s.top = top;
}

// Gradient of a class (lane m) for 16 rows, in P planes; rows: theirs, without a class past
// the last.
template <int P>
__device__ __forceinline__ void dlogits16(const GemmEpi &e, bool full, int m_end, int m, int n0, int left, float bias,
                                          const float4 *rows, float &col, float (&v)[16]) {
    const int c = e.class0 + m;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        const float4 r = rows[i];
        const int target = __float_as_int(r.z);
        float p = row_share(v[i] + bias, r);
        if (target == c) p -= 1.f;
        // (a row without a class is zero, whatever its logits are)
        v[i] = target >= 0 ? r.y * p : 0.f;
        col += v[i];
    }
    unsigned w[P][8];
    split16<P>(v, w);
    unsigned short *p = static_cast<unsigned short *>(e.out);
#pragma unroll
    for (int j = 0; j < P; ++j, p += e.out_plane) {
        if (full) store_plane<true>(p, e.ldo, true, m_end, m, n0, left, w[j]);
        else store_plane<false>(p, e.ldo, true, m_end, m, n0, left, w[j]);
    }
}

// ---------------------------------------------------------------------- GEN
__device__ __forceinline__ void cp_async4_part(unsigned dst, const void *src, unsigned bytes) {
    asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;\n" ::"r"(dst), "l"(src), "r"(bytes)
                 : "memory");
}
__device__ __forceinline__ void mma_ts(unsigned d, unsigned a, uint64_t b, uint32_t idesc, bool acc) {
    asm volatile(
        "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}\n" ::"r"(d),
        "r"(a), "l"(b), "r"(idesc), "r"((unsigned)acc)
        : "memory");
}
__device__ __forceinline__ void tmem_st8(unsigned taddr, const unsigned (&v)[8]) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};\n" ::"r"(taddr),
        "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7])
        : "memory");
}
// GEN: a warpgroup's registers per thread.  96 at launch (640 threads); 80 for TMA and MMA, 112
// for each of the two that drain and 88 for each of the two that split: 480, which is 5 x 96.
template <int N, bool MORE>
__device__ __forceinline__ void set_registers() {
    if constexpr (MORE) asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;\n" ::"n"(N));
    else asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;\n" ::"n"(N));
}
// What add has at 16 columns of a lane.
template <int KIND, int P>
__device__ __forceinline__ void fetch_add(Chunk16 &c, const ProblemArgs &p, int m, int n0, bool is, bool rows_full) {
    if (!is) return;
    const GemmEpi &e = p.e;
    if constexpr (KIND == GEMM_PLANES || KIND == GEMM_SYM) {
        const unsigned short *src = static_cast<const unsigned short *>(e.add);
        fetch_pairs<0, true>(c, src, e.lda, 0, m, n0, 16);
        fetch_pairs<1, true>(c, src + e.add_plane, e.lda, 0, m, n0, 16);
        if constexpr (P == 3) fetch_pairs<2, true>(c, src + 2 * e.add_plane, e.lda, 0, m, n0, 16);
    } else {
        const int left = p.n - n0;
        if (left <= 0) return;
        if (rows_full && left >= 16)
            fetch16<P == 3, true>(c, e.add, e.add_type, e.lda, e.pair & 4, p.m, m, n0, left);
        else
            fetch16<P == 3, false>(c, e.add, e.add_type, e.lda, e.pair & 4, p.m, m, n0, left);
    }
}

// ------------------------------------------------------------------- kernel
template <int P, int KIND, int CG, bool GEN>
__global__ void __launch_bounds__(GEN ? kGenThreads : 384, 1) gemm_kernel(const __grid_constant__ GemmArgs g) {
    constexpr int BK = GEN ? 32 : 64, KS = BK / 16;
    constexpr int PL = GEN ? 1 : P;  // stages (planes) of a block of terms
    constexpr bool DRAIN = P == 3;   // a block's sum at a time
    // Rings of stages, and as many warps that issue MMAs, each with a ring and an accumulator of
    // its own, which take the accumulators in turn: a block's each, or (g.stay: tiles of one
    // block, or of two and 128 columns, which have an accumulator each) a tile's.  (A warp's
    // waits come back behind the MMAs that it has issued: one alone left the tensor core idle
    // between accumulators, 1,204 clocks per block of 888.  And a ring has one consumer: a wait
    // for a phase two ahead passes at once.)
    constexpr int RINGS = DRAIN ? 2 : 1;
    constexpr int ACC = GEN ? 128 : kAccCols;
    extern __shared__ __align__(128) unsigned char smem_raw[];
    __shared__ Shared sh;
    // what belongs to the 16 columns that a warp is at: bias (STATS), rows (DLOGITS)
    using Column = std::conditional_t<KIND == GEMM_DLOGITS, float4, float>;
    constexpr bool COLUMNS = KIND == GEMM_STATS || KIND == GEMM_DLOGITS;
    constexpr bool PADDED = KIND == GEMM_PLANES || KIND == GEMM_SYM;
    __shared__ __align__(16) Column columns[COLUMNS ? kEpiWarps : 1][2][16];
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
    // (a cluster has one tile)
    const int first_unit = (int)blockIdx.x / (CG * g.cl), step = (int)gridDim.x / CG;

    if (tid == 0) {
        for (int i = 0; i < g.S; ++i) {
            mbar_init(&sh.full[i], GEN ? 1 + kGenWarps : 1);
            mbar_init(&sh.empty[i], 1);
        }
        for (int i = 0; i < 2; ++i) {
            mbar_init(&sh.tfull[i], 1);
            mbar_init(&sh.tempty[i], kEpiWarps * CG);
            mbar_init(&sh.done[i], 1);
        }
        if constexpr (GEN)
            for (int i = 0; i < g.raw; ++i) {
                mbar_init(&sh.raw_full[i], 1);
                mbar_init(&sh.raw_empty[i], kGenWarps);
            }
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
    // (each role waits for the kernel before it where it first needs memory: what it works
    // out before that, a first tile and its operands' maps, took 2,000 clocks)

    if (GEN && warp < 4) set_registers<80, false>();
    if (warp == 0) {
        // --------------------------------------------------------------- TMA
        if (elect_one()) {
            const int S = g.S / RINGS;
            int slot = 0, slot2 = 0;           // next stage of the block's ring, of the other
            unsigned par = 0, par2 = 0, ring = 0;
            unsigned issued = 0, issued2 = 0;
            bool ok = true, synced = false;
            for (int r = 0, u = first_unit; u < g.units && ok; u = unit_at(g, ++r, first_unit, step)) {
                const Tile t = tile_of<KIND, CG>(g, u, share);
                const ProblemArgs &p = g.p[t.q];
                const int m0 = (t.mt * CG + (int)rank) * kMT;
                const int bn = g.bn / CG, n0 = t.nt * g.bn + (int)rank * bn;
                const unsigned bytes = ((GEN ? 0 : p.a.bytes) + p.b.bytes) * CG;
                const bool a_mn = p.a.mn, b_mn = p.b.mn;
                const CUtensorMap *const map_a = &p.map_a, *const map_b = &p.map_b;
                const unsigned a_group = p.a.group_bytes, b_group = p.b.group_bytes;
                // (no prefetch.tensormap: with it every copy of the kernel came slower, 4096 rows of
                // 4096 -> 8192 in 179 us instead of 173)
                if (!synced) {
                    grid_dep_sync();
                    synced = true;
                }
                for (int kb = t.kb0; kb < t.kb1 && ok; ++kb) {
                    const int k = kb * BK;
#pragma unroll
                    for (int z = PL - 1; z >= 0; --z) {  // (in the order that they become free)
                        const int at = (int)ring * S + slot;
                        if (!(ok = wait_one(sh, &sh.empty[at], par ^ 1))) break;
                        uint64_t *const full = &sh.full[at];
                        if (rank == 0) arrive_expect(full, bytes);
                        const unsigned a = smem_addr(smem) + at * g.stage, b = a + g.b_off;
                        if (GEN) {
                        } else if (a_mn) {
                            tma_load<CG>(a, map_a, m0, k, z, full);
                            tma_load<CG>(a + a_group, map_a, m0 + 64, k, z, full);
                        } else {
                            tma_load<CG>(a, map_a, k, m0, z, full);
                        }
                        if (b_mn) {
                            for (int i = 0; i < bn; i += 64)
                                tma_load<CG>(b + (i >> 6) * b_group, map_b, n0 + i, k, z, full);
                        } else {
                            tma_load<CG>(b, map_b, k, n0, z, full);
                        }
                        ++issued;
                        if (++slot == S) {
                            slot = 0;
                            par ^= 1;
                        }
                    }
                    if (RINGS == 2 && (!g.stay || kb + 1 == t.kb1)) {
                        ring ^= 1;
                        swap(slot, slot2);
                        swap(par, par2);
                        swap(issued, issued2);
                    }
                }
            }
            if (!synced) grid_dep_sync();
            // no copy of its own under way when the CTA leaves
            if (rank == 0 || !ok)
                for (int i2 = 0; i2 < RINGS; ++i2, ring ^= 1, issued = issued2)
                    for (unsigned i = issued > (unsigned)S ? issued - S : 0; i < issued; ++i) {
                        const int at = (int)ring * S + (int)(i % S);
                        mbar_wait_bounded(rank == 0 ? &sh.full[at] : &sh.empty[at], i / S & 1, kPolls);
                    }
        }
        __syncwarp();
    } else if (warp == 1 || (RINGS == 2 && warp == 3)) {
        // --------------------------------------------------------------- MMA
        if (rank == 0 && elect_one()) {
            const unsigned ring = warp >> 1;  // this warp's, and its accumulator
            const int S = g.S / RINGS;
            int slot = 0;
            unsigned par = 0;
            unsigned use = 0;  // accumulators so far
            const bool drain = DRAIN && !g.stay;
            bool ok = true;
            const unsigned stage = g.stage >> 4;
            const uint64_t base = (uint64_t)((smem_addr(smem) >> 4) & 0x3FFFu) + ring * S * stage;
            for (int r = 0, u = first_unit; u < g.units && ok; u = unit_at(g, ++r, first_unit, step)) {
                const Tile t = tile_of<KIND, CG>(g, u, share);
                const ProblemArgs &p = g.p[t.q];
                const uint64_t da = p.a.desc + base, db = p.b.desc + base + (g.b_off >> 4);
                const unsigned ka = p.a.kstep, kb_ = p.b.kstep;
                [[maybe_unused]] const unsigned pb = p.b.plane;
                const uint32_t idesc = p.idesc;
                for (int kb = t.kb0; kb < t.kb1; ++kb) {
                    const bool first = drain || kb == t.kb0, last = drain || kb + 1 == t.kb1;
                    const unsigned buf = use & 1, round = use >> 1;
                    if (last) ++use;
                    if (RINGS == 2 && buf != ring) continue;  // the other warp's
                    if (first) {
                        if (!(ok = wait_one(sh, &sh.tempty[buf], (round & 1) ^ 1))) break;
                    }
                    // the stages of this block's planes, the last plane first
                    int at[PL];
#pragma unroll
                    for (int z = PL - 1; z >= 0; --z) {
                        at[z] = slot;
                        ok = ok && wait_one(sh, &sh.full[ring * S + slot], par);
                        if (++slot == S) {
                            slot = 0;
                            par ^= 1;
                        }
                    }
                    if (!ok) break;
                    tc_fence_after_sync();
                    // (three planes: each block's sum apart)
                    const unsigned d = tmem + buf * ACC + (DRAIN && !drain ? (kb - t.kb0) * 128 : 0);
                    bool acc = DRAIN ? false : !first;
                    auto product = [&](int i, int j) {
#pragma unroll
                        for (int s = 0; s < KS; ++s) {
                            if constexpr (GEN)
                                mma_ts(d, tmem + 2 * ACC + (ring * S + at[0]) * kGenCols + i * 16 + s * 8,
                                       db + at[0] * stage + j * pb + s * kb_, idesc, acc);
                            else
                                mma_ss<CG>(d, da + at[i] * stage + s * ka, db + at[j] * stage + s * kb_, idesc, acc);
                            acc = true;
                        }
                    };
                    if constexpr (P == 3) {
                        product(1, 1);
                        product(2, 0);
                        product(0, 2);
                        if constexpr (!GEN) commit<CG>(&sh.empty[ring * S + at[PL - 1]]);
                    }
                    if constexpr (P >= 2) {
                        product(1, 0);
                        product(0, 1);
                        if constexpr (!GEN) commit<CG>(&sh.empty[ring * S + at[PL > 1]]);
                    }
                    product(0, 0);
                    commit<CG>(&sh.empty[ring * S + at[0]]);
                    if (last) commit<CG>(&sh.tfull[buf]);
                }
            }
            // nothing in flight when the tensor memory is freed
            commit_here<CG>(&sh.done[ring]);
            mbar_wait_bounded(&sh.done[ring], 0, kPolls);
        }
        __syncwarp();
    } else if (GEN && warp == 2) {
        // ------------------------------------------------- raw copies by TMA
        // (no wait for the kernel before: the weights are the caller's, complete before the
        // first kernel of this call)
        const ProblemArgs &p = g.p[0];
        if (p.a.way != RAW_WORDS && elect_one()) {
            // (two rings, as the stages: each has one group of warps that reads it)
            const int R = g.raw / 2;
            int slot = 0;
            unsigned par = 0, ring = 0, issued = 0;
            bool ok = true;
            const bool mn = p.a.mn;
            for (int r = 0, u = first_unit; u < g.units && ok; u = unit_at(g, ++r, first_unit, step)) {
                const Tile t = tile_of<KIND, CG>(g, u, share);
                const int m0 = t.mt * kMT;
                for (int kb = t.kb0; kb < t.kb1; ++kb) {
                    const int at = (int)ring * R + slot;
                    if (!(ok = wait_one(sh, &sh.raw_empty[at], par ^ 1))) break;
                    uint64_t *const full = &sh.raw_full[at];
                    const unsigned d = smem_addr(smem) + g.S * g.stage + at * g.raw_bytes;
                    if (p.a.way == RAW_SHIFTED) {
                        const unsigned part = mn ? kShiftedPartMn : kShiftedPart;
                        const int x = mn ? m0 : kb * BK, y = (mn ? kb * BK : m0) / 4;
                        arrive_expect(full, 4 * part);
                        tma_load_2d(d, &p.map_a, x, y, full);
#pragma unroll
                        for (int i = 1; i < 4; ++i) tma_load_2d(d + i * part, &g.map_raw[i - 1], x, y, full);
                    } else if (mn) {
                        arrive_expect(full, kGenWarps * 4096);
#pragma unroll
                        for (int i = 0; i < kGenWarps; ++i)
                            tma_load_2d(d + i * 4096, &p.map_a, m0 + i * 32, kb * BK, full);
                    } else {
                        arrive_expect(full, kGenWarps * 4096);
                        tma_load_2d(d, &p.map_a, kb * BK, m0, full);
                    }
                    ++issued;
                    ring ^= 1;
                    if (ring == 0 && ++slot == R) {
                        slot = 0;
                        par ^= 1;
                    }
                }
            }
            for (unsigned i = issued > (unsigned)g.raw ? issued - g.raw : 0; i < issued; ++i)
                mbar_wait_bounded(&sh.raw_full[(i & 1) * R + (i >> 1) % R], (i >> 1) / R & 1, kPolls);
        }
        __syncwarp();
    } else if (warp >= 4 && warp < 4 + kEpiWarps) {
        // ---------------------------------------------------- drain, epilogue
        if constexpr (GEN) set_registers<112, true>();
        const int quarter = warp & 3, half = (warp - 4) >> 2;
        const unsigned tl = tmem + ((unsigned)(quarter * 32) << 16);
        const int chunks = g.bn / 16;  // this warp's: half, half + 2, ...
        [[maybe_unused]] const unsigned stash = smem_addr(smem);  // (where the stages were)
        grid_dep_sync();
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
        for (int r = 0, u = first_unit; u < g.units; u = unit_at(g, ++r, first_unit, step)) {
            const Tile t = tile_of<KIND, CG>(g, u, share);
            const ProblemArgs &p = g.p[t.q];
            const GemmEpi &e = p.e;
            const int m = (t.mt * CG + (int)rank) * kMT + quarter * 32 + lane, n0 = t.nt * g.bn;
            const bool in = m < p.m;
            [[maybe_unused]] const bool rows_full = m - lane + 32 <= p.m;  // of the whole warp
            // (SYM: the square on the diagonal is computed whole, what is below it is mirrored)
            [[maybe_unused]] const bool mirror = KIND == GEMM_SYM && t.mt * CG * kMT >= n0 + g.bn;
            [[maybe_unused]] float bias = 0.f, col = 0.f;
            [[maybe_unused]] const float alpha = KIND == GEMM_OUT && e.alpha_ptr ? *e.alpha_ptr : e.alpha;
            [[maybe_unused]] RunningSum run;
            [[maybe_unused]] int target = -1;
            if constexpr (KIND == GEMM_STATS) {
                if (in) {
                    const long long c = e.targets[m];
                    target = c >= 0 && c < p.n ? (int)c : -1;
                }
            } else {
                if (!PADDED && e.bias && in) bias = e.bias[m];
            }
            // the sums of the tile, in TMEM at tl + buf * ACC
            unsigned buf = use & 1;
            const bool drain = DRAIN && !g.stay;
            if (drain) {
                constexpr int CH = GEN ? 4 : 8;  // chunks of a warp at most
                float acc[CH][16];
#pragma unroll
                for (int c = 0; c < CH; ++c)
#pragma unroll
                    for (int i = 0; i < 16; ++i) acc[c][i] = 0.f;
                for (int kb = t.kb0; kb < t.kb1; ++kb, ++use) {
                    buf = use & 1;
                    if (!(ok = wait_warp(sh, &sh.tfull[buf], use >> 1 & 1))) break;
                    tc_fence_after_sync();
#pragma unroll
                    for (int c = 0; c < CH; ++c) {
                        if (2 * c + half < chunks) {
                            float v[16];
                            tmem_ld16(tl + buf * ACC + (2 * c + half) * 16, v);
#pragma unroll
                            for (int i = 0; i < 16; i += 2)
                                add2(acc[c][i], acc[c][i + 1], v[i], v[i + 1]);
                        }
                    }
                    // (the last: its columns take the sums, for a loop over chunks that is
                    // not unrolled: instructions fetched once per tile cost more)
                    if (kb + 1 < t.kb1) release(buf);
                }
                if (!ok) break;
#pragma unroll
                for (int c = 0; c < CH; ++c)
                    if (2 * c + half < chunks) tmem_st16(tl + buf * ACC + (2 * c + half) * 16, acc[c]);
                asm volatile("tcgen05.wait::st.sync.aligned;\n" ::: "memory");
            } else {
                ++use;
            }
            // (what a chunk of columns needs from memory is fetched one chunk ahead)
            [[maybe_unused]] Chunk16 add;
            [[maybe_unused]] Column column = {};
            auto fetch = [&](int c) {
                if constexpr (COLUMNS) {
                    const int n = n0 + c * 16 + (lane & 15);
                    const bool is = c < chunks && n < p.n;
                    if constexpr (KIND == GEMM_STATS)
                        column = !is ? -INFINITY : e.bias ? e.bias[n] : 0.f;
                    else
                        column = is ? e.rows[n] : make_float4(0.f, 0.f, __int_as_float(-1), 0.f);
                }
                if constexpr (!COLUMNS) fetch_add<KIND, P>(add, p, m, n0 + c * 16, c < chunks && e.add, rows_full);
            };
            if (g.cl == 1) fetch(half);
            if (!drain) {
                if (!(ok = wait_warp(sh, &sh.tfull[buf], (use - 1) >> 1 & 1))) break;
                tc_fence_after_sync();
            }
#pragma unroll 1
            for (int c = half; c < chunks; c += 2) {
                const int n = n0 + c * 16, left = p.n - n;
                float v[16];
                [[maybe_unused]] Column *const cols = columns[COLUMNS ? warp - 4 : 0][c >> 1 & 1];
                if constexpr (COLUMNS) {
                    if (lane < 16) cols[lane] = column;
                    __syncwarp();
                    fetch(c + 2);
                }
                tmem_ld16(tl + buf * ACC + c * 16, v);
                if (DRAIN && !drain && t.kb1 - t.kb0 > 1) {
                    float v2[16];
                    tmem_ld16(tl + buf * ACC + 128 + c * 16, v2);
#pragma unroll
                    for (int i = 0; i < 16; ++i) v[i] += v2[i];
                }
                if constexpr (KIND == GEMM_STATS) {
                    stats16(run, n, target, e.target_logit + m, cols, v);
                } else if constexpr (KIND == GEMM_DLOGITS) {
                    dlogits16<P>(e, rows_full && left >= 16, p.m, m, n, left, bias, cols, col, v);
                } else if (g.cl > 1) {  // to the cluster
                    const unsigned d = stash + (unsigned)(c * 4 + quarter) * 2048 + lane * 16;
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        asm volatile("st.shared.v4.f32 [%0], {%1, %2, %3, %4};\n" ::"r"(d + i * 512), "f"(v[4 * i]),
                                     "f"(v[4 * i + 1]), "f"(v[4 * i + 2]), "f"(v[4 * i + 3])
                                     : "memory");
                } else if constexpr (PADDED) {
                    finish_planes<P>(e, mirror, m, n, v, add);
                    if (e.add) fetch(c + 2);
                } else if (left > 0) {
                    const int row = n + t.group * p.n;  // (each group's outputs)
                    if (rows_full && left >= 16)
                        finish_out<P == 3, true>(e, p.m, m, row, left, alpha, bias, v, add, [&] { fetch(c + 2); });
                    else
                        finish_out<P == 3, false>(e, p.m, m, row, left, alpha, bias, v, add, [&] { fetch(c + 2); });
                }
            }
            release(buf);
            if constexpr (KIND == GEMM_STATS) {
                if (in) e.stats[(long long)(t.nt * 2 + half) * p.m + m] = make_float2(run.top, run.sum);
            }
            if constexpr (KIND == GEMM_DLOGITS) {
                if (in) e.col_part[(long long)(t.nt * 2 + half) * e.ld_col + m] = col;
            }
        }
        if constexpr (CG == 1 && !COLUMNS) {
            if (g.cl > 1) {
                // The sums of a tile's shares meet in shared memory, where each CTA has left its
                // own: each adds up a part of the columns, in the order of the shares, and does
                // their epilogue.  (Here, where these warps have their registers: for all warps
                // behind the roles the loads of four shares did not fit, 1.5 us more.)
                __syncwarp();
                cluster_sync_all();
                const Tile t = tile_of<KIND, CG>(g, first_unit, share);
                const ProblemArgs &p = g.p[0];
                const GemmEpi &e = p.e;
                const int m = t.mt * kMT + quarter * 32 + lane;
                const bool rows_full = m - lane + 32 <= p.m;
                [[maybe_unused]] const bool mirror = KIND == GEMM_SYM && t.mt * kMT >= (t.nt + 1) * g.bn;
                const float alpha = KIND == GEMM_OUT && e.alpha_ptr ? *e.alpha_ptr : e.alpha;
                const float bias = !PADDED && e.bias && m < p.m ? e.bias[m] : 0.f;
#pragma unroll 1
                for (int c = share + half * g.cl; c < g.bn / 16; c += 2 * g.cl) {
                    const int n = t.nt * g.bn + c * 16, left = p.n - n;
                    Chunk16 add;
                    fetch_add<KIND, P>(add, p, m, n, e.add != nullptr, rows_full);
                    const unsigned mine = smem_addr(smem) + (unsigned)(c * 4 + quarter) * 2048 + lane * 16;
                    float v[16];
#pragma unroll
                    for (int i = 0; i < 16; ++i) v[i] = 0.f;
#pragma unroll 4
                    for (int s = 0; s < g.cl; ++s) {
                        unsigned at;
                        asm("mapa.shared::cluster.u32 %0, %1, %2;\n" : "=r"(at) : "r"(mine), "r"(s));
                        float r[16];
#pragma unroll
                        for (int i = 0; i < 4; ++i)
                            asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];\n"
                                         : "=f"(r[4 * i]), "=f"(r[4 * i + 1]), "=f"(r[4 * i + 2]), "=f"(r[4 * i + 3])
                                         : "r"(at + i * 512)
                                         : "memory");
#pragma unroll
                        for (int i = 0; i < 16; ++i) v[i] += r[i];
                    }
                    if constexpr (PADDED) {
                        finish_planes<P>(e, mirror, m, n, v, add);
                    } else if (left > 0) {
                        if (rows_full && left >= 16)
                            finish_out<P == 3, true>(e, p.m, m, n, left, alpha, bias, v, add, [] {});
                        else
                            finish_out<P == 3, false>(e, p.m, m, n, left, alpha, bias, v, add, [] {});
                    }
                }
                __syncwarp();
                cluster_sync_all();  // (no CTA leaves while another reads from it)
            }
        }
    } else if (GEN && warp >= 12) {
        // ------------------------------------------ copy, split, store planes
        // Two groups of four warps take the blocks in turn, each those of one ring (one group
        // took 1,100 clocks per block for 300 instructions a warp, most of them waiting for the
        // one before: 4.4 TB/s of weights).  A warp has 32 rows (its TMEM lanes) x 32 terms of a
        // block.  Rows of k: [32][32] floats, the 16-byte pieces of a row permuted (TMA's
        // 128-byte swizzle) so that eight neighbouring rows read from all banks; rows of m: [32
        // terms][32].  Where TMA cannot read the matrix, the warp copies its own 32 lines of 128
        // bytes, element by element (a lane each: neighbours), so that no barrier lies between
        // copying and splitting (12 rows of 4097 -> 19456: 109 us, with shifted boxes 66).
        set_registers<88, false>();
        const int quarter = warp & 3, ring = (warp - 12) >> 2;
        const ProblemArgs &p = g.p[0];
        const bool mn = p.a.mn, vec = p.a.way != RAW_WORDS, shifted = p.a.way == RAW_SHIFTED;
        const long long ld = p.a.ld;
        const int slots = vec ? g.raw / 2 : kRawSlots;
        // (TMA: a block is the four warps' parts one after another; shifted: this lane's row, or
        // its first word of the terms 0 mod 4)
        const unsigned own = !shifted ? quarter * 4096
                             : mn     ? (quarter * 32 + lane) * 4
                                      : (lane & 3) * kShiftedPart + (quarter * 8 + (lane >> 2)) * 144 +
                                        g.shift[lane & 3] * 4;
        const unsigned raw = smem_addr(smem) + g.S * g.stage +
                             (vec ? ring * slots * g.raw_bytes + own : (warp - 12) * kRawSlots * 4096);
        const unsigned raw_step = vec ? g.raw_bytes : 4096;
        // this group's blocks (kb0: the block)
        struct Walk {
            int round, u;
            Tile t;
        };
        auto next = [&](Walk &w, int n) {
#pragma unroll 1
            for (; n > 0 && w.u < g.units; --n) {
                if (++w.t.kb0 < w.t.kb1) continue;
                w.u = unit_at(g, ++w.round, first_unit, step);
                if (w.u < g.units) w.t = tile_of<KIND, CG>(g, w.u, share);
            }
        };
        Walk at_split = {-1, first_unit, {}};
        next(at_split, 1 + ring);
        Walk at_copy = at_split;
        int cslot = 0;
        // (the weights are the caller's: no wait, as above)
        auto copy_next = [&]() {
            if (vec) return;
            if (at_copy.u < g.units) {
                const Tile &t = at_copy.t;
                const int row = t.mt * kMT + quarter * 32 + (mn ? lane : 0), k = t.kb0 * BK + (mn ? 0 : lane);
                // lines, and elements of a line from this lane's, that exist
                const int lines = mn ? p.k - k : p.m - row, along = mn ? p.m - row : p.k - k;
                const float *s = p.a.src + (mn ? (long long)k * ld + row : (long long)row * ld + k);
                const unsigned d = raw + cslot * raw_step;
#pragma unroll 4
                for (int j = 0; j < 32; ++j, s += ld) {
                    const unsigned at = mn ? lane * 4 : ((lane >> 2 ^ (j & 7)) << 4) + (lane & 3) * 4;
                    const bool is = along > 0 && lines > j;
                    cp_async4_part(d + j * 128 + at, is ? s : p.a.src, is ? 4 : 0);
                }
                next(at_copy, 2);
                if (++cslot == kRawSlots) cslot = 0;
            }
            cp_async_commit();
        };
        for (int i = 0; i < kRawSlots - 1; ++i) copy_next();
        const unsigned a_dst = tmem + 2 * ACC + ((unsigned)(quarter * 32) << 16);
        const int S = g.S / RINGS;
        int slot = 0, rslot = 0;  // (stages: as the TMA's)
        unsigned par = 0, rpar = 0;
        while (at_split.u < g.units) {
            const int raw_at = ring * slots + rslot;
            if (vec) {
                if (!wait_warp(sh, &sh.raw_full[raw_at], rpar)) break;
            } else {
                cp_async_wait<kRawSlots - 2>();
                __syncwarp();
            }
            const unsigned r = raw + rslot * raw_step;
            float v[32];
            if (shifted && mn) {
#pragma unroll
                for (int i = 0; i < 32; ++i)
                    asm volatile("ld.shared.f32 %0, [%1];\n"
                                 : "=f"(v[i])
                                 : "r"(r + (i & 3) * kShiftedPartMn + (i >> 2) * 528 + g.shift[i & 3] * 4));
            } else if (shifted) {  // (no two lanes in a bank: rows four apart lie 36 words apart)
#pragma unroll
                for (int i = 0; i < 32; ++i)
                    asm volatile("ld.shared.f32 %0, [%1];\n" : "=f"(v[i]) : "r"(r + i * 4));
            } else if (mn) {
#pragma unroll
                for (int i = 0; i < 32; ++i)
                    asm volatile("ld.shared.f32 %0, [%1];\n" : "=f"(v[i]) : "r"(r + i * 128 + lane * 4));
            } else {
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    asm volatile("ld.shared.v4.f32 {%0, %1, %2, %3}, [%4];\n"
                                 : "=f"(v[4 * i]), "=f"(v[4 * i + 1]), "=f"(v[4 * i + 2]), "=f"(v[4 * i + 3])
                                 : "r"(r + lane * 128 + ((i ^ (lane & 7)) << 4)));
            }
            const int at = ring * S + slot;
            if (!wait_warp(sh, &sh.empty[at], par ^ 1)) break;
            tc_fence_after_sync();
            const unsigned d = a_dst + at * kGenCols;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                unsigned w0[8], w1[8], w2[8];
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    planes3(v[16 * h + 2 * i], v[16 * h + 2 * i + 1], w0[i], w1[i], w2[i]);
                tmem_st8(d + 8 * h, w0);
                tmem_st8(d + 8 * h + 16, w1);
                tmem_st8(d + 8 * h + 32, w2);
            }
            __syncwarp();  // (all have read: the slot may be copied to)
            if (vec && lane == 0) arrive(&sh.raw_empty[raw_at]);
            copy_next();
            asm volatile("tcgen05.wait::st.sync.aligned;\n" ::: "memory");
            tc_fence_before_sync();
            __syncwarp();
            if (lane == 0) arrive(&sh.full[at]);
            if (++slot == S) {
                slot = 0;
                par ^= 1;
            }
            if (++rslot == slots) {
                rslot = 0;
                rpar ^= 1;
            }
            next(at_split, 2);
        }
        cp_async_wait<0>();
    }
    if constexpr (CG == 1 && !COLUMNS) {
        if (g.cl > 1 && (warp < 4 || warp >= 4 + kEpiWarps)) {  // (as the epilogue's warps)
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

}  // namespace

// The kernel of a plan, by translation unit.
template <int P, int KIND, int CG, bool GEN>
struct GemmKernel {
    static qcnn_status launch(const void *args, int ctas, size_t smem, cudaStream_t st) {
        const GemmArgs &g = *static_cast<const GemmArgs *>(args);
        const auto k = gemm_kernel<P, KIND, CG, GEN>;
        qcnn_status rc = allow_smem(reinterpret_cast<const void *>(k));
        if (rc != QCNN_OK) return rc;
        const int cluster = CG * g.cl;
        return launch_k(k, dim3(ctas), dim3(GEN ? kGenThreads : 384), smem, st,
                        dim3(cluster > 1 ? cluster : 0, 1, 1), g);
    }
};

}  // namespace qcnn
