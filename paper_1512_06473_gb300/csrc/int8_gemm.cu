// int8_gemm.cu -- products of 8-bit integers on the tensor cores (int8_gemm.cuh).
//
//   y[n][m] = act(xscale[n] (wscale[m] sum_k x[n][k] W[m][k]) + bias[m]) + r
//
// GB300's tensor cores multiply fp16 at many times their rate of 8-bit integers, and fp16 holds
// every code exactly: W is widened on its way, from bytes in shared memory to tensor memory, from where
// the MMAs take it as their operand A; x comes widened (fp16, of the pass that quantizes it) as B.  So W
// is read once, as bytes, and shared memory carries per 64 terms and 128 rows 8 KB of W in and out beside
// x's tile in and out.
//
// Sums.  Products of codes are integers of at most 2^14, sums of up to 1024 of them at most 2^24: fp32
// accumulators hold every one of them exactly.  After 1024 terms a sum is drained to fp32 registers and
// added there.
//
// Tile.  As gemm_kernel.cuh's: 128 (a pair of CTAs: 256) rows of m, TMEM lanes, x bn columns of n.  256
// columns are two accumulators of 128 that the MMAs of a block of 64 terms fill one after the other, so
// that draining the first overlaps the MMAs of the second; fewer columns take two accumulators in turn.
// TMEM: 256 columns of accumulators, eight stages of W, 64 terms in 32 columns each.
//
// Roles (16 warps): 0 TMA of x, 1 MMA, 2 TMEM and TMA of W, 4-11 drain and epilogue (two warps per TMEM
// lane quarter), 12-15 widen: a warp has its 32 rows of W, a lane a row, 128 terms at a time.
#define QCNN_UNIT_RECORDS
#include "int8_gemm.cuh"

#include "gemm_kernel.cuh"

#include <algorithm>
#include <array>
#include <map>
#include <mutex>

namespace qcnn {
namespace {

constexpr int kThreads = 512;
constexpr int kWStages = 8;            // stages of W in TMEM at most
constexpr int kWCols = 32;             // TMEM columns of one
constexpr int kRawTerms = 128;         // terms of a copy of W: 128 rows x 128 bytes
constexpr unsigned kRawBytes = 128 * kRawTerms;
constexpr int kRawStages = 4;
constexpr int kSumBlocks = 16;         // blocks of 64 terms whose sum is exact
constexpr size_t kSmem = 222 * 1024;   // dynamic, with 1 KB to align the stages
constexpr size_t kSmemFloor = 120 * 1024;  // one CTA per SM: all tensor memory is taken

struct Int8Args {
    CUtensorMap map_w, map_x;
    int m, n, kblocks, m_tiles, n_tiles, kb_per_split, group, units;
    int bn, S, cl, w_late;
    unsigned stage;  // bytes of a stage of x
    unsigned idesc;
    const float *xscale, *wscale;
    const int *sums;  // WIDE: of the magnitudes of x's codes, [n][segs], each of 1024 terms; null: segs 1
    int segs;
    GemmEpi e;
};
struct Int8Shared {
    uint64_t full[kWStages], empty[kWStages], raw_full[kRawStages], raw_empty[kRawStages], tfull[2], tempty[2], done;
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

// The largest sum of magnitudes of a segment in the 256 rows of x from n0 on: loads, and their maximum.
__device__ __forceinline__ void load_sums(const Int8Args &g, int n0, int seg, int (&v)[8]) {
    const int lane = threadIdx.x & 31;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int n = n0 + lane + 32 * i;
        v[i] = n < g.n && seg < g.segs ? g.sums[(long long)n * g.segs + seg] : 0;
    }
}
__device__ __forceinline__ int most_of(const int (&v)[8]) {
    int t = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) t = max(t, v[i]);
    return __reduce_max_sync(0xffffffffu, t);
}
// Where a sum in the accumulators ends (exclusive): the last segment, from k0's on, with which it is sure
// to stay exact, any code of W being at most 128.  used: the magnitudes in it so far.
__device__ __forceinline__ bool ends_here(int used, int next) { return used + next > (1 << 24) / 128; }

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

// An arrival on CTA 0 of the pair, of what this thread did to tensor memory.  (Its default order, of
// this CTA alone: with .release.cluster, which waits for what the thread has under way, a block of 64
// terms took 1,700 clocks instead of 600.)
__device__ __forceinline__ void arrive_first(uint64_t *bar) {
    asm volatile(
        "{\n\t.reg .b32 a;\n\t"
        "mapa.shared::cluster.u32 a, %0, 0;\n\t"
        "mbarrier.arrive.shared::cluster.b64 _, [a];\n\t}\n" ::"r"(smem_addr(bar))
        : "memory");
}
// 64 columns of this warp's lanes; tmem_ld_wait before they are used.
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
// 16 columns of a lane: sums v of row m (of m_end), columns n to n + left - 1, to the result.  xs: the
// columns' scales.  A warp's lanes are neighbours in the result; two-byte elements go in pairs where
// pairs are aligned (gemm_kernel.cuh).  The whole warp calls it.
__device__ __forceinline__ void int8_finish(const GemmEpi &e, int m_end, int m, int n, int left, float alpha, float bias,
                                            const float *xs, float (&v)[16]) {
    const bool f32 = e.out_type == GEMM_T_F32, odd = m & 1, in = m < m_end;
    const int count = in ? min(left, 16) : 0;
    unsigned r[16];
    if (e.add) {  // (on its way while the activation is computed)
        if (f32) {
            const float *p = static_cast<const float *>(e.add) + (long long)n * e.lda + m;
#pragma unroll
            for (int j = 0; j < 16; ++j) r[j] = j < count ? __float_as_uint(p[j * e.lda]) : 0;
        } else if (e.pair & 4) {
            const unsigned short *p = static_cast<const unsigned short *>(e.add) + (long long)(n + odd) * e.lda + (m - odd);
#pragma unroll
            for (int j = 0; j < 8; ++j)
                r[j] = 2 * j < count - odd ? *reinterpret_cast<const unsigned *>(p + 2 * j * e.lda) : 0;
        } else {
            const unsigned short *p = static_cast<const unsigned short *>(e.add) + (long long)n * e.lda + m;
#pragma unroll
            for (int j = 0; j < 16; ++j) r[j] = j < count ? (unsigned)p[j * e.lda] << 16 : 0;
        }
    }
    const float2 a2 = make_float2(alpha, alpha), b2 = make_float2(bias, bias);
#pragma unroll
    for (int j = 0; j < 16; j += 4) {
        const float4 s = *reinterpret_cast<const float4 *>(xs + j);
        float2 z = __ffma2_rn(a2, __fmul2_rn(make_float2(v[j], v[j + 1]), make_float2(s.x, s.y)), b2);
        v[j] = z.x, v[j + 1] = z.y;
        z = __ffma2_rn(a2, __fmul2_rn(make_float2(v[j + 2], v[j + 3]), make_float2(s.z, s.w)), b2);
        v[j + 2] = z.x, v[j + 3] = z.y;
    }
    act16(v, e.act);
    if (e.add) {
        if (!f32 && e.pair & 4) {
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const unsigned x = exchange(r[j], odd);
                add2(v[2 * j], v[2 * j + 1], __uint_as_float(x << 16), __uint_as_float(x & 0xffff0000u));
            }
        } else {
#pragma unroll
            for (int j = 0; j < 16; j += 2) add2(v[j], v[j + 1], __uint_as_float(r[j]), __uint_as_float(r[j + 1]));
        }
    }
    if (f32) {
        float *p = static_cast<float *>(e.out) + (long long)n * e.ldo + m;
#pragma unroll
        for (int j = 0; j < 16; ++j)
            if (j < count) p[j * e.ldo] = v[j];
    } else if (e.pair & 1) {
        unsigned short *p = static_cast<unsigned short *>(e.out) + (long long)(n + odd) * e.ldo + (m - odd);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const unsigned x = exchange(pack_bf16x2(v[2 * j], v[2 * j + 1]), odd);
            if (2 * j < count - odd) *reinterpret_cast<unsigned *>(p + 2 * j * e.ldo) = x;
        }
    } else {
        unsigned short *p = static_cast<unsigned short *>(e.out) + (long long)n * e.ldo + m;
#pragma unroll
        for (int j = 0; j < 16; ++j)
            if (j < count) p[j * e.ldo] = float_to_bf16(v[j]);
    }
}

// ------------------------------------------------------------------- kernel
// WIDE: tiles of 256 columns.
template <int CG, bool WIDE>
__global__ void __launch_bounds__(kThreads, 1) int8_kernel(const __grid_constant__ Int8Args g) {
    extern __shared__ __align__(128) unsigned char smem_raw[];
    __shared__ Int8Shared sh;
    __shared__ __align__(16) float column_scales[8][16];
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
    const int cols = WIDE ? 128 : g.bn;              // columns of one
    const int rows_x = cols / CG;                    // rows of x per accumulator, here
    const unsigned raw0 = smem_addr(smem) + g.S * g.stage;
    if (tid == 0) {
        for (int i = 0; i < g.S; ++i) {
            mbar_init(&sh.full[i], 1 + 4 * CG);
            mbar_init(&sh.empty[i], 1);
        }
        for (int i = 0; i < kRawStages; ++i) {
            mbar_init(&sh.raw_full[i], 1);
            mbar_init(&sh.raw_empty[i], 4);
        }
        for (int i = 0; i < 2; ++i) {
            mbar_init(&sh.tfull[i], 1);
            mbar_init(&sh.tempty[i], (WIDE ? 4 : 8) * CG);
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

    if (warp < 4) set_registers<40, false>();
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
                for (int kb = t.kb0; kb < t.kb1; ++kb) {
                    if (!(ok = wait_for(sh, &sh.empty[slot], par ^ 1))) break;
                    uint64_t *const full = &sh.full[slot];
                    if (rank == 0) arrive_expect(full, g.stage * CG);
                    const unsigned d = smem_addr(smem) + slot * g.stage;
#pragma unroll
                    for (int h = 0; h < NH; ++h)
                        tma_box<CG>(d + h * rows_x * 128, &g.map_x, kb * 64, n0 + h * 128, full);
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
        if (rank == 0) {
            const bool lead = elect_one();
            if (WIDE && g.sums) grid_dep_sync();
            int slot = 0;
            unsigned par = 0;
            unsigned sums = 0;  // in the accumulators, so far
            bool ok = true;
            const uint64_t desc = 1ull << 16 | (uint64_t)(1024 >> 4) << 32 | 1ull << 46 | 2ull << 61 |
                                  (uint64_t)((smem_addr(smem) >> 4) & 0x3FFFu);
            for (int u = first_unit; u < g.units && ok; u += step) {
                const Int8Tile t = int8_tile(g, u, share);
                bool first = true;  // of a sum
                [[maybe_unused]] int used = 0, more[8];
                if (WIDE && g.sums) {
                    load_sums(g, t.nt * 256, 0, more);
                    used = most_of(more);
                }
                for (int k0 = t.kb0; k0 < t.kb1 && ok; k0 += kSumBlocks) {
                    const int k1 = min(t.kb1, k0 + kSumBlocks);
                    if (WIDE && g.sums) load_sums(g, t.nt * 256, k0 / kSumBlocks + 1, more);
                    const unsigned buf = WIDE ? 0 : sums & 1, round = WIDE ? sums : sums >> 1;
                    bool end = true;
                    for (int kb = k0; kb < k1; ++kb) {
                        if (!(ok = warp_wait_for(sh, &sh.full[slot], par))) break;
                        tc_fence_after_sync();
                        if (WIDE && kb + 1 == k1 && k1 < t.kb1 && g.sums) {
                            const int next = most_of(more);
                            end = ends_here(used, next);
                            used = end ? next : used + next;
                        }
                        const bool last = end && kb + 1 == k1;
                        const unsigned a = tmem + 256 + slot * kWCols;
                        const uint64_t b = desc + (uint64_t)(slot * (g.stage >> 4));
#pragma unroll
                        for (int h = 0; h < NH; ++h) {
                            if (first) {
                                if (!(ok = warp_wait_for(sh, &sh.tempty[buf + h], (round & 1) ^ 1))) break;
                                tc_fence_after_sync();
                            }
                            const unsigned d = tmem + (buf + h) * 128;
                            if (lead) {
#pragma unroll
                                for (int s = 0; s < 4; ++s)
                                    mma_tmem<CG>(d, a + s * 8, b + h * (rows_x * 8) + s * 2, g.idesc, !first || s > 0);
                                if (last && h + 1 < NH) commit<CG>(&sh.tfull[buf + h]);
                            }
                        }
                        if (!ok) break;
                        first = false;
                        if (lead) {
                            commit<CG>(&sh.empty[slot]);
                            if (last) commit<CG>(&sh.tfull[buf + NH - 1]);
                        }
                        __syncwarp();
                        if (++slot == g.S) {
                            slot = 0;
                            par ^= 1;
                        }
                    }
                    if (end) {
                        first = true;
                        ++sums;
                    }
                }
            }
            // nothing in flight when the tensor memory is freed
            if (lead) {
                commit_here<CG>(&sh.done);
                mbar_wait_bounded(&sh.done, 0, kPolls);
            }
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
                for (int kb = t.kb0; kb < t.kb1; kb += 2) {
                    if (!(ok = wait_for(sh, &sh.raw_empty[slot], par ^ 1))) break;
                    arrive_expect(&sh.raw_full[slot], kRawBytes);
                    tma_load_2d(raw0 + slot * kRawBytes, &g.map_w, kb * 64, m0, &sh.raw_full[slot]);
                    ++issued;
                    if (++slot == kRawStages) {
                        slot = 0;
                        par ^= 1;
                    }
                }
            }
            for (unsigned i = issued > (unsigned)kRawStages ? issued - kRawStages : 0; i < issued; ++i)
                mbar_wait_bounded(&sh.raw_full[i % kRawStages], i / kRawStages & 1, kPolls);
        }
        __syncwarp();
    } else if (warp >= 4 && warp < 12) {
        // ---------------------------------------------------- drain, epilogue
        set_registers<200, true>();
        const int quarter = warp & 3, half = (warp - 4) >> 2;
        const unsigned tl = tmem + ((unsigned)(quarter * 32) << 16);
        grid_dep_sync();
        const GemmEpi &e = g.e;
        constexpr int CH = WIDE ? 8 : 4;  // chunks of 16 columns of a warp at most
        // this warp's chunk i: WIDE: of its accumulator; else every other one
        const int chunks = WIDE ? 8 : (g.bn / 16 - half + 1) / 2;
        auto chunk_at = [&](int i) { return WIDE ? half * 8 + i : 2 * i + half; };
        unsigned sums = 0;
        bool ok = true;
        float acc[CH][16];
        float *const scales = column_scales[warp - 4];
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
            [[maybe_unused]] int used = 0, more[8];
            if (WIDE && g.sums) {
                load_sums(g, n0, 0, more);
                used = most_of(more);
            }
            // (the residual's lines, from memory to the L2)
            if (WIDE && e.add) {
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int n = n0 + half * 128 + lane + 32 * i, m1 = m - lane;
                    if (n < g.n && m1 < g.m)
                        asm volatile("prefetch.global.L2 [%0];\n" ::"l"(
                            static_cast<const char *>(e.add) +
                            ((long long)n * e.lda + m1) * (e.add_type == GEMM_T_F32 ? 4 : 2)));
                }
            }
            bool first = true;
            for (int k0 = t.kb0; k0 < t.kb1; k0 += kSumBlocks) {
                if (WIDE && k0 + kSumBlocks < t.kb1 && g.sums) {  // (as the MMAs' warp)
                    load_sums(g, n0, k0 / kSumBlocks + 1, more);
                    const int next = most_of(more);
                    const bool end = ends_here(used, next);
                    used = end ? next : used + next;
                    if (!end) continue;
                }
                const unsigned buf = WIDE ? half : sums & 1;
                if (!(ok = warp_wait_for(sh, &sh.tfull[buf], (WIDE ? sums : sums >> 1) & 1))) break;
                ++sums;
                tc_fence_after_sync();
                const unsigned from = tl + buf * 128;
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
                            for (int i = 0; i < 16; i += 2) {
                                if (first) acc[c][i] = v[i], acc[c][i + 1] = v[i + 1];
                                else add2(acc[c][i], acc[c][i + 1], v[i], v[i + 1]);
                            }
                        }
                    }
                }
                first = false;
                release(buf);
            }
            if (!ok) break;
            const float alpha = m < g.m ? g.wscale[m] : 0.f, bias = e.bias && m < g.m ? e.bias[m] : 0.f;
            // (the sums move through the first chunk's registers: unrolled, the epilogue's instructions
            // would come eight times)
#pragma unroll 1
            for (int i = 0; i < chunks; ++i) {
                const int c = chunk_at(i), n = n0 + c * 16, left = g.n - n;
                float v[16];
#pragma unroll
                for (int j = 0; j < 16; ++j) v[j] = acc[0][j];
#pragma unroll
                for (int k = 0; k + 1 < CH; ++k)
#pragma unroll
                    for (int j = 0; j < 16; ++j) acc[k][j] = acc[k + 1][j];
                if (g.cl > 1) {  // to the cluster
                    const unsigned d = smem_addr(smem) + (unsigned)(c * 4 + quarter) * 2048 + lane * 16;
#pragma unroll
                    for (int j = 0; j < 4; ++j)
                        asm volatile("st.shared.v4.f32 [%0], {%1, %2, %3, %4};\n" ::"r"(d + j * 512), "f"(v[4 * j]),
                                     "f"(v[4 * j + 1]), "f"(v[4 * j + 2]), "f"(v[4 * j + 3])
                                     : "memory");
                } else if (left > 0) {
                    __syncwarp();  // (the chunk before has been read)
                    if (lane < 16) scales[lane] = lane < left ? g.xscale[n + lane] : 0.f;
                    __syncwarp();
                    int8_finish(e, g.m, m, n, left, alpha, bias, scales, v);
                }
            }
        }
        if constexpr (CG == 1) {
            if (g.cl > 1) {
                // The sums of a tile's shares meet in shared memory, where each CTA has left its own: each
                // adds up a part of the columns, in the order of the shares, and does their epilogue.
                __syncwarp();
                cluster_sync_all();
                const Int8Tile t = int8_tile(g, first_unit, share);
                const int m = t.mt * 128 + quarter * 32 + lane;
                const float alpha = m < g.m ? g.wscale[m] : 0.f, bias = e.bias && m < g.m ? e.bias[m] : 0.f;
#pragma unroll 1
                for (int c = share + half * g.cl; c < g.bn / 16; c += 2 * g.cl) {
                    const int n = t.nt * g.bn + c * 16, left = g.n - n;
                    if (left <= 0) break;
                    __syncwarp();
                    if (lane < 16) scales[lane] = lane < left ? g.xscale[n + lane] : 0.f;
                    __syncwarp();
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
                    int8_finish(e, g.m, m, n, left, alpha, bias, scales, v);
                }
                __syncwarp();
                cluster_sync_all();  // (no CTA leaves while another reads from it)
            }
        }
    } else if (warp >= 12) {
        // -------------------------------------------------------------- widen
        set_registers<72, false>();
        const int quarter = warp & 3;
        const unsigned a_dst = tmem + 256 + ((unsigned)(quarter * 32) << 16);
        const unsigned own = raw0 + (quarter * 32 + lane) * 128;  // (the pieces of a row permuted: 128-byte swizzle)
        int slot = 0, rslot = 0;
        unsigned par = 0, rpar = 0;
        bool ok = true;
        for (int u = first_unit; u < g.units && ok; u += step) {
            const Int8Tile t = int8_tile(g, u, share);
            for (int kb = t.kb0; kb < t.kb1 && ok; kb += 2) {
                if (!(ok = warp_wait_for(sh, &sh.raw_full[rslot], rpar))) break;
                const unsigned from = own + rslot * kRawBytes;
#pragma unroll
                for (int s = 0; s < 2; ++s) {
                    if (kb + s >= t.kb1) break;
                    unsigned w[16], v[32];
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];\n"
                                     : "=r"(w[4 * i]), "=r"(w[4 * i + 1]), "=r"(w[4 * i + 2]), "=r"(w[4 * i + 3])
                                     : "r"(from + (((4 * s + i) ^ (lane & 7)) << 4)));
#pragma unroll
                    for (int i = 0; i < 16; ++i) widen4(w[i], v[2 * i], v[2 * i + 1]);
                    if (!(ok = warp_wait_for(sh, &sh.empty[slot], par ^ 1))) break;
                    tc_fence_after_sync();
                    tmem_st32(a_dst + slot * kWCols, v);
                    asm volatile("tcgen05.wait::st.sync.aligned;\n" ::: "memory");
                    tc_fence_before_sync();
                    __syncwarp();
                    if (lane == 0) {
                        if constexpr (CG == 1) arrive(&sh.full[slot]);
                        else arrive_first(&sh.full[slot]);
                    }
                    if (++slot == g.S) {
                        slot = 0;
                        par ^= 1;
                    }
                }
                if (lane == 0) arrive(&sh.raw_empty[rslot]);
                if (++rslot == kRawStages) {
                    rslot = 0;
                    rpar ^= 1;
                }
            }
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
    return launch_k(k, dim3(ctas), dim3(kThreads), smem, st, dim3(cluster > 1 ? cluster : 0, 1, 1), g);
}

// Whether a matrix of two-byte elements can go in pairs of neighbours along m.
bool in_pairs(const void *p, int type, long long ld, int m) {
    return type != GEMM_T_F32 && p && reinterpret_cast<uintptr_t>(p) % 4 == 0 && ld % 2 == 0 && m % 2 == 0;
}

Int8Plan plan_int8_anew(int m, int n, int k, int sms) {
    Int8Plan best;
    const int kblocks = cdiv(k, 64);
    static const int tiles[5] = {16, 32, 64, 128, 256};
    for (int cg = 1; cg <= 2; ++cg)
        for (int bn : tiles) {
            if (cg == 2 && bn != 256) continue;
            if (bn > 16 && bn >= 2 * n) continue;
            const int mt = cdiv(m, 128 * cg), nt = cdiv(n, bn);
            const long long units = (long long)mt * nt;
            // clocks of a block of 64 terms: MMAs; bytes of W at the memory's rate when all SMs read, with
            // x's at TMA's; shared memory, in and out; the widening
            const double mma = 4 * (bn / 2 + 10.0), w = 8192.0, x = bn / cg * 128.0;
            const double per = std::max({mma, w / 23.0, (w + x) / 50.0, 2 * (w + x) / 128.0, 250.0});
            const double tail = 4500.0 + bn * 16.0;
            for (int cl = 1; cl <= 8; cl *= 2) {
                if (cl > 1 && (cg > 1 || bn > 128 || 2 * cl > kblocks)) break;
                const int kps = cdiv(cdiv(kblocks, cl), 2) * 2;
                if (cdiv(kblocks, kps) != cl) continue;
                const int slots = cl == 1 ? sms / cg
                                          : std::max(1, cluster_capacity(reinterpret_cast<const void *>(int8_kernel<1, false>),
                                                                         kThreads, cl, kSmem));
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
    const int cg = plan.cg, bn = plan.bn, wide = bn == 256;
    const int box = (wide ? 128 : bn) / cg;  // rows of x at a time
    qcnn_status rc = tensor_map(CU_TENSOR_MAP_DATA_TYPE_UINT8, p.W, p.k, p.m, p.ldw, kRawTerms, 128, true, &g.map_w);
    if (rc != QCNN_OK) return rc;
    rc = tensor_map(CU_TENSOR_MAP_DATA_TYPE_FLOAT16, p.x, p.k, p.n, p.ldx * 2, 64, box, true, &g.map_x);
    if (rc != QCNN_OK) return rc;
    g.m = p.m;
    g.n = p.n;
    g.kblocks = cdiv(p.k, 64);
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
    g.stage = (unsigned)(bn / cg * 128);
    g.S = (int)std::min<size_t>(kWStages, (kSmem - 1024 - kRawStages * (size_t)kRawBytes) / g.stage);
    // fp32 sums of fp16, 128 (256) rows x the columns of an accumulator
    g.idesc = (1u << 4) | (uint32_t)((wide ? 128 : bn) >> 3) << 17 | (uint32_t)(128 * cg >> 4) << 24;
    g.sums = wide && p.segs > 1 ? p.sums : nullptr;
    g.segs = p.segs;
    g.xscale = p.xscale;
    g.wscale = p.wscale;
    g.e = p.e;
    g.e.beta = 1.f;
    g.e.pair = (in_pairs(p.e.out, p.e.out_type, p.e.ldo, p.m) ? 1 : 0) |
               (in_pairs(p.e.add, p.e.add_type, p.e.lda, p.m) ? 4 : 0);
    const size_t stash = g.cl > 1 ? (size_t)bn * 512 : 0;
    const size_t smem = std::max({kSmemFloor, g.S * (size_t)g.stage + kRawStages * (size_t)kRawBytes + 1024, stash + 1024});
    const int ctas = g.cl > 1 ? g.units * g.cl : std::min(g.units, num_sms() / cg) * cg;
    if (cg == 2) return launch_of<2, true>(g, ctas, smem, st);
    return wide ? launch_of<1, true>(g, ctas, smem, st) : launch_of<1, false>(g, ctas, smem, st);
}

}  // namespace qcnn
