// gemm.cu -- plans and launches of the tensor-core products (gemm.cuh), and the pass that lays
// fp32 or unaligned data out as planes.
#include "gemm_kernel.cuh"

#include <algorithm>
#include <array>
#include <map>
#include <mutex>

namespace qcnn {

// (gemm_p1.cu, gemm_p2.cu, gemm_p3.cu, gemm_f32.cu)
using GemmLaunch = qcnn_status (*)(const void *, int, size_t, cudaStream_t);
GemmLaunch gemm_launch_p1(int kind, int cg);
const void *gemm_kernel_address();
GemmLaunch gemm_launch_p3(int kind, int cg);
GemmLaunch gemm_launch_planes(int planes, int kind, int cg);
GemmLaunch gemm_launch_f32();

namespace {

constexpr size_t kSmemMax = 222 * 1024;  // dynamic, with 1 KB to align the stages
// one CTA per SM, whatever it needs: all tensor memory is taken
constexpr size_t kSmemLeast = 120 * 1024;

using EncodeTiled = CUresult (*)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *,
                                 const cuuint64_t *, const cuuint64_t *, const cuuint32_t *,
                                 const cuuint32_t *, CUtensorMapInterleave, CUtensorMapSwizzle,
                                 CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
EncodeTiled encode_tiled() {
    static EncodeTiled f = nullptr;
    static std::once_flag once;
    std::call_once(once, [] {
        void *p = nullptr;
        cudaDriverEntryPointQueryResult q;
        if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &p, 12000, cudaEnableDefault,
                                             &q) == cudaSuccess &&
            q == cudaDriverEntryPointSuccess)
            f = reinterpret_cast<EncodeTiled>(p);
        cudaGetLastError();
    });
    return f;
}

// An operand of `rows` rows (this CTA's part of a tile); rows_all x k is its matrix.
qcnn_status set_operand(const GemmOperand &o, int P, bool gen, int rows, int rows_all, int k, OpArgs *a,
                        CUtensorMap *map) {
    const int bk = gemm_block_k(gen ? GEMM_F32 : P), box_planes = gen ? P : 1;
    a->mn = o.mn;
    a->group_bytes = box_planes * bk * 128;
    a->bytes = o.mn ? cdiv(rows, 64) * a->group_bytes : (unsigned)box_planes * rows * bk * 2;
    a->plane = o.mn ? bk * 128 / 16 : rows * bk * 2 / 16;
    a->kstep = o.mn ? 2048 / 16 : 32 / 16;
    const bool sw64 = !o.mn && bk == 32;
    const uint64_t sbo = sw64 ? 512 : 1024, lbo = o.mn ? a->group_bytes : 16;
    a->desc = (lbo >> 4) << 16 | (sbo >> 4) << 32 | 1ull << 46 | (uint64_t)(sw64 ? 4 : 2) << 61;
    const EncodeTiled enc = encode_tiled();
    if (!enc) return QCNN_ERR_CUDA;
    const cuuint64_t inner = o.mn ? rows_all : k, outer = o.mn ? k : rows_all;
    const cuuint64_t dims[3] = {inner, outer, (cuuint64_t)P};
    const cuuint64_t strides[2] = {(cuuint64_t)o.ld * 2, (cuuint64_t)(P > 1 ? o.plane : o.ld * outer) * 2};
    const cuuint32_t box[3] = {o.mn ? 64u : (cuuint32_t)bk, o.mn ? (cuuint32_t)bk : (cuuint32_t)rows,
                               (cuuint32_t)box_planes};
    const cuuint32_t steps[3] = {1, 1, 1};
    const CUresult r = enc(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<void *>(o.p), dims, strides,
                           box, steps, CU_TENSOR_MAP_INTERLEAVE_NONE,
                           sw64 ? CU_TENSOR_MAP_SWIZZLE_64B : CU_TENSOR_MAP_SWIZZLE_128B,
                           CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    if (r != CUDA_SUCCESS) return cuda_status(cudaErrorInvalidValue);
    return QCNN_OK;
}

// The map of an fp32 A: boxes of 32 terms x 128 rows, or of 32 rows x 32 terms where the rows
// are contiguous.
qcnn_status raw_map(const void *p, long long inner, long long outer, long long row_bytes, unsigned box_x,
                    unsigned box_y, bool swizzle, CUtensorMap *map) {
    const EncodeTiled enc = encode_tiled();
    if (!enc) return QCNN_ERR_CUDA;
    const cuuint64_t dims[2] = {(cuuint64_t)inner, (cuuint64_t)outer};
    const cuuint64_t strides[1] = {(cuuint64_t)row_bytes};
    const cuuint32_t box[2] = {box_x, box_y}, steps[2] = {1, 1};
    const CUresult r = enc(map, CU_TENSOR_MAP_DATA_TYPE_FLOAT32, 2, const_cast<void *>(p), dims, strides, box, steps,
                           CU_TENSOR_MAP_INTERLEAVE_NONE,
                           swizzle ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_NONE,
                           CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    return r == CUDA_SUCCESS ? QCNN_OK : cuda_status(cudaErrorInvalidValue);
}
// Maps and way of an fp32 A (RawWay).
qcnn_status set_raw(const GemmOperand &o, int rows, int k, GemmArgs *g) {
    ProblemArgs &p = g->p[0];
    const char *const base = static_cast<const char *>(o.p);
    const long long inner = o.mn ? rows : k, outer = o.mn ? k : rows;
    g->raw_bytes = kGenWarps * 4096;
    p.a.way = RAW_WORDS;
    if (reinterpret_cast<uintptr_t>(base) % 16) return QCNN_OK;
    if (o.ld % 4 == 0) {
        p.a.way = RAW_BOXES;
        return raw_map(base, inner, outer, o.ld * 4, 32, o.mn ? 32 : kMT, !o.mn, &p.map_a);
    }
    if (outer < 4) return QCNN_OK;  // (each map has rows)
    p.a.way = RAW_SHIFTED;
    g->raw_bytes = (unsigned)align_up(4 * (o.mn ? kShiftedPartMn : kShiftedPart), 128);
    for (int i = 0; i < 4; ++i) {
        // row i, i + 4, ...: from the boundary before row i on, which is in the matrix
        const long long at = i * o.ld * 4;
        g->shift[i] = (int)(at % 16 / 4);
        const qcnn_status rc = raw_map(base + at / 16 * 16, g->shift[i] + inner, (outer - i + 3) / 4, o.ld * 16,
                                       o.mn ? 132 : 36, o.mn ? 8 : 32, false, i ? &g->map_raw[i - 1] : &p.map_a);
        if (rc != QCNN_OK) return rc;
    }
    return QCNN_OK;
}

long long tiles_of(int kind, int m_tiles, int n_tiles, int per) {
    if (kind != GEMM_SYM) return (long long)m_tiles * n_tiles;
    long long t = 0;
    for (int i = 0; i < n_tiles; ++i) t += std::max(0, m_tiles - i * per);
    return t;
}

// Whether a matrix of two-byte elements can go in pairs of neighbours along m.
bool pairs(const void *p, int type, long long ld, int m) {
    return type != GEMM_T_F32 && p && reinterpret_cast<uintptr_t>(p) % 4 == 0 && ld % 2 == 0 && m % 2 == 0;
}

GemmLaunch launcher(const GemmPlan &p) {
    if (p.planes == GEMM_F32) return gemm_launch_f32();
    if (p.planes == 2 || p.kind == GEMM_SYM || p.kind == GEMM_PLANES)
        return gemm_launch_planes(p.planes, p.kind, p.cg);
    return p.planes == 1 ? gemm_launch_p1(p.kind, p.cg) : gemm_launch_p3(p.kind, p.cg);
}

// --------------------------------------------------------------- planes
template <typename T>
__global__ void __launch_bounds__(256) planes_kernel(PlanesJob j0, PlanesJob j1) {
    grid_dep_sync();
    if ((int)blockIdx.x < j0.blocks) planes_part<T>(j0, blockIdx.x);
    else planes_part<T>(j1, blockIdx.x - j0.blocks);
}

}  // namespace

// The tile, shares and pairing with the least estimated time.  Both sides of each choice, in
// us: tiles of a pair of CTAs (cg 2), 4096 x 4096 -> 8192 in bf16, 168 and 193 without; shares in
// clusters, 128 x 9216 -> 4096 in fp32, 56 and 121; shares kept apart, the logits of 128 x 4096 ->
// 1000, 20 and 25 (with the pass over their rows); a block's sum left in its accumulator
// (launch_gemm: stay), backward of 128 x 4096 -> 4096, 70 and 72; two products in a launch
// (gemm_together), backward of 3001 x 2048 -> 5003 in bf16, 114 and 141.
static GemmPlan plan_gemm_anew(int planes, int kind, int m, int n, int k, int max_groups, int sms) {
    GemmPlan best;
    const bool gen = planes == GEMM_F32;
    const int P = gen ? 3 : planes, bk = gemm_block_k(planes), kblocks = std::max(1, cdiv(k, bk));
    static const int tiles[5] = {16, 32, 64, 128, 256};
    const int mmas = (P == 1 ? 1 : P == 2 ? 3 : 6) * bk / 16;
    const bool whole = kind == GEMM_STATS || kind == GEMM_DLOGITS;  // (no shares)
    for (int cg = 1; cg <= (gen ? 1 : 2); ++cg) {
        for (int bn : tiles) {
            if (gen && bn > 128) continue;
            if (cg == 2 && bn != 256) continue;
            if (planes == 3 && cg == 1 && bn > 128) continue;  // (stages: launch_gemm)
            if (kind == GEMM_SYM && bn % (kMT * cg)) continue;
            if (bn > 16 && kind != GEMM_SYM && bn >= 2 * n) continue;
            const int mt = cdiv(m, kMT * cg), nt = cdiv(n, bn);
            const long long units = tiles_of(kind, mt, nt, bn / (kMT * cg));
            // Clocks of a block of terms: its MMAs, its bytes (TMA 50 bytes per clock and SM;
            // GEN: fp32 at the memory's rate when all SMs read, and 975 of 888 as measured),
            // or what goes through shared memory (128 bytes per clock: written once, read per
            // MMA).
            const double mma = mmas * (bn / 2 + 10.0), bytes = P * (kMT + bn / cg) * bk * 2.0;
            double per = std::max({mma, bytes / 50.0, (bytes + mmas * (kMT + bn / cg) * 32.0) / 128.0});
            if (gen) per = std::max({mma * 1.1, kMT * bk * 4 / 21.0, bn * 192.0 / 40.0, 600.0});
            // (three planes: a tile's sums go through registers, where they have no accumulator
            // for each block; with one, the next tile's come meanwhile)
            if (planes == 3 && kblocks == 2 && bn > 128) per += 1500.0;
            // (and of a tile: first loads, last sums, epilogue)
            const double tail = 4500.0 + bn * (kind == GEMM_OUT ? 16.0 : 24.0);
            for (int cl = 1; cl <= 8; cl *= 2) {
                if (cl > 1 && (cg > 1 || whole || cl > kblocks)) break;
                const int kps = cdiv(kblocks, cl);
                if (cdiv(kblocks, kps) != cl) continue;
                // (clusters do not span GPCs: fewer of eight CTAs than SMs / 8 are resident)
                const int slots =
                    cl == 1 ? sms / cg : std::max(1, cluster_capacity(gemm_kernel_address(), 384, cl, kSmemMax));
                const double waves = (double)((units + slots - 1) / slots);
                // (shares meet: two barriers of the cluster, bn / cl columns read from each)
                const double meet = cl > 1 ? 2500.0 + bn * 10.0 : 0.0;
                // (a cluster has one tile: nothing of the next runs during its epilogue)
                const double more = cl > 1 ? tail + meet : 1000.0;
                const double score = waves * kps * per + tail + meet + (waves - 1) * more;
                if (best.bn && score >= best.score) continue;
                best.planes = planes;
                best.kind = kind;
                best.cg = cg;
                best.bn = bn;
                best.splits = cl;
                best.groups = 1;
                best.kb_per_split = kps;
                best.score = score;
                best.n_tiles = nt;
            }
            for (int gr = 2; gr <= std::min(max_groups, kblocks) && cg == 1; ++gr) {
                const int kps = cdiv(kblocks, gr);
                if (cdiv(kblocks, kps) != gr) continue;
                // (the sums of the others, written and read back through the L2)
                const double waves = (double)((units * gr + sms - 1) / sms);
                const double score = waves * (kps * per + 1000.0) + tail + (gr - 1) * (double)m * n * 8.0 / 3500.0;
                if (score >= best.score) continue;
                best.planes = planes;
                best.kind = kind;
                best.cg = cg;
                best.bn = bn;
                best.splits = 1;
                best.groups = gr;
                best.kb_per_split = kps;
                best.score = score;
                best.n_tiles = nt;
            }
        }
    }
    return best;
}

GemmPlan plan_gemm(int planes, int kind, int m, int n, int k, int max_groups) {
    // (a plan takes some 5 us of host time, a small call has a few)
    static std::mutex mu;
    static std::map<std::array<int, 7>, GemmPlan> cache;
    const int sms = num_sms();
    const std::array<int, 7> key = {planes, kind, m, n, k, max_groups, sms};
    {
        std::lock_guard<std::mutex> g(mu);
        const auto it = cache.find(key);
        if (it != cache.end()) return it->second;
    }
    const GemmPlan p = plan_gemm_anew(planes, kind, m, n, k, max_groups, sms);
    std::lock_guard<std::mutex> g(mu);
    if (cache.size() >= 256) cache.clear();
    cache.emplace(key, p);
    return p;
}

bool gemm_together(const GemmPlan &a, int m_a, int n_a, int k_a, const GemmPlan &b, int m_b, int n_b, int k_b) {
    if (a.planes != b.planes || a.kind != b.kind || a.cg != b.cg || a.bn != b.bn || a.splits > 1 || b.splits > 1)
        return false;
    const int slots = num_sms() / a.cg;
    const long long ta = (long long)cdiv(m_a, kMT * a.cg) * cdiv(n_a, a.bn),
                    tb = (long long)cdiv(m_b, kMT * a.cg) * cdiv(n_b, a.bn);
    if (ta + tb > 64ll * slots) return false;  // (little is idle in the end)
    const long long ka = k_a + 128, kb = k_b + 128;  // (with a tile's own costs, in terms)
    const long long apart = cdiv((int)std::min<long long>(ta, 1 << 30), slots) * ka +
                            cdiv((int)std::min<long long>(tb, 1 << 30), slots) * kb;
    // the longest of the slots (tiles as unit_at deals them out)
    long long most = 0;
    const long long all = ta + tb;
    for (int i = 0; i < slots; ++i) {
        long long sum = 0;
        for (long long r = 0;; ++r) {
            const long long u = r * slots + (r == 1 ? slots - 1 - i : i);
            if (u >= all) break;
            sum += u < ta ? ka : kb;
        }
        most = std::max(most, sum);
    }
    return most < apart;
}

qcnn_status launch_gemm(const GemmPlan &plan, const GemmProblem *ps, int count, cudaStream_t st) {
    if (count > 1 && plan.splits * plan.groups > 1) return QCNN_ERR_UNSUPPORTED;
    const bool gen = plan.planes == GEMM_F32;
    const int P = gen ? 3 : plan.planes, cg = plan.cg, bnc = plan.bn / cg;
    GemmArgs g = {};
    g.stay = 1;
    unsigned a_bytes = 0, b_bytes = 0;
    for (int i = 0; i < count; ++i) {
        const GemmProblem &s = ps[i];
        ProblemArgs &p = g.p[i];
        qcnn_status rc = set_operand(s.b, P, gen, bnc, s.n, s.k, &p.b, &p.map_b);
        if (rc != QCNN_OK) return rc;
        if (gen) {
            p.a.mn = s.a.mn;
            p.a.src = static_cast<const float *>(s.a.p);
            p.a.ld = s.a.ld;
            if ((rc = set_raw(s.a, s.m, s.k, &g)) != QCNN_OK) return rc;
        } else if ((rc = set_operand(s.a, P, gen, kMT, s.m, s.k, &p.a, &p.map_a)) != QCNN_OK) {
            return rc;
        }
        a_bytes = std::max(a_bytes, p.a.bytes);
        b_bytes = std::max(b_bytes, p.b.bytes);
        // (A in TMEM has its terms along the columns, however it lay in memory)
        p.idesc = (1u << 4) | (1u << 7) | (1u << 10) | (s.a.mn && !gen ? 1u << 15 : 0) |
                  (s.b.mn ? 1u << 16 : 0) | (uint32_t)(plan.bn >> 3) << 17 | (uint32_t)(kMT * cg >> 4) << 24;
        p.m = s.m;
        p.n = s.n;
        p.k = s.k;
        p.kblocks = std::max(1, cdiv(s.k, gemm_block_k(plan.planes)));
        p.m_tiles = cdiv(s.m, kMT * cg);
        p.n_tiles = cdiv(s.n, plan.bn);
        p.kb_per_split = plan.splits > 1 || plan.groups > 1 ? plan.kb_per_split : p.kblocks;
        p.group = std::max(1, 16 / cg);
        p.e = s.e;
        p.e.pair = (pairs(s.e.out, s.e.out_type, s.e.ldo, s.m) ? 1 : 0) |
                   (pairs(s.e.pre, s.e.out_type, s.e.ldp, s.m) ? 2 : 0) |
                   (pairs(s.e.add, s.e.add_type, s.e.lda, s.m) ? 4 : 0);
        // (a plan for another k: a share without terms would never have its sum)
        const int shares = plan.splits * plan.groups;
        if ((shares - 1) * (long long)p.kb_per_split >= p.kblocks || shares * (long long)p.kb_per_split < p.kblocks)
            return QCNN_ERR_UNSUPPORTED;
        const long long tiles = tiles_of(plan.kind, p.m_tiles, p.n_tiles, plan.bn / (kMT * cg));
        if (tiles * plan.groups > (1 << 27)) return QCNN_ERR_UNSUPPORTED;
        p.units = (int)tiles;  // (of a group)
        g.units += p.units * plan.groups;
        if (p.kb_per_split > (!gen && plan.bn <= 128 ? 2 : 1)) g.stay = 0;
    }
    g.count = count;
    g.cl = plan.splits;
    g.groups = plan.groups;
    g.bn = plan.bn;
    g.b_off = a_bytes;  // (multiples of 1024: 128 rows; 64 rows of 128 bytes)
    g.stage = (unsigned)align_up(a_bytes + b_bytes, 1024);
    g.S = (int)std::min<size_t>(gen ? kGenStages : kStagesMax, (kSmemMax - 1024) / g.stage);
    if (gen) {  // raw copies: by TMA as many stages as there is room for
        g.raw = (int)std::min<size_t>(kRawMax, (kSmemMax - 1024 - g.S * (size_t)g.stage) / g.raw_bytes) & ~1;
        if (g.p[0].a.way == RAW_WORDS) g.raw = 2 * kRawSlots;
    }
    const size_t raw = g.raw * (size_t)g.raw_bytes;
    // (three planes: two rings, each with room for a block's planes)
    if (P == 3) g.S &= ~1;
    if (g.S < (gen ? 2 : P == 3 ? 6 : P)) return QCNN_ERR_UNSUPPORTED;
    const size_t smem = std::max(kSmemLeast, g.S * (size_t)g.stage + raw + 1024);
    const int ctas = g.cl > 1 ? g.units * g.cl : std::min(g.units, num_sms() / cg) * cg;
    return launcher(plan)(&g, ctas, smem, st);
}

PlanesJob planes_job(const void *src, int bf16, long long rows, int cols, long long ld, int planes, void *dst,
                     void *kept, const long long *classes, int Ct) {
    PlanesJob j;
    j.src = src;
    j.per_row = cdiv(cols, kPieceCols);
    j.all = rows * j.per_row;
    j.cols = cols;
    j.ld = ld;
    j.planes = planes;
    j.dst = static_cast<unsigned short *>(dst);
    j.kept = static_cast<unsigned short *>(kept);
    j.plane = rows * pad8(cols);
    j.classes = classes;
    j.Ct = Ct;
    j.vec = reinterpret_cast<uintptr_t>(src) % 16 == 0 && ld % (bf16 ? 8 : 4) == 0;
    j.blocks = (int)std::min<long long>((j.all + 7) / 8, (long long)num_sms() * 8);
    return j;
}
qcnn_status launch_planes(const PlanesJob &a, const PlanesJob &b, int bf16, cudaStream_t st) {
    const dim3 grid(a.blocks + b.blocks);
    if (!grid.x) return QCNN_OK;
    return launch_pdl(bf16 ? planes_kernel<unsigned short> : planes_kernel<float>, grid, dim3(256), 0, st, a, b);
}

}  // namespace qcnn
