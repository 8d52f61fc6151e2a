// Attention weight of a chunk's queries on every row of a cache:
//   mass[g][r] = decay * mass[g][r] + sum over tokens i that see row r and query heads h of KV head g of exp(s_ihr - lse_ih),
// s_ihr = scale * q_ih . k_gr, capped and biased as in a scored step, lse the softmax denominators that the step left.  (The paper prunes
// by attention weight in its Discussion and gives no scheme; this is the quantity that such schemes add up.)  It is the
// attention without its values: no running maximum, because the denominators are known, and sums over queries, not over keys.
//
// bf16 rows run on the tensor cores.  A tile is S^T = K Q^T, 128 keys of one KV head by up to 128 query rows (whole tokens of its G
// query heads), so that a thread has one key's row of tensor memory and the sum over queries is its own: what would be a reduction
// over lanes in the attention kernels costs nothing here.  An item is two key tiles, which stay in shared memory while the query
// tiles come by (L2 holds them); where the chunk is one query tile that one stays and the keys stream.
// What a tile of 128 x 128 needs: one exponential per score, 1024 cycles of the special-function unit, of which a quarter goes through the
// multiply-add pipe (not under a cap); shared memory (the MMAs' operands 512 cycles, half a query tile coming in 128, the columns'
// denominators 64).  None of these is full: 2048 tokens of 28 / 4 heads on 16 K rows keep the special-function pipe busy 66 % and the
// multiply-add pipe 50 % of the time, capped weights of 256 tokens on 31 K rows 60 % and 45 % of the cycles that an SM has work.  A
// decoded token is bound by the K plane's bytes.
#include <cstddef>
#include <type_traits>

#include "kvfold_internal.h"
#include "sm100_ptx.cuh"
#include "scores.cuh"

namespace kvf {
namespace {

// ---- tensor cores
constexpr int kTile = 128, kUnit = 2 * kTile;      // keys of a tile, of an item
constexpr uint32_t kPanel = 128 * 128, kTileBytes = 2 * kPanel;
constexpr int kGroups = 4;                     // groups of four warps of exponentials (a warp has a quarter of the lanes)
constexpr int kTcThreads = 128 + kGroups * 128;        // warp 0 TMA, warp 1 MMA, warps 2 and 3 what is to be known of the columns, the others exponentials
constexpr int kSlots = 6;                      // tiles in shared memory: many query tiles: four K slots, two Q slots; one: five and one
constexpr uint32_t kTmemCols = 512;            // two sets of two accumulators of 128 columns
constexpr int kColSlots = 8;
struct __align__(16) Cols {                    // what the exponentials need to know of a job's columns (query rows)
    float neg[kTile];                          // -lse * log2(e) (-inf: no such row, or it saw nothing)
    float2 bias[kTile];                        // slope in log2 units, distance of the item's first key; filled under slopes
    uint32_t seen[kTile];                      // keys of the item that it sees, [low half, high half); filled where some may not be
    int some, part;                            // does any column see a key of the item; may one not see all of them
    int pad[2];
};
enum { M_KFULL = 0, M_KEMPTY = M_KFULL + 5, M_QFULL = M_KEMPTY + 5, M_QEMPTY = M_QFULL + 4, M_DFULL = M_QEMPTY + 4, M_DEMPTY = M_DFULL + 2,
       M_SUM = M_DEMPTY + 2, M_TAKEN = M_SUM + 4, M_DRAIN = M_TAKEN + 4, M_CFULL, M_CEMPTY = M_CFULL + kColSlots, M_COUNT = M_CEMPTY + kColSlots };
struct MassCtl {
    unsigned long long bars[M_COUNT];
    uint32_t tmem_base;
    int abort;
    float sums[kGroups - 1][kUnit];            // the other groups' sums on their way to the first
};
constexpr uint32_t kOffCols = kSlots * kTileBytes;
constexpr uint32_t kOffMassCtl = kOffCols + (kColSlots * sizeof(Cols) + 1023) / 1024 * 1024;
constexpr uint32_t kMassSmem = kOffMassCtl + 4096 + 1024;
static_assert(sizeof(MassCtl) <= 4096 && kMassSmem <= 232448, "shared memory budget of one CTA");

__device__ __forceinline__ uint64_t desc_kmajor(uint32_t addr) {
    return (uint64_t)((addr >> 4) & 0x3FFFu) | ((uint64_t)1 << 16) | ((uint64_t)(1024 >> 4) << 32) | ((uint64_t)1 << 46) | ((uint64_t)2 << 61);
}
__device__ __forceinline__ void lds128(uint32_t at, float (&x)[4]) {
    asm volatile("ld.shared.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(x[0]), "=f"(x[1]), "=f"(x[2]), "=f"(x[3]) : "r"(at));
}

// 2^x of a pair of numbers without the special-function unit: x = i + f, |f| <= 1/2, 2^f = 1 + f c1 + ... + f^5 c5 (least relative
// error, 9e-8, by Lawson's reweighting; in fp32 1.6e-7, as good as ex2.approx), i added to the exponent.  Below 2^-126 off by less than
// 2^-126, from 2^128 on infinite; NaN counts as -inf.
__device__ __forceinline__ float2 exp2_fma(float2 x) {
    x.x = fminf(fmaxf(x.x, -127.f), 128.f);
    x.y = fminf(fmaxf(x.y, -127.f), 128.f);
    const float2 magic = both(12582912.f);                         // 1.5 * 2^23: the sum's low bits are the nearest whole number
    const float2 t = __fadd2_rn(x, magic);
    const float2 f = __fadd2_rn(x, __ffma2_rn(t, both(-1.f), magic));
    float2 y = __ffma2_rn(f, both(0.0013264727123542784f), both(0.009671512644823185f));
    y = __ffma2_rn(f, y, both(0.0555073374349718f));
    y = __ffma2_rn(f, y, both(0.24022242085262321f));
    y = __ffma2_rn(f, y, both(0.6931469775989922f));
    y = __ffma2_rn(f, y, both(1.f));
    return make_float2(__int_as_float(__float_as_int(y.x) + (__float_as_int(t.x) << 23)), __int_as_float(__float_as_int(y.y) + (__float_as_int(t.y) << 23)));
}

// What the roles have to agree on.  Item = (KV head, 256 keys, split of the query tiles); its jobs are query tiles [q0, q1).
struct MassWork {
    int nkt, nku, nq, toks, splits, one;       // key tiles and items' worth of keys of a KV head, query tiles, tokens of a query tile
    int64_t items;                             // (below 2^31)
    __device__ __forceinline__ void item(const MassArgs &a, int64_t i, int &kvh, int &ku, int &split, int &q0, int &q1) const {
        const uint32_t u = (uint32_t)i / (uint32_t)splits;
        split = (int)((uint32_t)i - u * (uint32_t)splits);
        kvh = (int)(u / (uint32_t)nku);
        ku = (int)u - kvh * nku;
        // (without ranges, tokens whose row lies below the item's keys see none of them)
        const int64_t ahead = (int64_t)ku * kUnit - (a.rows - a.n);
        int from = 0;
        if (a.self_rows && !(a.scored && (a.mods.first || a.mods.end)) && ahead > 0) from = (int)(ahead / toks);
        q0 = from + (int)((int64_t)split * (nq - from) / splits);
        q1 = from + (int)((int64_t)(split + 1) * (nq - from) / splits);
    }
};

// kOne: the chunk is one query tile of `ncols` columns (a multiple of 16).  kCap: scores are capped.
template <bool kOne, bool kCap>
__global__ void __launch_bounds__(kTcThreads, 1)
mass_tc_kernel(const MassArgs a, const MassWork w, const int ncols, const __grid_constant__ CUtensorMap map_q, const __grid_constant__ CUtensorMap map_k) {
    constexpr int SK = kOne ? 5 : 4, SQ = kOne ? 1 : 2;
    // Two groups share a job and the two pairs of groups take the jobs in turn, so that one pair's exponentials run while the other waits for
    // its scores (all four on each job: 289 us instead of 271).  Many query tiles: a group has half of the job's columns for both key
    // tiles (a thread has two keys, and what it reads of a column serves both).  One: all columns for one key tile.
    constexpr int kTurns = 2, kWarpsOfJob = 16 / kTurns;
    extern __shared__ uint8_t smem_raw[];
    const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
    uint8_t *smem = smem_raw + (base - smem_u32(smem_raw));
    MassCtl *ctl = reinterpret_cast<MassCtl *>(smem + kOffMassCtl);
    auto bar = [&](int i) { return base + kOffMassCtl + 8u * (uint32_t)i; };
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int64_t L = a.rows, P = L - (int64_t)a.n * a.self_rows;
    const int G = a.G;
    // items of this CTA: a contiguous range of them (kOne: the K rows of one stretch), else every gridDim-th
    const int64_t i0 = kOne ? blockIdx.x * w.items / gridDim.x : blockIdx.x, i1 = kOne ? (blockIdx.x + 1) * w.items / gridDim.x : w.items;
    const int64_t istep = kOne ? 1 : gridDim.x;

    if (threadIdx.x == 0) {
        for (int s = 0; s < SK; ++s) { mbar_init(bar(M_KFULL + s), 1); mbar_init(bar(M_KEMPTY + s), 1); }
        for (int s = 0; s < SQ; ++s) { mbar_init(bar(M_QFULL + s), 1); mbar_init(bar(M_QEMPTY + s), 1); }
        for (int s = 0; s < 2; ++s) { mbar_init(bar(M_DFULL + s), 1); mbar_init(bar(M_DEMPTY + s), kWarpsOfJob); }
        for (int s = 0; s < 4; ++s) { mbar_init(bar(M_SUM + s), kGroups - 1); mbar_init(bar(M_TAKEN + s), 1); }
        for (int s = 0; s < kColSlots; ++s) { mbar_init(bar(M_CFULL + s), 1); mbar_init(bar(M_CEMPTY + s), kWarpsOfJob); }
        mbar_init(bar(M_DRAIN), 1);
        ctl->abort = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 1) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&ctl->tmem_base)), "r"(kTmemCols) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    {
        // rows of a query tile behind its last token (G does not divide 128), which no copy fills
        const int from = w.toks * G * 128, bytes = (int)kPanel - from;
        for (int i = threadIdx.x * 16; i < 2 * SQ * bytes; i += kTcThreads * 16)
            *reinterpret_cast<uint4 *>(smem + (uint32_t)SK * kTileBytes + (uint32_t)(i / bytes) * kPanel + from + i % bytes) = make_uint4(0u, 0u, 0u, 0u);
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    }
    pdl_launch_dependents();
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    pdl_wait();          // nothing above reads what an earlier kernel wrote
    const uint32_t tmem = *reinterpret_cast<volatile uint32_t *>(&ctl->tmem_base);
    auto k_slot = [&](int s) { return base + (uint32_t)s * kTileBytes; };
    auto q_slot = [&](int s) { return base + (uint32_t)(SK + s) * kTileBytes; };

    if (warp == 0) {
        if (lane == 0) {
            // ------------------------------------------------------------------ TMA producer
            const uint32_t q_bytes = 2u * (uint32_t)(w.toks * G) * 128u;
            int kc = 0, qc = 0, held = -1;       // tiles loaded so far; kOne: KV head of the query tile held
            bool ok = true;
            for (int64_t i = i0; ok && i < i1; i += istep) {
                int kvh, ku, split, q0, q1;
                w.item(a, i, kvh, ku, split, q0, q1);
                if (q0 >= q1) continue;
                for (int kt = 2 * ku; kt < min(2 * ku + 2, w.nkt); ++kt, ++kc) {
                    ok = mbar_wait(bar(M_KEMPTY + kc % SK), ((kc / SK) & 1) ^ 1, ctl, a.status);
                    if (!ok) break;
                    const uint32_t kb = bar(M_KFULL + kc % SK), kd = k_slot(kc % SK);
                    mbar_expect_tx(kb, kTileBytes);
                    if (a.page_table) {
                        const int page = a.page_table[kt];
                        tma_load_4d(kd, &map_k, kb, 0, 0, kvh, page);
                        tma_load_4d(kd + kPanel, &map_k, kb, 64, 0, kvh, page);
                    } else {
                        tma_load_3d(kd, &map_k, kb, 0, kt * kTile, kvh);
                        tma_load_3d(kd + kPanel, &map_k, kb, 64, kt * kTile, kvh);
                    }
                }
                if (!ok) break;
                for (int q = q0; q < q1; ++q) {
                    if (kOne && held == kvh) break;
                    held = kvh;
                    ok = mbar_wait(bar(M_QEMPTY + qc % SQ), ((qc / SQ) & 1) ^ 1, ctl, a.status);
                    if (!ok) break;
                    const uint32_t qb = bar(M_QFULL + qc % SQ), qd = q_slot(qc % SQ);
                    mbar_expect_tx(qb, q_bytes);
                    tma_load_3d(qd, &map_q, qb, 0, kvh * G, q * w.toks);
                    tma_load_3d(qd + kPanel, &map_q, qb, 64, kvh * G, q * w.toks);
                    ++qc;
                }
            }
            // do not leave while a copy may still be writing into this CTA's shared memory
            for (int c = max(0, kc - SK); c < kc; ++c) mbar_wait_drain(bar(M_KFULL + c % SK), (c / SK) & 1, a.status);
            for (int c = max(0, qc - SQ); c < qc; ++c) mbar_wait_drain(bar(M_QFULL + c % SQ), (c / SQ) & 1, a.status);
        }
    } else if (warp == 1) {
        // ------------------------------------------------------------------ MMA issuer: the warp walks the loop, one thread of it issues
        const bool leader = elect_one();
        const uint32_t idesc = (1u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)(ncols >> 3) << 17) | ((128u >> 4) << 24);
        int kc = 0, qc = 0, jc = 0, held = -1;
        bool ok = true;
        for (int64_t i = i0; ok && i < i1; i += istep) {
            int kvh, ku, split, q0, q1;
            w.item(a, i, kvh, ku, split, q0, q1);
            if (q0 >= q1) continue;
            if (kOne && held >= 0 && held != kvh) {          // the last head's query tile has been read
                if (leader) tc_commit(bar(M_QEMPTY));
                ++qc;
            }
            const int tiles = min(2, w.nkt - 2 * ku);
            for (int q = q0; q < q1; ++q, ++jc) {
                // (what is not there to be waited for is asked for twice)
                const Phase acc = {bar(M_DEMPTY + (jc & 1)), (uint32_t)((jc >> 1) & 1) ^ 1u};
                const Phase k0 = q == q0 ? Phase{bar(M_KFULL + kc % SK), (uint32_t)(kc / SK) & 1u} : acc;
                const Phase k1 = q == q0 && tiles == 2 ? Phase{bar(M_KFULL + (kc + 1) % SK), (uint32_t)((kc + 1) / SK) & 1u} : acc;
                const Phase qt = !kOne || held != kvh ? Phase{bar(M_QFULL + qc % SQ), (uint32_t)(qc / SQ) & 1u} : acc;
                held = kvh;
                const Phase all[4] = {acc, k0, k1, qt};
                ok = mbar_wait4_warp(all, ctl, a.status);
                if (!ok) break;
                tc_fence_after();
                const uint64_t qdesc = desc_kmajor(q_slot(qc % SQ));
#pragma unroll
                for (int t = 0; t < 2; ++t) {
                    if (t >= tiles) break;
                    const uint64_t kdesc = desc_kmajor(k_slot((kc + t) % SK));
                    const uint32_t d = tmem + (uint32_t)(jc & 1) * 256u + (uint32_t)t * 128u;
#pragma unroll
                    for (int kk = 0; kk < 8; ++kk) {
                        const uint64_t off = (uint64_t)(((kk >> 2) * kPanel + (kk & 3) * 32) >> 4);
                        if (leader) tc_mma(d, kdesc + off, qdesc + off, idesc, kk > 0);
                    }
                    if (leader && q == q1 - 1) tc_commit(bar(M_KEMPTY + (kc + t) % SK));
                }
                if (leader) tc_commit(bar(M_DFULL + (jc & 1)));
                if (!kOne) {
                    if (leader) tc_commit(bar(M_QEMPTY + qc % SQ));
                    ++qc;
                }
            }
            kc += tiles;
        }
        // whatever made this warp leave its loop, tensor memory is released only after every MMA it issued has run
        if (leader) {
            tc_commit(bar(M_DRAIN));
            mbar_wait_drain(bar(M_DRAIN), 0, a.status);
        }
    } else if (warp < 4) {
        // ------------------------------------------------------------------ columns of the jobs, up to eight jobs ahead, two warps in turn
        const bool biased = a.scored && a.mods.slopes, ranged = a.scored && (a.mods.first || a.mods.end);
        // my four columns of a query tile: 32 apart, token and head within the group
        int tok_of[4], head_of[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            tok_of[k] = (lane + 32 * k) / G;
            head_of[k] = (lane + 32 * k) % G;
        }
        int jc = 0;
        bool ok = true;
        for (int64_t i = i0; ok && i < i1; i += istep) {
            int kvh, ku, split, q0, q1;
            w.item(a, i, kvh, ku, split, q0, q1);
            const int64_t key0 = (int64_t)ku * kUnit;
            for (int q = q0; q < q1; ++q, ++jc) {
                if ((jc & 1) != warp - 2) continue;
                float l[4];
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const int tok = q * w.toks + tok_of[k];
                    l[k] = tok_of[k] < w.toks && tok < a.n ? a.lse[(int64_t)tok * a.H + kvh * G + head_of[k]] : -INFINITY;
                }
                Cols *cols = reinterpret_cast<Cols *>(smem + kOffCols) + jc % kColSlots;
                ok = mbar_wait(bar(M_CEMPTY + jc % kColSlots), ((jc / kColSlots) & 1) ^ 1, ctl, a.status);
                ok = __all_sync(0xffffffffu, ok);
                if (!ok) break;
#pragma unroll
                for (int k = 0; k < 4; ++k) cols->neg[lane + 32 * k] = l[k] == -INFINITY ? -INFINITY : -l[k] * kLog2e;
                // does every token see all of the keys?  (without ranges known from the tile's first token)
                // (nor where a denominator is NaN: a pair's way through the multiply-add pipe would lose it)
                bool some = true, part = ranged || key0 + kUnit > P + (int64_t)(q * w.toks + 1) * a.self_rows;
                const bool odd = __any_sync(0xffffffffu, l[0] != l[0] || l[1] != l[1] || l[2] != l[2] || l[3] != l[3]);
                part = part || odd;
                if (part || biased) {
                    some = part = false;
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        const int tok = q * w.toks + tok_of[k];
                        uint32_t sees = 0u;
                        float2 bias = both(0.f);
                        if (tok_of[k] < w.toks && tok < a.n) {
                            const RowRange seen = a.scored ? seen_rows(a.mods, tok, tok, P, L, a.self_rows) : RowRange{0, P + (int64_t)(tok + 1) * a.self_rows};
                            const int lo = (int)min(max(seen.begin - key0, (int64_t)0), (int64_t)kUnit), hi = (int)min(max(seen.end - key0, (int64_t)0), (int64_t)kUnit);
                            if (lo < hi) {
                                sees = (uint32_t)lo | (uint32_t)hi << 16;
                                some = true;
                            }
                            part = part || odd || lo > 0 || hi < kUnit;
                            if (biased) bias = make_float2(a.mods.slopes[kvh * G + head_of[k]] * kLog2e, (float)(a.mods.pos0 + tok - key0));
                        }
                        cols->seen[lane + 32 * k] = sees;
                        cols->bias[lane + 32 * k] = bias;
                    }
                    some = __any_sync(0xffffffffu, some);
                    part = __any_sync(0xffffffffu, part);
                }
                if (lane == 0) {
                    cols->some = some;
                    cols->part = part;
                }
                __syncwarp();
                if (lane == 0) mbar_arrive(bar(M_CFULL + jc % kColSlots));
            }
        }
    } else {
        // ------------------------------------------------------------------ exponentials: a thread per key (kOne) or two
        const int group = (warp - 4) >> 2, quarter = warp & 3, r = quarter * 32 + lane;
        constexpr int NK = kOne ? 1 : 2;                 // keys of a thread: r of key tile t0, and of the next
        const int t0 = kOne ? group & 1 : 0, turn = group >> 1;
        const uint32_t t_acc = tmem + ((uint32_t)(quarter * 32) << 16) + (uint32_t)t0 * 128u;
        const bool biased = a.scored && a.mods.slopes;
        const float2 sl2 = both(a.scale_log2);
        int jc = 0, sums = 0;
        bool ok = true;
        for (int64_t i = i0; ok && i < i1; i += istep) {
            int kvh, ku, split, q0, q1;
            w.item(a, i, kvh, ku, split, q0, q1);
            const int64_t key0 = (int64_t)ku * kUnit;
            if (kOne && (jc & 1) != turn) { jc += q1 - q0; continue; }           // (kOne: an item is one job)
            // the weight so far, called for ahead of the work
            const bool last = w.splits == 1 && (kOne || group == 0);
            float before[NK];
#pragma unroll
            for (int t = 0; t < NK; ++t) {
                const int64_t key = key0 + (t0 + t) * kTile + r;
                before[t] = last && a.mass_in && a.decay != 0.f && key < a.held ? a.mass_in[(int64_t)kvh * a.in_stride + key] : 0.f;
            }
            float2 acc[NK][2];
#pragma unroll
            for (int t = 0; t < NK; ++t) acc[t][0] = acc[t][1] = both(0.f);
            for (int q = q0; q < q1; ++q, ++jc) {
                if (!kOne && (jc & 1) != turn) continue;
                const Cols *cols = reinterpret_cast<const Cols *>(smem + kOffCols) + jc % kColSlots;
                const uint32_t col0 = base + kOffCols + (uint32_t)(jc % kColSlots) * (uint32_t)sizeof(Cols);
                const Phase known = {bar(M_CFULL + jc % kColSlots), (uint32_t)(jc / kColSlots) & 1u}, full = {bar(M_DFULL + (jc & 1)), (uint32_t)(jc >> 1) & 1u};
                ok = mbar_wait(known.bar, known.parity, ctl, a.status) && mbar_wait(full.bar, full.parity, ctl, a.status);
                ok = __all_sync(0xffffffffu, ok);
                if (!ok) break;
                const bool some = *reinterpret_cast<const volatile int *>(&cols->some), part = *reinterpret_cast<const volatile int *>(&cols->part);
                tc_fence_after();
                const uint32_t t_job = t_acc + (uint32_t)(jc & 1) * 256u;
                constexpr int C = kOne ? 16 : 32;
                auto given_back = [&]() {            // my part of the accumulators
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(bar(M_DEMPTY + (jc & 1)));
                };
                const int from = kOne ? 0 : (group & 1) * (kTile / 2), to = kOne ? ncols : from + kTile / 2;
                if (some && (part || biased)) {
                    // (a way of its own, behind the branch of a whole job: beside the other it cost that 60 us of 340 in a launch whose jobs
                    // hardly ever take it)
#pragma unroll 1
                    for (int c0 = from; c0 < to; c0 += C)
#pragma unroll
                        for (int t = 0; t < NK; ++t) {
                            uint32_t v[C];
                            __syncwarp();
                            if constexpr (kOne) KVF_TMEM_LD16(v, 0, t_job + t * 128 + c0);
                            else KVF_TMEM_LD32(v, 0, t_job + t * 128 + c0);
                            tmem_wait_ld();
                            const int at = (t0 + t) * kTile + r;
#pragma unroll
                            for (int c = 0; c < C; ++c) {
                                const float s = __uint_as_float(v[c]);
                                const volatile Cols *col = cols;
                                float y = (kCap ? cap_any(a.mods, s) : s * sl2.x) + col->neg[c0 + c];
                                if (biased) y = fmaf(-col->bias[c0 + c].x, fabsf(col->bias[c0 + c].y - (float)at), y);
                                const uint32_t sees = col->seen[c0 + c];
                                acc[t][0].x += at >= (int)(sees & 0xFFFFu) && at < (int)(sees >> 16) ? ex2(y) : 0.f;
                            }
                        }
                } else if (some) {
#pragma unroll 1
                    for (int c0 = from; c0 < to; c0 += C) {
                        uint32_t v[NK][C];
                        __syncwarp();
#pragma unroll
                        for (int t = 0; t < NK; ++t) {
                            if constexpr (kOne) KVF_TMEM_LD16(v[t], 0, t_job + t * 128 + c0);
                            else KVF_TMEM_LD32(v[t], 0, t_job + t * 128 + c0);
                        }
                        tmem_wait_ld();
                        // (many query tiles: all that is left of the job is in registers now)
                        if (!kOne && c0 + C == to) given_back();
                        auto dot = [&](int t, int c) { return make_float2(__uint_as_float(v[t][c]), __uint_as_float(v[t][c + 1])); };
                        // (every fourth pair of exponentials goes through the multiply-add pipe, 286 -> 271 us; not under a cap, whose
                        // polynomials fill that pipe, 138 against 126)
                        auto sum_up = [&](auto exponent) {
#pragma unroll
                            for (int c = 0; c < C; c += 4) {
                                float n4[4];
                                lds128(col0 + (uint32_t)(c0 + c) * 4u, n4);
#pragma unroll
                                for (int t = 0; t < NK; ++t) {
                                    const float2 y0 = exponent(t, c, make_float2(n4[0], n4[1])), y1 = exponent(t, c + 2, make_float2(n4[2], n4[3]));
                                    acc[t][0] = __fadd2_rn(acc[t][0], make_float2(ex2(y0.x), ex2(y0.y)));
                                    acc[t][1] = __fadd2_rn(acc[t][1], !kCap && (c & 4) ? exp2_fma(y1) : make_float2(ex2(y1.x), ex2(y1.y)));
                                }
                            }
                        };
                        if constexpr (kCap) {
                            float far = 0.f;
#pragma unroll
                            for (int t = 0; t < NK; ++t)
#pragma unroll
                                for (int c = 0; c < C; ++c) far = fmaxf(far, fabsf(__uint_as_float(v[t][c])));
                            if (!__any_sync(0xffffffffu, far > a.mods.small_to)) {
                                sum_up([&](int t, int c, float2 n2) { return __ffma2_rn(dot(t, c), cap_small_over(a.mods, dot(t, c)), n2); });
                            } else {
                                const bool middle = !__any_sync(0xffffffffu, far > a.mods.middle_to);
#pragma unroll
                                for (int t = 0; t < NK; ++t)
#pragma unroll
                                    for (int c = 0; c < C; c += 2) {
                                        const float2 y = middle ? cap_middle(a.mods, dot(t, c)) : make_float2(cap_far(a.mods, dot(t, c).x * a.mods.cap_in), cap_far(a.mods, dot(t, c).y * a.mods.cap_in));
                                        v[t][c] = __float_as_uint(y.x);
                                        v[t][c + 1] = __float_as_uint(y.y);
                                    }
                                sum_up([&](int t, int c, float2 n2) { return __fadd2_rn(dot(t, c), n2); });
                            }
                        } else {
                            sum_up([&](int t, int c, float2 n2) { return __ffma2_rn(dot(t, c), sl2, n2); });
                        }
                    }
                }
                if (kOne || !some || part || biased) given_back();
                __syncwarp();
                if (lane == 0) mbar_arrive(bar(M_CEMPTY + jc % kColSlots));
            }
            if (!ok) break;
            float sum[NK];
#pragma unroll
            for (int t = 0; t < NK; ++t) {
                const float2 both_acc = __fadd2_rn(acc[t][0], acc[t][1]);
                sum[t] = both_acc.x + both_acc.y;
            }
            if (!kOne) {
                // the other groups' sums of the keys go to the first
                ++sums;
                if (group > 0) {
                    if (sums > 1) ok = mbar_wait(bar(M_TAKEN + quarter), (sums - 2) & 1, ctl, a.status);
                    ok = __all_sync(0xffffffffu, ok);
                    if (!ok) break;
#pragma unroll
                    for (int t = 0; t < NK; ++t) *reinterpret_cast<volatile float *>(&ctl->sums[group - 1][t * kTile + r]) = sum[t];
                    __syncwarp();
                    if (lane == 0) mbar_arrive(bar(M_SUM + quarter));
                    continue;
                }
                ok = mbar_wait(bar(M_SUM + quarter), (sums - 1) & 1, ctl, a.status);
                ok = __all_sync(0xffffffffu, ok);
                if (!ok) break;
#pragma unroll
                for (int t = 0; t < NK; ++t)
#pragma unroll
                    for (int o = 1; o < kGroups; ++o) sum[t] += *reinterpret_cast<volatile float *>(&ctl->sums[o - 1][t * kTile + r]);
                __syncwarp();
                if (lane == 0) mbar_arrive(bar(M_TAKEN + quarter));
            }
#pragma unroll
            for (int t = 0; t < NK; ++t) {
                const int64_t key = key0 + (t0 + t) * kTile + r;
                if (key >= L) continue;
                if (w.splits > 1) a.parts[((int64_t)split * a.Hkv + kvh) * L + key] = sum[t];
                else a.mass_out[(int64_t)kvh * a.out_stride + key] = fmaf(a.decay, before[t], sum[t]);
            }
        }
    }
    tc_fence_before();
    __syncthreads();
    if (warp == 1) {
        tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(kTmemCols) : "memory");
    }
}

// The splits' sums of a key, in order.
__global__ void __launch_bounds__(256) mass_sum_kernel(const MassArgs a, const int splits) {
    const int64_t key = (int64_t)blockIdx.x * 256 + threadIdx.x;
    const int kvh = blockIdx.y;
    pdl_launch_dependents();
    pdl_wait();
    if (key >= a.rows) return;
    float sum = 0.f;
    for (int s = 0; s < splits; ++s) sum += a.parts[((int64_t)s * a.Hkv + kvh) * a.rows + key];
    if (a.mass_in && a.decay != 0.f && key < a.held) sum = fmaf(a.decay, a.mass_in[(int64_t)kvh * a.in_stride + key], sum);
    a.mass_out[(int64_t)kvh * a.out_stride + key] = sum;
}

// ---- CUDA cores (fp32 caches, head_dim 64): 64 keys of one KV head a CTA, the query rows in tiles of 64, as attn_simt.cu has them
constexpr int BM = 64, BN = 64, kThreads = 256;

template <typename T> __device__ __forceinline__ void load16(const T *p, float *dst);
template <> __device__ __forceinline__ void load16<float>(const float *p, float *dst) { *reinterpret_cast<float4 *>(dst) = *reinterpret_cast<const float4 *>(p); }
template <> __device__ __forceinline__ void load16<__nv_bfloat16>(const __nv_bfloat16 *p, float *dst) {
    const uint4 v = *reinterpret_cast<const uint4 *>(p);
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        dst[2 * i] = __uint_as_float(w[i] << 16);
        dst[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
    }
}

template <typename T, int D>
__global__ void __launch_bounds__(kThreads, 2) mass_simt_kernel(const MassArgs a) {
    constexpr int S = D + 4, VEC = 16 / sizeof(T);
    extern __shared__ __align__(16) float smem[];
    float *Qs = smem, *Ks = Qs + BM * S;
    __shared__ float lse2[BM], slope[BM];
    __shared__ int64_t begin[BM], limit[BM];
    const int tid = threadIdx.x, ty = tid >> 4, tx = tid & 15;
    const int kvh = blockIdx.y, G = a.G, n = a.n;
    const int64_t key0 = (int64_t)blockIdx.x * BN, L = a.rows, P = L - (int64_t)n * a.self_rows;
    const T *q = reinterpret_cast<const T *>(a.q_rot);
    const T *K = reinterpret_cast<const T *>(a.k_plane) + (int64_t)kvh * a.capacity * D;
    auto load_row = [&](float *dst, const T *src, int c, bool there) {
        if (there) {
            load16<T>(src + c * VEC, dst + c * VEC);
        } else {
#pragma unroll
            for (int e = 0; e < VEC; ++e) dst[c * VEC + e] = 0.f;
        }
    };
    pdl_wait();
    for (int idx = tid; idx < BN * (D / VEC); idx += kThreads) {
        const int r = idx / (D / VEC), c = idx % (D / VEC);
        load_row(Ks + r * S, K + (key0 + r) * D, c, key0 + r < L);
    }
    float acc[4] = {0.f, 0.f, 0.f, 0.f};
    for (int row0 = 0; row0 < n * G; row0 += BM) {
        __syncthreads();
        for (int idx = tid; idx < BM * (D / VEC); idx += kThreads) {
            const int r = idx / (D / VEC), c = idx % (D / VEC), R = row0 + r, tok = R / G;
            load_row(Qs + r * S, q + ((int64_t)tok * a.H + kvh * G + R % G) * D, c, tok < n);
        }
        if (tid < BM) {
            const int R = row0 + tid, tok = R / G;
            // (a row without a token, or one that saw nothing, gives nothing: 2^-inf)
            lse2[tid] = INFINITY;
            begin[tid] = limit[tid] = 0;
            slope[tid] = 0.f;
            if (tok < n) {
                const float l = a.lse[(int64_t)tok * a.H + kvh * G + R % G];
                lse2[tid] = l == -INFINITY ? INFINITY : l * kLog2e;
                const RowRange seen = a.scored ? seen_rows(a.mods, tok, tok, P, L, a.self_rows) : RowRange{0, P + (int64_t)(tok + 1) * a.self_rows};
                begin[tid] = seen.begin;
                limit[tid] = seen.end;
                if (a.scored && a.mods.slopes) slope[tid] = a.mods.slopes[kvh * G + R % G] * kLog2e;
            }
        }
        __syncthreads();
        float s[4][4];
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) s[i][j] = 0.f;
#pragma unroll 4
        for (int k4 = 0; k4 < D / 4; ++k4) {
            float4 qa[4], kb[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) qa[i] = *reinterpret_cast<const float4 *>(Qs + (4 * ty + i) * S + k4 * 4);
#pragma unroll
            for (int j = 0; j < 4; ++j) kb[j] = *reinterpret_cast<const float4 *>(Ks + (tx + 16 * j) * S + k4 * 4);
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    s[i][j] = fmaf(qa[i].x, kb[j].x, s[i][j]);
                    s[i][j] = fmaf(qa[i].y, kb[j].y, s[i][j]);
                    s[i][j] = fmaf(qa[i].z, kb[j].z, s[i][j]);
                    s[i][j] = fmaf(qa[i].w, kb[j].w, s[i][j]);
                }
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int r = 4 * ty + i, tok = (row0 + r) / G;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int64_t key = key0 + tx + 16 * j;
                float x = s[i][j] * a.scale_log2;
                if (a.scored) {
                    if (a.mods.cap_out > 0.f) x = a.mods.cap_out * tanhf(s[i][j] * a.mods.cap_in);
                    const int64_t at = a.mods.pos0 + tok - key;
                    if (a.mods.slopes) x = fmaf(-slope[r], (float)(at < 0 ? -at : at), x);
                }
                if (key >= begin[r] && key < limit[r]) acc[j] += exp2f(x - lse2[r]);
            }
        }
    }
    // the sixteen threads of a key, in order
    __syncthreads();
#pragma unroll
    for (int j = 0; j < 4; ++j) Qs[ty * BN + tx + 16 * j] = acc[j];
    __syncthreads();
    if (tid < BN && key0 + tid < L) {
        const int64_t key = key0 + tid;
        float sum = 0.f;
#pragma unroll
        for (int t = 0; t < 16; ++t) sum += Qs[t * BN + tid];
        if (a.mass_in && a.decay != 0.f && key < a.held) sum = fmaf(a.decay, a.mass_in[(int64_t)kvh * a.in_stride + key], sum);
        a.mass_out[(int64_t)kvh * a.out_stride + key] = sum;
    }
}

template <typename T, int D>
cudaError_t launch_simt_t(const MassArgs &a, cudaStream_t s) {
    constexpr int smem = (int)sizeof(float) * (BM + BN) * (D + 4);
    static_assert(BM * (D + 4) >= 16 * BN, "the sums of a key reuse the query tile");
    cudaError_t e = raise_smem_limit_once(reinterpret_cast<const void *>(mass_simt_kernel<T, D>), smem);
    if (e != cudaSuccess) return e;
    return launch_pdl(mass_simt_kernel<T, D>, dim3((unsigned)((a.rows + BN - 1) / BN), a.Hkv), dim3(kThreads), smem, s, a);
}

}  // namespace

int mass_tile_tokens(int G) { return kTile / G; }

cudaError_t launch_mass_tc(const MassArgs &a, const CUtensorMap &map_q, const CUtensorMap &map_k, cudaStream_t s, int *launched) {
    *launched = 0;
    MassWork w;
    w.toks = mass_tile_tokens(a.G);
    w.nkt = (int)((a.rows + kTile - 1) / kTile);
    w.nku = (w.nkt + 1) / 2;
    w.nq = (a.n + w.toks - 1) / w.toks;
    w.one = w.nq == 1;
    const int64_t units = (int64_t)a.Hkv * w.nku;
    // Splits of the query tiles: as many as fill the waves of CTAs best (a tile for what an item costs besides)
    w.splits = 1;
    double least = 0.0;
    for (int sp = 1; sp <= w.nq && sp <= 16 && (int64_t)sp * a.Hkv * a.rows <= a.parts_cap; ++sp) {
        const double waves = (double)((units * sp + a.sms - 1) / a.sms), t = waves * ((double)w.nq / sp + 1.0) + (sp > 1 ? 2.0 : 0.0);
        if (sp == 1 || t < least) { least = t; w.splits = sp; }
    }
    w.items = units * w.splits;
    if (w.items >= (int64_t)1 << 31) return cudaErrorInvalidValue;          // (2^24 tiles of 128 rows for each of 16 heads, and beyond)
    const int ncols = w.one ? (a.n * a.G + 15) / 16 * 16 : kTile;
    const bool cap = a.scored && a.mods.cap_out > 0.f;
    auto kernel = w.one ? (cap ? mass_tc_kernel<true, true> : mass_tc_kernel<true, false>) : cap ? mass_tc_kernel<false, true> : mass_tc_kernel<false, false>;
    cudaError_t e = raise_smem_limit_once(reinterpret_cast<const void *>(kernel), (int)kMassSmem);
    if (e != cudaSuccess) return e;
    const int64_t ctas = w.items < a.sms ? w.items : a.sms;
    e = launch_pdl(kernel, dim3((unsigned)ctas), dim3(kTcThreads), kMassSmem, s, a, w, ncols, map_q, map_k);
    if (e != cudaSuccess) return e;
    *launched = 1;
    if (w.splits == 1) return e;
    e = launch_pdl(mass_sum_kernel, dim3((unsigned)((a.rows + 255) / 256), a.Hkv), dim3(256), 0, s, a, w.splits);
    if (e == cudaSuccess) *launched = 2;
    return e;
}

cudaError_t launch_mass_simt(const MassArgs &a, int dtype, cudaStream_t s, int *launched) {
    cudaError_t e;
    if (dtype == 0) e = a.d == 128 ? launch_simt_t<__nv_bfloat16, 128>(a, s) : launch_simt_t<__nv_bfloat16, 64>(a, s);
    else e = a.d == 128 ? launch_simt_t<float, 128>(a, s) : launch_simt_t<float, 64>(a, s);
    *launched = e == cudaSuccess;
    return e;
}

}  // namespace kvf
