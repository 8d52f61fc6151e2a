// Eviction: the rows of a cache that count most, moved in order into another one.
//
// The paper's Discussion perturbs a folded cache by attention-based pruning (an information-removing perturbation; no scheme is given).
// Here, for each KV head on its own, the first n_sink rows and the last n_recent stay, and of the m rows between them the `want` with the
// most accumulated attention weight (kvf_cache_mass); of rows with the same weight the lower ones.  Order is kept, so that "first" and
// "last" mean the same in the smaller cache.
//
// Select.  A weight is mapped to a 32-bit key that sorts as the weight does (NaN below everything, -0 as +0).  The want-th largest key is
// found by radix, eight bits at a time from the top: a histogram of the keys that agree with what is known so far, until all that are
// left in the bin are wanted.  A cluster of eight CTAs has one KV head (a CTA on its own, up to 4096 candidates): each takes an equal
// range of rows and each thread a piece of it, whose keys it keeps in registers (17 at most; in shared memory up to 51 200 of a
// CTA, else the weights are read again for each histogram); the histograms of all are added up through distributed shared memory.
// Then rows above the key, and as many of those equal to it as are wanted, from the lowest up, are counted thread by
// thread and written in order.  Counts are whole numbers, so that the order of the atomics changes nothing.
// What bounds it is latency: a sweep of the keys, a cluster barrier (1500 cycles), a look at eight histograms (1000) and a scan for every
// eight bits.  (Three histograms over 11, 11 and 10 bits: 64 KB from the peers at ~20 bytes a cycle each; numbering by ballots and
// the weights written here took half of the 26 us.)
//
// Move.  Rows are copied 16 bytes a thread, K and V rows of a KV head in one launch, eight loads in flight a thread; bound by memory
// (two reads and two writes of every row kept).
#include "kvfold_internal.h"
#include "sm100_ptx.cuh"

namespace kvf {
namespace {

constexpr int kBins = 256, kPasses = 4;
constexpr int kWide = 1024, kNarrow = 512;           // threads of a CTA of a cluster, of one on its own
constexpr int kOwn = 17;                             // keys that a thread keeps in registers, odd
constexpr int kHeldKeys = 51200;                     // keys of a CTA's range in shared memory
constexpr int64_t kOneCta = 8 * kNarrow;             // candidates up to which a KV head gets one CTA, not eight

struct SelectShared {
    uint32_t hist[kPasses][kBins];
    uint32_t scan[32];
    uint32_t found_bin, found_above, found_count;    // bin that the wanted key lies in, keys in the bins above it, in it
    uint32_t counts[2];                              // of this CTA's range: keys above the wanted key, keys equal to it
    uint32_t before[2];                              // of the ranges before it
};

__device__ __forceinline__ uint32_t key_of(float w) {
    if (w != w) return 0u;
    const uint32_t b = __float_as_uint(w + 0.f);     // (-0 + 0 = 0)
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}

// (No "memory": loads of one and the same phase may be in flight together.  What separates the phases is volatile too.)
__device__ __forceinline__ uint32_t peer_u32(const uint32_t *p, uint32_t rank) {
    uint32_t v;
    asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(v) : "r"(peer_smem(smem_u32(p), rank)));
    return v;
}
// Sum of x over the threads up to mine; `total` of all.  Two barriers; scan[32].
template <int kThreads>
__device__ __forceinline__ uint32_t block_scan(uint32_t x, uint32_t *scan, uint32_t &total) {
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const uint32_t y = __shfl_up_sync(0xffffffffu, x, o);
        if (lane >= o) x += y;
    }
    if (lane == 31) scan[warp] = x;
    __syncthreads();
    const uint32_t w = lane < kThreads / 32 ? scan[lane] : 0u;
    total = __reduce_add_sync(0xffffffffu, w);
    x += __reduce_add_sync(0xffffffffu, lane < warp ? w : 0u);
    __syncthreads();
    return x;
}

// kCtas: CTAs of a cluster.  kKeys: where a CTA's keys are: 0 its threads' registers, 1 shared memory, 2 nowhere (the weights are read again).
template <int kKeys, int kCtas>
__global__ void __launch_bounds__(kCtas > 1 ? kWide : kNarrow, 1) evict_select_kernel(const EvictArgs a) {
    constexpr int kThreads = kCtas > 1 ? kWide : kNarrow;
    auto meet = [&]() {
        if constexpr (kCtas > 1) cluster_sync_all();
    };
    extern __shared__ __align__(16) uint8_t smem_raw[];
    SelectShared &sh = *reinterpret_cast<SelectShared *>(smem_raw);
    uint32_t *held = reinterpret_cast<uint32_t *>(smem_raw + sizeof(SelectShared));
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const uint32_t rank = kCtas > 1 ? cluster_cta_rank() : 0u;
    const int g = blockIdx.x / kCtas;
    const float *mass = a.mass + (int64_t)g * a.mass_stride;
    int32_t *kept = a.kept + (int64_t)g * a.budget;
    const int64_t m = a.rows - a.n_sink - a.n_recent, want = a.budget - a.n_sink - a.n_recent;
    const int64_t per = (m + kCtas - 1) / kCtas;
    const int64_t at0 = min((int64_t)rank * per, m);                     // my range of the candidates
    const int mine = (int)(min(at0 + per, m) - at0);
    const float *w0 = mass + a.n_sink + at0;

    for (int i = tid; i < kPasses * kBins; i += kThreads) (&sh.hist[0][0])[i] = 0u;
    pdl_launch_dependents();
    __syncthreads();
    pdl_wait();                                                          // the weights are an earlier kernel's
    // Keys into shared memory in the order of the rows, a thread's piece out of it again.  (Sixteen loads in flight a thread; pieces of an
    // odd length, so that those of a warp's threads lie in different banks.)
    const int seg = ((mine + kThreads - 1) / kThreads) | 1, s0 = min(tid * seg, mine), s1 = min(s0 + seg, mine);
    uint32_t own[kKeys == 0 ? kOwn : 1];
    if constexpr (kKeys < 2) {
        for (int i = tid; i < mine; i += 16 * kThreads) {
            float x[16];
#pragma unroll
            for (int e = 0; e < 16; ++e) x[e] = i + e * kThreads < mine ? w0[i + e * kThreads] : 0.f;
#pragma unroll
            for (int e = 0; e < 16; ++e)
                if (i + e * kThreads < mine) held[i + e * kThreads] = key_of(x[e]);
        }
        __syncthreads();
    }
    if constexpr (kKeys == 0) {
#pragma unroll
        for (int e = 0; e < kOwn; ++e) own[e] = s0 + e < s1 ? held[s0 + e] : 0u;
    }
    // rows that stay whatever their weight
    for (int64_t i = (int64_t)rank * kThreads + tid; i < a.n_sink + a.n_recent; i += kCtas * kThreads) {
        const int64_t row = i < a.n_sink ? i : a.rows - a.n_recent + (i - a.n_sink);
        kept[i < a.n_sink ? i : a.budget - a.n_recent + (i - a.n_sink)] = (int32_t)row;
    }
    // f(key, its place in the range) for each of my keys, in order
    auto each = [&](auto f) {
        if constexpr (kKeys == 0) {
#pragma unroll
            for (int e = 0; e < kOwn; ++e)
                if (s0 + e < s1) f(own[e], s0 + e);
        } else {
#pragma unroll 4
            for (int i = s0; i < s1; ++i) f(kKeys == 1 ? held[i] : key_of(w0[i]), i);
        }
    };

    uint32_t known = 0u;                 // the wanted key's upper bits, as far as they are known
    uint32_t left = (uint32_t)want;      // the wanted key is the left-th largest of the keys that agree with them
    int bits = 0;                        // how many they are
#pragma unroll 1
    for (int pass = 0; pass < kPasses && want > 0; ++pass) {
        uint32_t *hist = sh.hist[pass];
        const int shift = 24 - 8 * pass;
        each([&](uint32_t k, int) {
            if (pass == 0 || k >> (shift + 8) == known) atomicAdd(&hist[(k >> shift) & 255u], 1u);
        });
        __syncthreads();
        meet();                          // everybody's histogram is complete (and stays: the next pass has another)
        // bins from the top down, one a thread
        uint32_t c = 0u;
        const int bin = kBins - 1 - tid;
        if (bin >= 0) {
            if constexpr (kCtas == 1) {
                c = hist[bin];
            } else {
                uint32_t got[kCtas];
#pragma unroll
                for (int r = 0; r < kCtas; ++r) got[r] = peer_u32(&hist[bin], (uint32_t)r);
#pragma unroll
                for (int r = 0; r < kCtas; ++r) c += got[r];
            }
        }
        uint32_t all;
        const uint32_t upto = block_scan<kThreads>(c, sh.scan, all);
        if (bin >= 0 && left > upto - c && left <= upto) {
            sh.found_bin = (uint32_t)bin;
            sh.found_above = upto - c;
            sh.found_count = c;
        }
        __syncthreads();
        known = known << 8 | sh.found_bin;
        left -= sh.found_above;
        bits += 8;
        if (left == sh.found_count) break;       // (what is in the bin is wanted, whatever the bits below; all CTAs see the same)
    }
    // Wanted are the keys whose upper bits are above `known`, and of those that have them `left`, from the lowest row up.
    const int lower = 32 - bits;
    uint32_t gt = 0u, eq = 0u;
    if (want > 0)
        each([&](uint32_t k, int) {
            gt += k >> lower > known;
            eq += k >> lower == known;
        });
    uint32_t gt_all, eq_all;
    uint32_t gt0 = block_scan<kThreads>(gt, sh.scan, gt_all) - gt, eq0 = block_scan<kThreads>(eq, sh.scan, eq_all) - eq;      // of rows below my piece
    uint32_t gt_before = 0u, eq_before = 0u;         // of the ranges before mine
    if constexpr (kCtas > 1) {
        if (tid == 0) {
            sh.counts[0] = gt_all;
            sh.counts[1] = eq_all;
        }
        __syncthreads();
        meet();
        if (warp == 0) {
            uint32_t x = 0u, y = 0u;
            if (lane < (int)rank) {
                x = peer_u32(&sh.counts[0], (uint32_t)lane);
                y = peer_u32(&sh.counts[1], (uint32_t)lane);
            }
            x = __reduce_add_sync(0xffffffffu, x);
            y = __reduce_add_sync(0xffffffffu, y);
            if (lane == 0) {
                sh.before[0] = x;
                sh.before[1] = y;
            }
        }
        __syncthreads();
        gt_before = sh.before[0];
        eq_before = sh.before[1];
        gt0 += gt_before;
        eq0 += eq_before;
        cluster_arrive_relaxed();        // (my looks at the partners are over; see the end)
    }
    // Numbers of the rows kept: through shared memory where the keys are no longer there, so that neighbours are written together (as they
    // come, 5400 cycles for 16 384 keys)
    const uint32_t first = gt_before + min(eq_before, left);             // kept rows of the ranges before mine
    if (want > 0)
        each([&](uint32_t k, int i) {
            const bool over = k >> lower > known, tie = k >> lower == known;
            if (over || (tie && eq0 < left)) {
                const uint32_t to = gt0 + min(eq0, left);
                const int32_t row = (int32_t)(a.n_sink + at0 + i);
                if (kKeys == 0) held[to - first] = (uint32_t)row;
                else kept[a.n_sink + to] = row;
            }
            gt0 += over;
            eq0 += tie;
        });
    if constexpr (kKeys == 0) {
        __syncthreads();
        const int count = want > 0 ? (int)(gt_all + min(eq_before + eq_all, left) - min(eq_before, left)) : 0;
        for (int i = tid; i < count; i += kThreads) kept[a.n_sink + first + i] = (int32_t)held[i];
    }
    if constexpr (kCtas > 1) {
        __syncwarp();
        cluster_wait();                  // nobody leaves while a partner may still read its counts
    }
}

constexpr int kMoveThreads = 256, kMoveItems = 8;
// A row is 2^lg units of 16 bytes in either plane.
__global__ void __launch_bounds__(kMoveThreads) evict_move_kernel(const EvictArgs a, const int lg, const int row_blocks) {
    const int units = 1 << lg;
    const int g = blockIdx.y;
    const int32_t *kept = a.kept + (int64_t)g * a.budget;
    const int64_t all = a.budget << (lg + 1);
    pdl_launch_dependents();
    pdl_wait();
    if ((int)blockIdx.x < row_blocks) {
        // the rows' weights and, of quantised storage, their scales: blocks of their own (in the threads that start a row they
        // cost 18 us of 59)
        for (int64_t r = (int64_t)blockIdx.x * (kMoveThreads * kMoveItems) + threadIdx.x, e = 0; e < kMoveItems && r < a.budget; ++e, r += kMoveThreads) {
            if (a.mass_out) a.mass_out[(int64_t)g * a.out_stride + r] = a.mass[(int64_t)g * a.mass_stride + kept[r]];
            if (a.from.k_scales) {
                const int64_t src = a.from.scale_offset(g, kept[r]), dst = a.to.scale_offset(g, r);
                a.to.k_scales[dst] = a.from.k_scales[src];
                a.to.v_scales[dst] = a.from.v_scales[src];
            }
        }
        return;
    }
    const int64_t i0 = (int64_t)(blockIdx.x - row_blocks) * (kMoveThreads * kMoveItems) + threadIdx.x;
    // (a thread's items are all K or all V of the same place in a row: 256 is a multiple of a row pair's units)
    const bool value = ((int)i0 & units) != 0;
    const int64_t in_row = ((int)i0 & (units - 1)) * 16;
    const char *from = (value ? a.from.v : a.from.k) + in_row;
    char *to = (value ? a.to.v : a.to.k) + in_row;
    int32_t row[kMoveItems];
    uint4 v[kMoveItems];
#pragma unroll
    for (int e = 0; e < kMoveItems; ++e) row[e] = i0 + e * kMoveThreads < all ? kept[(i0 + e * kMoveThreads) >> (lg + 1)] : -1;
#pragma unroll
    for (int e = 0; e < kMoveItems; ++e)
        if (row[e] >= 0) v[e] = *reinterpret_cast<const uint4 *>(from + a.from.offset(g, row[e]));
#pragma unroll
    for (int e = 0; e < kMoveItems; ++e)
        if (row[e] >= 0) *reinterpret_cast<uint4 *>(to + a.to.offset(g, (i0 + e * kMoveThreads) >> (lg + 1))) = v[e];
    if (a.range_limit > 0.f) {
        bool beyond = false;
#pragma unroll
        for (int e = 0; e < kMoveItems; ++e)
            if (row[e] >= 0)
                beyond = beyond || fabsf(__uint_as_float(v[e].x)) > a.range_limit || fabsf(__uint_as_float(v[e].y)) > a.range_limit ||
                         fabsf(__uint_as_float(v[e].z)) > a.range_limit || fabsf(__uint_as_float(v[e].w)) > a.range_limit;
        if (beyond) atomicCAS(a.status, 0, 7);
    }
    // value rows behind the last one, as an append leaves them
    if (i0 == threadIdx.x) {
        const int64_t rows = a.zero_end - a.budget;
        if (a.to.v_scales) {
            for (int64_t i = threadIdx.x; i < rows; i += kMoveThreads) a.to.v_scales[a.to.scale_offset(g, a.budget + i)] = 0.f;
        } else {
            for (int64_t i = threadIdx.x; i < rows << lg; i += kMoveThreads)
                *reinterpret_cast<uint4 *>(a.to.v + a.to.offset(g, a.budget + (i >> lg)) + (i & (units - 1)) * 16) = make_uint4(0u, 0u, 0u, 0u);
        }
    }
}

}  // namespace

template <int kKeys, int kCtas>
static cudaError_t launch_select(const EvictArgs &a, int64_t per, cudaStream_t s) {
    auto select = evict_select_kernel<kKeys, kCtas>;
    const cudaError_t e = raise_smem_limit_once(reinterpret_cast<const void *>(select), (int)(sizeof(SelectShared) + (size_t)kHeldKeys * 4));
    if (e != cudaSuccess) return e;
    return launch_pdl_cluster(kCtas, select, dim3((unsigned)(a.Hkv * kCtas)), dim3(kCtas > 1 ? kWide : kNarrow),
                              sizeof(SelectShared) + (kKeys < 2 ? (size_t)per * 4 : 0), s, a);
}

cudaError_t launch_evict(const EvictArgs &a, cudaStream_t s) {
    const int64_t m = a.rows - a.n_sink - a.n_recent, per = (m + 7) / 8;
    static_assert(sizeof(SelectShared) + (size_t)kHeldKeys * 4 <= 232448, "shared memory budget of one CTA");
    static_assert(kOneCta <= kOwn * kNarrow, "a thread's keys");
    cudaError_t e = m <= kOneCta        ? launch_select<0, 1>(a, m, s)
                    : per <= 16 * kWide ? launch_select<0, 8>(a, per, s)
                    : per <= kHeldKeys  ? launch_select<1, 8>(a, per, s)
                                        : launch_select<2, 8>(a, per, s);
    if (e != cudaSuccess) return e;
    int lg = 0;                                      // (rows are 64 to 512 bytes, a power of two)
    while (16 << lg < a.from.row_bytes) ++lg;
    const int64_t blocks = ((a.budget << (lg + 1)) + kMoveThreads * kMoveItems - 1) / (kMoveThreads * kMoveItems);
    const int64_t row_blocks = a.mass_out || a.from.k_scales ? (a.budget + kMoveThreads * kMoveItems - 1) / (kMoveThreads * kMoveItems) : 0;
    return launch_pdl(evict_move_kernel, dim3((unsigned)(row_blocks + blocks), a.Hkv), dim3(kMoveThreads), 0, s, a, lg, (int)row_blocks);
}

}  // namespace kvf
