// Eviction: the rows of a cache that count most, moved in order into another one.
//
// The paper's Discussion perturbs a folded cache by attention-based pruning (an information-removing perturbation; no scheme is given).
// Here, for each KV head on its own, the first n_sink rows and the last n_recent stay, and of the m rows between them the `want` with the
// most accumulated attention weight (kvf_cache_mass); of rows with the same weight the lower ones.  Order is kept, so that "first" and
// "last" mean the same in the smaller cache.
//
// Select.  A weight is mapped to a 32-bit key that sorts as the weight does (NaN below everything, -0 as +0).  The want-th largest key is
// found by radix, eight bits at a time from the top: a histogram of the keys that agree with what is known so far, until all that are
// left in the bin are wanted.  A cluster of CTAs has one KV head: each takes an equal range of rows, holds its keys in shared memory
// (51 200 of them; a longer range is read from global memory for each histogram), and adds up the histograms of all through
// distributed shared memory.  Then rows above the key, and as many of those equal to it as are wanted, from the lowest up, are counted
// thread by thread (a piece of the range each, of an odd length, so that 32 of them lie in different banks), and written in
// order.  Counts are whole numbers, so that the order of the atomics changes nothing.
// What bounds it is latency: a sweep of shared memory, a cluster barrier (1500 cycles), a look at eight histograms and a scan for every
// eight bits.  (Three histograms over 11, 11 and 10 bits: 64 KB from the peers at ~20 bytes a cycle each; numbering by ballots and
// the weights written here took half of the 26 us.)
//
// Move.  Rows are copied 16 bytes a thread, K and V rows of a KV head in one launch, eight loads in flight a thread; bound by memory
// (two reads and two writes of every row kept).
#include "kvfold_internal.h"
#include "sm100_ptx.cuh"

namespace kvf {
namespace {

constexpr int kSelectThreads = 1024;
constexpr int kBins = 256, kPasses = 4;
constexpr int kHeldKeys = 51200;                     // keys of a CTA's range in shared memory
constexpr int64_t kOneCta = 4096;                    // candidates up to which a KV head gets one CTA, not eight

struct SelectShared {
    uint32_t hist[kPasses][kBins];
    uint32_t scan[kSelectThreads / 32];
    uint32_t found_bin, found_above, found_count;    // bin that the wanted key lies in, keys in the bins above it, in it
    __align__(8) uint32_t counts[2];                 // of this CTA's range: keys above the wanted key, keys equal to it
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
__device__ __forceinline__ uint32_t block_scan(uint32_t x, uint32_t *scan, uint32_t &total) {
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const uint32_t y = __shfl_up_sync(0xffffffffu, x, o);
        if (lane >= o) x += y;
    }
    if (lane == 31) scan[warp] = x;
    __syncthreads();
    uint32_t below = lane < warp ? scan[lane] : 0u, all = scan[lane];
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
        below += __shfl_xor_sync(0xffffffffu, below, o);
        all += __shfl_xor_sync(0xffffffffu, all, o);
    }
    total = all;
    __syncthreads();
    return x + below;
}

// kCtas: CTAs of a cluster.  kHeld: the range's keys stay in shared memory.
template <bool kHeld, int kCtas>
__global__ void __launch_bounds__(kSelectThreads, 1) evict_select_kernel(const EvictArgs a) {
    auto meet = [&]() {
        if constexpr (kCtas > 1) cluster_sync_all();
    };
    extern __shared__ __align__(16) uint8_t smem_raw[];
    SelectShared &sh = *reinterpret_cast<SelectShared *>(smem_raw);
    uint32_t *held = reinterpret_cast<uint32_t *>(smem_raw + sizeof(SelectShared));
    const int tid = threadIdx.x, warp = tid >> 5;
    const uint32_t rank = kCtas > 1 ? cluster_cta_rank() : 0u;
    const int g = blockIdx.x / kCtas;
    const float *mass = a.mass + (int64_t)g * a.mass_stride;
    int32_t *kept = a.kept + (int64_t)g * a.budget;
    const int64_t m = a.rows - a.n_sink - a.n_recent, want = a.budget - a.n_sink - a.n_recent;
    const int64_t per = (m + kCtas - 1) / kCtas;
    const int64_t at0 = min((int64_t)rank * per, m);                     // my range of the candidates
    const int mine = (int)(min(at0 + per, m) - at0);
    const float *w0 = mass + a.n_sink + at0;

    for (int i = tid; i < kPasses * kBins; i += kSelectThreads) (&sh.hist[0][0])[i] = 0u;
    pdl_launch_dependents();
    __syncthreads();
    pdl_wait();                                                          // the weights are an earlier kernel's
    // rows that stay whatever their weight
    for (int64_t i = (int64_t)rank * kSelectThreads + tid; i < a.n_sink + a.n_recent; i += kCtas * kSelectThreads) {
        const int64_t row = i < a.n_sink ? i : a.rows - a.n_recent + (i - a.n_sink);
        kept[i < a.n_sink ? i : a.budget - a.n_recent + (i - a.n_sink)] = (int32_t)row;
    }
    auto key_at = [&](int i) { return kHeld ? held[i] : key_of(w0[i]); };

    uint32_t known = 0u;                 // the wanted key's upper bits, as far as they are known
    uint32_t left = (uint32_t)want;      // the wanted key is the left-th largest of the keys that agree with them
    int bits = 0;                        // how many they are
#pragma unroll 1
    for (int pass = 0; pass < kPasses && want > 0; ++pass) {
        uint32_t *hist = sh.hist[pass];
        const int shift = 24 - 8 * pass;
        if (pass == 0) {
            // (sixteen loads in flight a thread)
            for (int i = tid; i < mine; i += 16 * kSelectThreads) {
                float x[16];
#pragma unroll
                for (int e = 0; e < 16; ++e) x[e] = i + e * kSelectThreads < mine ? w0[i + e * kSelectThreads] : 0.f;
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                    if (i + e * kSelectThreads >= mine) break;
                    const uint32_t k = key_of(x[e]);
                    if (kHeld) held[i + e * kSelectThreads] = k;
                    atomicAdd(&hist[k >> 24], 1u);
                }
            }
        } else {
#pragma unroll 4
            for (int i = tid; i < mine; i += kSelectThreads) {
                const uint32_t k = key_at(i);
                if (k >> (shift + 8) == known) atomicAdd(&hist[(k >> shift) & 255u], 1u);
            }
        }
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
        const uint32_t upto = block_scan(c, sh.scan, all);
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
    auto above = [&](uint32_t k) { return bits > 0 && k >> lower > known; };
    auto equal = [&](uint32_t k) { return bits > 0 && k >> lower == known; };
    const int seg = ((mine + kSelectThreads - 1) / kSelectThreads) | 1, s0 = min(tid * seg, mine), s1 = min(s0 + seg, mine);
    uint32_t gt = 0u, eq = 0u;
#pragma unroll 4
    for (int i = s0; i < s1; ++i) {
        const uint32_t k = key_at(i);
        gt += above(k);
        eq += equal(k);
    }
    uint32_t gt_all, eq_all;
    uint32_t gt0 = block_scan(gt, sh.scan, gt_all) - gt, eq0 = block_scan(eq, sh.scan, eq_all) - eq;      // of rows below my piece
    if constexpr (kCtas > 1) {
        if (tid == 0) {
            sh.counts[0] = gt_all;
            sh.counts[1] = eq_all;
        }
        __syncthreads();
        meet();
        uint32_t got[2 * kCtas];
#pragma unroll
        for (int r = 0; r < 2 * kCtas; ++r) got[r] = peer_u32(&sh.counts[r & 1], (uint32_t)(r >> 1));
#pragma unroll
        for (int r = 0; r < kCtas; ++r)
            if (r < (int)rank) {
                gt0 += got[2 * r];
                eq0 += got[2 * r + 1];
            }
    }
#pragma unroll 4
    for (int i = s0; i < s1; ++i) {
        const uint32_t k = key_at(i);
        const bool over = above(k), tie = equal(k);
        if (over || (tie && eq0 < left)) kept[a.n_sink + gt0 + min(eq0, left)] = (int32_t)(a.n_sink + at0 + i);
        gt0 += over;
        eq0 += tie;
    }
    __syncthreads();
    meet();                              // nobody leaves while a partner may still read its counts
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

template <int kCtas>
static cudaError_t launch_select(const EvictArgs &a, cudaStream_t s) {
    const int64_t m = a.rows - a.n_sink - a.n_recent, per = (m + kCtas - 1) / kCtas;
    const bool held = per <= kHeldKeys;
    auto select = held ? evict_select_kernel<true, kCtas> : evict_select_kernel<false, kCtas>;
    cudaError_t e = raise_smem_limit_once(reinterpret_cast<const void *>(select), (int)(sizeof(SelectShared) + (size_t)kHeldKeys * 4));
    if (e != cudaSuccess) return e;
    return launch_pdl_cluster(kCtas, select, dim3((unsigned)(a.Hkv * kCtas)), dim3(kSelectThreads), sizeof(SelectShared) + (held ? (size_t)per * 4 : 0), s, a);
}

cudaError_t launch_evict(const EvictArgs &a, cudaStream_t s) {
    const int64_t m = a.rows - a.n_sink - a.n_recent;
    static_assert(sizeof(SelectShared) + (size_t)kHeldKeys * 4 <= 232448, "shared memory budget of one CTA");
    cudaError_t e = m <= kOneCta ? launch_select<1>(a, s) : launch_select<8>(a, s);
    if (e != cudaSuccess) return e;
    int lg = 0;                                      // (rows are 64 to 512 bytes, a power of two)
    while (16 << lg < a.from.row_bytes) ++lg;
    const int64_t blocks = ((a.budget << (lg + 1)) + kMoveThreads * kMoveItems - 1) / (kMoveThreads * kMoveItems);
    const int64_t row_blocks = a.mass_out || a.from.k_scales ? (a.budget + kMoveThreads * kMoveItems - 1) / (kMoveThreads * kMoveItems) : 0;
    return launch_pdl(evict_move_kernel, dim3((unsigned)(row_blocks + blocks), a.Hkv), dim3(kMoveThreads), 0, s, a, lg, (int)row_blocks);
}

}  // namespace kvf
