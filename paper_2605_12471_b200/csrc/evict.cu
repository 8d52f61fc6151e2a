// Eviction: the rows of a cache that count most, moved in order into another one.
//
// The paper's Discussion perturbs a folded cache by attention-based pruning (an information-removing perturbation; no scheme is given).
// Here, for each KV head on its own, the first n_sink rows and the last n_recent stay, and of the m rows between them the `want` with the
// most accumulated attention weight (kvf_cache_mass); of rows with the same weight the lower ones.  Order is kept, so that "first" and
// "last" mean the same in the smaller cache.
//
// Select.  A weight is mapped to a 32-bit key that sorts as the weight does (NaN below everything, -0 as +0).  The want-th largest key is
// found by radix: three histograms over 11, 11 and 10 bits, each of the keys that agree with what is known so far.  A cluster of
// CTAs has one KV head: each takes an equal range of rows, holds its keys in shared memory (49 152 of them; a longer range is read
// from global memory for each histogram), and adds up the histograms of all through distributed shared memory.  Then rows above the
// key, and as many of those equal to it as are wanted, from the lowest up, are numbered by ballots and written in order.  Counts
// are whole numbers, so that the order of the atomics changes nothing.
// What bounds it is latency: per histogram a sweep of shared memory, a cluster barrier and a scan.
//
// Move.  Rows are copied 16 bytes a thread, K and V rows of a KV head in one launch, eight loads in flight a thread; bound by memory
// (two reads and two writes of every row kept).
#include <mutex>
#include <utility>
#include <vector>

#include "kvfold_internal.h"
#include "sm100_ptx.cuh"

namespace kvf {
namespace {

constexpr int kSelectThreads = 1024;
constexpr int kBins = 2048;
constexpr int kHeldKeys = 49152;                     // keys of a CTA's range in shared memory
constexpr int64_t kOneCta = 4096, kEightCtas = 32768;  // candidates up to which a KV head gets one CTA, eight

struct SelectShared {
    uint32_t hist[3][kBins];
    uint32_t scan[kSelectThreads / 32];
    uint32_t found_bin, found_above;                 // bin that the wanted key lies in, keys above that bin
    __align__(8) uint32_t counts[2];                              // of this CTA's range: keys above the wanted key, keys equal to it
    uint32_t warp_gt[kSelectThreads / 32], warp_eq[kSelectThreads / 32];
};

__device__ __forceinline__ uint32_t key_of(float w) {
    if (w != w) return 0u;
    const uint32_t b = __float_as_uint(w + 0.f);     // (-0 + 0 = 0)
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}

// (No "memory": loads of one and the same phase may be in flight together.  What separates the phases is volatile too.)
__device__ __forceinline__ uint2 peer_pair(const uint32_t *p, uint32_t rank) {
    uint2 v;
    asm volatile("ld.shared::cluster.v2.u32 {%0, %1}, [%2];" : "=r"(v.x), "=r"(v.y) : "r"(peer_smem(smem_u32(p), rank)));
    return v;
}

// kCtas: CTAs of a cluster.  kHeld: the range's keys stay in shared memory.
template <bool kHeld, int kCtas>
__global__ void __launch_bounds__(kSelectThreads, 1) evict_select_kernel(const EvictArgs a) {
    constexpr int ctas = kCtas;
    auto meet = [&]() {
        if constexpr (kCtas > 1) cluster_sync_all();
    };
    extern __shared__ __align__(16) uint8_t smem_raw[];
    SelectShared &sh = *reinterpret_cast<SelectShared *>(smem_raw);
    uint32_t *held = reinterpret_cast<uint32_t *>(smem_raw + sizeof(SelectShared));
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const uint32_t rank = kCtas > 1 ? cluster_cta_rank() : 0u;
    const int g = blockIdx.x / ctas;
    const float *mass = a.mass + (int64_t)g * a.mass_stride;
    int32_t *kept = a.kept + (int64_t)g * a.budget;
    float *mass_out = a.mass_out ? a.mass_out + (int64_t)g * a.out_stride : nullptr;
    const int64_t m = a.rows - a.n_sink - a.n_recent, want = a.budget - a.n_sink - a.n_recent;
    const int64_t per = (m + ctas - 1) / ctas;
    const int64_t at0 = min((int64_t)rank * per, m);                     // my range of the candidates
    const int mine = (int)(min(at0 + per, m) - at0);
    const float *w0 = mass + a.n_sink + at0;

    for (int i = tid; i < 3 * kBins; i += kSelectThreads) sh.hist[0][i] = 0u;
    if (tid < 2) sh.counts[tid] = 0u;
    pdl_launch_dependents();
    __syncthreads();
    pdl_wait();                                                          // the weights are an earlier kernel's
    // rows that stay whatever their weight
    for (int64_t i = (int64_t)rank * kSelectThreads + tid; i < a.n_sink + a.n_recent; i += (int64_t)ctas * kSelectThreads) {
        const int64_t row = i < a.n_sink ? i : a.rows - a.n_recent + (i - a.n_sink);
        const int64_t to = i < a.n_sink ? i : a.budget - a.n_recent + (i - a.n_sink);
        kept[to] = (int32_t)row;
        if (mass_out) mass_out[to] = mass[row];
    }
    auto key_at = [&](int i) { return kHeld ? held[i] : key_of(w0[i]); };

    uint32_t known = 0u;                 // the wanted key's upper bits, as far as they are known
    uint32_t left = (uint32_t)want;      // the wanted key is the left-th largest of the keys that agree with them
#pragma unroll 1
    for (int pass = 0; pass < 3; ++pass) {
        const int shift = pass == 0 ? 21 : pass == 1 ? 10 : 0, bins = pass == 2 ? 1024 : kBins;
        uint32_t *hist = sh.hist[pass];
        if (pass == 0) {
            // (eight loads in flight a thread)
            for (int i = tid; i < mine; i += 8 * kSelectThreads) {
                float x[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) x[e] = i + e * kSelectThreads < mine ? w0[i + e * kSelectThreads] : 0.f;
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    if (i + e * kSelectThreads >= mine) break;
                    const uint32_t k = key_of(x[e]);
                    if (kHeld) held[i + e * kSelectThreads] = k;
                    atomicAdd(&hist[k >> 21], 1u);
                }
            }
        } else {
            const int above_shift = pass == 1 ? 21 : 10;
#pragma unroll 4
            for (int i = tid; i < mine; i += kSelectThreads) {
                const uint32_t k = key_at(i);
                if (k >> above_shift == known) atomicAdd(&hist[(k >> shift) & (bins - 1)], 1u);
            }
        }
        __syncthreads();
        meet();                          // everybody's histogram is complete (and stays: the next pass has another)
        // Bins from the top down, two a thread: thread t has bins top - 2 t and top - 2 t - 1.
        const int b0 = bins - 1 - 2 * tid;
        uint32_t c0 = 0u, c1 = 0u;
        if (b0 > 0) {
            if constexpr (kCtas == 1) {
                c0 = hist[b0];
                c1 = hist[b0 - 1];
            } else {
                uint2 got[kCtas];
#pragma unroll
                for (int r = 0; r < kCtas; ++r) got[r] = peer_pair(&hist[b0 - 1], (uint32_t)r);
#pragma unroll
                for (int r = 0; r < kCtas; ++r) {
                    c0 += got[r].y;
                    c1 += got[r].x;
                }
            }
        }
        uint32_t sum = c0 + c1;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const uint32_t x = __shfl_up_sync(0xffffffffu, sum, o);
            if (lane >= o) sum += x;
        }
        if (lane == 31) sh.scan[warp] = sum;
        __syncthreads();
        if (warp == 0) {
            uint32_t t = sh.scan[lane];
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const uint32_t x = __shfl_up_sync(0xffffffffu, t, o);
                if (lane >= o) t += x;
            }
            sh.scan[lane] = t;
        }
        __syncthreads();
        const uint32_t upto = sum + (warp ? sh.scan[warp - 1] : 0u), above = upto - c0 - c1;      // keys in bins above mine
        if (b0 > 0 && left > above && left <= upto) {
            const bool second = left > above + c0;
            sh.found_bin = (uint32_t)(second ? b0 - 1 : b0);
            sh.found_above = second ? above + c0 : above;
        }
        __syncthreads();
        if (want > 0) {
            known = pass == 0 ? sh.found_bin : pass == 1 ? known << 11 | sh.found_bin : known << 10 | sh.found_bin;
            left -= sh.found_above;
        }
        __syncthreads();
    }
    // `known` is the wanted key; `left` of the rows equal to it are kept.  Each warp has an equal piece of the range, in order.
    const int seg = ((mine + 31) / 32 + 31) / 32 * 32, s0 = min(warp * seg, mine), s1 = min(s0 + seg, mine);
    uint32_t gt = 0u, eq = 0u;
    if (want > 0)
        for (int i = s0; i < s1; i += 32) {
            const uint32_t k = i + lane < s1 ? key_at(i + lane) : 0u;
            const bool in = i + lane < s1;
            gt += __popc(__ballot_sync(0xffffffffu, in && k > known));
            eq += __popc(__ballot_sync(0xffffffffu, in && k == known));
        }
    if (lane == 0) { sh.warp_gt[warp] = gt; sh.warp_eq[warp] = eq; }
    __syncthreads();
    if (warp == 0) {
        uint32_t x = sh.warp_gt[lane], y = sh.warp_eq[lane];
        const uint32_t x0 = x, y0 = y;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const uint32_t u = __shfl_up_sync(0xffffffffu, x, o), v = __shfl_up_sync(0xffffffffu, y, o);
            if (lane >= o) { x += u; y += v; }
        }
        sh.warp_gt[lane] = x - x0;
        sh.warp_eq[lane] = y - y0;
        if (lane == 31) { sh.counts[0] = x; sh.counts[1] = y; }
    }
    __syncthreads();
    meet();
    uint32_t gt0 = sh.warp_gt[warp], eq0 = sh.warp_eq[warp];             // of rows below my warp's piece
    if constexpr (kCtas > 1) {
        uint2 got[kCtas];
#pragma unroll
        for (int r = 0; r < kCtas; ++r) got[r] = peer_pair(sh.counts, (uint32_t)r);
#pragma unroll
        for (int r = 0; r < kCtas; ++r)
            if (r < (int)rank) {
                gt0 += got[r].x;
                eq0 += got[r].y;
            }
    }
    if (want > 0)
        for (int i = s0; i < s1; i += 32) {
            const bool in = i + lane < s1;
            const uint32_t k = in ? key_at(i + lane) : 0u;
            const uint32_t bg = __ballot_sync(0xffffffffu, in && k > known), be = __ballot_sync(0xffffffffu, in && k == known);
            const uint32_t below = (1u << lane) - 1u;
            const uint32_t ng = gt0 + __popc(bg & below), ne = eq0 + __popc(be & below);      // rows of either kind below mine
            if (in && (k > known || (k == known && ne < left))) {
                const int64_t to = a.n_sink + ng + min(ne, left), row = a.n_sink + at0 + i + lane;
                kept[to] = (int32_t)row;
                if (mass_out) mass_out[to] = w0[i + lane];
            }
            gt0 += __popc(bg);
            eq0 += __popc(be);
        }
    __syncthreads();
    meet();                              // nobody leaves while a partner may still read its counts
}

constexpr int kMoveThreads = 256, kMoveItems = 8;
// A row is 2^lg units of 16 bytes in either plane.
__global__ void __launch_bounds__(kMoveThreads) evict_move_kernel(const EvictArgs a, const int lg) {
    const int units = 1 << lg;
    const int g = blockIdx.y;
    const int32_t *kept = a.kept + (int64_t)g * a.budget;
    const int64_t all = a.budget << (lg + 1);
    const int64_t i0 = (int64_t)blockIdx.x * (kMoveThreads * kMoveItems) + threadIdx.x;
    pdl_launch_dependents();
    pdl_wait();
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
    // row scales of quantised storage, by the thread that starts a row; value rows behind the last one as an append leaves them
    if (a.from.k_scales)
        for (int e = 0; e < kMoveItems; ++e) {
            const int64_t i = i0 + e * kMoveThreads;
            if (i >= all || ((int)i & (2 * units - 1)) != 0) continue;
            const int64_t r = i >> (lg + 1), src = a.from.scale_offset(g, kept[r]), dst = a.to.scale_offset(g, r);
            a.to.k_scales[dst] = a.from.k_scales[src];
            a.to.v_scales[dst] = a.from.v_scales[src];
        }
    if (blockIdx.x == 0) {
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

// Clusters of that many CTAs the device holds at once (queried once per device).
template <int kCtas>
static int select_clusters() {
    static std::mutex mu;
    static std::vector<std::pair<int, int>> seen;
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess) return 0;
    std::lock_guard<std::mutex> lock(mu);
    for (auto &d : seen)
        if (d.first == dev) return d.second;
    auto kernel = evict_select_kernel<true, kCtas>;
    const size_t most = sizeof(SelectShared) + (size_t)kHeldKeys * 4;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(kCtas);
    cfg.blockDim = dim3(kSelectThreads);
    cfg.dynamicSmemBytes = most;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = kCtas; attr[0].val.clusterDim.y = 1; attr[0].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    int clusters = 0;
    if ((kCtas > 8 && (cudaFuncSetAttribute(kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1) != cudaSuccess ||
                       cudaFuncSetAttribute(evict_select_kernel<false, kCtas>, cudaFuncAttributeNonPortableClusterSizeAllowed, 1) != cudaSuccess)) ||
        raise_smem_limit_once(reinterpret_cast<const void *>(kernel), (int)most) != cudaSuccess ||
        cudaOccupancyMaxActiveClusters(&clusters, kernel, &cfg) != cudaSuccess) {
        cudaGetLastError();
        clusters = 0;
    }
    seen.push_back({dev, clusters});
    return clusters;
}

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
    cudaError_t e = m <= kOneCta                                        ? launch_select<1>(a, s)
                    : m > kEightCtas && select_clusters<16>() >= a.Hkv ? launch_select<16>(a, s)
                                                                        : launch_select<8>(a, s);
    if (e != cudaSuccess) return e;
    int lg = 0;                                      // (rows are 64 to 512 bytes, a power of two)
    while (16 << lg < a.from.row_bytes) ++lg;
    const int64_t blocks = ((a.budget << (lg + 1)) + kMoveThreads * kMoveItems - 1) / (kMoveThreads * kMoveItems);
    return launch_pdl(evict_move_kernel, dim3((unsigned)blocks, a.Hkv), dim3(kMoveThreads), 0, s, a, lg);
}

}  // namespace kvf
