// Attention weight of a chunk's queries on every row of a cache:
//   mass[g][r] = decay * mass[g][r] + sum over tokens i that see row r and query heads h of KV head g of exp(s_ihr - lse_ih),
// s_ihr = scale * q_ih . k_gr, capped and biased as in a scored step, lse the softmax denominators that the step left.  (The paper prunes
// by attention weight in its Discussion and gives no scheme; this is the quantity that such schemes add up.)  It is the
// attention without its values: no running maximum, because the denominators are known, and sums over queries, not over keys.
#include "kvfold_internal.h"
#include "scores.cuh"

namespace kvf {
namespace {

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

cudaError_t launch_mass_simt(const MassArgs &a, int dtype, cudaStream_t s) {
    if (dtype == 0) return a.d == 128 ? launch_simt_t<__nv_bfloat16, 128>(a, s) : launch_simt_t<__nv_bfloat16, 64>(a, s);
    return a.d == 128 ? launch_simt_t<float, 128>(a, s) : launch_simt_t<float, 64>(a, s);
}

}  // namespace kvf
