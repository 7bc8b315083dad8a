// Log-probabilities of given tokens, entropy and the most probable alternatives of rows of logits, in one pass over them.
//
// In powers of two, with y_i = log2(e) / T (x_i - m), m the largest logit so far: log2 p_i = y_i - log2 Z, Z = sum 2^y, and
// H = log2 Z - W / Z, W = sum 2^y y; raising m by d / (log2(e) / T) turns (Z, W) into (Z f, (W - d Z) f), f = 2^-d.  (The difference
// comes before the product: logits may be of any size, the type's lowest number as a mask among them.)  A thread keeps
// (m, Z, W) of its part of a row.  Threads are joined in a CTA and CTAs, up to 16 to a row, in a cluster, always in the same
// order, in fp32; the row's results are made of the joined sums in fp64.
//
// Alternatives: the n-th largest of the threads' maxima is no larger than the row's n-th largest logit, so only threads whose
// maximum reaches it look through their part again, and what they find (a few more than n) is sorted as (value, lowest token)
// keys by one warp.  Where far more logits pass (many equal ones), the n largest are found one after the other instead.
#include <cstdio>
#include <cstring>

#include <cooperative_groups.h>

#include "attn_body.cuh"

namespace cg = cooperative_groups;

#define LP_THREADS 256
#define LP_WARPS (LP_THREADS / 32)
#define LP_MAX_CLUSTER 16
static_assert(HIVIS_LOGPROBS_MAX_IDS <= 32 && HIVIS_LOGPROBS_MAX_TOP <= 32, "a lane each");
#define LP_CAND 512               // candidates a CTA keeps, and a cluster

struct LogprobArgs {
    const void* logits;
    long long ld;
    int n_rows, V;
    float scale;                  // log2(e) / T
    const int32_t* ids;           // nullable
    int n_ids, top_n;
    float *out_lp, *out_h, *out_top_lp;     // nullable
    int32_t* out_top;
    int slice;                    // logits per CTA, a multiple of 8
};

struct LpSum {
    float m, z, w;                // z = 0: nothing yet, m means nothing
};
__device__ __forceinline__ float lp_exp2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
// the sums of a set with another, at least as high, m
__device__ __forceinline__ LpSum lp_raise(const LpSum& s, float m, float scale) {
    if (s.z == 0.f) return LpSum{m, 0.f, 0.f};
    const float d = m == s.m ? 0.f : scale * (m - s.m), f = lp_exp2(-d);
    return LpSum{m, s.z * f, f > 0.f ? fmaf(-d, s.z, s.w) * f : 0.f};
}
__device__ __forceinline__ float lp_m(const LpSum& s) { return s.z == 0.f ? -INFINITY : s.m; }

// 16 bytes of logits at a time; a vector that is not wholly inside the row is read one by one
template <typename T>
struct LpVec {
    static constexpr int N = 16 / (int)sizeof(T);
};
template <typename T>
__device__ __forceinline__ void lp_load(const T* row, int i, int lo, int hi, bool vec, float (&x)[LpVec<T>::N]) {
    constexpr int N = LpVec<T>::N;
    if (vec && i >= lo && i + N <= hi) {
        const uint4 v = ld_stream((const uint4*)(row + i));
        if constexpr (N == 8) {
            x[0] = bf16_lo(v.x); x[1] = bf16_hi(v.x); x[2] = bf16_lo(v.y); x[3] = bf16_hi(v.y);
            x[4] = bf16_lo(v.z); x[5] = bf16_hi(v.z); x[6] = bf16_lo(v.w); x[7] = bf16_hi(v.w);
        } else {
            x[0] = __uint_as_float(v.x); x[1] = __uint_as_float(v.y); x[2] = __uint_as_float(v.z); x[3] = __uint_as_float(v.w);
        }
    } else {
#pragma unroll
        for (int e = 0; e < N; ++e) x[e] = i + e >= lo && i + e < hi ? load_as_float<T>(row, i + e) : -INFINITY;
    }
}
template <int N>
__device__ __forceinline__ void lp_add(LpSum& s, float& most, const float (&x)[N], float scale) {
    float m = x[0];
#pragma unroll
    for (int e = 1; e < N; ++e) m = fmaxf(m, x[e]);
    if (m > most) {
        most = m;
        s = lp_raise(s, m, scale);
    }
#pragma unroll
    for (int e = 0; e < N; ++e) {
        const float y = scale * (x[e] - s.m), p = lp_exp2(y);
        s.z += p;
        s.w = fmaf(p, fmaxf(y, -1e30f), s.w);            // (a logit of -infinity adds nothing)
    }
}

__device__ __forceinline__ float lp_zero(float x) { return x + 0.f; }                  // (-0 counts as 0)

// a warp's 32 values, largest first
__device__ __forceinline__ float lp_sort(float v, int lane) {
#pragma unroll
    for (int k = 2; k <= 32; k <<= 1)
#pragma unroll
        for (int j = k >> 1; j > 0; j >>= 1) {
            const float o = __shfl_xor_sync(0xffffffffu, v, j);
            const bool up = ((lane & j) == 0) == ((lane & k) == 0);      // this lane takes the larger one
            v = up ? fmaxf(v, o) : fminf(v, o);
        }
    return v;
}
__device__ __forceinline__ u64 lp_sort(u64 v, int lane) {
#pragma unroll
    for (int k = 2; k <= 32; k <<= 1)
#pragma unroll
        for (int j = k >> 1; j > 0; j >>= 1) {
            const u64 o = __shfl_xor_sync(0xffffffffu, v, j);
            const bool up = ((lane & j) == 0) == ((lane & k) == 0);
            v = up == (v > o) ? v : o;
        }
    return v;
}
// the 32 largest of two sets sorted so
__device__ __forceinline__ float lp_merge(float v, float o, int lane) {
    v = fmaxf(v, __shfl_sync(0xffffffffu, o, 31 - lane));
#pragma unroll
    for (int j = 16; j > 0; j >>= 1) {
        const float p = __shfl_xor_sync(0xffffffffu, v, j);
        v = (lane & j) == 0 ? fmaxf(v, p) : fminf(v, p);
    }
    return v;
}
__device__ __forceinline__ u64 lp_merge(u64 v, u64 o, int lane) {
    o = __shfl_sync(0xffffffffu, o, 31 - lane);
    v = v > o ? v : o;
#pragma unroll
    for (int j = 16; j > 0; j >>= 1) {
        const u64 p = __shfl_xor_sync(0xffffffffu, v, j);
        v = ((lane & j) == 0) == (v > p) ? v : p;
    }
    return v;
}

// The largest keys of `cand` (count of them; all different, 0 = none) by one warp, sorted: lane i has the i-th.
__device__ __forceinline__ u64 lp_select(const u64* cand, int count, int lane) {
    u64 best = lp_sort(lane < count ? cand[lane] : 0ull, lane);
    for (int i = 32; i < count; i += 32) best = lp_merge(best, lp_sort(i + lane < count ? cand[i + lane] : 0ull, lane), lane);
    return best;
}

template <typename T, bool TOP>
__global__ void __launch_bounds__(LP_THREADS) logprob_kernel(const __grid_constant__ LogprobArgs a) {
    constexpr int N = LpVec<T>::N;
    __shared__ LpSum s_sum[LP_WARPS], s_cta;
    __shared__ float s_max[LP_WARPS][32];
    __shared__ u64 s_cand[LP_CAND], s_top[32], s_red[LP_WARPS];
    __shared__ int s_count;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int S = gridDim.x, rank = blockIdx.x, r = blockIdx.y + gridDim.y * blockIdx.z;
    pdl_wait();
    pdl_trigger();
    if (r >= a.n_rows) return;                               // (whole clusters)
    const T* row = (const T*)a.logits + (long long)r * a.ld;
    // vectors start on 16-byte boundaries: `skew` logits before the row's first one belong to the first of them
    const int skew = (int)(((uintptr_t)row & 15u) / sizeof(T));
    const int lo = min(a.V, max(0, rank * a.slice - skew)), hi = rank == S - 1 ? a.V : min(a.V, (rank + 1) * a.slice - skew);
    const int first = rank * a.slice - skew + tid * N;
    // the tokens asked for: their logits are on their way meanwhile
    float asked = -INFINITY;
    if (rank == 0 && warp == 0 && lane < a.n_ids) {
        const int id = a.ids[(long long)r * a.n_ids + lane];
        if (id >= 0 && id < a.V) asked = load_as_float<T>(row, id);
    }
    LpSum s = {0.f, 0.f, 0.f};
    float most = -INFINITY;
    for (int i = first; i < hi; i += 4 * LP_THREADS * N) {
        float x[4][N];
#pragma unroll
        for (int u = 0; u < 4; ++u) lp_load<T>(row, i + u * LP_THREADS * N, lo, hi, true, x[u]);
#pragma unroll
        for (int u = 0; u < 4; ++u) lp_add<N>(s, most, x[u], a.scale);
    }
    // ---- the CTA's sums
    {
        float m = lp_m(s);
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
        LpSum d = lp_raise(s, m, a.scale);
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) {
            d.z += __shfl_xor_sync(0xffffffffu, d.z, o);
            d.w += __shfl_xor_sync(0xffffffffu, d.w, o);
        }
        if (lane == 0) s_sum[warp] = d;
    }
    if (TOP) {
        s_max[warp][lane] = lp_sort(most, lane);
        if (tid == 0) s_count = 0;
    }
    __syncthreads();
    if (tid == 0) {
        float m = -INFINITY;
        for (int w = 0; w < LP_WARPS; ++w) m = fmaxf(m, lp_m(s_sum[w]));
        LpSum d = {m, 0.f, 0.f};
        for (int w = 0; w < LP_WARPS; ++w) {
            const LpSum e = lp_raise(s_sum[w], m, a.scale);
            d.z += e.z;
            d.w += e.w;
        }
        s_cta = d;
    }
    if (TOP) {
        // the n-th largest of the threads' maxima
        float v = s_max[0][lane];
#pragma unroll
        for (int w = 1; w < LP_WARPS; ++w) v = lp_merge(v, s_max[w][lane], lane);
        const float bar = __shfl_sync(0xffffffffu, v, a.top_n - 1);
        if (most > -INFINITY && most >= bar) {
            for (int i = first; i < hi; i += LP_THREADS * N) {
                float x[N];
                lp_load<T>(row, i, lo, hi, true, x);
#pragma unroll
                for (int e = 0; e < N; ++e)
                    if (x[e] >= bar && x[e] > -INFINITY) {
                        const int at = atomicAdd(&s_count, 1);
                        if (at < LP_CAND) s_cand[at] = pack_key(lp_zero(x[e]), i + e);
                    }
            }
        }
        __syncthreads();
        const int count = s_count;
        if (count <= LP_CAND) {
            if (warp == 0) {
                const u64 best = lp_select(s_cand, count, lane);
                s_top[lane] = lane < a.top_n ? best : 0ull;
            }
        } else {
            // too many: one after the other
            u64 below = ~0ull;
            for (int k = 0; k < a.top_n; ++k) {
                u64 best = 0ull;
                for (int i = first; i < hi; i += LP_THREADS * N) {
                    float x[N];
                    lp_load<T>(row, i, lo, hi, true, x);
#pragma unroll
                    for (int e = 0; e < N; ++e)
                        if (x[e] >= bar && x[e] > -INFINITY) {
                            const u64 key = pack_key(lp_zero(x[e]), i + e);
                            if (key < below && key > best) best = key;
                        }
                }
#pragma unroll
                for (int o = 16; o > 0; o >>= 1) {
                    const u64 other = __shfl_xor_sync(0xffffffffu, best, o);
                    best = best > other ? best : other;
                }
                if (lane == 0) s_red[warp] = best;
                __syncthreads();
                for (int w = 0; w < LP_WARPS; ++w) best = best > s_red[w] ? best : s_red[w];
                below = best;
                if (tid == 0) s_top[k] = best;
                __syncthreads();
            }
            if (tid < 32 && tid >= a.top_n) s_top[tid] = 0ull;
        }
    }
    cg::cluster_group cluster = cg::this_cluster();
    if (S > 1) cluster.sync();
    else __syncthreads();
    // ---- the row, by the first warp of the first CTA
    if (rank == 0 && warp == 0) {
        LpSum d = {0.f, 0.f, 0.f};
        if (lane < S) d = *(S > 1 ? cluster.map_shared_rank(&s_cta, lane) : &s_cta);
        float m = lp_m(d);
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
        d = lp_raise(d, m, a.scale);
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) {
            d.z += __shfl_xor_sync(0xffffffffu, d.z, o);
            d.w += __shfl_xor_sync(0xffffffffu, d.w, o);
        }
        const bool mass = !(d.z == 0.f);                      // (a NaN counts as mass: it has to come out)
        const double ln2 = 0.69314718055994531, log_z = log2((double)d.z), scale = (double)a.scale;
        auto logprob = [&](float x) { return !mass || x == -INFINITY ? -INFINITY : (float)((scale * ((double)x - (double)m) - log_z) * ln2); };
        if (a.out_lp && lane < a.n_ids) a.out_lp[(long long)r * a.n_ids + lane] = logprob(asked);
        if (a.out_h && lane == 0) a.out_h[r] = mass ? (float)((log_z - (double)d.w / (double)d.z) * ln2) : 0.f;
        if (TOP) {
            u64 best = s_top[lane];
            for (int c = 1; c < S; ++c) best = lp_merge(best, *cluster.map_shared_rank(s_top + lane, c), lane);
            if (lane < a.top_n) {
                const int id = best ? key_index(best) : -1;
                a.out_top[(long long)r * a.top_n + lane] = id;
                a.out_top_lp[(long long)r * a.top_n + lane] = id >= 0 ? logprob(load_as_float<T>(row, id)) : -INFINITY;
            }
        }
    }
    if (S > 1) cluster.sync();
}

template <typename T, bool TOP>
static cudaError_t lp_launch(LogprobArgs& a, int dev, int num_sms, cudaStream_t st) {
    auto kernel = logprob_kernel<T, TOP>;
    static bool attr_set[HIVIS_MAX_DEVICES] = {false};
    if (dev < 0 || dev >= HIVIS_MAX_DEVICES || !attr_set[dev]) {
        const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
        if (e != cudaSuccess) return e;
        if (dev >= 0 && dev < HIVIS_MAX_DEVICES) attr_set[dev] = true;
    }
    // CTAs per row: enough to fill the GPU, each with a few thousand logits at least
    int S = 1;
    while (S < LP_MAX_CLUSTER && (long long)a.n_rows * S < 4ll * num_sms && a.V / (2 * S) >= 2048) S *= 2;
    a.slice = ((a.V + 8 + S - 1) / S + 7) / 8 * 8;
    cudaLaunchConfig_t cfg = {};
    const int y = a.n_rows < 32768 ? a.n_rows : 32768;
    cfg.gridDim = dim3((unsigned)S, (unsigned)y, (unsigned)((a.n_rows + y - 1) / y));
    cfg.blockDim = dim3(LP_THREADS);
    cfg.stream = st;
    cudaLaunchAttribute at[2] = {};
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    at[1].id = cudaLaunchAttributeClusterDimension;
    at[1].val.clusterDim.x = (unsigned)S;
    at[1].val.clusterDim.y = at[1].val.clusterDim.z = 1;
    cfg.attrs = at;
    cfg.numAttrs = 2;
    return cudaLaunchKernelEx(&cfg, kernel, a);
}

#define LP_FAIL(code, ...)                                    \
    do {                                                      \
        char msg_[200];                                       \
        snprintf(msg_, sizeof(msg_), __VA_ARGS__);            \
        hivis_set_global_error(msg_);                         \
        return code;                                          \
    } while (0)

extern "C" int hivis_logprobs(int n_rows, int vocab, const void* logits, int logits_dtype, int64_t ld, float temperature,
                              const int32_t* ids, int n_ids, int top_n, float* out_logprobs, float* out_entropy,
                              int32_t* out_top_ids, float* out_top_logprobs, void* stream) {
    if (n_rows < 0 || n_rows > (1 << 30)) LP_FAIL(HIVIS_ERR_CAPACITY, "hivis_logprobs: n_rows=%d out of range", n_rows);
    if (vocab < 1 || vocab > HIVIS_LOGPROBS_MAX_VOCAB) LP_FAIL(HIVIS_ERR_SHAPE, "hivis_logprobs: vocab=%d outside [1,%d]", vocab, HIVIS_LOGPROBS_MAX_VOCAB);
    if (logits_dtype != HIVIS_F32 && logits_dtype != HIVIS_BF16) LP_FAIL(HIVIS_ERR_DTYPE, "hivis_logprobs: unknown logits dtype");
    if (ld < vocab) LP_FAIL(HIVIS_ERR_SHAPE, "hivis_logprobs: ld is less than vocab");
    if (!(temperature > 0.f) || !(temperature < 3e38f)) LP_FAIL(HIVIS_ERR_ARG, "hivis_logprobs: temperature must be positive");
    if (n_ids < 0 || n_ids > HIVIS_LOGPROBS_MAX_IDS) LP_FAIL(HIVIS_ERR_CAPACITY, "hivis_logprobs: n_ids=%d outside [0,%d]", n_ids, HIVIS_LOGPROBS_MAX_IDS);
    if (top_n < 0 || top_n > HIVIS_LOGPROBS_MAX_TOP) LP_FAIL(HIVIS_ERR_CAPACITY, "hivis_logprobs: top_n=%d outside [0,%d]", top_n, HIVIS_LOGPROBS_MAX_TOP);
    if (n_rows == 0) return HIVIS_OK;
    if (!logits) LP_FAIL(HIVIS_ERR_ARG, "hivis_logprobs: logits is null");
    if (n_ids > 0 && (!ids || !out_logprobs)) LP_FAIL(HIVIS_ERR_ARG, "hivis_logprobs: ids and out_logprobs go with n_ids");
    if (top_n > 0 && (!out_top_ids || !out_top_logprobs)) LP_FAIL(HIVIS_ERR_ARG, "hivis_logprobs: out_top_ids and out_top_logprobs go with top_n");
    if (n_ids == 0 && top_n == 0 && !out_entropy) LP_FAIL(HIVIS_ERR_ARG, "hivis_logprobs: nothing is asked for");
    const void* ptrs[] = {logits, ids, out_logprobs, out_entropy, out_top_ids, out_top_logprobs};
    for (const void* p : ptrs)
        if (p && (((uintptr_t)p) & 15u)) LP_FAIL(HIVIS_ERR_ARG, "hivis_logprobs: device pointer not 16-byte aligned");
    LogprobArgs a;
    memset(&a, 0, sizeof(a));
    a.logits = logits; a.ld = ld; a.n_rows = n_rows; a.V = vocab;
    a.scale = (float)(1.4426950408889634 / (double)temperature);
    a.ids = ids; a.n_ids = n_ids; a.top_n = top_n;
    a.out_lp = n_ids > 0 ? out_logprobs : nullptr; a.out_h = out_entropy; a.out_top = out_top_ids; a.out_top_lp = out_top_logprobs;
    int dev = 0, sms = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e == cudaSuccess) e = cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev);
    cudaStream_t st = (cudaStream_t)stream;
    if (e == cudaSuccess) {
        if (logits_dtype == HIVIS_BF16) e = top_n ? lp_launch<bf16, true>(a, dev, sms, st) : lp_launch<bf16, false>(a, dev, sms, st);
        else e = top_n ? lp_launch<float, true>(a, dev, sms, st) : lp_launch<float, false>(a, dev, sms, st);
    }
    if (e != cudaSuccess) {
        cudaGetLastError();
        LP_FAIL(HIVIS_ERR_CUDA, "hivis_logprobs: launch failed: %s", cudaGetErrorString(e));
    }
    return HIVIS_OK;
}
