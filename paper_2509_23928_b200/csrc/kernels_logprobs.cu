// Log-probabilities of given tokens, entropy and the most probable alternatives of rows of logits, in one pass over them.
//
// In powers of two, with y_i = log2(e) / T x_i - c: log2 p_i = y_i - log2 Z, Z = sum 2^y, and H = log2 Z - W / Z, W = sum 2^y y, for any
// c near the largest logit's.  A thread takes c from its first 32 (bf16) or 16 logits and raises it only when later ones are above
// it by 2^3 (with 2^60 the rounding of y in the largest terms cost a digit: 9.7e-7 of the results) - raising by d turns (Z, W) into (Z f, (W - d Z) f), f = 2^-d - so that a logit costs one multiply-add for y, the
// exponential, and one operation for each sum.  Threads are joined in a CTA and CTAs, up to 16 to a row, in a cluster, always in
// the same order, in fp32; the row's results are made of the joined sums in fp64.
// A CTA whose largest logit is so far from zero that y would lose it (|log2(e) / T x| > 2^28: a row of the type's lowest number, say)
// goes over its part again with y = log2(e) / T (x - max).
//
// Alternatives: a thread remembers its largest logit.  The n-th largest of the threads' maxima is no larger than the n-th largest
// logit, so only parts of threads whose maximum reaches it are looked through again, a warp to a part, and what they hold (a
// few more than n) is sorted as (value, lowest token) keys by one warp.  Where far more logits pass (many equal ones), the n
// largest are found one after the other instead.
#include <cstdio>
#include <cstring>

#include <cooperative_groups.h>

#include "attn_body.cuh"

namespace cg = cooperative_groups;

#define LP_MAX_CLUSTER 16
static_assert(HIVIS_LOGPROBS_MAX_IDS <= 32 && HIVIS_LOGPROBS_MAX_TOP <= 32, "a lane each");
#define LP_CAND 512               // candidates a CTA keeps, and a cluster

struct LogprobArgs {
    const void* logits;
    long long ld;
    int n_rows, V;
    float scale;                  // log2(e) / T
    uint32_t low;                 // bf16: a pair of the number that stands for -infinity in the sums
    const int32_t* ids;           // nullable
    int n_ids, top_n;
    float *out_lp, *out_h, *out_top_lp;     // nullable
    int32_t* out_top;
    int slice;                    // logits per CTA, a multiple of 8
};

#define LP_FAR 0x1p28f            // |c| is at most this
#define LP_RISE 3.f               // y beyond which c is raised: y is rounded to 2^-24 of itself

struct LpSum {
    float c, z, w;
};
__device__ __forceinline__ float lp_exp2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
// (Z, W) for a reference higher by d
__device__ __forceinline__ void lp_lower(float& z, float& w, float d) {
    const float f = lp_exp2(-d);
    w = f > 0.f ? fmaf(-d, z, w) * f : 0.f;
    z = z == 0.f ? 0.f : z * f;
}

// 16 bytes of logits; a vector that is not wholly inside [lo, hi) is read one by one, with -infinity for what is outside
template <typename T>
struct LpVec {
    static constexpr int N = 16 / (int)sizeof(T);
    // Threads to a CTA; 1024 to an SM.  Smaller CTAs even out the last wave of many rows (1021 fp32 rows of 50257: 41 us with 128
    // threads, 45 with 256); with eight bf16 logits to a load a row needs the 256 (512 rows of 152064: 49 us, 55).
    static constexpr int THREADS = sizeof(T) == 2 ? 256 : 128;
};
template <typename T>
__device__ __forceinline__ uint4 lp_load(const T* row, int i, int lo, int hi) {
    constexpr int N = LpVec<T>::N;
    if (i >= lo && i + N <= hi) return ld_stream((const uint4*)(row + i));
    uint32_t w[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) w[k] = N == 8 ? 0xFF80FF80u : 0xFF800000u;
#pragma unroll
    for (int e = 0; e < N; ++e)
        if (i + e >= lo && i + e < hi) {
            if constexpr (N == 8) {
                const uint32_t x = ((const unsigned short*)row)[i + e];
                w[e / 2] = e & 1 ? (w[e / 2] & 0xFFFFu) | (x << 16) : (w[e / 2] & 0xFFFF0000u) | x;
            } else {
                w[e] = ((const uint32_t*)row)[i + e];
            }
        }
    return make_uint4(w[0], w[1], w[2], w[3]);
}
template <typename T>
__device__ __forceinline__ void lp_values(const uint4& v, float (&x)[LpVec<T>::N]) {
    if constexpr (sizeof(T) == 2) {
        x[0] = bf16_lo(v.x); x[1] = bf16_hi(v.x); x[2] = bf16_lo(v.y); x[3] = bf16_hi(v.y);
        x[4] = bf16_lo(v.z); x[5] = bf16_hi(v.z); x[6] = bf16_lo(v.w); x[7] = bf16_hi(v.w);
    } else {
        x[0] = __uint_as_float(v.x); x[1] = __uint_as_float(v.y); x[2] = __uint_as_float(v.z); x[3] = __uint_as_float(v.w);
    }
}

__device__ __forceinline__ __nv_bfloat162 lp_bf2(uint32_t w) { return *(const __nv_bfloat162*)&w; }
__device__ __forceinline__ uint32_t lp_w(const __nv_bfloat162& h) { return *(const uint32_t*)&h; }
// the largest of the numbers of some vectors (NaNs left out)
template <typename T, int U>
__device__ __forceinline__ float lp_most(const uint4 (&v)[U]) {
    if constexpr (sizeof(T) == 2) {
        __nv_bfloat162 m = __hmax2(__hmax2(lp_bf2(v[0].x), lp_bf2(v[0].y)), __hmax2(lp_bf2(v[0].z), lp_bf2(v[0].w)));
#pragma unroll
        for (int u = 1; u < U; ++u) m = __hmax2(m, __hmax2(__hmax2(lp_bf2(v[u].x), lp_bf2(v[u].y)), __hmax2(lp_bf2(v[u].z), lp_bf2(v[u].w))));
        return fmaxf(bf16_lo(lp_w(m)), bf16_hi(lp_w(m)));
    } else {
        float m = -INFINITY;
#pragma unroll
        for (int u = 0; u < U; ++u)
            m = fmaxf(fmaxf(m, fmaxf(__uint_as_float(v[u].x), __uint_as_float(v[u].y))), fmaxf(__uint_as_float(v[u].z), __uint_as_float(v[u].w)));
        return m;
    }
}
// The sums of some vectors' logits.  y stays finite, so that 2^y y of a logit of -infinity is 0 and no NaN: a clamp of y, and for bf16 of
// the logits, two at a time, to a number `low` that is without mass at any reference (lp_low).
template <typename T, int U>
__device__ __forceinline__ void lp_add(LpSum& s, const uint4 (&v)[U], float scale, uint32_t low2) {
    constexpr int N = LpVec<T>::N;
#pragma unroll
    for (int u = 0; u < U; ++u) {
        float x[N];
        if constexpr (sizeof(T) == 2) {
            const __nv_bfloat162 low = lp_bf2(low2);
            const uint4 t = make_uint4(lp_w(__hmax2_nan(lp_bf2(v[u].x), low)), lp_w(__hmax2_nan(lp_bf2(v[u].y), low)),
                                       lp_w(__hmax2_nan(lp_bf2(v[u].z), low)), lp_w(__hmax2_nan(lp_bf2(v[u].w), low)));
            lp_values<T>(t, x);
        } else {
            lp_values<T>(v[u], x);
        }
#pragma unroll
        for (int e = 0; e < N; ++e) {
            const float y = fmaf(scale, x[e], -s.c), p = lp_exp2(y);
            s.z += p;
            s.w = fmaf(p, sizeof(T) == 2 ? y : fmaxf(y, -1e38f), s.w);
        }
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

// What a CTA found out about its part of a row: sums relative to c, and whether some logit is not -infinity.
struct LpPart {
    double c;
    float z, w;
};

template <typename T, bool TOP>
__global__ void __launch_bounds__(LpVec<T>::THREADS, 1024 / LpVec<T>::THREADS) logprob_kernel(const __grid_constant__ LogprobArgs a) {
    constexpr int LP_THREADS = LpVec<T>::THREADS, LP_WARPS = LP_THREADS / 32;
    constexpr int N = LpVec<T>::N, U = 4, STRIDE = LP_THREADS * N;
    __shared__ LpSum s_sum[LP_WARPS];
    __shared__ float s_most[LP_WARPS], s_max[LP_WARPS][32], s_bar;
    __shared__ LpPart s_part;
    __shared__ u64 s_cand[LP_CAND], s_top[32], s_red[LP_WARPS];
    __shared__ int s_list[LP_THREADS], s_listed, s_count;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int S = gridDim.x, rank = blockIdx.x, r = blockIdx.y + gridDim.y * blockIdx.z;
    pdl_wait();
    pdl_trigger();
    if (r >= a.n_rows) return;                               // (whole clusters)
    const T* row = (const T*)a.logits + (long long)r * a.ld;
    // vectors start on 16-byte boundaries: `skew` logits before the row's first one belong to the first of them
    const int skew = (int)(((uintptr_t)row & 15u) / sizeof(T));
    const int lo = min(a.V, max(0, rank * a.slice - skew)), hi = rank == S - 1 ? a.V : min(a.V, (rank + 1) * a.slice - skew);
    const int begin = rank * a.slice - skew, first = begin + tid * N;
    // the tokens asked for: their logits are on their way meanwhile
    float asked = -INFINITY;
    if (rank == 0 && warp == 0 && lane < a.n_ids) {
        const int id = a.ids[(long long)r * a.n_ids + lane];
        if (id >= 0 && id < a.V) asked = load_as_float<T>(row, id);
    }
    LpSum s = {-LP_FAR, 0.f, 0.f};
    float most = -INFINITY;
    uint4 next[U];
#pragma unroll
    for (int u = 0; u < U; ++u) next[u] = lp_load<T>(row, first + u * STRIDE, lo, hi);
    for (int i = first; i < hi; i += U * STRIDE) {
        uint4 v[U];
#pragma unroll
        for (int u = 0; u < U; ++u) v[u] = next[u];
        if (i + U * STRIDE < hi) {
#pragma unroll
            for (int u = 0; u < U; ++u) next[u] = lp_load<T>(row, i + (U + u) * STRIDE, lo, hi);
        }
        const float m = lp_most<T>(v);
        most = fmaxf(most, m);
        const float c = fminf(fmaxf(a.scale * m, -LP_FAR), LP_FAR);
        if (c > s.c + (s.z == 0.f ? 0.f : LP_RISE)) {
            lp_lower(s.z, s.w, c - s.c);
            s.c = c;
        }
        lp_add<T>(s, v, a.scale, a.low);
    }
    // ---- the CTA's sums
    {
        float c = s.z == 0.f ? -INFINITY : s.c, m = most;
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) {
            c = fmaxf(c, __shfl_xor_sync(0xffffffffu, c, o));
            m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
        }
        if (s.z == 0.f) s.w = 0.f;
        else lp_lower(s.z, s.w, c - s.c);
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) {
            s.z += __shfl_xor_sync(0xffffffffu, s.z, o);
            s.w += __shfl_xor_sync(0xffffffffu, s.w, o);
        }
        if (lane == 0) {
            s_sum[warp] = LpSum{c, s.z, s.w};
            s_most[warp] = m;
        }
    }
    if (TOP) {
        s_max[warp][lane] = lp_sort(most, lane);
        if (tid == 0) s_count = s_listed = 0;
    }
    __syncthreads();
    float cta_most = s_most[0];
#pragma unroll
    for (int w = 1; w < LP_WARPS; ++w) cta_most = fmaxf(cta_most, s_most[w]);
    const bool far = cta_most > -INFINITY && !(fabsf(a.scale * cta_most) < 0.5f * LP_FAR);
    if (far) {
        // relative to the largest logit itself
        float z = 0.f, w = 0.f;
        for (int i = first; i < hi; i += STRIDE) {
            float x[N];
            lp_values<T>(lp_load<T>(row, i, lo, hi), x);
#pragma unroll
            for (int e = 0; e < N; ++e) {
                const float y = a.scale * (x[e] - cta_most), p = x[e] == cta_most && fabsf(cta_most) < INFINITY ? 1.f : lp_exp2(y);
                z += p;
                if (p > 0.f && p < 1.f) w = fmaf(p, y, w);
            }
        }
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) {
            z += __shfl_xor_sync(0xffffffffu, z, o);
            w += __shfl_xor_sync(0xffffffffu, w, o);
        }
        __syncthreads();                                     // (s_most has been read)
        if (lane == 0) s_sum[warp] = LpSum{0.f, z, w};
        __syncthreads();
    }
    if (tid == 0) {
        float c = -INFINITY, z = 0.f, w = 0.f;
#pragma unroll
        for (int k = 0; k < LP_WARPS; ++k) c = fmaxf(c, s_sum[k].c);
#pragma unroll
        for (int k = 0; k < LP_WARPS; ++k) {
            LpSum e = s_sum[k];
            if (e.z == 0.f) continue;
            lp_lower(e.z, e.w, c - e.c);
            z += e.z;
            w += e.w;
        }
        s_part = LpPart{far ? (double)a.scale * (double)cta_most : z == 0.f ? -INFINITY : (double)c, z, w};
    }
    if (TOP) {
        // the n-th largest of the threads' maxima
        if (warp == 1) {
            float v = s_max[0][lane];
#pragma unroll
            for (int w = 1; w < LP_WARPS; ++w) v = lp_merge(v, s_max[w][lane], lane);
            if (lane == a.top_n - 1) s_bar = v;
        }
        __syncthreads();
        const float bar = s_bar;
        if (most > -INFINITY && most >= bar) s_list[atomicAdd(&s_listed, 1)] = tid;
        __syncthreads();
        const int listed = s_listed;
        for (int k = warp; k < listed; k += LP_WARPS) {
            const int from = begin + s_list[k] * N;
            for (int i = from + lane * STRIDE; i < hi; i += 32 * STRIDE) {
                float x[N];
                lp_values<T>(lp_load<T>(row, i, lo, hi), x);
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
                for (int i = first; i < hi; i += STRIDE) {
                    float x[N];
                    lp_values<T>(lp_load<T>(row, i, lo, hi), x);
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
        LpPart d = {-INFINITY, 0.f, 0.f};
        if (lane < S) d = *(S > 1 ? cluster.map_shared_rank(&s_part, lane) : &s_part);
        double c = d.c;
#pragma unroll
        for (int o = 8; o > 0; o >>= 1) c = fmax(c, __shfl_xor_sync(0xffffffffu, c, o));
        c = __shfl_sync(0xffffffffu, c, 0);
        if (d.z == 0.f) d.w = 0.f;
        else lp_lower(d.z, d.w, (float)(c - d.c));
#pragma unroll
        for (int o = 8; o > 0; o >>= 1) {
            d.z += __shfl_xor_sync(0xffffffffu, d.z, o);
            d.w += __shfl_xor_sync(0xffffffffu, d.w, o);
        }
        d.z = __shfl_sync(0xffffffffu, d.z, 0);
        d.w = __shfl_sync(0xffffffffu, d.w, 0);
        const bool mass = !(d.z == 0.f);                      // (a NaN counts as mass: it has to come out)
        const double ln2 = 0.69314718055994531, log_z = log2((double)d.z), scale = (double)a.scale;
        // (-infinity - log Z: -infinity, or NaN in a row that is)
        auto logprob = [&](float x) { return !mass ? -INFINITY : (float)((scale * (double)x - c - log_z) * ln2); };
        if (a.out_lp && lane < a.n_ids) a.out_lp[(long long)r * a.n_ids + lane] = logprob(asked);
        if (a.out_h && lane == 0) a.out_h[r] = mass ? (float)((log_z - (double)d.w / (double)d.z) * ln2) : 0.f;
        if (TOP) {
            u64 best = s_top[lane];
            for (int k = 1; k < S; ++k) best = lp_merge(best, *cluster.map_shared_rank(s_top + lane, k), lane);
            if (lane < a.top_n) {
                const int id = best ? key_index(best) : -1;
                a.out_top[(long long)r * a.top_n + lane] = id;
                a.out_top_lp[(long long)r * a.top_n + lane] = id >= 0 ? logprob(load_as_float<T>(row, id)) : -INFINITY;
            }
        }
    }
    if (S > 1) cluster.sync();
}

// For bf16: the logit that takes -infinity's place, as a pair.  scale * low has to be finite (1e37) and so far below every reference, which is
// -LP_FAR at least, that 2^y is 0: at the smallest scale that is taken (T below 1e30) -3.3e38 comes to -4.7e8, LP_FAR is 2.7e8.  A finite
// logit below it is as far from the largest one, or its CTA goes over its part again relative to that one.
static uint32_t lp_low(float scale) {
    const double most = 1e37 / (double)scale;
    const uint32_t b = __bfloat16_as_ushort(__float2bfloat16((float)(most < 3.3e38 ? -most : -3.3e38)));
    return b << 16 | b;
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
    // CTAs per row: the first power of two that comes to half of what the GPU holds at once, each with a few thousand logits at least.  A CTA
    // costs some microseconds beside its logits.  Rows of 152064, in a graph: 56 of fp32 take 8.3 us with 16 CTAs each (which this gives
    // them; 16 CTAs of 128 threads are as many warps as 8 of 256), 8.2 with 8, 10.3 with 4; 56 of bf16 8.9 with 8 (this), 7.7 with 4, 11.9 with
    // 16; 512 of bf16 with 20 alternatives 43 with one (this), 46 with two; 1021 fp32 rows of 50257 38 with one (this), 45 with two.
    int S = 1;
    while (S < LP_MAX_CLUSTER && (long long)a.n_rows * S < (long long)num_sms * 512 / LpVec<T>::THREADS && a.V / (2 * S) >= 8 * LpVec<T>::THREADS) S *= 2;
    a.slice = ((a.V + 8 + S - 1) / S + 7) / 8 * 8;
    const int y = a.n_rows < 32768 ? a.n_rows : 32768;
    const dim3 grid((unsigned)S, (unsigned)y, (unsigned)((a.n_rows + y - 1) / y));
    return launch_cluster_pdl(kernel, S, grid, dim3(LpVec<T>::THREADS), 0, st, a);
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
    if (!(temperature > 1e-30f) || !(temperature < 1e30f)) LP_FAIL(HIVIS_ERR_ARG, "hivis_logprobs: temperature outside (1e-30, 1e30)");
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
    a.low = lp_low(a.scale);
    a.ids = ids; a.n_ids = n_ids; a.top_n = top_n;
    a.out_lp = n_ids > 0 ? out_logprobs : nullptr; a.out_h = out_entropy; a.out_top = out_top_ids; a.out_top_lp = out_top_logprobs;
    int dev = 0, sms = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e == cudaSuccess) e = device_sms(dev, &sms);
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
