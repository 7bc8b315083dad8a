// What the attention kernels over a 4-bit cache share: arguments, which rows a query sees, bounded waits, taking codes apart.
#pragma once
#include "kv4.cuh"

#define KV4_MAX_CLUSTER 16
#define KV4_WAIT_LIMIT (1 << 20)     // polls of a barrier before a warp gives up (each may suspend for a while)

struct Kv4AttnArgs {
    Kv4View c;
    SlotList sl;
    const int* rows;           // [B] rows of the cache that each sequence holds, the new ones among them
    const void* q;             // [B * n_q][q_ld], heads side by side
    long long q_ld;
    int n_q, Hq, G, ncol;      // G: query heads per KV head; ncol = n_q * G columns
    float scale_log2;          // scale * log2(e)
    const uint32_t* mask;      // nullable: [B][n_q][mask_words], over the last mask_rows rows
    int mask_rows, mask_words;
    void* out;                 // [B * n_q][out_ld]
    long long out_ld;
    int n_blocks;              // blocks of 8 NT columns
    int rows_add;              // added to rows[b]
    bf16* out_h;               // drafts: bf16 copy of out, its rounding remainders lo_rows rows further on if that is not 0
    int lo_rows;
};

// Element types of a draft step: queries in fp32, rounded to fp16 like the probabilities; results in fp32 and in bf16.
struct Kv4DraftIo {};
template <typename T> struct Kv4Io { typedef T Query; static constexpr bool SPLIT = sizeof(T) == 4; };
template <> struct Kv4Io<Kv4DraftIo> { typedef float Query; static constexpr bool SPLIT = false; };

__device__ __forceinline__ uint32_t kv4_saddr(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }
__device__ __forceinline__ bool kv4_wait(uint32_t bar, uint32_t parity) {
    for (int i = 0; i < KV4_WAIT_LIMIT; ++i) {
        uint32_t done;
        asm volatile("{\n\t.reg .pred p;\n\tmbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\tselp.u32 %0, 1, 0, p;\n\t}"
                     : "=r"(done) : "r"(bar), "r"(parity) : "memory");
        if (done) return true;
    }
    return false;
}
// one tile into shared memory; the barrier's phase ends when it is there (one lane)
__device__ __forceinline__ void kv4_fetch(uint32_t dst, const unsigned char* src, uint32_t bytes, uint32_t bar) {
    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];"
                 ::"r"(dst), "l"(src), "r"(bytes), "r"(bar) : "memory");
}
template <typename T>
__device__ __forceinline__ void kv4_load8(const void* p, long long i, float (&x)[8]) {
    if constexpr (sizeof(T) == 2) {
        const uint4 w = __ldg((const uint4*)((const bf16*)p + i));
        x[0] = bf16_lo(w.x); x[1] = bf16_hi(w.x); x[2] = bf16_lo(w.y); x[3] = bf16_hi(w.y);
        x[4] = bf16_lo(w.z); x[5] = bf16_hi(w.z); x[6] = bf16_lo(w.w); x[7] = bf16_hi(w.w);
    } else {
        const float4 u = __ldg((const float4*)((const float*)p + i)), w = __ldg((const float4*)((const float*)p + i + 4));
        x[0] = u.x; x[1] = u.y; x[2] = u.z; x[3] = u.w; x[4] = w.x; x[5] = w.y; x[6] = w.z; x[7] = w.w;
    }
}

__device__ __forceinline__ uint32_t kv4_half2(float x, float y) {
    const __half2 h = __floats2half2_rn(x, y);
    return *(const uint32_t*)&h;
}
__device__ __forceinline__ float2 kv4_unhalf2(uint32_t w) { return __half22float2(*(const __half2*)&w); }
__device__ __forceinline__ float kv4_exp2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
// 2^e, -126 <= e <= 127
__device__ __forceinline__ float kv4_pow2(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }
// What a column's scores are multiplied with, 2^e f (e may lie beyond fp32's exponents): neither 0 nor infinite, so that a score of
// -infinity (a row that is not seen) stays one and a score of 0 stays 0.
__device__ __forceinline__ float kv4_factor(int e, float f) {
    return fminf(fmaxf(f * kv4_pow2(e / 2) * kv4_pow2(e - e / 2), __uint_as_float(1u)), 3.402823466e38f);
}

// Nibbles 0 and 4 of a word as n, nibbles 1 and 5 as 16 n, two fp16 numbers: subnormal ones (of 2^-24) by a mask alone, or whole ones.
// The tensor core lines products up by their factors' exponent fields, and a subnormal's is ten bits above its value: sums of
// subnormal products keep about 2^-16 of themselves (measured: 1.9e-5), too few for fp32 results.
template <bool WHOLE>
__device__ __forceinline__ uint32_t kv4_lo(uint32_t w) {
    if constexpr (!WHOLE) return w & 0x000F000Fu;
    const uint32_t x = (w & 0x000F000Fu) | 0x64006400u;             // 1024 + n
    const __half2 h = __hsub2(*(const __half2*)&x, __floats2half2_rn(1024.f, 1024.f));
    return *(const uint32_t*)&h;
}
template <bool WHOLE>
__device__ __forceinline__ uint32_t kv4_hi(uint32_t w) {
    if constexpr (!WHOLE) return w & 0x00F000F0u;
    const uint32_t x = (w & 0x00F000F0u) | 0x64006400u;
    const __half2 h = __hsub2(*(const __half2*)&x, __floats2half2_rn(1024.f, 1024.f));
    return *(const uint32_t*)&h;
}

// a column's four channels from ch on: the sum of its rows over the sum of their weights
template <typename T>
__device__ __forceinline__ void kv4_put(const Kv4AttnArgs& a, int b, int h, int j, int ch, int dh, const float4& o, float l) {
    const float inv = l == 0.f ? 0.f : 1.f / l;                    // nothing visible: zeros
    const long long at = (long long)(b * a.n_q + j / a.G) * a.out_ld + (h * a.G + j % a.G) * dh + ch;
    if constexpr (sizeof(T) == 2) {
        const __nv_bfloat162 u = __floats2bfloat162_rn(o.x * inv, o.y * inv), v = __floats2bfloat162_rn(o.z * inv, o.w * inv);
        *(uint2*)((bf16*)a.out + at) = make_uint2(*(const unsigned*)&u, *(const unsigned*)&v);
    } else if constexpr (sizeof(T) == 1) {
        const float x[4] = {o.x * inv, o.y * inv, o.z * inv, o.w * inv};
        *(float4*)((float*)a.out + at) = make_float4(x[0], x[1], x[2], x[3]);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const bf16 hi = __float2bfloat16_rn(x[i]);
            a.out_h[at + i] = hi;
            if (a.lo_rows > 0) a.out_h[at + a.lo_rows * a.out_ld + i] = __float2bfloat16_rn(x[i] - __bfloat162float(hi));
        }
    } else {
        *(float4*)((float*)a.out + at) = make_float4(o.x * inv, o.y * inv, o.z * inv, o.w * inv);
    }
}

// The running maximum of a column that has seen no row: fp32's lowest number, as good a reference as any for scores next to it, and a
// difference with it is never NaN.
#define KV4_NOTHING -3.402823466e38f

// Two columns' scores above their maxima.  The product is rounded before the difference, as the maxima are: by one fused operation the
// largest score itself would be off its maximum by what the product lost, whole powers of two from 2^25 on.
// (Single products: the compiler fuses a pair's with the sum.)
__device__ __forceinline__ void kv4_above(float s0, float s1, float f0, float f1, u64 minus_m, float& y0, float& y1) {
    kv4_unpack2(kv4_add2(kv4_pack2(__fmul_rn(s0, f0), __fmul_rn(s1, f1)), minus_m), y0, y1);
}

// How far the maximum may fall behind: p < 2^8.
#define KV4_LAZY 8.f

struct Kv4Sight {              // which rows the columns see
    int nrows, n_q, mask_rows;
    const uint32_t* mask;      // of the sequence; nullable
    int mask_words;
    __device__ __forceinline__ bool operator()(int r, int i) const {
        if (!mask) return r <= nrows - n_q + i;
        const int k = r - (nrows - mask_rows);
        return k < 0 || (r < nrows && ((mask[(long long)i * mask_words + (k >> 5)] >> (k & 31)) & 1u));
    }
};

template <int Q>
__device__ __forceinline__ void kv4_lds(const unsigned char* p, uint32_t (&w)[Q]) {
    if constexpr (Q == 4) {
        const uint4 x = *(const uint4*)p;
        w[0] = x.x; w[1] = x.y; w[2] = x.z; w[3] = x.w;
    } else {
        const uint2 x = *(const uint2*)p;
        w[0] = x.x; w[1] = x.y;
    }
}

// CTAs per (sequence, KV head, block of columns): as many as the GPU holds at once, but no more than the cache's full length has
// steps for their warps.  Eight or sixteen, or less than eight: clusters of nine, say, leave a third of a GPC's places empty.
inline int kv4_cluster(int units, int max_len, int step_rows, int resident, int largest = KV4_MAX_CLUSTER) {
    const int most = max_len / step_rows, want = resident / units;
    const int s = want < most ? want : most;
    return s < 1 ? 1 : s < 8 ? s : s < largest ? 8 : largest;
}

// bf16, many columns (kernels_kv4_tc.cu).
cudaError_t launch_kv4_attn_tc(Kv4AttnArgs& a, int dev, int num_sms, cudaStream_t st);
