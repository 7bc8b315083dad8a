// The 4-bit key/value cache: rows go in (quantised), come out (as fp32 values), and are attended over.  No call needs a context
// or a workspace.  kv4.cuh has the format.
#include <cstdio>
#include <cstring>

#include <cooperative_groups.h>

#include "kv4.cuh"

namespace cg = cooperative_groups;

// ------------------------------------------------------------------------------------------------ rows in and out
struct Kv4RowsArgs {
    Kv4View c;
    SlotList sl;
    CuSeqlens cu;              // packed rows: sequence b owns [cu.v[b], cu.v[b + 1])
    CuSeqlens pairs;           // first pair of rows of each sequence: half its rows and one, whichever way its start is aligned
    const int* start;          // [B] cache row of each sequence's first packed row
    const void *k, *v;         // packed rows [.][ld]
    long long ld;
    float *out_k, *out_v;      // read: [.][Hkv * dh]
};

// DH / 8 lanes a row: a lane has 8 neighbouring channels, four lanes a group.  Two halves of 2 * DH / 8 lanes take the two rows
// of a pair, which share the words of their V codes.
struct Kv4Place {
    int b, h, slot, w, c;      // sequence, KV head, slot, group, lane of the group
    int row, packed;           // cache row; row of the packed input, -1: none
};
template <int DH>
__device__ __forceinline__ Kv4Place kv4_place(const Kv4RowsArgs& a) {
    constexpr int LR = DH / 8;
    Kv4Place p;
    const long long t = (long long)blockIdx.x * blockDim.x + threadIdx.x;
    const long long unit = t / (2 * LR);
    const int l = (int)(t % LR), odd = (int)(t / LR) & 1;
    const int pair = (int)(unit / a.c.Hkv);
    p.h = (int)(unit % a.c.Hkv);
    p.w = l >> 2;
    p.c = l & 3;
    p.packed = -1;
    p.row = 0;
    int lo = 0, hi = a.sl.n;                              // the sequence that owns the pair
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (a.pairs.v[mid] <= pair) lo = mid;
        else hi = mid;
    }
    p.b = lo;
    p.slot = a.sl.slot[lo];
    if (pair >= a.pairs.v[a.sl.n]) return p;
    const int start = a.start[lo], n = a.cu.v[lo + 1] - a.cu.v[lo];
    if (start < 0 || start >= a.c.max_len) return p;
    p.row = ((start >> 1) + (pair - a.pairs.v[lo])) * 2 + odd;
    const int i = p.row - start;
    if (i >= 0 && i < n && p.row < a.c.max_len) p.packed = a.cu.v[lo] + i;
    return p;
}

template <typename T>
__device__ __forceinline__ void kv4_load8(const void* p, long long i, float (&x)[8]) {
    if constexpr (sizeof(T) == 2) {
        const uint4 w = ld_stream((const uint4*)((const bf16*)p + i));
        x[0] = bf16_lo(w.x); x[1] = bf16_hi(w.x); x[2] = bf16_lo(w.y); x[3] = bf16_hi(w.y);
        x[4] = bf16_lo(w.z); x[5] = bf16_hi(w.z); x[6] = bf16_lo(w.w); x[7] = bf16_hi(w.w);
    } else {
        const float4 u = __ldg((const float4*)((const float*)p + i)), w = __ldg((const float4*)((const float*)p + i + 4));
        x[0] = u.x; x[1] = u.y; x[2] = u.z; x[3] = u.w; x[4] = w.x; x[5] = w.y; x[6] = w.z; x[7] = w.w;
    }
}

// parameters of the group whose 32 values the four lanes of a quad hold (every lane of the warp takes part)
__device__ __forceinline__ uint32_t kv4_group_params(const float (&x)[8]) {
    float lo = x[0], hi = x[0];
    bool finite = true;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        lo = fminf(lo, x[i]);
        hi = fmaxf(hi, x[i]);
        finite &= fabsf(x[i]) < INFINITY;
    }
#pragma unroll
    for (int o = 1; o < 4; o <<= 1) {
        lo = fminf(lo, __shfl_xor_sync(0xffffffffu, lo, o));
        hi = fmaxf(hi, __shfl_xor_sync(0xffffffffu, hi, o));
    }
    const unsigned bad = __ballot_sync(0xffffffffu, !finite);
    return kv4_params(lo, hi, ((bad >> (threadIdx.x & 28)) & 15u) == 0u);
}

// One row's 8 channels of K and of V into the cache.  `live`: the lane has a row; every lane of the warp takes part.
template <int DH>
__device__ __forceinline__ void kv4_store_row(const Kv4View& c, const Kv4Place& p, bool live, const float (&k)[8], const float (&v)[8]) {
    constexpr int LR = DH / 8;
    const uint32_t kp = kv4_group_params(k), vp = kv4_group_params(v);
    const uint32_t kw = kv4_codes8(k, kp), vw = kv4_codes8(v, vp);
    const uint32_t other = __shfl_xor_sync(0xffffffffu, vw, LR);
    const bool both = __shfl_xor_sync(0xffffffffu, live ? 1 : 0, LR) != 0 && live;
    if (!live) return;
    const long long r0 = kv4_row0(c, p.slot, p.h), row = r0 + p.row;
    *(uint32_t*)(c.k_codes + kv4_k_offset(DH, row, p.w, p.c)) = kw;
    if (p.c == 0) {
        c.k_params[row * (DH / 32) + p.w] = kp;
        c.v_params[row * (DH / 32) + p.w] = vp;
    }
    const bool odd = (p.row & 1) != 0;
    if (both) {
        // the pair's words are whole: the even row's lane writes the first, the odd row's the second
        const uint32_t word = odd ? ((other >> 16) | (vw & 0xFFFF0000u)) : ((vw & 0xFFFFu) | (other << 16));
        *(uint32_t*)(c.v_codes + kv4_v_offset(DH, row & ~1ll, p.w, 2 * p.c + (odd ? 1 : 0))) = word;
    } else {
        *(uint16_t*)(c.v_codes + kv4_v_offset(DH, row, p.w, 2 * p.c)) = (uint16_t)vw;
        *(uint16_t*)(c.v_codes + kv4_v_offset(DH, row, p.w, 2 * p.c + 1)) = (uint16_t)(vw >> 16);
    }
}

template <int DH, typename T>
__global__ void __launch_bounds__(256) kv4_append_kernel(const __grid_constant__ Kv4RowsArgs a) {
    pdl_wait();
    pdl_trigger();
    const Kv4Place p = kv4_place<DH>(a);
    float k[8] = {0.f}, v[8] = {0.f};
    if (p.packed >= 0) {
        const long long i = (long long)p.packed * a.ld + p.h * DH + 32 * p.w + 8 * p.c;
        kv4_load8<T>(a.k, i, k);
        kv4_load8<T>(a.v, i, v);
    }
    kv4_store_row<DH>(a.c, p, p.packed >= 0, k, v);
}

template <int DH>
__global__ void __launch_bounds__(256) kv4_read_kernel(const __grid_constant__ Kv4RowsArgs a) {
    pdl_wait();
    pdl_trigger();
    const Kv4Place p = kv4_place<DH>(a);
    if (p.packed < 0) return;
    const long long row = kv4_row0(a.c, p.slot, p.h) + p.row;
    const uint32_t kp = a.c.k_params[row * (DH / 32) + p.w], vp = a.c.v_params[row * (DH / 32) + p.w];
    const uint32_t kw = *(const uint32_t*)(a.c.k_codes + kv4_k_offset(DH, row, p.w, p.c));
    const uint32_t v0 = *(const uint16_t*)(a.c.v_codes + kv4_v_offset(DH, row, p.w, 2 * p.c));
    const uint32_t v1 = *(const uint16_t*)(a.c.v_codes + kv4_v_offset(DH, row, p.w, 2 * p.c + 1));
    const uint32_t vw = v0 | (v1 << 16);
    float k[8], v[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        k[i] = fmaf((float)((kw >> (4 * i)) & 15u), kv4_scale(kp), kv4_min(kp));
        v[i] = fmaf((float)((vw >> (4 * i)) & 15u), kv4_scale(vp), kv4_min(vp));
    }
    const long long o = ((long long)p.packed * a.c.Hkv + p.h) * DH + 32 * p.w + 8 * p.c;
#pragma unroll
    for (int q = 0; q < 2; ++q) {
        *(float4*)(a.out_k + o + 4 * q) = make_float4(k[4 * q], k[4 * q + 1], k[4 * q + 2], k[4 * q + 3]);
        *(float4*)(a.out_v + o + 4 * q) = make_float4(v[4 * q], v[4 * q + 1], v[4 * q + 2], v[4 * q + 3]);
    }
}

// ------------------------------------------------------------------------------------------------ attention
// For each KV head the queries of all its rows and query heads are the columns of one problem: S^T = K Q^T and O^T = V^T P^T with
// the cache as the A operand of mma.m16n8k16 (16 keys, or 16 channels) and eight queries as B, so that one query costs no more
// than eight.  For bf16 codes reach the tensor core as fp16 subnormals (n 2^-24: a mask, no conversion), every second nibble as 16 n with
// its query, or its output, scaled by 1/16.  Scales stay outside: per group of 32 channels S = sum s_g (q_g . n) + m_g sum(q_g),
// and O_g = sum_r (p_r s_rg) n_r + sum_r p_r m_rg, the second sums in fp32 beside the products.
//
// Precision.  bf16 queries are exact in fp16 once their row is scaled by a power of two (what is below 2^-29 of the row's largest
// is rounded there); probabilities are rounded to fp16's 11 bits, 2^-12 of each, which the 2^-9 of the bf16 result hides.  fp32
// queries and their probabilities go in as two fp16 numbers (22 bits), the codes as whole numbers, and the products of 16 rows are
// added up in fp32 outside the tensor core.
//
// A cluster of up to 16 CTAs shares one (sequence, KV head, block of columns); a warp takes every (4 * CTAs)-th tile of 16 rows and
// keeps its own maximum, sum and output.  They are joined in shared memory, then over the cluster, always in the same order.
#define KV4_WARPS 4
#define KV4_MAX_CLUSTER 16

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
};

template <int Q>
struct Kv4Tile {               // a lane's part of 16 rows: chunk lane % 4 of the keys lane / 4 and lane / 4 + 8; chunk lane / 4 of the
    uint32_t k0[Q], k1[Q], v0[Q], v1[Q];        // pairs of values lane % 4 and lane % 4 + 4; the parameters of its two keys' rows
    uint32_t kp0[Q], kp1[Q], vp0[Q], vp1[Q];
};
template <int Q>
__device__ __forceinline__ void kv4_ld(const void* p, uint32_t (&w)[Q]) {
    if constexpr (Q == 4) {
        const uint4 x = ld_stream((const uint4*)p);
        w[0] = x.x; w[1] = x.y; w[2] = x.z; w[3] = x.w;
    } else {
        const uint2 x = __ldg((const uint2*)p);
        w[0] = x.x; w[1] = x.y;
    }
}
template <int DH>
__device__ __forceinline__ void kv4_load_tile(const Kv4View& c, long long row, int lane, Kv4Tile<DH / 32>& t) {
    constexpr int Q = DH / 32, RB = DH / 2, CH = DH / 8;
    const int g = lane >> 2, l = lane & 3;
    kv4_ld<Q>(c.k_codes + (row + g) * RB + l * CH, t.k0);
    kv4_ld<Q>(c.k_codes + (row + g + 8) * RB + l * CH, t.k1);
    kv4_ld<Q>(c.k_params + (row + g) * Q, t.kp0);
    kv4_ld<Q>(c.k_params + (row + g + 8) * Q, t.kp1);
    kv4_ld<Q>(c.v_codes + (row + 2 * l) * RB + g * CH, t.v0);
    kv4_ld<Q>(c.v_codes + (row + 2 * l + 8) * RB + g * CH, t.v1);
    kv4_ld<Q>(c.v_params + (row + g) * Q, t.vp0);
    kv4_ld<Q>(c.v_params + (row + g + 8) * Q, t.vp1);
}

__device__ __forceinline__ void kv4_mma(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                 : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t kv4_half2(float x, float y) {
    const __half2 h = __floats2half2_rn(x, y);
    return *(const uint32_t*)&h;
}
__device__ __forceinline__ float2 kv4_unhalf2(uint32_t w) { return __half22float2(*(const __half2*)&w); }
__device__ __forceinline__ uint32_t kv4_transpose(uint32_t x) {
    uint32_t y;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
    return y;
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

// ---- the state of a warp: running maximum, sum and output of its columns
template <int DH, int NT>
struct Kv4State {
    float m[NT][2], l[NT][2];          // of columns 2 (lane % 4) and + 1 of every block of eight; l: this lane's rows only
    float o[NT][DH / 16][4];           // V^T P^T, scaled by R and the codes' unit
    float mn[NT][DH / 32][2];          // sum of p m per group, this lane's rows only
    float R;                           // power of two that brings the values' scales to 2^5 .. 2^6
};

template <int DH, int NT>
__device__ __forceinline__ void kv4_rescale(Kv4State<DH, NT>& st, int t, float f0, float f1) {
#pragma unroll
    for (int i = 0; i < DH / 16; ++i) { st.o[t][i][0] *= f0; st.o[t][i][1] *= f1; st.o[t][i][2] *= f0; st.o[t][i][3] *= f1; }
#pragma unroll
    for (int w = 0; w < DH / 32; ++w) { st.mn[t][w][0] *= f0; st.mn[t][w][1] *= f1; }
    st.l[t][0] *= f0;
    st.l[t][1] *= f1;
}
__device__ __forceinline__ float kv4_max_rows(float x) {       // over the lanes that hold other rows of the same columns
    x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 4));
    x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 8));
    return fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 16));
}
__device__ __forceinline__ float kv4_sum_rows(float x) {
    x += __shfl_xor_sync(0xffffffffu, x, 4);
    x += __shfl_xor_sync(0xffffffffu, x, 8);
    return x + __shfl_xor_sync(0xffffffffu, x, 16);
}

template <int DH, int NT, typename T>
__global__ void __launch_bounds__(KV4_WARPS * 32) kv4_attn_kernel(const __grid_constant__ Kv4AttnArgs a) {
    constexpr int Q = DH / 32, NB = 8 * NT, LDO = DH + 4;
    constexpr bool SPLIT = sizeof(T) == 4;
    constexpr float UNIT = SPLIT ? 1.f : 0x1p-24f;     // what a code of 1 is to the tensor core
    constexpr float LAZY = 8.f;        // the running maximum is raised once a score is above it by 2^8 (see the state's R: p s R < 2^14)
    extern __shared__ float sm[];
    float* sO = sm;                                 // [warp][column][LDO]
    float* sM = sO + KV4_WARPS * NB * LDO;          // [warp][column]
    float* sL = sM + KV4_WARPS * NB;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g = lane >> 2, c = lane & 3;
    const int b = blockIdx.z, h = blockIdx.y / a.n_blocks, j0 = (blockIdx.y % a.n_blocks) * NB;
    const int rank = blockIdx.x, S = gridDim.x;     // (a cluster is the x extent of the grid)
    pdl_wait();
    pdl_trigger();
    const int nrows = min(max(a.rows[b], 0), a.c.max_len);
    const int i_first = j0 / a.G, i_last = min(j0 + NB, a.ncol) - 1 < 0 ? 0 : (min(j0 + NB, a.ncol) - 1) / a.G;
    // rows [0, clear) are visible to every column of the block, rows from `end` on to none
    const int clear = max(0, a.mask ? nrows - a.mask_rows : nrows - a.n_q + i_first + 1);
    const int end = max(0, a.mask ? nrows : nrows - a.n_q + i_last + 1);
    const int ntile = (end + 15) >> 4;
    const long long row0 = kv4_row0(a.c, a.sl.slot[b], h);

    int t = rank * KV4_WARPS + warp;
    const int step = S * KV4_WARPS;
    Kv4Tile<Q> tile;
    if (t < ntile) kv4_load_tile<DH>(a.c, row0 + t * 16, lane, tile);

    // ---- queries: column lane / 4 of every block of eight, channels 32 w + 8 (lane % 4) + 0..7 of every group
    uint32_t qb[NT][2 * Q][2], ql[SPLIT ? NT : 1][2 * Q][2];
    float fq[NT][2], qs[NT][Q][2];      // of columns 2 c and 2 c + 1: what a sum is to be multiplied with; sum of q per group
    int ci[NT][2];                      // query row of those columns
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        const int j = j0 + 8 * n + g;
        float x[Q][8], mx = 0.f;
#pragma unroll
        for (int w = 0; w < Q; ++w) {
            if (j < a.ncol) {
                const long long at = (long long)(b * a.n_q + j / a.G) * a.q_ld + (h * a.G + j % a.G) * DH + 32 * w + 8 * c;
                kv4_load8<T>(a.q, at, x[w]);
            } else {
#pragma unroll
                for (int i = 0; i < 8; ++i) x[w][i] = 0.f;
            }
#pragma unroll
            for (int i = 0; i < 8; ++i) mx = fmaxf(mx, fabsf(x[w][i]));
        }
        mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 1));
        mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 2));
        const int e = mx > 0.f ? min(max(ilogbf(mx), -100), 100) : 0;
        const float up = scalbnf(1.f, 14 - e);
        float sum[Q];
#pragma unroll
        for (int w = 0; w < Q; ++w) {
            sum[w] = 0.f;
#pragma unroll
            for (int i = 0; i < 8; ++i) x[w][i] *= up;
#pragma unroll
            for (int s = 0; s < 2; ++s) {
                const float y[4] = {x[w][2 * s], x[w][2 * s + 4], x[w][2 * s + 1], x[w][2 * s + 5]};
#pragma unroll
                for (int r = 0; r < 2; ++r) {
                    const uint32_t hi = kv4_half2(y[2 * r], y[2 * r + 1]);
                    const float2 back = kv4_unhalf2(hi);
                    const float f = r ? 0.0625f : 1.f;
                    sum[w] += back.x + back.y;
                    qb[n][2 * w + s][r] = kv4_half2(back.x * f, back.y * f);
                    if constexpr (SPLIT) {
                        const uint32_t lo = kv4_half2(y[2 * r] - back.x, y[2 * r + 1] - back.y);
                        const float2 bl = kv4_unhalf2(lo);
                        sum[w] += bl.x + bl.y;
                        ql[n][2 * w + s][r] = kv4_half2(bl.x * f, bl.y * f);
                    }
                }
            }
            sum[w] += __shfl_xor_sync(0xffffffffu, sum[w], 1);
            sum[w] += __shfl_xor_sync(0xffffffffu, sum[w], 2);
            sum[w] *= UNIT;                                       // in the unit of the products
        }
        const float f = scalbnf(a.scale_log2, e - 14) * (1.f / UNIT);
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            const int from = (2 * c + s) * 4;                     // a lane with lane / 4 = 2 c + s
            fq[n][s] = __shfl_sync(0xffffffffu, f, from);
#pragma unroll
            for (int w = 0; w < Q; ++w) qs[n][w][s] = __shfl_sync(0xffffffffu, sum[w], from);
            const int jc = j0 + 8 * n + 2 * c + s;
            ci[n][s] = jc < a.ncol ? jc / a.G : 0;
        }
    }

    Kv4State<DH, NT> st;
#pragma unroll
    for (int n = 0; n < NT; ++n) {
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            st.m[n][s] = -INFINITY;
            st.l[n][s] = 0.f;
#pragma unroll
            for (int w = 0; w < Q; ++w) st.mn[n][w][s] = 0.f;
        }
#pragma unroll
        for (int i = 0; i < DH / 16; ++i)
#pragma unroll
            for (int s = 0; s < 4; ++s) st.o[n][i][s] = 0.f;
    }
    st.R = 0x1p120f;

    for (; t < ntile; t += step) {
        Kv4Tile<Q> cur = tile;
        if (t + step < ntile) kv4_load_tile<DH>(a.c, row0 + (t + step) * 16, lane, tile);
        const int r0 = t * 16 + g, r1 = r0 + 8;                   // this lane's rows
        const bool edge = t * 16 + 16 > clear;                    // some row is not for every column
        if (edge) {
            // what lies behind the last row is anything at all
#pragma unroll
            for (int w = 0; w < Q; ++w) {
                if (r0 >= nrows) cur.kp0[w] = cur.vp0[w] = 0u;
                if (r1 >= nrows) cur.kp1[w] = cur.vp1[w] = 0u;
            }
        }
        // ---- scores
        float s[NT][4];
#pragma unroll
        for (int n = 0; n < NT; ++n) s[n][0] = s[n][1] = s[n][2] = s[n][3] = 0.f;
#pragma unroll
        for (int w = 0; w < Q; ++w) {
            const uint32_t x0 = cur.k0[w], x1 = cur.k1[w], y0 = x0 >> 8, y1 = x1 >> 8;
            const uint32_t f0 = kv4_lo<SPLIT>(x0), f1 = kv4_lo<SPLIT>(x1), f2 = kv4_hi<SPLIT>(x0), f3 = kv4_hi<SPLIT>(x1);
            const uint32_t h0 = kv4_lo<SPLIT>(y0), h1 = kv4_lo<SPLIT>(y1), h2 = kv4_hi<SPLIT>(y0), h3 = kv4_hi<SPLIT>(y1);
            const float sc0 = kv4_scale(cur.kp0[w]), sc1 = kv4_scale(cur.kp1[w]), mn0 = kv4_min(cur.kp0[w]), mn1 = kv4_min(cur.kp1[w]);
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                float d[4] = {0.f, 0.f, 0.f, 0.f};
                kv4_mma(d, f0, f1, f2, f3, qb[n][2 * w][0], qb[n][2 * w][1]);
                kv4_mma(d, h0, h1, h2, h3, qb[n][2 * w + 1][0], qb[n][2 * w + 1][1]);
                if constexpr (SPLIT) {
                    kv4_mma(d, f0, f1, f2, f3, ql[n][2 * w][0], ql[n][2 * w][1]);
                    kv4_mma(d, h0, h1, h2, h3, ql[n][2 * w + 1][0], ql[n][2 * w + 1][1]);
                }
                s[n][0] = fmaf(mn0, qs[n][w][0], fmaf(sc0, d[0], s[n][0]));
                s[n][1] = fmaf(mn0, qs[n][w][1], fmaf(sc0, d[1], s[n][1]));
                s[n][2] = fmaf(mn1, qs[n][w][0], fmaf(sc1, d[2], s[n][2]));
                s[n][3] = fmaf(mn1, qs[n][w][1], fmaf(sc1, d[3], s[n][3]));
            }
        }
        bool raise = edge;
#pragma unroll
        for (int n = 0; n < NT; ++n) {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                s[n][e] *= fq[n][e & 1];
                if (edge) {
                    const int r = e < 2 ? r0 : r1, i = ci[n][e & 1];
                    bool see;
                    if (!a.mask) {
                        see = r <= nrows - a.n_q + i;
                    } else {
                        const int k = r - (nrows - a.mask_rows);
                        see = k < 0 || (r < nrows && ((a.mask[((long long)b * a.n_q + i) * a.mask_words + (k >> 5)] >> (k & 31)) & 1u));
                    }
                    if (!see) s[n][e] = -INFINITY;
                }
                raise |= s[n][e] > st.m[n][e & 1] + LAZY;
            }
        }
        if (__any_sync(0xffffffffu, raise)) {
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                float f[2];
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const float m = fmaxf(st.m[n][e], kv4_max_rows(fmaxf(s[n][e], s[n][e + 2])));
                    f[e] = m == st.m[n][e] ? 1.f : exp2f(st.m[n][e] - m);
                    st.m[n][e] = m;
                }
                kv4_rescale<DH, NT>(st, n, f[0], f[1]);
            }
        }
        // ---- the values' scales, as multiples of 1 / R
        {
            uint32_t top = 0u;
#pragma unroll
            for (int w = 0; w < Q; ++w) top = max(top, max(cur.vp0[w], cur.vp1[w]));
            if (__any_sync(0xffffffffu, top >= __float_as_uint(64.f / st.R))) {
                uint32_t fin = 0u;                                  // (rows that hold a NaN decide nothing)
#pragma unroll
                for (int w = 0; w < Q; ++w) {
                    if (cur.vp0[w] < 0x7F800000u) fin = max(fin, cur.vp0[w]);
                    if (cur.vp1[w] < 0x7F800000u) fin = max(fin, cur.vp1[w]);
                }
                fin = __reduce_max_sync(0xffffffffu, fin);
                const float R = __uint_as_float((uint32_t)(127 + 5 + 127 - min(max((int)(fin >> 23), 12), 250)) << 23);
                if (R < st.R) {
                    const float f = R / st.R;
#pragma unroll
                    for (int n = 0; n < NT; ++n)
#pragma unroll
                        for (int i = 0; i < DH / 16; ++i)
#pragma unroll
                            for (int e = 0; e < 4; ++e) st.o[n][i][e] *= f;
                    st.R = R;
                }
            }
        }
        // ---- probabilities, and the part of the output that the codes do not carry
#pragma unroll
        for (int n = 0; n < NT; ++n) {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float m = st.m[n][e & 1];
                s[n][e] = exp2f(s[n][e] - (m == -INFINITY ? 0.f : m));
            }
            st.l[n][0] += s[n][0] + s[n][2];
            st.l[n][1] += s[n][1] + s[n][3];
        }
#pragma unroll
        for (int w = 0; w < Q; ++w) {
            const float a0 = kv4_scale(cur.vp0[w]) * st.R, a1 = kv4_scale(cur.vp1[w]) * st.R, mn0 = kv4_min(cur.vp0[w]), mn1 = kv4_min(cur.vp1[w]);
            const uint32_t x0 = cur.v0[w], x1 = cur.v1[w], y0 = x0 >> 8, y1 = x1 >> 8;
            const uint32_t f0 = kv4_lo<SPLIT>(x0), f1 = kv4_hi<SPLIT>(x0), f2 = kv4_lo<SPLIT>(x1), f3 = kv4_hi<SPLIT>(x1);
            const uint32_t g0 = kv4_lo<SPLIT>(y0), g1 = kv4_hi<SPLIT>(y0), g2 = kv4_lo<SPLIT>(y1), g3 = kv4_hi<SPLIT>(y1);
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                float p[4] = {s[n][0] * a0, s[n][1] * a0, s[n][2] * a1, s[n][3] * a1};
                if (edge) {
                    // a column that does not see the row takes nothing of it, not even a NaN
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        if (s[n][e] == 0.f) p[e] = 0.f;
                    st.mn[n][w][0] += (s[n][0] == 0.f ? 0.f : s[n][0] * mn0) + (s[n][2] == 0.f ? 0.f : s[n][2] * mn1);
                    st.mn[n][w][1] += (s[n][1] == 0.f ? 0.f : s[n][1] * mn0) + (s[n][3] == 0.f ? 0.f : s[n][3] * mn1);
                } else {
                    st.mn[n][w][0] = fmaf(s[n][0], mn0, fmaf(s[n][2], mn1, st.mn[n][w][0]));
                    st.mn[n][w][1] = fmaf(s[n][1], mn0, fmaf(s[n][3], mn1, st.mn[n][w][1]));
                }
                const uint32_t h0 = kv4_half2(p[0], p[1]), h1 = kv4_half2(p[2], p[3]);
                const uint32_t b0 = kv4_transpose(h0), b1 = kv4_transpose(h1);
                if constexpr (SPLIT) {
                    const float2 w0 = kv4_unhalf2(h0), w1 = kv4_unhalf2(h1);
                    const uint32_t c0 = kv4_transpose(kv4_half2(p[0] - w0.x, p[1] - w0.y)), c1 = kv4_transpose(kv4_half2(p[2] - w1.x, p[3] - w1.y));
                    float d[4] = {0.f, 0.f, 0.f, 0.f}, u[4] = {0.f, 0.f, 0.f, 0.f};
                    kv4_mma(d, f0, f1, f2, f3, c0, c1);
                    kv4_mma(d, f0, f1, f2, f3, b0, b1);
                    kv4_mma(u, g0, g1, g2, g3, c0, c1);
                    kv4_mma(u, g0, g1, g2, g3, b0, b1);
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        st.o[n][2 * w][e] += d[e];
                        st.o[n][2 * w + 1][e] += u[e];
                    }
                } else {
                    kv4_mma(st.o[n][2 * w], f0, f1, f2, f3, b0, b1);
                    kv4_mma(st.o[n][2 * w + 1], g0, g1, g2, g3, b0, b1);
                }
            }
        }
    }

    // ---- this warp's columns to shared memory: maximum, sum, output
    const float down = (1.f / UNIT) / st.R;
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            const int col = 8 * n + 2 * c + s;
            const float l = kv4_sum_rows(st.l[n][s]);
            if (g == 0) {
                sM[warp * NB + col] = st.m[n][s];
                sL[warp * NB + col] = l;
            }
#pragma unroll
            for (int w = 0; w < Q; ++w) {
                const float m = kv4_sum_rows(st.mn[n][w][s]);
                // channels 32 w + 4 g + 0..3: rows g and g + 8 of the two blocks of 16, the latter sixteenfold
                *(float4*)(sO + (warp * NB + col) * LDO + 32 * w + 4 * g) =
                    make_float4(fmaf(st.o[n][2 * w][s], down, m), fmaf(st.o[n][2 * w][2 + s], down * 0.0625f, m),
                                fmaf(st.o[n][2 * w + 1][s], down, m), fmaf(st.o[n][2 * w + 1][2 + s], down * 0.0625f, m));
            }
        }
    __syncthreads();
    // ---- the four warps of the CTA, into the first one's place
    const int cols = min(NB, a.ncol - j0);
    for (int i = tid; i < cols * (DH / 4); i += KV4_WARPS * 32) {
        const int col = i / (DH / 4), ch = (i % (DH / 4)) * 4;
        float m = -INFINITY;
#pragma unroll
        for (int w = 0; w < KV4_WARPS; ++w) m = fmaxf(m, sM[w * NB + col]);
        float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
        for (int w = 0; w < KV4_WARPS; ++w) {
            const float mw = sM[w * NB + col];
            if (mw == -INFINITY && m > -INFINITY) continue;        // (nothing seen; where every warp saw nothing all is zero)
            const float f = m == mw ? 1.f : exp2f(mw - m);
            const float4 x = *(const float4*)(sO + (w * NB + col) * LDO + ch);
            o.x = fmaf(x.x, f, o.x); o.y = fmaf(x.y, f, o.y); o.z = fmaf(x.z, f, o.z); o.w = fmaf(x.w, f, o.w);
        }
        *(float4*)(sO + col * LDO + ch) = o;
    }
    __syncthreads();
    if (tid < cols) {
        float m = -INFINITY, l = 0.f;
#pragma unroll
        for (int w = 0; w < KV4_WARPS; ++w) m = fmaxf(m, sM[w * NB + tid]);
#pragma unroll
        for (int w = 0; w < KV4_WARPS; ++w) {
            const float mw = sM[w * NB + tid];
            if (mw > -INFINITY || mw != mw) l = fmaf(sL[w * NB + tid], m == mw ? 1.f : exp2f(mw - m), l);
        }
        sM[tid] = m;
        sL[tid] = l;
    }
    cg::cluster_group cluster = cg::this_cluster();
    if (S > 1) cluster.sync();
    else __syncthreads();
    // ---- the CTAs of the cluster: each writes its share of the columns' channels
    for (int i = rank * KV4_WARPS * 32 + tid; i < cols * (DH / 4); i += S * KV4_WARPS * 32) {
        const int col = i / (DH / 4), ch = (i % (DH / 4)) * 4;
        float m = -INFINITY;
        for (int r = 0; r < S; ++r) m = fmaxf(m, *(S > 1 ? cluster.map_shared_rank(sM + col, r) : sM + col));
        float l = 0.f;
        float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
        for (int r = 0; r < S; ++r) {
            const float mr = *(S > 1 ? cluster.map_shared_rank(sM + col, r) : sM + col);
            const float lr = *(S > 1 ? cluster.map_shared_rank(sL + col, r) : sL + col);
            const float4 x = *(const float4*)(S > 1 ? cluster.map_shared_rank(sO + col * LDO + ch, r) : sO + col * LDO + ch);
            if (mr == -INFINITY && m > -INFINITY) continue;
            const float f = m == mr ? 1.f : exp2f(mr - m);
            l = fmaf(lr, f, l);
            o.x = fmaf(x.x, f, o.x); o.y = fmaf(x.y, f, o.y); o.z = fmaf(x.z, f, o.z); o.w = fmaf(x.w, f, o.w);
        }
        const float inv = l == 0.f ? 0.f : 1.f / l;                // nothing visible: zeros
        const int j = j0 + col;
        const long long at = (long long)(b * a.n_q + j / a.G) * a.out_ld + (h * a.G + j % a.G) * DH + ch;
        if constexpr (sizeof(T) == 2) {
            const __nv_bfloat162 u = __floats2bfloat162_rn(o.x * inv, o.y * inv), v = __floats2bfloat162_rn(o.z * inv, o.w * inv);
            *(uint2*)((bf16*)a.out + at) = make_uint2(*(const unsigned*)&u, *(const unsigned*)&v);
        } else {
            *(float4*)((float*)a.out + at) = make_float4(o.x * inv, o.y * inv, o.z * inv, o.w * inv);
        }
    }
    if (S > 1) cluster.sync();          // nobody leaves while its shared memory may still be read
}

// CTAs per (sequence, KV head, block of columns): a power of two, so many that the GPU's SMs have about four CTAs each, but not
// more than there are tiles of 16 rows for their warps at the cache's full length.
static int kv4_cluster(int units, int max_len, int num_sms) {
    int s = 1;
    while (s < KV4_MAX_CLUSTER && units * s < 4 * num_sms && s * 2 * KV4_WARPS * 16 <= max_len) s *= 2;
    return s;
}

template <int DH, int NT, typename T>
static cudaError_t kv4_launch_attn(Kv4AttnArgs& a, int dev, int num_sms, cudaStream_t st) {
    constexpr int NB = 8 * NT;
    const size_t smem = sizeof(float) * KV4_WARPS * NB * (DH + 4 + 2);
    auto kernel = kv4_attn_kernel<DH, NT, T>;
    static bool attr_set[HIVIS_MAX_DEVICES] = {false};
    if (dev < 0 || dev >= HIVIS_MAX_DEVICES || !attr_set[dev]) {
        cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
        if (e == cudaSuccess) e = cudaFuncSetAttribute(kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
        if (e != cudaSuccess) return e;
        if (dev >= 0 && dev < HIVIS_MAX_DEVICES) attr_set[dev] = true;
    }
    a.n_blocks = (a.ncol + NB - 1) / NB;
    const int S = kv4_cluster(a.sl.n * a.c.Hkv * a.n_blocks, a.c.max_len, num_sms);
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)S, (unsigned)(a.c.Hkv * a.n_blocks), (unsigned)a.sl.n);
    cfg.blockDim = dim3(KV4_WARPS * 32);
    cfg.dynamicSmemBytes = smem;
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

template <int DH, typename T>
static cudaError_t kv4_launch_attn_n(Kv4AttnArgs& a, int dev, int num_sms, cudaStream_t st) {
    if (a.ncol <= 8) return kv4_launch_attn<DH, 1, T>(a, dev, num_sms, st);
    return kv4_launch_attn<DH, 2, T>(a, dev, num_sms, st);
}

// ------------------------------------------------------------------------------------------------ C entries
#define KV4_FAIL(code, ...)                                   \
    do {                                                      \
        char msg_[200];                                       \
        snprintf(msg_, sizeof(msg_), __VA_ARGS__);            \
        hivis_set_global_error(msg_);                         \
        return code;                                          \
    } while (0)

static bool kv4_misaligned(const void* p) { return (((uintptr_t)p) & 15u) != 0; }

static int kv4_check(const char* who, const hivis_kv4_cache* cache, int B, const int* slots_host, Kv4View* c, SlotList* sl) {
    if (!cache) KV4_FAIL(HIVIS_ERR_ARG, "%s: null cache", who);
    if (cache->struct_size != sizeof(hivis_kv4_cache)) KV4_FAIL(HIVIS_ERR_ARG, "%s: struct_size mismatch", who);
    if (cache->head_dim != 64 && cache->head_dim != 128) KV4_FAIL(HIVIS_ERR_SHAPE, "%s: head_dim must be 64 or 128", who);
    if (cache->n_kv_heads < 1 || cache->n_kv_heads > 65535 || cache->n_slots < 1) KV4_FAIL(HIVIS_ERR_SHAPE, "%s: n_kv_heads or n_slots out of range", who);
    if (cache->max_len < 32 || cache->max_len % 32 || cache->max_len > (1 << 28))
        KV4_FAIL(HIVIS_ERR_SHAPE, "%s: max_len must be a positive multiple of 32, at most 2^28", who);
    if (!cache->k_codes || !cache->v_codes || !cache->k_params || !cache->v_params) KV4_FAIL(HIVIS_ERR_ARG, "%s: null buffer in the cache", who);
    if (kv4_misaligned(cache->k_codes) || kv4_misaligned(cache->v_codes) || kv4_misaligned(cache->k_params) || kv4_misaligned(cache->v_params))
        KV4_FAIL(HIVIS_ERR_ARG, "%s: a cache buffer is not 16-byte aligned", who);
    if (B < 1 || B > HIVIS_MAX_BATCH) KV4_FAIL(HIVIS_ERR_CAPACITY, "%s: B=%d outside [1,%d]", who, B, HIVIS_MAX_BATCH);
    sl->n = B;
    for (int b = 0; b < B; ++b) {
        const int s = slots_host ? slots_host[b] : b;
        if (s < 0 || s >= cache->n_slots) KV4_FAIL(HIVIS_ERR_ARG, "%s: slot %d out of range", who, s);
        for (int i = 0; i < b; ++i)
            if (sl->slot[i] == s) KV4_FAIL(HIVIS_ERR_ARG, "%s: slot %d listed twice", who, s);
        sl->slot[b] = s;
    }
    c->k_codes = (unsigned char*)cache->k_codes;
    c->v_codes = (unsigned char*)cache->v_codes;
    c->k_params = (uint32_t*)cache->k_params;
    c->v_params = (uint32_t*)cache->v_params;
    c->n_slots = cache->n_slots; c->Hkv = cache->n_kv_heads; c->max_len = cache->max_len; c->dh = cache->head_dim;
    return HIVIS_OK;
}

static int kv4_check_rows(const char* who, const hivis_kv4_cache* cache, int B, const int* slots_host, const int32_t* cu_seqlens_host,
                          const int32_t* start_rows, Kv4RowsArgs* a) {
    memset(a, 0, sizeof(*a));
    int rc = kv4_check(who, cache, B, slots_host, &a->c, &a->sl);
    if (rc) return rc;
    if (!cu_seqlens_host || !start_rows) KV4_FAIL(HIVIS_ERR_ARG, "%s: null argument", who);
    if (kv4_misaligned(start_rows)) KV4_FAIL(HIVIS_ERR_ARG, "%s: device pointer not 16-byte aligned", who);
    if (cu_seqlens_host[0] != 0) KV4_FAIL(HIVIS_ERR_ARG, "%s: cu_seqlens must start at 0", who);
    for (int b = 0; b < B; ++b) {
        const long long n = (long long)cu_seqlens_host[b + 1] - cu_seqlens_host[b];
        if (n < 0) KV4_FAIL(HIVIS_ERR_ARG, "%s: cu_seqlens must not fall", who);
        if (n > cache->max_len) KV4_FAIL(HIVIS_ERR_CAPACITY, "%s: sequence %d brings %lld rows > max_len %d", who, b, n, cache->max_len);
        a->cu.v[b + 1] = cu_seqlens_host[b + 1];
        a->pairs.v[b + 1] = a->pairs.v[b] + (n > 0 ? (int)(n / 2) + 1 : 0);
    }
    a->start = start_rows;
    return HIVIS_OK;
}

static dim3 kv4_rows_grid(const Kv4RowsArgs& a) {
    const long long threads = (long long)a.pairs.v[a.sl.n] * a.c.Hkv * (a.c.dh / 4);
    return dim3((unsigned)((threads + 255) / 256));
}
static bool kv4_rows_too_many(const Kv4RowsArgs& a) {
    return ((long long)a.pairs.v[a.sl.n] * a.c.Hkv * (a.c.dh / 4) + 255) / 256 > 0x7FFFFFFFll;
}

static int kv4_cuda(const char* who, cudaError_t e) {
    if (e == cudaSuccess) return HIVIS_OK;
    cudaGetLastError();
    KV4_FAIL(HIVIS_ERR_CUDA, "%s: launch failed: %s", who, cudaGetErrorString(e));
}

extern "C" int hivis_kv4_append(const hivis_kv4_cache* cache, int B, const int* seq_slots_host, const int32_t* cu_seqlens_host,
                                const int32_t* start_rows, const void* k, const void* v, int dtype, int64_t ld, void* stream) {
    const char* who = "hivis_kv4_append";
    Kv4RowsArgs a;
    int rc = kv4_check_rows(who, cache, B, seq_slots_host, cu_seqlens_host, start_rows, &a);
    if (rc) return rc;
    if (dtype != HIVIS_F32 && dtype != HIVIS_BF16) KV4_FAIL(HIVIS_ERR_DTYPE, "%s: unknown dtype", who);
    if (a.cu.v[B] == 0) return HIVIS_OK;
    if (!k || !v) KV4_FAIL(HIVIS_ERR_ARG, "%s: null argument", who);
    if (kv4_misaligned(k) || kv4_misaligned(v)) KV4_FAIL(HIVIS_ERR_ARG, "%s: device pointer not 16-byte aligned", who);
    if (ld % 8 || ld < (int64_t)a.c.Hkv * a.c.dh) KV4_FAIL(HIVIS_ERR_SHAPE, "%s: ld must be a multiple of 8 of at least n_kv_heads * head_dim", who);
    if (kv4_rows_too_many(a)) KV4_FAIL(HIVIS_ERR_CAPACITY, "%s: too many rows for one call", who);
    a.k = k; a.v = v; a.ld = ld;
    const dim3 grid = kv4_rows_grid(a), block(256);
    cudaStream_t st = (cudaStream_t)stream;
    cudaError_t e;
    if (dtype == HIVIS_BF16) e = a.c.dh == 128 ? launch_pdl(kv4_append_kernel<128, bf16>, grid, block, 0, st, a) : launch_pdl(kv4_append_kernel<64, bf16>, grid, block, 0, st, a);
    else e = a.c.dh == 128 ? launch_pdl(kv4_append_kernel<128, float>, grid, block, 0, st, a) : launch_pdl(kv4_append_kernel<64, float>, grid, block, 0, st, a);
    return kv4_cuda(who, e);
}

extern "C" int hivis_kv4_read(const hivis_kv4_cache* cache, int B, const int* seq_slots_host, const int32_t* cu_seqlens_host,
                              const int32_t* start_rows, float* out_k, float* out_v, void* stream) {
    const char* who = "hivis_kv4_read";
    Kv4RowsArgs a;
    int rc = kv4_check_rows(who, cache, B, seq_slots_host, cu_seqlens_host, start_rows, &a);
    if (rc) return rc;
    if (a.cu.v[B] == 0) return HIVIS_OK;
    if (!out_k || !out_v) KV4_FAIL(HIVIS_ERR_ARG, "%s: null argument", who);
    if (kv4_misaligned(out_k) || kv4_misaligned(out_v)) KV4_FAIL(HIVIS_ERR_ARG, "%s: device pointer not 16-byte aligned", who);
    if (kv4_rows_too_many(a)) KV4_FAIL(HIVIS_ERR_CAPACITY, "%s: too many rows for one call", who);
    a.out_k = out_k; a.out_v = out_v;
    const dim3 grid = kv4_rows_grid(a), block(256);
    cudaStream_t st = (cudaStream_t)stream;
    return kv4_cuda(who, a.c.dh == 128 ? launch_pdl(kv4_read_kernel<128>, grid, block, 0, st, a) : launch_pdl(kv4_read_kernel<64>, grid, block, 0, st, a));
}

extern "C" int hivis_kv4_attention(const hivis_kv4_cache* cache, int B, const int* seq_slots_host, const int32_t* rows, int n_q,
                                   int n_q_heads, const void* q, int dtype, int64_t q_ld, float scale, const uint32_t* mask,
                                   int mask_rows, void* out, int64_t out_ld, void* stream) {
    const char* who = "hivis_kv4_attention";
    Kv4AttnArgs a;
    memset(&a, 0, sizeof(a));
    int rc = kv4_check(who, cache, B, seq_slots_host, &a.c, &a.sl);
    if (rc) return rc;
    if (dtype != HIVIS_F32 && dtype != HIVIS_BF16) KV4_FAIL(HIVIS_ERR_DTYPE, "%s: unknown dtype", who);
    if (!rows || !q || !out) KV4_FAIL(HIVIS_ERR_ARG, "%s: null argument", who);
    if (kv4_misaligned(rows) || kv4_misaligned(q) || kv4_misaligned(out) || kv4_misaligned(mask))
        KV4_FAIL(HIVIS_ERR_ARG, "%s: device pointer not 16-byte aligned", who);
    if (n_q < 1 || n_q > HIVIS_KV4_MAX_QUERIES) KV4_FAIL(HIVIS_ERR_CAPACITY, "%s: n_q=%d outside [1,%d]", who, n_q, HIVIS_KV4_MAX_QUERIES);
    if (n_q_heads < 1 || n_q_heads % a.c.Hkv) KV4_FAIL(HIVIS_ERR_SHAPE, "%s: n_q_heads must be a multiple of n_kv_heads", who);
    if (q_ld % 8 || out_ld % 8 || q_ld < (int64_t)n_q_heads * a.c.dh || out_ld < (int64_t)n_q_heads * a.c.dh)
        KV4_FAIL(HIVIS_ERR_SHAPE, "%s: q_ld and out_ld must be multiples of 8 of at least n_q_heads * head_dim", who);
    if (!(scale > 0.f) || !(scale < 3e38f)) KV4_FAIL(HIVIS_ERR_ARG, "%s: scale must be positive", who);
    if (mask && (mask_rows < 1 || mask_rows > HIVIS_KV4_MAX_MASK))
        KV4_FAIL(HIVIS_ERR_CAPACITY, "%s: mask_rows=%d outside [1,%d]", who, mask_rows, HIVIS_KV4_MAX_MASK);
    a.rows = rows; a.q = q; a.q_ld = q_ld; a.n_q = n_q; a.Hq = n_q_heads; a.G = n_q_heads / a.c.Hkv; a.ncol = n_q * a.G;
    a.scale_log2 = (float)((double)scale * 1.4426950408889634);
    a.mask = mask; a.mask_rows = mask ? mask_rows : 0; a.mask_words = (a.mask_rows + 31) / 32;
    a.out = out; a.out_ld = out_ld;
    if ((long long)a.c.Hkv * ((a.ncol + 7) / 8) > 65535) KV4_FAIL(HIVIS_ERR_SHAPE, "%s: too many heads and queries for one call", who);
    int dev = 0, sms = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e == cudaSuccess) e = cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev);
    if (e != cudaSuccess) return kv4_cuda(who, e);
    cudaStream_t st = (cudaStream_t)stream;
    if (dtype == HIVIS_BF16) e = a.c.dh == 128 ? kv4_launch_attn_n<128, bf16>(a, dev, sms, st) : kv4_launch_attn_n<64, bf16>(a, dev, sms, st);
    else e = a.c.dh == 128 ? kv4_launch_attn_n<128, float>(a, dev, sms, st) : kv4_launch_attn_n<64, float>(a, dev, sms, st);
    return kv4_cuda(who, e);
}
