// The 4-bit key/value cache: rows go in (quantised), come out (as fp32 values), and are attended over, for callers with a cache of
// their own (no context or workspace) and for the drafter contexts that keep theirs so.  kv4.cuh has the format.
#include <cstdio>
#include <cstring>
#include <type_traits>

#include <cooperative_groups.h>

#include "attn_body.cuh"
#include "kv4_attn.cuh"

namespace cg = cooperative_groups;

// ------------------------------------------------------------------------------------------------ rows in and out
struct Kv4RowsArgs {
    Kv4View c;
    SlotList sl;
    CuSeqlens cu;              // packed rows: sequence b owns [cu.v[b], cu.v[b + 1])
    CuSeqlens pairs;           // append: first pair of rows of each sequence: half its rows and one, whichever way its start is aligned
    const int* start;          // [B] cache row of each sequence's first packed row; nullptr: start_host for all
    int start_host;
    const void *k, *v;         // packed rows [.][ld]
    long long ld;
    float *out_k, *out_v;      // read: [.][Hkv * dh]
    int heads_log2;            // heads side by side in a CTA
};

// the entry of a rising list (at most HIVIS_MAX_BATCH of them) that i lies in
__device__ __forceinline__ int kv4_owner(const CuSeqlens& first, int n, int i) {
    int lo = 0, hi = n;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (first.v[mid] <= i) lo = mid;
        else hi = mid;
    }
    return lo;
}

struct Kv4Place {
    int h, slot, row, w, c;    // KV head, slot, cache row, group, lane of the group
};

// parameters of the group whose 32 values the four lanes of a quad hold (every lane of the warp takes part)
__device__ __forceinline__ uint32_t kv4_group_params(const float (&x)[8]) {
    float lo = kv4_min_nan(kv4_min_nan(kv4_min_nan(x[0], x[1]), kv4_min_nan(x[2], x[3])), kv4_min_nan(kv4_min_nan(x[4], x[5]), kv4_min_nan(x[6], x[7])));
    float hi = kv4_max_nan(kv4_max_nan(kv4_max_nan(x[0], x[1]), kv4_max_nan(x[2], x[3])), kv4_max_nan(kv4_max_nan(x[4], x[5]), kv4_max_nan(x[6], x[7])));
#pragma unroll
    for (int o = 1; o < 4; o <<= 1) {
        lo = kv4_min_nan(lo, __shfl_xor_sync(0xffffffffu, lo, o));
        hi = kv4_max_nan(hi, __shfl_xor_sync(0xffffffffu, hi, o));
    }
    return kv4_params(lo, hi);
}

// One row's 8 channels of K and of V into the cache (four lanes a group).  `live`: the lane has some; every lane of the warp takes part.
template <int DH>
__device__ __forceinline__ void kv4_store_row(const Kv4View& c, const Kv4Place& p, bool live, const float (&k)[8], const float (&v)[8]) {
    const uint32_t kp = kv4_group_params(k), vp = kv4_group_params(v);
    const uint32_t kw = kv4_codes8<true>(k, kp), vw = kv4_codes8<true>(v, vp);
    if (!live) return;
    unsigned char* tile = kv4_tile(c, p.slot, p.h, p.row);
    const int r = p.row % KV4_TILE;
    *(uint32_t*)(tile + kv4_k_at(DH, r, p.w, p.c)) = kw;
    if (p.c == 0) {
        *(uint16_t*)(tile + kv4_s_at(DH, 0, r, p.w)) = (uint16_t)(kp >> 16);
        *(uint16_t*)(tile + kv4_m_at(DH, 0, r, p.w)) = (uint16_t)kp;
        *(uint16_t*)(tile + kv4_s_at(DH, 1, r, p.w)) = (uint16_t)(vp >> 16);
        *(uint16_t*)(tile + kv4_m_at(DH, 1, r, p.w)) = (uint16_t)vp;
    }
    *(uint16_t*)(tile + kv4_v_at(DH, r, p.w, 2 * p.c)) = (uint16_t)vw;
    *(uint16_t*)(tile + kv4_v_at(DH, r, p.w, 2 * p.c + 1)) = (uint16_t)(vw >> 16);
}

// Append: a lane has one group of 32 channels of a row, first K's, then V's, so that nothing is shared but the words of the V codes,
// which the two rows of a pair exchange (DH / 32 lanes further on).  The values are read twice, the second time from L1: for their
// range, then eight at a time for their codes.  6144 rows of 32 heads, bf16: 35 us (their bytes: 20), issue slots 70 % in use; 62 us with
// 8 channels a lane and shuffles for the groups (most of it went into finding the place and the parameters for too few values), 57 us
// with everything unrolled (a third of that waiting for code), 47 us with values next to a tie decided in eight unrolled branches, 37 us in a loop
// that ties take too.
template <int DH, typename T>
__global__ void __launch_bounds__(128) kv4_append_kernel(const __grid_constant__ Kv4RowsArgs a) {
    constexpr int Q = DH / 32, UNITS = 128 / (2 * Q);
    pdl_wait();
    pdl_trigger();
    const int w = threadIdx.x % Q, odd = (threadIdx.x / Q) & 1, unit = threadIdx.x / (2 * Q);
    const int h = (blockIdx.y << a.heads_log2) + (unit & ((1 << a.heads_log2) - 1));
    const int pair = blockIdx.x * (UNITS >> a.heads_log2) + (unit >> a.heads_log2);
    const int b = kv4_owner(a.pairs, a.sl.n, pair);
    int row = 0, packed = -1;
    if (pair < a.pairs.v[a.sl.n] && h < a.c.Hkv) {
        const int start = a.start[b], n = a.cu.v[b + 1] - a.cu.v[b];
        if (start >= 0 && start < a.c.max_len) {
            row = ((start >> 1) + (pair - a.pairs.v[b])) * 2 + odd;
            const int i = row - start;
            if (i >= 0 && i < n && row < a.c.max_len) packed = a.cu.v[b] + i;
        }
    }
    const bool live = packed >= 0, both = __shfl_xor_sync(0xffffffffu, live ? 1 : 0, Q) != 0 && live;
    const long long at = (long long)packed * a.ld + h * DH + 32 * w;
    unsigned char* tile = kv4_tile(a.c, a.sl.slot[b], h, row);
    const int r = row % KV4_TILE;
#pragma unroll 1
    for (int which = 0; which < 2; ++which) {
        const void* src = which == 0 ? a.k : a.v;
        uint32_t params = 0u;
        if (live) {
            float lo, hi;
            if constexpr (sizeof(T) == 2) {
                uint4 u[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) u[i] = __ldg((const uint4*)((const bf16*)src + at) + i);
                const uint32_t* x = (const uint32_t*)u;
                auto two = [&](int i) { return *(const __nv_bfloat162*)&x[i]; };
                __nv_bfloat162 m = two(0), n = two(0);
#pragma unroll
                for (int i = 1; i < 16; ++i) {
                    m = __hmin2_nan(m, two(i));
                    n = __hmax2_nan(n, two(i));
                }
                lo = kv4_min_nan(__low2float(m), __high2float(m));
                hi = kv4_max_nan(__low2float(n), __high2float(n));
            } else {
                float4 u[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) u[i] = __ldg((const float4*)((const float*)src + at) + i);
                const float* x = (const float*)u;
                lo = hi = x[0];
#pragma unroll
                for (int i = 1; i < 32; ++i) {
                    lo = kv4_min_nan(lo, x[i]);
                    hi = kv4_max_nan(hi, x[i]);
                }
            }
            params = kv4_params(lo, hi);
            *(uint16_t*)(tile + kv4_s_at(DH, which, r, w)) = (uint16_t)(params >> 16);
            *(uint16_t*)(tile + kv4_m_at(DH, which, r, w)) = (uint16_t)params;
        }
#pragma unroll 1
        for (int c = 0; c < 4; ++c) {
            float x[8];
            uint32_t codes = 0u;
            if (live) {
                kv4_load8<T>(src, at + 8 * c, x);
                codes = kv4_codes8<sizeof(T) == 2>(x, params);
            }
            if (which == 0) {
                if (live) *(uint32_t*)(tile + kv4_k_at(DH, r, w, c)) = codes;
                continue;
            }
            const uint32_t other = __shfl_xor_sync(0xffffffffu, codes, Q);
            if (both) {
                // the pair's words are whole: the even row's lane writes the first, the odd row's the second
                const uint32_t word = odd ? ((other >> 16) | (codes & 0xFFFF0000u)) : ((codes & 0xFFFFu) | (other << 16));
                *(uint32_t*)(tile + kv4_v_at(DH, r & ~1, w, 2 * c + odd)) = word;
            } else if (live) {
                *(uint16_t*)(tile + kv4_v_at(DH, r, w, 2 * c)) = (uint16_t)codes;
                *(uint16_t*)(tile + kv4_v_at(DH, r, w, 2 * c + 1)) = (uint16_t)(codes >> 16);
            }
        }
    }
}

// Read: a lane has four neighbouring channels of a row, so that a warp writes whole lines, and four rows one after the other, whose
// place is found once unless a tile or a sequence ends between them: 42 us for the same rows (their bytes: 36), 46 with every place on its own.
#define KV4_READ_ROWS 4
template <int DH>
__global__ void __launch_bounds__(256) kv4_read_kernel(const __grid_constant__ Kv4RowsArgs a) {
    constexpr int LR = DH / 4, UNITS = 256 / LR;
    pdl_wait();
    pdl_trigger();
    const int l = threadIdx.x % LR, unit = threadIdx.x / LR, per = UNITS >> a.heads_log2;
    const int h = (blockIdx.y << a.heads_log2) + (unit & ((1 << a.heads_log2) - 1));
    const int j0 = (blockIdx.x * per + (unit >> a.heads_log2)) * KV4_READ_ROWS, total = a.cu.v[a.sl.n];
    if (h >= a.c.Hkv || j0 >= total) return;
    int b = kv4_owner(a.cu, a.sl.n, j0), last = 0, row = 0;
    const int w = l >> 3, at_k = kv4_k_at(DH, 0, w, (l >> 1) & 3) + 2 * (l & 1), at_v = kv4_v_at(DH, 0, w, l & 7);
    const long long head_stride = (long long)(a.c.max_len / KV4_TILE) * kv4_tile_bytes(DH);
    const unsigned char* tile = nullptr;
    uint32_t kw[KV4_READ_ROWS], vw[KV4_READ_ROWS], p[KV4_READ_ROWS][4];
    bool live[KV4_READ_ROWS], inside = false;
#pragma unroll
    for (int u = 0; u < KV4_READ_ROWS; ++u) {
        const int j = j0 + u;
        live[u] = j < total;
        if (!live[u]) break;
        if (u == 0 || j == last) {
            while (j >= a.cu.v[b + 1]) ++b;
            last = a.cu.v[b + 1];
            const int start = a.start ? a.start[b] : a.start_host;
            inside = start >= 0 && start < a.c.max_len;
            row = start + (j - a.cu.v[b]);
            tile = a.c.data + ((long long)a.sl.slot[b] * a.c.Hkv + h) * head_stride + (long long)(row / KV4_TILE) * kv4_tile_bytes(DH);
        } else {
            row += 1;
            if (row % KV4_TILE == 0) tile += kv4_tile_bytes(DH);
        }
        live[u] = inside && row < a.c.max_len;
        if (!live[u]) continue;
        const int r = row % KV4_TILE;
        auto half = [&](int at) { return (uint32_t)__ldg((const unsigned short*)(tile + at)); };
        kw[u] = half(at_k + r * (DH / 2));
        vw[u] = half(at_v + (r & ~1) * (DH / 2) + (r & 1) * 2);
        p[u][0] = half(kv4_s_at(DH, 0, r, w));
        p[u][1] = half(kv4_m_at(DH, 0, r, w));
        p[u][2] = half(kv4_s_at(DH, 1, r, w));
        p[u][3] = half(kv4_m_at(DH, 1, r, w));
    }
    auto value = [](uint32_t codes, int i, uint32_t s, uint32_t m) {
        const float n = __uint_as_float(((codes >> (4 * i)) & 15u) | 0x4B000000u) - 8388608.f;
        return fmaf(n, __uint_as_float(s << 16), __uint_as_float(m << 16));
    };
#pragma unroll
    for (int u = 0; u < KV4_READ_ROWS; ++u) {
        const int j = j0 + u;
        if (j >= total) break;
        if (!live[u]) continue;
        const long long o = ((long long)j * a.c.Hkv + h) * DH + 4 * l;
        *(float4*)(a.out_k + o) = make_float4(value(kw[u], 0, p[u][0], p[u][1]), value(kw[u], 1, p[u][0], p[u][1]),
                                              value(kw[u], 2, p[u][0], p[u][1]), value(kw[u], 3, p[u][0], p[u][1]));
        *(float4*)(a.out_v + o) = make_float4(value(vw[u], 0, p[u][2], p[u][3]), value(vw[u], 1, p[u][2], p[u][3]),
                                              value(vw[u], 2, p[u][2], p[u][3]), value(vw[u], 3, p[u][2], p[u][3]));
    }
}

// ------------------------------------------------------------------------------------------------ rows of a drafter context
// A CTA has one KV head of one row: its first warp rotates and quantises the row (half its lanes: a row alone has no partner), the
// others rotate the head group's queries.  The angles are made once per CTA (fp64, see rope_cs).
template <int DH>
__global__ void __launch_bounds__(128) kv4_put_kernel(Kv4View c, const float* kv, int ld, int k_col, const int* slots, const int* rows,
                                                      int row_add, const double* inv_freq, int G, float* q_out) {
    constexpr int LR = DH / 8, HALF = DH / 2;
    __shared__ float2 s_cs[HALF];
    pdl_wait();
    pdl_trigger();
    const int h = blockIdx.x, j = blockIdx.y, row = rows[j];
    if (row < 0 || row + row_add >= c.max_len) return;
    if (threadIdx.x < HALF) {
        float cs, sn;
        rope_cs(row + row_add, inv_freq[threadIdx.x], cs, sn);
        s_cs[threadIdx.x] = make_float2(cs, sn);
    }
    __syncthreads();
    const float* in = kv + (long long)j * ld;
    if (threadIdx.x < 32) {
        const int lane = threadIdx.x, l = lane % LR;
        const bool live = lane < LR;
        const float* k = in + k_col + h * DH;
        const float* v = k + (long long)c.Hkv * DH;
        float x[8], y[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int e = 8 * l + i;
            const float own = k[e], other = k[e ^ HALF];
            const float2 t = s_cs[e % HALF];
            x[i] = __bfloat162float(__float2bfloat16_rn(e < HALF ? own * t.x - other * t.y : own * t.x + other * t.y));
            y[i] = __bfloat162float(__float2bfloat16_rn(v[e]));
        }
        Kv4Place p;
        p.h = h; p.slot = slots[j]; p.w = l >> 2; p.c = l & 3; p.row = row + row_add;
        kv4_store_row<DH>(c, p, live, x, y);
    } else if (q_out) {
        for (int i = threadIdx.x - 32; i < G * HALF; i += 96) {
            const int g = i / HALF, e = i % HALF, at = (h * G + g) * DH + e;
            const float2 t = s_cs[e];
            const float lo = in[at], hi = in[at + HALF];
            float* out = q_out + (long long)j * G * c.Hkv * DH + at;
            out[0] = lo * t.x - hi * t.y;
            out[HALF] = hi * t.x + lo * t.y;
        }
    }
}

long long kv4_bytes(const Kv4View& c) { return (long long)c.n_slots * c.Hkv * (c.max_len / KV4_TILE) * kv4_tile_bytes(c.dh); }

cudaError_t launch_kv4_put(const Kv4View& c, int n, const float* kv, int ld, int k_col, const int* slots, const int* rows, int row_add,
                           const double* inv_freq, int G, float* q_out, cudaStream_t st) {
    const dim3 grid((unsigned)c.Hkv, (unsigned)n);
    if (c.dh == 128) return launch_pdl(kv4_put_kernel<128>, grid, dim3(128), 0, st, c, kv, ld, k_col, slots, rows, row_add, inv_freq, G, q_out);
    return launch_pdl(kv4_put_kernel<64>, grid, dim3(128), 0, st, c, kv, ld, k_col, slots, rows, row_add, inv_freq, G, q_out);
}

// ------------------------------------------------------------------------------------------------ attention
// For each KV head the queries of all its rows and query heads are the columns of one problem: S^T = K Q^T and O^T = V^T P^T with
// the cache as the A operand of mma.m16n8k16 (16 keys, or 16 channels) and eight queries as B, so that one query costs no more
// than eight.  For bf16 codes reach the tensor core as fp16 subnormals (n 2^-24: a mask, no conversion), every second nibble as 16 n
// with its query, or its output, scaled by 1/16.  Scales stay outside: per group of 32 channels S = sum s_g (q_g . n) + m_g sum(q_g),
// and O_g = sum_r (p_r s_rg) n_r + sum_r p_r m_rg.  The second sum of S is one more product, of the m as they are stored (bf16)
// and sum(q_g) in three bf16 parts.
//
// Precision.  bf16 queries are exact in fp16 once their row is scaled by a power of two (what is below 2^-29 of the row's largest
// is rounded there); probabilities are rounded to fp16's 11 bits, 2^-12 of each, which the 2^-9 of the bf16 result hides.  fp32
// queries and their probabilities go in as two fp16 numbers (22 bits), the codes as whole numbers, and the products of 16 rows are
// added up in fp32 outside the tensor core.
// Weights meet the values' scales in fp16, p s R.  R is a column's own power of two and follows the largest p s that the column has met,
// which it keeps between 2^3 and 2^15, as the maximum follows the scores: rows that a column does not see, and rows whose weight is next to
// nothing, take no bits from the others, whatever they hold (64 sequences x 4 KV heads x 8 columns of 4096 rows 43.5 us, 48 to 50 where every
// step has a row 2^20 larger).  What a warp does for one column depends on that column's rows alone, to the bit.
//
// A cluster of up to 16 CTAs shares one (sequence, KV head, block of columns); a warp takes every (warps of the cluster)-th step of
// 16 or 32 rows, which bulk copies bring into its own ring, and keeps its own maximum, sum and output.  They are joined in
// shared memory, then over the cluster, always in the same order.
#define KV4_RING 4                   // tiles in a warp's ring


__device__ __forceinline__ void kv4_mma(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                 : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
// the first of a sum
__device__ __forceinline__ void kv4_mma0(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%10,%10,%10,%10};"
                 : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3])
                 : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "f"(0.f));
}
__device__ __forceinline__ void kv4_mma0_bf16(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%10,%10,%10,%10};"
                 : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3])
                 : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "f"(0.f));
}
__device__ __forceinline__ uint32_t kv4_transpose(uint32_t x) {
    uint32_t y;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
    return y;
}
// The number bf16 w's half h (0 lower, 1 upper) stands for.
__device__ __forceinline__ float kv4_bf(uint32_t w, int h) { return h ? bf16_hi(w) : bf16_lo(w); }

// ---- what a warp keeps: the queries, and the running maximum, sum and output of its columns
template <int DH, int NT, bool SPLIT>
struct Kv4Warp {
    static constexpr int Q = DH / 32;
    uint32_t q[NT][2 * Q][2];                   // B fragments of the queries
    uint32_t ql[SPLIT ? NT : 1][2 * Q][2];      // fp32: what the first rounding left
    uint32_t qm[SPLIT ? 1 : NT][2];             // B fragment of sum(q_g) in bf16 parts
    float qs[SPLIT ? NT : 1][Q][2];             // fp32: sum(q_g) of columns 2 (lane % 4) and + 1
    float fq[NT][2];                            // of those columns: what a sum is to be multiplied with
    float m[NT][2], l[NT][2];                   // l: this lane's rows only
    float o[NT][2 * Q][4];                      // V^T P^T, scaled by R and the codes' unit
    float mn[NT][Q][2];                         // sum of p m per group, this lane's rows only
    float R[NT][2];                             // powers of two that bring those columns' p s below 2^15
    uint32_t r_limit;                           // the bf16 scale from which on one of them may be too large
};

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

// A score above its column's maximum.  Products are rounded first, as for two (kv4_above); fp32 keeps what a fused operation has of them where
// the maximum is small enough for that to be a fraction.
template <bool SPLIT>
__device__ __forceinline__ float kv4_above1(float s, float f, float m) {
    const float y = __fadd_rn(__fmul_rn(s, f), -m);
    return SPLIT && fabsf(m) < 0x1p22f ? fmaf(s, f, -m) : y;
}

// U tiles of 16 rows from `row` on.  EDGE: some of the rows are not for every column, or not there at all.  Two tiles at a time: the
// chain from a tile's codes to its output is a thousand cycles long, and one tile alone leaves a warp waiting for most of them.
template <int DH, int NT, bool SPLIT, int U, bool EDGE>
__device__ __forceinline__ void kv4_rows(Kv4Warp<DH, NT, SPLIT>& st, const unsigned char* tile, int row, int lane, int j0, int G,
                                         const Kv4Sight& sight) {
    constexpr int Q = DH / 32, CH = DH / 8, H = Q / 2, TB = kv4_tile_bytes(DH);
    const int g = lane >> 2, c = lane & 3;
    float s[U][NT][4];
#pragma unroll
    for (int u = 0; u < U; ++u) {
        uint32_t p0[Q], p1[Q], k0[Q], k1[Q];                      // s of the groups two by two, then m; codes: of this lane's rows g, g + 8
        kv4_lds<Q>(tile + u * TB + 16 * DH + g * CH, p0);
        kv4_lds<Q>(tile + u * TB + 17 * DH + g * CH, p1);
        kv4_lds<Q>(tile + u * TB + g * (DH / 2) + c * CH, k0);
        kv4_lds<Q>(tile + u * TB + (g + 8) * (DH / 2) + c * CH, k1);
        if constexpr (!SPLIT) {
            // the lane's columns of A: the m of groups 2 c and 2 c + 1, the groups over and over again
            const uint32_t m0 = H == 2 && (c & 1) ? p0[Q - 1] : p0[H], m1 = H == 2 && (c & 1) ? p1[Q - 1] : p1[H];
#pragma unroll
            for (int n = 0; n < NT; ++n) kv4_mma0_bf16(s[u][n], m0, m1, m0, m1, st.qm[n][0], st.qm[n][1]);
        } else {
#pragma unroll
            for (int n = 0; n < NT; ++n) s[u][n][0] = s[u][n][1] = s[u][n][2] = s[u][n][3] = 0.f;
        }
#pragma unroll
        for (int w = 0; w < Q; ++w) {
            const uint32_t x0 = k0[w], x1 = k1[w], y0 = x0 >> 8, y1 = x1 >> 8;
            const uint32_t f0 = kv4_lo<SPLIT>(x0), f1 = kv4_lo<SPLIT>(x1), f2 = kv4_hi<SPLIT>(x0), f3 = kv4_hi<SPLIT>(x1);
            const uint32_t h0 = kv4_lo<SPLIT>(y0), h1 = kv4_lo<SPLIT>(y1), h2 = kv4_hi<SPLIT>(y0), h3 = kv4_hi<SPLIT>(y1);
            const float sc0 = kv4_bf(p0[w >> 1], w & 1), sc1 = kv4_bf(p1[w >> 1], w & 1);
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                float d[4];
                kv4_mma0(d, f0, f1, f2, f3, st.q[n][2 * w][0], st.q[n][2 * w][1]);
                kv4_mma(d, h0, h1, h2, h3, st.q[n][2 * w + 1][0], st.q[n][2 * w + 1][1]);
                if constexpr (SPLIT) {
                    kv4_mma(d, f0, f1, f2, f3, st.ql[n][2 * w][0], st.ql[n][2 * w][1]);
                    kv4_mma(d, h0, h1, h2, h3, st.ql[n][2 * w + 1][0], st.ql[n][2 * w + 1][1]);
                    const float mn0 = kv4_bf(p0[H + (w >> 1)], w & 1), mn1 = kv4_bf(p1[H + (w >> 1)], w & 1);
                    s[u][n][0] = fmaf(mn0, st.qs[n][w][0], s[u][n][0]);
                    s[u][n][1] = fmaf(mn0, st.qs[n][w][1], s[u][n][1]);
                    s[u][n][2] = fmaf(mn1, st.qs[n][w][0], s[u][n][2]);
                    s[u][n][3] = fmaf(mn1, st.qs[n][w][1], s[u][n][3]);
                }
                s[u][n][0] = fmaf(sc0, d[0], s[u][n][0]);
                s[u][n][1] = fmaf(sc0, d[1], s[u][n][1]);
                s[u][n][2] = fmaf(sc1, d[2], s[u][n][2]);
                s[u][n][3] = fmaf(sc1, d[3], s[u][n][3]);
            }
        }
    }
    // ---- scores above the running maximum, in powers of two
    float p[U][NT][4], top = -INFINITY;
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int e = 0; e < 4; e += 2) {
                if constexpr (EDGE) {
#pragma unroll
                    for (int i = 0; i < 2; ++i)
                        if (!sight(row + 16 * u + g + 4 * e, min((j0 + 8 * n + 2 * c + i) / G, sight.n_q - 1))) s[u][n][e + i] = -INFINITY;
                }
                if constexpr (SPLIT) {
                    p[u][n][e] = kv4_above1<true>(s[u][n][e], st.fq[n][0], st.m[n][0]);
                    p[u][n][e + 1] = kv4_above1<true>(s[u][n][e + 1], st.fq[n][1], st.m[n][1]);
                } else {
                    kv4_above(s[u][n][e], s[u][n][e + 1], st.fq[n][0], st.fq[n][1], kv4_pack2(-st.m[n][0], -st.m[n][1]), p[u][n][e], p[u][n][e + 1]);
                }
                top = fmaxf(top, fmaxf(p[u][n][e], p[u][n][e + 1]));
            }
    // ---- the values' scales
    uint32_t a0[U][Q], a1[U][Q];                                    // s of the lane's rows' pairs, a word a group
    const uint32_t mine = g & 1 ? 0x3244u : 0x1044u;                // the lane's rows are the even or the odd ones of their pairs
    uint32_t big = 0u;
#pragma unroll
    for (int u = 0; u < U; ++u) {
        kv4_lds<Q>(tile + u * TB + 18 * DH + (g >> 1) * (DH / 4), a0[u]);
        kv4_lds<Q>(tile + u * TB + 19 * DH + (g >> 1) * (DH / 4), a1[u]);
        if constexpr (EDGE) {
            // what lies behind the last row is anything at all
            const int pair = row + 16 * u + (g & 6);
#pragma unroll
            for (int w = 0; w < Q; ++w) {
                if (pair >= sight.nrows) a0[u][w] = 0u;
                if (pair + 1 >= sight.nrows) a0[u][w] &= 0xFFFFu;
                if (pair + 8 >= sight.nrows) a1[u][w] = 0u;
                if (pair + 9 >= sight.nrows) a1[u][w] &= 0xFFFFu;
            }
        }
#pragma unroll
        for (int w = 0; w < Q; ++w) big = __vmaxu2(big, __vmaxu2(a0[u][w], a1[u][w]));
    }
    // ---- The columns' maxima and their R, by what each of them sees: a maximum is raised by whole powers of two, which R takes from the
    // outputs' scale, once a score is above it by KV4_LAZY, R lowered once a p s R may reach 2^15.  Neither can be while no score is so far up
    // and every scale is below r_limit = 2^7 / (the largest R) - compared by halves of words; no scale is negative, a NaN's is above all.
    if (__any_sync(0xffffffffu, top > KV4_LAZY || max(big >> 16, big & 0xFFFFu) >= st.r_limit)) {
        float s0[U], s1[U];                                         // the rows' scales are below 2^s0, 2^s1 (those of groups that hold a NaN decide nothing)
#pragma unroll
        for (int u = 0; u < U; ++u) {
            uint32_t x0 = 0u, x1 = 0u;
#pragma unroll
            for (int w = 0; w < Q; ++w) {
                const uint32_t y0 = __byte_perm(a0[u][w], 0u, mine) >> 16, y1 = __byte_perm(a1[u][w], 0u, mine) >> 16;
                if (y0 < 0x7F80u) x0 = max(x0, y0);
                if (y1 < 0x7F80u) x1 = max(x1, y1);
            }
            s0[u] = x0 ? (float)((int)(x0 >> 7) - 126) : -INFINITY;
            s1[u] = x1 ? (float)((int)(x1 >> 7) - 126) : -INFINITY;
        }
        int most = -200;                                            // the largest R's exponent
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                float z = -INFINITY, t = -INFINITY;
#pragma unroll
                for (int u = 0; u < U; ++u) z = fmaxf(z, fmaxf(s[u][n][e], s[u][n][e + 2]));
                z = kv4_max_rows(z);
                const float old = st.m[n][e], above = kv4_above1<SPLIT>(z, st.fq[n][e], old);
                const bool rise = above > KV4_LAZY;
                const float m = !rise ? old : above < 0x1p20f && fabsf(old) < 0x1p22f ? old + floorf(above) : __fmul_rn(z, st.fq[n][e]);
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    p[u][n][e] = kv4_above1<SPLIT>(s[u][n][e], st.fq[n][e], m);
                    p[u][n][e + 2] = kv4_above1<SPLIT>(s[u][n][e + 2], st.fq[n][e], m);
                    t = fmaxf(t, fmaxf(p[u][n][e] + s0[u], p[u][n][e + 2] + s1[u]));
                }
                t = kv4_max_rows(t);                                // the step's p s are below 2^t
                const int was = (int)(__float_as_uint(st.R[n][e]) >> 23) - 127;
                int now = min(was + (rise ? __float2int_rn(fminf(m - old, 300.f)) : 0), 119);
                if (t + (float)now > (rise ? 6.f : 15.f)) now = max(5 - (int)ceilf(t), -125);
                const float f = kv4_exp2(old - m), fo = kv4_exp2((old - m) + (float)(now - was));
                st.m[n][e] = m;
                st.R[n][e] = kv4_pow2(now);
                most = max(most, now);
                st.l[n][e] *= f;
#pragma unroll
                for (int w = 0; w < Q; ++w) {
                    st.mn[n][w][e] *= f;
                    st.o[n][2 * w][e] *= fo; st.o[n][2 * w][e + 2] *= fo;
                    st.o[n][2 * w + 1][e] *= fo; st.o[n][2 * w + 1][e + 2] *= fo;
                }
            }
        most = max(most, __shfl_xor_sync(0xffffffffu, most, 1));
        most = max(most, __shfl_xor_sync(0xffffffffu, most, 2));
        st.r_limit = (uint32_t)(127 + 7 - most) << 7;
    }
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int u = 0; u < U; ++u) {
#pragma unroll
            for (int e = 0; e < 4; ++e) p[u][n][e] = kv4_exp2(p[u][n][e]);
            st.l[n][0] += p[u][n][0] + p[u][n][2];
            st.l[n][1] += p[u][n][1] + p[u][n][3];
        }
    // ---- the values
#pragma unroll
    for (int u = 0; u < U; ++u) {
        uint32_t v0[Q], v1[Q];
        kv4_lds<Q>(tile + u * TB + 8 * DH + c * DH + g * CH, v0);
        kv4_lds<Q>(tile + u * TB + 8 * DH + (c + 4) * DH + g * CH, v1);
        float pr[NT][4];
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int e = 0; e < 4; ++e) pr[n][e] = p[u][n][e] * st.R[n][e & 1];
        uint32_t q0[Q], q1[Q];                                      // m likewise
        kv4_lds<Q>(tile + u * TB + 18 * DH + (g >> 1) * (DH / 4) + CH, q0);
        kv4_lds<Q>(tile + u * TB + 19 * DH + (g >> 1) * (DH / 4) + CH, q1);
#pragma unroll
        for (int w = 0; w < Q; ++w) {
            const float sc0 = __uint_as_float(__byte_perm(a0[u][w], 0u, mine)), sc1 = __uint_as_float(__byte_perm(a1[u][w], 0u, mine));
            const float mn0 = __uint_as_float(__byte_perm(q0[w], 0u, mine)), mn1 = __uint_as_float(__byte_perm(q1[w], 0u, mine));
            uint32_t f0, f1, f2, f3, g0, g1, g2, g3;
            if constexpr (SPLIT) {
                const uint32_t y0 = v0[w] >> 8, y1 = v1[w] >> 8;
                f0 = kv4_lo<true>(v0[w]); f1 = kv4_hi<true>(v0[w]); f2 = kv4_lo<true>(v1[w]); f3 = kv4_hi<true>(v1[w]);
                g0 = kv4_lo<true>(y0); g1 = kv4_hi<true>(y0); g2 = kv4_lo<true>(y1); g3 = kv4_hi<true>(y1);
            } else {
                // whole bytes, n + 16 n', for the first of two channels: the second one's sum is taken off in the end
                f0 = v0[w] & 0x00FF00FFu; f2 = v1[w] & 0x00FF00FFu;
                g0 = __byte_perm(v0[w], 0u, 0x4341); g2 = __byte_perm(v1[w], 0u, 0x4341);
                f1 = kv4_hi<false>(f0); f3 = kv4_hi<false>(f2); g1 = kv4_hi<false>(g0); g3 = kv4_hi<false>(g2);
            }
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                float ps[4] = {pr[n][0] * sc0, pr[n][1] * sc0, pr[n][2] * sc1, pr[n][3] * sc1};
                const float* pp = p[u][n];
                if constexpr (EDGE) {
                    // a column that does not see the row takes nothing of it, not even a NaN
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        if (pp[e] == 0.f) ps[e] = 0.f;
                    st.mn[n][w][0] += (pp[0] == 0.f ? 0.f : pp[0] * mn0) + (pp[2] == 0.f ? 0.f : pp[2] * mn1);
                    st.mn[n][w][1] += (pp[1] == 0.f ? 0.f : pp[1] * mn0) + (pp[3] == 0.f ? 0.f : pp[3] * mn1);
                } else {
                    st.mn[n][w][0] = fmaf(pp[0], mn0, fmaf(pp[2], mn1, st.mn[n][w][0]));
                    st.mn[n][w][1] = fmaf(pp[1], mn0, fmaf(pp[3], mn1, st.mn[n][w][1]));
                }
                const uint32_t h0 = kv4_half2(ps[0], ps[1]), h1 = kv4_half2(ps[2], ps[3]);
                const uint32_t b0 = kv4_transpose(h0), b1 = kv4_transpose(h1);
                if constexpr (SPLIT) {
                    const float2 w0 = kv4_unhalf2(h0), w1 = kv4_unhalf2(h1);
                    // (what the first rounding left, 2^11 times: as far from fp16's smallest number as the first part)
                    const uint32_t c0 = kv4_transpose(kv4_half2((ps[0] - w0.x) * 0x1p11f, (ps[1] - w0.y) * 0x1p11f));
                    const uint32_t c1 = kv4_transpose(kv4_half2((ps[2] - w1.x) * 0x1p11f, (ps[3] - w1.y) * 0x1p11f));
                    auto add = [](float (&o)[4], const float (&hi)[4], const float (&lo)[4]) {
#pragma unroll
                        for (int e = 0; e < 4; ++e) o[e] += fmaf(lo[e], 0x1p-11f, hi[e]);
                    };
                    float d[4], f[4];
                    kv4_mma0(d, f0, f1, f2, f3, b0, b1);
                    kv4_mma0(f, f0, f1, f2, f3, c0, c1);
                    add(st.o[n][2 * w], d, f);
                    kv4_mma0(d, g0, g1, g2, g3, b0, b1);
                    kv4_mma0(f, g0, g1, g2, g3, c0, c1);
                    add(st.o[n][2 * w + 1], d, f);
                } else {
                    kv4_mma(st.o[n][2 * w], f0, f1, f2, f3, b0, b1);
                    kv4_mma(st.o[n][2 * w + 1], g0, g1, g2, g3, b0, b1);
                }
            }
        }
    }
}

// B fragment of sum(q_g) = hi + mid + lo, eight bits each.  Rows 2 c, 2 c + 1 of B: groups 2 (c % (Q / 2)) and + 1, part c / (Q / 2) (four
// groups: lo comes in rows 2 c + 8, 2 c + 9 of c = 0, 1; two groups: c = 3 has nothing).
template <int Q>
__device__ __forceinline__ void kv4_sum_parts(const float (&sum)[Q], int c, uint32_t (&qm)[2]) {
    float part[Q][3];
#pragma unroll
    for (int w = 0; w < Q; ++w) {
        part[w][0] = __bfloat162float(__float2bfloat16_rn(sum[w]));
        part[w][1] = __bfloat162float(__float2bfloat16_rn(sum[w] - part[w][0]));
        part[w][2] = sum[w] - part[w][0] - part[w][1];
    }
    auto pair = [](float x, float y) {
        const __nv_bfloat162 v = __floats2bfloat162_rn(x, y);
        return *(const uint32_t*)&v;
    };
    if constexpr (Q == 4) {
        const uint32_t b00 = pair(part[0][0], part[1][0]), b01 = pair(part[2][0], part[3][0]);
        const uint32_t b10 = pair(part[0][1], part[1][1]), b11 = pair(part[2][1], part[3][1]);
        const uint32_t b20 = pair(part[0][2], part[1][2]), b21 = pair(part[2][2], part[3][2]);
        qm[0] = c == 0 ? b00 : c == 1 ? b01 : c == 2 ? b10 : b11;
        qm[1] = c == 0 ? b20 : c == 1 ? b21 : 0u;
    } else {
        const uint32_t b0 = pair(part[0][0], part[1][0]), b1 = pair(part[0][1], part[1][1]), b2 = pair(part[0][2], part[1][2]);
        qm[0] = c == 0 ? b0 : c == 1 ? b1 : c == 2 ? b2 : 0u;
        qm[1] = 0u;
    }
}

// The queries as B fragments: column lane / 4 of every block of eight, channels 32 w + 8 (lane % 4) + 0..7 of every group.
template <int DH, int NT, typename T>
__device__ __forceinline__ void kv4_load_queries(Kv4Warp<DH, NT, Kv4Io<T>::SPLIT>& st, const Kv4AttnArgs& a, int b, int h, int j0, int lane) {
    constexpr bool SPLIT = Kv4Io<T>::SPLIT;
    constexpr int Q = DH / 32;
    constexpr float UNIT = SPLIT ? 1.f : 0x1p-24f;                // what a code of 1 is to the tensor core
    const int g = lane >> 2, c = lane & 3;
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        const int j = j0 + 8 * n + g;
        float x[Q][8], mx = 0.f;
#pragma unroll
        for (int w = 0; w < Q; ++w) {
            if (j < a.ncol) {
                const long long at = (long long)(b * a.n_q + j / a.G) * a.q_ld + (h * a.G + j % a.G) * DH + 32 * w + 8 * c;
                kv4_load8<typename Kv4Io<T>::Query>(a.q, at, x[w]);
            } else {
#pragma unroll
                for (int i = 0; i < 8; ++i) x[w][i] = 0.f;
            }
#pragma unroll
            for (int i = 0; i < 8; ++i) mx = fmaxf(mx, fabsf(x[w][i]));
        }
        mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 1));
        mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 2));
        // the row's largest number to 2^14 .. 2^15 (a row of zeros, or below 2^-100, as far as that goes)
        const int e = mx > 0.f ? min(max((int)(__float_as_uint(mx) >> 23) - 127, -100), 127) : 0;
        const float up = kv4_pow2(14 - e);
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
                    st.q[n][2 * w + s][r] = kv4_half2(back.x * f, back.y * f);
                    if constexpr (SPLIT) {
                        const uint32_t lo = kv4_half2(y[2 * r] - back.x, y[2 * r + 1] - back.y);
                        const float2 bl = kv4_unhalf2(lo);
                        sum[w] += bl.x + bl.y;
                        st.ql[n][2 * w + s][r] = kv4_half2(bl.x * f, bl.y * f);
                    }
                }
            }
            sum[w] += __shfl_xor_sync(0xffffffffu, sum[w], 1);
            sum[w] += __shfl_xor_sync(0xffffffffu, sum[w], 2);
            sum[w] *= UNIT;                                       // in the unit of the products
        }
        if constexpr (!SPLIT) {
            kv4_sum_parts<Q>(sum, c, st.qm[n]);
        }
        const float f = kv4_factor(e - 14 + (SPLIT ? 0 : 24), a.scale_log2);       // (the unit of the products in it)
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            const int from = (2 * c + s) * 4;                     // a lane with lane / 4 = 2 c + s
            st.fq[n][s] = __shfl_sync(0xffffffffu, f, from);
            if constexpr (SPLIT) {
#pragma unroll
                for (int w = 0; w < Q; ++w) st.qs[n][w][s] = __shfl_sync(0xffffffffu, sum[w], from);
            }
        }
    }
}

// Shared memory: the warps' rings, and over them, once they are used up, [warp][column][DH + 4] outputs, maxima and sums.
template <int DH, int NT>
__host__ __device__ constexpr size_t kv4_smem(int warps) {
    const size_t ring = (size_t)warps * KV4_RING * kv4_tile_bytes(DH), join = sizeof(float) * 8 * NT * (warps * (DH + 4 + 2) + 2);
    return ring > join ? ring : join;
}

template <int DH, int NT, typename T, int U, int WARPS, int CTAS>
__global__ void __launch_bounds__(WARPS * 32, CTAS) kv4_attn_kernel(const __grid_constant__ Kv4AttnArgs a) {
    constexpr bool SPLIT = Kv4Io<T>::SPLIT;
    constexpr int Q = DH / 32, NB = 8 * NT, LDO = DH + 4, TB = kv4_tile_bytes(DH), ROWS = KV4_TILE * U, STAGES = KV4_RING / U;
    constexpr float UNIT = SPLIT ? 1.f : 0x1p-24f;
    extern __shared__ __align__(128) unsigned char kv4_sm[];
    __shared__ u64 bars[WARPS][STAGES];
    float* sO = (float*)kv4_sm;                     // [warp][column][LDO]
    float* sM = sO + WARPS * NB * LDO;              // [warp][column]
    float* sL = sM + WARPS * NB;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g = lane >> 2, c = lane & 3;
    const int b = blockIdx.z, h = blockIdx.y / a.n_blocks, j0 = (blockIdx.y % a.n_blocks) * NB;
    const int rank = blockIdx.x, S = gridDim.x;     // (a cluster is the x extent of the grid)
    const uint32_t bar = kv4_saddr(bars[warp]), ring = kv4_saddr(kv4_sm) + warp * KV4_RING * TB;
    if (lane < STAGES) asm volatile("mbarrier.init.shared::cta.b64 [%0], 1;" ::"r"(bar + lane * 8) : "memory");
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("fence.proxy.async;" ::: "memory");
    __syncwarp();
    pdl_wait();
    pdl_trigger();
    Kv4Sight sight;
    sight.nrows = min(max(a.rows[b] + a.rows_add, 0), a.c.max_len);
    sight.n_q = a.n_q; sight.mask_rows = a.mask_rows; sight.mask_words = a.mask_words;
    sight.mask = a.mask ? a.mask + (long long)b * a.n_q * a.mask_words : nullptr;
    const int i_first = j0 / a.G, i_last = (min(j0 + NB, a.ncol) - 1) / a.G;
    // rows [0, clear) are visible to every column of the block, rows from `end` on to none
    const int clear = max(0, a.mask ? sight.nrows - a.mask_rows : sight.nrows - a.n_q + i_first + 1);
    const int end = max(0, a.mask ? sight.nrows : sight.nrows - a.n_q + i_last + 1);
    const int nstep = (end + ROWS - 1) / ROWS, nfull = clear / ROWS;         // steps of U tiles; those before `clear`
    const unsigned char* base = kv4_tile(a.c, a.sl.slot[b], h, 0);
    const int first = rank * WARPS + warp, step = S * WARPS;

    int ahead = first;                              // the next step to be fetched
#pragma unroll
    for (int i = 0; i < STAGES; ++i) {
        if (ahead < nstep && lane == 0) kv4_fetch(ring + i * U * TB, base + (long long)ahead * (U * TB), U * TB, bar + i * 8);
        ahead += step;
    }
    Kv4Warp<DH, NT, SPLIT> st;
    kv4_load_queries<DH, NT, T>(st, a, b, h, j0, lane);
#pragma unroll
    for (int n = 0; n < NT; ++n) {
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            st.m[n][s] = KV4_NOTHING;
            st.l[n][s] = 0.f;
            st.R[n][s] = 0x1p119f;
#pragma unroll
            for (int w = 0; w < Q; ++w) st.mn[n][w][s] = 0.f;
        }
#pragma unroll
        for (int i = 0; i < 2 * Q; ++i)
#pragma unroll
            for (int s = 0; s < 4; ++s) st.o[n][i][s] = 0.f;
    }
    st.r_limit = 0u;

    bool ok = true;
    uint32_t stage = 0, parity = 0;
    for (int t = first; t < nstep; t += step) {
        ok = kv4_wait(bar + stage * 8, parity);
        if (!ok) break;
        const unsigned char* tile = kv4_sm + (warp * KV4_RING + stage * U) * TB;
        if (t < nfull) kv4_rows<DH, NT, SPLIT, U, false>(st, tile, t * ROWS, lane, j0, a.G, sight);
        else kv4_rows<DH, NT, SPLIT, U, true>(st, tile, t * ROWS, lane, j0, a.G, sight);
        __syncwarp();
        if (ahead < nstep && lane == 0) kv4_fetch(ring + stage * U * TB, base + (long long)ahead * (U * TB), U * TB, bar + stage * 8);
        ahead += step;
        if (++stage == STAGES) { stage = 0; parity ^= 1u; }
    }
    if (!ok) {
        // a copy has not come: what is in flight is waited for once more, and the result is NaN
        for (int i = 0; i < STAGES; ++i) {
            kv4_wait(bar + stage * 8, parity);
            if (++stage == STAGES) { stage = 0; parity ^= 1u; }
        }
#pragma unroll
        for (int n = 0; n < NT; ++n) st.l[n][0] = st.l[n][1] = __uint_as_float(0x7FC00000u);
    }
    __syncthreads();                                // every ring is used up

    // ---- this warp's columns to shared memory: maximum, sum, output
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            const int col = 8 * n + 2 * c + s;
            // 1 / R (the unit apart: values next to fp32's ends pass through numbers of their own size)
            const float down = __uint_as_float((254u << 23) - __float_as_uint(st.R[n][s]));
            const float l = kv4_sum_rows(st.l[n][s]);
            if (g == 0) {
                sM[warp * NB + col] = st.m[n][s];
                sL[warp * NB + col] = l;
            }
#pragma unroll
            for (int w = 0; w < Q; ++w) {
                const float m = kv4_sum_rows(st.mn[n][w][s]);
                // channels 32 w + 4 g + 0..3: rows g and g + 8 of the two blocks of 16, the latter sixteenfold, the former (bf16) with
                // the latter added
                const float x1 = st.o[n][2 * w][2 + s], y1 = st.o[n][2 * w + 1][2 + s];
                const float x0 = st.o[n][2 * w][s] - (SPLIT ? 0.f : x1), y0 = st.o[n][2 * w + 1][s] - (SPLIT ? 0.f : y1);
                *(float4*)(sO + (warp * NB + col) * LDO + 32 * w + 4 * g) =
                    make_float4(fmaf(x0 * down, 1.f / UNIT, m), fmaf(x1 * down, 0.0625f / UNIT, m), fmaf(y0 * down, 1.f / UNIT, m),
                                fmaf(y1 * down, 0.0625f / UNIT, m));
            }
        }
    __syncthreads();
    // ---- the warps of the CTA, into the first one's place
    const int cols = min(NB, a.ncol - j0);
    for (int i = tid; i < cols * (DH / 4); i += WARPS * 32) {
        const int col = i / (DH / 4), ch = (i % (DH / 4)) * 4;
        float m = KV4_NOTHING, l = 0.f;
#pragma unroll
        for (int w = 0; w < WARPS; ++w) m = fmaxf(m, sM[w * NB + col]);
        float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
        for (int w = 0; w < WARPS; ++w) {
            const float f = kv4_exp2(sM[w * NB + col] - m);
            const float4 x = *(const float4*)(sO + (w * NB + col) * LDO + ch);
            l = fmaf(sL[w * NB + col], f, l);
            o.x = fmaf(x.x, f, o.x); o.y = fmaf(x.y, f, o.y); o.z = fmaf(x.z, f, o.z); o.w = fmaf(x.w, f, o.w);
        }
        if (S == 1) {
            kv4_put<T>(a, b, h, j0 + col, ch, DH, o, l);
        } else {
            *(float4*)(sO + col * LDO + ch) = o;
            // (maxima and sums for the cluster go behind those of the warps, which other threads still read)
            if (ch == 0) {
                sM[2 * WARPS * NB + col] = m;
                sM[2 * WARPS * NB + NB + col] = l;
            }
        }
    }
    if (S == 1) return;
    // ---- the CTAs of the cluster: each writes its share of the columns' channels
    cg::cluster_group cluster = cg::this_cluster();
    cluster.sync();
    const float* cM = sM + 2 * WARPS * NB;
    for (int i = rank * WARPS * 32 + tid; i < cols * (DH / 4); i += S * WARPS * 32) {
        const int col = i / (DH / 4), ch = (i % (DH / 4)) * 4;
        float m = KV4_NOTHING, l = 0.f;
        for (int r = 0; r < S; ++r) m = fmaxf(m, *cluster.map_shared_rank(cM + col, r));
        float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
        for (int r = 0; r < S; ++r) {
            const float f = kv4_exp2(*cluster.map_shared_rank(cM + col, r) - m);
            const float4 x = *(const float4*)cluster.map_shared_rank(sO + col * LDO + ch, r);
            l = fmaf(*cluster.map_shared_rank(cM + NB + col, r), f, l);
            o.x = fmaf(x.x, f, o.x); o.y = fmaf(x.y, f, o.y); o.z = fmaf(x.z, f, o.z); o.w = fmaf(x.w, f, o.w);
        }
        kv4_put<T>(a, b, h, j0 + col, ch, DH, o, l);
    }
    cluster.sync();          // nobody leaves while its shared memory may still be read
}

static cudaError_t kv4_launch(void (*kernel)(Kv4AttnArgs), bool* attr_set, Kv4AttnArgs& a, int columns, int threads, size_t smem, int step_rows,
                              int resident, int dev, cudaStream_t st) {
    if (dev < 0 || dev >= HIVIS_MAX_DEVICES || !attr_set[dev]) {
        cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
        if (e == cudaSuccess) e = cudaFuncSetAttribute(kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
        if (e != cudaSuccess) return e;
        if (dev >= 0 && dev < HIVIS_MAX_DEVICES) attr_set[dev] = true;
    }
    a.n_blocks = (a.ncol + columns - 1) / columns;
    const int S = kv4_cluster(a.sl.n * a.c.Hkv * a.n_blocks, a.c.max_len, step_rows, resident);
    const dim3 grid((unsigned)S, (unsigned)(a.c.Hkv * a.n_blocks), (unsigned)a.sl.n);
    return launch_cluster_pdl(kernel, S, grid, dim3((unsigned)threads), smem, st, a);
}
template <int DH, int NT, typename T, int U, int WARPS, int CTAS>
static cudaError_t kv4_launch_attn(Kv4AttnArgs& a, int dev, int num_sms, cudaStream_t st) {
    static bool attr_set[HIVIS_MAX_DEVICES] = {false};
    return kv4_launch(kv4_attn_kernel<DH, NT, T, U, WARPS, CTAS>, attr_set, a, 8 * NT, WARPS * 32, kv4_smem<DH, NT>(WARPS),
                      WARPS * U * KV4_TILE, num_sms * CTAS, dev, st);
}
template <int DH, typename T>
static cudaError_t kv4_launch_attn_n(Kv4AttnArgs& a, int dev, int num_sms, cudaStream_t st) {
    if constexpr (sizeof(T) == 4) {
        if (a.ncol <= 8) return kv4_launch_attn<DH, 1, T, 1, 4, 2>(a, dev, num_sms, st);
        return kv4_launch_attn<DH, 2, T, 1, 4, 2>(a, dev, num_sms, st);
    } else {
        // Blocks of 64 columns, whose codes are taken apart once (kernels_kv4_tc.cu), or of 16 here.  The rule is set for large batches of long
        // caches: 64 sequences x 4 KV heads of 4096 rows, head_dim 128, 16 columns take 132 us there and 95 here, 17 to 32 133 and 155 to 159,
        // 64 136 and 249; head_dim 64, where taking apart is half the work, 32 x 8 of 2048 rows: 48 columns 71 and 56, 49 71 and 74.  Where a
        // CTA has less to do it costs more than it saves, most of all with many short sequences, whose units of one step pay a CTA's
        // set-up each: 64 x 32 of 32 rows, 17 columns 166 there and 95 here, 64 191 and 183; of 512 rows 257 and 178, 275 and 378; one
        // sequence of 32 heads x 2240 rows 20.5 and 19.0, 21.0 and 27.3, of 4 heads x 2048 rows 14.9 and 11.8, 15.4 and 14.1; head_dim 64,
        // 64 x 32 of 64 rows, 49 columns 155 and 107.
        // Registers: head_dim 128 spills, by ptxas, 32 bytes a thread at eight columns and four CTAs to an SM, 104 (bf16) and 60 (fp32) at sixteen.
        if (std::is_same<T, bf16>::value && a.ncol > (DH == 128 ? 16 : 48)) return launch_kv4_attn_tc(a, dev, num_sms, st);
        if (a.ncol > 8) return kv4_launch_attn<DH, 2, T, 1, 4, 3>(a, dev, num_sms, st);
        // Few (sequence, KV head) pairs do not fill the GPU with clusters of 16: a warp then gets more registers (nothing spilled)
        // instead of a fourth neighbour.  4 x 4 pairs of 9 001 to 32 768 rows: 24.6 us, 29.1 with 128 registers; 16 x 32 pairs of
        // 2176 rows, where four to an SM count: 48.7 us, 45.1 with 128.
        if (a.sl.n * a.c.Hkv * KV4_MAX_CLUSTER < num_sms * 3) return kv4_launch_attn<DH, 1, T, 2, 4, 3>(a, dev, num_sms, st);
        return kv4_launch_attn<DH, 1, T, 2, 4, 4>(a, dev, num_sms, st);
    }
}

cudaError_t launch_kv4_draft_attention(const Kv4View& c, const SlotList& sl, const int* pos0, int step, int G, const float* q, float scale,
                                       float* attn, bf16* attn_h, int lo_rows, int num_sms, cudaStream_t st) {
    Kv4AttnArgs a;
    memset(&a, 0, sizeof(a));
    a.c = c; a.sl = sl; a.rows = pos0; a.rows_add = step + 1;
    a.q = q; a.n_q = 1; a.G = a.ncol = G; a.Hq = G * c.Hkv; a.q_ld = a.out_ld = (long long)a.Hq * c.dh;
    a.scale_log2 = (float)((double)scale * 1.4426950408889634);
    a.out = attn; a.out_h = attn_h; a.lo_rows = lo_rows;
    int dev = 0;
    const cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    return c.dh == 128 ? kv4_launch_attn_n<128, Kv4DraftIo>(a, dev, num_sms, st) : kv4_launch_attn_n<64, Kv4DraftIo>(a, dev, num_sms, st);
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
    if (!cache->data || kv4_misaligned(cache->data)) KV4_FAIL(HIVIS_ERR_ARG, "%s: the cache's buffer is null or not 16-byte aligned", who);
    if (B < 1 || B > HIVIS_MAX_BATCH) KV4_FAIL(HIVIS_ERR_CAPACITY, "%s: B=%d outside [1,%d]", who, B, HIVIS_MAX_BATCH);
    sl->n = B;
    for (int b = 0; b < B; ++b) {
        const int s = slots_host ? slots_host[b] : b;
        if (s < 0 || s >= cache->n_slots) KV4_FAIL(HIVIS_ERR_ARG, "%s: slot %d out of range", who, s);
        for (int i = 0; i < b; ++i)
            if (sl->slot[i] == s) KV4_FAIL(HIVIS_ERR_ARG, "%s: slot %d listed twice", who, s);
        sl->slot[b] = s;
    }
    c->data = (unsigned char*)cache->data;
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

// A CTA's `units` places are heads side by side (as many as there are, to a power of two) of neighbouring rows or pairs, `rounds` of
// them after one another.
static bool kv4_rows_grid(Kv4RowsArgs* a, int units, int rounds, int items, dim3* grid) {
    a->heads_log2 = 0;
    while ((1 << a->heads_log2) < units && (1 << a->heads_log2) < a->c.Hkv) a->heads_log2 += 1;
    const int per = (units >> a->heads_log2) * rounds;
    const long long y = (a->c.Hkv + (1 << a->heads_log2) - 1) >> a->heads_log2;
    *grid = dim3((unsigned)(((long long)items + per - 1) / per), (unsigned)y);
    return y <= 65535;
}

cudaError_t launch_kv4_read_slot(const Kv4View& c, int slot, int row0, int n, float* out_k, float* out_v, cudaStream_t st) {
    if (n <= 0) return cudaSuccess;
    Kv4RowsArgs a;
    memset(&a, 0, sizeof(a));
    a.c = c; a.sl.n = 1; a.sl.slot[0] = slot; a.cu.v[1] = n; a.start_host = row0;
    a.out_k = out_k; a.out_v = out_v;
    dim3 grid;
    if (!kv4_rows_grid(&a, 256 / (c.dh / 4), KV4_READ_ROWS, n, &grid)) return cudaErrorInvalidValue;
    return c.dh == 128 ? launch_pdl(kv4_read_kernel<128>, grid, dim3(256), 0, st, a) : launch_pdl(kv4_read_kernel<64>, grid, dim3(256), 0, st, a);
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
    a.k = k; a.v = v; a.ld = ld;
    dim3 grid;
    const dim3 block(128);
    if (!kv4_rows_grid(&a, 128 / (a.c.dh / 16), 1, a.pairs.v[B], &grid)) KV4_FAIL(HIVIS_ERR_SHAPE, "%s: too many heads", who);
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
    a.out_k = out_k; a.out_v = out_v;
    dim3 grid;
    const dim3 block(256);
    if (!kv4_rows_grid(&a, 256 / (a.c.dh / 4), KV4_READ_ROWS, a.cu.v[B], &grid)) KV4_FAIL(HIVIS_ERR_SHAPE, "%s: too many heads", who);
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
    if (!(scale > 0.f) || !(scale < 1e38f)) KV4_FAIL(HIVIS_ERR_ARG, "%s: scale must be positive and less than 1e38", who);
    if (mask && (mask_rows < 1 || mask_rows > HIVIS_KV4_MAX_MASK))
        KV4_FAIL(HIVIS_ERR_CAPACITY, "%s: mask_rows=%d outside [1,%d]", who, mask_rows, HIVIS_KV4_MAX_MASK);
    a.rows = rows; a.q = q; a.q_ld = q_ld; a.n_q = n_q; a.Hq = n_q_heads; a.G = n_q_heads / a.c.Hkv; a.ncol = n_q * a.G;
    a.scale_log2 = (float)((double)scale * 1.4426950408889634);
    a.mask = mask; a.mask_rows = mask ? mask_rows : 0; a.mask_words = (a.mask_rows + 31) / 32;
    a.out = out; a.out_ld = out_ld;
    if ((long long)a.c.Hkv * ((a.ncol + 7) / 8) > 65535) KV4_FAIL(HIVIS_ERR_SHAPE, "%s: too many heads and queries for one call", who);
    int dev = 0, sms = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e == cudaSuccess) e = device_sms(dev, &sms);
    if (e != cudaSuccess) return kv4_cuda(who, e);
    cudaStream_t st = (cudaStream_t)stream;
    if (dtype == HIVIS_BF16) e = a.c.dh == 128 ? kv4_launch_attn_n<128, bf16>(a, dev, sms, st) : kv4_launch_attn_n<64, bf16>(a, dev, sms, st);
    else e = a.c.dh == 128 ? kv4_launch_attn_n<128, float>(a, dev, sms, st) : kv4_launch_attn_n<64, float>(a, dev, sms, st);
    return kv4_cuda(who, e);
}
