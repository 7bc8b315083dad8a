// Attention of many columns (queries x query heads of a KV head) over a 4-bit cache, on the tcgen05 tensor cores.
//
// A CTA has 64 columns and takes 128 rows of the cache at a time:
//   S^T [128 rows x 64 columns] = K Q^T      A = K's values, B = the queries, accumulators in tensor memory
//   P^T = 2^(S^T f - m)                      a thread has one row and half the columns
//   O^T [channels x 64] += V^T P^T           A = V's values, B = the probabilities
// Eight warps take the codes apart, eight others have the probabilities: rows' values t + 1 are made while the probabilities of rows t
// are.  Values m + s n are written as fp16 numbers (11 bits, like the probabilities; a bf16 result has 8) to shared memory in the
// layouts that tcgen05.mma reads (rows of 128 bytes, 128-byte swizzle).  A word of K codes has eight channels of a row: 16 bytes of
// that row, the channels of a group in the order of the nibbles, and the queries' in the same.  Two words of V codes have four channels
// each of two neighbouring rows: 16 bytes of either row, channels of two groups side by side; V^T and P^T are read transposed, a row
// of the cache to 128 bytes, and the results' channels put in order when they leave.
// Keys are scaled by a power of two of their row (which the row's scores undo), so that fp16's range holds them; probabilities are written
// for a running maximum that is raised once a score is above it by 2^8.  Values share one power of two, that of rows up to 2^KT_SPAN times
// as large as the smallest the CTA met first.  A row that lies outside (far larger or smaller than most, or not seen at all and holding
// anything) gets one of its own, 2^-d of that: its probabilities are written 2^d times as large, and a column in which that leaves fp16's range has all
// its probabilities, and its outputs, scaled by 2^c.  Steps with such a row cost a second maximum and exponential, and the outputs' way
// through registers: where every step has one, 64 sequences x 4 KV heads x 56 columns of 4096 rows take 278 us, where none has, 135 to 139.
// So a column gets what the rows that it sees and gives weight make of it; others can move the scale that most rows share, which shifts
// roundings at most.
// (ptxas: 128 registers, 14 bytes spilled at head_dim 128, 8 at 64.)
//
// What bounds it: 64 sequences x 4 KV heads x 56 columns of 4096 rows take 139 us, 217 TFLOP/s, and 64 columns as long as 17: about 3500
// cycles go by for 128 rows, of which the codes' warps (two to a scheduler) are busy all the time and the others two thirds.  Shared memory
// is in use for some 2500 of them: values and probabilities are written (640), read by the products at 128 bytes a cycle (16 of
// 6 KB: 790), codes, parameters and columns' scales read by the warps.  What was measured on the way: one group of eight warps that does everything in turn 238 us; two groups 161; keys' codes as
// subnormal factors and all loads before all stores 152; sums of weights added up beside the probabilities instead of a product with ones,
// and two steps' P and V in shared memory, 134; stores without bank conflicts 131; values' codes as whole numbers, for rows far below the
// largest, 137; scales and maxima that go by what a column sees 139 (138 without).  Products started by other warps than now are no help: by the probabilities' 142, by warps of their own, which leave the
// others fewer registers, 139 instead of 131.
#include <cstring>

#include <cooperative_groups.h>

#include "kv4_attn.cuh"

namespace cg = cooperative_groups;

namespace {

constexpr int KT_COLS = 64, KT_ROWS = 128, KT_GROUP = 256, KT_THREADS = 2 * KT_GROUP, KT_STAGES = 3, KT_CLUSTER = 8, KT_TILES = KT_ROWS / KV4_TILE;
constexpr uint32_t KT_TMEM = 256;                                     // columns: S^T of two steps, O^T
// Probabilities are held as 2^KT_LIFT p, below 2^15: fp16 has them to 2^-31 of a column's largest.
#define KT_LIFT 7.f
// Values' exponents: the rows that share a scale lie in (base - KT_WINDOW, base], base = KT_SPAN above the smallest of the first step with any.
constexpr int KT_SPAN = 10, KT_WINDOW = 16, KT_LEAST = -98, KT_MOST = 131;
constexpr uint32_t KT_S = 0, KT_O = 128;

// Shared memory, every block 1024-byte aligned.  K: [64 channels a block][128 rows][128 bytes], Q: [64 channels a block][64][128 bytes];
// V, two steps': [64 channels a block][128 rows][128 bytes] (head_dim 64: and a block of zeros, the products' other 64 rows);
// P, two steps': [128 rows][128 bytes].
template <int DH>
struct KtSmem {
    static constexpr int KB = DH / 64;                                 // blocks of 64 channels
    static constexpr int RAW = KT_TILES * kv4_tile_bytes(DH);
    static constexpr int K = KT_STAGES * RAW, V = K + KB * 16384, P = V + (DH == 128 ? 4 : 3) * 16384, Q = P + 2 * 16384;
    static constexpr int END = Q + KB * 8192;
    static constexpr int LDO = DH + 32;                                // results: groups of channels 1024 / DH words apart, no bank twice
    static constexpr int BYTES = END + 1024;                           // (the base is aligned by hand)
    static_assert(RAW % 1024 == 0 && KT_COLS * LDO * 4 <= END && BYTES <= 227 * 1024, "layout");
};

// fp16 operands, fp32 accumulators, M = 128, N = 64; ROWS: both operands with the products' axis along 128-byte rows, else across them
template <bool ROWS>
__device__ __forceinline__ void kt_mma(uint32_t d, u64 a, u64 b, uint32_t accumulate) {
    constexpr uint32_t IDESC = (1u << 4) | (ROWS ? 0u : 3u << 15) | ((KT_COLS >> 3) << 17) | ((128 >> 4) << 24);
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\ttcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}"
                 ::"r"(d), "l"(a), "l"(b), "r"(IDESC), "r"(accumulate) : "memory");
}
// 128-byte rows, 128-byte swizzle, groups of 8 rows 1024 bytes apart; blocks of 64 elements across `apart` bytes apart
__device__ __forceinline__ u64 kt_desc(uint32_t addr, uint32_t apart = 16) {
    const uint32_t lo = ((addr >> 4) & 0x3FFFu) | ((apart >> 4) << 16), hi = (1024u >> 4) | (1u << 14) | (2u << 29);
    return ((u64)hi << 32) | lo;
}
__device__ __forceinline__ void kt_commit(uint32_t bar) {
    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void kt_fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void kt_fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void kt_fence_smem() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }
__device__ __forceinline__ bool kt_elect() {
    uint32_t p;
    __syncwarp();
    asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(p));
    return p != 0;
}
template <int ID>
__device__ __forceinline__ void kt_sync() { asm volatile("barrier.cta.sync %0, %1;" ::"n"(ID), "n"(KT_GROUP) : "memory"); }
template <int ID>
__device__ __forceinline__ bool kt_sync_or(bool x) {
    uint32_t r;
    asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.u32 p, %1, 0;\n\tbarrier.cta.red.or.pred q, %2, %3, p;\n\tselp.u32 %0, 1, 0, q;\n\t}"
                 : "=r"(r) : "r"((uint32_t)x), "n"(ID), "n"(KT_GROUP) : "memory");
    return r != 0;
}
__device__ __forceinline__ void kt_arrive(uint32_t bar) { asm volatile("mbarrier.arrive.release.cta.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory"); }
#define KT_R(v, i) "=r"(v[i]), "=r"(v[i + 1]), "=r"(v[i + 2]), "=r"(v[i + 3]), "=r"(v[i + 4]), "=r"(v[i + 5]), "=r"(v[i + 6]), "=r"(v[i + 7])
#define KT_W(v, i) "r"(v[i]), "r"(v[i + 1]), "r"(v[i + 2]), "r"(v[i + 3]), "r"(v[i + 4]), "r"(v[i + 5]), "r"(v[i + 6]), "r"(v[i + 7])
// 32 columns of the 32 tensor-memory lanes that this warp may touch
__device__ __forceinline__ void kt_ld32(uint32_t t, uint32_t (&r)[32]) {
    __syncwarp();
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,"
        "%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
        : KT_R(r, 0), KT_R(r, 8), KT_R(r, 16), KT_R(r, 24) : "r"(t) : "memory");
    asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
}
// 16 columns
__device__ __forceinline__ void kt_ld16(uint32_t t, uint32_t (&r)[16]) {
    __syncwarp();
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];"
                 : KT_R(r, 0), KT_R(r, 8) : "r"(t) : "memory");
    asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
}
__device__ __forceinline__ void kt_st32(uint32_t t, const uint32_t (&r)[32]) {
    __syncwarp();
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x32.b32 [%32], {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,"
        "%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31};"
        ::KT_W(r, 0), KT_W(r, 8), KT_W(r, 16), KT_W(r, 24), "r"(t) : "memory");
    asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory");
}

__device__ __forceinline__ uint32_t kt_h2(const __half2& h) { return *(const uint32_t*)&h; }
__device__ __forceinline__ __half2 kt_as_h2(uint32_t w) { return *(const __half2*)&w; }

// The eight values of a word of codes, in the nibbles' order (0 and 4, 1 and 5, 2 and 6, 3 and 7), for s, s / 16 and m as pairs.
// Not WHOLE: a code in an fp16's lowest bits is the subnormal n 2^-24, four bits further up 16 n 2^-24, and s has 2^24 in it.
template <bool WHOLE>
__device__ __forceinline__ void kt_values(uint32_t x, const __half2& s, const __half2& s16, const __half2& m, uint32_t (&v)[4]) {
    const uint32_t y = x >> 8;
    v[0] = kt_h2(__hfma2(kt_as_h2(kv4_lo<WHOLE>(x)), s, m));
    v[1] = kt_h2(__hfma2(kt_as_h2(kv4_hi<WHOLE>(x)), s16, m));
    v[2] = kt_h2(__hfma2(kt_as_h2(kv4_lo<WHOLE>(y)), s, m));
    v[3] = kt_h2(__hfma2(kt_as_h2(kv4_hi<WHOLE>(y)), s16, m));
}
// 2^e, -149 <= e <= 127
__device__ __forceinline__ float kt_pow2(int e) { return __uint_as_float(e < -126 ? 1u << (e + 149) : (uint32_t)(e + 127) << 23); }
// Which of the 32 rows from r0 on query i sees.
__device__ __forceinline__ uint32_t kt_window(const Kv4Sight& s, int r0, int i) {
    const int end = s.mask ? s.nrows : s.nrows - s.n_q + i + 1;        // (none from here on)
    uint32_t w = 0xFFFFFFFFu;
    if (s.mask) {
        const int k = r0 - (s.nrows - s.mask_rows);
        const uint32_t* m = s.mask + (long long)i * s.mask_words;
        if (k >= 0) {
            const int at = k >> 5;
            const uint32_t lo = at < s.mask_words ? m[at] : 0u, hi = at + 1 < s.mask_words ? m[at + 1] : 0u;
            w = __funnelshift_r(lo, hi, k);
        } else if (k > -32) {
            w = (m[0] << -k) | ((1u << -k) - 1u);
        }
    }
    const int n = end - r0;
    return n >= 32 ? w : n <= 0 ? 0u : w & ((1u << n) - 1u);
}
// The larger of |m| and 16 s over halves of words (bf16; 0x0200 where both are 0).
// Keys: below 2^(e + 1), they are scaled by 2^-(e + 6) and stay below 2^-4, s 2^24 below 2^15; a rounding is 2^-20 of its row's largest at
// most, or half a step of its own.  Values: by 2^(13 - e), below 2^15, roundings 2^-38 of the largest.
__device__ __forceinline__ uint32_t kt_reach(uint32_t s, uint32_t m) { return __vmaxu2(m & 0x7FFF7FFFu, s + 0x02000200u); }
#define KT_ZERO 0x0200u

template <int DH>
__global__ void __launch_bounds__(KT_THREADS, 1) kv4_tc_kernel(const __grid_constant__ Kv4AttnArgs a) {
    typedef KtSmem<DH> M;
    constexpr int APART = 1024 / DH, Q = DH / 32, KB = M::KB, H = Q / 2, TB = kv4_tile_bytes(DH), LDO = M::LDO;
    extern __shared__ unsigned char kt_raw[];
    // rows' codes; of even and odd steps: S^T is there (and what goes with it); V is there; O^T is there, P and V may be overwritten
    __shared__ u64 bars[KT_STAGES + 6];
    __shared__ uint32_t s_tmem, s_poison[KT_COLS], s_nan[2][KT_ROWS];
    __shared__ __align__(16) float s_f[KT_COLS], s_m[KT_COLS];         // what a column's scores are to be multiplied with; KT_LIFT less its maximum
    __shared__ float2 s_part[KT_CLUSTER][KT_COLS];
    // of the rows: what undoes their keys' scale, d; of the columns: c, what their sums and their outputs are multiplied with
    __shared__ float s_rk[2][KT_ROWS], s_d[2][KT_ROWS], s_top[4][KT_COLS], s_c[KT_COLS], s_fall[KT_COLS], s_fall_o[KT_COLS], s_inv[KT_COLS];
    __shared__ int s_least[8], s_has_nan[2], s_apart[2], s_base;
    unsigned char* sm = (unsigned char*)(((uintptr_t)kt_raw + 1023) & ~(uintptr_t)1023);
    const uint32_t smem = kv4_saddr(sm), bar = kv4_saddr(bars), bar_s = bar + 8 * KT_STAGES, bar_v = bar_s + 16, bar_o = bar_v + 16;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int b = blockIdx.z, h = blockIdx.y / a.n_blocks, j0 = (blockIdx.y % a.n_blocks) * KT_COLS;
    const int rank = blockIdx.x, S = gridDim.x;
    if (tid < KT_STAGES + 6) {
        const int n = tid < KT_STAGES || tid >= KT_STAGES + 4 ? 1 : tid < KT_STAGES + 2 ? 2 : KT_GROUP / 32;
        asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar + tid * 8), "r"(n) : "memory");
    }
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("fence.proxy.async;" ::: "memory");
    if (tid < KT_COLS) {
        s_poison[tid] = 0u;
        s_c[tid] = 0.f;
    }
    if (warp == 0) {
        __syncwarp();
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(kv4_saddr(&s_tmem)), "r"(KT_TMEM) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    if (DH == 64)
        for (int i = tid; i < 1024; i += KT_THREADS) *(uint4*)(sm + M::V + 2 * 16384 + 16 * i) = make_uint4(0u, 0u, 0u, 0u);
    kt_fence_before();
    __syncthreads();
    kt_fence_after();
    const uint32_t tmem = s_tmem;
    // (waited for before the first access to another CTA's shared memory: all have started)
    if (S > 1) asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory");
    pdl_wait();
    pdl_trigger();
    Kv4Sight sight;
    sight.nrows = min(max(a.rows[b] + a.rows_add, 0), a.c.max_len);
    sight.n_q = a.n_q; sight.mask_rows = a.mask_rows; sight.mask_words = a.mask_words;
    sight.mask = a.mask ? a.mask + (long long)b * a.n_q * a.mask_words : nullptr;
    const int i_first = j0 / a.G, i_last = (min(j0 + KT_COLS, a.ncol) - 1) / a.G;
    // rows [0, clear) are visible to every column of the block, rows from `end` on to none
    const int clear = max(0, a.mask ? sight.nrows - a.mask_rows : sight.nrows - a.n_q + i_first + 1);
    const int end = max(0, a.mask ? sight.nrows : sight.nrows - a.n_q + i_last + 1);
    const int ntile = (end + KV4_TILE - 1) / KV4_TILE, nstep = (ntile + KT_TILES - 1) / KT_TILES, nfull = clear / KT_ROWS;
    const unsigned char* base = kv4_tile(a.c, a.sl.slot[b], h, 0);
    auto fetch = [&](int t, int stage) {                               // (one thread)
        kv4_fetch(smem + stage * M::RAW, base + (long long)t * M::RAW, (uint32_t)(min(KT_TILES, ntile - t * KT_TILES) * TB), bar + stage * 8);
    };
    if (tid == 0) {
#pragma unroll
        for (int i = 0; i < KT_STAGES; ++i)
            if (rank + i * S < nstep) fetch(rank + i * S, i);
    }
    // ---- queries: a thread has a quarter of a column's channels; its row scaled by a power of two, so that bf16 is exact in fp16
    if (tid < KT_GROUP) {
        const int col = tid >> 2, c = tid & 3, j = j0 + col;
        float x[Q][8], mx = 0.f;
#pragma unroll
        for (int w = 0; w < Q; ++w) {
            if (j < a.ncol) {
                kv4_load8<bf16>(a.q, (long long)(b * a.n_q + j / a.G) * a.q_ld + (h * a.G + j % a.G) * DH + 32 * w + 8 * c, x[w]);
            } else {
#pragma unroll
                for (int i = 0; i < 8; ++i) x[w][i] = 0.f;
            }
#pragma unroll
            for (int i = 0; i < 8; ++i) mx = fmaxf(mx, fabsf(x[w][i]));
        }
        mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 1));
        mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 2));
        const int e = mx > 0.f ? min(max((int)(__float_as_uint(mx) >> 23) - 127, -100), 127) : 0;
        const float up = kv4_pow2(14 - e);
        if (c == 0) {
            s_f[col] = kv4_factor(e + 2, a.scale_log2);                // (2^-14 of the queries' scaling, 2^16 of the keys')
            s_m[col] = -KV4_NOTHING;
        }
#pragma unroll
        for (int w = 0; w < Q; ++w) {
            const float* y = x[w];
            const int chunk = (w & 1) * 4 + c;
            *(uint4*)(sm + M::Q + (w >> 1) * 8192 + col * 128 + ((chunk ^ (col & 7)) << 4)) =
                make_uint4(kv4_half2(y[0] * up, y[4] * up), kv4_half2(y[1] * up, y[5] * up), kv4_half2(y[2] * up, y[6] * up), kv4_half2(y[3] * up, y[7] * up));
        }
    }
    kt_fence_smem();
    __syncthreads();

    bool ok = true;                        // (once a wait has run out, the others do not wait: the CTA comes to its end)
    int n = 0;                             // steps taken
    if (warp < KT_GROUP / 32) {
        // ================ codes into values
        int base = KT_LEAST;                                           // |m| and 16 s of a row in the window are below 2^(base + 1)
        uint32_t above = 0u, below = 0u;                               // its ends in kt_reach's numbers (above 0: no row has had values yet)
        int stage = 0;
        uint32_t parity = 0;
        const __half2 sixteenth = __floats2half2_rn(0.0625f, 0.0625f);
        for (int t = rank; t < nstep; t += S, ++n) {
            if (ok) ok = kv4_wait(bar + stage * 8, parity);
            if (ok && n > 1) ok = kv4_wait(bar_o + 8 * (n & 1), ((n >> 1) - 1) & 1);
            const unsigned char* step = sm + stage * M::RAW;
            const bool edge = t >= nfull;
            // keys: a thread has half the chunks of a row, neighbouring rows' at different places (no bank twice); values: a quarter of the
            // groups of four channels of a pair of rows, so that the banks of eight pairs' loads differ, and of four pairs' stores
            const int r = tid & 127, c0 = (tid >> 7) * 2 + (r >> 1), pr = tid & 63, part = tid >> 6;
            const int swap = (pr & 4) | ((pr ^ (pr << 1)) & 2) | ((pr >> 1) & 1);
            const unsigned char *ktile = step + (r / KV4_TILE) * TB, *vtile = step + (pr / (KV4_TILE / 2)) * TB;
            uint32_t kp[Q], kx[2][Q], sw[Q], mw[Q], vx[2][Q];
            kv4_lds<Q>(ktile + kv4_s_at(DH, 0, r % KV4_TILE, 0), kp);      // s of the groups two by two, then m
            kv4_lds<Q>(vtile + kv4_s_at(DH, 1, 2 * pr % KV4_TILE, 0), sw);
            kv4_lds<Q>(vtile + kv4_m_at(DH, 1, 2 * pr % KV4_TILE, 0), mw);
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                kv4_lds<Q>(ktile + kv4_k_at(DH, r % KV4_TILE, 0, (c0 + i) & 3), kx[i]);
                kv4_lds<Q>(vtile + kv4_v_at(DH, 2 * pr % KV4_TILE, 0, (2 * part + i) ^ swap), vx[i]);
            }
            // ---- keys
            uint32_t big = 0u;
            {
#pragma unroll
                for (int w = 0; w < H; ++w) big = __vmaxu2(big, kt_reach(kp[w], kp[H + w]));
                const uint32_t top = max(big >> 16, big & 0xFFFFu);
                const int e = min(max((int)(top >> 7) - 127, -98), 130);   // all are below 2^(e + 1); a NaN stays one
                const float up = kt_pow2(-6 - e), up24 = kv4_pow2(18 - e);
                if (tid < KT_ROWS) s_rk[n & 1][r] = kv4_pow2(e - 10);
                __half2 s1[Q], m1[Q];
#pragma unroll
                for (int w = 0; w < Q; ++w) {
                    const float x = (w & 1 ? bf16_hi(kp[w >> 1]) : bf16_lo(kp[w >> 1])) * up24, y = (w & 1 ? bf16_hi(kp[H + (w >> 1)]) : bf16_lo(kp[H + (w >> 1)])) * up;
                    s1[w] = __floats2half2_rn(x, x);
                    m1[w] = __floats2half2_rn(y, y);
                }
                if (ok && n > 0) ok = kv4_wait(bar_s + 8 * ((n - 1) & 1), ((n - 1) >> 1) & 1);
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    const int c = (c0 + i) & 3;
#pragma unroll
                    for (int w = 0; w < Q; ++w) {
                        uint32_t v[4];
                        kt_values<false>(kx[i][w], s1[w], __hmul2(s1[w], sixteenth), m1[w], v);
                        *(uint4*)(sm + M::K + (w >> 1) * 16384 + r * 128 + ((((w & 1) * 4 + c) ^ (r & 7)) << 4)) = make_uint4(v[0], v[1], v[2], v[3]);
                    }
                }
            }
            // ---- the values' parameters
            uint32_t keep = 0xFFFFFFFFu;
            if (edge) {
                // nothing was fetched behind `end`
                const int r = t * KT_ROWS + 2 * pr;
                keep = r + 1 < end ? 0xFFFFFFFFu : r < end ? 0xFFFFu : 0u;
#pragma unroll
                for (int w = 0; w < Q; ++w) { sw[w] &= keep; mw[w] &= keep; }
            }
            uint32_t signs = 0u;                                       // (of scales: of rows that were never written)
#pragma unroll
            for (int w = 0; w < Q; ++w) {
                big = w ? __vmaxu2(big, kt_reach(sw[w], mw[w])) : kt_reach(sw[w], mw[w]);
                signs |= sw[w];
            }
            kt_fence_smem();
            // (of eight pairs of rows, four start with the odd one: no bank twice)
            const int flip = pr >> 2 & 1;
            float R0 = kv4_pow2(13 - base), R1 = R0;                   // of the pair's rows, in that order
            bool apart = false;
            // (an infinite or NaN parameter, or a row outside the window; behind `end` there is none)
            if (edge) big = (big & keep) | (below << 16 | below) & ~keep;
            const uint32_t b0 = big & 0xFFFFu, b1 = big >> 16;
            const bool unusual = kt_sync_or<1>((signs & 0x80008000u) != 0u || max(b0, b1) >= above || min(b0, b1) < below);
            if (unusual) {
                uint32_t nan = 0u, x0 = 0u, x1 = 0u;                   // groups of the pair's rows that hold a NaN: bits w and 4 + w
#pragma unroll
                for (int w = 0; w < Q; ++w)
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        const uint32_t x = (sw[w] >> (16 * i)) & 0xFFFFu, y = (mw[w] >> (16 * i)) & 0x7FFFu;
                        if (x < 0x7F80u && y < 0x7F80u) (i ? x1 : x0) = max(i ? x1 : x0, max(x + 0x0200u, y));
                        else nan |= 1u << (4 * i + w);
                    }
                const int e0 = max((int)(x0 >> 7) - 127, KT_LEAST), e1 = max((int)(x1 >> 7) - 127, KT_LEAST);
                if (above == 0u) {
                    int least = __reduce_min_sync(0xffffffffu, min(x0 > KT_ZERO ? e0 : KT_MOST + 1, x1 > KT_ZERO ? e1 : KT_MOST + 1));
                    if (lane == 0) s_least[warp] = least;
                    kt_sync<1>();
#pragma unroll
                    for (int w = 0; w < 8; ++w) least = min(least, s_least[w]);
                    if (least <= KT_MOST) {
                        base = min(least + KT_SPAN, KT_MOST);
                        above = min((uint32_t)(base + 1 + 127) << 7, 0x7F80u);
                        below = base - KT_WINDOW < KT_LEAST ? KT_ZERO + 1u : (uint32_t)(base - KT_WINDOW + 1 + 127) << 7;
                    }
                }
                int d0 = e0 <= base && e0 > base - KT_WINDOW ? 0 : e0 - base, d1 = e1 <= base && e1 > base - KT_WINDOW ? 0 : e1 - base;
                R0 = kv4_pow2(13 - base - (flip ? d1 : d0));
                R1 = kv4_pow2(13 - base - (flip ? d0 : d1));
                // (rows of zeros have weight and no values: a column does not go by them)
                if (x0 <= KT_ZERO) d0 = keep & 0xFFFFu ? -300 : 0;
                if (x1 <= KT_ZERO) d1 = keep >> 16 ? -300 : 0;
                if (part == 0) {
                    s_nan[n & 1][2 * pr] = nan & 15u;
                    s_nan[n & 1][2 * pr + 1] = nan >> 4;
                    s_d[n & 1][2 * pr] = (float)d0;
                    s_d[n & 1][2 * pr + 1] = (float)d1;
                }
                apart = kt_sync_or<1>(d0 != 0 || d1 != 0);
                if (edge && nan) {
                    // columns that do not see the row take nothing of it: left out here, put in where the probabilities are
#pragma unroll
                    for (int w = 0; w < Q; ++w) {
                        const uint32_t keep = (nan >> w & 1u ? 0u : 0xFFFFu) | (nan >> (4 + w) & 1u ? 0u : 0xFFFF0000u);
                        sw[w] &= keep;
                        mw[w] &= keep;
                    }
                }
            }
            if (warp == 0 && kt_elect()) {
                s_apart[n & 1] = apart;
                s_has_nan[n & 1] = unusual && edge;
                kt_fence_after();
#pragma unroll
                for (int kb = 0; kb < KB; ++kb)
#pragma unroll
                    for (int k = 0; k < 4; ++k)
                        kt_mma<true>(tmem + KT_S + (n & 1) * KT_COLS, kt_desc(smem + M::K + kb * 16384) + 2 * k, kt_desc(smem + M::Q + kb * 8192) + 2 * k, kb | k ? 1u : 0u);
                kt_commit(bar_s + 8 * (n & 1));
                kt_arrive(bar_s + 8 * (n & 1));
                // the step before this one's codes have been read (if they have not come, their barrier takes no second arrival)
                if (ok && n > 0 && t + (KT_STAGES - 1) * S < nstep) fetch(t + (KT_STAGES - 1) * S, stage == 0 ? KT_STAGES - 1 : stage - 1);
            }
            __syncwarp();
#pragma unroll
            for (int w = 0; w < Q; ++w) {
                sw[w] = __byte_perm(sw[w], 0u, flip ? 0x1032 : 0x3210);
                mw[w] = __byte_perm(mw[w], 0u, flip ? 0x1032 : 0x3210);
            }
            // ---- values: four channels of a group and of its neighbour, of two rows
            __half2 s1[2][H], m1[2][H];
#pragma unroll
            for (int w = 0; w < H; ++w) {
                s1[0][w] = __floats2half2_rn(bf16_lo(sw[2 * w]) * R0, bf16_lo(sw[2 * w + 1]) * R0);
                s1[1][w] = __floats2half2_rn(bf16_hi(sw[2 * w]) * R1, bf16_hi(sw[2 * w + 1]) * R1);
                m1[0][w] = __floats2half2_rn(bf16_lo(mw[2 * w]) * R0, bf16_lo(mw[2 * w + 1]) * R0);
                m1[1][w] = __floats2half2_rn(bf16_hi(mw[2 * w]) * R1, bf16_hi(mw[2 * w + 1]) * R1);
            }
            unsigned char* to = sm + M::V + (n & 1) * KB * 16384;
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const int g = (2 * part + i) ^ swap;
#pragma unroll
                for (int w = 0; w < H; ++w)
#pragma unroll
                    for (int o = 0; o < 2; ++o) {
                        uint32_t v[4];
                        kt_values<true>(__byte_perm(vx[i][2 * w], vx[i][2 * w + 1], o ^ flip ? 0x7632 : 0x5410), s1[o][w], __hmul2(s1[o][w], sixteenth), m1[o][w], v);
                        const int chunk = H * g + w, row = 2 * pr + (o ^ flip);
                        *(uint4*)(to + (chunk >> 3) * 16384 + row * 128 + (((chunk & 7) ^ (row & 7)) << 4)) = make_uint4(v[0], v[1], v[2], v[3]);
                    }
            }
            kt_fence_smem();
            __syncwarp();
            if (lane == 0) kt_arrive(bar_v + 8 * (n & 1));
            if (++stage == KT_STAGES) { stage = 0; parity ^= 1u; }
        }
        if (tid == 0) s_base = base;
    } else {
        // ================ scores into probabilities
        const int quarter = warp & 3, half = (warp - KT_GROUP / 32) >> 2;
        const uint32_t my_tmem = tmem + ((uint32_t)(quarter * 32) << 16) + half * 32;     // this warp's lanes, its half of the columns
        const int row = quarter * 32 + lane;
        float l[32];                                                   // sums of this row's weights, every 128th row's
#pragma unroll
        for (int i = 0; i < 32; ++i) l[i] = 0.f;
        bool scaled = false;                                           // some column's c is not 0 (the same in all of these threads)
        // the columns' largest of the rows' x: lane L of the warp gets that of its column L, by halving what each lane has to compare
        auto largest = [&](float (&x)[32]) {
#pragma unroll
            for (int o = 16; o > 0; o >>= 1) {
                const bool high = (lane & o) != 0;
#pragma unroll
                for (int i = 0; i < 16; ++i)
                    if (i < o) {
                        const float keep = high ? x[i + o] : x[i], give = high ? x[i] : x[i + o];
                        x[i] = fmaxf(keep, __shfl_xor_sync(0xffffffffu, give, o));
                    }
            }
            s_top[quarter][half * 32 + lane] = x[0];
            kt_sync<2>();
        };
        for (int t = rank; t < nstep; t += S, ++n) {
            if (ok) ok = kv4_wait(bar_s + 8 * (n & 1), (n >> 1) & 1);
            kt_fence_after();
            const bool apart = s_apart[n & 1] || scaled;
            const float rk = s_rk[n & 1][row];
            float y[32], top = -INFINITY;                              // by how much scores are above the columns' maxima
            float counts = 1.f;                                        // what the probabilities written count for in the sums
            uint32_t see = 0xFFFFFFFFu;
            {
                uint32_t raw[32];
                kt_ld32(my_tmem + KT_S + (n & 1) * KT_COLS, raw);
#pragma unroll
                for (int i = 0; i < 32; i += 4) {
                    const float4 f = *(const float4*)(s_f + half * 32 + i);
                    const ulonglong2 m = *(const ulonglong2*)(s_m + half * 32 + i);
                    float t[4];
#pragma unroll
                    for (int k = 0; k < 4; k += 2) kv4_unpack2(kv4_mul2(kv4_pack2(__uint_as_float(raw[i + k]), __uint_as_float(raw[i + k + 1])), kv4_pack2(rk, rk)), t[k], t[k + 1]);
                    kv4_above(t[0], t[1], f.x, f.y, m.x, y[i], y[i + 1]);
                    kv4_above(t[2], t[3], f.z, f.w, m.y, y[i + 2], y[i + 3]);
                }
            }
            if (t >= nfull) {
                const uint32_t mine = kt_window(sight, t * KT_ROWS + quarter * 32, min((j0 + half * 32 + lane) / a.G, a.n_q - 1));
                see = 0u;
#pragma unroll
                for (int i = 0; i < 32; ++i) {
                    see |= (__shfl_sync(0xffffffffu, mine, i) >> lane & 1u) << i;
                    if (!(see >> i & 1u)) y[i] = -INFINITY;
                }
            }
#pragma unroll
            for (int i = 0; i < 32; ++i) top = fmaxf(top, y[i]);
            if (ok && n > 1) ok = kv4_wait(bar_o + 8 * (n & 1), ((n >> 1) - 1) & 1);       // P may be overwritten
            if (kt_sync_or<2>(top > KV4_LAZY + KT_LIFT || apart)) {
                uint32_t raw[32];
                kt_ld32(my_tmem + KT_S + (n & 1) * KT_COLS, raw);
                float x[32];
#pragma unroll
                for (int i = 0; i < 32; ++i) {
                    y[i] = __fmul_rn(__uint_as_float(raw[i]) * rk, s_f[half * 32 + i]);
                    if (!(see >> i & 1u)) y[i] = -INFINITY;
                    x[i] = y[i];
                }
                largest(x);
                float d = 0.f, old = 0.f, m = 0.f;                     // old, m: of the column that this thread looks after, if any
                const int c = tid - KT_GROUP;
                if (c < KT_COLS) {
                    // (a column's own scores decide)
                    const float z = fmaxf(fmaxf(s_top[0][c], s_top[1][c]), fmaxf(s_top[2][c], s_top[3][c]));
                    old = -s_m[c];
                    m = z - old > KV4_LAZY + KT_LIFT ? z - KT_LIFT : old;
                    s_m[c] = -m;
                    s_fall[c] = s_fall_o[c] = kv4_exp2(old - m);
                }
                kt_sync<2>();
#pragma unroll
                for (int i = 0; i < 32; ++i) y[i] += s_m[half * 32 + i];
                if (apart) {
                    // what the rows' 2^d does to the probabilities: below 2^15, and not next to nothing where the maximum has been raised
                    d = s_apart[n & 1] ? s_d[n & 1][row] : 0.f;
#pragma unroll
                    for (int i = 0; i < 32; ++i) x[i] = y[i] + d;
                    largest(x);
                    bool some = false;
                    if (c < KT_COLS) {
                        const float z = fmaxf(fmaxf(s_top[0][c], s_top[1][c]), fmaxf(s_top[2][c], s_top[3][c])), was = s_c[c];
                        float now = was;
                        if (z + was > 15.f) now = KT_LIFT - ceilf(z);
                        else if (m > old && z + was < 0.f) now = fminf(KT_LIFT - ceilf(z), was + floorf(fminf(m - old, 300.f)));
                        now = fminf(now, 300.f);
                        s_c[c] = now;
                        s_fall_o[c] = kv4_exp2((old - m) + (now - was));
                        some = now != 0.f;
                    }
                    scaled = kt_sync_or<2>(some);
                }
                if (n > 0) {
                    if (ok) ok = kv4_wait(bar_o + 8 * ((n - 1) & 1), ((n - 1) >> 1) & 1);
                    kt_fence_after();
                    uint32_t o[32];
                    kt_ld32(my_tmem + KT_O, o);
#pragma unroll
                    for (int i = 0; i < 32; ++i) {
                        l[i] *= s_fall[half * 32 + i];
                        o[i] = __float_as_uint(__uint_as_float(o[i]) * s_fall_o[half * 32 + i]);
                    }
                    kt_st32(my_tmem + KT_O, o);
                }
                if (apart) {
                    // the sums take the weights themselves
                    counts = 0.f;
#pragma unroll
                    for (int i = 0; i < 32; ++i) {
                        l[i] += kv4_exp2(y[i]);
                        y[i] += d + s_c[half * 32 + i];
                    }
                }
            }
            // ---- probabilities
#pragma unroll
            for (int i = 0; i < 32; i += 8) {
                uint32_t v[4];
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const float p0 = kv4_exp2(y[i + 2 * k]), p1 = kv4_exp2(y[i + 2 * k + 1]);
                    l[i + 2 * k] = fmaf(p0, counts, l[i + 2 * k]);
                    l[i + 2 * k + 1] = fmaf(p1, counts, l[i + 2 * k + 1]);
                    v[k] = kv4_half2(p0, p1);
                }
                const int chunk = half * 4 + i / 8;
                *(uint4*)(sm + M::P + (n & 1) * 16384 + row * 128 + ((chunk ^ (row & 7)) << 4)) = make_uint4(v[0], v[1], v[2], v[3]);
            }
            if (s_has_nan[n & 1]) {
                // rows that hold a NaN: every column that sees them has it in that group's channels
                const uint32_t mine = s_nan[n & 1][row];
                if (mine) {
#pragma unroll 1
                    for (int i = 0; i < 32; ++i)
                        if (see >> i & 1u) atomicOr(&s_poison[half * 32 + i], mine);
                }
            }
            kt_fence_smem();
            kt_fence_before();
            kt_sync<2>();
            if (warp == KT_GROUP / 32) {
                if (ok) ok = kv4_wait(bar_v + 8 * (n & 1), (n >> 1) & 1);
                if (kt_elect()) {
                    kt_fence_after();
#pragma unroll
                    for (int k = 0; k < KT_ROWS / 16; ++k)
                        kt_mma<false>(tmem + KT_O, kt_desc(smem + M::V + (n & 1) * KB * 16384, DH == 64 ? (2 - (n & 1)) * 16384 : 16384) + 128 * k,
                                      kt_desc(smem + M::P + (n & 1) * 16384) + 128 * k, n || k ? 1u : 0u);
                    kt_commit(bar_o + 8 * (n & 1));
                }
                __syncwarp();
            }
        }
        // the columns' sums, by halving
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) {
            const bool high = (lane & o) != 0;
#pragma unroll
            for (int i = 0; i < 16; ++i)
                if (i < o) l[i] = (high ? l[i + o] : l[i]) + __shfl_xor_sync(0xffffffffu, high ? l[i] : l[i + o], o);
        }
        kt_sync<2>();
        s_top[quarter][half * 32 + lane] = l[0];
    }
    // ---- the CTA's columns: maximum, sum, output (over the sum before the scale is undone: a mean is no larger than its values)
    if (ok && n > 0) ok = kv4_wait(bar_o + 8 * ((n - 1) & 1), ((n - 1) >> 1) & 1);
    if (!ok) {
        // a copy or a product has not come: time for what is in flight, and the result is NaN
        const long long t0 = clock64();
        while (clock64() - t0 < 4000000ll) {}
    }
    ok = __syncthreads_and(ok) != 0;
    kt_fence_after();
    // (every thread sends one column's maximum and sum to one of the cluster's CTAs)
    cg::cluster_group cluster = cg::this_cluster();
    static_assert(KT_THREADS == KT_COLS * KT_CLUSTER, "a column of a CTA to a thread");
    if (S > 1) asm volatile("barrier.cluster.wait.aligned;" ::: "memory");
    if (tid < S * KT_COLS) {
        const int col = tid % KT_COLS;
        const float l = ok ? (s_top[0][col] + s_top[1][col]) + (s_top[2][col] + s_top[3][col]) : __uint_as_float(0x7FC00000u);
        *(S > 1 ? cluster.map_shared_rank(&s_part[rank][col], tid / KT_COLS) : &s_part[0][col]) = make_float2(-s_m[col], l);
        if (tid < KT_COLS) s_inv[col] = l == 0.f ? 0.f : 1.f / l;      // nothing visible: zeros
    }
    __syncthreads();
    float* sO = (float*)sm;
    if (n == 0) {
        // (no row at all: zeros)
        for (int i = tid; i < KT_COLS * LDO; i += KT_THREADS) sO[i] = 0.f;
    } else {
        // a warp has a quarter of the lanes, 16 columns
        const int quarter = warp & 3, col = (warp >> 2) * 16;
        uint32_t o[16];
        if (quarter * 32 < DH) {
            kt_ld16(tmem + ((uint32_t)(quarter * 32) << 16) + col + KT_O, o);
            const int at = quarter * 32 + lane, w = at % (4 * Q) / 8 * 2 + (at & 1), ch = 32 * w + at / (4 * Q) * 4 + (at >> 1 & 3);
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const int e = min(max(s_base - 13 - (int)s_c[col + i], -250), 250);
                sO[(col + i) * LDO + ch + APART * w] = s_poison[col + i] >> w & 1u ? __uint_as_float(0x7FC00000u)
                                                                                  : __uint_as_float(o[i]) * s_inv[col + i] * kv4_pow2(e / 2) * kv4_pow2(e - e / 2);
            }
        }
    }
    kt_fence_before();
    __syncthreads();
    if (warp == 0) {
        __syncwarp();
        kt_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(KT_TMEM) : "memory");
    }
    // ---- the CTAs of the cluster: each writes its share of the columns' channels
    if (S > 1) cluster.sync();
    else __syncthreads();
    const int cols = min(KT_COLS, a.ncol - j0);
    for (int i = rank * KT_THREADS + tid; i < cols * (DH / 4); i += S * KT_THREADS) {
        const int col = i / (DH / 4), ch = (i % (DH / 4)) * 4;
        float m = KV4_NOTHING, l = 0.f;
        float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
        for (int r = 0; r < S; ++r) m = fmaxf(m, s_part[r][col].x);
        for (int r = 0; r < S; ++r) l = fmaf(s_part[r][col].y, kv4_exp2(s_part[r][col].x - m), l);
        const float inv = l == 0.f ? 0.f : 1.f / l;
#pragma unroll 4
        for (int r = 0; r < S; ++r) {
            const float f = s_part[r][col].y * kv4_exp2(s_part[r][col].x - m) * inv;
            const float4 y = *(const float4*)(S > 1 ? cluster.map_shared_rank(sO + col * LDO + ch + ch / 32 * APART, r) : sO + col * LDO + ch + ch / 32 * APART);
            x.x = fmaf(y.x, f, x.x); x.y = fmaf(y.y, f, x.y); x.z = fmaf(y.z, f, x.z); x.w = fmaf(y.w, f, x.w);
        }
        kv4_put<bf16>(a, b, h, j0 + col, ch, DH, x, 1.f);
    }
    if (S > 1) cluster.sync();          // nobody leaves while its shared memory may still be read
}

template <int DH>
cudaError_t kt_launch(Kv4AttnArgs& a, int dev, int num_sms, cudaStream_t st) {
    static bool attr_set[HIVIS_MAX_DEVICES] = {false};
    auto kernel = kv4_tc_kernel<DH>;
    if (dev < 0 || dev >= HIVIS_MAX_DEVICES || !attr_set[dev]) {
        cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, KtSmem<DH>::BYTES);
        if (e == cudaSuccess) e = cudaFuncSetAttribute(kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
        if (e != cudaSuccess) return e;
        if (dev >= 0 && dev < HIVIS_MAX_DEVICES) attr_set[dev] = true;
    }
    a.n_blocks = (a.ncol + KT_COLS - 1) / KT_COLS;
    // a CTA has an SM to itself: sixteen would have to find a whole GPC free (8 x 64 columns of 2048 rows: 24 us, with eight 12)
    const int S = kv4_cluster(a.sl.n * a.c.Hkv * a.n_blocks, a.c.max_len, KT_ROWS, num_sms, KT_CLUSTER);
    const dim3 grid((unsigned)S, (unsigned)(a.c.Hkv * a.n_blocks), (unsigned)a.sl.n);
    return launch_cluster_pdl(kernel, S, grid, dim3(KT_THREADS), KtSmem<DH>::BYTES, st, a);
}

}  // namespace

cudaError_t launch_kv4_attn_tc(Kv4AttnArgs& a, int dev, int num_sms, cudaStream_t st) {
    return a.c.dh == 128 ? kt_launch<128>(a, dev, num_sms, st) : kt_launch<64>(a, dev, num_sms, st);
}
