// A key/value cache held in 4 bits: the format, shared by the kernels that write, read and attend over it.
//
// Per cache row, KV head and group of 32 channels: m = the smallest value rounded down to bf16, s = (the largest - m) / 15
// rounded up to bf16, and per channel the integer n in 0..15 nearest to (x - m) / s (the lower one on a tie); the channel
// stands for m + s n.  Rounded this way round, m and m + 15 s enclose the group, so no value is off by more than s / 2.
// A group that holds a NaN or an infinity, or whose range overflows, gets m = s = NaN.
//
// Rows lie in tiles of 16, [slot][KV head][row / 16], 20 dh bytes each, so that one copy brings everything the attention needs of 16
// rows: the codes of K (16 rows of dh / 2 bytes), those of V, then per row s and m of K's groups (dh / 32 bf16 numbers each), then per
// pair of rows s and m of V's groups (dh / 32 words each, the even row's number in the lower half, the odd row's in the upper).
// Codes are in the order in which mma.m16n8k16 wants them as its A operand, so that the attention takes them from memory to the
// tensor core with a mask and a shift:
//   K  (A = keys: 16 rows x 16 channels).  A row is four chunks of dh / 8 bytes, chunk c for the lanes with lane % 4 = c; word w
//      of a chunk holds channels 32 w + 8 c + i, nibble i.
//   V  (A = values transposed: 16 channels x 16 rows).  A register holds one channel of two neighbouring rows, so rows 2 p and
//      2 p + 1 share dh / 4 words: word u = (dh / 32) g + w holds channels 32 w + 4 g + i, nibble i of the even row in the lower
//      half and of the odd row in the upper half.  A row owns whole 16-bit halves: writing it leaves its neighbour alone.
#pragma once
#include "hivis_internal.cuh"

#include <cuda_fp16.h>

#define KV4_GROUP 32
#define KV4_TILE 16
__host__ __device__ __forceinline__ constexpr int kv4_tile_bytes(int dh) { return 20 * dh; }

// the tile of a head that holds `row`
__device__ __forceinline__ unsigned char* kv4_tile(const Kv4View& c, int slot, int h, int row) {
    return c.data + (((long long)slot * c.Hkv + h) * (c.max_len / KV4_TILE) + row / KV4_TILE) * kv4_tile_bytes(c.dh);
}

// A group's parameters in one word: s in the upper half, m in the lower.
__device__ __forceinline__ float kv4_scale(uint32_t w) { return __uint_as_float(w & 0xFFFF0000u); }
__device__ __forceinline__ float kv4_min(uint32_t w) { return __uint_as_float(w << 16); }

// Parameters of a group whose smallest and largest value are lo and hi.  m: rounded down.  s: the smallest bf16 number with 15 s >=
// hi - m (NaN where lo or hi is not finite: taken with min and max that keep a NaN).  15 s is an fp32 number, so the difference may be rounded up before it is compared; a product with 1 / 15 finds s up to
// one bf16 step.
__device__ __forceinline__ uint32_t kv4_params(float lo, float hi) {
    const uint32_t m = __bfloat16_as_ushort(__float2bfloat16_rd(lo));
    const float d = __fsub_ru(hi, __uint_as_float(m << 16));
    uint32_t s = (__float_as_uint(d * (1.f / 15.f)) + 0xFFFFu) & 0xFFFF0000u;
    if (15.f * __uint_as_float(s) < d) s += 0x10000u;
    else if (s && 15.f * __uint_as_float(s - 0x10000u) >= d) s -= 0x10000u;
    // (lo so low that it rounds to -infinity; a range beyond fp32's)
    return fabsf(lo) < INFINITY && (m & 0x7F80u) != 0x7F80u && s < 0x7F800000u && d < INFINITY ? s | m : 0x7FC07FC0u;
}

// The code of x, decided without error; n is an integer next to the quotient or the one beside it.  x - m may need more than 24 bits:
// e is what d = x - m lost.  r = d - n s is exact (n s has 12 bits, and the difference no bit below d's last), and so are the
// comparisons with s / 2, a multiple of d's last bit.
__device__ __forceinline__ unsigned kv4_code_exact(float x, float m, float s, float n, float up) {
    float d = x - m;
    const float bb = d - x;
    float e = (x - (d - bb)) - (m + bb);
    d *= up;                                                // (a power of two, for both sides of the quotient)
    e *= up;
    s *= up;
    const float r = fmaf(-n, s, d), half = 0.5f * s;
    if (r > half || (r == half && e > 0.f)) n += 1.f;
    else if (r < -half || (r == -half && e <= 0.f)) n -= 1.f;
    return (unsigned)fminf(fmaxf(n, 0.f), 15.f);
}

// min and max that keep a NaN
__device__ __forceinline__ float kv4_min_nan(float x, float y) {
    float r;
    asm("min.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(x), "f"(y));
    return r;
}
__device__ __forceinline__ float kv4_max_nan(float x, float y) {
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(x), "f"(y));
    return r;
}
// two fp32 operations at once
__device__ __forceinline__ u64 kv4_pack2(float x, float y) {
    u64 r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(x), "f"(y));
    return r;
}
__device__ __forceinline__ void kv4_unpack2(u64 v, float& x, float& y) { asm("mov.b64 {%0, %1}, %2;" : "=f"(x), "=f"(y) : "l"(v)); }
__device__ __forceinline__ u64 kv4_mul2(u64 a, u64 b) {
    u64 r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ u64 kv4_add2(u64 a, u64 b) {
    u64 r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}

__device__ __forceinline__ u64 kv4_fma2(u64 a, u64 b, u64 c) {
    u64 r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
    return r;
}

// Codes of 8 values as 8 nibbles.  t = (x - m) / s comes from a product with an approximate reciprocal, off by less than 2^-18, and n
// is the integer next to t - 2^-17: never above the code, and at a tie the lower one.  r = (x - m) - n s is exact but for what x - m
// lost, at most 2^-20 s, so that n is the code where r is below s / 2 by more than that.  Of bf16 values one in some hundreds is a tie:
// r = s / 2 says so where x - m is exact, which it is if neither x nor m is below 2^-12 s (both are then multiples of 2^-20 s, and their
// difference is below 2^4 s).  The exact form decides about what is left.  BF16: whether the values are bf16 numbers.
template <bool BF16>
__device__ __forceinline__ uint32_t kv4_codes8(const float (&x)[8], uint32_t params) {
    const float m = kv4_min(params), s = kv4_scale(params);
    uint32_t w = 0u;
    if (s >= 1e-30f) {
        constexpr float MAGIC = 12582912.f;                 // 1.5 * 2^23: the nearest integer in the low bits
        const float lim = s * (0.5f - 0x1p-18f), half = 0.5f * s;
        float inv, off = 0.f, r[8], u[8];
        asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(inv) : "f"(s));
        const u64 mm = kv4_pack2(-m, -m), ii = kv4_pack2(inv, inv), ss = kv4_pack2(-s, -s), up = kv4_pack2(MAGIC, MAGIC), down = kv4_pack2(-MAGIC, -MAGIC),
                  less = kv4_pack2(-0x1p-17f, -0x1p-17f);
#pragma unroll
        for (int i = 0; i < 8; i += 2) {
            const u64 d = kv4_add2(kv4_pack2(x[i], x[i + 1]), mm), uu = kv4_add2(kv4_fma2(d, ii, less), up);
            kv4_unpack2(kv4_fma2(kv4_add2(uu, down), ss, d), r[i], r[i + 1]);
            kv4_unpack2(uu, u[i], u[i + 1]);
            off = fmaxf(off, fmaxf(r[i], r[i + 1]));
        }
#pragma unroll
        for (int i = 7; i >= 0; --i) w = w * 16u + __float_as_uint(u[i]);      // (0x4B400000 above n: together 0x3F400000 in 32 bits)
        w -= 0x3F400000u;
        if (off > lim) {
            uint32_t which = 0u;
#pragma unroll
            for (int i = 0; i < 8; ++i) which |= r[i] > lim ? 1u << i : 0u;
            if (BF16) {
                uint32_t ties = 0u;
                float least = m == 0.f ? s : fabsf(m);
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    ties |= r[i] == half ? 1u << i : 0u;
                    least = fminf(least, fabsf(x[i]));
                }
                if (least >= s * 0x1p-12f) which &= ~ties;
            }
#pragma unroll 1
            for (; which; which &= which - 1u) {
                const int i = __ffs((int)which) - 1;
                float y = x[0];
#pragma unroll
                for (int k = 1; k < 8; ++k) y = i == k ? x[k] : y;
                w = (w & ~(15u << (4 * i))) | (kv4_code_exact(y, m, s, (float)(w >> (4 * i) & 15u), 1.f) << (4 * i));
            }
        }
    } else if (s > 0.f) {
        // (a NaN group and one of equal values keep zeros)
#pragma unroll
        for (int i = 0; i < 8; ++i) w |= kv4_code_exact(x[i], m, s, rintf((x[i] - m) * 0x1p96f / (s * 0x1p96f)), 0x1p96f) << (4 * i);
    }
    return w;
}

// Offsets in a tile, r = row % 16.  The 8 codes of channels [32 w + 8 c, + 8): K, one word; V, the lower four nibbles into the row's
// half of word g = 2 c of the group, the upper four into that of g = 2 c + 1.  Parameters of group w (which: 0 K, 1 V).
__device__ __forceinline__ int kv4_k_at(int dh, int r, int w, int c) { return r * (dh / 2) + c * (dh / 8) + w * 4; }
__device__ __forceinline__ int kv4_v_at(int dh, int r, int w, int g) { return 8 * dh + (r & ~1) * (dh / 2) + ((dh / 32) * g + w) * 4 + (r & 1) * 2; }
__device__ __forceinline__ int kv4_s_at(int dh, int which, int r, int w) {
    return which == 0 ? 16 * dh + r * (dh / 8) + 2 * w : 18 * dh + (r >> 1) * (dh / 4) + 4 * w + 2 * (r & 1);
}
__device__ __forceinline__ int kv4_m_at(int dh, int which, int r, int w) { return kv4_s_at(dh, which, r, w) + (which == 0 ? dh / 16 : dh / 8); }

// One lane's 32 values - channels 32 w .. 32 w + 31 of row r, bf16 numbers - into a tile; which: 0 K, 1 V.
__device__ __forceinline__ void kv4_store32(unsigned char* tile, int dh, int which, int r, int w, const float (&x)[32]) {
    float lo = x[0], hi = x[0];
#pragma unroll
    for (int i = 1; i < 32; ++i) {
        lo = kv4_min_nan(lo, x[i]);
        hi = kv4_max_nan(hi, x[i]);
    }
    const uint32_t params = kv4_params(lo, hi);
    *(uint16_t*)(tile + kv4_s_at(dh, which, r, w)) = (uint16_t)(params >> 16);
    *(uint16_t*)(tile + kv4_m_at(dh, which, r, w)) = (uint16_t)params;
#pragma unroll
    for (int c = 0; c < 4; ++c) {
        float y[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) y[i] = x[8 * c + i];
        const uint32_t codes = kv4_codes8<true>(y, params);
        if (which == 0) {
            *(uint32_t*)(tile + kv4_k_at(dh, r, w, c)) = codes;
        } else {
            *(uint16_t*)(tile + kv4_v_at(dh, r, w, 2 * c)) = (uint16_t)codes;
            *(uint16_t*)(tile + kv4_v_at(dh, r, w, 2 * c + 1)) = (uint16_t)(codes >> 16);
        }
    }
}
