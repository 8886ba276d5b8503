// mc_kv4.cuh -- the 4-bit form of a cached row: groups of 64 elements as s (c - z), c and z of 4 bits,
// s of 4 significant bits (mc.h has the layout).  s (c - z) is exact in bf16 and fp16.
#pragma once
#include "mc_attn.h"

namespace mc {

constexpr int kKv4Group = 64;
__host__ __device__ constexpr int kv4_code_bytes(int D) { return D / 2; }   // of a row
__host__ __device__ constexpr int kv4_word_bytes(int D) { return D / 32; }  // of a row: 16 bits a group
__host__ __device__ constexpr int kv4_row_bytes(int D) { return kv4_code_bytes(D) + kv4_word_bytes(D); }

// Address of (page, head): a block of codes [page_size][D / 2] and, behind them, words [page_size][D / 64].
// (KvView's k and v are bytes here, page_stride counts them.)
template <int D>
__device__ __forceinline__ int64_t kv4_offset(const KvView &c, int page, int h)
{
    return page * c.page_stride + (int64_t)h * (c.page_size * kv4_row_bytes(D));
}
template <int D>
__device__ __forceinline__ const uint8_t *kv4_block(const KvView &c, const uint16_t *side, int page, int h)
{
    return reinterpret_cast<const uint8_t *>(side) + kv4_offset<D>(c, page, h);
}

__device__ __forceinline__ float kv4_scale(uint32_t word) { return __uint_as_float((word & 0xfff0u) << 16); }

// Larger of two pairs, NaN if either is one.
template <bool BF16>
__device__ __forceinline__ uint32_t max2(uint32_t a, uint32_t b)
{
    uint32_t r;
    if (BF16) asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    else asm("max.NaN.f16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
}

template <bool BF16>
__device__ __forceinline__ uint32_t min2(uint32_t a, uint32_t b)
{
    uint32_t r;
    if (BF16) asm("min.NaN.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    else asm("min.NaN.f16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
}

// Codes held to z - most .. z + most, where more steps than `most` pass the type's largest number.
template <bool BF16>
__device__ __noinline__ uint32_t kv4_held(uint32_t codes, int z, int most)
{
    uint32_t r = 0;
    for (int i = 0; i < 32; i += 4) r |= (uint32_t)max(z - most, min(z + most, (int)(codes >> i & 15))) << i;
    return r;
}

// A group's 64 elements, 8 in each of 8 neighbouring lanes (x: pairs of them, in order): returns the lane's
// word of codes, and the group's scale and zero point in `word`.  All 8 lanes take part.
//
// s is the span's mantissa m, 24 bits, times 16 / 15, rounded up to four: n = ceil(16 m / (15 * 2^20)), 9 .. 18.
// Quotients x / s that are not halves lie at least 2^-12 from them (s has 4 bits, x at most 11 and at
// least an ulp of 2^-12 s where it matters), so half of that added makes the approximate reciprocal's rounding
// that of the exact one with halves upward.
template <bool BF16>
__device__ __forceinline__ uint32_t kv4_quantise(const uint32_t (&x)[4], uint32_t &word)
{
    constexpr float kTie = 0x1p-14f, kShift = 12582912.f;  // 1.5 * 2^23: integers stand in the low bits
    constexpr float kMost = BF16 ? 0x1.fep127f : 65504.f;
    constexpr uint32_t kLeast = BF16 ? (127u - 100) << 23 : (127u - 20) << 23;
    uint32_t top = max2<BF16>(max2<BF16>(x[0], x[1]), max2<BF16>(x[2], x[3]));
    uint32_t low = min2<BF16>(min2<BF16>(x[0], x[1]), min2<BF16>(x[2], x[3])) ^ 0x80008000u;
    // (largest, largest of the negatives) in one register
    uint32_t ends = max2<BF16>(__byte_perm(top, low, 0x5410), __byte_perm(top, low, 0x7632));
#pragma unroll
    for (int m = 4; m >= 1; m >>= 1) ends = max2<BF16>(ends, __shfl_xor_sync(0xffffffffu, ends, m));
    ends = max2<BF16>(ends, 0u);
    const float2 e = unpack2<BF16>(ends);  // hi, -lo
    const uint32_t span = __float_as_uint(fmaf(e.x, 0.0625f, e.y * 0.0625f));
    const bool odd = span >= 0x7f800000u;  // infinite or NaN
    const uint32_t m = (span & 0x7fffffu) | 0x800000u, n = (16u * m + (15u << 20) - 1) / (15u << 20);
    uint32_t bits = span & 0x7f800000u;
    bits += n <= 16 ? (n - 8) << 20 : (1u << 23) + (1u << 20);
    bits = max(bits, kLeast);
    const float s = __uint_as_float(bits), inv = rcp(s);
    const float zs = fmaf(e.y, inv, kTie) + kShift, z = zs - kShift;  // (not negative, at most 15)
    word = odd ? 0x7ff0u : (bits >> 16) | (__float_as_uint(zs) & 15u);
    const float base = kShift + z;
    uint32_t r = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {  // (no quotient rounds below -z)
        const float2 f = unpack2<BF16>(x[i]);
        float a, b;
        unpair2(add2(fma2(pair2(f.x, f.y), pair2(inv, inv), pair2(kTie, kTie)), pair2(base, base)), a, b);
        r += __byte_perm(__float_as_uint(fminf(a, kShift + 15.f)), __float_as_uint(fminf(b, kShift + 15.f)), 0x5410) << (4 * i);
    }
    if (kMost * inv < 16.f && !odd) r = kv4_held<BF16>(r, (int)z, (int)(kMost * inv));
    return odd ? 0u : r;
}

// Elements 2 i and 2 i + 1 of a row.
template <int D>
__device__ __forceinline__ float2 kv4_pair(const KvView &c, const uint16_t *side, int page, int h, int row, int i)
{
    const uint8_t *block = kv4_block<D>(c, side, page, h);
    const int g = i / 32, at = i % 32 / 4 * (D / kKv4Group) + g, j = 4 * (i % 4);
    const uint32_t codes = *reinterpret_cast<const uint32_t *>(block + row * kv4_code_bytes(D) + 4 * at);
    const uint32_t word = *reinterpret_cast<const uint16_t *>(block + c.page_size * kv4_code_bytes(D) + row * kv4_word_bytes(D) + 2 * g);
    const float s = kv4_scale(word);
    const int z = word & 15;
    return make_float2(s * (float)((int)(codes >> j & 15) - z), s * (float)((int)(codes >> (16 + j) & 15) - z));
}

// The eight elements of a word of codes as pairs of the type, exactly: (2^k + c) - (2^k + z), with the code
// in the low mantissa bits of 2^k, then the scale.
template <bool BF16>
struct Kv4Pairs {
    static constexpr uint32_t kMagic = BF16 ? 0x43004300u : 0x64006400u;  // 128, 1024
    static __device__ __forceinline__ uint32_t zeros(uint32_t word) { return (word & 15u) * 0x10001u + kMagic; }
    static __device__ __forceinline__ uint32_t magic(uint32_t w, int j) { return lop_and_or(w >> (4 * j), 0x000f000fu, kMagic); }
    static __device__ __forceinline__ uint32_t sub(uint32_t a, uint32_t b)
    {
        uint32_t r;
        if (BF16) asm("sub.rn.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
        else asm("sub.rn.f16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
        return r;
    }
    static __device__ __forceinline__ uint32_t mul(uint32_t a, uint32_t b)
    {
        uint32_t r;
        if (BF16) asm("mul.rn.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
        else asm("mul.rn.f16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
        return r;
    }
    // a group's scale, twice
    static __device__ __forceinline__ uint32_t scales(uint32_t word)
    {
        if (BF16) return (word & 0xfff0u) * 0x10001u;
        const float s = kv4_scale(word);
        return pack2<BF16>(s, s);
    }
};

}  // namespace mc
