// mc_attn_row.cuh -- a row of attention by the definition, key by key: what the kernels fall back to where a hidden
// key is infinite or NaN.  Q4: over the 4-bit cache.
#pragma once
#include <math.h>

#include "mc_kv4.cuh"

namespace mc {

// Whether a key or value in the rows [from, to) of head h of sequence b is infinite or NaN.
// `warps` warps look, 16 rows at a time each, this one as number `warp`; the answer is the warp's.
template <int D, bool BF16, bool Q4>
__device__ __noinline__ bool odd_keys(const AttnParams &p, int b, int h, int from, int to, int warp, int warps, int lane)
{
    constexpr uint32_t kExp = BF16 ? 0x7f80u : 0x7c00u;  // infinities and NaN have the exponent's bits all set
    bool odd = false;
    for (int j = (from & ~15) + 16 * warp; j < to; j += 16 * warps) {
        int row;
        const int i = p.c.page.div(j, row), page = seq_page(p.b, p.c, b, i, nullptr);
        if (page < 0) continue;
        if constexpr (Q4) {  // a lane's row of one side: the groups' scales
            const int r = lane & 15;
            const uint8_t *words = kv4_block<D>(p.c, lane < 16 ? p.c.k : p.c.v, page, h) + p.c.page_size * kv4_code_bytes(D) +
                                   (row + r) * kv4_word_bytes(D);
            if (j + r < from || j + r >= to) continue;
#pragma unroll
            for (int g = 0; g < D / kKv4Group; ++g) odd |= (reinterpret_cast<const uint16_t *>(words)[g] & 0x7f80u) == 0x7f80u;
            continue;
        }
        const int64_t at = page * p.c.page_stride + ((int64_t)h * p.c.page_size + row) * D;
#pragma unroll 2
        for (int c = lane; c < 2 * D; c += 32) {  // 16-byte chunks of the 16 rows
            const int r = j + c / (D / 8);
            if (r < from || r >= to) continue;
            const uint4 k = *reinterpret_cast<const uint4 *>(p.c.k + at + 8 * c), v = *reinterpret_cast<const uint4 *>(p.c.v + at + 8 * c);
            const uint32_t w[8] = {k.x, k.y, k.z, k.w, v.x, v.y, v.z, v.w};
#pragma unroll
            for (int e = 0; e < 8; ++e) odd |= (w[e] & kExp) == kExp || (w[e] >> 16 & kExp) == kExp;
        }
    }
    return __any_sync(0xffffffffu, odd);
}

// One row by the definition, by a warp, key by key: what the kernels fall back to for a row
// whose sum came out infinite or NaN and which hides a key that is.  They multiply hidden keys'
// values by weights of 0, which an infinite or NaN value survives; here a hidden key is not
// touched.  Where the keys that it hides are finite, the row is what those that it sees make it,
// and stays.  (Slow, and meant to be: finite caches never come here.)
template <int D, bool BF16, bool Q4>
__device__ __noinline__ void exact_row(const AttnParams &p, int b, int pos, int len, int prefix, int token, int head, int lane)
{
    constexpr int kPer = D / 64;  // 32-bit words a lane holds of a row
    float2 q[kPer], o[kPer];
#pragma unroll
    for (int e = 0; e < kPer; ++e) {
        q[e] = unpack2<BF16>(*reinterpret_cast<const uint32_t *>(p.q + token * p.q_stride + head * D + 2 * (lane * kPer + e)));
        o[e] = make_float2(0.f, 0.f);
    }
    const int h = p.by_group.div(head), end = pos < 0 ? 0 : min(len, max(pos + 1, prefix));
    const float slope = p.slopes ? __ldg(p.slopes + head) * kLog2e : 0.f;
    float m = -INFINITY, l = 0.f;
#pragma unroll 1
    for (int j = p.window ? max(0, pos - p.window + 1) : 0; j < end; ++j) {
        int row;
        const int i = p.c.page.div(j, row), page = seq_page(p.b, p.c, b, i, p.status);
        const int64_t at = Q4 ? 0 : page * p.c.page_stride + ((int64_t)h * p.c.page_size + row) * D;
        float x = 0.f;
        float2 v[kPer];
#pragma unroll
        for (int e = 0; e < kPer; ++e) {
            float2 k;
            if constexpr (Q4) {
                k = page < 0 ? make_float2(0.f, 0.f) : kv4_pair<D>(p.c, p.c.k, page, h, row, lane * kPer + e);
                v[e] = page < 0 ? make_float2(0.f, 0.f) : kv4_pair<D>(p.c, p.c.v, page, h, row, lane * kPer + e);
            } else {
                const int64_t w = at + 2 * (lane * kPer + e);
                k = unpack2<BF16>(page < 0 ? 0u : *reinterpret_cast<const uint32_t *>(p.c.k + w));
                v[e] = unpack2<BF16>(page < 0 ? 0u : *reinterpret_cast<const uint32_t *>(p.c.v + w));
            }
            x = fmaf(q[e].x, k.x, fmaf(q[e].y, k.y, x));
        }
#pragma unroll
        for (int d = 16; d >= 1; d >>= 1) x += __shfl_xor_sync(0xffffffffu, x, d);
        x *= p.scale;
        if (p.cap > 0.f) x = capped(x, p.cap);
        x = fmaf(slope, (float)(j - pos), x);
        const float top = fmaxf(m, x), keep = top == m ? 1.f : ex2(m - top), pr = x == -INFINITY ? 0.f : ex2(x - top);
        m = top;
        l = fmaf(l, keep, pr);
#pragma unroll
        for (int e = 0; e < kPer; ++e) o[e] = make_float2(fmaf(o[e].x, keep, pr * v[e].x), fmaf(o[e].y, keep, pr * v[e].y));
    }
    const float inv = 1.f / l;
#pragma unroll
    for (int e = 0; e < kPer; ++e)
        *reinterpret_cast<uint32_t *>(p.out + token * p.out_stride + head * D + 2 * (lane * kPer + e)) =
            l == 0.f ? 0u : pack2<BF16>(o[e].x * inv, o[e].y * inv);
    if (p.lse && lane == 0) p.lse[(int64_t)token * p.q_heads + head] = l == 0.f ? -INFINITY : (m + log2f(l)) * kLn2;
}

}  // namespace mc
