// mc_attn.h -- what the paged-attention kernels share: their parameter blocks and the
// device reading of a batch (lengths, positions, pages), checked against its bounds.
#pragma once
#include <atomic>

#include "mc_kernels.h"

namespace mc {

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;
constexpr float kTanhOne = 8.5f;  // from here on tanh is 1
constexpr int kMaxLen = 1 << 30;  // keys of a sequence, so that positions and windows stay in 32 bits

// Division of 0 .. 2^31 - 1 by a number fixed for the call: the high product is the quotient
// or one less.
struct FastDiv {
    uint32_t d, m;
    FastDiv() = default;
    explicit FastDiv(uint32_t by) : d(by), m(by == 1 ? 0xffffffffu : (uint32_t)(((uint64_t)1 << 32) / by)) {}
#ifdef __CUDACC__
    __device__ __forceinline__ int div(int n, int &rest) const
    {
        uint32_t q = __umulhi((uint32_t)n, m), r = (uint32_t)n - q * d;
        if (r >= d) {
            ++q;
            r -= d;
        }
        rest = (int)r;
        return (int)q;
    }
    __device__ __forceinline__ int div(int n) const
    {
        int r;
        return div(n, r);
    }
#endif
};

struct KvView {
    uint16_t *k, *v;
    int64_t page_stride;
    int num_pages, page_size, kv_heads;
    FastDiv page;  // by page_size
};

struct BatchView {
    const int32_t *lens, *table, *cu_q;
    int seqs, tokens, table_width;
};

struct AttnParams {
    KvView c;
    BatchView b;
    const uint16_t *q;
    int64_t q_stride;
    int q_heads, group;  // group = q_heads / kv_heads
    FastDiv by_group;
    float scale;         // q . k in units of log 2; with a cap: of the cap
    float cap;           // the cap in units of log 2; 0: none
    int window;          // 0: none
    const float *slopes;
    const int32_t *prefix;
    uint16_t *out;
    int64_t out_stride;
    float *lse;
    int32_t *status;
    uint8_t *part;       // partial results of split items
};

struct AppendParams {
    KvView c;
    BatchView b;
    const uint16_t *q, *k, *v;
    int64_t q_stride, k_stride, v_stride;
    int q_heads;
    const uint16_t *q_norm, *k_norm;
    float eps;
    const float *rope;
    int rope_rows, rot, interleaved;
    FastDiv per_token;  // warps of a token
    uint16_t *q_out;
    int32_t *status;
};

// Keys that a row of the page table has pages for.
__device__ __forceinline__ int seq_room(const BatchView &bv, const KvView &c)
{
    const int64_t room = (int64_t)bv.table_width * c.page_size;
    return (int)(room < kMaxLen ? room : kMaxLen);
}

// Length of sequence b, cut to what its table row can hold.
__device__ __forceinline__ int seq_len(const BatchView &bv, const KvView &c, int b, int32_t *status)
{
    const int len = __ldg(bv.lens + b), room = seq_room(bv, c);
    if (len > room) {
        set_status(status, MC_ERR_RANGE);
        return room;
    }
    return len < 0 ? 0 : len;
}

// a / b and a * c / d (rounded down) for b, c, d > 0, in 32 bits where they fit: a 64-bit
// division is a few hundred cycles at the start of every CTA.
__device__ __forceinline__ int64_t div64(int64_t a, int64_t b)
{
    return ((a | b) >> 32) == 0 ? (int64_t)((uint32_t)a / (uint32_t)b) : a / b;
}
__device__ __forceinline__ int64_t muldiv64(int64_t a, int c, int d)  // c <= d < 2^15
{
    const int64_t q = div64(a, d);
    return q * c + (uint32_t)((uint32_t)(a - q * d) * (uint32_t)c) / (uint32_t)d;
}

// New tokens of sequence b: their first row and count (0 where cu_q is not sound).
__device__ __forceinline__ int seq_rows(const BatchView &bv, int b, int &first, int32_t *status)
{
    if (!bv.cu_q) {
        first = b;
        return 1;
    }
    const int lo = __ldg(bv.cu_q + b), hi = __ldg(bv.cu_q + b + 1);
    first = lo;
    if (lo < 0 || hi < lo || hi > bv.tokens) {
        set_status(status, MC_ERR_RANGE);
        first = 0;
        return 0;
    }
    return hi - lo;
}

// Page that holds the rows [i * page_size, ...) of sequence b, or -1.
__device__ __forceinline__ int seq_page(const BatchView &bv, const KvView &c, int b, int i, int32_t *status)
{
    const int page = __ldg(bv.table + (int64_t)b * bv.table_width + i);
    if ((unsigned)page >= (unsigned)c.num_pages) {
        set_status(status, MC_ERR_RANGE);
        return -1;
    }
    return page;
}

// A token's sequence, position and length, found by the whole warp.
struct TokenPlace {
    int seq, pos;  // seq < 0: padding; pos < 0: no position
};

// Sequence of token row t: the largest b with cu_q[b] <= t, found by the whole warp (32
// probes a round); -1 for a padding row.  Ends for any contents of cu_q.
__device__ __forceinline__ int token_seq(const BatchView &bv, int t, int lane)
{
    if (!bv.cu_q) return t;
    int lo = 0, hi = bv.seqs;
    if (t >= __ldg(bv.cu_q + hi)) return -1;
    while (hi - lo > 1) {
        const int step = (hi - lo - 1 + 31) / 32;
        const int i = lo + (lane + 1) * step;
        const int n = __popc(__ballot_sync(0xffffffffu, i < hi && __ldg(bv.cu_q + i) <= t));
        const int top = lo + (n + 1) * step;
        lo += n * step;
        hi = top < hi ? top : hi;
    }
    return lo;
}

// Where token row t is.  Up to 31 sequences every lane reads one boundary and one length, so
// that all comes with one memory round trip; more are searched.  Positions follow from lengths
// that are not cut: a token that its table row has no page for has no position, and the ones
// before it keep theirs.
__device__ __forceinline__ int placed(const BatchView &bv, const KvView &c, int pos, int32_t *status)
{
    if (pos < seq_room(bv, c)) return pos;
    set_status(status, MC_ERR_RANGE);
    return -1;
}
__device__ __forceinline__ TokenPlace token_place(const BatchView &bv, const KvView &c, int t, int lane, int32_t *status)
{
    if (bv.cu_q && bv.seqs < 32) {
        const int cu = lane <= bv.seqs ? __ldg(bv.cu_q + lane) : 0x7fffffff;
        const int mine = lane < bv.seqs ? max(0, __ldg(bv.lens + lane)) : 0;
        const int s = __popc(__ballot_sync(0xffffffffu, lane > 0 && lane <= bv.seqs && cu <= t));
        const int first = __shfl_sync(0xffffffffu, cu, s), end = __shfl_sync(0xffffffffu, cu, s + 1 < 32 ? s + 1 : 31);
        const int len = __shfl_sync(0xffffffffu, mine, s);
        if (s >= bv.seqs) return {-1, -1};
        if (first < 0 || first > t || end <= t || end > bv.tokens) {
            set_status(status, MC_ERR_RANGE);
            return {s, -1};
        }
        return {s, placed(bv, c, len - (end - first) + (t - first), status)};
    }
    const int s = token_seq(bv, t, lane);
    if (s < 0) return {-1, -1};
    int first;
    const int n = seq_rows(bv, s, first, status), len = max(0, __ldg(bv.lens + s));
    return {s, t >= first && t - first < n ? placed(bv, c, len - n + (t - first), status) : -1};
}

template <bool BF16>
__device__ __forceinline__ float2 unpack2(uint32_t w)
{
    if (BF16) return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u));
    return __half22float2(*reinterpret_cast<const __half2 *>(&w));
}

template <bool BF16>
__device__ __forceinline__ uint32_t pack2(float lo, float hi)
{
    uint32_t r;
    if (BF16) asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    else asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}

__device__ __forceinline__ uint64_t pair2(float lo, float hi)
{
    uint64_t r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(lo), "f"(hi));
    return r;
}

__device__ __forceinline__ void unpair2(uint64_t v, float &lo, float &hi)
{
    asm("mov.b64 {%0, %1}, %2;" : "=f"(lo), "=f"(hi) : "l"(v));
}

// Two fp32 operations for one issue slot (the pipe takes as long as for two: what is saved
// is issue: one by one, the prefill softmax of 128 keys takes 1610 cycles instead of 1340).
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c)
{
    uint64_t r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
    return r;
}

__device__ __forceinline__ uint64_t mul2(uint64_t a, uint64_t b)
{
    uint64_t r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}

__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b)
{
    uint64_t r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}

__device__ __forceinline__ float ex2(float x)
{
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}

__device__ __forceinline__ float rcp(float x)
{
    float r;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}

// y within [-kTanhOne, kTanhOne]; NaN stays.
__device__ __forceinline__ float clamped(float y)
{
    float r;
    asm("{\n\t.reg .f32 t;\n\tmin.NaN.f32 t, %1, %2;\n\tmax.NaN.f32 %0, t, %3;\n\t}" : "=f"(r) : "f"(y), "f"(kTanhOne), "f"(-kTanhOne));
    return r;
}

// top * tanh(y), as top * y P(y^2) / Q(y^2) with polynomials of degree 4 that start at 1 (a fit of
// tanh(y) / y on Chebyshev nodes over |y| <= 8.5, its relative error evened out by reweighting:
// 1.3e-8; beyond, tanh is 1 to fp32), for two scores with one reciprocal, that of the denominators'
// product (at most 1.6e5).  In fp32 off by 4.3e-7 of the result at most and 9e-8 in the mean, however
// large the cap: formed from 2^x, as 1 - 2 / (1 + 2^x), it is off by 2^-23 of the cap, a score of 1.5
// under a cap of 10^6 by 0.2.  (tanh.approx, at 2^-11, would move a score of 20 by 0.01.)
// A NaN in either makes both NaN.
__device__ __forceinline__ uint64_t capped2(uint64_t y2, float top)
{
    constexpr float P[4] = {0.134158394f, 3.53705402e-3f, 2.12989525e-5f, 1.43323659e-8f};
    constexpr float Q[4] = {0.467491656f, 2.60343995e-2f, 3.35373107e-4f, 8.17163198e-7f};
    float a, b;
    unpair2(y2, a, b);
    const uint64_t y = pair2(clamped(a), clamped(b)), u = mul2(y, y), one = pair2(1.f, 1.f);
    uint64_t n = pair2(P[3], P[3]), d = pair2(Q[3], Q[3]);
#pragma unroll
    for (int i = 2; i >= 0; --i) {
        n = fma2(n, u, pair2(P[i], P[i]));
        d = fma2(d, u, pair2(Q[i], Q[i]));
    }
    n = mul2(fma2(n, u, one), y);
    d = fma2(d, u, one);
    unpair2(d, a, b);
    const float r = top * rcp(a * b);
    return mul2(n, mul2(pair2(b, a), pair2(r, r)));
}
// The same for |y| <= 3/4, as top * y R(y^2) with a polynomial of degree 5 (fitted the same way, 3.3e-8;
// in fp32 1.3e-7 at most).
constexpr float kTanhNear = 0.75f;
__device__ __forceinline__ uint64_t capped2_near(uint64_t y, float top)
{
    constexpr float R[5] = {-0.333330684f, 0.133265212f, -5.33902597e-2f, 1.96649155e-2f, -4.76949155e-3f};
    const uint64_t u = mul2(y, y);
    uint64_t r = pair2(R[4], R[4]);
#pragma unroll
    for (int i = 3; i >= 0; --i) r = fma2(r, u, pair2(R[i], R[i]));
    return mul2(mul2(fma2(r, u, pair2(1.f, 1.f)), y), pair2(top, top));
}
__device__ __forceinline__ float capped(float y, float top)
{
    float a, b;
    unpair2(capped2(pair2(y, y), top), a, b);
    return a;
}

// Weights are 2^(x - m).  When a score passes m by more than kLazy, m moves to kBelow under the row's
// maximum, so that a row's largest weight lies in 2^7 .. 2^15, inside fp16: a weight keeps its 11 bits
// down to 2^-21 of the largest one, and 2^-32 of it is what rounds to zero.  (With the largest at 1,
// 8192 keys 17 below one other counted 41 % too much: their weights, 4e-8, are subnormal.)
constexpr float kBelow = 7.f, kLazy = 15.f;

int launch_append(AppendParams p, int head_dim, bool bf16, cudaStream_t st);

// Whether a key or value in the rows [from, to) of head h of sequence b is infinite or NaN.
// `warps` warps look, 16 rows at a time each, this one as number `warp`; the answer is the warp's.
template <int D, bool BF16>
__device__ __noinline__ bool odd_keys(const AttnParams &p, int b, int h, int from, int to, int warp, int warps, int lane)
{
    constexpr uint32_t kExp = BF16 ? 0x7f80u : 0x7c00u;  // infinities and NaN have the exponent's bits all set
    bool odd = false;
    for (int j = (from & ~15) + 16 * warp; j < to; j += 16 * warps) {
        int row;
        const int i = p.c.page.div(j, row), page = seq_page(p.b, p.c, b, i, nullptr);
        if (page < 0) continue;
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
template <int D, bool BF16>
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
        const int64_t at = page * p.c.page_stride + ((int64_t)h * p.c.page_size + row) * D;
        float x = 0.f;
        float2 v[kPer];
#pragma unroll
        for (int e = 0; e < kPer; ++e) {
            const int64_t w = at + 2 * (lane * kPer + e);
            const float2 k = unpack2<BF16>(page < 0 ? 0u : *reinterpret_cast<const uint32_t *>(p.c.k + w));
            v[e] = unpack2<BF16>(page < 0 ? 0u : *reinterpret_cast<const uint32_t *>(p.c.v + w));
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

constexpr int kAttnMaxSms = 160;  // SMs that the workspace has room for (the GB300's 152)
// SMs of the current device, asked for once per device.
cudaError_t sm_count(int *out);
// A kernel's shared-memory size, set once on each device.
struct SmemAttr {
    std::atomic<uint64_t> done{0};
    cudaError_t set(const void *kernel, int bytes)
    {
        int dev = 0;
        cudaError_t e = cudaGetDevice(&dev);
        if (e != cudaSuccess) return e;
        const uint64_t bit = dev < 64 ? (uint64_t)1 << dev : 0;
        if (bit & done.load(std::memory_order_relaxed)) return cudaSuccess;
        e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
        if (e == cudaSuccess) done.fetch_or(bit, std::memory_order_relaxed);
        return e;
    }
};
size_t decode_part_bytes(int head_dim);
int launch_decode(const AttnParams &p, int head_dim, bool bf16, int rows, cudaStream_t st);
size_t prefill_part_bytes(int head_dim);
int launch_prefill(const AttnParams &p, int head_dim, bool bf16, cudaStream_t st);

}  // namespace mc
