// mc_attn.h -- what the paged-attention kernels share: their parameter blocks and the
// device reading of a batch (lengths, positions, pages), checked against its bounds.
#pragma once
#include "mc_kernels.h"

namespace mc {

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;
constexpr int kMaxLen = 1 << 30;  // keys of a sequence, so that positions and windows stay in 32 bits

struct KvView {
    uint16_t *k, *v;
    int64_t page_stride;
    int num_pages, page_size, kv_heads;
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
    float scale;         // of q . k; with a cap: of tanh's argument (scale / softcap)
    float softcap;       // 0: none
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
    uint16_t *q_out;
    int32_t *status;
};

// Length of sequence b, cut to what its table row can hold.
__device__ __forceinline__ int seq_len(const BatchView &bv, const KvView &c, int b, int32_t *status)
{
    const int len = __ldg(bv.lens + b);
    const int64_t room = (int64_t)bv.table_width * c.page_size, cap = room < kMaxLen ? room : kMaxLen;
    if (len > cap) {
        set_status(status, MC_ERR_RANGE);
        return (int)cap;
    }
    return len < 0 ? 0 : len;
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

__device__ __forceinline__ float ex2(float x)
{
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}

// cap * tanh(x) with x already divided by the cap, as cap - 2 cap / (1 + e^2x): exact to
// a few units of fp32 relative to the cap (tanh.approx, at 2^-11, would move a score of 20
// by 0.01, a probability by 1 %).  e^2x may overflow to infinity: the quotient is then 0.
__device__ __forceinline__ float capped(float x, float cap)
{
    return fmaf(__fdividef(1.f, 1.f + ex2(x * (2.f * kLog2e))), -2.f * cap, cap);
}

int launch_append(const AppendParams &p, int head_dim, bool bf16, cudaStream_t st);
constexpr int kAttnMaxSms = 160;  // SMs that the workspace has room for (the GB300's 152)
// SMs of the current device, asked for once per device.
cudaError_t sm_count(int *out);
size_t decode_part_bytes(int head_dim, int group);
int launch_decode(const AttnParams &p, int head_dim, bool bf16, cudaStream_t st);
size_t prefill_part_bytes(int head_dim);
int launch_prefill(const AttnParams &p, int head_dim, bool bf16, cudaStream_t st);

}  // namespace mc
