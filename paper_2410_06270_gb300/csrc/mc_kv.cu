// mc_kv.cu -- mc_kv_append: new tokens into the paged key-value cache, with the per-head
// norms and the position rotation on the way.
#include <math.h>

#include "mc_attn.h"
#include "mc_host.h"
#include "mc_profile.h"

namespace mc {

constexpr int kAppendPasses = 4;  // rows a half or quarter warp takes, loads first
constexpr int kAppendThreads = 128;

__device__ __forceinline__ void turned(float &a, float &b, float c, float s)
{
    const float t = a;
    a = t * c - b * s;
    b = b * c + t * s;
}

// A head's row of D elements is shared by D / 8 lanes; a warp's 256 / D rows times
// kAppendPasses are heads of one token (its queries, keys, then values), so the token's
// position, page and rotation are found once for them.  A lane holds two runs of four
// elements, chosen so that both members of every pair that the rotation turns lie in it
// (runs 4i and rot/2 + 4i, or 8i and 8i + 4 for interleaved pairs): no exchange between
// lanes but the norm's sum.
template <int D, bool BF16>
__global__ void __launch_bounds__(kAppendThreads) append_kernel(const AppendParams p)
{
    constexpr int kLanes = D / 8, kRows = 32 / kLanes;
    pdl_trigger();
    pdl_wait();
    const int lane = threadIdx.x & 31, li = lane % kLanes;
    const int heads = p.q_heads + 2 * p.c.kv_heads;
    const int per = (heads + kRows * kAppendPasses - 1) / (kRows * kAppendPasses);  // warps per token
    const int64_t warp = (int64_t)blockIdx.x * (kAppendThreads / 32) + (threadIdx.x >> 5);
    if (warp >= (int64_t)p.b.tokens * per) return;
    const int t = (int)(warp / per), h0 = (int)(warp % per) * kRows * kAppendPasses + lane / kLanes;

    const bool turn = p.interleaved ? 8 * li < p.rot : 4 * li < p.rot / 2;
    const int run = p.interleaved || !turn ? 8 * li : 4 * li;
    int ea = run, eb = run + 4;
    if (!p.interleaved) {
        if (turn) eb = p.rot / 2 + run;
        else ea = p.rot + 8 * (li - p.rot / 8), eb = ea + 4;
    }

    uint2 a[kAppendPasses], b[kAppendPasses];
#pragma unroll
    for (int i = 0; i < kAppendPasses; ++i) {
        const int h = h0 + i * kRows;
        const uint16_t *src = nullptr;
        if (h < p.q_heads) src = p.q + t * p.q_stride + h * D;
        else if (h < p.q_heads + p.c.kv_heads) src = p.k + t * p.k_stride + (h - p.q_heads) * D;
        else if (h < heads) src = p.v + t * p.v_stride + (h - p.q_heads - p.c.kv_heads) * D;
        a[i] = b[i] = make_uint2(0, 0);
        if (src) {
            a[i] = *reinterpret_cast<const uint2 *>(src + ea);
            b[i] = *reinterpret_cast<const uint2 *>(src + eb);
        }
    }

    const TokenPlace place = token_place(p.b, p.c, t, lane, p.status);
    const int s = place.seq;
    if (s < 0) return;  // padding
    int pos = place.pos, row = 0;
    int64_t at = -1;  // the row's element offset in the cache
    float4 cs = make_float4(1.f, 1.f, 1.f, 1.f), sn = make_float4(0.f, 0.f, 0.f, 0.f);
    if (pos >= 0) {
        const int i = p.c.page.div(pos, row);
        const int page = seq_page(p.b, p.c, s, i, p.status);
        if (page >= 0) at = page * p.c.page_stride + (int64_t)row * D;
        if (p.rot) {
            if (pos >= p.rope_rows) {
                set_status(p.status, MC_ERR_RANGE);
                pos = -1;
                at = -1;
            } else if (turn) {
                const float *r = p.rope + (int64_t)pos * p.rot + 4 * li;
                cs = *reinterpret_cast<const float4 *>(r);
                sn = *reinterpret_cast<const float4 *>(r + p.rot / 2);
            }
        }
    }

#pragma unroll
    for (int i = 0; i < kAppendPasses; ++i) {
        const int h = h0 + i * kRows;
        const bool is_q = h < p.q_heads, is_k = !is_q && h < p.q_heads + p.c.kv_heads;
        float x[8];
        *reinterpret_cast<float2 *>(x) = unpack2<BF16>(a[i].x);
        *reinterpret_cast<float2 *>(x + 2) = unpack2<BF16>(a[i].y);
        *reinterpret_cast<float2 *>(x + 4) = unpack2<BF16>(b[i].x);
        *reinterpret_cast<float2 *>(x + 6) = unpack2<BF16>(b[i].y);
        const uint16_t *gain = is_q ? p.q_norm : is_k ? p.k_norm : nullptr;
        // the sum is formed by every lane (a warp may hold rows of both kinds)
        float ss = 0.f;
#pragma unroll
        for (int e = 0; e < 8; ++e) ss = fmaf(x[e], x[e], ss);
#pragma unroll
        for (int m = kLanes / 2; m >= 1; m >>= 1) ss += __shfl_xor_sync(0xffffffffu, ss, m);
        if (gain) {
            const float inv = rsqrtf(ss * (1.f / D) + p.eps);
            const uint2 ga = *reinterpret_cast<const uint2 *>(gain + ea), gb = *reinterpret_cast<const uint2 *>(gain + eb);
            const uint32_t g[4] = {ga.x, ga.y, gb.x, gb.y};
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float2 f = unpack2<BF16>(g[e]);
                x[2 * e] *= inv * f.x;
                x[2 * e + 1] *= inv * f.y;
            }
        }
        if (turn && (is_q || is_k)) {
            const float c4[4] = {cs.x, cs.y, cs.z, cs.w}, s4[4] = {sn.x, sn.y, sn.z, sn.w};
            // (two static forms: indices chosen at run time put x into local memory)
            if (p.interleaved) {
#pragma unroll
                for (int e = 0; e < 4; ++e) turned(x[2 * e], x[2 * e + 1], c4[e], s4[e]);
            } else {
#pragma unroll
                for (int e = 0; e < 4; ++e) turned(x[e], x[e + 4], c4[e], s4[e]);
            }
        }
        if (pos < 0) {
#pragma unroll
            for (int e = 0; e < 8; ++e) x[e] = 0.f;
        }
        uint16_t *dst = nullptr;
        if (is_q) dst = p.q_out + ((int64_t)t * p.q_heads + h) * D;
        else if (h < heads && at >= 0)
            dst = (is_k ? p.c.k : p.c.v) + at + (int64_t)(h - p.q_heads - (is_k ? 0 : p.c.kv_heads)) * p.c.page_size * D;
        if (dst) {
            *reinterpret_cast<uint2 *>(dst + ea) = make_uint2(pack2<BF16>(x[0], x[1]), pack2<BF16>(x[2], x[3]));
            *reinterpret_cast<uint2 *>(dst + eb) = make_uint2(pack2<BF16>(x[4], x[5]), pack2<BF16>(x[6], x[7]));
        }
    }
}

int launch_append(const AppendParams &p, int head_dim, bool bf16, cudaStream_t st)
{
    const int rows = 256 / head_dim * kAppendPasses, heads = p.q_heads + 2 * p.c.kv_heads;
    const int64_t warps = (int64_t)p.b.tokens * ((heads + rows - 1) / rows);
    const int64_t ctas = (warps + kAppendThreads / 32 - 1) / (kAppendThreads / 32);
    if (ctas > 0x7fffffff) return set_error(MC_ERR_UNSUPPORTED, "%d tokens of %d heads in one call", p.b.tokens, heads);
    auto k = head_dim == 64 ? (bf16 ? append_kernel<64, true> : append_kernel<64, false>)
                            : (bf16 ? append_kernel<128, true> : append_kernel<128, false>);
    profile_begin(kKAppend, st);
    cudaError_t e = launch_k(k, dim3((unsigned)ctas), dim3(kAppendThreads), 0, st, p);
    profile_end(kKAppend, st);
    if (e != cudaSuccess) return set_error(MC_ERR_CUDA, "append launch: %s", cudaGetErrorString(e));
    return MC_OK;
}

}  // namespace mc
