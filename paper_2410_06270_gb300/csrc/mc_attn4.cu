// mc_attn4.cu -- attention over the 4-bit cache, a warp per token and head.
#include "mc_attn_row.cuh"
#include "mc_host.h"
#include "mc_profile.h"

namespace mc {

template <int D, bool BF16>
__global__ void __launch_bounds__(128) rows4_kernel(const AttnParams p)
{
    pdl_trigger();
    pdl_wait();
    const int lane = threadIdx.x & 31, t = blockIdx.x, head = blockIdx.y * 4 + (threadIdx.x >> 5);
    if (head >= p.q_heads) return;
    const int b = token_seq(p.b, t, lane);
    if (b < 0) return;
    int first;
    const int n = seq_rows(p.b, b, first, p.status), len = seq_len(p.b, p.c, b, p.status);
    if (t < first || t >= first + n) return;
    exact_row<D, BF16, true>(p, b, len - n + (t - first), len, p.prefix ? p.prefix[b] : 0, t, head, lane);
}

int launch_rows4(const AttnParams &p, int head_dim, bool bf16, cudaStream_t st)
{
    auto k = head_dim == 64 ? (bf16 ? rows4_kernel<64, true> : rows4_kernel<64, false>)
                            : (bf16 ? rows4_kernel<128, true> : rows4_kernel<128, false>);
    profile_begin(kKAttnDecode, st);
    const cudaError_t e = launch_k(k, dim3(p.b.tokens, (p.q_heads + 3) / 4), dim3(128), 0, st, p);
    profile_end(kKAttnDecode, st);
    if (e != cudaSuccess) return set_error(MC_ERR_CUDA, "attention launch: %s", cudaGetErrorString(e));
    return MC_OK;
}

}  // namespace mc
