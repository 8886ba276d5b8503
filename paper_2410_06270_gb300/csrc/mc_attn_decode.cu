// mc_attn_decode.cu -- attention of few rows per sequence: the launch, and the kernels over the 16-bit cache.
#include "mc_attn_decode.cuh"

namespace mc {

extern template cudaError_t launch_decode_d<true>(const AttnParams &, int, bool, int, int, cudaStream_t);

size_t decode_part_bytes(int head_dim)
{
    return kDecMaxCtas * sizeof(OpenItem) + 2 * kAttnMaxSms * 2 * 4 * dec_part_floats(head_dim, kDecMaxTiles);
}

// rows: what most sequences have, (token, head of the group) each; the smallest slice that
// holds them is taken, and sequences with more take several.
int launch_decode(const AttnParams &p, int head_dim, bool bf16, bool q4, int rows, cudaStream_t st)
{
    int nsm = 0;
    cudaError_t e = sm_count(&nsm);
    if (e == cudaSuccess) {
        const int sms = nsm < kAttnMaxSms ? nsm : kAttnMaxSms;
        e = q4 ? launch_decode_d<true>(p, head_dim, bf16, rows, sms, st) : launch_decode_d<false>(p, head_dim, bf16, rows, sms, st);
    }
    if (e != cudaSuccess) return set_error(MC_ERR_CUDA, "decode launch: %s", cudaGetErrorString(e));
    return MC_OK;
}

}  // namespace mc
