// mc_attn_prefill.cu -- attention of many new tokens per sequence: the launch's choices, and the kernels over the
// 16-bit cache.
#include "mc_attn_prefill.cuh"

namespace mc {

extern template cudaError_t launch_prefill_d<true>(const PfParams &, int, bool, int, int, cudaStream_t);

size_t prefill_part_bytes(int head_dim)
{
    return kAttnMaxSms * (sizeof(PfOpen) + sizeof(int32_t) + 2 * 4 * pf_part_floats(head_dim));
}

int launch_prefill(const AttnParams &a, int head_dim, bool bf16, bool q4, cudaStream_t st)
{
    if ((int64_t)a.b.tokens * a.group > 0x7fffffff - kPfRows)
        return set_error(MC_ERR_UNSUPPORTED, "%d tokens of %d heads a group in one call", a.b.tokens, a.group);
    PfParams p;
    p.a = a;
    p.open = reinterpret_cast<PfOpen *>(a.part);
    p.odd = reinterpret_cast<int32_t *>(p.open + kAttnMaxSms);
    p.part = reinterpret_cast<float *>(p.odd + kAttnMaxSms);
    p.timeout_ns = wait_bound_ns();
    p.debug = debug_flags();
    p.q_boxes = kPfTile % a.group == 0 && a.q_stride < (int64_t)1 << 38;
    p.out32 = (uintptr_t)a.out % 32 == 0 && a.out_stride % 16 == 0;
    p.box_rows = q4 ? 1 : std::min(a.c.page_size & -a.c.page_size, kPfKeys);  // (the 4-bit cache's keys come one by one)
    const int mode = a.cap > 0.f ? kPfCap : a.slopes ? kPfBias : kPfPlain;
    int nsm = 0;
    cudaError_t e = sm_count(&nsm);
    if (e == cudaSuccess) {
        const int ctas = nsm < kAttnMaxSms ? nsm : kAttnMaxSms;
        e = q4 ? launch_prefill_d<true>(p, head_dim, bf16, mode, ctas, st) : launch_prefill_d<false>(p, head_dim, bf16, mode, ctas, st);
    }
    if (e != cudaSuccess) return set_error(MC_ERR_CUDA, "prefill launch: %s", cudaGetErrorString(e));
    return MC_OK;
}

}  // namespace mc
