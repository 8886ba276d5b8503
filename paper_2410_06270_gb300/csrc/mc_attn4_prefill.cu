// mc_attn4_prefill.cu -- attention of many new tokens per sequence: the kernels over the 4-bit cache.
#include "mc_attn_prefill.cuh"

namespace mc {

template cudaError_t launch_prefill_d<true>(const PfParams &, int, bool, int, int, cudaStream_t);

}  // namespace mc
