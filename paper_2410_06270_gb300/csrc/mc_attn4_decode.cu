// mc_attn4_decode.cu -- attention of few rows per sequence: the kernels over the 4-bit cache.
#include "mc_attn_decode.cuh"

namespace mc {

template cudaError_t launch_decode_d<true>(const AttnParams &, int, bool, int, int, cudaStream_t);

}  // namespace mc
