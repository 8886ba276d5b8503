// mc_profile.h -- optional per-kernel CUDA-event timing of the library's own
// launches (enabled with mc_profile_enable; off by default, no cost when off).
#pragma once
#include <cuda_runtime.h>

namespace mc {

enum KernelId {
    kKRoute = 0,
    kKPermute,
    kKGemvW13,
    kKGemvW2,
    kKCombine,
    kKFragX,      // decode path: activations -> vector blocks
    kKGemmW13,
    kKGemmW2,
    kKRmsnorm,
    kKImportance,
    kKXImg,       // prefill path: activations -> SW128 images
    kKAppend,     // new tokens into the key-value cache
    kKAttnDecode,
    kKAttnPrefill,
    kKAttnJoin,   // partial results of items split over the cache's length
    kKRead,       // rows of the 4-bit cache in 16 bits
    kKPlan,       // pages and slots of a step
    kKUnpack,     // keys of the 4-bit cache in 16 bits for a call
    kKResidual,   // norms, gate and residual sum between blocks
    kKCount
};

bool profile_on();
// Record an event pair around one launch on `st`; call begin before and end
// after the launch.  No-ops when profiling is off.
void profile_begin(int id, cudaStream_t st);
void profile_end(int id, cudaStream_t st);

}  // namespace mc
