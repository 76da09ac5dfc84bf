// coded_core_bf16.cu -- the attention core for bf16 queries over a cache in 8 bits.
#include "coded_run.cuh"

template rs_status rs::flash_launch_coded<true>(const FlashArgs &, int, const CUtensorMap &, const CUtensorMap &,
                                                     const CUtensorMap &, const char *, cudaStream_t);
