// coded_core_f16.cu -- the attention core for fp16 queries over a cache in 8 bits.
#include "coded_run.cuh"

template rs_status rs::flash_launch_coded<false>(const FlashArgs &, int, const CUtensorMap &, const CUtensorMap &,
                                                     const CUtensorMap &, const char *, cudaStream_t);
