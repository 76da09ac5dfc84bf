// flash_bf16.cu -- the attention core for bf16 queries, keys and values.
#include "flash_run.cuh"

template rs_status rs::flash_launch<true>(const FlashArgs &, int, const CUtensorMap &, const CUtensorMap &,
                                                const CUtensorMap &, const char *, cudaStream_t);
