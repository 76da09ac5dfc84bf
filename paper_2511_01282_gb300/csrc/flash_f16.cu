// flash_f16.cu -- the attention core for fp16 queries, keys and values.
#include "flash_run.cuh"

template rs_status rs::flash_launch<false>(const FlashArgs &, int, const CUtensorMap &, const CUtensorMap &,
                                                const CUtensorMap &, const char *, cudaStream_t);
