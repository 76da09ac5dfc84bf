// flash_coded.h -- the attention core over a cache in 8 bits, as rs_coded_attn calls it.
#pragma once

#include "coded.cuh"

namespace rs {

struct FlashCoded {
    const uint16_t *q;
    int64_t q_stride;
    int dtype;
    const int32_t *off, *parents;
    int B, T, max_new, Hq, Hkv, D;
    float scale;
    uint16_t *out;
    float *lse;
    int32_t *status;
    void *workspace;  // of flash_coded_workspace bytes
};
size_t flash_coded_workspace(int B, int T, int Hq, int Hkv, int D);
rs_status flash_coded(const char *what, const FlashCoded &f, const CodedPool &pool, cudaStream_t st);

}  // namespace rs
