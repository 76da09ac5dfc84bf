// coded_run.cuh -- launches of the attention core over a cache in 8 bits for one type
// of queries (included by one source file per type, so that they compile side by side).
#pragma once

#include "coded_core.cuh"
#include "flash_run.cuh"

namespace rs {

template <int D, bool BF16>
rs_status coded_launch_d(const FlashArgs &a, const CUtensorMap &tmq, const CUtensorMap &tmk, const CUtensorMap &tmv,
                         const char *what, cudaStream_t st) {
    // per device: 0 not asked, 1 ready, -1 built with too few registers for the
    // warpgroups' split (a raise that cannot be granted would wait for ever)
    static std::atomic<int> ready[64];
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) {
        set_error("%s: no current device", what);
        return RS_ERR_CUDA;
    }
    if (ready[dev].load() == 0) {
        cudaFuncAttributes fa;
        const cudaError_t e1 = cudaFuncGetAttributes(&fa, coded_core<D, BF16>);
        const cudaError_t e2 = cudaFuncSetAttribute(coded_core<D, BF16>, cudaFuncAttributeMaxDynamicSharedMemorySize, CoSmem<D>::kTotal);
        if (e1 != cudaSuccess || e2 != cudaSuccess) {
            set_error("%s: kernel attributes: %s", what, cudaGetErrorString(e1 != cudaSuccess ? e1 : e2));
            return RS_ERR_CUDA;
        }
        const int need = kCoThreads * 128;
        ready[dev].store(fa.numRegs * kCoThreads >= need ? 1 : -1);
    }
    if (ready[dev].load() != 1) {
        set_error("%s: attention kernel built with too few registers per thread", what);
        return RS_ERR_CUDA;
    }
    launch_pdl(coded_core<D, BF16>, dim3(a.grid), dim3(kCoThreads), CoSmem<D>::kTotal, st, a, tmq, tmk, tmv);
    RS_CHECK_LAUNCH(what);
    launch_full(flash_combine<D, BF16>, dim3(std::max(a.grid - 1, 1), a.comb_blocks), dim3(kFlCombThreads), 0, st, a);
    RS_CHECK_LAUNCH(what);
    launch_pdl(coded_nan<D>, dim3(32), dim3(kNanThreads), 0, st, a);
    RS_CHECK_LAUNCH(what);
    return RS_OK;
}

template <bool BF16>
rs_status flash_launch_coded(const FlashArgs &a, int D, const CUtensorMap &tmq, const CUtensorMap &tmk, const CUtensorMap &tmv,
                             const char *what, cudaStream_t st) {
    return D == 128 ? coded_launch_d<128, BF16>(a, tmq, tmk, tmv, what, st) : coded_launch_d<64, BF16>(a, tmq, tmk, tmv, what, st);
}

}  // namespace rs
