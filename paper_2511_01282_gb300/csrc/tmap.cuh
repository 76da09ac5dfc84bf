// tmap.cuh -- host helpers of the attention and cache calls: tensor maps over
// rows of heads, checks of the page arguments, the limit of bounded waits.
#pragma once

#include <cuda.h>
#include <cudaTypedefs.h>
#include <stdlib.h>

#include <algorithm>
#include <mutex>

#include "attn_core.cuh"
#include "common.cuh"

namespace rs {

inline PFN_cuTensorMapEncodeTiled_v12000 tmap_encode() {
    static std::once_flag once;
    static PFN_cuTensorMapEncodeTiled_v12000 fn = nullptr;
    std::call_once(once, [] {
        void *p = nullptr;
        cudaDriverEntryPointQueryResult q;
        if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &p, 12000, cudaEnableDefault, &q) == cudaSuccess &&
            q == cudaDriverEntryPointSuccess)
            fn = reinterpret_cast<PFN_cuTensorMapEncodeTiled_v12000>(p);
    });
    return fn;
}

// Rows of `heads` heads of D 16-bit values, `stride` values from row to row,
// viewed as (D, heads, rows); boxes of 64 columns x box_heads x box_rows,
// 128-byte swizzled (the K-major layout of the products), zeros past the rows.
inline bool rows_map(CUtensorMap *m, const void *base, bool bf16, int D, int heads, long long rows, int64_t stride,
                     int box_heads, int box_rows) {
    auto fn = tmap_encode();
    if (!fn) return false;
    cuuint64_t dims[3] = {(cuuint64_t)D, (cuuint64_t)heads, (cuuint64_t)std::max(rows, 1ll)};
    cuuint64_t strides[2] = {(cuuint64_t)D * 2, (cuuint64_t)stride * 2};
    cuuint32_t box[3] = {64, (cuuint32_t)box_heads, (cuuint32_t)box_rows};
    cuuint32_t estr[3] = {1, 1, 1};
    return fn(m, bf16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 3, const_cast<void *>(base), dims,
              strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
              CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

inline int page_log2(int page_size) {
    int l = 0;
    while ((1 << l) < page_size) ++l;
    return l;
}

// A page holds a power of two of tokens, 8 at least (one swizzle atom of a TMA
// copy); all slots of the pool are numbered in 31 bits.
inline rs_status check_pages(const char *what, int n_pages, int page_size, int max_pages) {
    RS_CHECK_ARG(n_pages >= 0 && max_pages >= 0, "%s: negative size", what);
    if (page_size < 8 || page_size > 65536 || (page_size & (page_size - 1))) {
        set_error("%s: page size %d unsupported (a power of two, 8 to 65536)", what, page_size);
        return RS_ERR_UNSUPPORTED;
    }
    RS_CHECK_ARG((long long)n_pages * page_size < (1ll << 31) - kBN, "%s: %d pages of %d tokens: 2^31 slots or more", what,
                 n_pages, page_size);
    RS_CHECK_ARG((long long)max_pages * page_size < (1ll << 31) - 65536, "%s: max_pages=%d of %d tokens: 2^31 slots or more",
                 what, max_pages, page_size);
    return RS_OK;
}

// Clock cycles a pipeline wait may take; RS_DEBUG_WAIT_LIMIT (a test hook)
// shortens it so that the time-out path can be exercised.
inline long long wait_limit() {
    if (const char *e = getenv("RS_DEBUG_WAIT_LIMIT")) {
        const long long v = atoll(e);
        if (v > 0) return v;
    }
    return kWaitLimit;
}

}  // namespace rs
