// tmap.cuh -- host helpers of the attention and cache calls: tensor maps over
// rows of heads, checks of the page arguments, the limit of bounded waits.
#pragma once

#include <cuda.h>
#include <cudaTypedefs.h>
#include <math.h>
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

// Sizes and types that the attention calls share.
constexpr int kBatchMax = 4096;  // requests per call (a prefix over them lives in shared memory)
inline rs_status check_sizes(const char *what, int dtype, int B, int T, int Hq, int Hkv, int D, float scale) {
    RS_CHECK_ARG(B >= 0 && T >= 0, "%s: negative size", what);
    RS_CHECK_ARG(dtype == RS_BF16 || dtype == RS_F16, "%s: dtype %d is neither RS_BF16 nor RS_F16", what, dtype);
    if (D != 64 && D != 128) {
        set_error("%s: head dim %d unsupported (64 or 128)", what, D);
        return RS_ERR_UNSUPPORTED;
    }
    if (Hkv < 1 || Hq < 1 || Hq % Hkv != 0 || Hq / Hkv > kBM) {
        set_error("%s: Hq=%d must be a multiple of Hkv=%d, 1 to %d times", what, Hq, Hkv, kBM);
        return RS_ERR_UNSUPPORTED;
    }
    RS_CHECK_ARG(T <= 1 << 30, "%s: T=%d above 2^30", what, T);
    RS_CHECK_ARG(B <= kBatchMax, "%s: B=%d above %d", what, B, kBatchMax);
    RS_CHECK_ARG(isfinite(scale) && scale > 0.f, "%s: scale must be finite and > 0", what);
    return RS_OK;
}

inline rs_status check_stride(const char *what, const char *name, const void *p, int64_t stride, int heads, int D) {
    RS_CHECK_ARG((reinterpret_cast<uintptr_t>(p) & 15) == 0, "%s: %s must be 16-byte aligned", what, name);
    RS_CHECK_ARG(stride >= (int64_t)heads * D && stride % 8 == 0 && stride < (1ll << 38),
                 "%s: %s rows of %lld elements: at least heads x D, a multiple of 8", what, name, (long long)stride);
    return RS_OK;
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
