// coded_attn.cu -- rs_coded_attn: attention over a cache in 8 bits.  Requests of a
// few rows go to coded_rows (coded_rows.cuh), longer chunks and trees to the
// attention core (flash.cuh).
#include <math.h>

#include <algorithm>
#include <atomic>

#include "coded_rows.cuh"
#include "flash_coded.h"
#include "tmap.cuh"

namespace rs {
namespace {

// Tiles of eight rows that the calls' requests need at most: 1, 2 or 4; 0: more rows
// than coded_rows takes.  The core works on 128 rows a KV head, whatever is in them.
// 64 requests with trees behind 1024 to 8191 keys, 32 / 8 heads of 128, bf16, few rows and core:
// 8 rows 122 and 180 us, 16 rows 163 and 181, 32 rows 618 and 185 (the third tile's registers do not
// fit); heads of 64: 82 and 164, 127 and 166, 212 and 169.  So four tiles are too many where caches are long.
int row_tiles(int max_new, int G) {
    const long long rows = (long long)max_new * G;
    return rows <= 8 ? 1 : rows <= 16 ? 2 : rows <= kRowMax ? 4 : 0;
}
int per_sm(int tiles) { return tiles == 1 ? 3 : 2; }

struct Work {
    RowsArgs a;
    size_t bytes;
};
Work carve(void *base, int B, int Hkv, int D, int tiles) {
    Work w{};
    RowsArgs &a = w.a;
    a.grid = per_sm(tiles) * num_sms();
    a.most_hw = Hkv % 4 == 0 ? 4 : Hkv % 2 == 0 ? 2 : 1;
    Carve cv(base);
    a.req = cv.take<int4>((size_t)B);
    a.cum = cv.take<long long>((size_t)B + 1);
    a.start = cv.take<int4>((size_t)a.grid);
    a.flag = cv.take<unsigned char>((size_t)B * Hkv + a.grid);
    a.part_lse = cv.take<float>(2 * (size_t)a.grid * a.most_hw * 8 * tiles);
    a.part_o = cv.take<float>(2 * (size_t)a.grid * a.most_hw * 8 * tiles * D);
    w.bytes = cv.used();
    return w;
}

bool sizes_ok(int B, int T, int max_new, int Hq, int Hkv, int D) {
    return B >= 0 && T >= 0 && max_new >= 0 && Hkv >= 1 && Hq >= 1 && Hq % Hkv == 0 && Hq / Hkv <= kBM && (D == 64 || D == 128) &&
           B <= kBatchMax && T <= 1 << 30;
}

template <int D, int NT, bool TREE>
rs_status launch_rows(const RowsArgs &a, cudaStream_t st) {
    CUtensorMap tmk, tmv;
    const long long slots = (long long)a.c.n_pages << a.c.page_log2;
    const void *any = a.req;  // no pages: nothing is read
    if (!codes_map(&tmk, slots ? a.c.k : any, D, a.Hkv, slots, kCodeBlock, true) ||
        !codes_map(&tmv, slots ? a.c.v : any, D, a.Hkv, slots, kCodeBlock, true)) {
        set_error("rs_coded_attn: cuTensorMapEncodeTiled failed");
        return RS_ERR_CUDA;
    }
    constexpr int kBytes = RowsShape<D, NT>::kBytes;
    static std::atomic<int> ready[64];
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) {
        set_error("rs_coded_attn: no current device");
        return RS_ERR_CUDA;
    }
    if (!ready[dev].load()) {
        cudaError_t e = cudaFuncSetAttribute(coded_rows<D, NT, TREE>, cudaFuncAttributeMaxDynamicSharedMemorySize, kBytes);
        // the same division of L1 for both kernels: changing it between them takes an SM 1.5 us
        if (e == cudaSuccess) e = cudaFuncSetAttribute(coded_join<D>, cudaFuncAttributePreferredSharedMemoryCarveout, 100);
        if (e != cudaSuccess) {
            set_error("rs_coded_attn: kernel attributes: %s", cudaGetErrorString(e));
            return RS_ERR_CUDA;
        }
        ready[dev].store(1);
    }
    launch_pdl(coded_rows<D, NT, TREE>, dim3(a.grid), dim3(kRowThreads), kBytes, st, a, tmk, tmv);
    RS_CHECK_LAUNCH("rs_coded_attn");
    const int each = std::min((a.most_hw * std::min(a.max_new * a.G, kRowMax) + kRowWarps - 1) / kRowWarps, 8);
    launch_pdl(coded_join<D>, dim3(a.grid, std::max(each, 1)), dim3(kRowThreads), 0, st, a, NT);
    RS_CHECK_LAUNCH("rs_coded_attn");
    return RS_OK;
}
template <int D, bool TREE>
rs_status launch_tiles(const RowsArgs &a, int tiles, cudaStream_t st) {
    return tiles == 1 ? launch_rows<D, 1, TREE>(a, st) : tiles == 2 ? launch_rows<D, 2, TREE>(a, st) : launch_rows<D, 4, TREE>(a, st);
}

}  // namespace
}  // namespace rs

using namespace rs;

extern "C" size_t rs_coded_attn_workspace_size(int B, int T, int max_new, int Hq, int Hkv, int D) {
    if (!sizes_ok(B, T, max_new, Hq, Hkv, D)) return 0;
    const int tiles = row_tiles(max_new, Hq / Hkv);
    return tiles ? carve(nullptr, B, Hkv, D, tiles).bytes : flash_coded_workspace(B, T, Hq, Hkv, D);
}

extern "C" rs_status rs_coded_attn(const uint16_t *q, int64_t q_stride, int dtype, const int32_t *new_off,
                                   const int32_t *parents, int B, int T, int max_new, int Hq, int Hkv, int D,
                                   const uint8_t *k_codes, const uint8_t *v_codes, const int8_t *k_exps, const int8_t *v_exps,
                                   int n_pages, int page_size, const int32_t *page_table, int max_pages, const int32_t *ctx_len,
                                   float scale, uint16_t *out, float *lse, int32_t *status, void *workspace,
                                   size_t workspace_bytes, void *stream) {
    clear_error();
    const char *what = "rs_coded_attn";
    rs_status st = check_sizes(what, dtype, B, T, Hq, Hkv, D, scale);
    if (st != RS_OK) return st;
    RS_CHECK_ARG(max_new >= 0, "%s: max_new=%d is negative", what, max_new);
    if ((long long)B * Hkv > 1 << 20) {
        set_error("%s: %d requests of %d KV heads: above 2^20", what, B, Hkv);
        return RS_ERR_UNSUPPORTED;
    }
    if ((st = check_coded_pages(what, n_pages, page_size, max_pages)) != RS_OK) return st;
    RS_CHECK_ARG(B == 0 || (new_off && ctx_len && status && (page_table || max_pages == 0)), "%s: null request pointer", what);
    RS_CHECK_ARG(T == 0 || (q && out && lse), "%s: null row pointer", what);
    RS_CHECK_ARG(n_pages == 0 || (k_codes && v_codes && k_exps && v_exps), "%s: null page pointer", what);
    if ((st = check_stride(what, "q", q, q_stride, Hq, D)) != RS_OK) return st;
    RS_CHECK_ARG((((uintptr_t)k_codes | (uintptr_t)v_codes) & 15) == 0, "%s: pages must be 16-byte aligned", what);
    RS_CHECK_ARG((((uintptr_t)out | (uintptr_t)workspace) & 31) == 0, "%s: out and workspace must be 32-byte aligned", what);
    if (B == 0) return RS_OK;
    const int G = Hq / Hkv, tiles = row_tiles(max_new, G);
    const size_t need = rs_coded_attn_workspace_size(B, T, max_new, Hq, Hkv, D);
    if (workspace_bytes < need || !workspace) {
        set_error("%s: workspace %zu bytes < %zu required", what, workspace_bytes, need);
        return RS_ERR_CAPACITY;
    }
    // a cache without pages: no request with rows passes its check
    const CodedPool pool{const_cast<uint8_t *>(k_codes), const_cast<uint8_t *>(v_codes), const_cast<int8_t *>(k_exps),
                         const_cast<int8_t *>(v_exps), page_table ? page_table : new_off, ctx_len, n_pages, page_log2(page_size),
                         n_pages ? max_pages : 0};
    if (!tiles) {
        const FlashCoded f{q, q_stride, dtype, new_off, parents, B, T, max_new, Hq, Hkv, D, scale, out, lse, status, workspace};
        return flash_coded(what, f, pool, (cudaStream_t)stream);
    }
    Work w = carve(workspace, B, Hkv, D, tiles);
    RowsArgs &a = w.a;
    a.q = q;
    a.q_stride = q_stride;
    a.off = new_off;
    a.parents = parents;
    a.c = pool;
    a.B = B;
    a.T = T;
    a.max_new = max_new;
    a.Hq = Hq;
    a.Hkv = Hkv;
    a.G = G;
    a.bf16 = dtype == RS_BF16;
    a.scale = scale;
    a.wait_limit = wait_limit();
    a.out = out;
    a.lse = lse;
    a.status = status;
    const cudaStream_t s = (cudaStream_t)stream;
    if (parents) return D == 128 ? launch_tiles<128, true>(a, tiles, s) : launch_tiles<64, true>(a, tiles, s);
    return D == 128 ? launch_tiles<128, false>(a, tiles, s) : launch_tiles<64, false>(a, tiles, s);
}
