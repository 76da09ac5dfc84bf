// flash.cu -- rs_prompt_attn and rs_paged_attn (and rs_coded_attn's long chunks): the
// plan of the work and the host side of the attention core (flash.cuh).
// Launches: flash_plan (one CTA, and one per request for draft trees) ->
// flash_kernel (a CTA per SM) -> flash_combine; over a cache in 8 bits coded_core
// in the place of flash_kernel, and coded_nan at the end.
#include <cudaTypedefs.h>
#include <math.h>

#include <algorithm>
#include <mutex>

#include "common.cuh"
#include "flash.cuh"
#include "flash_coded.h"
#include "tmap.cuh"

namespace rs {
namespace {

constexpr int kPlanThreads = 1024;

struct Add {
    template <class T>
    __device__ __forceinline__ T operator()(T x, T y) const { return x + y; }
};
struct Max {
    template <class T>
    __device__ __forceinline__ T operator()(T x, T y) const { return x > y ? x : y; }
};
template <class T, class Op>
__device__ __forceinline__ T warp_scan(T x, Op op) {
    const int lane = threadIdx.x & 31;
    for (int o = 1; o < 32; o <<= 1) {
        const T y = __shfl_up_sync(0xffffffffu, x, o);
        if (lane >= o) x = op(x, y);
    }
    return x;
}
// Inclusive prefix over the block, on top of `carry` (kept by every thread).
template <class T, class Op = Add>
__device__ __forceinline__ T block_scan(T v, T &carry, T *s_w, Op op = Op()) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    T x = warp_scan(v, op);
    if (lane == 31) s_w[warp] = x;
    __syncthreads();
    const T w = warp_scan(lane < (int)(blockDim.x >> 5) ? s_w[lane] : T(0), op);
    const T before = __shfl_sync(0xffffffffu, w, warp > 0 ? warp - 1 : 0);
    if (warp > 0) x = op(x, before);
    x = op(x, carry);
    carry = op(carry, __shfl_sync(0xffffffffu, w, 31));
    __syncthreads();
    return x;
}

// A request's rows and keys against the arrays: 0, or the status that rejects it.
// rq: first row, rows to work on, ctx, rows of its own (to be emptied if it is rejected).
__device__ __forceinline__ int check_rows(const FlashArgs &a, int b, int4 &rq) {
    const int n0 = a.off[b], n1 = a.off[b + 1], ctx = a.ctx ? a.ctx[b] : 0;
    rq = make_int4(0, 0, 0, 0);
    if (n0 < 0 || n1 < n0 || n1 > a.T) return RS_ST_BAD_OFFSET;
    rq = make_int4(n0, 0, 0, n1 - n0);
    if (ctx < 0 || (a.page_table && (long long)ctx + (n1 - n0) > ((long long)a.max_pages << a.page_log2))) return RS_ST_BAD_OFFSET;
    if (n1 - n0 > a.max_new || (a.anc && n1 - n0 > RS_MAX_NODES)) return RS_ST_TOO_LARGE;
    rq = make_int4(n0, n1 - n0, ctx, n1 - n0);
    return 0;
}

// A draft tree: its parents and every node's ancestor set.
__device__ void plan_tree(const FlashArgs &a, const int32_t *parents, uint32_t *anc, int b) {
    __shared__ int s_par[RS_MAX_NODES];
    int4 rq;
    int st = check_rows(a, b, rq);
    int late = 0;  // an earlier request starts behind this one
    for (int i = threadIdx.x; i < b; i += blockDim.x) late |= a.off[i] > a.off[b];
    if (__syncthreads_or(late)) {
        st = RS_ST_BAD_OFFSET;
        rq = make_int4(0, 0, 0, 0);
    }
    int bad = 0;
    for (int i = threadIdx.x; i < rq.y; i += blockDim.x) {
        const int pa = parents[rq.x + i];
        s_par[i] = pa;
        bad |= i == 0 ? pa != -1 : (pa < 0 || pa >= i);
    }
    if (__syncthreads_or(bad)) st = RS_ST_BAD_TREE;
    for (int i = threadIdx.x; i < rq.y; i += blockDim.x) {
        uint32_t bits[kAncWords] = {};
        if (st == 0) {
            for (int x = i; x >= 0; x = s_par[x]) {
#pragma unroll
                for (int w = 0; w < kAncWords; ++w) bits[w] |= (x >> 5) == w ? 1u << (x & 31) : 0u;
            }
        }
#pragma unroll
        for (int w = 0; w < kAncWords; ++w) anc[(long long)(rq.x + i) * kAncWords + w] = bits[w];
    }
    if (threadIdx.x == 0) a.status[b] = st;
}

// Block 0: the pairs of row tiles of all requests end to end and the prefix of
// their costs.  Blocks 1 ..: the draft trees.
__global__ void __launch_bounds__(kPlanThreads)
flash_plan(FlashArgs a, const int32_t *parents, uint32_t *anc, double kv_bytes, double l2) {
    pdl_wait_prev();
    pdl_launch_next();
    if (blockIdx.x > 0) {
        plan_tree(a, parents, anc, blockIdx.x - 1);
        return;
    }
    __shared__ int s_pref[kBatchMax + 1];  // pairs before each request
    __shared__ int s_wi[32];
    __shared__ long long s_wl[32];
    const int tid = threadIdx.x;
    int pairs = 0, latest = 0;
    long long tiles = 0, keys = 0;  // about how many key tiles one KV head has; keys of all requests
    for (int base = 0; base < a.B; base += blockDim.x) {
        const int b = base + tid;
        int4 rq = make_int4(0, 0, 0, 0);
        int st = 0, mine = 0;
        if (b < a.B) {
            st = check_rows(a, b, rq);
        }
        // a request that starts before an earlier one is rejected: what is left
        // shares no rows, and its pairs fit the table
        const int start = b < a.B ? a.off[b] : 0;
        if (block_scan(start, latest, s_wi, Max()) > start && b < a.B) {
            st = RS_ST_BAD_OFFSET;
            rq = make_int4(0, 0, 0, 0);
        }
        if (b < a.B) {
            mine = (rq.y + 2 * a.tq - 1) / (2 * a.tq);
        }
        const int end = block_scan(mine, pairs, s_wi);
        if (b < a.B) {
            s_pref[b + 1] = end;
            a.req[b] = rq;
            if (!a.anc) a.status[b] = st;
        }
        long long t = 0;
        if (rq.y > 0) t = (long long)mine * (pair_keys(a, rq.y, rq.z, 0) + (long long)pair_keys(a, rq.y, rq.z, mine - 1)) / (2 * kBN) + 1;
        block_scan(t, tiles, s_wl);
        block_scan((long long)(rq.y > 0 ? rq.y + rq.z : 0), keys, s_wl);
    }
    if (tid == 0) s_pref[0] = 0;
    __syncthreads();
    const int M = pairs;
    const long long per = tiles * a.Hkv / (2 * a.grid);
    const int beta = (int)(per * a.single < a.start ? per * a.single : a.start);
    long long carry = 0;
    for (int base = 0; base < M; base += blockDim.x) {
        const int i = base + tid;
        long long cost = 0;
        if (i < M) {
            int lo = 0, hi = a.B - 1;  // last b with s_pref[b] <= i: a request with rows
            while (lo < hi) {
                const int mid = (lo + hi + 1) >> 1;
                if (s_pref[mid] <= i) lo = mid;
                else hi = mid - 1;
            }
            const int4 rq = a.req[lo];
            const int p = i - s_pref[lo];
            a.ent[i] = make_int4(lo, p, rq.x, rq.y);
            a.ent_ctx[i] = rq.z;
            cost = tile_cost(a, rq.y, p) * pair_tiles(a, rq.y, rq.z, p) + beta;
        }
        const long long end = block_scan(cost, carry, s_wl);
        if (i < M) a.cum[i + 1] = end;
    }
    if (tid == 0) {
        a.cum[0] = 0;
        a.n_pairs[0] = M;
        a.n_pairs[1] = beta;
        // groups of KV heads whose keys and values fill half of L2 each, where all are
        // more than it holds and a share stays long (200 key tiles) for its two more pieces
        int phases = 1;
        const double used = (double)keys * kv_bytes;
        while (phases < a.max_phases && used > 1.5 * l2 && used > 0.5 * l2 * phases && tiles * a.Hkv / (a.grid * 2 * phases) >= 200) phases *= 2;
        a.n_pairs[2] = phases;
        a.n_pairs[3] = 0;
    }
}

int flash_grid() { return std::min(num_sms(), kAttnMaxGrid); }

// tokens of a row tile
int flash_tq(int G) { return kBM / G; }

// groups of KV heads that a call may be worked off in (the workspace holds their
// partial slots): several only where requests have several pairs of row tiles, so
// that keys are read again
int max_phases(int B, int T, int Hkv, int tq) {
    int p = 1;
    while ((long long)T > 2ll * tq * B && p < kFlMaxPhases && 2 * p <= Hkv) p *= 2;
    return p;
}

struct Work {
    FlashArgs a;
    uint32_t *anc;
    size_t bytes;
};
// trees: rows may be draft trees' (their ancestor sets)
Work carve(void *base, int B, int T, int Hq, int Hkv, int D, bool trees) {
    Work w{};
    const int tq = flash_tq(Hq / Hkv);
    const size_t grid = (size_t)flash_grid(), F = (size_t)max_phases(B, T, Hkv, tq);
    FlashArgs &a = w.a;
    const size_t pairs = (size_t)(T / (2 * tq) + B);  // disjoint requests have no more
    Carve cv(base);
    a.req = cv.take<int4>((size_t)B);
    a.cum = cv.take<long long>(pairs + 1);
    a.ent = cv.take<int4>(pairs);
    a.ent_ctx = cv.take<int>(pairs);
    a.n_pairs = cv.take<int>(4);
    a.bound = cv.take<int4>(F * (grid + 1));
    if (trees) w.anc = cv.take<uint32_t>((size_t)T * kAncWords);
    a.part_m = cv.take<float>(2 * grid * F * kFlRows);
    a.part_l = cv.take<float>(2 * grid * F * kFlRows);
    a.part_o = cv.take<float>(2 * grid * F * kFlRows * (size_t)D);
    w.bytes = cv.used();
    return w;
}

bool sizes_ok(int B, int T, int Hq, int Hkv, int D) {
    return B >= 0 && T >= 0 && Hkv >= 1 && Hq >= 1 && Hq % Hkv == 0 && Hq / Hkv <= kBM && (D == 64 || D == 128) && B <= kBatchMax;
}

size_t workspace_size(int B, int T, int Hq, int Hkv, int D, bool trees) {
    return sizes_ok(B, T, Hq, Hkv, D) ? carve(nullptr, B, T, Hq, Hkv, D, trees).bytes : 0;
}

// The launches of the calls.  a: everything but what comes out of the sizes (coded: of
// the cache in 8 bits, k and v its codes).
rs_status flash_run(const char *what, Work &w, int dtype, int D, const void *q, int64_t q_stride, const void *k,
                    int64_t k_stride, const void *v, int64_t v_stride, long long kv_rows, const int32_t *parents,
                    bool coded, cudaStream_t st) {
    FlashArgs &a = w.a;
    const int type = dtype == RS_BF16;
    a.G = a.Hq / a.Hkv;
    a.tq = flash_tq(a.G);
    a.grid = flash_grid();
    a.anc = parents ? w.anc : nullptr;
    a.single = fl_single(D);
    a.start = fl_start(D);
    a.wait_limit = wait_limit();
    const double token = (coded ? 2.0 : 4.0) * a.Hkv * D;  // bytes
    const double bytes = token * (double)kv_rows;
    a.kv_stream = bytes > 0.5 * (double)l2_bytes();
    a.max_phases = bytes > 1.5 * (double)l2_bytes() ? max_phases(a.B, a.T, a.Hkv, a.tq) : 1;
    // rows of a segment, by the average request, and how many of them a block of eight warps joins
    const int rows = std::min((a.T + a.B - 1) / a.B, 2 * a.tq) * a.G, each = 8 * ((long long)a.T * a.Hq <= 4096 ? 1 : 4);
    a.comb_blocks = std::max((rows + each - 1) / each, 1);
    const int box = a.page_table ? std::min(1 << a.page_log2, kBN) : kBN;
    CUtensorMap tmq, tmk, tmv;
    if (!rows_map(&tmq, q, type, D, a.Hq, a.T, q_stride, a.G, a.tq) ||
        !(coded ? codes_map(&tmk, k, D, a.Hkv, kv_rows, box, false) : rows_map(&tmk, k, type, D, a.Hkv, kv_rows, k_stride, 1, box)) ||
        !(coded ? codes_map(&tmv, v, D, a.Hkv, kv_rows, box, false) : rows_map(&tmv, v, type, D, a.Hkv, kv_rows, v_stride, 1, box))) {
        set_error("%s: cuTensorMapEncodeTiled failed", what);
        return RS_ERR_CUDA;
    }
    // a thread per request and per pair, as far as a block goes (fewer warps, shorter barriers)
    const int wide = std::max(a.B, a.T / (2 * a.tq) + a.B);
    const int threads = std::min(std::max((wide + 31) / 32 * 32, parents ? RS_MAX_NODES : 32), kPlanThreads);
    launch_pdl(flash_plan, dim3(1 + (parents ? a.B : 0)), dim3(threads), 0, st, a, parents, w.anc, token,
               (double)l2_bytes());
    RS_CHECK_LAUNCH(what);
    if (coded) return type ? flash_launch_coded<true>(a, D, tmq, tmk, tmv, what, st) : flash_launch_coded<false>(a, D, tmq, tmk, tmv, what, st);
    return type ? flash_launch<true>(a, D, tmq, tmk, tmv, what, st) : flash_launch<false>(a, D, tmq, tmk, tmv, what, st);
}

}  // namespace

size_t flash_coded_workspace(int B, int T, int Hq, int Hkv, int D) { return workspace_size(B, T, Hq, Hkv, D, true); }

rs_status flash_coded(const char *what, const FlashCoded &f, const CodedPool &pool, cudaStream_t st) {
    Work w = carve(f.workspace, f.B, f.T, f.Hq, f.Hkv, f.D, true);
    FlashArgs &a = w.a;
    a.off = f.off;
    a.ctx = pool.ctx;
    a.page_table = pool.table;
    a.max_pages = pool.max_pages;
    a.n_pages = pool.n_pages;
    a.page_log2 = pool.page_log2;
    a.coded = pool;
    a.B = f.B;
    a.T = f.T;
    a.max_new = f.max_new;
    a.Hq = f.Hq;
    a.Hkv = f.Hkv;
    a.scale = f.scale;
    a.out = f.out;
    a.lse = f.lse;
    a.status = f.status;
    return flash_run(what, w, f.dtype, f.D, f.T ? f.q : f.workspace, f.q_stride, pool.n_pages ? pool.k : f.workspace, 0,
                     pool.n_pages ? pool.v : f.workspace, 0, (long long)pool.n_pages << pool.page_log2, f.parents, true, st);
}

}  // namespace rs

using namespace rs;

extern "C" size_t rs_prompt_attn_workspace_size(int B, int T, int Hq, int Hkv, int D) {
    return workspace_size(B, T, Hq, Hkv, D, false);
}

extern "C" rs_status rs_prompt_attn(const uint16_t *q, int64_t q_stride, const uint16_t *k, int64_t k_stride,
                                    const uint16_t *v, int64_t v_stride, int dtype, const int32_t *seq_off, int B, int T,
                                    int Hq, int Hkv, int D, float scale, uint16_t *out, float *lse, int32_t *status,
                                    void *workspace, size_t workspace_bytes, void *stream) {
    clear_error();
    const char *what = "rs_prompt_attn";
    rs_status st = check_sizes(what, dtype, B, T, Hq, Hkv, D, scale);
    if (st != RS_OK) return st;
    RS_CHECK_ARG(B == 0 || (seq_off && status), "%s: null request pointer", what);
    RS_CHECK_ARG(T == 0 || (q && k && v && out && lse), "%s: null row pointer", what);
    if ((st = check_stride(what, "q", q, q_stride, Hq, D)) != RS_OK) return st;
    if ((st = check_stride(what, "k", k, k_stride, Hkv, D)) != RS_OK) return st;
    if ((st = check_stride(what, "v", v, v_stride, Hkv, D)) != RS_OK) return st;
    RS_CHECK_ARG((((uintptr_t)out | (uintptr_t)workspace) & 31) == 0, "%s: out and workspace must be 32-byte aligned", what);
    if (B == 0) return RS_OK;
    Work w = carve(workspace, B, T, Hq, Hkv, D, false);
    if (workspace_bytes < w.bytes || !workspace) {
        set_error("%s: workspace %zu bytes < %zu required", what, workspace_bytes, w.bytes);
        return RS_ERR_CAPACITY;
    }
    FlashArgs &a = w.a;
    a.off = seq_off;
    a.B = B;
    a.T = T;
    a.max_new = T;
    a.Hq = Hq;
    a.Hkv = Hkv;
    a.scale = scale;
    a.out = out;
    a.lse = lse;
    a.status = status;
    // no rows: nothing is read, the maps only need some address
    const void *any = workspace;
    return flash_run(what, w, dtype, D, T ? q : any, q_stride, T ? k : any, k_stride, T ? v : any, v_stride, T, nullptr,
                     false, (cudaStream_t)stream);
}

extern "C" size_t rs_paged_attn_workspace_size(int B, int T, int Hq, int Hkv, int D) {
    return workspace_size(B, T, Hq, Hkv, D, true);
}

extern "C" rs_status rs_paged_attn(const uint16_t *q, int64_t q_stride, int dtype, const int32_t *new_off,
                                   const int32_t *parents, int B, int T, int Hq, int Hkv, int D, const uint16_t *k_pages,
                                   const uint16_t *v_pages, int n_pages, int page_size, const int32_t *page_table,
                                   int max_pages, const int32_t *ctx_len, float scale, uint16_t *out, float *lse,
                                   int32_t *status, void *workspace, size_t workspace_bytes, void *stream) {
    clear_error();
    const char *what = "rs_paged_attn";
    rs_status st = check_sizes(what, dtype, B, T, Hq, Hkv, D, scale);
    if (st != RS_OK) return st;
    if ((st = check_pages(what, n_pages, page_size, max_pages)) != RS_OK) return st;
    RS_CHECK_ARG(B == 0 || (new_off && ctx_len && status && (page_table || max_pages == 0)), "%s: null request pointer", what);
    RS_CHECK_ARG(T == 0 || (q && out && lse), "%s: null row pointer", what);
    RS_CHECK_ARG(n_pages == 0 || (k_pages && v_pages), "%s: null page pointer", what);
    if ((st = check_stride(what, "q", q, q_stride, Hq, D)) != RS_OK) return st;
    RS_CHECK_ARG((((uintptr_t)k_pages | (uintptr_t)v_pages) & 15) == 0, "%s: pages must be 16-byte aligned", what);
    RS_CHECK_ARG((((uintptr_t)out | (uintptr_t)workspace) & 31) == 0, "%s: out and workspace must be 32-byte aligned", what);
    if (B == 0) return RS_OK;
    Work w = carve(workspace, B, T, Hq, Hkv, D, true);
    if (workspace_bytes < w.bytes || !workspace) {
        set_error("%s: workspace %zu bytes < %zu required", what, workspace_bytes, w.bytes);
        return RS_ERR_CAPACITY;
    }
    FlashArgs &a = w.a;
    a.off = new_off;
    a.ctx = ctx_len;
    // a cache without pages: no request with rows passes its check
    a.page_table = page_table ? page_table : new_off;
    a.max_pages = n_pages ? max_pages : 0;
    a.n_pages = n_pages;
    a.page_log2 = page_log2(page_size);
    a.B = B;
    a.T = T;
    a.max_new = T;
    a.Hq = Hq;
    a.Hkv = Hkv;
    a.scale = scale;
    a.out = out;
    a.lse = lse;
    a.status = status;
    const void *any = workspace;
    const int64_t row = (int64_t)Hkv * D;
    return flash_run(what, w, dtype, D, T ? q : any, q_stride, n_pages ? k_pages : any, row, n_pages ? v_pages : any, row,
                     (long long)n_pages * page_size, parents, false, (cudaStream_t)stream);
}
