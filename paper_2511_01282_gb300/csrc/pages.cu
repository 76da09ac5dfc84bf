// pages.cu -- rs_pages_copy and rs_pages_compact: pages of a cache copied by a
// list of pairs, and a pool's used pages moved below its free ones.
#include "coded.cuh"
#include "tmap.cuh"

namespace rs {
namespace {

// All that a cache keeps about a page: its keys and values, their exponents (8-bit
// caches), and a run of weights and positions for each KV head.
struct Pages {
    char *data[2], *exps[2];
    uint32_t *each[2];            // weights, positions: [Hkv, slots]
    long long data_bytes;         // of a page, a multiple of 16
    long long slots;
    int exp_bytes, Hkv, page_size, n_pages, units;
};

// A block copies a page in units: 16 KB of keys or values, all loads of a thread
// under way before its first store, and one unit for the small arrays.
// Bound: 2 bytes moved a byte: 2500 pages of 133 KB, 666 MB, in 99 us, 6.7 TB/s (with 64
// blocks an SM, which take a few units each; 8 that take many 106 us, a unit of 32 KB 104).
constexpr int kCopyThreads = 256, kCopyWords = 4;  // 16-byte words of a thread
constexpr int kCopyUnit = kCopyThreads * kCopyWords * 16;

__host__ __device__ inline int data_units(const Pages &p) { return (int)((p.data_bytes + kCopyUnit - 1) / kCopyUnit); }

__device__ __forceinline__ void copy_unit(const Pages &p, int from, int to, int unit) {
    const int per = data_units(p);
    if (unit < 2 * per) {
        char *base = unit >= per ? p.data[1] : p.data[0];
        const long long at = (long long)(unit >= per ? unit - per : unit) * (kCopyUnit / 16), words = p.data_bytes / 16;
        const uint4 *src = reinterpret_cast<const uint4 *>(base + from * p.data_bytes) + at;
        uint4 *dst = reinterpret_cast<uint4 *>(base + to * p.data_bytes) + at;
        uint4 x[kCopyWords];
#pragma unroll
        for (int u = 0; u < kCopyWords; ++u)
            if (at + u * kCopyThreads + threadIdx.x < words) x[u] = src[u * kCopyThreads + threadIdx.x];
#pragma unroll
        for (int u = 0; u < kCopyWords; ++u)
            if (at + u * kCopyThreads + threadIdx.x < words) dst[u * kCopyThreads + threadIdx.x] = x[u];
        return;
    }
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        if (p.exps[i]) {
            const char *src = p.exps[i] + (long long)from * p.exp_bytes;
            char *dst = p.exps[i] + (long long)to * p.exp_bytes;
            for (int j = threadIdx.x; j < p.exp_bytes; j += kCopyThreads) dst[j] = src[j];
        }
        if (p.each[i])
            for (int j = threadIdx.x; j < p.Hkv * p.page_size; j += kCopyThreads) {
                const int h = j / p.page_size, s = j - h * p.page_size;
                uint32_t *row = p.each[i] + h * p.slots + s;
                row[(long long)to * p.page_size] = row[(long long)from * p.page_size];
            }
    }
}

__device__ __forceinline__ bool in_pool(const Pages &p, int id) { return id >= 0 && id < p.n_pages; }

// pairs [n, 2]: from, to.  Block 0 also looks all of them over for the status.
__global__ void __launch_bounds__(kCopyThreads)
pages_copy(Pages p, const int2 *pairs, int n, int32_t *status) {
    pdl_enter();
    if (blockIdx.x == 0) {
        int bad = 0;
        for (int i = threadIdx.x; i < n; i += kCopyThreads) bad |= !in_pool(p, pairs[i].x) || !in_pool(p, pairs[i].y);
        bad = __syncthreads_or(bad);
        if (threadIdx.x == 0) *status = bad ? RS_ST_BAD_PAGE : 0;
    }
    const long long total = (long long)n * p.units;
    for (long long w = blockIdx.x; w < total; w += gridDim.x) {
        const int i = (int)(w / p.units);
        const int2 pr = pairs[i];
        if (pr.x == pr.y || !in_pool(p, pr.x) || !in_pool(p, pr.y)) continue;
        copy_unit(p, pr.x, pr.y, (int)(w - (long long)i * p.units));
    }
}

// Used pages (refs > 0): U of them.  The r-th used page at U or above moves to the
// r-th free one below U.  One block; a warp takes runs of 512 pages, whose counts and
// places within the run are votes' bits.
// Bound: latency, of two passes over the counts and one over the moves: 16384 pages
// 10 us (25 with 16 pages in a row to a thread, whose loads and stores are 32 lines each).
constexpr int kPlanThreads = 1024, kPlanEach = 16, kPlanRound = kPlanThreads * kPlanEach;
static_assert(kPlanRound < 1 << 16, "two counts in a word");
__global__ void __launch_bounds__(kPlanThreads)
compact_plan(int n, int32_t *refs, int32_t *new_id, int32_t *n_moves, int2 *moves) {
    pdl_enter();
    __shared__ int s_w[kPlanThreads / 32];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const unsigned below = (1u << lane) - 1u;
    auto first_of = [&](int base) { return base + warp * (32 * kPlanEach) + lane; };  // this lane's pages: every 32nd from there
    auto load = [&](int at, int (&r)[kPlanEach]) {
#pragma unroll
        for (int i = 0; i < kPlanEach; ++i) r[i] = at + 32 * i < n ? refs[at + 32 * i] : 0;
    };
    // v of every warp: the sum of the earlier ones', and of all
    auto prefix = [&](int v, int &sum) {
        if (lane == 0) s_w[warp] = v;
        __syncthreads();
        int x = s_w[lane];
        for (int o = 1; o < 32; o <<= 1) {
            const int y = __shfl_up_sync(0xffffffffu, x, o);
            if (lane >= o) x += y;
        }
        sum = __shfl_sync(0xffffffffu, x, 31);
        const int incl = __shfl_sync(0xffffffffu, x, warp);
        __syncthreads();
        return incl - v;
    };
    int U = 0;
    for (int base = 0; base < n; base += kPlanRound) {
        int r[kPlanEach];
        load(first_of(base), r);
#pragma unroll
        for (int i = 0; i < kPlanEach; ++i) U += __popc(__ballot_sync(0xffffffffu, r[i] > 0));
    }
    const int mine = U;
    prefix(mine, U);
    int holes = 0, above = 0;  // free pages below U, used ones from U on
    for (int base = 0; base < n; base += kPlanRound) {
        const int at = first_of(base);
        int r[kPlanEach], counts = 0, sum;
        unsigned hole[kPlanEach], high[kPlanEach];
        load(at, r);
#pragma unroll
        for (int i = 0; i < kPlanEach; ++i) {
            hole[i] = __ballot_sync(0xffffffffu, at + 32 * i < U && r[i] <= 0);  // (U <= n)
            high[i] = __ballot_sync(0xffffffffu, at + 32 * i >= U && r[i] > 0);
            counts += __popc(hole[i]) | __popc(high[i]) << 16;
        }
        const int before = prefix(counts, sum);
        int ph = holes + (before & 0xffff), pu = above + (before >> 16);
        holes += sum & 0xffff;
        above += sum >> 16;
#pragma unroll
        for (int i = 0; i < kPlanEach; ++i) {
            const int id = at + 32 * i;
            if (id < n) new_id[id] = r[i] > 0 ? id : -1;
            if (hole[i] >> lane & 1u) moves[ph + __popc(hole[i] & below)].y = id;
            if (high[i] >> lane & 1u) moves[pu + __popc(high[i] & below)].x = id;
            ph += __popc(hole[i]);
            pu += __popc(high[i]);
        }
    }
    __syncthreads();
    for (int i = threadIdx.x; i < above; i += kPlanThreads) {
        const int2 m = moves[i];
        new_id[m.x] = m.y;
        refs[m.y] = refs[m.x];
        refs[m.x] = 0;
    }
    if (threadIdx.x == 0) *n_moves = above;
}

// The moves (sources and destinations are all different pages), and the tables.
__global__ void __launch_bounds__(kCopyThreads)
compact_move(Pages p, const int32_t *n_moves, const int2 *moves, const int32_t *new_id, int32_t *table, int max_pages,
             const int32_t *held, int B, int32_t *status) {
    pdl_enter();
    for (int b = blockIdx.x; b < B; b += gridDim.x) {
        const int n = held[b];
        int st = 0;
        if (n < 0 || n > max_pages) {
            st = RS_ST_BAD_OFFSET;
        } else {
            for (int i = threadIdx.x; i < n; i += kCopyThreads) {
                int32_t *e = table + (long long)b * max_pages + i;
                const int id = *e, to = in_pool(p, id) ? new_id[id] : -1;
                if (to < 0) st = RS_ST_BAD_PAGE;
                else if (to != id) *e = to;
            }
        }
        const int bad_page = __syncthreads_or(st == RS_ST_BAD_PAGE);
        if (threadIdx.x == 0) status[b] = bad_page ? RS_ST_BAD_PAGE : st;
    }
    const long long total = (long long)*n_moves * p.units;
    for (long long w = blockIdx.x; w < total; w += gridDim.x) {
        const int i = (int)(w / p.units);
        const int2 m = moves[i];
        copy_unit(p, m.x, m.y, (int)(w - (long long)i * p.units));
    }
}

// The pool's arrays, checked.
rs_status make_pages(const char *what, Pages &p, void *k, void *v, int8_t *ke, int8_t *ve, float *weights, int32_t *positions,
                     int bits, int Hkv, int D, int n_pages, int page_size) {
    RS_CHECK_ARG(bits == 8 || bits == 16, "%s: bits=%d: 8 or 16", what, bits);
    if (D != 64 && D != 128) {
        set_error("%s: head dim %d unsupported (64 or 128)", what, D);
        return RS_ERR_UNSUPPORTED;
    }
    RS_CHECK_ARG(Hkv >= 1 && Hkv <= 65535, "%s: Hkv=%d out of range", what, Hkv);
    const rs_status st = bits == 8 ? check_coded_pages(what, n_pages, page_size, 0) : check_pages(what, n_pages, page_size, 0);
    if (st != RS_OK) return st;
    RS_CHECK_ARG((long long)Hkv * page_size <= 1 << 30, "%s: %d heads of %d tokens: above 2^30", what, Hkv, page_size);
    RS_CHECK_ARG(n_pages == 0 || (k && v), "%s: null page pointer", what);
    RS_CHECK_ARG((((uintptr_t)k | (uintptr_t)v) & 15) == 0, "%s: pages must be 16-byte aligned", what);
    RS_CHECK_ARG(n_pages == 0 || bits == 16 || (ke && ve), "%s: an 8-bit cache without exponents", what);
    RS_CHECK_ARG(bits == 8 || (!ke && !ve), "%s: exponents of a 16-bit cache", what);
    p = Pages{};
    p.data[0] = static_cast<char *>(k);
    p.data[1] = static_cast<char *>(v);
    p.exps[0] = reinterpret_cast<char *>(ke);
    p.exps[1] = reinterpret_cast<char *>(ve);
    p.each[0] = reinterpret_cast<uint32_t *>(weights);
    p.each[1] = reinterpret_cast<uint32_t *>(positions);
    p.data_bytes = (long long)page_size * Hkv * D * (bits / 8);
    p.slots = (long long)n_pages * page_size;
    p.exp_bytes = page_size / kCodeBlock * Hkv;
    p.Hkv = Hkv;
    p.page_size = page_size;
    p.n_pages = n_pages;
    p.units = 2 * data_units(p) + (ke || weights || positions ? 1 : 0);
    return RS_OK;
}

unsigned copy_grid(long long units) { return (unsigned)std::max(1ll, std::min(units, 64ll * num_sms())); }

struct CompactWork {
    int32_t *n_moves;
    int2 *moves;
    size_t bytes;
};
CompactWork carve(void *base, int n_pages) {
    Carve cv(base);
    CompactWork w;
    w.n_moves = cv.take<int32_t>(1);
    w.moves = cv.take<int2>((size_t)n_pages / 2 + 1);  // as many holes as moves
    w.bytes = cv.used();
    return w;
}

}  // namespace
}  // namespace rs

using namespace rs;

extern "C" rs_status rs_pages_copy(void *k_pages, void *v_pages, int8_t *k_exps, int8_t *v_exps, float *weights, int32_t *positions,
                                   int bits, int Hkv, int D, int n_pages, int page_size, const int32_t *pairs, int n,
                                   int32_t *status, void *stream) {
    clear_error();
    const char *what = "rs_pages_copy";
    Pages p;
    const rs_status st = make_pages(what, p, k_pages, v_pages, k_exps, v_exps, weights, positions, bits, Hkv, D, n_pages, page_size);
    if (st != RS_OK) return st;
    RS_CHECK_ARG(n >= 0 && n <= 1 << 30, "%s: n=%d out of range (0 to 2^30)", what, n);
    RS_CHECK_ARG(status && (n == 0 || pairs), "%s: null pointer", what);
    RS_CHECK_ARG((reinterpret_cast<uintptr_t>(pairs) & 7) == 0, "%s: pairs must be 8-byte aligned", what);
    launch_pdl(pages_copy, dim3(copy_grid((long long)n * p.units)), dim3(kCopyThreads), 0, (cudaStream_t)stream, p,
               reinterpret_cast<const int2 *>(pairs), n, status);
    RS_CHECK_LAUNCH(what);
    return RS_OK;
}

extern "C" size_t rs_pages_compact_workspace_size(int n_pages) { return n_pages < 0 ? 0 : carve(nullptr, n_pages).bytes; }

extern "C" rs_status rs_pages_compact(void *k_pages, void *v_pages, int8_t *k_exps, int8_t *v_exps, float *weights,
                                      int32_t *positions, int bits, int Hkv, int D, int n_pages, int page_size, int32_t *page_table,
                                      int max_pages, const int32_t *held, int B, int32_t *refs, int32_t *new_id, int32_t *status,
                                      void *workspace, size_t workspace_bytes, void *stream) {
    clear_error();
    const char *what = "rs_pages_compact";
    Pages p;
    rs_status st = make_pages(what, p, k_pages, v_pages, k_exps, v_exps, weights, positions, bits, Hkv, D, n_pages, page_size);
    if (st != RS_OK) return st;
    if ((st = check_pages(what, n_pages, page_size, max_pages)) != RS_OK) return st;
    RS_CHECK_ARG(B >= 0 && B <= 1 << 30, "%s: B=%d out of range (0 to 2^30)", what, B);
    RS_CHECK_ARG(B == 0 || (held && status && (page_table || max_pages == 0)), "%s: null request pointer", what);
    RS_CHECK_ARG(n_pages == 0 || (refs && new_id), "%s: null page pointer", what);
    const CompactWork w = carve(workspace, n_pages);
    if (workspace_bytes < w.bytes || !workspace) {
        set_error("%s: workspace %zu bytes < %zu required", what, workspace_bytes, w.bytes);
        return RS_ERR_CAPACITY;
    }
    RS_CHECK_ARG((reinterpret_cast<uintptr_t>(workspace) & 15) == 0, "%s: workspace must be 16-byte aligned", what);
    const cudaStream_t s = (cudaStream_t)stream;
    launch_pdl(compact_plan, dim3(1), dim3(kPlanThreads), 0, s, n_pages, refs, new_id, w.n_moves, w.moves);
    RS_CHECK_LAUNCH(what);
    launch_pdl(compact_move, dim3(copy_grid((long long)n_pages / 2 * p.units + B)), dim3(kCopyThreads), 0, s, p, w.n_moves, w.moves,
               new_id, page_table, max_pages, held, B, status);
    RS_CHECK_LAUNCH(what);
    return RS_OK;
}
