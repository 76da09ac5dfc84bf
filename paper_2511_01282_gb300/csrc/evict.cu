// evict.cu -- rs_paged_evict: cuts every request's cache down to a budget of
// tokens per KV head, by accumulated attention weight.
//
// Of the slots s < len of one (request, head) the first `budget` in the order
// (recent ones, then weight descending, then slot ascending) stay.  The kept
// slots behind the budget then move into the holes below it, both in ascending
// order: the holes and the movers are disjoint, so all moves are independent,
// and tokens that already lie below the budget are not touched.
// Launches: evict_select (a CTA per (request, head): the list of moves) ->
// evict_move.
// Bound: weights and positions read once, the movers' rows read and written.
#include <algorithm>

#include "common.cuh"
#include "tmap.cuh"

namespace rs {
namespace {

struct EvictArgs {
    uint16_t *k, *v;
    const int32_t *table, *len, *next_pos;
    float *weights;
    int32_t *positions, *new_len, *status;
    int2 *moves;      // [B][Hkv][budget] (from, to) rows of the pool
    int *n_moves;     // [B][Hkv]
    int B, Hkv, D, n_pages, page_log2, max_pages, budget, recent;
};

// Weights as unsigned keys of the same order; NaN comes last, -0 equals 0.
__device__ __forceinline__ uint32_t weight_key(float w) {
    if (w != w) return 0u;
    const uint32_t u = __float_as_uint(w + 0.f);
    return (u >> 31) ? ~u : (u | 0x80000000u);
}

constexpr int kSelThreads = 1024;

// Inclusive prefix of two small counts at once (16 bits each would overflow:
// two ints) over the block, on top of a carry that every thread keeps.
__device__ __forceinline__ int block_prefix(int v, int &carry, int *s_w) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    int x = v;
    for (int o = 1; o < 32; o <<= 1) {
        const int y = __shfl_up_sync(0xffffffffu, x, o);
        if (lane >= o) x += y;
    }
    if (lane == 31) s_w[warp] = x;
    __syncthreads();
    int w = s_w[lane];
    for (int o = 1; o < 32; o <<= 1) {
        const int y = __shfl_up_sync(0xffffffffu, w, o);
        if (lane >= o) w += y;
    }
    const int before = __shfl_sync(0xffffffffu, w, warp ? warp - 1 : 0);
    x += carry + (warp ? before : 0);
    carry += __shfl_sync(0xffffffffu, w, 31);
    __syncthreads();
    return x;
}

__global__ void __launch_bounds__(kSelThreads)
evict_select(EvictArgs a) {
    pdl_enter();
    __shared__ int s_hist[256], s_w[32];
    __shared__ uint32_t s_prefix;
    __shared__ int s_left;
    const int h = blockIdx.x, b = blockIdx.y, tid = threadIdx.x;
    const int len = a.len[b];
    const int32_t *table = a.table + (long long)b * a.max_pages;
    const int pmask = (1 << a.page_log2) - 1;
    const long long slots = (long long)a.n_pages << a.page_log2;
    int st = 0, bad = 0;
    if (len < 0 || len > ((long long)a.max_pages << a.page_log2)) {
        st = RS_ST_BAD_OFFSET;
    } else if (len > a.budget) {
        for (int p = tid; p <= (len - 1) >> a.page_log2; p += kSelThreads) bad |= table[p] < 0 || table[p] >= a.n_pages;
    }
    if (__syncthreads_or(bad)) st = RS_ST_BAD_PAGE;
    const bool work = st == 0 && len > a.budget;
    if (tid == 0) {
        if (!work) a.n_moves[b * a.Hkv + h] = 0;
        if (h == 0) {
            a.status[b] = st;
            a.new_len[b] = work ? a.budget : len;
        }
    }
    if (!work) return;
    const float *weights = a.weights + h * slots;
    const int32_t *positions = a.positions ? a.positions + h * slots : nullptr;
    const long long newest = (long long)a.next_pos[b] - a.recent;
    auto row_of = [&](int s) -> long long { return ((long long)table[s >> a.page_log2] << a.page_log2) + (s & pmask); };
    auto key_of = [&](int s) -> uint32_t {
        const long long r = row_of(s);
        return positions[r] >= newest ? 0xffffffffu : weight_key(weights[r]);
    };
    // the budget-th largest key, eight bits at a time
    uint32_t prefix = 0;
    int left = a.budget;  // of the keys that share the prefix, how many stay
    for (int shift = 24; shift >= 0; shift -= 8) {
        if (tid < 256) s_hist[tid] = 0;
        __syncthreads();
        for (int s = tid; s < len; s += kSelThreads) {
            const uint32_t k = key_of(s);
            if (shift == 24 || (k >> (shift + 8)) == (prefix >> (shift + 8))) atomicAdd(&s_hist[(k >> shift) & 255u], 1);
        }
        __syncthreads();
        if (tid < 32) {  // lane: eight digits, highest first
            int sum = 0;
            for (int i = 0; i < 8; ++i) sum += s_hist[255 - (tid * 8 + i)];
            int incl = sum;
            for (int o = 1; o < 32; o <<= 1) {
                const int y = __shfl_up_sync(0xffffffffu, incl, o);
                if (tid >= o) incl += y;
            }
            int above = incl - sum;
            if (above < left && incl >= left) {
                for (int i = 0; i < 8; ++i) {
                    const int d = 255 - (tid * 8 + i), n = s_hist[d];
                    if (above + n >= left) {
                        s_prefix = prefix | ((uint32_t)d << shift);
                        s_left = left - above;
                        break;
                    }
                    above += n;
                }
            }
        }
        __syncthreads();
        prefix = s_prefix;
        left = s_left;
    }
    // in slot order: keys above the threshold stay, and the first `left` equal to it
    int2 *moves = a.moves + ((long long)b * a.Hkv + h) * a.budget;
    int ties = 0, holes = 0, movers = 0;
    for (int base = 0; base < len; base += kSelThreads) {
        const int s = base + tid;
        const uint32_t k = s < len ? key_of(s) : 0u;
        const int tie = s < len && k == prefix;
        const int rank = block_prefix(tie, ties, s_w);
        const bool kept = s < len && (k > prefix || (tie && rank <= left));
        const int hole = s < a.budget && !kept, mover = s >= a.budget && kept;
        if (base < a.budget) {
            const int i = block_prefix(hole, holes, s_w);
            if (hole) moves[i - 1].y = (int)row_of(s);
        }
        if (base + kSelThreads > a.budget) {
            const int i = block_prefix(mover, movers, s_w);
            if (mover) moves[i - 1].x = (int)row_of(s);
        }
    }
    if (tid == 0) a.n_moves[b * a.Hkv + h] = movers;
}

constexpr int kMoveThreads = 256;

// D / 8 lanes move one token's row of K and of V; the first also its weight
// and position.
__global__ void __launch_bounds__(kMoveThreads)
evict_move(EvictArgs a) {
    pdl_enter();
    const int lanes = a.D / 8, sub = threadIdx.x % lanes;
    const int bh = blockIdx.y, h = bh % a.Hkv;
    const int n = a.n_moves[bh];
    const int2 *moves = a.moves + (long long)bh * a.budget;
    const long long slots = (long long)a.n_pages << a.page_log2;
    const int per = kMoveThreads / lanes;
    for (int i = blockIdx.x * per + threadIdx.x / lanes; i < n; i += gridDim.x * per) {
        const int2 m = moves[i];
        const long long from = ((long long)m.x * a.Hkv + h) * lanes + sub, to = ((long long)m.y * a.Hkv + h) * lanes + sub;
        const uint4 x = reinterpret_cast<const uint4 *>(a.k)[from], y = reinterpret_cast<const uint4 *>(a.v)[from];
        reinterpret_cast<uint4 *>(a.k)[to] = x;
        reinterpret_cast<uint4 *>(a.v)[to] = y;
        if (sub == 0) {
            a.weights[h * slots + m.y] = a.weights[h * slots + m.x];
            a.positions[h * slots + m.y] = a.positions[h * slots + m.x];
        }
    }
}

size_t carve(EvictArgs &a, void *base, int B, int Hkv, int budget) {
    Carve cv(base);
    a.n_moves = cv.take<int>((size_t)B * Hkv);
    a.moves = cv.take<int2>((size_t)B * Hkv * budget);
    return cv.used();
}

constexpr int kEvictMaxB = 4096;

}  // namespace
}  // namespace rs

using namespace rs;

extern "C" size_t rs_paged_evict_workspace_size(int B, int Hkv, int budget) {
    if (B < 0 || B > kEvictMaxB || Hkv < 1 || Hkv > 65535 || budget < 1 || (long long)B * Hkv > 65535) return 0;
    EvictArgs a{};
    return carve(a, nullptr, B, Hkv, budget);
}

extern "C" rs_status rs_paged_evict(uint16_t *k_pages, uint16_t *v_pages, int Hkv, int D, int n_pages, int page_size,
                                    const int32_t *page_table, int max_pages, const int32_t *cache_len, const int32_t *next_pos,
                                    int B, int budget, int recent, float *weights, int32_t *positions, int32_t *new_len,
                                    int32_t *status, void *workspace, size_t workspace_bytes, void *stream) {
    clear_error();
    const char *what = "rs_paged_evict";
    RS_CHECK_ARG(B >= 0 && B <= kEvictMaxB, "%s: B=%d out of range (0 to %d)", what, B, kEvictMaxB);
    if (D != 64 && D != 128) {
        set_error("%s: head dim %d unsupported (64 or 128)", what, D);
        return RS_ERR_UNSUPPORTED;
    }
    RS_CHECK_ARG(Hkv >= 1 && (long long)B * Hkv <= 65535, "%s: B x Hkv = %d x %d out of range (at most 65535)", what, B, Hkv);
    const rs_status st = check_pages(what, n_pages, page_size, max_pages);
    if (st != RS_OK) return st;
    RS_CHECK_ARG(budget >= 1, "%s: budget=%d must be at least 1", what, budget);
    RS_CHECK_ARG(recent >= 0 && recent <= budget, "%s: recent=%d out of range (0 to budget)", what, recent);
    RS_CHECK_ARG(B == 0 || (cache_len && next_pos && new_len && status && (page_table || max_pages == 0)), "%s: null request pointer", what);
    RS_CHECK_ARG(n_pages == 0 || (k_pages && v_pages && weights && positions), "%s: null page pointer", what);
    RS_CHECK_ARG((((uintptr_t)k_pages | (uintptr_t)v_pages | (uintptr_t)workspace) & 15) == 0,
                 "%s: pages and workspace must be 16-byte aligned", what);
    if (B == 0) return RS_OK;
    EvictArgs a{};
    const size_t need = carve(a, workspace, B, Hkv, budget);
    if (workspace_bytes < need || !workspace) {
        set_error("%s: workspace %zu bytes < %zu required", what, workspace_bytes, need);
        return RS_ERR_CAPACITY;
    }
    a.k = k_pages;
    a.v = v_pages;
    a.table = page_table;
    a.len = cache_len;
    a.next_pos = next_pos;
    a.weights = weights;
    a.positions = positions;
    a.new_len = new_len;
    a.status = status;
    a.B = B;
    a.Hkv = Hkv;
    a.D = D;
    a.n_pages = n_pages;
    a.page_log2 = page_log2(page_size);
    a.max_pages = n_pages ? max_pages : 0;
    a.budget = budget;
    a.recent = recent;
    launch_pdl(evict_select, dim3(Hkv, B), dim3(kSelThreads), 0, (cudaStream_t)stream, a);
    RS_CHECK_LAUNCH(what);
    const int per = kMoveThreads / (D / 8);
    const int chunks = std::max(1, std::min((budget + per - 1) / per, 16 * num_sms() / (B * Hkv) + 1));
    launch_pdl(evict_move, dim3(chunks, B * Hkv), dim3(kMoveThreads), 0, (cudaStream_t)stream, a);
    RS_CHECK_LAUNCH(what);
    return RS_OK;
}
