// paged.cu -- rs_paged_append: keys and values of new tokens into the pages of
// their requests.
#include "common.cuh"
#include "tmap.cuh"

namespace rs {
namespace {

struct AppendArgs {
    const uint16_t *k, *v;
    long long k_stride, v_stride;
    const int32_t *pos, *off;
    uint16_t *k_pages, *v_pages;
    const int32_t *table, *ctx;
    float *weights;
    int32_t *positions, *status;
    int B, T, Hkv, D, n_pages, page_log2, max_pages;
};

// A warp per new token: its request is found in the offsets (32 ways at a
// time), its slot in the page table; then the token's Hkv heads of K and of V
// move as 16-byte words, all loads of a round under way before its stores.
// Bound: 8 Hkv D bytes a token (read and written once): prompts of 500-8000 tokens,
// 281 MB, in 46 us, 6.05 TB/s; single tokens of 16 requests 3.6 us, the launch.
constexpr int kAppThreads = 256;

__global__ void __launch_bounds__(kAppThreads)
paged_append(AppendArgs a) {
    pdl_enter();
    const int lane = threadIdx.x & 31;
    const int w0 = blockIdx.x * (kAppThreads / 32) + (threadIdx.x >> 5), warps = gridDim.x * (kAppThreads / 32);
    // offsets that decrease anywhere belong to no batch: every request is rejected
    int bad = 0;
    for (int b = lane; b < a.B; b += 32) bad |= a.off[b] > a.off[b + 1];
    const bool ordered = !__any_sync(0xffffffffu, bad) && a.off[0] >= 0 && a.off[a.B] <= a.T;
    for (int b = w0; b < a.B; b += warps) {  // a warp per request: its slots and their pages
        const int n = a.off[b + 1] - a.off[b], ctx = a.ctx[b];
        int st = 0;
        if (!ordered || ctx < 0 || (long long)ctx + n > ((long long)a.max_pages << a.page_log2)) {
            st = RS_ST_BAD_OFFSET;
        } else if (n > 0) {
            for (int p = (ctx >> a.page_log2) + lane; p <= (ctx + n - 1) >> a.page_log2; p += 32) {
                const int id = a.table[(long long)b * a.max_pages + p];
                if (id < 0 || id >= a.n_pages) st = RS_ST_BAD_PAGE;
            }
        }
        st = __reduce_or_sync(0xffffffffu, st);
        if (lane == 0) a.status[b] = st;
    }
    if (!ordered) return;
    for (int i = w0; i < a.T; i += warps) {
        int lo = 0, hi = a.B;  // last b with off[b] <= i
        while (hi - lo > 1) {
            const int step = (hi - lo + 31) / 32, at = lo + lane * step;
            const unsigned m = __ballot_sync(0xffffffffu, at < hi && a.off[at] <= i) | 1u;
            lo += (31 - __clz(m)) * step;
            hi = min(lo + step, hi);
        }
        const int n0 = a.off[lo], n1 = a.off[lo + 1], ctx = a.ctx[lo];
        if (i < n0 || i >= n1 || ctx < 0 || (long long)ctx + (n1 - n0) > ((long long)a.max_pages << a.page_log2)) continue;
        const int s = ctx + (i - n0);
        const int id = a.table[(long long)lo * a.max_pages + (s >> a.page_log2)];
        if (id < 0 || id >= a.n_pages) continue;
        const long long slot = ((long long)id << a.page_log2) + (s & ((1 << a.page_log2) - 1));
        const int words = a.Hkv * a.D / 8;
        const uint4 *ks = reinterpret_cast<const uint4 *>(a.k + i * a.k_stride);
        const uint4 *vs = reinterpret_cast<const uint4 *>(a.v + i * a.v_stride);
        uint4 *kd = reinterpret_cast<uint4 *>(a.k_pages) + slot * words, *vd = reinterpret_cast<uint4 *>(a.v_pages) + slot * words;
        for (int c = lane; c < words; c += 128) {
            uint4 x[4], y[4];
#pragma unroll
            for (int u = 0; u < 4; ++u)
                if (c + u * 32 < words) {
                    x[u] = ks[c + u * 32];
                    y[u] = vs[c + u * 32];
                }
#pragma unroll
            for (int u = 0; u < 4; ++u)
                if (c + u * 32 < words) {
                    kd[c + u * 32] = x[u];
                    vd[c + u * 32] = y[u];
                }
        }
        const long long slots = (long long)a.n_pages << a.page_log2;
        for (int h = lane; h < a.Hkv; h += 32) {
            if (a.weights) a.weights[h * slots + slot] = 0.f;
            if (a.positions) a.positions[h * slots + slot] = a.pos ? a.pos[i] : s;
        }
    }
}

}  // namespace
}  // namespace rs

using namespace rs;

extern "C" rs_status rs_paged_append(const uint16_t *k, int64_t k_stride, const uint16_t *v, int64_t v_stride,
                                     const int32_t *pos, const int32_t *new_off, int B, int T, int Hkv, int D,
                                     uint16_t *k_pages, uint16_t *v_pages, int n_pages, int page_size,
                                     const int32_t *page_table, int max_pages, const int32_t *ctx_len, float *weights,
                                     int32_t *positions, int32_t *status, void *stream) {
    clear_error();
    const char *what = "rs_paged_append";
    RS_CHECK_ARG(B >= 0 && T >= 0, "%s: negative size", what);
    RS_CHECK_ARG(T <= 1 << 30, "%s: T=%d above 2^30", what, T);  // a warp's next token stays an int
    RS_CHECK_ARG(B <= 1 << 30, "%s: B=%d above 2^30", what, B);
    if (D != 64 && D != 128) {
        set_error("%s: head dim %d unsupported (64 or 128)", what, D);
        return RS_ERR_UNSUPPORTED;
    }
    RS_CHECK_ARG(Hkv >= 1 && Hkv <= 65536, "%s: Hkv=%d out of range", what, Hkv);
    const rs_status st = check_pages(what, n_pages, page_size, max_pages);
    if (st != RS_OK) return st;
    RS_CHECK_ARG(B == 0 || (new_off && ctx_len && status && (page_table || max_pages == 0)), "%s: null request pointer", what);
    RS_CHECK_ARG(T == 0 || (k && v), "%s: null row pointer", what);
    RS_CHECK_ARG(n_pages == 0 || (k_pages && v_pages), "%s: null page pointer", what);
    RS_CHECK_ARG((((uintptr_t)k | (uintptr_t)v | (uintptr_t)k_pages | (uintptr_t)v_pages) & 15) == 0,
                 "%s: k, v and pages must be 16-byte aligned", what);
    RS_CHECK_ARG(k_stride >= (int64_t)Hkv * D && v_stride >= (int64_t)Hkv * D && k_stride % 8 == 0 && v_stride % 8 == 0,
                 "%s: rows of k and v: at least Hkv x D elements, a multiple of 8", what);
    if (B == 0) return RS_OK;
    AppendArgs a{k, v, k_stride, v_stride, pos, new_off, k_pages, v_pages, page_table, ctx_len, weights, positions, status,
                 B, T, Hkv, D, n_pages, page_log2(page_size), n_pages ? max_pages : 0};
    const long long blocks = ((long long)std::max(T, (B + 31) / 32) + kAppThreads / 32 - 1) / (kAppThreads / 32);
    launch_pdl(paged_append, dim3((unsigned)std::min(blocks, 8ll * num_sms())), dim3(kAppThreads), 0, (cudaStream_t)stream, a);
    RS_CHECK_LAUNCH(what);
    return RS_OK;
}
