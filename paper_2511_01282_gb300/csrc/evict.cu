// evict.cu -- rs_paged_evict: cuts every request's cache down to a budget of
// tokens per KV head, by accumulated attention weight.
//
// Of the slots s < len of one (request, head) the first `budget` in the order
// (recent ones by slot, then the others by weight descending and slot ascending) stay.  The kept
// slots behind the budget then move into the holes below it, both in ascending
// order: the holes and the movers are disjoint, so all moves are independent,
// and tokens that already lie below the budget are not touched.
// Launches: evict_select (a CTA or a cluster per (request, head): the list of
// moves) -> evict_move.
// Bound: weights and positions read once, the movers' rows read and written (4
// caches of 32768 tokens to 4096, 8 heads, D = 128: select 24 us, a chain of passes
// and barriers; move 24; 50 in a graph.  16 of 2112 to 2048: 16 us).
#include <algorithm>
#include <atomic>

#include "common.cuh"
#include "sm100.cuh"
#include "tmap.cuh"

namespace rs {
namespace {

struct EvictArgs {
    uint16_t *k, *v;
    const int32_t *table, *len, *next_pos;
    float *weights;
    int32_t *positions, *new_len, *status;
    int2 *moves;      // [B][Hkv][budget] (from, to) slots of the request
    int *n_moves;     // [B][Hkv]
    int B, Hkv, D, n_pages, page_log2, max_pages, budget, recent;
    int cluster, held;  // CTAs of evict_select per (request, head); the longest cache whose keys they hold
};

// Weights as unsigned keys of the same order; NaN comes last, -0 equals 0.
__device__ __forceinline__ uint32_t weight_key(float w) {
    if (w != w) return 0u;
    const uint32_t u = __float_as_uint(w + 0.f);
    return (u >> 31) ? ~u : (u | 0x80000000u);
}

// evict_select: a cluster of CTAs per (request, head), each over a part of the
// slots (more than one where there are fewer pairs than SMs and the caches are
// long: 32768 tokens of 32 pairs took one CTA each 37 us).  A warp owns a run of
// consecutive slots, 32 at a time.  The keys
// are read once into shared memory, as many as it holds (49152 tokens a CTA);
// longer caches are read again in each pass.  (In registers, with every loop
// unrolled, 32 keys a thread took twice as long: the code runs once and is all
// instruction misses.)  The budget-th largest key is
// found by three digits of 11, 11 and 10 bits (the sign, the exponent and two bits
// of the fraction are the first, so that weights of one distribution spread over
// many counters); a warp whose lanes all hold one digit counts once.  Then the
// ties, the holes and the movers are ranked in slot order by ballots and two
// prefixes over the 32 warps.
// Bound: latency (table, then weights and positions; the passes' counters).
constexpr int kSelThreads = 1024;
constexpr int kSelKeys = 49152;
constexpr int kSelBins = 2048;

constexpr int kSelLeast = 4096;  // slots of a CTA, at least, where a cluster shares them

struct SelShared {
    int hist[kSelBins];
    int warp[3][32];
    int total[3];  // of the CTA: ties, holes, movers
    uint32_t prefix;
    int left;
};

// (MANY: a cluster of more than one; alone, the CTA's own barrier and memory do,
// 10 us for 14 on 2112 tokens.)
template <bool MANY>
__device__ __forceinline__ int cluster_read(const int *p, int rank) {
    if (!MANY) return *p;
    uint32_t at = sm100::smem_u32(p);
    int v;
    asm volatile("{\n\t.reg .b32 a;\n\tmapa.shared::cluster.u32 a, %1, %2;\n\tld.shared::cluster.u32 %0, [a];\n\t}"
                 : "=r"(v)
                 : "r"(at), "r"(rank)
                 : "memory");
    return v;
}
// Every CTA's earlier shared-memory writes are there for the others.
template <bool MANY>
__device__ __forceinline__ void cluster_sync() {
    if (MANY) {
        cluster_arrive_release();
        cluster_wait();
    } else {
        __syncthreads();
    }
}

// Exclusive prefix of the warps' counts in row, and their sum (whole block).
__device__ __forceinline__ int warps_before(int (&row)[32], int count, int &sum) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    if (lane == 0) row[warp] = count;
    __syncthreads();
    const int v = row[lane];
    sum = __reduce_add_sync(0xffffffffu, v);
    return __reduce_add_sync(0xffffffffu, lane < warp ? v : 0);
}

struct SelKeys {
    const int32_t *table, *positions;
    const float *weights;
    long long newest;
    int page_log2;
    // pool rows of N slots, 32 apart, then their keys: the loads of a step go out together
    template <int N>
    __device__ __forceinline__ void read(int s, int len, uint32_t (&k)[N]) const {
        int id[N];
        float w[N];
        int32_t p[N];
#pragma unroll
        for (int i = 0; i < N; ++i) id[i] = s + 32 * i < len ? table[(s + 32 * i) >> page_log2] : 0;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int at = s + 32 * i;
            const long long r = ((long long)id[i] << page_log2) + (at & ((1 << page_log2) - 1));
            w[i] = at < len ? weights[r] : 0.f;
            p[i] = at < len ? positions[r] : 0;
        }
#pragma unroll
        for (int i = 0; i < N; ++i) k[i] = p[i] >= newest ? 0xffffffffu : weight_key(w[i]);
    }
};

template <bool MANY, bool HELD>
__device__ __forceinline__ void select_moves(const EvictArgs &a, SelShared &sh, uint32_t *keys, int len, int bh, int rank,
                                             const SelKeys &src) {
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, cs = MANY ? a.cluster : 1;
    const int steps = (len + kSelThreads * cs - 1) / (kSelThreads * cs);  // of 32 slots a warp
    const int first = (rank * (kSelThreads / 32) + warp) * steps * 32 + lane;
    // the CTAs' counts before this one's, and their sum
    auto ctas_before = [&](int i, int &sum) {
        int before = 0;
        sum = 0;
        for (int r = 0; r < cs; ++r) {
            const int v = cluster_read<MANY>(&sh.total[i], r);
            sum += v;
            before += r < rank ? v : 0;
        }
        return before;
    };
    constexpr int kAtOnce = 8;
    if (HELD) {
#pragma unroll 1
        for (int i = 0; i < steps; i += kAtOnce) {
            uint32_t k[kAtOnce];
            src.read(first + i * 32, len, k);
#pragma unroll
            for (int j = 0; j < kAtOnce; ++j)
                if (i + j < steps) keys[(i + j) * kSelThreads + tid] = k[j];
        }
    }
    // use(slot, key, in): every step of the warp, in order
    auto each = [&](auto use) {
        if (HELD) {
#pragma unroll 2
            for (int i = 0; i < steps; ++i) use(first + i * 32, keys[i * kSelThreads + tid], first + i * 32 < len);
        } else {
#pragma unroll 1
            for (int i = 0; i < steps; i += kAtOnce) {
                uint32_t k[kAtOnce];
                src.read(first + i * 32, len, k);
#pragma unroll
                for (int j = 0; j < kAtOnce; ++j)
                    if (i + j < steps) use(first + (i + j) * 32, k[j], first + (i + j) * 32 < len);
            }
        }
    };
    uint32_t prefix = 0;
    int left = a.budget;  // of the keys that share the prefix, how many stay
#pragma unroll 1
    for (int pass = 0; pass < 3; ++pass) {
        const int bits = pass == 2 ? 10 : 11, shift = pass == 0 ? 21 : pass == 1 ? 10 : 0, bins = 1 << bits;
        for (int i = tid; i < bins; i += kSelThreads) sh.hist[i] = 0;
        __syncthreads();
        each([&](int, uint32_t k, bool in) {
            const bool on = in && (pass == 0 || (k >> (shift + bits)) == (prefix >> (shift + bits)));
            const unsigned m = __ballot_sync(0xffffffffu, on);
            if (m == 0) return;
            const int d = (int)((k >> shift) & (uint32_t)(bins - 1));
            const int d0 = __shfl_sync(0xffffffffu, d, __ffs(m) - 1);
            if (__all_sync(0xffffffffu, !on || d == d0)) {
                if (lane == 0) atomicAdd(&sh.hist[d0], __popc(m));
            } else if (on) {
                atomicAdd(&sh.hist[d], 1);
            }
        });
        cluster_sync<MANY>();
        // thread t owns bins / 1024 digits, the highest first, of all CTAs
        const int per = bins / kSelThreads;
        int mine = 0, own[2] = {0, 0};
        for (int i = 0; i < per; ++i) {
            for (int r = 0; r < cs; ++r) own[i] += cluster_read<MANY>(&sh.hist[bins - 1 - (tid * per + i)], r);
            mine += own[i];
        }
        int incl = mine;
        for (int o = 1; o < 32; o <<= 1) {
            const int y = __shfl_up_sync(0xffffffffu, incl, o);
            if (lane >= o) incl += y;
        }
        int all;
        const int before = warps_before(sh.warp[pass], __shfl_sync(0xffffffffu, incl, 31), all);
        int above = before + incl - mine;
        if (above < left && above + mine >= left) {
            for (int i = 0; i < per; ++i) {
                const int d = bins - 1 - (tid * per + i), n = own[i];
                if (above + n >= left) {
                    sh.prefix = prefix | ((uint32_t)d << shift);
                    sh.left = left - above;
                    break;
                }
                above += n;
            }
        }
        cluster_sync<MANY>();  // the counters have been read everywhere
        prefix = sh.prefix;
        left = sh.left;
    }
    // keys above the threshold stay, and the first `left` equal to it
    const unsigned below = (1u << lane) - 1u;
    int ties = 0, sum;
    each([&](int, uint32_t k, bool in) { ties += __popc(__ballot_sync(0xffffffffu, in && k == prefix)); });
    int ties0 = warps_before(sh.warp[0], ties, sum);
    if (tid == 0) sh.total[0] = sum;
    cluster_sync<MANY>();
    ties0 += ctas_before(0, sum);
    auto marks = [&](int s, uint32_t k, bool in, int &tie_rank, bool &hole, bool &mover) {
        const bool tie = in && k == prefix;
        const unsigned m = __ballot_sync(0xffffffffu, tie);
        const bool kept = in && (k > prefix || (tie && tie_rank + __popc(m & below) < left));
        tie_rank += __popc(m);
        hole = s < a.budget && in && !kept;
        mover = s >= a.budget && kept;
    };
    int tie_rank = ties0, holes = 0, movers = 0;
    each([&](int s, uint32_t k, bool in) {
        bool hole, mover;
        marks(s, k, in, tie_rank, hole, mover);
        holes += __popc(__ballot_sync(0xffffffffu, hole));
        movers += __popc(__ballot_sync(0xffffffffu, mover));
    });
    int n;
    int hole_at = warps_before(sh.warp[1], holes, n);
    if (tid == 0) sh.total[1] = n;
    int mover_at = warps_before(sh.warp[2], movers, n);
    if (tid == 0) sh.total[2] = n;
    cluster_sync<MANY>();
    hole_at += ctas_before(1, n);
    mover_at += ctas_before(2, n);
    int2 *moves = a.moves + (long long)bh * a.budget;
    tie_rank = ties0;
    each([&](int s, uint32_t k, bool in) {
        bool hole, mover;
        marks(s, k, in, tie_rank, hole, mover);
        const unsigned mh = __ballot_sync(0xffffffffu, hole), mm = __ballot_sync(0xffffffffu, mover);
        if (hole) moves[hole_at + __popc(mh & below)].y = s;
        if (mover) moves[mover_at + __popc(mm & below)].x = s;
        hole_at += __popc(mh);
        mover_at += __popc(mm);
    });
    if (tid == 0 && rank == 0) a.n_moves[bh] = n;
    cluster_sync<MANY>();  // no CTA leaves while another reads its counts
}

template <bool MANY>
__global__ void __launch_bounds__(kSelThreads)
evict_select(EvictArgs a) {
    pdl_enter();
    __shared__ SelShared sh;
    extern __shared__ uint32_t s_keys[];
    const int cs = MANY ? a.cluster : 1, h = blockIdx.x / cs, rank = blockIdx.x % cs, b = blockIdx.y, tid = threadIdx.x;
    const int len = a.len[b];
    const int32_t *table = a.table + (long long)b * a.max_pages;
    const long long slots = (long long)a.n_pages << a.page_log2;
    int st = 0, bad = 0;
    if (len < 0 || len > ((long long)a.max_pages << a.page_log2)) {
        st = RS_ST_BAD_OFFSET;
    } else if (len > a.budget) {
        for (int p = tid; p <= (len - 1) >> a.page_log2; p += kSelThreads) bad |= table[p] < 0 || table[p] >= a.n_pages;
    }
    if (__syncthreads_or(bad)) st = RS_ST_BAD_PAGE;
    const bool work = st == 0 && len > a.budget;
    const int bh = b * a.Hkv + h;
    if (tid == 0 && rank == 0) {
        if (!work) a.n_moves[bh] = 0;
        if (h == 0) {
            a.status[b] = st;
            a.new_len[b] = work ? a.budget : len;
        }
    }
    if (!work) return;
    const SelKeys src{table, a.positions + h * slots, a.weights + h * slots, (long long)a.next_pos[b] - a.recent, a.page_log2};
    if (len <= a.held) select_moves<MANY, true>(a, sh, s_keys, len, bh, rank, src);
    else select_moves<MANY, false>(a, sh, s_keys, len, bh, rank, src);
}

constexpr int kMoveThreads = 256;

// D / 8 lanes move one token's row of K and of V; the first also its weight
// and position.  Bound: HBM, in rows of 2 D bytes: 3600 tokens of 32 heads, 119 MB,
// in 24 us, 4.9 TB/s, behind a list entry and two table entries each (all of a
// token's reads before its writes: 16 requests 105 -> 97 us; 2 to 4 tokens at a time
// are no faster).
__global__ void __launch_bounds__(kMoveThreads)
evict_move(EvictArgs a) {
    pdl_enter();
    const int lanes = a.D / 8, sub = threadIdx.x % lanes;
    const int bh = blockIdx.y, h = bh % a.Hkv;
    const int n = a.n_moves[bh];
    const int2 *moves = a.moves + (long long)bh * a.budget;
    const long long slots = (long long)a.n_pages << a.page_log2;
    const int32_t *table = a.table + (long long)(bh / a.Hkv) * a.max_pages;
    const int pmask = (1 << a.page_log2) - 1;
    const int per = kMoveThreads / lanes;
    for (int i = blockIdx.x * per + threadIdx.x / lanes; i < n; i += gridDim.x * per) {
        const int2 slot = moves[i];
        const int2 m = make_int2((table[slot.x >> a.page_log2] << a.page_log2) + (slot.x & pmask),
                                 (table[slot.y >> a.page_log2] << a.page_log2) + (slot.y & pmask));
        const long long from = ((long long)m.x * a.Hkv + h) * lanes + sub, to = ((long long)m.y * a.Hkv + h) * lanes + sub;
        const uint4 x = reinterpret_cast<const uint4 *>(a.k)[from], y = reinterpret_cast<const uint4 *>(a.v)[from];
        float w = 0.f;
        int32_t pos = 0;
        if (sub == 0) {
            w = a.weights[h * slots + m.x];
            pos = a.positions[h * slots + m.x];
        }
        reinterpret_cast<uint4 *>(a.k)[to] = x;
        reinterpret_cast<uint4 *>(a.v)[to] = y;
        if (sub == 0) {
            a.weights[h * slots + m.y] = w;
            a.positions[h * slots + m.y] = pos;
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
    // as many CTAs as share the longest cache that the page tables allow, and its keys
    const long long most = (long long)a.max_pages << a.page_log2;
    a.cluster = 1;
    while (a.cluster < 8 && B * Hkv * a.cluster * 2 <= num_sms() && most / (a.cluster * 2) >= kSelLeast) a.cluster *= 2;
    const long long steps = std::min((most + kSelThreads * a.cluster - 1) / (kSelThreads * a.cluster), (long long)(kSelKeys / kSelThreads));
    a.held = (int)steps * kSelThreads * a.cluster;
    const size_t smem = (size_t)steps * kSelThreads * sizeof(uint32_t);
    static std::atomic<int> ready[64];
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) {
        set_error("%s: no current device", what);
        return RS_ERR_CUDA;
    }
    if (!ready[dev].load()) {
        const int most_smem = kSelKeys * (int)sizeof(uint32_t);
        const cudaError_t e1 = cudaFuncSetAttribute(evict_select<false>, cudaFuncAttributeMaxDynamicSharedMemorySize, most_smem);
        const cudaError_t e2 = cudaFuncSetAttribute(evict_select<true>, cudaFuncAttributeMaxDynamicSharedMemorySize, most_smem);
        if (e1 != cudaSuccess || e2 != cudaSuccess) {
            set_error("%s: cudaFuncSetAttribute: %s", what, cudaGetErrorString(e1 != cudaSuccess ? e1 : e2));
            return RS_ERR_CUDA;
        }
        ready[dev].store(1);
    }
    cudaStream_t s = (cudaStream_t)stream;
    if (a.cluster > 1) launch_pdl_cluster(evict_select<true>, dim3(Hkv * a.cluster, B), dim3(kSelThreads), smem, s, a.cluster, a);
    else launch_pdl(evict_select<false>, dim3(Hkv, B), dim3(kSelThreads), smem, s, a);
    RS_CHECK_LAUNCH(what);
    const int per = kMoveThreads / (D / 8);
    const int chunks = std::max(1, std::min((budget + per - 1) / per, 16 * num_sms() / (B * Hkv) + 1));
    launch_pdl(evict_move, dim3(chunks, B * Hkv), dim3(kMoveThreads), 0, (cudaStream_t)stream, a);
    RS_CHECK_LAUNCH(what);
    return RS_OK;
}
