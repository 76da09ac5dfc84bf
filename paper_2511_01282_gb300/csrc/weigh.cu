// weigh.cu -- rs_paged_weights: attention weight that the rows of a chunk give
// to every cached key, added up per KV head:
//     w_j += sum_{rows i that see j} sum_{heads h of the group} exp(scale q_ih.k_j - lse_ih).
//
// The product runs with the keys as its rows, S^T = K Q^T, so that a thread
// holds one key's scores of 128 (token, head) columns and its sum stays in a
// register: no exchange between threads, and K, which is read once, stays in
// shared memory while the Q tiles pass by.  Work: a segment is (KV head,
// request, 128 keys), its units the Q tiles of tq = 128 / G tokens that see
// the keys.  The segments lie end to end, a CTA takes an equal share of their
// cost, and the sums of a segment that a share's end cuts are joined by
// weigh_combine in order (no atomics: the same bits every time).
// Bound: K and the weights, read once, for single tokens; the exponentials and
// the product (2 D flop each) for long chunks.
//
// Warps: 0-3 and 4-7 two warpgroups that take turns at the Q tiles, 8 TMA, 9
// MMA issue.  Tensor memory: four S buffers of 128 columns.
#include <math.h>

#include <algorithm>
#include <atomic>

#include "common.cuh"
#include "tmap.cuh"

namespace rs {
namespace {

using namespace sm100;

constexpr int kWgThreads = 320;
constexpr int kWgBeta = 2;  // cost of a segment's start (its K tile), in Q tiles

struct WeighArgs {
    const int32_t *off, *ctx, *table;
    const float *lse;
    float *weights;
    int32_t *status;
    int4 *req;        // first row, rows (0: nothing to do), ctx
    long long *cum;   // [B + 1] cost prefix of one KV head
    int4 *bound;      // [CTA] start of its share: (KV head, request, key tile, Q tile)
    float *part;      // [2 grid][128]
    int B, T, Hq, Hkv, G, tq, grid, max_pages, n_pages, page_log2;
    float scale;
    long long wait_limit;
};

__device__ __forceinline__ int key_tiles(int4 rq) { return rq.y > 0 ? (rq.z + rq.y + kBN - 1) / kBN : 0; }
// first Q tile that sees key tile jt, and the cost of the request's tiles before
// jt: (Q tiles + beta) tq each, 128 less for every tile that lies behind the
// cached tokens (what it sees, up to rounding: the split needs no more)
__device__ __forceinline__ int first_q(const WeighArgs &a, int4 rq, int jt) { return max(0, jt * kBN - rq.z) / a.tq; }
__device__ __forceinline__ long long tiles_cost(const WeighArgs &a, int4 rq, int jt) {
    const long long full = (long long)((rq.y + a.tq - 1) / a.tq + kWgBeta) * a.tq;
    const long long m = max(0, jt - (rq.z + kBN - 1) / kBN);
    return full * jt - (long long)kBN * (m * (m - 1) / 2);
}

// Where cost position x falls (whole warp): 32-way searches for the request
// and for its key tile.
__device__ __forceinline__ int4 weigh_locate(const WeighArgs &a, long long x) {
    const long long C = a.cum[a.B];
    if (C == 0 || x >= a.Hkv * C) return make_int4(a.Hkv, 0, 0, 0);
    const int lane = threadIdx.x & 31;
    const int kvh = (int)(x / C);
    long long rem = x - kvh * C;
    int lo = 0, hi = a.B;
    while (hi - lo > 1) {
        const int step = (hi - lo + 31) / 32, at = lo + lane * step;
        const unsigned m = __ballot_sync(0xffffffffu, at < hi && a.cum[at] <= rem);
        lo += (31 - __clz(m)) * step;
        hi = min(lo + step, hi);
    }
    const int b = lo;
    const int4 rq = a.req[b];
    rem -= a.cum[b];
    lo = 0;
    hi = key_tiles(rq);
    while (hi - lo > 1) {
        const int step = (hi - lo + 31) / 32, at = lo + lane * step;
        const unsigned m = __ballot_sync(0xffffffffu, at < hi && tiles_cost(a, rq, at) <= rem);
        lo += (31 - __clz(m)) * step;
        hi = min(lo + step, hi);
    }
    rem -= tiles_cost(a, rq, lo) + kWgBeta * a.tq;
    const int nq = (rq.y + a.tq - 1) / a.tq - first_q(a, rq, lo);
    return make_int4(kvh, b, lo, rem > 0 ? min((int)(rem / a.tq), nq - 1) : 0);
}

__global__ void __launch_bounds__(1024)
weigh_plan(WeighArgs a) {
    // weigh_kernel takes whole SMs: it launches once earlier work has left them
    pdl_wait_prev();
    pdl_launch_next();
    __shared__ long long s_w[32];
    __shared__ int s_m[32];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    long long carry = 0;
    int latest = 0;
    for (int base = 0; base < a.B; base += 1024) {
        const int b = base + threadIdx.x;
        int n0 = 0, n1 = 0, ctx = 0, st = 0;
        if (b < a.B) {
            n0 = a.off[b];
            n1 = a.off[b + 1];
            ctx = a.ctx[b];
        }
        // a request that starts before an earlier one is rejected
        int mx = n0;
        for (int o = 1; o < 32; o <<= 1) {
            const int y = __shfl_up_sync(0xffffffffu, mx, o);
            if (lane >= o) mx = max(mx, y);
        }
        if (lane == 31) s_m[warp] = mx;
        __syncthreads();
        for (int w = 0; w < warp; ++w) mx = max(mx, s_m[w]);
        mx = max(mx, latest);
        for (int w = 0; w < 32; ++w) latest = max(latest, s_m[w]);
        if (n0 < 0 || n1 < n0 || n1 > a.T || mx > n0 || ctx < 0 ||
            (long long)ctx + (n1 - n0) > ((long long)a.max_pages << a.page_log2))
            st = RS_ST_BAD_OFFSET;
        const int4 rq = st || b >= a.B ? make_int4(0, 0, 0, 0) : make_int4(n0, n1 - n0, ctx, 0);
        long long x = tiles_cost(a, rq, key_tiles(rq));
        for (int o = 1; o < 32; o <<= 1) {
            const long long y = __shfl_up_sync(0xffffffffu, x, o);
            if (lane >= o) x += y;
        }
        if (lane == 31) s_w[warp] = x;
        __syncthreads();
        x += carry;
        for (int w = 0; w < warp; ++w) x += s_w[w];
        for (int w = 0; w < 32; ++w) carry += s_w[w];
        if (b < a.B) {
            a.req[b] = rq;
            a.cum[b + 1] = x;
            a.status[b] = st;
        }
        __syncthreads();
    }
    if (threadIdx.x == 0) a.cum[0] = 0;
}

struct WgPiece {
    int kvh, b, jt, q0, q1;  // Q tiles [q0, q1), counted from the first that sees the keys
    int4 rq;
    int slot;                // -1: the segment is complete here
};
struct WgCursor {
    const WeighArgs &a;
    int4 at, end;
    __device__ __forceinline__ WgCursor(const WeighArgs &a_, int4 lo, int4 hi) : a(a_), at(lo), end(hi) {}
    __device__ __forceinline__ bool next(WgPiece &pc) {
        for (;;) {
            const bool same_b = at.x == end.x && at.y == end.y;
            if (at.x > end.x || (at.x == end.x && at.y > end.y) ||
                (same_b && (at.z > end.z || (at.z == end.z && at.w >= end.w))))
                return false;
            const int4 rq = a.req[at.y];
            if (at.z >= key_tiles(rq)) {  // next request, next head
                at.z = at.w = 0;
                if (++at.y == a.B) {
                    at.y = 0;
                    ++at.x;
                }
                continue;
            }
            const int nq = (rq.y + a.tq - 1) / a.tq - first_q(a, rq, at.z);
            pc.kvh = at.x;
            pc.b = at.y;
            pc.jt = at.z;
            pc.rq = rq;
            pc.q0 = at.w;
            pc.q1 = same_b && at.z == end.z ? end.w : nq;
            pc.slot = pc.q0 > 0 ? 2 * (int)blockIdx.x : pc.q1 < nq ? 2 * (int)blockIdx.x + 1 : -1;
            ++at.z;
            at.w = 0;
            return true;
        }
    }
};

// The pool row of key j of request b, or -1 where its page lies outside.
__device__ __forceinline__ long long key_slot(const WeighArgs &a, int b, int j) {
    const int id = a.table[(long long)b * a.max_pages + (j >> a.page_log2)];
    if (id < 0 || id >= a.n_pages) return -1;
    return ((long long)id << a.page_log2) + (j & ((1 << a.page_log2) - 1));
}

template <int D>
struct WgSmem {
    static constexpr int kTile = kBN * D * 2;
    static constexpr int kNK = 2, kNQ = 4, kNS = 4;
    static constexpr int kK = 0, kQ = kNK * kTile;
    static constexpr int kLse = kQ + kNQ * kTile;      // [8 warps][2][128] floats
    static constexpr int kSum = kLse + 8 * 2 * 512;    // [128] floats, from one warpgroup to the other
    static constexpr int kBar = kSum + 512;
    static constexpr int kNumBars = 2 * (kNK + kNQ + kNS) + 3;
    static constexpr int kMisc = kBar + kNumBars * 8;
    static constexpr int kBounds = (kMisc + 8 + 15) / 16 * 16;
    static constexpr int kTotal = kBounds + 32 + 1024;
    static_assert(kTotal <= 232448, "shared memory of one CTA");
};

template <int D, bool BF16>
__global__ void __launch_bounds__(kWgThreads, 1)
weigh_kernel(WeighArgs a, const __grid_constant__ CUtensorMap tmq, const __grid_constant__ CUtensorMap tmk) {
    using S = WgSmem<D>;
    constexpr int NK = S::kNK, NQ = S::kNQ, NS = S::kNS;
    extern __shared__ unsigned char smem_raw[];
    unsigned char *smem = reinterpret_cast<unsigned char *>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) &
                                                            ~uintptr_t(1023));
    uint64_t *bars = reinterpret_cast<uint64_t *>(smem + S::kBar);
    uint64_t *kfull = bars, *kempty = kfull + NK, *qfull = kempty + NK, *qempty = qfull + NQ;
    uint64_t *sfull = qempty + NQ, *sempty = sfull + NS, *given = sempty + NS, *taken = given + 1, *drain = taken + 1;
    uint32_t *s_tmem = reinterpret_cast<uint32_t *>(smem + S::kMisc);
    volatile int *s_abort = reinterpret_cast<volatile int *>(smem + S::kMisc + 4);
    int4 *s_bound = reinterpret_cast<int4 *>(smem + S::kBounds);
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    constexpr int kKB = D / 64;

    if (tid == 0) {
        for (int s = 0; s < NK; ++s) {
            mbar_init(&kfull[s], 1);
            mbar_init(&kempty[s], 1);
        }
        for (int s = 0; s < NQ; ++s) {
            mbar_init(&qfull[s], 1);
            mbar_init(&qempty[s], kBM);
        }
        for (int s = 0; s < NS; ++s) {
            mbar_init(&sfull[s], 1);
            mbar_init(&sempty[s], kBM);
        }
        mbar_init(given, kBM);
        mbar_init(taken, kBM);
        mbar_init(drain, 1);
        *s_abort = 0;
        fence_mbar_init();
    }
    if (warp == kMmaWarp) tmem_alloc(s_tmem, kTmemCols);
    if (warp == kTmaWarp && lane == 0) {
        prefetch_tmap(&tmq);
        prefetch_tmap(&tmk);
    }
    // rows of the Q tiles that no token fills (G does not divide 128) are never
    // copied to: zeroed once, their scores are 0
    const int idle = kBN - a.tq * a.G;
    for (int e = tid; e < NQ * kKB * idle * 8; e += kWgThreads) {
        const int t = e / (idle * 8), c = e - t * idle * 8;
        *reinterpret_cast<uint4 *>(smem + S::kQ + t * 16384 + a.tq * a.G * 128 + c * 16) = make_uint4(0, 0, 0, 0);
    }
    fence_async_smem();
    pdl_wait_prev();
    pdl_launch_next();
    if (warp < 2) {
        const long long L = a.Hkv * a.cum[a.B];
        const int4 at = weigh_locate(a, L * (blockIdx.x + warp) / a.grid);
        if (lane == 0) {
            s_bound[warp] = at;
            if (warp == 0) a.bound[blockIdx.x] = at;
            else if ((int)blockIdx.x == a.grid - 1) a.bound[a.grid] = at;
        }
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = *s_tmem;
    WgCursor cur(a, s_bound[0], s_bound[1]);
    WgPiece pc;

    if (warp == kTmaWarp) {
        // ---------------------------------------------------------- TMA producer
        const int page = 1 << a.page_log2, box = page < kBN ? page : kBN;
        const uint32_t q_tx = (uint32_t)(a.tq * a.G) * D * 2;
        uint32_t g = 0, piece = 0;
        bool ok = true;
        while (ok && cur.next(pc)) {
            const int ks = (int)(piece % NK);
            const int key = pc.jt * kBN + lane * box, keys = pc.rq.z + pc.rq.y;
            int row = -1;
            if (lane * box < kBN && key < keys) {
                const long long s = key_slot(a, pc.b, key);
                row = s < 0 ? a.n_pages << a.page_log2 : (int)s;  // outside the pool: the copy fills zeros
            }
            const uint32_t tx = (uint32_t)__popc(__ballot_sync(0xffffffffu, row >= 0)) * (uint32_t)(box * D * 2);
            if (!(ok = warp_wait(&kempty[ks], ((piece / NK) & 1) ^ 1, s_abort, a.wait_limit))) break;
            if (lane == 0) mbar_expect_tx(&kfull[ks], tx);
            __syncwarp();
            if (row >= 0) {
#pragma unroll
                for (int kb = 0; kb < kKB; ++kb)
                    tma_load_3d(smem + S::kK + ks * S::kTile + kb * 16384 + lane * box * 128, &tmk, &kfull[ks], kb * 64, pc.kvh, row);
            }
            ++piece;
            const int q_first = first_q(a, pc.rq, pc.jt);
            for (int qt = pc.q0; qt < pc.q1; ++qt, ++g) {
                const int qs = (int)(g % NQ);
                if (!(ok = warp_wait(&qempty[qs], ((g / NQ) & 1) ^ 1, s_abort, a.wait_limit))) break;
                if (lane == 0) {
                    mbar_expect_tx(&qfull[qs], q_tx);
#pragma unroll
                    for (int kb = 0; kb < kKB; ++kb)
                        tma_load_3d(smem + S::kQ + qs * S::kTile + kb * 16384, &tmq, &qfull[qs], kb * 64, pc.kvh * a.G,
                                    pc.rq.x + (q_first + qt) * a.tq);
                }
                __syncwarp();
            }
        }
        if (!ok) {  // let the copies already issued land before the CTA exits
            volatile int no_abort = 0;
            for (uint32_t t = piece >= NK ? piece - NK : 0; t < piece; ++t) mbar_wait(&kfull[t % NK], (t / NK) & 1, &no_abort, kWaitLimit);
            for (uint32_t t = g >= NQ ? g - NQ : 0; t < g; ++t) mbar_wait(&qfull[t % NQ], (t / NQ) & 1, &no_abort, kWaitLimit);
        }
    } else if (warp == kMmaWarp) {
        if (lane == 0) {
            // ------------------------------------------------------ MMA issuer
            constexpr uint32_t id = idesc_16_f32(BF16, kBN, kBM, false);
            const uint64_t d0 = sdesc_sw128(smem_u32(smem + S::kK), 16, 1024);
            const uint32_t d_hi = (uint32_t)(d0 >> 32), k_lo0 = (uint32_t)d0;
            const uint32_t q_lo0 = (uint32_t)sdesc_sw128(smem_u32(smem + S::kQ), 16, 1024);
            uint32_t g = 0, piece = 0;
            bool ok = true;
            auto wait = [&](uint64_t *bar, uint32_t par) -> bool { return ok = mbar_wait(bar, par & 1, s_abort, a.wait_limit); };
            while (ok && cur.next(pc)) {
                const uint32_t ks = piece % NK;
                if (!wait(&kfull[ks], piece / NK)) break;
                for (int qt = pc.q0; qt < pc.q1; ++qt, ++g) {
                    const uint32_t qs = g % NQ, buf = g % NS;
                    if (!wait(&qfull[qs], g / NQ)) break;
                    if (!wait(&sempty[buf], (g / NS) ^ 1)) break;
                    tc_fence_after();
                    uint32_t k_lo = k_lo0 + ks * (S::kTile >> 4), q_lo = q_lo0 + qs * (S::kTile >> 4);
                    asm volatile("" : "+r"(k_lo), "+r"(q_lo));
#pragma unroll
                    for (int kk = 0; kk < D / 16; ++kk) {
                        const uint32_t o = (uint32_t)(((kk >> 2) * 16384 + (kk & 3) * 32) >> 4);
                        umma_ss(tmem + buf * 128, desc_of(k_lo + o, d_hi), desc_of(q_lo + o, d_hi), id, kk > 0);
                    }
                    umma_commit(&sfull[buf]);
                }
                if (!ok) break;
                umma_commit(&kempty[ks]);
                ++piece;
            }
            if (!ok) {
                umma_commit(drain);
                volatile int no_abort = 0;
                mbar_wait(drain, 0, &no_abort, kWaitLimit);
            }
        }
        __syncwarp();
    } else {
        // ---------------------------------------------------------- sums (a thread per key)
        const int x = warp >> 2, r = tid & (kBN - 1);
        const uint32_t lane_off = (uint32_t)((warp & 3) * 32) << 16;
        const float c = a.scale * 1.4426950408889634f;
        float *s_lse = reinterpret_cast<float *>(smem + S::kLse) + warp * 256;
        float *s_sum = reinterpret_cast<float *>(smem + S::kSum);
        uint32_t g = 0, gifts = 0;
        bool ok = true;
        while (ok && cur.next(pc)) {
            const int n = pc.q1 - pc.q0, key = pc.jt * kBN + r, keys = pc.rq.z + pc.rq.y;
            const int q_first = first_q(a, pc.rq, pc.jt);
            float2 sum = make_float2(0.f, 0.f);
            for (int t = 0; t < n; ++t) {
                const uint32_t gt = g + t;
                if ((int)(gt & 1) != x) continue;
                const int buf = (int)(gt % NS), tok0 = (q_first + pc.q0 + t) * a.tq;
                // the columns' lse in the log2 domain; +inf for those that count for nothing
                float *lse = s_lse + ((gt >> 1) & 1) * 128;
                bool odd = false;
                for (int e = lane; e < 128; e += 32) {
                    const int tk = e / a.G, tok = tok0 + tk;
                    float l = INFINITY;
                    if (tk < a.tq && tok < pc.rq.y) {
                        l = a.lse[(long long)(pc.rq.x + tok) * a.Hq + pc.kvh * a.G + (e - tk * a.G)] * 1.4426950408889634f;
                        if (!isfinite(l)) {
                            l = INFINITY;
                            odd = true;
                        }
                    }
                    lse[e] = l;
                }
                __syncwarp();
                // columns [lo, hi) see the key: its token is cached or not later than theirs
                const int lo = max(0, key - pc.rq.z - tok0) * a.G, hi = min(a.tq, pc.rq.y - tok0) * a.G;
                const bool checked = __any_sync(0xffffffffu, odd || lo > 0 || hi < a.tq * a.G);
                if (!(ok = warp_wait(&sfull[buf], (gt / NS) & 1, s_abort, a.wait_limit))) break;
                tc_fence_after();
                warp_arrive(&qempty[gt % NQ]);
                uint32_t xa[32], xb[32], xc[32], xd[32];
                const uint32_t s_tm = tmem + lane_off + buf * 128;
                tmem_ld32(s_tm, xa);
                tmem_ld32(s_tm + 32, xb);
                tmem_ld32(s_tm + 64, xc);
                tmem_ld32(s_tm + 96, xd);
                tmem_wait_ld();
                tmem_regs_ready(xa);
                tmem_regs_ready(xb);
                tmem_regs_ready(xc);
                tmem_regs_ready(xd);
                tc_fence_before();
                warp_arrive(&sempty[buf]);
                const float2 c2 = make_float2(c, c);
                auto add = [&](const uint32_t(&s)[32], int base) {
#pragma unroll
                    for (int e = 0; e < 32; e += 4) {
                        const float4 l = *reinterpret_cast<const float4 *>(lse + base + e);
                        float2 u = fma2(make_float2(__uint_as_float(s[e]), __uint_as_float(s[e + 1])), c2, make_float2(-l.x, -l.y));
                        float2 v = fma2(make_float2(__uint_as_float(s[e + 2]), __uint_as_float(s[e + 3])), c2, make_float2(-l.z, -l.w));
                        if (checked) {  // by selection: what is hidden may be NaN
                            const int i = base + e;
                            u.x = i >= lo && i < hi && l.x != INFINITY ? u.x : -INFINITY;
                            u.y = i + 1 >= lo && i + 1 < hi && l.y != INFINITY ? u.y : -INFINITY;
                            v.x = i + 2 >= lo && i + 2 < hi && l.z != INFINITY ? v.x : -INFINITY;
                            v.y = i + 3 >= lo && i + 3 < hi && l.w != INFINITY ? v.y : -INFINITY;
                        }
                        sum = add2(sum, add2(make_float2(ex2(u.x), ex2(u.y)), make_float2(ex2(v.x), ex2(v.y))));
                    }
                };
                add(xa, 0);
                add(xb, 32);
                add(xc, 64);
                add(xd, 96);
            }
            if (!ok) break;
            float total = sum.x + sum.y;
            // the warpgroup of the last tile adds what the other one has and writes
            const bool writer = (int)((g + n - 1) & 1) == x;
            if (n > 1) {
                if (!writer) {
                    if (gifts > 0 && !(ok = warp_wait(taken, (gifts - 1) & 1, s_abort, a.wait_limit))) break;
                    s_sum[r] = total;
                    warp_arrive(given);
                } else {
                    if (!(ok = warp_wait(given, gifts & 1, s_abort, a.wait_limit))) break;
                    total += s_sum[r];
                    warp_arrive(taken);
                }
                ++gifts;
            }
            if (writer && key < keys) {
                if (pc.slot >= 0) {
                    a.part[pc.slot * kBN + r] = total;
                } else {
                    const long long s = key_slot(a, pc.b, key);
                    if (s < 0) atomicOr(&a.status[pc.b], RS_ST_BAD_PAGE);
                    else a.weights[((long long)pc.kvh * a.n_pages << a.page_log2) + s] += total;
                }
            }
            g += n;
        }
    }
    __syncthreads();
    if (warp == kMmaWarp) {
        tc_fence_after();
        tmem_dealloc(tmem, kTmemCols);
    }
    if (tid == 0 && *s_abort) {  // any role gave up: flag every request this CTA touches
        WgCursor again(a, s_bound[0], s_bound[1]);
        while (again.next(pc)) atomicOr(&a.status[pc.b], RS_ST_TIMEOUT);
    }
}

// Joins the sums of the segments that the shares' ends cut: block c looks at
// where CTA c + 1's share starts and, if that is the first cut of a segment,
// adds up its pieces in order.
__global__ void __launch_bounds__(kBN)
weigh_combine(WeighArgs a) {
    pdl_enter();
    const int c = blockIdx.x + 1, r = threadIdx.x;
    const int4 at = a.bound[c], before = a.bound[c - 1];
    auto same = [&](int4 p) { return p.x == at.x && p.y == at.y && p.z == at.z && p.w > 0; };
    if (at.w == 0 || same(before)) return;
    float total = a.part[(2 * (c - 1) + 1) * kBN + r];
    for (int c1 = c; c1 < a.grid; ++c1) {
        const int4 p = a.bound[c1], q = a.bound[c1 + 1];
        if (!same(p)) break;
        if (same(q) && q.w == p.w) continue;  // an empty share
        total += a.part[2 * c1 * kBN + r];
    }
    const int4 rq = a.req[at.y];
    const int key = at.z * kBN + r;
    if (key >= rq.z + rq.y) return;
    const long long s = key_slot(a, at.y, key);
    if (s < 0) atomicOr(&a.status[at.y], RS_ST_BAD_PAGE);
    else a.weights[((long long)at.x * a.n_pages << a.page_log2) + s] += total;
}

size_t carve(WeighArgs &a, void *base, int B, int grid) {
    Carve cv(base);
    a.req = cv.take<int4>((size_t)B);
    a.cum = cv.take<long long>((size_t)B + 1);
    a.bound = cv.take<int4>((size_t)grid + 1);
    a.part = cv.take<float>(2 * (size_t)grid * kBN);
    return cv.used();
}

int weigh_grid() { return std::min(num_sms(), kAttnMaxGrid); }

template <int D, bool BF16>
rs_status weigh_launch(const WeighArgs &a, const CUtensorMap &tmq, const CUtensorMap &tmk, const char *what, cudaStream_t st) {
    static std::atomic<int> ready[64];
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) {
        set_error("%s: no current device", what);
        return RS_ERR_CUDA;
    }
    if (!ready[dev].load()) {
        const cudaError_t e = cudaFuncSetAttribute(weigh_kernel<D, BF16>, cudaFuncAttributeMaxDynamicSharedMemorySize, WgSmem<D>::kTotal);
        if (e != cudaSuccess) {
            set_error("%s: cudaFuncSetAttribute: %s", what, cudaGetErrorString(e));
            return RS_ERR_CUDA;
        }
        ready[dev].store(1);
    }
    launch_pdl(weigh_plan, dim3(1), dim3(1024), 0, st, a);
    RS_CHECK_LAUNCH(what);
    launch_pdl(weigh_kernel<D, BF16>, dim3(a.grid), dim3(kWgThreads), WgSmem<D>::kTotal, st, a, tmq, tmk);
    RS_CHECK_LAUNCH(what);
    if (a.grid > 1) {
        launch_pdl(weigh_combine, dim3(a.grid - 1), dim3(kBN), 0, st, a);
        RS_CHECK_LAUNCH(what);
    }
    return RS_OK;
}

}  // namespace
}  // namespace rs

using namespace rs;

extern "C" size_t rs_paged_weights_workspace_size(int B, int T, int Hq, int Hkv, int D) {
    if (B < 0 || B > kBatchMax || T < 0 || Hkv < 1 || Hq < 1 || Hq % Hkv != 0 || Hq / Hkv > kBM || (D != 64 && D != 128)) return 0;
    WeighArgs a{};
    return carve(a, nullptr, B, weigh_grid());
}

extern "C" rs_status rs_paged_weights(const uint16_t *q, int64_t q_stride, int dtype, const float *lse, const int32_t *new_off,
                                      int B, int T, int Hq, int Hkv, int D, const uint16_t *k_pages, int n_pages, int page_size,
                                      const int32_t *page_table, int max_pages, const int32_t *ctx_len, float scale,
                                      float *weights, int32_t *status, void *workspace, size_t workspace_bytes, void *stream) {
    clear_error();
    const char *what = "rs_paged_weights";
    rs_status st = check_sizes(what, dtype, B, T, Hq, Hkv, D, scale);
    if (st != RS_OK) return st;
    if ((st = check_pages(what, n_pages, page_size, max_pages)) != RS_OK) return st;
    RS_CHECK_ARG(B == 0 || (new_off && ctx_len && status && (page_table || max_pages == 0)), "%s: null request pointer", what);
    RS_CHECK_ARG(T == 0 || (q && lse), "%s: null row pointer", what);
    RS_CHECK_ARG(n_pages == 0 || (k_pages && weights), "%s: null page pointer", what);
    if ((st = check_stride(what, "q", q, q_stride, Hq, D)) != RS_OK) return st;
    RS_CHECK_ARG((((uintptr_t)k_pages | (uintptr_t)workspace) & 15) == 0, "%s: pages and workspace must be 16-byte aligned", what);
    if (B == 0) return RS_OK;
    WeighArgs a{};
    a.grid = weigh_grid();
    const size_t need = carve(a, workspace, B, a.grid);
    if (workspace_bytes < need || !workspace) {
        set_error("%s: workspace %zu bytes < %zu required", what, workspace_bytes, need);
        return RS_ERR_CAPACITY;
    }
    a.off = new_off;
    a.ctx = ctx_len;
    a.table = page_table;
    a.lse = lse;
    a.weights = weights;
    a.status = status;
    a.B = B;
    a.T = T;
    a.Hq = Hq;
    a.Hkv = Hkv;
    a.G = Hq / Hkv;
    a.tq = kBM / a.G;
    a.max_pages = n_pages ? max_pages : 0;
    a.n_pages = n_pages;
    a.page_log2 = page_log2(page_size);
    a.scale = scale;
    a.wait_limit = wait_limit();
    const bool bf16 = dtype == RS_BF16;
    CUtensorMap tmq, tmk;
    if (!rows_map(&tmq, T ? q : workspace, bf16, D, Hq, T, q_stride, a.G, a.tq) ||
        !rows_map(&tmk, n_pages ? k_pages : workspace, bf16, D, Hkv, (long long)n_pages * page_size, (int64_t)Hkv * D, 1,
                  std::min(page_size, kBN))) {
        set_error("%s: cuTensorMapEncodeTiled failed", what);
        return RS_ERR_CUDA;
    }
    cudaStream_t s = (cudaStream_t)stream;
    if (D == 128) return bf16 ? weigh_launch<128, true>(a, tmq, tmk, what, s) : weigh_launch<128, false>(a, tmq, tmk, what, s);
    return bf16 ? weigh_launch<64, true>(a, tmq, tmk, what, s) : weigh_launch<64, false>(a, tmq, tmk, what, s);
}
