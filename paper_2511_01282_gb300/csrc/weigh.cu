// weigh.cu -- rs_paged_weights: attention weight that the rows of a chunk give
// to every cached key, added up per KV head:
//     w_j += sum_{rows i that see j} sum_{heads h of the group} exp(scale q_ih.k_j - lse_ih).
//
// The product runs with the keys as its rows, S^T = K Q^T, so that a thread
// holds one key's scores of up to 128 (token, head) columns and its sum stays in
// a register: no exchange between threads, and K, which is read once, stays in
// shared memory while the Q tiles pass by.  A segment is (KV head, request, 256
// keys): two key tiles, so that a Q tile serves 256 keys (with one they would ask
// L2 for 12 TB/s).  Its units are the Q tiles of tq tokens
// that see the keys; tq follows the average chunk, up to 128 / G, so that single
// tokens neither copy nor multiply rows they do not have.  The segments lie end
// to end, a CTA takes an equal share of their cost, and the sums of a segment that
// a share's end cuts are joined by weigh_combine in order (the same bits every time).
// Bound: K and the weights, read once, for single tokens (16 requests of up to 8191
// keys, D = 64: 80 MB in 22 us).  Chunks: shared memory, which the products read at
// its full rate (8 KB each 64 cycles) while Q tiles are written to it and each warp
// reads the columns' lse; then the exponentials (4 cycles a warp for 32 keys).  Four
// prompts of 1000-4000 tokens, D = 128: 116 us, 1060 TFLOP/s of the rows and keys that see each other.
//
// Warps: 0 and 1 issue the products of a key tile each (one warp for both spent as
// long on waits as on products), 2 copies K, 3 copies Q and reads its columns' lse
// (K and Q by one warp: single tokens 33 -> 36 us).  Four warpgroups sum, one for
// each key tile and parity of the Q tiles, which is its S buffer of 128 columns of
// tensor memory: with two, the waits of a tile's chain were not covered (129 us
// against 116).  At a segment's end the two of a key tile join their sums in shared
// memory in a fixed order.
#include <math.h>

#include <algorithm>
#include <atomic>

#include "common.cuh"
#include "roles.cuh"
#include "tmap.cuh"

namespace rs {
namespace {

using namespace sm100;

constexpr int kWgThreads = 640;
constexpr int kWgKeys = 2 * kBN;  // keys of a segment
// A warpgroup hands its part of a segment's sums to the other of its key tile in one of
// these places.  It can not get kNL + 1 segments ahead: the columns' lse of its tiles
// would have to be there, for which the other has finished all but kNL tiles before.
constexpr int kJoins = 8;
constexpr int kWgBeta = 2;  // cost of a segment's start (its K tiles), in Q tiles

struct WeighArgs {
    const int32_t *off, *ctx, *table;
    const float *lse;
    float *weights;
    int32_t *status;
    int4 *req;        // first row, rows (0: nothing to do), ctx
    long long *cum;   // [B + 1] cost prefix of one KV head
    int4 *bound;      // [CTA] start of its share: (KV head, request, key pair, Q tile)
    float *part;      // [2 grid][256]
    int B, T, Hq, Hkv, G, tq, grid, max_pages, n_pages, page_log2;
    float scale;
    long long wait_limit;
};

__device__ __forceinline__ int key_tiles(int4 rq) { return rq.y > 0 ? (rq.z + rq.y + kWgKeys - 1) / kWgKeys : 0; }
// first Q tile that sees key pair jt, and the cost of the request's pairs before
// jt: (Q tiles + beta) tq each, 256 less for every one that lies behind the
// cached tokens (what it sees, up to rounding: the split needs no more)
__device__ __forceinline__ int first_q(const WeighArgs &a, int4 rq, int jt) {
    const int behind = jt * kWgKeys - rq.z;  // most often none: no division
    return behind > 0 ? behind / a.tq : 0;
}
__device__ __forceinline__ long long tiles_cost(const WeighArgs &a, int4 rq, int jt) {
    const long long full = (long long)((rq.y + a.tq - 1) / a.tq + kWgBeta) * a.tq;
    const long long m = max(0, jt - (rq.z + kWgKeys - 1) / kWgKeys);
    return full * jt - (long long)kWgKeys * (m * (m - 1) / 2);
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

// The requests' checks and the prefix of their costs: a thread per request, as far as a
// block goes (1024 threads for a few requests: 1.4 us more a call).
__global__ void __launch_bounds__(1024)
weigh_plan(WeighArgs a) {
    // weigh_kernel takes whole SMs: it launches once earlier work has left them
    pdl_wait_prev();
    pdl_launch_next();
    __shared__ long long s_w[32];
    __shared__ int s_m[32];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
    long long carry = 0;
    int latest = 0;
    for (int base = 0; base < a.B; base += blockDim.x) {
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
        for (int w = 0; w < warps; ++w) latest = max(latest, s_m[w]);
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
        for (int w = 0; w < warps; ++w) carry += s_w[w];
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
    int kvh, b, jt, q_first, q0, q1;  // Q tiles [q0, q1), counted from q_first, the first that sees the keys
    int4 rq;
    int slot;                // -1: the segment is complete here
};
struct WgCursor {
    const WeighArgs &a;
    int4 at, end, rq;
    int rq_of = -1, nq_all = 0;  // the request that rq describes, its Q tiles
    __device__ __forceinline__ WgCursor(const WeighArgs &a_, int4 lo, int4 hi) : a(a_), at(lo), end(hi) {}
    __device__ __forceinline__ bool next(WgPiece &pc) {
        for (;;) {
            const bool same_b = at.x == end.x && at.y == end.y;
            if (at.x > end.x || (at.x == end.x && at.y > end.y) ||
                (same_b && (at.z > end.z || (at.z == end.z && at.w >= end.w))))
                return false;
            if (rq_of != at.y) {
                rq = a.req[at.y];
                rq_of = at.y;
                nq_all = (rq.y + a.tq - 1) / a.tq;
            }
            if (at.z >= key_tiles(rq)) {  // next request, next head
                at.z = at.w = 0;
                if (++at.y == a.B) {
                    at.y = 0;
                    ++at.x;
                }
                continue;
            }
            pc.q_first = first_q(a, rq, at.z);
            const int nq = nq_all - pc.q_first;
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
    static constexpr int kNK = D == 128 ? 2 : 4, kNQ = D == 128 ? 2 : 4, kNL = 4;  // key pairs, Q tiles, columns' lse
    static constexpr int kK = 0, kQ = kNK * 2 * kTile;
    static constexpr int kLse = kQ + kNQ * kTile;     // [kNL][128] floats: -lse in the log2 domain
    static constexpr int kMask = kLse + kNL * 512;    // [kNL][4] words: the columns that count
    static_assert(kMask % 16 == 0, "16-byte reads");
    static constexpr int kJoin = kMask + kNL * 16;  // [2][kJoins][128] floats: sums of a segment's other Q tiles
    static constexpr int kBar = kJoin + 2 * kJoins * 512;
    static constexpr int kNumBars = 2 * (kNK + kNQ + kNL + 4) + 2 * kJoins + 2;
    static constexpr int kMisc = kBar + kNumBars * 8;
    static constexpr int kBounds = (kMisc + 8 + 15) / 16 * 16;
    static constexpr int kTotal = kBounds + 32 + 1024;
    static_assert(kTotal <= 232448, "shared memory of one CTA");
};

// sum += 2^(c s_i + nl_i) over 32 columns, two at a time; the statements in an
// order that keeps the other work between the exponentials (see exp_pairs).
__device__ __forceinline__ void exp_sums(const uint32_t (&s)[32], float2 c, uint32_t nl, uint64_t (&sum)[4]) {
    constexpr int kAhead = 4, kBehind = 4;  // pairs of columns
    constexpr int kRead = 2;                // 16-byte reads of nl ahead of their use
    float2 d[16], p[16];
    ulonglong2 l[8];
    auto read = [&](int i) {
        if (i < 8) asm volatile("ld.shared.v2.b64 {%0, %1}, [%2];" : "=l"(l[i].x), "=l"(l[i].y) : "r"(nl + 16 * i));
    };
    auto fma1 = [&](int e) {
        if (e % 2 == 0) read(e / 2 + kRead);
        const float2 v = make_float2(__uint_as_float(s[2 * e]), __uint_as_float(s[2 * e + 1]));
        uint64_t r;
        asm volatile("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(as_b64(v)), "l"(as_b64(c)), "l"(e % 2 ? l[e / 2].y : l[e / 2].x));
        d[e] = as_float2(r);
    };
#pragma unroll
    for (int i = 0; i < kRead; ++i) read(i);
#pragma unroll
    for (int e = 0; e < kAhead; ++e) fma1(e);
#pragma unroll
    for (int e = 0; e < 16 + kBehind; ++e) {
        if (e < 16) {
            asm volatile("ex2.approx.ftz.f32 %0, %1;" : "=f"(p[e].x) : "f"(d[e].x));
            asm volatile("ex2.approx.ftz.f32 %0, %1;" : "=f"(p[e].y) : "f"(d[e].y));
        }
        if (e + kAhead < 16) fma1(e + kAhead);
        if (e >= kBehind) asm volatile("add.rn.f32x2 %0, %0, %1;" : "+l"(sum[e & 3]) : "l"(as_b64(p[e - kBehind])));
    }
}

template <int D, bool BF16>
__global__ void __launch_bounds__(kWgThreads, 1)
weigh_kernel(WeighArgs a, const __grid_constant__ CUtensorMap tmq, const __grid_constant__ CUtensorMap tmk) {
    using S = WgSmem<D>;
    constexpr uint32_t NK = S::kNK, NQ = S::kNQ, NL = S::kNL;
    extern __shared__ unsigned char smem_raw[];
    unsigned char *smem = reinterpret_cast<unsigned char *>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) &
                                                            ~uintptr_t(1023));
    uint64_t *bars = reinterpret_cast<uint64_t *>(smem + S::kBar);
    uint64_t *kfull = bars, *kempty = kfull + NK, *qfull = kempty + NK, *qempty = qfull + NQ;
    uint64_t *lfull = qempty + NQ, *lempty = lfull + NL, *sfull = lempty + NL, *sempty = sfull + 4, *joined = sempty + 4, *drain = joined + 2 * kJoins;
    uint32_t *s_tmem = reinterpret_cast<uint32_t *>(smem + S::kMisc);
    volatile int *s_abort = reinterpret_cast<volatile int *>(smem + S::kMisc + 4);
    int4 *s_bound = reinterpret_cast<int4 *>(smem + S::kBounds);
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    constexpr int kKB = D / 64;

    if (tid == 0) {
        for (uint32_t s = 0; s < NK; ++s) {
            mbar_init(&kfull[s], 1);
            mbar_init(&kempty[s], 2);  // a commit for each key tile
        }
        for (uint32_t s = 0; s < NQ; ++s) {
            mbar_init(&qfull[s], 1);
            mbar_init(&qempty[s], 2);
        }
        for (uint32_t s = 0; s < NL; ++s) {
            mbar_init(&lfull[s], 32);
            mbar_init(&lempty[s], 2 * kBM);
        }
        for (int s = 0; s < 4; ++s) {  // buffer y of key tile x: 2 x + y
            mbar_init(&sfull[s], 1);
            mbar_init(&sempty[s], kBM);
        }
        for (int s = 0; s < 2 * kJoins; ++s) mbar_init(&joined[s], kBM);
        mbar_init(&drain[0], 1);
        mbar_init(&drain[1], 1);
        *s_abort = 0;
        fence_mbar_init();
    }
    if (warp == 0) tmem_alloc(s_tmem, kTmemCols);
    if (warp == 3 && lane == 0) {
        prefetch_tmap(&tmq);
        prefetch_tmap(&tmk);
    }
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
    const int cols = a.tq * a.G;
    bool ok = true;

    if (warp < 4) {
        if (warp < 2) {
            // ------------------------------------------------------ products of key tile x (whole warp, one lane issues)
            const uint32_t x = (uint32_t)warp;
            // columns in units of 16, the product's granularity
            const uint32_t id = (idesc_16_f32(BF16, kBN, 16, false) & ~(0x3fu << 17)) | ((uint32_t)((cols + 15) / 16 * 2) << 17);
            const uint64_t d0 = sdesc_sw128(smem_u32(smem + S::kK), 16, 1024);
            const uint32_t d_hi = (uint32_t)(d0 >> 32), k_lo0 = (uint32_t)d0;
            const uint32_t q_lo0 = (uint32_t)sdesc_sw128(smem_u32(smem + S::kQ), 16, 1024);
            const uint32_t tm = uniform(tmem + x * 256), idu = uniform(id);
            constexpr uint32_t kTileDesc = S::kTile >> 4;
            uint32_t g = 0, piece = 0;  // Q tiles, segments
            auto wait = [&](uint64_t *b1, uint32_t p1, uint64_t *b2, uint32_t p2) -> bool {
                return ok = quick_wait2(b1, p1 & 1, b2, p2 & 1, s_abort, a.wait_limit);
            };
            while (ok && cur.next(pc)) {
                const uint32_t ks = piece % NK;
                const bool here = pc.rq.z + pc.rq.y > pc.jt * kWgKeys + (int)x * kBN;
                const uint32_t k_lo = uniform(k_lo0 + (2 * ks + x) * kTileDesc);
                if (!wait(&kfull[ks], piece / NK, &kfull[ks], piece / NK)) break;
                for (int qt = pc.q0; qt < pc.q1; ++qt, ++g) {
                    const uint32_t qs = g % NQ;
                    const uint32_t buf = 2 * x + (g & 1);
                    if (!wait(&qfull[qs], g / NQ, &sempty[buf], (g >> 1) ^ 1)) break;
                    tc_fence_after();
                    const uint32_t q_lo = uniform(q_lo0 + qs * kTileDesc), d = uniform(tm + (g & 1) * 128);
                    if (elect_one()) {
                        if (here) {  // (else the commits alone arrive)
#pragma unroll
                            for (int kk = 0; kk < D / 16; ++kk) {
                                const uint32_t o = (uint32_t)(((kk >> 2) * 16384 + (kk & 3) * 32) >> 4);
                                umma_ss(d, desc_of(k_lo + o, d_hi), desc_of(q_lo + o, d_hi), idu, kk > 0);
                            }
                        }
                        umma_commit(&sfull[buf]);
                        umma_commit(&qempty[qs]);
                        if (qt == pc.q1 - 1) umma_commit(&kempty[ks]);
                    }
                    __syncwarp();
                }
                ++piece;
            }
            if (!ok) {
                if (elect_one()) umma_commit(&drain[x]);
                __syncwarp();
                volatile int no_abort = 0;
                mbar_wait(&drain[x], 0, &no_abort, kWaitLimit);
            }
        } else if (warp == 2) {
            // ------------------------------------------------------ key pairs; lane x copies page x
            const int page = 1 << a.page_log2, box = page < kBN ? page : kBN;
            uint32_t piece = 0;
            // pool row of lane x's copy; the table is read a segment ahead
            auto row_of = [&](const WgPiece &p) -> int {
                const int key = p.jt * kWgKeys + lane * box;
                if (lane * box >= kWgKeys || key >= p.rq.z + p.rq.y) return -1;
                const long long s = key_slot(a, p.b, key);
                return s < 0 ? a.n_pages << a.page_log2 : (int)s;  // outside the pool: the copy fills zeros
            };
            bool more = cur.next(pc);
            int row = more ? row_of(pc) : -1;
            while (more) {
                const uint32_t ks = piece % NK;
                const int kvh = pc.kvh, from = row;
                more = cur.next(pc);
                row = more ? row_of(pc) : -1;
                const uint32_t tx = (uint32_t)__popc(__ballot_sync(0xffffffffu, from >= 0)) * (uint32_t)(box * D * 2);
                if (!(ok = warp_wait(&kempty[ks], ((piece / NK) & 1) ^ 1, s_abort, a.wait_limit))) break;
                if (lane == 0) mbar_expect_tx(&kfull[ks], tx);
                __syncwarp();
                if (from >= 0) {
                    const int at = lane * box;  // key tile at / 128, its row at % 128
                    unsigned char *dst = smem + S::kK + (2 * ks + at / kBN) * S::kTile + at % kBN * 128;
#pragma unroll
                    for (int kb = 0; kb < kKB; ++kb) tma_load_3d(dst + kb * 16384, &tmk, &kfull[ks], kb * 64, kvh, from);
                }
                __syncwarp();
                ++piece;
            }
            if (!ok) {
                volatile int no_abort = 0;
                for (uint32_t t = piece >= NK ? piece - NK : 0; t < piece; ++t) mbar_wait(&kfull[t % NK], (t / NK) & 1, &no_abort, kWaitLimit);
            }
        } else {
            // ------------------------------------------------------ Q tiles, their columns' lse
            const uint32_t q_tx = (uint32_t)cols * D * 2;
            uint32_t g = 0;
            int tk[4], hg[4];  // column c = 32 i + lane: token c / G of the tile, head c % G of the group
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                tk[i] = (32 * i + lane) / a.G;
                hg[i] = 32 * i + lane - tk[i] * a.G;
            }
            while (ok && cur.next(pc)) {
                const int q_first = pc.q_first;
                auto read = [&](int qt, float(&v)[4]) {
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const int tok = (q_first + qt) * a.tq + tk[i];
                        v[i] = INFINITY;
                        if (tk[i] < a.tq && tok < pc.rq.y) v[i] = a.lse[(long long)(pc.rq.x + tok) * a.Hq + pc.kvh * a.G + hg[i]];
                    }
                };
                float next[4];
                read(pc.q0, next);
                for (int qt = pc.q0; qt < pc.q1; ++qt, ++g) {
                    const uint32_t ls = g % NL, qs = g % NQ;
                    if (!(ok = warp_wait(&qempty[qs], ((g / NQ) & 1) ^ 1, s_abort, a.wait_limit))) break;
                    if (lane == 0) {
                        mbar_expect_tx(&qfull[qs], q_tx);
#pragma unroll
                        for (int kb = 0; kb < kKB; ++kb)
                            tma_load_3d(smem + S::kQ + qs * S::kTile + kb * 16384, &tmq, &qfull[qs], kb * 64, pc.kvh * a.G,
                                        pc.rq.x + (q_first + qt) * a.tq);
                    }
                    __syncwarp();
                    float v[4];
                    uint32_t m[4];
#pragma unroll
                    for (int i = 0; i < 4; ++i) v[i] = next[i];
                    if (qt + 1 < pc.q1) read(qt + 1, next);
#pragma unroll
                    for (int i = 0; i < 4; ++i) m[i] = __ballot_sync(0xffffffffu, isfinite(v[i]));
                    if (!(ok = warp_wait(&lempty[ls], ((g / NL) & 1) ^ 1, s_abort, a.wait_limit))) {
                        ++g;  // its Q tile is under way
                        break;
                    }
                    float *nl = reinterpret_cast<float *>(smem + S::kLse) + ls * 128;
#pragma unroll
                    for (int i = 0; i < 4; ++i) nl[32 * i + lane] = isfinite(v[i]) ? v[i] * -1.4426950408889634f : 0.f;
                    if (lane < 4)
                        reinterpret_cast<uint32_t *>(smem + S::kMask)[ls * 4 + lane] = lane == 0 ? m[0] : lane == 1 ? m[1] : lane == 2 ? m[2] : m[3];
                    warp_arrive(&lfull[ls]);
                }
            }
            if (!ok) {  // let the copies already issued land before the CTA exits
                volatile int no_abort = 0;
                for (uint32_t t = g >= NQ ? g - NQ : 0; t < g; ++t) mbar_wait(&qfull[t % NQ], (t / NQ) & 1, &no_abort, kWaitLimit);
            }
        }
    } else {
        // ---------------------------------------------------------- sums (a thread per key)
        // x: the key tile; y: Q tiles of this parity
        const int x = (warp - 4) >> 3, r = tid & (kBN - 1);
        const uint32_t y = (uint32_t)(warp >> 2) - 1 & 1, buf = 2 * x + y;
        const uint32_t s_tm = tmem + ((uint32_t)((warp & 3) * 32) << 16) + buf * 128;
        const float2 c2 = make_float2(a.scale * 1.4426950408889634f, a.scale * 1.4426950408889634f);
        const int chunks = (cols + 31) / 32;
        uint32_t g = 0, joins = 0;  // Q tiles, segments of more than one
        while (ok && cur.next(pc)) {
            const int key = pc.jt * kWgKeys + x * kBN + r, keys = pc.rq.z + pc.rq.y, n = pc.q1 - pc.q0;
            const bool here = keys > pc.jt * kWgKeys + x * kBN;  // this key tile has keys
            const bool last = ((g + n - 1) & 1) == y;            // the segment's last Q tile is this warpgroup's
            const long long slot = last && key < keys ? key_slot(a, pc.b, key) : -1;
            const int rel = key - pc.rq.z - (pc.q_first + pc.q0) * a.tq;  // the key's token, counted from the first Q tile's
            uint64_t sum[4] = {0, 0, 0, 0};  // pairs of floats
#pragma unroll 1
            for (uint32_t t = g + ((g ^ y) & 1); t < g + n; t += 2) {
                const uint32_t ls = t % NL;
                if (!(ok = quick_wait2(&lfull[ls], (t / NL) & 1, &sfull[buf], (t >> 1) & 1, s_abort, a.wait_limit))) break;
                tc_fence_after();
                const uint32_t nl = smem_u32(smem + S::kLse) + ls * 512;
                const uint32_t *mask = reinterpret_cast<const uint32_t *>(smem + S::kMask) + ls * 4;
                // columns from lo on see the key: its token is cached or not later than theirs
                const int lo = max(0, rel - (int)(t - g) * a.tq) * a.G;
                const uint4 m = *reinterpret_cast<const uint4 *>(mask);
                const bool open = __all_sync(0xffffffffu, lo == 0 && (m.x & m.y & m.z & m.w) == 0xffffffffu);
#pragma unroll 1
                for (int ch = 0; ch < (here ? chunks : 0); ++ch) {
                    uint32_t v[32];
                    tmem_ld32(s_tm + ch * 32, v);
                    tmem_wait_ld();
                    tmem_regs_ready(v);
                    if (ch == chunks - 1) {
                        tc_fence_before();
                        warp_arrive(&sempty[buf]);
                    }
                    if (!open) {  // by selection: what is hidden may be NaN
                        const int l = lo - ch * 32;
                        hide(v, mask[ch] & (l <= 0 ? 0xffffffffu : l >= 32 ? 0u : ~((1u << l) - 1u)));
                    }
                    exp_sums(v, c2, nl + ch * 128, sum);
                }
                if (!here) {
                    tc_fence_before();
                    warp_arrive(&sempty[buf]);
                }
                warp_arrive(&lempty[ls]);
            }
            if (!ok) break;
            g += n;
            const float2 t2 = add2(add2(as_float2(sum[0]), as_float2(sum[1])), add2(as_float2(sum[2]), as_float2(sum[3])));
            float total = t2.x + t2.y;
            if (n > 1) {  // join both warpgroups' sums
                const uint32_t place = x * kJoins + joins % kJoins;
                float *other = reinterpret_cast<float *>(smem + S::kJoin) + place * kBN + r;
                if (!last) {
                    *other = total;
                    warp_arrive(&joined[place]);
                } else {
                    if (!(ok = quick_wait(&joined[place], (joins / kJoins) & 1, s_abort, a.wait_limit))) break;
                    total += *other;
                }
                ++joins;
            }
            if (last && key < keys) {
                if (pc.slot >= 0) a.part[pc.slot * kWgKeys + x * kBN + r] = total;
                else if (slot < 0) atomicOr(&a.status[pc.b], RS_ST_BAD_PAGE);
                else atomicAdd(&a.weights[((long long)pc.kvh * a.n_pages << a.page_log2) + slot], total);  // the key's only one
            }
        }
    }
    __syncthreads();
    if (warp == 0) {
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
__global__ void __launch_bounds__(kWgKeys)
weigh_combine(WeighArgs a) {
    pdl_enter();
    const int c = blockIdx.x + 1, r = threadIdx.x;
    const int4 at = a.bound[c], before = a.bound[c - 1];
    auto same = [&](int4 p) { return p.x == at.x && p.y == at.y && p.z == at.z && p.w > 0; };
    if (at.w == 0 || same(before)) return;
    float total = a.part[(2 * (c - 1) + 1) * kWgKeys + r];
    for (int c1 = c; c1 < a.grid; ++c1) {
        const int4 p = a.bound[c1], q = a.bound[c1 + 1];
        if (!same(p)) break;
        if (same(q) && q.w == p.w) continue;  // an empty share
        total += a.part[2 * c1 * kWgKeys + r];
    }
    const int4 rq = a.req[at.y];
    const int key = at.z * kWgKeys + r;
    if (key >= rq.z + rq.y) return;
    const long long s = key_slot(a, at.y, key);
    if (s < 0) atomicOr(&a.status[at.y], RS_ST_BAD_PAGE);
    else atomicAdd(&a.weights[((long long)at.x * a.n_pages << a.page_log2) + s], total);
}

size_t carve(WeighArgs &a, void *base, int B, int grid) {
    Carve cv(base);
    a.req = cv.take<int4>((size_t)B);
    a.cum = cv.take<long long>((size_t)B + 1);
    a.bound = cv.take<int4>((size_t)grid + 1);
    a.part = cv.take<float>(2 * (size_t)grid * kWgKeys);
    return cv.used();
}

int weigh_grid() { return std::min(num_sms(), kAttnMaxGrid); }

template <int D, bool BF16>
rs_status weigh_launch(const WeighArgs &a, const CUtensorMap &tmq, const CUtensorMap &tmk, const char *what, cudaStream_t st) {
    static std::atomic<bool> ready[64];  // per device
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) {
        set_error("%s: no current device", what);
        return RS_ERR_CUDA;
    }
    if (!ready[dev].load()) {
        const cudaError_t e = cudaFuncSetAttribute(weigh_kernel<D, BF16>, cudaFuncAttributeMaxDynamicSharedMemorySize, WgSmem<D>::kTotal);
        if (e != cudaSuccess) {
            set_error("%s: kernel attributes: %s", what, cudaGetErrorString(e));
            return RS_ERR_CUDA;
        }
        ready[dev].store(true);
    }
    launch_pdl(weigh_plan, dim3(1), dim3(std::min((a.B + 31) / 32 * 32, 1024)), 0, st, a);  // a thread per request
    RS_CHECK_LAUNCH(what);
    launch_pdl(weigh_kernel<D, BF16>, dim3(a.grid), dim3(kWgThreads), WgSmem<D>::kTotal, st, a, tmq, tmk);
    RS_CHECK_LAUNCH(what);
    if (a.grid > 1) {
        launch_pdl(weigh_combine, dim3(a.grid - 1), dim3(kWgKeys), 0, st, a);
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
    // tokens of a Q tile: the average chunk, as far as 128 columns hold them
    a.tq = std::max(1, std::min(kBM / a.G, (T + B - 1) / B));
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
