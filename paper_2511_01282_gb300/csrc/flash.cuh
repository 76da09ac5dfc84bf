// flash.cuh -- causal attention of packed rows against contiguous keys (whole
// prompts) or against a paged KV cache (chunks of new tokens, draft trees,
// single tokens).
//
// Row i of a request with n new tokens behind ctx cached ones computes
//     o_i = sum_j p_ij v_j,  p_ij = exp(scale q_i.k_j - lse_i),
//     lse_i = log sum_j exp(scale q_i.k_j),
// over the keys j it sees: j <= ctx + i (causal), or the ctx cached ones and
// the ancestors of node i and itself (tree).  One pass over the keys keeps the
// running maximum m and sum l of every row and the unnormalised O in tensor
// memory: S = Q K^T, P = 2^(c S - m), O += P V, l += sum P (fp32), O rescaled
// only where m grows by more than 2^8.  P is rounded to the type of V for the
// second product: at most half a step relative to each term, as the inputs.
//
// Work: a segment is (KV head, request, pair of row tiles); a row tile is
// tq = 128 / G tokens x G query heads (G = Hq / Hkv; the rows that do not fill
// 128 are idle), so that any G is one TMA box of Q and a K/V tile of 128 keys
// serves 2 tq tokens of all heads of its group.  flash_plan lays the pairs of
// all requests end to end with the prefix of their costs; the KV heads follow
// each other along one axis, and every CTA takes an equal share of the axis
// (in `phases` shares, one per group of KV heads, where all heads' K/V would
// not stay in L2).  A segment cut by a share's end leaves partial (O, m, l),
// which flash_combine joins in key order: no atomics, the same bits each run.
//
// Warps: 0-3 softmax of row tile A (thread = row), 4-7 of tile B, 8 TMA, 9 MMA
// issue, 10-11 idle (they only give registers up).  A pair whose second tile
// is empty runs in half mode: A's S is double buffered.  Tensor memory: O_A
// [0, 128), O_B [128, 256), S/P buffers [256, 384) and [384, 512).
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "attn_core.cuh"

namespace rs {

constexpr int kFlThreads = 384;
constexpr uint32_t kFlRegsSoft = 216, kFlRegsProd = 72;
static_assert(2 * 128 * kFlRegsSoft + 128 * kFlRegsProd == kFlThreads * 168, "register split");
constexpr int kFlMaxPhases = 4;   // groups of KV heads
constexpr int kFlRows = 2 * kBM;  // rows of a segment and of a partial slot
constexpr int kFlWF = 5, kFlWH = 3;  // cost of a key tile for a pair and for a single row tile
constexpr int kFlSegCost = 8;        // cost of a segment's start, in single-tile key tiles, at most
constexpr uint32_t kFlTmS = 256;

struct FlashArgs {
    const int32_t *off, *ctx;    // ctx: null for prompts
    const uint32_t *anc;         // ancestor sets of tree nodes, or null: causal
    const int32_t *page_table;   // null: keys of request b are rows off[b] ..
    int max_pages, n_pages, page_log2;
    int4 *req;                   // per request: first row, rows (0: rejected), ctx
    long long *cum;              // [pairs + 1] cost prefix of the pairs of one KV head
    int2 *ent;                   // [pairs] (request, pair)
    int *n_pairs;
    int4 *bound;                 // [phase][CTA] where the CTA's share starts: (head in phase, pair, tile)
    float *part_o, *part_m, *part_l;
    int phases, grid;
    int B, T, Hq, Hkv, G, tq;
    int kv_stream;               // K/V is large next to L2: tiles read once are evicted first
    float scale;
    uint16_t *out;
    float *lse;
    int32_t *status;
    long long wait_limit;
};

// keys of pair p of a request: what its last token sees
__device__ __forceinline__ int pair_keys(const FlashArgs &a, int4 rq, int p) {
    return rq.z + (a.anc ? rq.y : min(rq.y, (p + 1) * 2 * a.tq));
}

struct FlPiece {
    int b, p, kvh, j0, j1, keys;  // key tiles [j0, j1), keys of the segment
    int n0, n, ctx;
    int slot;                     // partial slot, -1: the segment is complete here
    bool full;                    // the second row tile has rows
};

// A CTA's pieces in order; every role walks them by itself.
struct FlCursor {
    const FlashArgs &a;
    const int4 *bounds;  // shared: [phase][2]
    int M, f = -1, s = 0, t = 0, s_end = -1, t_end = 0;
    __device__ __forceinline__ FlCursor(const FlashArgs &a_, const int4 *b, int M_) : a(a_), bounds(b), M(M_) {}
    __device__ __forceinline__ bool next(FlPiece &pc) {
        for (;;) {
            if (s > s_end || (s == s_end && t >= t_end)) {
                if (++f >= a.phases) return false;
                const int4 lo = bounds[2 * f], hi = bounds[2 * f + 1];
                s = lo.x * M + lo.y;
                t = lo.z;
                s_end = hi.x * M + hi.y;
                t_end = hi.z;
                continue;
            }
            const int hh = s / M;
            const int2 e = a.ent[s - hh * M];
            const int4 rq = a.req[e.x];
            pc.b = e.x;
            pc.p = e.y;
            pc.n0 = rq.x;
            pc.n = rq.y;
            pc.ctx = rq.z;
            pc.kvh = f * a.Hkv / a.phases + hh;
            pc.keys = pair_keys(a, rq, e.y);
            const int nt = (pc.keys + kBN - 1) / kBN;
            pc.j0 = t;
            pc.j1 = s == s_end ? t_end : nt;
            pc.full = rq.y - e.y * 2 * a.tq > a.tq;
            const int share = 2 * (f * a.grid + (int)blockIdx.x);
            pc.slot = t > 0 ? share : (pc.j1 < nt ? share + 1 : -1);
            ++s;
            t = 0;
            return true;
        }
    }
};

__device__ __forceinline__ int seg_cost(const FlashArgs &a, int4 rq, int p, int beta) {
    const int w = rq.y - p * 2 * a.tq > a.tq ? kFlWF : kFlWH;
    return w * ((pair_keys(a, rq, p) + kBN - 1) / kBN) + beta;
}

// Where cost position x of a phase of hn heads falls: (head, pair, tile).
// Whole warp; the pair is searched 32 ways at a time.
__device__ __forceinline__ int4 fl_locate(const FlashArgs &a, long long x, int hn, int M, int beta) {
    const long long C = a.cum[M];
    if (M == 0 || x >= hn * C) return make_int4(hn, 0, 0, 0);
    const int hh = (int)(x / C);
    const long long rem = x - hh * C;
    int lo = 0, hi = M;  // cum[lo] <= rem < cum[hi]
    while (hi - lo > 1) {
        const int step = (hi - lo + 31) / 32;
        const int at = lo + (int)(threadIdx.x & 31) * step;
        const unsigned m = __ballot_sync(0xffffffffu, at < hi && a.cum[at] <= rem);
        lo += (31 - __clz(m)) * step;
        hi = min(lo + step, hi);
    }
    const int2 e = a.ent[lo];
    const int4 rq = a.req[e.x];
    const int w = rq.y - e.y * 2 * a.tq > a.tq ? kFlWF : kFlWH;
    const long long in = rem - a.cum[lo] - beta;
    return make_int4(hh, lo, in > 0 ? (int)(in / w) : 0, 0);
}

template <bool BF16>
__device__ __forceinline__ uint32_t pack16(float lo, float hi) {
    if (BF16) return pack_bf16x2(lo, hi);
    __half2 v = __floats2half2_rn(lo, hi);
    return *reinterpret_cast<uint32_t *>(&v);
}
// fp16 holds P times 2^7: P <= 2^8 then stays below its largest value, and the
// smallest weights keep seven more bits above its subnormals.
template <bool BF16>
constexpr float kFlBias = BF16 ? 0.f : 7.f;

template <int D>
struct FlSmem {
    static constexpr int kTile = kBN * D * 2;
    static constexpr int kNS = D == 128 ? 2 : 4;
    static constexpr int kK = 0, kV = kNS * kTile, kQ = 2 * kNS * kTile;
    static constexpr int kStage = kQ + 2 * kTile;        // 4 KB per softmax warp
    static constexpr int kBar = kStage + 8 * 4096;
    static constexpr int kNumBars = 4 * kNS + 12;
    static constexpr int kMisc = kBar + kNumBars * 8;    // tensor memory base, abort flag
    static constexpr int kBounds = (kMisc + 8 + 15) / 16 * 16;
    static constexpr int kBytes = kBounds + 2 * kFlMaxPhases * 16;
    static constexpr int kTotal = kBytes + 1024;         // the base is rounded up to 1 KB
    static_assert(kTotal <= 232448, "shared memory of one CTA");
};

template <int D, bool BF16>
__global__ void __launch_bounds__(kFlThreads, 1)
flash_kernel(FlashArgs a, const __grid_constant__ CUtensorMap tmq, const __grid_constant__ CUtensorMap tmk,
             const __grid_constant__ CUtensorMap tmv) {
    using namespace sm100;
    using S = FlSmem<D>;
    constexpr int NS = S::kNS;
    extern __shared__ unsigned char smem_raw[];
    unsigned char *smem = reinterpret_cast<unsigned char *>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) &
                                                            ~uintptr_t(1023));
    uint64_t *bars = reinterpret_cast<uint64_t *>(smem + S::kBar);
    uint64_t *kfull = bars, *vfull = kfull + NS, *kempty = vfull + NS, *vempty = kempty + NS;
    uint64_t *sfull = vempty + NS, *pfull = sfull + 2, *qfull = pfull + 2, *qfree = qfull + 2;
    uint64_t *ofree = qfree + 2, *drain = ofree + 1;
    uint32_t *s_tmem = reinterpret_cast<uint32_t *>(smem + S::kMisc);
    volatile int *s_abort = reinterpret_cast<volatile int *>(smem + S::kMisc + 4);
    int4 *s_bound = reinterpret_cast<int4 *>(smem + S::kBounds);

    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    if (tid == 0) {
        for (int s = 0; s < NS; ++s) {
            mbar_init(&kfull[s], 1);
            mbar_init(&vfull[s], 1);
            mbar_init(&kempty[s], kBM);  // the softmax warps that see the last S reading K arrive
            mbar_init(&vempty[s], 1);
        }
        for (int s = 0; s < 2; ++s) {
            mbar_init(&sfull[s], 1);
            mbar_init(&pfull[s], kBM);
            mbar_init(&qfull[s], 1);
            mbar_init(&qfree[s], kBM);
        }
        mbar_init(ofree, kSoftThreads);
        mbar_init(drain, 1);
        *s_abort = 0;
        fence_mbar_init();
    }
    if (warp == kMmaWarp) tmem_alloc(s_tmem, kTmemCols);
    if (warp == kTmaWarp && lane == 0) {
        prefetch_tmap(&tmq);
        prefetch_tmap(&tmk);
        prefetch_tmap(&tmv);
    }
    pdl_wait_prev();
    pdl_launch_next();
    const int M = a.n_pairs[0], beta = a.n_pairs[1];
    if (warp < 2 * a.phases) {  // the two ends of every phase's share, a warp each
        const int f = warp >> 1, h0 = f * a.Hkv / a.phases, hn = (f + 1) * a.Hkv / a.phases - h0;
        const long long L = hn * a.cum[M];
        const int4 at = fl_locate(a, L * (blockIdx.x + (warp & 1)) / a.grid, hn, M, beta);
        if (lane == 0) {
            s_bound[warp] = at;
            if (!(warp & 1)) a.bound[f * (a.grid + 1) + blockIdx.x] = at;
            else if ((int)blockIdx.x == a.grid - 1) a.bound[f * (a.grid + 1) + a.grid] = at;
        }
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = *s_tmem;
    const int G = a.G, tq = a.tq;
    constexpr int kKB = D / 64;  // 64-column swizzle blocks per row
    FlCursor cur(a, s_bound, M);
    FlPiece pc;

    if (warp >= kTmaWarp) {
      reg_dealloc<kFlRegsProd>();
      if (warp == kTmaWarp) {
        // ---------------------------------------------------------- TMA producer
        // Whole warp: in a paged cache lane x copies page x of the tile.
        const uint32_t q_tx = (uint32_t)(tq * G) * D * 2;
        const int page = a.page_table ? 1 << a.page_log2 : kBN;
        const int box = page < kBN ? page : kBN;      // keys per copy
        const uint64_t once = l2_evict_first_policy();
        uint32_t g = 0, quse[2] = {0, 0};
        bool ok = true;
        while (ok && cur.next(pc)) {
            const int32_t *table = a.page_table ? a.page_table + (long long)pc.b * a.max_pages : nullptr;
            const bool evict = a.kv_stream && pc.n <= 2 * tq;
            // rows of the pool where lane x's copy of tile jt starts
            auto row_of = [&](int jt) -> int {
                const int key = jt * kBN + lane * box;
                if (lane * box >= kBN || key >= pc.keys) return -1;
                if (!table) return pc.n0 + key;
                const int id = table[key >> a.page_log2];
                if (id < 0 || id >= a.n_pages) {  // nothing outside the pool is read: the copy fills zeros
                    atomicOr(&a.status[pc.b], RS_ST_BAD_PAGE);
                    return a.n_pages << a.page_log2;
                }
                return (id << a.page_log2) + (key & (page - 1));
            };
            int row = row_of(pc.j0);
            for (int jt = pc.j0; jt < pc.j1; ++jt, ++g) {
                const int st = (int)(g % NS);
                const uint32_t free_par = ((g / NS) & 1) ^ 1;
                const int next_row = jt + 1 < pc.j1 ? row_of(jt + 1) : -1;
                const uint32_t tx = (uint32_t)__popc(__ballot_sync(0xffffffffu, row >= 0)) * (uint32_t)(box * D * 2);
                unsigned char *sk = smem + S::kK + st * S::kTile + lane * box * 128;
                unsigned char *sv = smem + S::kV + st * S::kTile + lane * box * 128;
                if (!(ok = warp_wait(&kempty[st], free_par, s_abort, a.wait_limit))) break;
                if (lane == 0) mbar_expect_tx(&kfull[st], tx);
                __syncwarp();
                if (row >= 0) {
#pragma unroll
                    for (int kb = 0; kb < kKB; ++kb) {
                        if (evict) tma_load_3d_hint(sk + kb * 16384, &tmk, &kfull[st], kb * 64, pc.kvh, row, once);
                        else tma_load_3d(sk + kb * 16384, &tmk, &kfull[st], kb * 64, pc.kvh, row);
                    }
                }
                if (jt == pc.j0) {  // the piece's Q tiles, once its previous S products are done with the buffers
                    for (int x = 0; x < (pc.full ? 2 : 1); ++x) {
                        if (quse[x] > 0 && !(ok = warp_wait(&qfree[x], (quse[x] - 1) & 1, s_abort, a.wait_limit))) break;
                        ++quse[x];
                        if (lane == 0) {
                            mbar_expect_tx(&qfull[x], q_tx);
#pragma unroll
                            for (int kb = 0; kb < kKB; ++kb)
                                tma_load_3d(smem + S::kQ + x * S::kTile + kb * 16384, &tmq, &qfull[x], kb * 64, pc.kvh * G,
                                            pc.n0 + (pc.p * 2 + x) * tq);
                        }
                        __syncwarp();
                    }
                }
                if (!ok || !(ok = warp_wait(&vempty[st], free_par, s_abort, a.wait_limit))) {
                    volatile int no_abort = 0;  // this tile's K copy is in flight: let it land
                    mbar_wait(&kfull[st], (g / NS) & 1, &no_abort, kWaitLimit);
                    break;
                }
                if (lane == 0) mbar_expect_tx(&vfull[st], tx);
                __syncwarp();
                if (row >= 0) {
#pragma unroll
                    for (int kb = 0; kb < kKB; ++kb) {
                        if (evict) tma_load_3d_hint(sv + kb * 16384, &tmv, &vfull[st], kb * 64, pc.kvh, row, once);
                        else tma_load_3d(sv + kb * 16384, &tmv, &vfull[st], kb * 64, pc.kvh, row);
                    }
                }
                row = next_row;
            }
        }
        if (!ok) {  // let the copies already issued land before the CTA exits
            for (uint32_t t = g >= NS ? g - NS : 0; t < g; ++t) {
                volatile int no_abort = 0;
                mbar_wait(&kfull[t % NS], (t / NS) & 1, &no_abort, kWaitLimit);
                mbar_wait(&vfull[t % NS], (t / NS) & 1, &no_abort, kWaitLimit);
            }
            for (int x = 0; x < 2; ++x)
                if (quse[x] > 0) {
                    volatile int no_abort = 0;
                    mbar_wait(&qfull[x], (quse[x] - 1) & 1, &no_abort, kWaitLimit);
                }
        }
      } else if (warp == kMmaWarp) {
       if (lane == 0) {
        // ---------------------------------------------------------- MMA issuer
        constexpr uint32_t idS = idesc_16_f32(BF16, kBM, kBN, false);
        constexpr uint32_t idO = idesc_16_f32(BF16, kBM, D, true);
        const uint64_t dK0 = sdesc_sw128(smem_u32(smem + S::kK), 16, 1024);
        const uint32_t d_hi = (uint32_t)(dK0 >> 32);
        const uint32_t k_lo0 = (uint32_t)dK0;
        const uint32_t q_lo0 = (uint32_t)sdesc_sw128(smem_u32(smem + S::kQ), 16, 1024);
        const uint32_t v_lo0 = (uint32_t)sdesc_sw128(smem_u32(smem + S::kV), 16384, 1024);
        constexpr uint32_t kTileDesc = S::kTile >> 4;
        uint32_t g = 0, use0 = 0, use1 = 0, quse0 = 0, quse1 = 0;
        int piece = 0;
        bool ok = true;
        // S of key tile t for row tile x into buffer buf
        auto issue_s = [=](uint32_t t, int x, int buf) {
            uint32_t k_lo = k_lo0 + (t % NS) * kTileDesc, q_lo = q_lo0 + (uint32_t)x * kTileDesc;
            asm volatile("" : "+r"(k_lo), "+r"(q_lo));  // offsets rebuilt per burst, not kept for every stage
            const uint32_t d_s = tmem + kFlTmS + (uint32_t)buf * 128;
#pragma unroll
            for (int kk = 0; kk < D / 16; ++kk) {
                const uint32_t off = (uint32_t)(((kk >> 2) * 16384 + (kk & 3) * 32) >> 4);
                umma_ss(d_s, desc_of(q_lo + off, d_hi), desc_of(k_lo + off, d_hi), idS, kk > 0);
            }
            umma_commit(&sfull[buf]);
        };
        // O of row tile x += P (buffer buf) V of key tile t
        auto issue_pv = [=](uint32_t t, int x, int buf, bool acc) {
            uint32_t v_lo = v_lo0 + (t % NS) * kTileDesc;
            asm volatile("" : "+r"(v_lo));
            const uint32_t p_tm = tmem + kFlTmS + (uint32_t)buf * 128;
#pragma unroll
            for (int ks = 0; ks < kBN / 16; ++ks)
                umma_ts(tmem + (uint32_t)x * 128, p_tm + ks * 8, desc_of(v_lo + (uint32_t)((ks * 2048) >> 4), d_hi), idO,
                        (acc || ks > 0) ? 1u : 0u);
        };
        auto wait = [&](uint64_t *bar, uint32_t par) -> bool { return ok = mbar_wait(bar, par & 1, s_abort, a.wait_limit); };
        while (ok && cur.next(pc)) {
            const int n = pc.j1 - pc.j0;
            if (!wait(&qfull[0], quse0++)) break;
            if (pc.full && !wait(&qfull[1], quse1++)) break;
            if (!wait(&kfull[g % NS], g / NS)) break;
            tc_fence_after();
            issue_s(g, 0, 0);
            if (pc.full) issue_s(g, 1, 1);
            for (int tl = 0; tl < n; ++tl) {
                const uint32_t t = g + tl;
                const bool more = tl + 1 < n;
                const int b = pc.full ? 0 : tl & 1;
                if (!pc.full && more) {
                    if (!wait(&kfull[(t + 1) % NS], (t + 1) / NS)) break;
                    tc_fence_after();
                    issue_s(t + 1, 0, b ^ 1);
                }
                if (!wait(&pfull[b], pc.full ? use0 + tl : (b ? use1 : use0) + (tl >> 1))) break;
                if (!wait(&vfull[t % NS], t / NS)) break;
                if (tl == 0 && piece > 0 && !wait(ofree, (uint32_t)(piece - 1))) break;
                tc_fence_after();
                issue_pv(t, 0, b, tl > 0);
                if (pc.full) {
                    if (more) {
                        if (!wait(&kfull[(t + 1) % NS], (t + 1) / NS)) break;
                        tc_fence_after();
                        issue_s(t + 1, 0, 0);
                    }
                    if (!wait(&pfull[1], use1 + tl)) break;
                    tc_fence_after();
                    issue_pv(t, 1, 1, tl > 0);
                }
                umma_commit(&vempty[t % NS]);
                if (pc.full && more) issue_s(t + 1, 1, 1);
            }
            use0 += pc.full ? n : (n + 1) >> 1;
            use1 += pc.full ? n : n >> 1;
            g += n;
            ++piece;
        }
        if (!ok) {  // drain the MMAs in flight before tensor memory is released
            umma_commit(drain);
            volatile int no_abort = 0;
            mbar_wait(drain, 0, &no_abort, kWaitLimit);
        }
       }
       __syncwarp();
      }
    } else {
        reg_alloc<kFlRegsSoft>();
        // ---------------------------------------------------------- softmax / epilogue (rows)
        const int x = warp >> 2;        // row tile of this warpgroup
        const int r = tid & (kBM - 1);  // row of the tile == tensor memory lane
        const uint32_t lane_off = (uint32_t)((warp & 3) * 32) << 16;
        const float cexp = a.scale * 1.4426950408889634f;  // scores -> log2 domain (scale > 0)
        const int rt = r / G, rg = r - rt * G;
        unsigned char *stage = smem + S::kStage + warp * 4096;
        uint32_t g = 0, use0 = 0, use1 = 0;
        int piece = 0;
        bool ok = true;
        while (ok && cur.next(pc)) {
            const int n = pc.j1 - pc.j0;
            const bool active = x == 0 || pc.full;
            if (active) {
                const int tok = (pc.p * 2 + x) * tq + rt;
                const bool valid = rt < tq && tok < pc.n;
                const unsigned vmask = __ballot_sync(0xffffffffu, valid);
                // keys that every row of the tile sees
                const int open = pc.ctx + (a.anc ? 0 : (pc.p * 2 + x) * tq + 1);
                const int seen = pc.ctx + tok + 1;  // causal: keys this row sees
                float m_used = -INFINITY, l = 0.f;
                for (int tl = 0; tl < n; ++tl) {
                    const uint32_t t = g + tl;
                    const int key0 = (pc.j0 + tl) * kBN;
                    const int b = pc.full ? x : (tl & 1);
                    const uint32_t par = (pc.full ? (b ? use1 : use0) + tl : (b ? use1 : use0) + (tl >> 1)) & 1;
                    const bool masked = key0 + kBN > open;
                    uint32_t anc[kAncWords];
#pragma unroll
                    for (int w = 0; w < kAncWords; ++w)
                        anc[w] = (a.anc && valid && masked) ? a.anc[(long long)(pc.n0 + tok) * kAncWords + w] : 0u;
                    if (!(ok = warp_wait(&sfull[b], par, s_abort, a.wait_limit))) break;
                    tc_fence_after();
                    // every S reading K of this tile is complete (S_A was issued before S_B)
                    if (x == 1 || !pc.full) warp_arrive(&kempty[t % NS]);
                    // the tile's S was the last to read Q: its buffer is free
                    if (tl == n - 1) warp_arrive(&qfree[x]);
                    if (x == 0 && key0 + kBN > pc.keys) {
                        // slots behind the last key hold anything, NaN too: their V rows are zeroed
                        if (!(ok = warp_wait(&vfull[t % NS], (t / NS) & 1, s_abort, a.wait_limit))) break;
                        unsigned char *sv = smem + S::kV + (t % NS) * S::kTile;
                        const int first = pc.keys - key0, count = (kBN - first) * 8;
                        for (int e = r; e < count * kKB; e += kBM) {
                            const int kb = e / count, c = e - kb * count;
                            *reinterpret_cast<uint4 *>(sv + kb * 16384 + first * 128 + c * 16) = make_uint4(0, 0, 0, 0);
                        }
                        fence_async_smem();
                    }
                    if (vmask == 0) {  // no rows in this warp: its P feeds rows that are never read
                        warp_arrive(&pfull[b]);
                        continue;
                    }
                    const uint32_t s_tm = tmem + lane_off + kFlTmS + (uint32_t)b * 128;
                    float s[kBN];
                    {
                        uint32_t xa[32], xb[32], xc[32], xd[32];
                        tmem_ld32(s_tm, xa);
                        tmem_ld32(s_tm + 32, xb);
                        tmem_ld32(s_tm + 64, xc);
                        tmem_ld32(s_tm + 96, xd);
                        tmem_wait_ld();
                        tmem_regs_ready(xa);
                        tmem_regs_ready(xb);
                        tmem_regs_ready(xc);
                        tmem_regs_ready(xd);
#pragma unroll
                        for (int e = 0; e < 32; ++e) {
                            s[e] = __uint_as_float(xa[e]);
                            s[32 + e] = __uint_as_float(xb[e]);
                            s[64 + e] = __uint_as_float(xc[e]);
                            s[96 + e] = __uint_as_float(xd[e]);
                        }
                    }
                    if (masked) {
#pragma unroll
                        for (int ch = 0; ch < kBN / 32; ++ch) {
                            const int base = key0 + ch * 32;
                            uint32_t msk;
                            if (a.anc) {
                                msk = tree_window(anc, base - pc.ctx);
                            } else {
                                const int c = seen - base;
                                msk = c >= 32 ? 0xffffffffu : c <= 0 ? 0u : (1u << c) - 1u;
                            }
#pragma unroll
                            for (int e = 0; e < 32; ++e)
                                if (!((msk >> e) & 1u)) s[ch * 32 + e] = -INFINITY;
                        }
                    }
                    float mx4[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
                    for (int j = 0; j < kBN; j += 2) mx4[(j >> 1) & 3] = fmaxf(mx4[(j >> 1) & 3], fmaxf(s[j], s[j + 1]));
                    const float mt = fmaxf(fmaxf(mx4[0], mx4[1]), fmaxf(mx4[2], mx4[3])) * cexp;
                    // lazy rescale: move the reference maximum only when it grows
                    // by more than 2^8 (warp-wide O pass, factor 1 for other rows)
                    const bool grow = mt > m_used + 8.f;
                    const float corr = grow ? ex2(m_used - mt) : 1.f;  // 0 when m_used is -inf
                    if (grow) {
                        l *= corr;
                        m_used = mt;
                    }
                    const float nb = (m_used == -INFINITY) ? 0.f : kFlBias<BF16> - m_used;
                    const float2 c2 = make_float2(cexp, cexp), nb2 = make_float2(nb, nb);
                    float2 sum2[4] = {};
#pragma unroll
                    for (int hh = 0; hh < 2; ++hh) {
                        uint32_t xp[32];
#pragma unroll
                        for (int e = 0; e < 32; ++e) {
                            const float2 d = fma2(make_float2(s[hh * 64 + 2 * e], s[hh * 64 + 2 * e + 1]), c2, nb2);
                            const float2 p = make_float2(ex2(d.x), ex2(d.y));
                            sum2[e & 3] = add2(sum2[e & 3], p);
                            xp[e] = pack16<BF16>(p.x, p.y);
                        }
                        tmem_st32(s_tm + hh * 32, xp);
                    }
                    const float2 sum = add2(add2(sum2[0], sum2[1]), add2(sum2[2], sum2[3]));
                    l += sum.x + sum.y;
                    if (tl > 0 && __any_sync(0xffffffffu, grow)) {
                        // O must hold P V of the previous tile: in full mode that
                        // P V was issued before this S; in half mode after it
                        if (!pc.full) {
                            const uint32_t pv = t - 1;
                            if (!(ok = warp_wait(&vempty[pv % NS], (pv / NS) & 1, s_abort, a.wait_limit))) break;
                            tc_fence_after();
                        }
#pragma unroll
                        for (int ch = 0; ch < D / 32; ++ch) {
                            uint32_t xo[32];
                            const uint32_t o_tm = tmem + lane_off + (uint32_t)x * 128 + ch * 32;
                            tmem_ld32(o_tm, xo);
                            tmem_wait_ld();
                            tmem_regs_ready(xo);
#pragma unroll
                            for (int e = 0; e < 32; ++e) xo[e] = __float_as_uint(__uint_as_float(xo[e]) * corr);
                            tmem_st32(o_tm, xo);
                        }
                    }
                    tmem_wait_st();
                    tc_fence_before();
                    warp_arrive(&pfull[b]);
                }
                if (ok) {  // P V of the last tile (its V stage's release is committed after it)
                    const uint32_t pv = g + n - 1;
                    ok = warp_wait(&vempty[pv % NS], (pv / NS) & 1, s_abort, a.wait_limit);
                }
                if (!ok) break;
                tc_fence_after();
                if (vmask) {
                    const long long orow = (long long)(pc.n0 + tok) * a.Hq + pc.kvh * G + rg;
                    if (pc.slot < 0) {
                        // rows leave through shared memory, 64 columns at a time, so that a
                        // store writes whole 128-byte lines (16-byte chunk c of row r at
                        // c ^ (r & 7): no bank conflicts either way)
                        const float f = l > 0.f ? 1.f / l : l;  // no key with weight: 0; NaN stays
                        uint16_t *dst = a.out + orow * D;
#pragma unroll 1
                        for (int ch = 0; ch < D / 64; ++ch) {
#pragma unroll
                            for (int hh = 0; hh < 2; ++hh) {
                                uint32_t xo[32];
                                tmem_ld32(tmem + lane_off + (uint32_t)x * 128 + ch * 64 + hh * 32, xo);
                                tmem_wait_ld();
                                tmem_regs_ready(xo);
#pragma unroll
                                for (int e = 0; e < 4; ++e) {
                                    uint4 v;
                                    v.x = pack16<BF16>(__uint_as_float(xo[8 * e]) * f, __uint_as_float(xo[8 * e + 1]) * f);
                                    v.y = pack16<BF16>(__uint_as_float(xo[8 * e + 2]) * f, __uint_as_float(xo[8 * e + 3]) * f);
                                    v.z = pack16<BF16>(__uint_as_float(xo[8 * e + 4]) * f, __uint_as_float(xo[8 * e + 5]) * f);
                                    v.w = pack16<BF16>(__uint_as_float(xo[8 * e + 6]) * f, __uint_as_float(xo[8 * e + 7]) * f);
                                    *reinterpret_cast<uint4 *>(stage + lane * 128 + (((hh * 4 + e) ^ (lane & 7)) << 4)) = v;
                                }
                            }
                            __syncwarp();
#pragma unroll
                            for (int it = 0; it < 8; ++it) {
                                const int rw = it * 4 + (lane >> 3);  // row of the warp this lane writes
                                uint16_t *d = reinterpret_cast<uint16_t *>(
                                    __shfl_sync(0xffffffffu, reinterpret_cast<unsigned long long>(dst), rw));
                                const uint4 v = *reinterpret_cast<const uint4 *>(stage + rw * 128 + (((lane & 7) ^ (rw & 7)) << 4));
                                if ((vmask >> rw) & 1u) *reinterpret_cast<uint4 *>(d + ch * 64 + (lane & 7) * 8) = v;
                            }
                            __syncwarp();
                        }
                        if (valid) a.lse[orow] = l > 0.f ? (m_used - kFlBias<BF16> + log2f(l)) * 0.6931471805599453f
                                                         : (l == 0.f ? -INFINITY : l);
                    } else {
                        const long long prow = (long long)pc.slot * kFlRows + x * kBM + r;
#pragma unroll 1
                        for (int ch = 0; ch < D / 32; ++ch) {
                            uint32_t xo[32];
                            tmem_ld32(tmem + lane_off + (uint32_t)x * 128 + ch * 32, xo);
                            tmem_wait_ld();
                            tmem_regs_ready(xo);
                            if (valid) {
                                uint4 *d = reinterpret_cast<uint4 *>(a.part_o + prow * D + ch * 32);
#pragma unroll
                                for (int e = 0; e < 8; ++e) d[e] = make_uint4(xo[4 * e], xo[4 * e + 1], xo[4 * e + 2], xo[4 * e + 3]);
                            }
                        }
                        if (valid) {
                            a.part_m[prow] = m_used - kFlBias<BF16>;
                            a.part_l[prow] = l;
                        }
                    }
                    tc_fence_before();
                }
            }
            use0 += pc.full ? n : (n + 1) >> 1;
            use1 += pc.full ? n : n >> 1;
            warp_arrive(ofree);
            // the tile-B warps may not run ahead through pieces in which they have nothing to do
            if (x == 1 && !(ok = warp_wait(ofree, (uint32_t)(piece & 1), s_abort, a.wait_limit))) break;
            ++piece;
            g += n;
        }
    }
    __syncthreads();
    if (warp == kMmaWarp) {
        tc_fence_after();
        tmem_dealloc(tmem, kTmemCols);
    }
    if (tid == 0 && *s_abort) {  // any role gave up: flag every request this CTA touches
        FlCursor again(a, s_bound, M);
        while (again.next(pc)) atomicOr(&a.status[pc.b], RS_ST_TIMEOUT);
    }
}

template <bool BF16>
rs_status flash_launch(const FlashArgs &a, int D, const CUtensorMap &tmq, const CUtensorMap &tmk, const CUtensorMap &tmv,
                       const char *what, cudaStream_t st);

}  // namespace rs
