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
// (in up to four phases, each for a group of KV heads, where all heads' K/V
// would not stay in L2: a prompt of 65536 tokens 25.1 -> 21.9 ms; the plan knows
// what is cached and decides).  A segment cut by a share's end leaves partial (O, m, l),
// which flash_combine joins in key order: no atomics, the same bits each run.
//
// Bound: long prompts at D = 128, the tensor cores (16384 tokens, 32 heads on 8: 1.48
// ms, 1480 TFLOP/s); at D = 64, whose products are half as long, the softmax warps
// (issue slots 52 % full, each warp's chain of wait, maximum, exponentials and store;
// 16 prompts of up to 4095 tokens: 518 us, 732 TFLOP/s, a tenth of it segments'
// starts); single tokens, HBM (64 requests, 1.21 GB: 187 us, 6.5 TB/s); those of one
// request, the latency of three launches (2048 keys: 19 us).
//
// Warps: 0 and 1 MMA issue for row tiles A and B, 2 and 3 TMA (K and Q, V), 4-7
// softmax of tile A (thread = row), 8-11 of tile B.  Tensor memory (512 columns):
//   D = 64: O_A O_B (64 each), S_A S_B (128 each), P_A P_B (64 each).  S of the
//     next key tile is issued as soon as its softmax has read the last one, so
//     that a softmax finds its next S ready and the exponentials bound the loop.
//   D = 128: O_A O_B (128 each), S_A S_B (128 each), P written over S: S of the
//     next tile follows P V of this one.  The two row tiles take turns, and P goes
//     to the product in two halves.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <type_traits>

#include "attn_core.cuh"
#include "roles.cuh"

namespace rs {

constexpr int kFlThreads = 384;
constexpr int kFlMmaWarp = 0, kFlTmaWarp = 2, kFlSoftWarp = 4;  // two warps issue products, two copy
// (with 56 registers the product warps spill: 56 bytes at D = 128, with 88 12, and packed
// prompts take 525 us for 518; the softmax warps' code is the same from 200 up)
constexpr uint32_t kFlRegsSoft = 208, kFlRegsProd = 88;
static_assert(2 * 128 * kFlRegsSoft + 128 * kFlRegsProd == kFlThreads * 168, "register split");
constexpr int kFlMaxPhases = 4;   // groups of KV heads
constexpr int kFlRows = 2 * kBM;  // rows of a segment and of a partial slot
// What a CTA's time goes to, in eighths of a key tile of a pair: a key tile where
// only the first row tile has rows, and a segment's start (the first copies and
// products, the epilogue).  Fitted to every CTA's cycles over packed prompts, chunks
// and a long prompt: 2650, 1900 and 5000 cycles at D = 64; 2850, 2500 and 7200 at D = 128.
constexpr int kFlPair = 8;
constexpr int fl_single(int D) { return D == 64 ? 6 : 7; }
constexpr int fl_start(int D) { return D == 64 ? 15 : 20; }
// Tensor memory columns
template <int D>
struct FlTm {
    static constexpr bool kApart = D == 64;  // P has columns of its own
    __host__ __device__ static constexpr uint32_t o(int x) { return (uint32_t)(x * D); }
    __host__ __device__ static constexpr uint32_t s(int x) { return (uint32_t)(2 * D + x * 128); }
    __host__ __device__ static constexpr uint32_t p(int x) { return kApart ? (uint32_t)(384 + x * 64) : s(x); }
};

struct FlashArgs {
    const int32_t *off, *ctx;    // ctx: null for prompts
    const uint32_t *anc;         // ancestor sets of tree nodes, or null: causal
    const int32_t *page_table;   // null: keys of request b are rows off[b] ..
    int max_pages, n_pages, page_log2;
    int4 *req;                   // per request: first row, rows (0: rejected), ctx, rows of its own
    long long *cum;              // [pairs + 1] cost prefix of the pairs of one KV head
    int4 *ent;                   // [pairs] request, pair, first row and rows of the request
    int *ent_ctx;                // [pairs] its ctx
    int *n_pairs;                // pairs, cost of a segment's start, phases (the plan's choices)
    int4 *bound;                 // [phase][CTA] where the CTA's share starts: (head in phase, pair, tile)
    float *part_o, *part_m, *part_l;
    int max_phases, grid;
    int single, start;           // costs: fl_single, fl_start
    int comb_blocks;             // blocks of flash_combine per cut segment
    int B, T, Hq, Hkv, G, tq;
    int kv_stream;               // K/V is large next to L2: tiles read once are evicted first
    float scale;
    uint16_t *out;
    float *lse;
    int32_t *status;
    long long wait_limit;
};

// keys of pair p of a request of n rows behind ctx: what its last token sees
__device__ __forceinline__ int pair_keys(const FlashArgs &a, int n, int ctx, int p) {
    return ctx + (a.anc ? n : min(n, (p + 1) * 2 * a.tq));
}
__device__ __forceinline__ int pair_tiles(const FlashArgs &a, int n, int ctx, int p) {
    return (pair_keys(a, n, ctx, p) + kBN - 1) / kBN;
}
// Key tiles that some row of row tile x of the pair sees.  The first row tile's may end
// before the pair's (causal): P V is left out there, where P is 0 and V may hold NaN.
__device__ __forceinline__ int row_tiles(const FlashArgs &a, int n, int ctx, int p, int x) {
    return (ctx + (a.anc ? n : min(n, (2 * p + x + 1) * a.tq)) + kBN - 1) / kBN;
}
// cost of one of its key tiles
__device__ __forceinline__ int tile_cost(const FlashArgs &a, int n, int p) {
    return n - p * 2 * a.tq > a.tq ? kFlPair : a.single;
}

struct FlPiece {
    int b, p, kvh, j0, j1, keys;  // key tiles [j0, j1), keys of the segment
    int n0, n, ctx;
    int slot;                     // partial slot, -1: the segment is complete here
    bool full;                    // the second row tile has rows
};

// A CTA's pieces in order; every role walks them by itself.  The next piece's
// record is loaded a piece ahead.
struct FlCursor {
    const FlashArgs &a;
    const int4 *bounds;  // shared: [phase][2]
    int M, f = -1, h0 = 0, hh = 0, i = 0, t = 0;  // phase, its first head, head in it, pair, key tile
    int hh_end = -1, i_end = 0, t_end = 0;
    int at = -1, ctx = 0;                 // the pair whose record is at hand
    int4 e;
    __device__ __forceinline__ FlCursor(const FlashArgs &a_, const int4 *b, int M_) : a(a_), bounds(b), M(M_) {}
    __device__ __forceinline__ void load(int k) {
        at = k;
        e = a.ent[k];
        ctx = a.ent_ctx[k];
    }
    __device__ __forceinline__ bool next(FlPiece &pc) {
        while (hh > hh_end || (hh == hh_end && (i > i_end || (i == i_end && t >= t_end)))) {
            const int phases = a.n_pairs[2];
            if (++f >= phases) return false;
            h0 = f * a.Hkv / phases;
            const int4 lo = bounds[2 * f], hi = bounds[2 * f + 1];
            hh = lo.x;
            i = lo.y;
            t = lo.z;
            hh_end = hi.x;
            i_end = hi.y;
            t_end = hi.z;
        }
        if (at != i) load(i);
        pc.b = e.x;
        pc.p = e.y;
        pc.n0 = e.z;
        pc.n = e.w;
        pc.ctx = ctx;
        pc.kvh = h0 + hh;
        pc.keys = pair_keys(a, e.w, ctx, e.y);
        const int nt = (pc.keys + kBN - 1) / kBN;
        pc.j0 = t;
        pc.j1 = hh == hh_end && i == i_end ? t_end : nt;
        pc.full = e.w - e.y * 2 * a.tq > a.tq;
        const int share = 2 * (f * a.grid + (int)blockIdx.x);
        pc.slot = t > 0 ? share : (pc.j1 < nt ? share + 1 : -1);
        t = 0;
        if (++i == M) {
            i = 0;
            ++hh;
        }
        load(i);
        return true;
    }
};

// Where cost position x of a phase of hn heads falls: (head, pair, tile).
// No piece shorter than half a segment's start is cut off (64 sequences of 256
// tokens, 96.7 -> 93.0 us; 32 of up to 1000 at D = 128, 159.7 -> 156.1).
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
    const int4 e = a.ent[lo];
    const int w = tile_cost(a, e.w, e.y), in = (int)(rem - a.cum[lo]) - beta;
    if (2 * in < beta) return make_int4(hh, lo, 0, 0);
    if (2 * (w * pair_tiles(a, e.w, a.ent_ctx[lo], e.y) - in) < beta) return lo + 1 < M ? make_int4(hh, lo + 1, 0, 0) : make_int4(hh + 1, 0, 0, 0);
    return make_int4(hh, lo, in / w, 0);
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

// 64 weights of a row: xp = 2^(c s + nb) in 16 bits, their fp32 sums added to
// sum4.  The exponentials (4 cycles a warp) bound it; volatile statements keep
// the other instructions between them, where the compiler's own order puts
// them into bursts (a probe of two warps per scheduler: 1360 cycles for both
// warps' 128 weights against 1600).
template <bool BF16>
__device__ __forceinline__ void exp_pairs(const uint32_t (&s0)[32], const uint32_t (&s1)[32], float c, float nb,
                                          float (&sum4)[4], uint32_t (&xp)[32]) {
    constexpr int kAhead = 4, kBehind = 4;  // pairs
    float d[64], p[64];
    auto fma1 = [&](int i) {
        const float v = __uint_as_float(i < 32 ? s0[i] : s1[i - 32]);
        asm volatile("fma.rn.f32 %0, %1, %2, %3;" : "=f"(d[i]) : "f"(v), "f"(c), "f"(nb));
    };
#pragma unroll
    for (int i = 0; i < 2 * kAhead; ++i) fma1(i);
#pragma unroll
    for (int e = 0; e < 32 + kBehind; ++e) {
        if (e < 32) {
            asm volatile("ex2.approx.ftz.f32 %0, %1;" : "=f"(p[2 * e]) : "f"(d[2 * e]));
            asm volatile("ex2.approx.ftz.f32 %0, %1;" : "=f"(p[2 * e + 1]) : "f"(d[2 * e + 1]));
        }
        if (e + kAhead < 32) {
            fma1(2 * (e + kAhead));
            fma1(2 * (e + kAhead) + 1);
        }
        if (e >= kBehind) {
            const int q = e - kBehind;
            asm volatile("add.rn.f32 %0, %0, %1;" : "+f"(sum4[(2 * q) & 3]) : "f"(p[2 * q]));
            asm volatile("add.rn.f32 %0, %0, %1;" : "+f"(sum4[(2 * q + 1) & 3]) : "f"(p[2 * q + 1]));
            if (BF16) asm volatile("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(xp[q]) : "f"(p[2 * q + 1]), "f"(p[2 * q]));
            else asm volatile("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(xp[q]) : "f"(p[2 * q + 1]), "f"(p[2 * q]));
        }
    }
}

// 32 bytes in one store (p 32-byte aligned): a whole sector, so that a thread
// may write its own row.
__device__ __forceinline__ void store32(void *p, const uint32_t *v) {
    asm volatile("st.global.v8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};" ::"l"(p), "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]),
                 "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7])
                 : "memory");
}

template <int D>
struct FlSmem {
    static constexpr int kTile = kBN * D * 2;
    static constexpr int kNK = D == 128 ? 3 : 4, kNV = D == 128 ? 2 : 4;  // stages of K and V
    static constexpr int kK = 0, kV = kNK * kTile, kQ = kV + kNV * kTile;
    static constexpr int kBar = kQ + 2 * kTile;
    static constexpr int kNumBars = 2 * kNK + 2 * kNV + 20;
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
    constexpr uint32_t NK = S::kNK, NV = S::kNV;
    extern __shared__ unsigned char smem_raw[];
    unsigned char *smem = reinterpret_cast<unsigned char *>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) &
                                                            ~uintptr_t(1023));
    uint64_t *bars = reinterpret_cast<uint64_t *>(smem + S::kBar);
    uint64_t *kfull = bars, *kempty = kfull + NK, *vfull = kempty + NK, *vempty = vfull + NV;
    // per row tile: S there, S read (kApart), P there (its two halves), P V complete,
    // Q there, Q read, O read, turn at the tensor core
    uint64_t *sfull = vempty + NV, *sfree = sfull + 2, *pfull = sfree + 2, *pfull2 = pfull + 2, *pvdone = pfull2 + 2;
    uint64_t *qfull = pvdone + 2, *qfree = qfull + 2, *ofree = qfree + 2, *turn = ofree + 2;
    uint64_t *drain = turn + 2;
    uint32_t *s_tmem = reinterpret_cast<uint32_t *>(smem + S::kMisc);
    volatile int *s_abort = reinterpret_cast<volatile int *>(smem + S::kMisc + 4);
    int4 *s_bound = reinterpret_cast<int4 *>(smem + S::kBounds);

    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    if (tid == 0) {
        for (int s = 0; s < (int)NK; ++s) {
            mbar_init(&kfull[s], 1);
            mbar_init(&kempty[s], 2);  // a commit for each row tile
        }
        for (int s = 0; s < (int)NV; ++s) {
            mbar_init(&vfull[s], 1);
            mbar_init(&vempty[s], 2);
        }
        for (int x = 0; x < 2; ++x) {
            mbar_init(&sfull[x], 1);
            mbar_init(&sfree[x], kBM);
            mbar_init(&pfull[x], kBM);
            mbar_init(&pfull2[x], kBM);
            mbar_init(&pvdone[x], 1);
            mbar_init(&qfull[x], 1);
            mbar_init(&qfree[x], kBM);
            mbar_init(&ofree[x], kBM);
            mbar_init(&turn[x], 1);
            mbar_init(&drain[x], 1);
        }
        *s_abort = 0;
        fence_mbar_init();
    }
    if (warp == kFlMmaWarp) tmem_alloc(s_tmem, kTmemCols);
    if (warp == kFlTmaWarp && lane == 0) {
        prefetch_tmap(&tmq);
        prefetch_tmap(&tmk);
        prefetch_tmap(&tmv);
    }
    pdl_wait_prev();
    pdl_launch_next();
    const int M = a.n_pairs[0], beta = a.n_pairs[1], phases = a.n_pairs[2];
    if (warp < 2 * phases) {  // the two ends of every phase's share, a warp each
        const int f = warp >> 1, h0 = f * a.Hkv / phases, hn = (f + 1) * a.Hkv / phases - h0;
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
    using Tm = FlTm<D>;
    constexpr bool kApart = Tm::kApart;
    constexpr int kParts = kApart ? 1 : 2;  // P goes to the product in so many parts
    constexpr int kKB = D / 64;  // 64-column swizzle blocks per row
    FlCursor cur(a, s_bound, M);
    FlPiece pc;

    if (warp < kFlSoftWarp) {
      reg_dealloc<kFlRegsProd>();
      if (warp >= kFlTmaWarp) {
        // ---------------------------------------------------------- TMA producers
        // One warp for K (and Q), one for V.  Whole warps: in a paged cache lane x
        // copies page x of the tile (a copy takes a warp some 75 cycles to issue, and
        // a tile in pages of 16 tokens is 16 copies: with one warp for both they bound
        // long chunks, 665 us for 500).
        const bool is_v = warp == kFlTmaWarp + 1;
        const CUtensorMap *map = is_v ? &tmv : &tmk;
        uint64_t *full = is_v ? vfull : kfull, *empty = is_v ? vempty : kempty;
        unsigned char *ring = smem + (is_v ? S::kV : S::kK);
        const uint32_t stages = is_v ? NV : NK;
        const uint32_t q_tx = (uint32_t)(tq * G) * D * 2;
        const int page = a.page_table ? 1 << a.page_log2 : kBN;
        const int box = page < kBN ? page : kBN;      // keys per copy
        const uint64_t once = l2_evict_first_policy();
        uint32_t st = 0, phase = 0, quse[2] = {0, 0};  // stage, its phase; Q tiles copied
        uint32_t used = 0;                             // stages in use so far (at most all)
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
            for (int jt = pc.j0; jt < pc.j1; ++jt) {
                const int next_row = jt + 1 < pc.j1 ? row_of(jt + 1) : -1;
                const uint32_t tx = (uint32_t)__popc(__ballot_sync(0xffffffffu, row >= 0)) * (uint32_t)(box * D * 2);
                if (!(ok = warp_wait(&empty[st], phase ^ 1, s_abort, a.wait_limit))) break;
                if (lane == 0) mbar_expect_tx(&full[st], tx);
                __syncwarp();
                if (row >= 0) {
                    unsigned char *dst = ring + st * S::kTile + lane * box * 128;
#pragma unroll
                    for (int kb = 0; kb < kKB; ++kb) {
                        if (evict) tma_load_3d_hint(dst + kb * 16384, map, &full[st], kb * 64, pc.kvh, row, once);
                        else tma_load_3d(dst + kb * 16384, map, &full[st], kb * 64, pc.kvh, row);
                    }
                }
                __syncwarp();
                used = min(used + 1, stages);
                if (++st == stages) {
                    st = 0;
                    phase ^= 1;
                }
                row = next_row;
                if (is_v || jt != pc.j0) continue;
                // the piece's Q tiles, once its previous S products are done with the buffers
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
                if (!ok) break;
            }
        }
        if (!ok) {  // let the copies already issued land before the CTA exits
            volatile int no_abort = 0;
            for (uint32_t u = 0; u < used; ++u) {
                if (st == 0) {
                    st = stages;
                    phase ^= 1;
                }
                --st;
                mbar_wait(&full[st], phase, &no_abort, kWaitLimit);
            }
            for (int x = 0; x < 2; ++x)
                if (quse[x] > 0) mbar_wait(&qfull[x], (quse[x] - 1) & 1, &no_abort, kWaitLimit);
        }
      } else if (warp <= kFlMmaWarp + 1) {
        // ---------------------------------------------------------- MMA issuers, one per row tile
        // The whole warp walks the loop, so that descriptors and addresses are the
        // same in all lanes and stay in uniform registers; one elected lane issues.
        // A wait costs some 110 cycles even for a phase that is complete, which two
        // warps and waits for two barriers at a time keep off the tensor core.
        const int x = warp - kFlMmaWarp;
        constexpr uint32_t idS = idesc_16_f32(BF16, kBM, kBN, false);
        constexpr uint32_t idO = idesc_16_f32(BF16, kBM, D, true);
        const uint64_t dK0 = sdesc_sw128(smem_u32(smem + S::kK), 16, 1024);
        const uint32_t d_hi = (uint32_t)(dK0 >> 32);
        const uint32_t k_lo0 = (uint32_t)dK0;
        const uint32_t q_lo0 = (uint32_t)sdesc_sw128(smem_u32(smem + S::kQ), 16, 1024);
        const uint32_t v_lo0 = (uint32_t)sdesc_sw128(smem_u32(smem + S::kV), 16384, 1024);
        constexpr uint32_t kTileDesc = S::kTile >> 4;
        const uint32_t tm = uniform(tmem), xu = uniform((uint32_t)x);
        const uint32_t q_lo = q_lo0 + xu * kTileDesc, s_tm = tm + Tm::s(0) + xu * 128;
        const uint32_t o_tm = tm + Tm::o(0) + xu * D, p_tm = tm + Tm::p(0) + xu * (kApart ? 64 : 128);
        uint32_t g = 0, done = 0, pieces = 0, turns = 0;  // key tiles of the CTA; key tiles, pieces of this row tile
        bool ok = true;
        auto wait = [&](uint64_t *b1, uint32_t p1, uint64_t *b2, uint32_t p2) -> bool {
            return ok = quick_wait2(b1, p1 & 1, b2, p2 & 1, s_abort, a.wait_limit);
        };
        // S of key tile t (K and, at D = 64, S's columns are there)
        auto issue_s = [&](uint32_t t) {
            tc_fence_after();
            const uint32_t k_lo = uniform(k_lo0 + (t % NK) * kTileDesc);
            if (elect_one()) {
#pragma unroll
                for (int kk = 0; kk < D / 16; ++kk) {
                    const uint32_t off = (uint32_t)(((kk >> 2) * 16384 + (kk & 3) * 32) >> 4);
                    umma_ss(s_tm, desc_of(q_lo + off, d_hi), desc_of(k_lo + off, d_hi), idS, kk > 0);
                }
                umma_commit(&sfull[x]);
                umma_commit(&kempty[t % NK]);
                if (!pc.full) umma_commit(&kempty[t % NK]);  // for the row tile that is not there
            }
            __syncwarp();
        };
        while (ok && cur.next(pc)) {
            const int n = pc.j1 - pc.j0;
            if (x == 1 && !pc.full) {
                g += n;
                continue;
            }
            if (!wait(&kfull[g % NK], g / NK, &qfull[x], pieces)) break;
            if (kApart && done > 0 && !wait(&sfree[x], done - 1, &sfree[x], done - 1)) break;
            issue_s(g);
            // of the piece's key tiles, those that some row of the row tile sees; the others go
            // through without P V (by a predicate: a branch around it cost a prompt of 16384
            // tokens 3 %)
            const int seen = (int)uniform((uint32_t)min(n, row_tiles(a, pc.n, pc.ctx, pc.p, x) - pc.j0));
#pragma unroll 1
            for (int tl = 0; tl < n; ++tl, ++done) {
                const uint32_t t = g + tl, st = t % NV;
                const bool more = tl + 1 < n;
                if (kApart) {  // S of the next tile goes ahead of this one's P V
                    if (more) {
                        if (!wait(&kfull[(t + 1) % NK], (t + 1) / NK, &sfree[x], done)) break;
                        issue_s(t + 1);
                    }
                    if (!wait(&vfull[st], t / NV, &pfull[x], done)) break;
                } else {
                    // what does not depend on the softmax first; then P and, where both row
                    // tiles are at work, the turn: they alternate, so that one's softmax
                    // runs beside the other's products
                    const uint32_t tn = t + 1;
                    if (!wait(&vfull[st], t / NV, more ? &kfull[tn % NK] : &vfull[st], more ? tn / NK : t / NV)) break;
                    const bool must = pc.full && (x == 1 || turns > 0);
                    if (!wait(&pfull[x], done, must ? &turn[x] : &pfull[x], must ? turns - (x == 0 ? 1 : 0) : done)) break;
                }
                if (tl == 0 && pieces > 0 && !wait(&ofree[x], pieces - 1, &ofree[x], pieces - 1)) break;
                tc_fence_after();
                const uint32_t v_lo = uniform(v_lo0 + st * kTileDesc);
#pragma unroll
                for (int part = 0; part < kParts; ++part) {
                    if (part > 0) {
                        if (!wait(&pfull2[x], done, &pfull2[x], done)) break;
                        tc_fence_after();
                    }
                    if (elect_one()) {
#pragma unroll
                        for (int ks = part * 8 / kParts; ks < (part + 1) * 8 / kParts; ++ks)
                            umma_ts_if(tl < seen, o_tm, p_tm + ks * 8, desc_of(v_lo + (uint32_t)((ks * 2048) >> 4), d_hi), idO,
                                       (tl > 0 || ks > 0) ? 1u : 0u);
                        if (part == kParts - 1) {
                            umma_commit(&pvdone[x]);
                            umma_commit(&vempty[st]);
                            if (!pc.full) umma_commit(&vempty[st]);
                        }
                    }
                    __syncwarp();
                }
                if (!ok) break;
                if (!kApart) {
                    if (more) issue_s(t + 1);
                    if (pc.full) {
                        if (lane == 0) mbar_arrive_cnt(&turn[x ^ 1], 1);
                        __syncwarp();
                        ++turns;
                    }
                }
            }
            ++pieces;
            g += n;
        }
        if (!ok) {  // drain the MMAs in flight before tensor memory is released
            if (elect_one()) umma_commit(&drain[x]);
            __syncwarp();
            volatile int no_abort = 0;
            mbar_wait(&drain[x], 0, &no_abort, kWaitLimit);
        }
      }
    } else {
        reg_alloc<kFlRegsSoft>();
        // ---------------------------------------------------------- softmax / epilogue (rows)
        const int x = (warp - kFlSoftWarp) >> 2;  // row tile of this warpgroup
        const int r = tid & (kBM - 1);  // row of the tile == tensor memory lane
        const uint32_t lane_off = (uint32_t)((warp & 3) * 32) << 16;
        const float cexp = a.scale * 1.4426950408889634f;  // scores -> log2 domain (scale > 0)
        const int rt = r / G, rg = r - rt * G;
        const uint32_t s_tm0 = tmem + lane_off + Tm::s(0) + (uint32_t)x * 128;
        const uint32_t p_tm0 = tmem + lane_off + Tm::p(0) + (uint32_t)x * (kApart ? 64 : 128);
        uint32_t g = 0, done = 0;  // key tiles of the CTA; of this row tile
        bool ok = true;
        while (ok && cur.next(pc)) {
            const int n = pc.j1 - pc.j0;
            if (x == 1 && !pc.full) {
                g += n;
                continue;
            }
            const int tok0 = (pc.p * 2 + x) * tq, tok = tok0 + rt;
            const bool valid = rt < tq && tok < pc.n;
            const unsigned vmask = __ballot_sync(0xffffffffu, valid);
            const int open = pc.ctx + (a.anc ? 0 : tok0 + 1);  // keys that every row of the tile sees
            const int seen = pc.ctx + tok + 1;                 // causal: keys this row sees
            float m_used = -INFINITY, l = 0.f;
            // One key tile; masked: some row does not see all of the keys.
            auto tile = [&](auto masked_t, int tl) -> bool {
                constexpr bool masked = decltype(masked_t)::value;
                const uint32_t t = g + tl;
                const int key0 = (pc.j0 + tl) * kBN;
                uint32_t mk[4] = {};                    // the keys this row sees
                if (masked) {
                    if (a.anc) {
                        uint32_t anc[kAncWords];
#pragma unroll
                        for (int w = 0; w < kAncWords; ++w) anc[w] = valid ? a.anc[(long long)(pc.n0 + tok) * kAncWords + w] : 0u;
#pragma unroll
                        for (int ch = 0; ch < 4; ++ch) mk[ch] = tree_window(anc, key0 + ch * 32 - pc.ctx);
                    } else {
#pragma unroll
                        for (int ch = 0; ch < 4; ++ch) {
                            const int c = seen - key0 - ch * 32;
                            mk[ch] = c >= 32 ? 0xffffffffu : c <= 0 ? 0u : (1u << c) - 1u;
                        }
                    }
                }
                if (!(ok = quick_wait(&sfull[x], done & 1, s_abort, a.wait_limit))) return false;
                tc_fence_after();
                // the piece's last S has read Q: its buffer is free
                if (tl == n - 1) warp_arrive(&qfree[x]);
                if (key0 + kBN > pc.keys) {
                    // slots behind the last key hold anything, NaN too: their V rows are zeroed (by
                    // each row tile for its own product)
                    if (!(ok = quick_wait(&vfull[t % NV], (t / NV) & 1, s_abort, a.wait_limit))) return false;
                    unsigned char *sv = smem + S::kV + (t % NV) * S::kTile;
                    const int first = pc.keys - key0, count = (kBN - first) * 8;
#pragma unroll 1
                    for (int e = r; e < count * kKB; e += kBM) {
                        const int kb = e / count, c = e - kb * count;
                        *reinterpret_cast<uint4 *>(sv + kb * 16384 + first * 128 + c * 16) = make_uint4(0, 0, 0, 0);
                    }
                    fence_async_smem();
                }
                // P V of the last tile must be complete before P's columns (where they are
                // apart) are written; at D = 128 S was issued behind it
                auto wait_idle = [&]() -> bool {
                    if (!kApart || done == 0) return true;
                    if (!(ok = quick_wait(&pvdone[x], (done - 1) & 1, s_abort, a.wait_limit))) return false;
                    tc_fence_after();
                    return true;
                };
                if (vmask == 0) {  // no rows in this warp: its P feeds rows that are never read
                    if (kApart) warp_arrive(&sfree[x]);
                    // (the next S may be there already: no arrival for it before this P is used)
                    if (!wait_idle()) return false;
                    warp_arrive(&pfull[x]);
                    if (!kApart) warp_arrive(&pfull2[x]);
                    ++done;
                    return true;
                }
                const uint32_t s_tm = s_tm0, p_tm = p_tm0;
                // the row's maximum; 64 keys at a time, here and below: tensor memory is
                // read again at little cost, and the exponentials' loop, which is not
                // unrolled, stays small enough for the instruction cache
                float mx[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
                for (int hh = 0; hh < 2; ++hh) {
                    uint32_t va[32], vb[32];
                    tmem_ld32(s_tm + hh * 64, va);
                    tmem_ld32(s_tm + hh * 64 + 32, vb);
                    tmem_wait_ld();
                    tmem_regs_ready(va);
                    tmem_regs_ready(vb);
                    if (masked) {
                        hide(va, hh ? mk[2] : mk[0]);
                        hide(vb, hh ? mk[3] : mk[1]);
                    }
#pragma unroll
                    for (int e = 0; e < 32; ++e)
                        mx[e & 3] = fmaxf(mx[e & 3], fmaxf(__uint_as_float(va[e]), __uint_as_float(vb[e])));
                }
                const float mt = fmaxf(fmaxf(mx[0], mx[1]), fmaxf(mx[2], mx[3])) * cexp;
                // lazy rescale: move the reference maximum only when it grows
                // by more than 2^8 (warp-wide O pass, factor 1 for other rows)
                const bool grow = mt > m_used + 8.f;
                const float corr = grow ? ex2(m_used - mt) : 1.f;  // 0 when m_used is -inf
                if (grow) {
                    l *= corr;
                    m_used = mt;
                }
                if (tl > 0 && __any_sync(0xffffffffu, grow)) {
                    if (!wait_idle()) return false;
#pragma unroll 1
                    for (int ch = 0; ch < D / 32; ++ch) {
                        uint32_t xo[32];
                        const uint32_t o_tm = tmem + lane_off + Tm::o(x) + ch * 32;
                        tmem_ld32(o_tm, xo);
                        tmem_wait_ld();
                        tmem_regs_ready(xo);
#pragma unroll
                        for (int e = 0; e < 32; ++e) xo[e] = __float_as_uint(__uint_as_float(xo[e]) * corr);
                        tmem_st32(o_tm, xo);
                    }
                }
                const float nb = (m_used == -INFINITY) ? 0.f : kFlBias<BF16> - m_used;
                float sum4[4] = {l, 0.f, 0.f, 0.f};
#pragma unroll 1
                for (int hh = 0; hh < 2; ++hh) {
                    uint32_t va[32], vb[32], xp[32];
                    tmem_ld32(s_tm + hh * 64, va);
                    tmem_ld32(s_tm + hh * 64 + 32, vb);
                    tmem_wait_ld();
                    tmem_regs_ready(va);
                    tmem_regs_ready(vb);
                    if (masked) {
                        hide(va, hh ? mk[2] : mk[0]);
                        hide(vb, hh ? mk[3] : mk[1]);
                    }
                    if (kApart && hh) {  // S has been read: the next one may be written
                        tc_fence_before();
                        warp_arrive(&sfree[x]);
                    }
                    exp_pairs<BF16>(va, vb, cexp, nb, sum4, xp);
                    if (kApart && !hh && !wait_idle()) return false;
                    tmem_st32(p_tm + hh * 32, xp);
                    if (!kApart || hh) {
                        tmem_wait_st();
                        tc_fence_before();
                        warp_arrive(kApart || !hh ? &pfull[x] : &pfull2[x]);
                    }
                }
                l = (sum4[0] + sum4[1]) + (sum4[2] + sum4[3]);
                ++done;
                return true;
            };
            int tl = 0;
            const int n_open = min(n, open / kBN - pc.j0);
#pragma unroll 1
            for (; ok && tl < n_open; ++tl) tile(std::false_type(), tl);
#pragma unroll 1
            for (; ok && tl < n; ++tl) tile(std::true_type(), tl);
            // P V of the last tile; that of the tile before it is known to be complete (by
            // the wait above or by the order of the products), as a phase's parity demands
            if (!ok || !(ok = quick_wait(&pvdone[x], (done - 1) & 1, s_abort, a.wait_limit))) break;
            tc_fence_after();
            if (vmask) {
                const long long orow = (long long)(pc.n0 + tok) * a.Hq + pc.kvh * G + rg;
                const long long prow = (long long)pc.slot * kFlRows + x * kBM + r;
                const bool final = pc.slot < 0;
                const float f = l > 0.f ? 1.f / l : l;  // NaN stays
                // no key with weight: zeros, whatever V held or, where the row tile sees none of
                // the piece's keys, was in the columns
#pragma unroll 1
                for (int ch = 0; ch < D / 32; ++ch) {
                    uint32_t xo[32];
                    tmem_ld32(tmem + lane_off + Tm::o(0) + (uint32_t)x * D + ch * 32, xo);
                    tmem_wait_ld();
                    tmem_regs_ready(xo);
                    if (!valid) continue;
                    if (l == 0.f) {
#pragma unroll
                        for (int e = 0; e < 32; ++e) xo[e] = 0u;
                    }
                    if (final) {
                        uint32_t v[16];
#pragma unroll
                        for (int e = 0; e < 16; ++e) v[e] = pack16<BF16>(__uint_as_float(xo[2 * e]) * f, __uint_as_float(xo[2 * e + 1]) * f);
                        store32(a.out + orow * D + ch * 32, v);
                        store32(a.out + orow * D + ch * 32 + 16, v + 8);
                    } else {
#pragma unroll
                        for (int e = 0; e < 4; ++e) store32(a.part_o + prow * D + ch * 32 + 8 * e, xo + 8 * e);
                    }
                }
                if (valid && final) {
                    a.lse[orow] = l > 0.f ? (m_used - kFlBias<BF16> + log2f(l)) * 0.6931471805599453f : (l == 0.f ? -INFINITY : l);
                } else if (valid) {
                    a.part_m[prow] = m_used - kFlBias<BF16>;
                    a.part_l[prow] = l;
                }
            }
            tc_fence_before();
            warp_arrive(&ofree[x]);
            g += n;
        }
    }
    __syncthreads();
    if (warp == kFlMmaWarp) {
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
