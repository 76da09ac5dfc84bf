// coded_rows.cuh -- attention of a few rows over an 8-bit cache: single tokens,
// short chunks and trees of up to 32 rows (tokens x query heads of a group).
//
// Row r of a request (token i = r / G, query head of the group r % G) computes
//     o_r = sum_j p_rj v_j,  p_rj = exp(scale q_r.k_j - lse_r),
//     k_j = K_j 2^(ek),  v_j = V_j 2^(ev)     (codes, exponents of j's 16 slots)
// over the keys it sees, in one pass with a running maximum.  S^T = K Q^T and
// O^T = V^T P^T: keys, and then the head's columns, are the 16 rows of the tensor
// core's products and the attention's rows its 8 columns, so that a code goes from
// memory to the register that the product reads it from, as fp16, without shared
// memory tiles or shuffles (the order of D within the sums is free, and V's pairs
// of keys are two bytes of two words).  Codes are exact in fp16; the exponents go
// where they cost nothing: ek into the scores' factor, ev into the exponent of
//     P'_rj = 2^(s_rj + ev - R_r + 7),   O'_r = sum P'_rj V_j,
// with R_r a running bound of s + ev (the largest P' is 2^7 to 2^15 in fp16: weights times
// 2^ev are rounded by up to 2^-11 down to 2^-21 of the largest, by up to 2^-32 of the
// largest below that).  l_r = sum 2^(s - m_r) has
// its own bound m_r, so that it does not depend on the values' sizes.  Both move
// only when they would be exceeded by 2^8.  bf16 queries are scaled by a power of two
// per row, so that fp16 holds them (what lies 2^-39 below a row's largest is lost).
//
// Work: units are blocks of 16 keys of a request and a group of up to four KV heads;
// all units in a row are cut into equal shares, a CTA each.  A CTA's warps are its heads
// (where there are fewer than four, several warps share a head and take its blocks in
// turn), so that the heads' codes of a token, 128 bytes each and next to one another,
// are read at about the same time.  A warp has a ring of its own that TMA fills, a
// block's K and V a box each (with cp.async instead, 16 bytes a lane, an SM does not have
// enough under way: 4.7 TB/s, whatever the kernel does with the bytes).  Two blocks at a
// time: one is a chain of some 2600 cycles (copies read, eight products in a row, maxima,
// exponentials, a transpose, products), which the twelve warps of an SM do not fill.  Pieces of a cut
// (request, head) are joined in order by coded_join: the same bits every time.
//
// NaN in V of a new token is for the rows that see it, where the products give it to all of a warp's: a piece whose
// results hold NaN is done again without (a check for each block takes 3 to 7 % of short caches' calls).
//
// Bound: HBM, of 2 D bytes a key and KV head.  Measured: single tokens of 64 requests behind 1024 to 8191
// keys, 32 / 8 heads of 128, 605 MB, 111-114 us, 5.4 TB/s (107 with the copies alone; 183 from a cache in 16
// bits); of one request behind 2048 keys 13.7 us, two launches and their chains of reads.  K and V in rings of
// their own, K refilled as soon as it is in registers, took 119.
#pragma once

#include "attn_core.cuh"
#include "coded.cuh"
#include "roles.cuh"

namespace rs {

constexpr int kRowThreads = 128, kRowWarps = kRowThreads / 32;
constexpr int kRowMax = 32;        // rows of a request and KV head

struct RowsArgs {
    const uint16_t *q;
    long long q_stride;
    const int32_t *off, *parents;
    CodedPool c;
    int B, T, max_new, Hq, Hkv, G, bf16, grid;
    int most_hw;          // heads of a group at most (4, 2 or 1)
    float scale;
    long long wait_limit;
    uint16_t *out;
    float *lse;
    int32_t *status;
    // workspace
    int4 *req;            // first row, rows of its own, ctx, status (of the arguments)
    long long *cum;       // blocks before each request (of one KV head); [B]: all
    int4 *start;          // per CTA: request, group, first block, CTAs in use (0: nothing to do) and heads of a group << 24
    unsigned char *flag;  // per piece, numbered (request, group) + CTA: status bits
    float *part_o, *part_lse;  // two slots a CTA: the piece that it goes on with, the one that it begins
};

// What is wrong with request b's rows and keys; rq: first row, rows of its own, ctx.
__device__ __forceinline__ int rows_check(const RowsArgs &a, int b, int latest, int4 &rq) {
    const int n0 = a.off[b], n1 = a.off[b + 1], ctx = a.c.ctx[b];
    rq = make_int4(0, 0, 0, 0);
    if (n0 < 0 || n1 < n0 || n1 > a.T || n0 < latest) return RS_ST_BAD_OFFSET;
    rq = make_int4(n0, n1 - n0, ctx, 0);
    if (ctx < 0 || (long long)ctx + (n1 - n0) > ((long long)a.c.max_pages << a.c.page_log2)) return RS_ST_BAD_OFFSET;
    return n1 - n0 > a.max_new ? RS_ST_TOO_LARGE : 0;
}
__device__ __forceinline__ int rows_blocks(const int4 &rq, int st) {
    return st || rq.y == 0 ? 0 : (int)(((long long)rq.z + rq.y + kCodeBlock - 1) / kCodeBlock);
}
// the CTA whose share holds unit x (of W, shares [W c / n, W (c + 1) / n))
__device__ __forceinline__ int owner(long long x, long long W, int n) { return (int)(((x + 1) * n - 1) / W); }

// Where a CTA's share begins, and the walk over its pieces.
struct RowsWalk {
    int b, h, j, nb;      // request, group, block; blocks of the request
    int latest;           // largest first row of the requests so far
    int4 rq;
    long long left;       // units of the share that are left
};

__device__ __forceinline__ long long warp_prefix(long long v) {
    for (int o = 1; o < 32; o <<= 1) {
        const long long y = __shfl_up_sync(0xffffffffu, v, o);
        if ((int)(threadIdx.x & 31) >= o) v += y;
    }
    return v;
}

// The whole block: every thread counts the units of a run of requests; the one whose
// run holds the share's start finds it.  CTA 0 writes the requests' records.
__device__ __forceinline__ RowsWalk rows_plan(const RowsArgs &a, int &used, int &hw) {
    __shared__ long long s_sum[kRowWarps];
    __shared__ int s_late[kRowWarps], s_live;  // s_live: requests with keys
    __shared__ RowsWalk s_walk;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int each = (a.B + kRowThreads - 1) / kRowThreads;
    if (tid == 0) s_live = 0;
    const int b0 = min(tid * each, a.B), b1 = min(b0 + each, a.B);
    int late = INT_MIN;
    for (int b = b0; b < b1; ++b) late = max(late, a.off[b]);
    // largest first row before this thread's requests
    int x = late;
    for (int o = 1; o < 32; o <<= 1) {
        const int y = __shfl_up_sync(0xffffffffu, x, o);
        if (lane >= o) x = max(x, y);
    }
    if (lane == 31) s_late[warp] = x;
    x = __shfl_up_sync(0xffffffffu, x, 1);
    if (lane == 0) x = INT_MIN;
    __syncthreads();
    for (int w = 0; w < warp; ++w) x = max(x, s_late[w]);
    const int before = x;
    long long mine = 0;
    int live = 0;
    for (int b = b0; b < b1; ++b) {
        int4 rq;
        const int st = rows_check(a, b, x, rq);
        const int nb = rows_blocks(rq, st);
        mine += nb;
        live += nb > 0;
        x = max(x, a.off[b]);
    }
    live = __reduce_add_sync(0xffffffffu, live);
    if (lane == 0 && live) atomicAdd(&s_live, live);
    const long long incl = warp_prefix(mine);
    if (lane == 31) s_sum[warp] = incl;
    __syncthreads();
    long long first = incl - mine, total = 0;
    for (int w = 0; w < kRowWarps; ++w) {
        if (w < warp) first += s_sum[w];
        total += s_sum[w];
    }
    // Heads side by side read HBM better, warps side by side at one head leave fewer pieces to
    // join: the first where every warp has 16 blocks and more, and where requests are so short (four
    // blocks on average) that a head leaves most warps without any
    hw = total * a.Hkv >= 16ll * kRowWarps * a.grid || total <= 4ll * s_live ? a.most_hw : 1;
    const int groups = a.Hkv / hw;
    const long long W = total * groups;
    // shares of at least two steps a warp: shorter ones cost more to join than they save; but a share a
    // segment, as many as there are CTAs for, since a segment's own cost is that of many blocks (25 requests of
    // up to 4 tokens, 16 heads, no cache: 106 us with 25 CTAs).  With few segments a whole number of shares
    // each, at least one: a CTA has one piece then (of requests of one length)
    const int least = 4 * kRowWarps / hw;
    const long long segments = (long long)s_live * groups;
    const long long fit = min(max((W + least - 1) / least, segments), (long long)a.grid);
    used = (int)(2 * segments > a.grid ? fit : segments * max(fit / max(segments, 1ll), 1ll));
    const int c = blockIdx.x;
    const long long lo = c < used ? W * c / used : 0, hi = c < used ? W * (c + 1) / used : 0;
    if (c == 0 || (c < used && lo >= first * groups && lo < (first + mine) * groups)) {
        long long at = first;
        int l = before;
        for (int b = b0; b < b1; ++b) {
            int4 rq;
            const int st = rows_check(a, b, l, rq);
            const int nb = rows_blocks(rq, st);
            l = max(l, a.off[b]);
            if (c == 0) {
                a.req[b] = make_int4(rq.x, rq.y, rq.z, st);
                a.cum[b] = at;
            }
            if (c < used && lo >= at * groups && lo < (at + nb) * groups) {
                const long long in = lo - at * groups;
                s_walk = RowsWalk{b, (int)(in / nb), (int)(in % nb), nb, l, rq, hi - lo};
            }
            at += nb;
        }
    }
    if (c == 0 && tid == 0) a.cum[a.B] = total;
    __syncthreads();
    RowsWalk w{};
    if (c < used) w = s_walk;
    if (tid == 0) a.start[c] = make_int4(w.b, w.h, w.j, used | hw << 24);
    return w;
}
// behind a piece of `done` units: the next one
__device__ __forceinline__ void rows_next(const RowsArgs &a, RowsWalk &w, int done, int groups) {
    w.left -= done;
    if (w.left <= 0) return;
    w.j = 0;
    if (++w.h < groups) return;
    w.h = 0;
    do {
        ++w.b;
        const int st = rows_check(a, w.b, w.latest, w.rq);
        w.nb = rows_blocks(w.rq, st);
        w.latest = max(w.latest, a.off[w.b]);
    } while (w.nb == 0);
}

__device__ __forceinline__ void mma_f16(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                 : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
// an 8 x 8 matrix of 16-bit values transposed across the warp
__device__ __forceinline__ uint32_t transpose8(uint32_t x) {
    uint32_t y;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
    return y;
}
__device__ __forceinline__ uint32_t half2_of(float lo, float hi) {
    uint32_t r;
    asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}
__device__ __forceinline__ float2 float2_of(uint32_t x, bool bf16) {
    if (bf16) return make_float2(__uint_as_float(x << 16), __uint_as_float(x & 0xffff0000u));
    return __half22float2(*reinterpret_cast<const __half2 *>(&x));
}
__device__ __forceinline__ uint32_t pair_of(float lo, float hi, bool bf16) {
    uint32_t r;
    if (!bf16) return half2_of(lo, hi);
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}

template <int D, int NT>
struct RowsShape {
    static constexpr int kKLoads = D == 128 ? 4 : 2;  // words of a block's K that a lane reads
    static constexpr int kBlocks = NT == 4 ? 1 : 2;        // blocks of a step (four tiles of O fill the registers)
    static constexpr int kStages = (D == 128 ? 4 : 8) / kBlocks;
    static constexpr int kBlockBytes = 32 * D;             // 16 keys, K and V
    static constexpr int kStageBytes = kBlocks * kBlockBytes;  // of a warp
    static constexpr int kRing = kRowWarps * kStages * kStageBytes;
    static constexpr int kRows = 8 * NT;
    static constexpr int kRowStride = D + 4;               // floats, of a warp's O in shared memory
    static constexpr int kMerge = kRowWarps * kRows * (kRowStride + 1) * 4;
    static constexpr int kBytes = (kRing > kMerge ? kRing : kMerge) + 1024;  // the base is rounded up to 1 KB
    static constexpr int kPerSm = NT == 1 ? 3 : 2;
};

template <int D, int NT, bool TREE>
__global__ void __launch_bounds__(kRowThreads, RowsShape<D, NT>::kPerSm)
coded_rows(RowsArgs a, const __grid_constant__ CUtensorMap tmk, const __grid_constant__ CUtensorMap tmv) {
    using Sh = RowsShape<D, NT>;
    constexpr int kS = Sh::kStages, kBl = Sh::kBlocks, kSteps = D / 16, kTiles = D / 16;  // k-steps of K Q^T, 16-column tiles of O^T
    extern __shared__ unsigned char smem_raw[];
    // (an offset and not a rounded address, which would make all loads generic ones)
    unsigned char *smem = smem_raw + (-sm100::smem_u32(smem_raw) & 1023u);
    __shared__ uint64_t s_full[kRowWarps][kS];
    __shared__ int s_gave_up;
    __shared__ uint32_t s_anc[32];  // a tree's ancestor sets
    volatile int *s_abort = &s_gave_up;
    if (threadIdx.x == 0) {
        for (int i = 0; i < kRowWarps * kS; ++i) sm100::mbar_init(&s_full[0][0] + i, 1);
        s_gave_up = 0;
        sm100::fence_mbar_init();
        sm100::prefetch_tmap(&tmk);
        sm100::prefetch_tmap(&tmv);
    }
    // the joining kernel is let in at the end: its blocks, waiting beside these, cost 64 single
    // tokens 27 us of 138
    pdl_wait_prev();
    int used, hw;
    RowsWalk w = rows_plan(a, used, hw);
    const int groups = a.Hkv / hw;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int g = lane >> 2, t = lane & 3;
    unsigned char *ring = smem + warp * kS * Sh::kStageBytes;
    const float cexp = fminf(a.scale * 1.4426950408889634f, 3.402823466e38f);
    const bool bf16 = a.bf16;
    const int head = warp % hw, kw = warp / hw, KW = kRowWarps / hw;  // head of the group; the warp's place among the head's
    uint32_t filled = 0, drained = 0;  // stages of this warp's ring, over all pieces
    bool begun = false;
    // NaN in V of a key that some row does not see reaches all rows by the product's 0 x NaN.  A piece with such keys
    // whose results hold NaN is done again with 0 in its place, and the rows that see the key get it at the end.
    bool clean = false;
    while (w.left > 0) {
        const int b = w.b, h = w.h * hw + head, j0 = w.j, nb = w.nb;
        const int j1 = (int)min((long long)nb, j0 + w.left);
        const int n0 = w.rq.x, n = w.rq.y, ctx = w.rq.z, R = n * a.G, keys = ctx + n;
        int flag = 0;
        float o[NT][kTiles][4], m[NT][2], l[NT][2], ref[NT][2];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
            for (int i = 0; i < kTiles; ++i)
#pragma unroll
                for (int e = 0; e < 4; ++e) o[nt][i][e] = 0.f;
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                m[nt][e] = ref[nt][e] = -INFINITY;
                l[nt][e] = 0.f;
            }
        }

        // This warp's steps: blocks j0 + kBl kw .., KW kBl apart.  Lane x looks up the x-th block of
        // 32: its number in the pool and its exponents, 32 blocks ahead.
        constexpr int kBatch = 32 / kBl;  // steps
        const int steps_all = (j1 - j0 + kBl - 1) / kBl, mine = steps_all > kw ? (steps_all - kw + KW - 1) / KW : 0;
        const int32_t *table = a.c.table + (long long)b * a.c.max_pages;
        const int in_page = (1 << (a.c.page_log2 - kCodeBlockLog2)) - 1;
        auto block_at = [&](int bat) { return j0 + kBl * (kw + KW * (bat * kBatch + lane / kBl)) + lane % kBl; };
        auto page_of = [&](int bat) -> int {
            const int j = block_at(bat);
            return j < j1 ? table[j >> (a.c.page_log2 - kCodeBlockLog2)] : 0;
        };
        auto block_of = [&](int bat, int id) -> int {  // -1: not this CTA's, or a bad page
            const int j = block_at(bat);
            if (j >= j1) return -1;
            if (id < 0 || id >= a.c.n_pages) {
                flag |= RS_ST_BAD_PAGE;
                return -1;
            }
            return (id << (a.c.page_log2 - kCodeBlockLog2)) + (j & in_page);
        };
        auto exps_of = [&](int blk) -> int {  // (ek, ev) as two bytes
            if (blk < 0) return 0;
            const long long at = (long long)blk * a.Hkv + h;
            return (int)(uint8_t)a.c.ke[at] | (int)(uint8_t)a.c.ve[at] << 8;
        };
        // the ring's words, as the boxes are swizzled: 16-byte word c of row r
        auto word = [&](int r, int c) { return D == 128 ? r * 128 + ((c ^ (r & 7)) * 16) : r * 64 + ((c ^ (r >> 1 & 3)) * 16); };
        int blk = -1, exps = 0, blk_next = -1, exps_next = 0, id_next = 0;
        // copies step it (of this warp) into its stage; cur: the batch of blk
        auto issue = [&](int it, int cur) {
            if (it >= mine) return;
            int at[kBl], n_at = 0;
#pragma unroll
            for (int u = 0; u < kBl; ++u) {
                at[u] = __shfl_sync(0xffffffffu, it / kBatch == cur ? blk : blk_next, it % kBatch * kBl + u);
                n_at += at[u] >= 0;
            }
            if (lane == 0) {
                uint64_t *bar = &s_full[warp][filled % kS];
                unsigned char *dst = ring + filled % kS * Sh::kStageBytes;
                sm100::mbar_expect_tx(bar, (uint32_t)(n_at * Sh::kBlockBytes));
#pragma unroll
                for (int u = 0; u < kBl; ++u)
                    if (at[u] >= 0) {
                        sm100::tma_load_3d(dst + u * Sh::kBlockBytes, &tmk, bar, 0, h, at[u] * kCodeBlock);
                        sm100::tma_load_3d(dst + u * Sh::kBlockBytes + kCodeBlock * D, &tmv, bar, 0, h, at[u] * kCodeBlock);
                    }
            }
            __syncwarp();
            ++filled;
        };
        if (mine > 0) {
            blk = block_of(0, page_of(0));
            for (int it = 0; it < kS; ++it) issue(it, 0);
            exps = exps_of(blk);
        }
        uint32_t anc = 0;  // lane i: node i's ancestors and itself
        if (TREE) {
            const int pa = lane < n ? a.parents[n0 + lane] : -1;
            const bool bad = lane < n && (lane == 0 ? pa != -1 : pa < 0 || pa >= lane);
            if (__any_sync(0xffffffffu, bad)) {
                flag |= RS_ST_BAD_TREE;
            } else {
                int x = lane < n ? lane : -1;
                while (__any_sync(0xffffffffu, x >= 0)) {
                    if (x >= 0) anc |= 1u << x;
                    const int up = __shfl_sync(0xffffffffu, pa, max(x, 0));
                    x = x >= 0 ? up : -1;
                }
            }
        }
        if (TREE && warp == 0) s_anc[lane] = anc;
        // the queries, as the product's second operand: row nt 8 + g; this lane's columns are
        // those of the codes that it reads
        uint32_t qf[NT][kSteps][2];
        float factor[NT][2];   // scores -> log2 domain, rows nt 8 + 2 t (+ 1)
        int limit[NT][2];      // keys that the row sees (causal)
        uint32_t see[NT][2];   // its ancestors (tree)
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            const int r = nt * 8 + g;
            uint4 x[D / 32];   // 16 columns at 16 t of each 64
#pragma unroll
            for (int u = 0; u < D / 32; ++u) x[u] = make_uint4(0, 0, 0, 0);
            if (r < R) {
                const int i = r / a.G;
                const uint4 *src = reinterpret_cast<const uint4 *>(a.q + (n0 + i) * a.q_stride + (long long)(h * a.G + r - i * a.G) * D);
#pragma unroll
                for (int u = 0; u < D / 64; ++u) {
                    x[2 * u] = src[8 * u + 2 * t];
                    x[2 * u + 1] = src[8 * u + 2 * t + 1];
                }
            }
            int shift = 0;
            if (bf16) {
                uint32_t most = 0;
#pragma unroll
                for (int u = 0; u < D / 32; ++u) {
                    const uint32_t v[4] = {x[u].x, x[u].y, x[u].z, x[u].w};
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const uint32_t lo = (v[e] << 16) & 0x7fffffffu, hi = v[e] & 0x7fff0000u;
                        most = max(most, max(lo < 0x7f800000u ? lo : 0u, hi < 0x7f800000u ? hi : 0u));
                    }
                }
                most = max(most, __shfl_xor_sync(0xffffffffu, most, 1));
                most = max(most, __shfl_xor_sync(0xffffffffu, most, 2));
                shift = most ? max((int)(most >> 23) - 127 - 14, -112) : 0;
            }
            const float down = pow2i(-shift);
#pragma unroll
            for (int s = 0; s < kSteps; ++s) {  // 4 columns of this lane: word s % 4 of its 16
                const uint4 &v = x[s / 2];
                const uint32_t v0 = s & 1 ? v.z : v.x, v1 = s & 1 ? v.w : v.y;
                if (bf16) {
                    const float2 p = float2_of(v0, true), q = float2_of(v1, true);
                    qf[nt][s][0] = half2_of(p.x * down, p.y * down);
                    qf[nt][s][1] = half2_of(q.x * down, q.y * down);
                } else {
                    qf[nt][s][0] = v0;
                    qf[nt][s][1] = v1;
                }
            }
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const int row = nt * 8 + 2 * t + e, i = row / a.G;
                factor[nt][e] = finite_mul(cexp, pow2i(__shfl_sync(0xffffffffu, shift, (2 * t + e) * 4)));
                limit[nt][e] = row < R ? ctx + i + 1 : 0;
                see[nt][e] = TREE ? __shfl_sync(0xffffffffu, anc, min(i, 31)) : 0;
                if (row >= R) see[nt][e] = 0;
            }
        }
        const int open = TREE ? ctx : ctx + 1;  // keys that every row sees

        if (!(flag & RS_ST_BAD_TREE)) {  // (else nothing is computed: the request's rows are emptied)
#pragma unroll 1
            for (int it = 0; it < mine && !(flag & RS_ST_TIMEOUT);) {  // (two loops: what is rare stays out of the inner one)
                const int stop = clean ? it + 1 : mine;
                const int hidden = j0 + kBl * (kw + KW * it);  // the step's first block
                if (clean && (hidden + kBl) * kCodeBlock > open) {
                    unsigned char *v = ring + drained % kS * Sh::kStageBytes + kCodeBlock * D;
                    if (!quick_wait(&s_full[warp][drained % kS], drained / kS & 1, s_abort, a.wait_limit)) {
                        flag |= RS_ST_TIMEOUT;
                        break;
                    }
#pragma unroll 1
                    for (int u = 0; u < kBl; ++u, v += Sh::kBlockBytes)
                        if ((hidden + u + 1) * kCodeBlock > open)
                            for (int i = lane; i < D; i += 32) {  // 16-byte words of the block's V
                                uint4 *p = reinterpret_cast<uint4 *>(v) + i;
                                *p = make_uint4(without_nan(p->x), without_nan(p->y), without_nan(p->z), without_nan(p->w));
                            }
                    sm100::fence_async_smem();  // (the stage is copied to again)
                    __syncwarp();
                }
#pragma unroll 1
                for (; it < stop; ++it) {
                    const int cur = it / kBatch;
                    // the lookups of the next batch, a step at a time
                    if (it % kBatch == 2) id_next = page_of(cur + 1);
                    if (it % kBatch == 5) {
                        blk_next = block_of(cur + 1, id_next);
                        exps_next = exps_of(blk_next);
                    }
                    if (!quick_wait(&s_full[warp][drained % kS], drained / kS & 1, s_abort, a.wait_limit)) {
                        flag |= RS_ST_TIMEOUT;
                        break;
                    }
                    const unsigned char *src = ring + drained % kS * Sh::kStageBytes;
                    ++drained;
                    const int block0 = j0 + kBl * (kw + KW * it), key0 = block0 * kCodeBlock;
                    float s[kBl][NT][4], evf[kBl], two_ek[kBl];
#pragma unroll
                    for (int u = 0; u < kBl; ++u) {
                        const int e2 = __shfl_sync(0xffffffffu, exps, it % kBatch * kBl + u);
                        two_ek[u] = pow2i(code_exp((int)(int8_t)(e2 & 255), bf16));
                        evf[u] = (float)code_exp((int)(int8_t)(e2 >> 8), bf16);
                    }
                    // S^T: keys g and g + 8 of a block, rows 2 t and 2 t + 1 of every tile; even and odd
                    // steps are summed apart
                    uint4 kc[kBl][Sh::kKLoads];
#pragma unroll
                    for (int u = 0; u < kBl; ++u)
#pragma unroll
                        for (int i = 0; i < Sh::kKLoads; ++i)
                            kc[u][i] = *reinterpret_cast<const uint4 *>(src + u * Sh::kBlockBytes + word(i / (D / 64) * 8 + g, i % (D / 64) * 4 + t));
                    float s1[kBl][NT][4];
#pragma unroll
                    for (int u = 0; u < kBl; ++u)
#pragma unroll
                        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                            for (int e = 0; e < 4; ++e) s[u][nt][e] = s1[u][nt][e] = 0.f;
#pragma unroll
                    for (int k = 0; k < kSteps; ++k)
#pragma unroll
                        for (int u = 0; u < kBl; ++u) {
                            const uint4 &x = kc[u][k / 4], &y = kc[u][D / 64 + k / 4];
                            const uint32_t wx = (k & 3) == 0 ? x.x : (k & 3) == 1 ? x.y : (k & 3) == 2 ? x.z : x.w;
                            const uint32_t wy = (k & 3) == 0 ? y.x : (k & 3) == 1 ? y.y : (k & 3) == 2 ? y.z : y.w;
                            uint32_t a0, a1, a2, a3;
                            decode4(wx, a0, a2);
                            decode4(wy, a1, a3);
#pragma unroll
                            for (int nt = 0; nt < NT; ++nt) mma_f16(NT < 4 && (k & 1) ? s1[u][nt] : s[u][nt], a0, a1, a2, a3, qf[nt][k][0], qf[nt][k][1]);
                        }
                    const bool masked = key0 + kBl * kCodeBlock > open || block0 + kBl > j1;
                    bool grow = false;
#pragma unroll
                    for (int u = 0; u < kBl; ++u)
#pragma unroll
                        for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
                            for (int e = 0; e < 4; ++e) s[u][nt][e] = (NT < 4 ? s[u][nt][e] + s1[u][nt][e] : s[u][nt][e]) * finite_mul(factor[nt][e & 1], two_ek[u]);
                            if (masked) {
#pragma unroll
                                for (int e = 0; e < 4; ++e) {
                                    const int key = key0 + u * kCodeBlock + g + (e >> 1) * 8, node = key - ctx;
                                    const bool on = TREE ? node < 0 || (node < 32 && ((see[nt][e & 1] >> node) & 1u)) : key < limit[nt][e & 1];
                                    if (!on || block0 + u >= j1) s[u][nt][e] = -INFINITY;
                                }
                            }
#pragma unroll
                            for (int e = 0; e < 2; ++e) {
                                const float x = fmaxf(s[u][nt][e], s[u][nt][e + 2]);
                                grow |= x > m[nt][e] + 8.f || x + evf[u] > ref[nt][e] + 8.f;
                            }
                        }
                    if (__any_sync(0xffffffffu, grow)) {
#pragma unroll
                        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                            for (int e = 0; e < 2; ++e) {
                                float x = -INFINITY, y = -INFINITY;  // the largest score, and with its block's ev
#pragma unroll
                                for (int u = 0; u < kBl; ++u) {
                                    const float z = fmaxf(s[u][nt][e], s[u][nt][e + 2]);
                                    x = fmaxf(x, z);
                                    y = fmaxf(y, z + evf[u]);
                                }
#pragma unroll
                                for (int d = 4; d < 32; d *= 2) {
                                    x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, d));
                                    y = fmaxf(y, __shfl_xor_sync(0xffffffffu, y, d));
                                }
                                if (x > m[nt][e] + 8.f) {
                                    l[nt][e] *= sm100::ex2(m[nt][e] - x);
                                    m[nt][e] = x;
                                }
                                if (y > ref[nt][e] + 8.f) {
                                    const float f = sm100::ex2(ref[nt][e] - y);
                                    ref[nt][e] = y;
#pragma unroll
                                    for (int i = 0; i < kTiles; ++i) {
                                        o[nt][i][e] *= f;
                                        o[nt][i][e + 2] *= f;
                                    }
                                }
                            }
                    }
#pragma unroll
                    for (int u = 0; u < kBl; ++u) {
                        uint32_t pb[NT][2];  // P'^T as the product's second operand
#pragma unroll
                        for (int nt = 0; nt < NT; ++nt) {
                            float p[4];
#pragma unroll
                            for (int e = 0; e < 2; ++e) {
                                const float nm = m[nt][e] == -INFINITY ? 0.f : m[nt][e];
                                const float nr = ref[nt][e] == -INFINITY ? 0.f : evf[u] + 7.f - ref[nt][e];
                                l[nt][e] += sm100::ex2(s[u][nt][e] - nm) + sm100::ex2(s[u][nt][e + 2] - nm);
                                p[e] = sm100::ex2(s[u][nt][e] + nr);
                                p[e + 2] = sm100::ex2(s[u][nt][e + 2] + nr);
                            }
                            pb[nt][0] = transpose8(half2_of(p[0], p[1]));
                            pb[nt][1] = transpose8(half2_of(p[2], p[3]));
                        }
                        uint32_t vc[4][D / 32];
#pragma unroll
                        for (int y = 0; y < 4; ++y) {
                            const int key = 2 * t + (y & 1) + 8 * (y >> 1);
                            const unsigned char *q = src + u * Sh::kBlockBytes + kCodeBlock * D +
                                                     (D == 128 ? word(key, g) : word(key, g >> 1) + (g & 1) * 8);
                            if constexpr (D == 128) {
                                const uint4 x = *reinterpret_cast<const uint4 *>(q);
                                vc[y][0] = x.x, vc[y][1] = x.y, vc[y][2] = x.z, vc[y][3] = x.w;
                            } else {
                                const uint2 x = *reinterpret_cast<const uint2 *>(q);
                                vc[y][0] = x.x, vc[y][1] = x.y;
                            }
                        }
                        if (key0 + (u + 1) * kCodeBlock > keys || block0 + u >= j1) {  // slots behind the last key hold anything
#pragma unroll
                            for (int y = 0; y < 4; ++y)
                                if (block0 + u >= j1 || key0 + u * kCodeBlock + 2 * t + (y & 1) + 8 * (y >> 1) >= keys) {
#pragma unroll
                                    for (int i = 0; i < D / 32; ++i) vc[y][i] = 0;
                                }
                        }
                        // O^T: columns D / 8 g + 2 i (+ 1) of tile i
#pragma unroll
                        for (int i = 0; i < kTiles; ++i) {
                            const uint32_t pick = i & 1 ? 0x7362u : 0x5140u;
                            uint32_t a0, a1, a2, a3;
                            decode4(__byte_perm(vc[0][i / 2], vc[1][i / 2], pick), a0, a1);
                            decode4(__byte_perm(vc[2][i / 2], vc[3][i / 2], pick), a2, a3);
#pragma unroll
                            for (int nt = 0; nt < NT; ++nt) mma_f16(o[nt][i], a0, a1, a2, a3, pb[nt][0], pb[nt][1]);
                        }
                    }
                    __syncwarp();  // all have read the stage
                    issue(it + kS, cur);
                    if (it % kBatch == kBatch - 1) {
                        blk = blk_next;
                        exps = exps_next;
                    }
                }
            }
        }
        for (; drained < filled; ++drained) {  // given up: what is on its way lands first
            volatile int no_abort = 0;
            sm100::mbar_wait(&s_full[warp][drained % kS], drained / kS & 1, &no_abort, kWaitLimit);
        }
        flag = __reduce_or_sync(0xffffffffu, flag);

        // The warps' results are joined: each one's O / l and log2 sum.
        __syncthreads();  // the ring is free
        float *s_o = reinterpret_cast<float *>(smem) + warp * Sh::kRows * Sh::kRowStride;
        float *s_lse = reinterpret_cast<float *>(smem) + kRowWarps * Sh::kRows * Sh::kRowStride;
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                float x = l[nt][e];
                x += __shfl_xor_sync(0xffffffffu, x, 4);
                x += __shfl_xor_sync(0xffffffffu, x, 8);
                x += __shfl_xor_sync(0xffffffffu, x, 16);
                const int row = nt * 8 + 2 * t + e;
                // l >= 1 where there is a weight (the one that set m): the quotient stays finite.  Where V's exponents are
                // the smallest, the power is below fp32's normal numbers: 2^64 of it then goes to the product
                const float up = ref[nt][e] - 7.f - m[nt][e];
                const bool small = up < -60.f;
                const float f = x == 0.f ? 0.f : sm100::ex2(small ? up + 64.f : up) / x, f2 = small ? 0x1p-64f : 1.f;
                if (g == 0) s_lse[warp * Sh::kRows + row] = x == 0.f ? -INFINITY : m[nt][e] + log2f(x);
                float *dst = s_o + row * Sh::kRowStride + D / 8 * g;
#pragma unroll
                for (int i = 0; i < kTiles; ++i) {
                    // 0 x NaN of a row without weights
                    *reinterpret_cast<float2 *>(dst + 2 * i) =
                        x == 0.f ? make_float2(0.f, 0.f) : make_float2(o[nt][i][e] * f * f2, o[nt][i][e + 2] * f * f2);
                }
            }
        __shared__ int s_flag;
        if (tid == 0) s_flag = 0;
        __syncthreads();
        if (lane == 0 && flag) atomicOr(&s_flag, flag);
        const bool final = j0 == 0 && j1 == nb;
        const int slot = 2 * blockIdx.x + (j0 == 0 ? 1 : 0);
        const float *all = reinterpret_cast<const float *>(smem);
        bool nan = false;
        for (int i = tid; i < hw * R * (D / 4); i += kRowThreads) {
            const int hr = i / (D / 4), col = i % (D / 4) * 4, hx = hr / R, row = hr - hx * R;  // head of the group, row
            float top = -INFINITY;
            for (int x = hx; x < kRowWarps; x += hw) top = fmaxf(top, s_lse[x * Sh::kRows + row]);
            float sum = 0.f;
            float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
            for (int x = hx; x < kRowWarps; x += hw) {
                const float z = s_lse[x * Sh::kRows + row];
                if (z == -INFINITY) continue;
                const float p = sm100::ex2(z - top);
                const float4 y = *reinterpret_cast<const float4 *>(all + (x * Sh::kRows + row) * Sh::kRowStride + col);
                sum += p;
                v.x = fmaf(p, y.x, v.x);
                v.y = fmaf(p, y.y, v.y);
                v.z = fmaf(p, y.z, v.z);
                v.w = fmaf(p, y.w, v.w);
            }
            const float f = sum == 0.f ? 0.f : 1.f / sum, z2 = sum == 0.f ? -INFINITY : top + log2f(sum);
            v = make_float4(v.x * f, v.y * f, v.z * f, v.w * f);
            const float any = (v.x + v.y) + (v.z + v.w);
            nan |= any != any;
            if (final) {
                const int tok = row / a.G;
                const long long orow = (long long)(n0 + tok) * a.Hq + (w.h * hw + hx) * a.G + (row - tok * a.G);
                *reinterpret_cast<uint2 *>(a.out + orow * D + col) = make_uint2(pair_of(v.x, v.y, bf16), pair_of(v.z, v.w, bf16));
                if (col == 0) a.lse[orow] = z2 * 0.6931471805599453f;
            } else {
                *reinterpret_cast<float4 *>(a.part_o + ((long long)(slot * hw + hx) * Sh::kRows + row) * D + col) = v;
                if (col == 0) a.part_lse[(slot * hw + hx) * Sh::kRows + row] = z2;
            }
        }
        if (clean) {  // over what this thread has just stored
#pragma unroll 1
            for (int i = tid; i < hw * R * (D / 4); i += kRowThreads) {
                const int hr = i / (D / 4), col = i % (D / 4) * 4, hx = hr / R, row = hr - hx * R, tok = row / a.G;
                const int last = min(TREE ? keys : ctx + tok + 1, j1 * kCodeBlock);
                uint32_t at = 0;
#pragma unroll 1
                for (int key = max(open, j0 * kCodeBlock) & -kCodeBlock; key < last; ++key) {  // (from the first block that was changed)
                    if (TREE && key >= ctx && !(s_anc[tok] >> (key - ctx) & 1u)) continue;
                    const int id = table[key >> a.c.page_log2];
                    if (id < 0 || id >= a.c.n_pages) continue;  // (the request is rejected)
                    const long long slot = ((long long)id << a.c.page_log2) + (key & ((1 << a.c.page_log2) - 1));
                    at |= nan_codes(*reinterpret_cast<const uint32_t *>(a.c.v + (slot * a.Hkv + w.h * hw + hx) * D + col));
                }
                const long long orow = (long long)(n0 + tok) * a.Hq + (w.h * hw + hx) * a.G + (row - tok * a.G);
#pragma unroll 1
                for (int e = 0; e < 4; ++e, at >>= 8)
                    if (at & 0x80u) {
                        if (final) a.out[orow * D + col + e] = 0x7fff;
                        else a.part_o[((long long)(slot * hw + hx) * Sh::kRows + row) * D + col + e] = NAN;
                    }
            }
        }
        sm100::fence_async_smem();  // the ring is copied to again
        if (__syncthreads_or(nan && !clean && open < keys && j1 * kCodeBlock > open)) {
            clean = true;
            continue;
        }
        clean = false;
        if (tid == 0) {
            const long long piece = (long long)b * groups + w.h + blockIdx.x;
            a.flag[piece] = (unsigned char)s_flag;
            if (!begun && j0 == 0 && blockIdx.x > 0) a.flag[piece - 1] = 0;  // a number that no piece has
        }
        begun = true;
        rows_next(a, w, j1 - j0, groups);
    }
    pdl_launch_next();
}

// Joins the pieces of the segments that the shares' ends cut (the blocks of the share
// that holds a segment's second piece, as many as give a warp a row: one request's pieces
// have few such shares), a row to a warp, lanes the pieces' sums first
// and then the columns; empties the rows of rejected requests; writes the statuses.
template <int D>
__global__ void __launch_bounds__(kRowThreads)
coded_join(RowsArgs a, int row_tiles) {
    pdl_wait_prev();
    pdl_launch_next();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int4 at = a.start[min((int)blockIdx.x + 1, a.grid - 1)];
    const int hw = at.w >> 24, used = at.w & 0xffffff, groups = a.Hkv / hw;
    const long long total = a.cum[a.B], W = total * groups;
    // the flags of request b's pieces, whose units are [lo, hi) (whole warp)
    auto flags_of = [&](int b, long long lo, long long hi) -> int {
        int bits = 0;
        if (hi > lo) {
            const long long first = (long long)b * groups + owner(lo, W, used), last = (long long)(b + 1) * groups - 1 + owner(hi - 1, W, used);
            for (long long i = first + lane; i <= last; i += 32) bits |= a.flag[i];
        }
        return (int)__reduce_or_sync(0xffffffffu, bits);
    };
    const int blocks = gridDim.x * gridDim.y;
    // (the last blocks first: those with pieces to join are at the front)
    for (int b = (blocks - 1 - (int)(blockIdx.y * gridDim.x + blockIdx.x)) * kRowWarps + warp; b < a.B; b += blocks * kRowWarps) {
        const int4 rq = a.req[b];
        const int st = rq.w | flags_of(b, a.cum[b] * groups, a.cum[b + 1] * groups);
        if (lane == 0) a.status[b] = st;
        if (!st) continue;
        const long long rows = (long long)rq.y * a.Hq;  // none where another request may have them
        uint4 *o = reinterpret_cast<uint4 *>(a.out + (long long)rq.x * a.Hq * D);
        for (long long i = lane; i < rows * (D / 8); i += 32) o[i] = make_uint4(0, 0, 0, 0);
        for (long long i = lane; i < rows; i += 32) a.lse[(long long)rq.x * a.Hq + i] = 0.f;
    }
    const int c = blockIdx.x + 1;
    if (c >= used) return;
    if (at.z == 0) return;  // it begins with a segment
    const int4 rq = a.req[at.x];
    const long long nb = a.cum[at.x + 1] - a.cum[at.x];
    const long long x0 = a.cum[at.x] * groups + at.y * nb;
    const int c0 = owner(x0, W, used), c1 = owner(x0 + nb - 1, W, used);
    if (c0 != c - 1) return;  // not the second piece
    const bool bad = rq.w != 0 || flags_of(at.x, x0 - at.y * nb, x0 + (groups - at.y) * nb) != 0;
    const int pieces = c1 - c0 + 1, rows = 8 * row_tiles;
    constexpr int kC = D / 32;  // columns of a lane
    const int R = rq.y * a.G;
    for (int hr = blockIdx.y * kRowWarps + warp; hr < hw * R; hr += gridDim.y * kRowWarps) {
        const int hx = hr / R, row = hr - hx * R;  // head of the group, row
        float top = -INFINITY, sum = 0.f, acc[kC] = {};
        for (int p0 = 0; p0 < pieces; p0 += 32) {
            const int cnt = min(pieces - p0, 32);
            auto slot = [&](int p) { return 2 * (c0 + p) + (p == 0 ? 1 : 0); };
            const float z = lane < cnt ? a.part_lse[(slot(p0 + lane) * hw + hx) * rows + row] : -INFINITY;
            const float next = fmaxf(top, warp_max(z));
            const float old = next == -INFINITY ? 1.f : sm100::ex2(top - next);
            const float wt = z == -INFINITY ? 0.f : sm100::ex2(z - (next == -INFINITY ? 0.f : next));
            top = next;
            sum = sum * old + warp_sum(wt);
#pragma unroll
            for (int j = 0; j < kC; ++j) acc[j] *= old;
#pragma unroll 8
            for (int p = 0; p < cnt; ++p) {
                const float f = __shfl_sync(0xffffffffu, wt, p);
                const float *src = a.part_o + ((long long)(slot(p0 + p) * hw + hx) * rows + row) * D + lane * kC;
                float v[kC];
                if constexpr (kC == 4) *reinterpret_cast<float4 *>(v) = *reinterpret_cast<const float4 *>(src);
                else *reinterpret_cast<float2 *>(v) = *reinterpret_cast<const float2 *>(src);
#pragma unroll
                for (int j = 0; j < kC; ++j) acc[j] = fmaf(f, v[j], acc[j]);
            }
        }
        if (bad) break;
        const float f = sum == 0.f ? 0.f : 1.f / sum;
        const int tok = row / a.G;
        const long long orow = (long long)(rq.x + tok) * a.Hq + (at.y * hw + hx) * a.G + (row - tok * a.G);
        uint32_t *d = reinterpret_cast<uint32_t *>(a.out + orow * D + lane * kC);
#pragma unroll
        for (int j = 0; j < kC / 2; ++j) d[j] = pair_of(acc[2 * j] * f, acc[2 * j + 1] * f, a.bf16);
        if (lane == 0) a.lse[orow] = sum == 0.f ? -INFINITY : (top + log2f(sum)) * 0.6931471805599453f;
    }
}

}  // namespace rs
