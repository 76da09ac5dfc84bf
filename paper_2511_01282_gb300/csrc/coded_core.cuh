// coded_core.cuh -- the attention core over a cache in 8 bits: long chunks and
// draft trees.  Plan, pieces and joining are flash.cuh's; so is the arithmetic, but
// for what the codes change:
//
// Products take codes as fp16, which holds them exactly; the exponents, one for 16 keys,
// go into the softmax:
//     S_rj = q_r.K_j,  s_rj = c 2^(ek) S_rj,  P'_rj = 2^(s_rj + ev - R_r + 7),
//     O'_r = sum P'_rj V_j,  l_r = sum 2^(s_rj - m_r) = sum_blocks 2^(R_r - 7 - ev - m_r) sum P'_rj
// with m_r and R_r running bounds of s and of s + ev, moved only when they are exceeded
// by 2^8 (the largest P' is 2^7 to 2^15 in fp16: weights times 2^ev are rounded by up to 2^-11 down to
// 2^-21 of the largest, by up to 2^-32 of the largest below that).  Where ev is so far below R - m that P' would vanish in fp32 while the
// weight counts, l is summed from its own exponentials.  bf16 queries are scaled by a
// power of two per row into fp16 (what lies 2^-39 below a row's largest is lost).  The
// converting warps are the scarcer: with code 2^e in bf16 tiles (five instructions for two
// codes and not one) the trees below took 1356 us, with code 2^(e - E) in fp16 (E the tile's
// largest; one multiplication, and one exponent in the softmax) 460 us and the chunks 515.
//
// A segment with two row tiles is worked off as in flash.cuh, a row tile to a
// softmax warpgroup.  With one (trees, short chunks), the two take turns at the key
// tiles, each with its own m, R, l and O over the same rows, and the first joins both:
// the chain of one row tile, product, softmax, product, took 2500 cycles a key tile
// where its bytes take 1500.
//
// NaN in V of a key that only some rows see stays out of the products (coded_nan): the converting warps look for it
// in the tiles with such keys, which costs chunks and trees behind a cache nothing that shows (308 us the trees, 438 the
// chunks, 436 before) and short prompts without one 6 % (46 of 757 tokens, 224 us and 210).
//
// Warps: 0 and 1 MMA issue, 2 Q, 3 copies codes, 4-7 and 8-11 softmax, 12-15 codes to
// tiles.  Codes come by TMA, two tiles (64 KB at D = 128) ahead; the converting warps load
// nothing themselves, as their fences, which hand a tile to the tensor core, would wait for
// what is on its way (4.2 us a key tile).  K and V tiles share one ring, K a tile ahead:
// K0 K1 V0 K2 V1 ... V(n-1).
//
// Measured (replayed in a graph): four trees of 65 nodes over 32768 keys (40 heads of 128, bf16) 308 us, 4.4 TB/s
// (the cache in 16 bits takes 414), near what shared memory passes: 224 KB a key tile (products 96, tiles
// written 64, codes written and read 64) in 2200 cycles; 200 to 1000 new tokens behind 4000 to
// 32000 (four requests, 32 / 8 heads of 64, fp16) 438 us, bound by the softmax warps, which share
// their schedulers with the converting ones (in 16 bits 375 us).
#pragma once

#include "coded.cuh"
#include "flash.cuh"

namespace rs {

constexpr int kCoThreads = 512, kCoQWarp = 2, kCoCopyWarp = 3, kCoDecodeWarp = 12;
// (fewer for the issuing warps than they could use: 2 % less time than 176 / 80 / 80)
constexpr uint32_t kCoRegsSoft = 184, kCoRegsProd = 64, kCoRegsDecode = 80;
static_assert(2 * 128 * kCoRegsSoft + 128 * (kCoRegsProd + kCoRegsDecode) == kCoThreads * 128, "register split");

template <int D>
struct CoSmem {
    static constexpr int kTile = kBN * D * 2;
    static constexpr int kNR = D == 128 ? 3 : 8;             // stages of fp16 tiles
    static constexpr int kNC = D == 128 ? 4 : 6;             // stages of codes
    // Tiles whose exponents are kept.  They are written for up to four tiles when the first one's K is
    // about to be copied, so when K of kNC / 2 tiles before is in the ring, so when position kNR before
    // that one is free: at kNR = 3 the products of tile t - 5 are done (and t + 3 takes its place), at
    // 8 S of tile t - 7, whose softmax reads on.
    static constexpr int kExps = D == 128 ? 8 : 16;
    static constexpr int kRing = 0, kQ = kNR * kTile, kCodes = kQ + 2 * kTile;
    static constexpr int kBar = kCodes + kNC * kBN * D;
    static constexpr int kNumBars = 2 * kNR + 2 * kNC + 23;
    static constexpr int kMisc = kBar + kNumBars * 8;        // tensor memory base, abort flag
    static constexpr int kBounds = (kMisc + 8 + 15) / 16 * 16;
    static constexpr int kExp = kBounds + 2 * kFlMaxPhases * 16;  // [tile][block]: 2^ek and ev, each a float's upper half
    static constexpr int kShift = kExp + kExps * 32;         // int8 [row tile][row]
    static constexpr int kStat = kShift + 2 * kBM;           // float2 [row]: the second warpgroup's sums
    static constexpr int kBytes = kStat + kBM * 8;
    static constexpr int kTotal = kBytes + 1024;             // the base is rounded up to 1 KB
    static_assert(kTotal <= 232448, "shared memory of one CTA");
};

// The n key tiles of a piece in the ring's order: positions 0 .. 2 n - 1.
__device__ __forceinline__ int k_at(int tl) { return tl == 0 ? 0 : 2 * tl - 1; }
__device__ __forceinline__ int v_at(int tl, int n) { return tl == n - 1 ? 2 * n - 1 : 2 * tl + 2; }
__device__ __forceinline__ int tile_at(int pos, int n) { return pos == 2 * n - 1 ? n - 1 : pos == 0 ? 0 : (pos & 1) ? (pos + 1) / 2 : pos / 2 - 1; }

// 64 weights of a row as exp_pairs gives them, in fp16, with a factor, an offset and a sum for each block
// of 16 keys; arguments and sums two to an instruction.
__device__ __forceinline__ void exp_blocks(const uint32_t (&s0)[32], const uint32_t (&s1)[32], const float (&c)[4], const float (&nb)[4],
                                           float (&sum)[4], uint32_t (&xp)[32]) {
    constexpr int kAhead = 4, kBehind = 4;  // pairs
    float2 d[32], p[32];
    uint64_t both[4];
    auto fma1 = [&](int i) {
        const float2 v = i < 16 ? make_float2(__uint_as_float(s0[2 * i]), __uint_as_float(s0[2 * i + 1]))
                                : make_float2(__uint_as_float(s1[2 * i - 32]), __uint_as_float(s1[2 * i - 31]));
        uint64_t r;
        asm volatile("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(as_b64(v)), "l"(as_b64(make_float2(c[i / 8], c[i / 8]))), "l"(as_b64(make_float2(nb[i / 8], nb[i / 8]))));
        d[i] = as_float2(r);
    };
#pragma unroll
    for (int i = 0; i < kAhead; ++i) fma1(i);
#pragma unroll
    for (int e = 0; e < 32 + kBehind; ++e) {
        if (e < 32) {
            asm volatile("ex2.approx.ftz.f32 %0, %1;" : "=f"(p[e].x) : "f"(d[e].x));
            asm volatile("ex2.approx.ftz.f32 %0, %1;" : "=f"(p[e].y) : "f"(d[e].y));
        }
        if (e + kAhead < 32) fma1(e + kAhead);
        if (e >= kBehind) {
            const int q = e - kBehind, b = q / 8;
            if (q % 8 == 0) both[b] = as_b64(p[q]);
            else asm volatile("add.rn.f32x2 %0, %0, %1;" : "+l"(both[b]) : "l"(as_b64(p[q])));
            asm volatile("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(xp[q]) : "f"(p[q].y), "f"(p[q].x));
        }
    }
#pragma unroll
    for (int b = 0; b < 4; ++b) sum[b] = as_float2(both[b]).x + as_float2(both[b]).y;
}

template <int D, bool BF16>
__global__ void __launch_bounds__(kCoThreads, 1)
coded_core(FlashArgs a, const __grid_constant__ CUtensorMap tmq, const __grid_constant__ CUtensorMap tmk,
           const __grid_constant__ CUtensorMap tmv) {
    using namespace sm100;
    using S = CoSmem<D>;
    constexpr uint32_t NR = S::kNR, NC = S::kNC;
    extern __shared__ unsigned char smem_raw[];
    // (an offset and not a rounded address: the compiler then knows it for shared memory, whose
    // loads and stores are several times as fast as generic ones)
    unsigned char *smem = smem_raw + (-smem_u32(smem_raw) & 1023u);
    uint64_t *bars = reinterpret_cast<uint64_t *>(smem + S::kBar);
    uint64_t *full = bars, *empty = full + NR, *cfull = empty + NR, *cempty = cfull + NC;  // tiles, codes
    // per softmax: S there, S read (kApart), P there (its two halves), P V complete, Q copied,
    // Q as fp16, Q read, O read, turn at the tensor core; and the second one's sums there
    uint64_t *sfull = cempty + NC, *sfree = sfull + 2, *pfull = sfree + 2, *pfull2 = pfull + 2, *pvdone = pfull2 + 2;
    uint64_t *qfull = pvdone + 2, *qready = qfull + 2, *qfree = qready + 2, *ofree = qfree + 2, *turn = ofree + 2;
    uint64_t *drain = turn + 2, *other = drain + 2;
    uint32_t *s_tmem = reinterpret_cast<uint32_t *>(smem + S::kMisc);
    volatile int *s_abort = reinterpret_cast<volatile int *>(smem + S::kMisc + 4);
    int4 *s_bound = reinterpret_cast<int4 *>(smem + S::kBounds);
    unsigned char *s_exp = smem + S::kExp;
    int8_t *s_shift = reinterpret_cast<int8_t *>(smem + S::kShift);
    float2 *s_stat = reinterpret_cast<float2 *>(smem + S::kStat);

    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    if (tid == 0) {
        for (int s = 0; s < (int)NR; ++s) {
            mbar_init(&full[s], 128);
            mbar_init(&empty[s], 2);  // one for each issuing warp
        }
        for (int s = 0; s < (int)NC; ++s) {
            mbar_init(&cfull[s], 1);
            mbar_init(&cempty[s], 128);
        }
        for (int x = 0; x < 2; ++x) {
            mbar_init(&sfull[x], 1);
            mbar_init(&sfree[x], kBM);
            mbar_init(&pfull[x], kBM);
            mbar_init(&pfull2[x], kBM);
            mbar_init(&pvdone[x], 1);
            mbar_init(&qfull[x], 1);
            mbar_init(&qready[x], 128);
            mbar_init(&qfree[x], kBM);
            mbar_init(&ofree[x], kBM);
            mbar_init(&turn[x], 1);
            mbar_init(&drain[x], 1);
        }
        mbar_init(other, kBM);
        *s_abort = 0;
        fence_mbar_init();
    }
    if (warp == kFlMmaWarp) tmem_alloc(s_tmem, kTmemCols);
    if (warp == kCoQWarp && lane == 0) {
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
    FlPiece pc{};
    // whether softmax (and issuing warp) x has key tiles in a piece of n: with one row tile
    // they alternate, the first one first
    auto takes_part = [&](int x) { return x == 0 || pc.full || pc.j1 - pc.j0 > 1; };

    if (warp < kFlSoftWarp) {
      reg_dealloc<kCoRegsProd>();
      if (warp == kCoQWarp) {
        // ---------------------------------------------------------- Q tiles (one row tile: twice the same)
        const uint32_t q_tx = (uint32_t)(tq * G) * D * 2;
        uint32_t quse[2] = {0, 0};
        bool ok = true;
        while (ok && cur.next(pc)) {
            for (int x = 0; x < 2; ++x) {
                if (!takes_part(x)) continue;
                if (quse[x] > 0 && !(ok = warp_wait(&qfree[x], (quse[x] - 1) & 1, s_abort, a.wait_limit))) break;
                ++quse[x];
                if (lane == 0) {
                    mbar_expect_tx(&qfull[x], q_tx);
#pragma unroll
                    for (int kb = 0; kb < kKB; ++kb)
                        tma_load_3d(smem + S::kQ + x * S::kTile + kb * 16384, &tmq, &qfull[x], kb * 64, pc.kvh * G,
                                    pc.n0 + (pc.p * 2 + (pc.full ? x : 0)) * tq);
                }
                __syncwarp();
            }
        }
        if (!ok) {  // let the copies already issued land before the CTA exits
            volatile int no_abort = 0;
            for (int x = 0; x < 2; ++x)
                if (quse[x] > 0) mbar_wait(&qfull[x], (quse[x] - 1) & 1, &no_abort, kWaitLimit);
        }
      } else if (warp == kCoCopyWarp) {
        // ---------------------------------------------------------- codes and exponents
        // Lane x copies page x of a tile.  The pages and the exponents of four tiles' 32 blocks are looked
        // up by a lane each, four tiles ahead and in three steps, as each waits for the one before
        // (looked up a tile ahead in one go they took 1.6 us a tile, and bound trees).
        const int page = 1 << a.page_log2, box = page < kBN ? page : kBN;  // keys per copy
        const int in_page = (page >> kCodeBlockLog2) - 1;
        constexpr int kBlocks = kBN / kCodeBlock, kBatch = 32 / kBlocks;   // of a tile; tiles of a batch
        const CodedPool &pool = a.coded;
        const uint64_t once = l2_evict_first_policy();
        const int lane_block = min(lane * (box >> kCodeBlockLog2), kBlocks - 1);  // of a tile: where the lane's copy starts
        uint32_t c = 0, g = 0, st = 0, phase = 0;  // positions copied; the next one's stage, and which use of it
        bool ok = true;
        auto free_stage = [&]() -> bool { return ok = quick_wait(&cempty[st], phase ^ 1, s_abort, a.wait_limit); };
        while (ok && cur.next(pc)) {
            const int n = pc.j1 - pc.j0;
            const int32_t *table = a.page_table + (long long)pc.b * a.max_pages;
            const bool evict = a.kv_stream && pc.n <= 2 * tq;
            // this lane's block of batch `bat`; its page: -1 none, -2 a bad one
            auto block_at = [&](int bat) { return (pc.j0 + bat * kBatch) * kBlocks + lane; };
            auto there = [&](int bat) { return bat * kBatch + lane / kBlocks < n && (long long)block_at(bat) * kCodeBlock < pc.keys; };
            auto page_of = [&](int bat) { return there(bat) ? table[block_at(bat) >> (a.page_log2 - kCodeBlockLog2)] : -1; };
            auto checked = [&](int bat, int id) -> int {
                if (!there(bat)) return -1;
                if (id >= 0 && id < a.n_pages) return id;
                atomicOr(&a.status[pc.b], RS_ST_BAD_PAGE);  // nothing outside the pool is read: the copy fills zeros
                return -2;
            };
            auto exp_at = [&](int bat, int id) { return (((long long)id << (a.page_log2 - kCodeBlockLog2)) + (block_at(bat) & in_page)) * a.Hkv + pc.kvh; };
            // (a block without keys or of a bad page: any exponent, as its codes are 0)
            auto scales = [&](int id, int ek, int ev) -> uint32_t {  // (whole numbers of eight bits fit half a float)
                return id < 0 ? 0x3f800000u : __float_as_uint(pow2i(code_exp(ek, BF16))) | __float_as_uint((float)code_exp(ev, BF16)) >> 16;
            };
            int id = checked(0, page_of(0)), id1 = -1, ek1 = 0, ev1 = 0;
            uint32_t exps = scales(id, id >= 0 ? pool.ke[exp_at(0, id)] : 0, id >= 0 ? pool.ve[exp_at(0, id)] : 0);
            auto copy = [&](const CUtensorMap *map, int from, uint32_t tx) {
                if (lane == 0) mbar_expect_tx(&cfull[st], tx);
                __syncwarp();
                if (from >= 0) {
                    unsigned char *dst = smem + S::kCodes + st * (kBN * D) + lane * box * D;
                    if (evict) tma_load_3d_hint(dst, map, &cfull[st], 0, pc.kvh, from, once);
                    else tma_load_3d(dst, map, &cfull[st], 0, pc.kvh, from);
                }
                ++c;
                if (++st == NC) {
                    st = 0;
                    phase ^= 1;
                }
            };
            // row of the pool where the lane's copy of the tile starts (-1: none), bytes of all copies
            int row = -1;
            uint32_t tx = 0;
            for (int tl = 0; tl <= n; ++tl) {  // K of tile tl, V of the one before
                const int last = row;
                const uint32_t last_tx = tx;
                if (tl < n) {
                    const int bat = tl / kBatch, q = tl % kBatch;
                    if (q == 0 && tl > 0) {
                        id = id1;
                        exps = scales(id, ek1, ev1);
                    }
                    const int from = __shfl_sync(0xffffffffu, id, q * kBlocks + lane_block);
                    row = lane * box >= kBN || from == -1 ? -1
                          : from < 0 ? a.n_pages << a.page_log2 : (from << a.page_log2) + (((pc.j0 + tl) * kBN) & (page - 1));
                    tx = (uint32_t)__popc(__ballot_sync(0xffffffffu, row >= 0)) * (uint32_t)(box * D);
                    if (q == 0) id1 = page_of(bat + 1);
                    if (q == 1) {
                        id1 = checked(bat + 1, id1);
                        if (id1 >= 0) {
                            const long long at = exp_at(bat + 1, id1);
                            ek1 = pool.ke[at];
                            ev1 = pool.ve[at];
                        }
                    }
                    if (!free_stage()) break;
                    if (q == 0)  // the batch's exponents
                        *reinterpret_cast<uint32_t *>(s_exp + ((g + tl + lane / kBlocks) % S::kExps) * 32 + lane % kBlocks * 4) = exps;
                    __syncwarp();
                    copy(&tmk, row, tx);
                }
                if (tl > 0) {
                    if (!free_stage()) break;
                    copy(&tmv, last, last_tx);
                }
            }
            g += n;
        }
        if (!ok) {  // let the copies already issued land before the CTA exits
            volatile int no_abort = 0;
            for (uint32_t u = min(c, NC); u > 0; --u) {
                --c;
                mbar_wait(&cfull[c % NC], c / NC & 1, &no_abort, kWaitLimit);
            }
        }
      } else {
        // ---------------------------------------------------------- MMA issuers, one per softmax
        const int x = warp - kFlMmaWarp;
        constexpr uint32_t idS = idesc_16_f32(false, kBM, kBN, false);
        constexpr uint32_t idO = idesc_16_f32(false, kBM, D, true);
        const uint64_t dK0 = sdesc_sw128(smem_u32(smem + S::kRing), 16, 1024);
        const uint32_t d_hi = (uint32_t)(dK0 >> 32);
        const uint32_t k_lo0 = (uint32_t)dK0;
        const uint32_t q_lo0 = (uint32_t)sdesc_sw128(smem_u32(smem + S::kQ), 16, 1024);
        const uint32_t v_lo0 = (uint32_t)sdesc_sw128(smem_u32(smem + S::kRing), 16384, 1024);
        constexpr uint32_t kTileDesc = S::kTile >> 4;
        const uint32_t tm = uniform(tmem), xu = uniform((uint32_t)x);
        const uint32_t q_lo = q_lo0 + xu * kTileDesc, s_tm = tm + Tm::s(0) + xu * 128;
        const uint32_t o_tm = tm + Tm::o(0) + xu * D, p_tm = tm + Tm::p(0) + xu * (kApart ? 64 : 128);
        uint64_t *const q_there = BF16 ? qready : qfull;
        uint32_t g = 0, done = 0, pieces = 0, turns = 0;  // key tiles of the CTA; key tiles, pieces of this softmax
        bool ok = true;
        auto wait = [&](uint64_t *b1, uint32_t p1, uint64_t *b2, uint32_t p2) -> bool {
            return ok = quick_wait2(b1, p1 & 1, b2, p2 & 1, s_abort, a.wait_limit);
        };
        // Positions of the ring that this warp does not use are given back, one by one, so that
        // it is never two uses of a stage behind (a wait's parity tells only neighbours apart).
        int pos = 0;
        auto give = [&](int to, int n, int own) -> bool {  // own: parity of its tiles, 2: all are, 3: none
            for (; pos < to; ++pos) {
                if (own == 2 || (own < 2 && (tile_at(pos, n) & 1) == own)) continue;
                const uint32_t p = 2 * g + pos;
                if (!wait(&full[p % NR], p / NR, &full[p % NR], p / NR)) return false;
                if (lane == 0) mbar_arrive_cnt(&empty[p % NR], 1);
                __syncwarp();
            }
            return true;
        };
        // S of key tile tl of the piece (K and, at D = 64, S's columns are there)
        auto issue_s = [&](int tl) {
            const uint32_t st = (2 * g + k_at(tl)) % NR;
            tc_fence_after();
            const uint32_t k_lo = uniform(k_lo0 + st * kTileDesc);
            if (elect_one()) {
#pragma unroll
                for (int kk = 0; kk < D / 16; ++kk) {
                    const uint32_t off = (uint32_t)(((kk >> 2) * 16384 + (kk & 3) * 32) >> 4);
                    umma_ss(s_tm, desc_of(q_lo + off, d_hi), desc_of(k_lo + off, d_hi), idS, kk > 0);
                }
                umma_commit(&sfull[x]);
                umma_commit(&empty[st]);
            }
            __syncwarp();
        };
        while (ok && cur.next(pc)) {
            const int n = pc.j1 - pc.j0;
            const int step = pc.full ? 1 : 2, first = pc.full ? 0 : x, own = !takes_part(x) ? 3 : pc.full ? 2 : x;
            pos = 0;
            if (own == 3) {
                if (!give(2 * n, n, own)) break;
                g += n;
                continue;
            }
            if (!give(k_at(first), n, own)) break;
            const uint32_t p0 = 2 * g + k_at(first);
            if (!wait(&q_there[x], pieces, &full[p0 % NR], p0 / NR)) break;
            if (kApart && done > 0 && !wait(&sfree[x], done - 1, &sfree[x], done - 1)) break;
            issue_s(first);
            // key tiles of the piece that some row of the row tile sees
            const int seen = (int)uniform((uint32_t)min(n, row_tiles(a, pc.n, pc.ctx, pc.p, pc.full ? x : 0) - pc.j0));
#pragma unroll 1
            for (int tl = first; tl < n; tl += step, ++done) {
                const int next = tl + step;
                const bool more = next < n;
                const uint32_t pv = 2 * g + v_at(tl, n), pk = 2 * g + k_at(next), st = pv % NR;
                if (kApart) {  // S of the next tile goes ahead of this one's P V
                    if (more) {
                        if (!give(k_at(next), n, own)) break;
                        if (!wait(&full[pk % NR], pk / NR, &sfree[x], done)) break;
                        issue_s(next);
                    }
                    if (!give(v_at(tl, n), n, own)) break;
                    if (!wait(&full[st], pv / NR, &pfull[x], done)) break;
                } else {
                    // what does not depend on the softmax first; then P and, where both row tiles are
                    // at work, the turn
                    if (!give(v_at(tl, n), n, own)) break;
                    if (more && !give(k_at(next), n, own)) break;
                    if (!wait(&full[st], pv / NR, more ? &full[pk % NR] : &full[st], more ? pk / NR : pv / NR)) break;
                    const bool must = pc.full && (x == 1 || turns > 0);
                    if (!wait(&pfull[x], done, must ? &turn[x] : &pfull[x], must ? turns - (x == 0 ? 1 : 0) : done)) break;
                }
                if (tl == first && pieces > 0 && !wait(&ofree[x], pieces - 1, &ofree[x], pieces - 1)) break;
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
                                       (tl > first || ks > 0) ? 1u : 0u);
                        if (part == kParts - 1) {
                            umma_commit(&pvdone[x]);
                            umma_commit(&empty[st]);
                        }
                    }
                    __syncwarp();
                }
                if (!ok) break;
                if (!kApart) {
                    if (more) issue_s(next);
                    if (pc.full) {
                        if (lane == 0) mbar_arrive_cnt(&turn[x ^ 1], 1);
                        __syncwarp();
                        ++turns;
                    }
                }
            }
            if (!ok || !give(2 * n, n, own)) break;
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
    } else if (warp < kCoDecodeWarp) {
        reg_alloc<kCoRegsSoft>();
        // ---------------------------------------------------------- softmax / epilogue (rows)
        const int x = (warp - kFlSoftWarp) >> 2;
        const int r = tid & (kBM - 1);  // row of the tile == tensor memory lane
        const uint32_t lane_off = (uint32_t)((warp & 3) * 32) << 16;
        const float cexp = fminf(a.scale * 1.4426950408889634f, 3.402823466e38f);  // scores -> log2 domain (scale > 0)
        const int rt = r / G, rg = r - rt * G;
        const uint32_t s_tm = tmem + lane_off + Tm::s(0) + (uint32_t)x * 128;
        const uint32_t p_tm = tmem + lane_off + Tm::p(0) + (uint32_t)x * (kApart ? 64 : 128);
        uint32_t g = 0, done = 0, both = 0;  // key tiles of the CTA; of this softmax; pieces that the two have shared
        bool ok = true;
        while (ok && cur.next(pc)) {
            const int n = pc.j1 - pc.j0;
            if (!takes_part(x)) {
                g += n;
                continue;
            }
            const int step = pc.full ? 1 : 2, first = pc.full ? 0 : x;
            const bool shared = !pc.full && n > 1;
            const int tok0 = (pc.p * 2 + (pc.full ? x : 0)) * tq, tok = tok0 + rt;
            const bool valid = rt < tq && tok < pc.n;
            const unsigned vmask = __ballot_sync(0xffffffffu, valid);
            const int open = pc.ctx + (a.anc ? 0 : tok0 + 1);  // keys that every row of the tile sees
            const int seen = pc.ctx + tok + 1;                 // causal: keys this row sees
            float m = -INFINITY, ref = -INFINITY, l = 0.f, rowf = cexp;
            // One key tile; masked: some row does not see all of the keys.  The kernel's roles share an
            // instruction cache: what is rare is one small loop, and nothing is compiled twice (masks within
            // the loads and sums of their own in registers took the chunks 523 us and not 464).
            auto tile = [&](bool masked, int tl) -> bool {
                const uint32_t t = g + tl;
                const int key0 = (pc.j0 + tl) * kBN;
                if (!(ok = quick_wait(&sfull[x], done & 1, s_abort, a.wait_limit))) return false;
                tc_fence_after();
                if (BF16 && tl == first) rowf = finite_mul(cexp, pow2i(s_shift[x * kBM + r]));
                // the piece's last S has read Q: its buffer is free
                if (tl + step >= n) warp_arrive(&qfree[x]);
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
                    if (!wait_idle()) return false;
                    warp_arrive(&pfull[x]);
                    if (!kApart) warp_arrive(&pfull2[x]);
                    ++done;
                    return true;
                }
                if (masked) {  // hidden scores are replaced where they are: what follows knows nothing of them
                    uint32_t anc[kAncWords];
                    if (a.anc)
#pragma unroll
                        for (int w = 0; w < kAncWords; ++w) anc[w] = valid ? a.anc[(long long)(pc.n0 + tok) * kAncWords + w] : 0u;
#pragma unroll 1
                    for (int k0 = 0; k0 < kBN; k0 += 32) {
                        uint32_t va[32];
                        const int c = seen - key0 - k0;
                        const uint32_t mk = a.anc ? tree_window(anc, key0 + k0 - pc.ctx) : c >= 32 ? 0xffffffffu : c <= 0 ? 0u : (1u << c) - 1u;
                        tmem_ld32(s_tm + k0, va);
                        tmem_wait_ld();
                        tmem_regs_ready(va);
                        hide(va, mk);
                        tmem_st32(s_tm + k0, va);
                    }
                    tmem_wait_st();
                }
                const uint4 *exps = reinterpret_cast<const uint4 *>(s_exp + (t % S::kExps) * 32);  // of four blocks each
                auto word = [](const uint4 &e4, int b) { return b == 0 ? e4.x : b == 1 ? e4.y : b == 2 ? e4.z : e4.w; };
                // (factors are not 0: hidden scores stay -inf)
                auto factor = [&](const uint4 &e4, int b) { return fmaxf(finite_mul(rowf, __uint_as_float(word(e4, b) & 0xffff0000u)), 0x1p-126f); };
                auto offset = [&](const uint4 &e4, int b) { return __uint_as_float(word(e4, b) << 16); };
                auto load64 = [&](int hh, uint32_t (&va)[32], uint32_t (&vb)[32]) {
                    tmem_ld32(s_tm + hh * 64, va);
                    tmem_ld32(s_tm + hh * 64 + 32, vb);
                    tmem_wait_ld();
                    tmem_regs_ready(va);
                    tmem_regs_ready(vb);
                };
                // the row's maxima, of the scores and with their blocks' ev, 64 keys at a time
                float mt = -INFINITY, rmax = -INFINITY, ev_min = INFINITY;
#pragma unroll
                for (int hh = 0; hh < 2; ++hh) {
                    uint32_t va[32], vb[32];
                    load64(hh, va, vb);
                    const uint4 e4 = exps[hh];
#pragma unroll
                    for (int b = 0; b < 4; ++b) {
                        const uint32_t *v = (b < 2 ? va : vb) + b % 2 * 16;
                        float x[2] = {-INFINITY, -INFINITY};
#pragma unroll
                        for (int e = 0; e < 16; e += 2)
                            asm("max.f32 %0, %0, %1, %2;" : "+f"(x[e >> 1 & 1]) : "f"(__uint_as_float(v[e])), "f"(__uint_as_float(v[e + 1])));
                        const float top = fmaxf(x[0], x[1]) * factor(e4, b);
                        mt = fmaxf(mt, top);
                        rmax = fmaxf(rmax, top + offset(e4, b));
                        ev_min = fminf(ev_min, offset(e4, b));
                    }
                }
                // lazy rescale: a bound moves only when it is exceeded by more than 2^8
                if (mt > m + 8.f) {
                    l *= ex2(m - mt);
                    m = mt;
                }
                const bool grow = rmax > ref + 8.f;
                const float corr = grow ? ex2(ref - rmax) : 1.f;  // 0 when ref is -inf
                if (grow) ref = rmax;
                if (tl > first && __any_sync(0xffffffffu, grow)) {
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
                const float mn = m == -INFINITY ? 0.f : m, up = ref == -INFINITY ? 0.f : 7.f - ref;
                // P' may vanish in fp32 while its keys count for l (values 2^90 below others'): then l is
                // summed by itself
                const bool apart = __any_sync(0xffffffffu, -up - ev_min - mn > 90.f);
                if (apart) {
#pragma unroll 1
                    for (int k0 = 0; k0 < kBN; k0 += 32) {
                        uint32_t va[32];
                        tmem_ld32(s_tm + k0, va);
                        tmem_wait_ld();
                        tmem_regs_ready(va);
                        const uint4 e4 = exps[k0 / 64];
                        const float c0 = factor(e4, k0 & 32 ? 2 : 0), c1 = factor(e4, k0 & 32 ? 3 : 1);
#pragma unroll
                        for (int e = 0; e < 32; ++e) l += ex2(fmaf(__uint_as_float(va[e]), e < 16 ? c0 : c1, -mn));
                    }
                }
#pragma unroll(kApart ? 2 : 1)
                for (int hh = 0; hh < 2; ++hh) {
                    uint32_t va[32], vb[32], xp[32];
                    load64(hh, va, vb);
                    if (kApart && hh) {  // S has been read: the next one may be written
                        tc_fence_before();
                        warp_arrive(&sfree[x]);
                    }
                    const uint4 e4 = exps[hh];
                    float c[4], nb[4], sum[4];
#pragma unroll
                    for (int b = 0; b < 4; ++b) {
                        c[b] = factor(e4, b);
                        nb[b] = offset(e4, b) + up;
                    }
                    exp_blocks(va, vb, c, nb, sum, xp);
                    if (kApart && !hh && !wait_idle()) return false;
                    tmem_st32(p_tm + hh * 32, xp);
                    if (!apart) {
#pragma unroll
                        for (int b = 0; b < 4; ++b) l = fmaf(sum[b], ex2(-nb[b] - mn), l);
                    }
                    if (!kApart || hh) {
                        tmem_wait_st();
                        tc_fence_before();
                        warp_arrive(kApart || !hh ? &pfull[x] : &pfull2[x]);
                    }
                }
                ++done;
                return true;
            };
            const int n_open = min(n, open / kBN - pc.j0);
#pragma unroll 1
            for (int tl = first; ok && tl < n; tl += step) tile(tl >= n_open, tl);
            if (!ok || !(ok = quick_wait(&pvdone[x], (done - 1) & 1, s_abort, a.wait_limit))) break;
            tc_fence_after();
            // log2 of the sum of the weights, and what O' has to be multiplied with, as a power of two
            float z = l == 0.f ? -INFINITY : m + log2f(l), up2 = l == 0.f ? 0.f : ref - 7.f - z;
            if (shared && x == 1) {
                s_stat[r] = make_float2(z, up2);
                tc_fence_before();
                warp_arrive(other);
                g += n;
                continue;
            }
            float z1 = -INFINITY, up1 = 0.f;
            if (shared) {
                if (!(ok = quick_wait(other, both & 1, s_abort, a.wait_limit))) break;
                ++both;
                tc_fence_after();
                z1 = s_stat[r].x;
                up1 = s_stat[r].y;
            }
            if (vmask) {
                const float top = fmaxf(z, z1);
                const float w0 = z == -INFINITY ? 0.f : ex2(z - top), w1 = z1 == -INFINITY ? 0.f : ex2(z1 - top);
                const float sum = w0 + w1, inv = sum == 0.f ? 0.f : 1.f / sum;
                // (in two steps: the power alone may be out of range)
                const float h0 = ex2(0.5f * up2), f0 = h0 * (w0 * inv), h1 = ex2(0.5f * up1), f1 = h1 * (w1 * inv);
                const float zz = sum == 0.f ? -INFINITY : top + log2f(sum);
                const long long orow = (long long)(pc.n0 + tok) * a.Hq + pc.kvh * G + rg;
                const long long prow = (long long)pc.slot * kFlRows + (pc.full ? x : 0) * kBM + r;
                const bool final = pc.slot < 0;
#pragma unroll 1
                for (int ch = 0; ch < D / 32; ++ch) {
                    uint32_t xo[32];
                    tmem_ld32(tmem + lane_off + Tm::o(0) + (uint32_t)x * D + ch * 32, xo);
                    tmem_wait_ld();
                    tmem_regs_ready(xo);
#pragma unroll
                    for (int e = 0; e < 32; ++e)  // without weights the columns may hold anything
                        xo[e] = w0 == 0.f ? 0u : __float_as_uint(__uint_as_float(xo[e]) * h0 * f0);
                    if (shared) {
                        uint32_t y[32];
                        tmem_ld32(tmem + lane_off + Tm::o(1) + ch * 32, y);
                        tmem_wait_ld();
                        tmem_regs_ready(y);
                        if (w1 != 0.f) {
#pragma unroll
                            for (int e = 0; e < 32; ++e) xo[e] = __float_as_uint(fmaf(__uint_as_float(y[e]) * h1, f1, __uint_as_float(xo[e])));
                        }
                    }
                    if (!valid) continue;
                    if (final) {
                        uint32_t v[16];
#pragma unroll
                        for (int e = 0; e < 16; ++e) v[e] = pack16<BF16>(__uint_as_float(xo[2 * e]), __uint_as_float(xo[2 * e + 1]));
                        store32(a.out + orow * D + ch * 32, v);
                        store32(a.out + orow * D + ch * 32 + 16, v + 8);
                    } else {
#pragma unroll
                        for (int e = 0; e < 4; ++e) store32(a.part_o + prow * D + ch * 32 + 8 * e, xo + 8 * e);
                    }
                }
                if (valid && final) {
                    a.lse[orow] = zz * 0.6931471805599453f;
                } else if (valid) {  // O / l, and l as part of the maximum; NaN in l, which joining keeps
                    a.part_m[prow] = zz;
                    a.part_l[prow] = sum == 0.f ? 0.f : 1.f + 0.f * sum;
                }
            }
            tc_fence_before();
            warp_arrive(&ofree[x]);
            if (shared) warp_arrive(&ofree[1]);
            g += n;
        }
    } else {
        reg_dealloc<kCoRegsDecode>();
        // ---------------------------------------------------------- codes to tiles
        // Four warps turn a copied tile into fp16, each a quarter of its rows; a lane has 16 codes of
        // a row, 32 bytes of the tile.  (Two groups of four that take turns need registers that the
        // softmax warps miss more.)
        constexpr int kRowLanes = D / 16, kRowsStep = 128 / kRowLanes, kLoads = kBN / kRowsStep;
        const int ci = tid & 127, part = ci % kRowLanes, row0 = ci / kRowLanes;
        uint32_t st = 0, phase = 0, cst = 0, cphase = 0;  // stages of tiles and codes, and which use of them
        uint32_t qphase = 0;                              // bit x: of Q tile x
        bool ok = true;
        while (ok && cur.next(pc)) {
            const int n = pc.j1 - pc.j0, tail = pc.keys - (pc.j1 - 1) * kBN;  // keys of the last tile
            // NaN in V of a key that some row does not see would reach all rows by the product's 0 x NaN.  In V from this
            // position on, the first with keys that not every row of the piece sees, it is looked for first and becomes
            // 0 (the rows that see the key get it from coded_nan).
            const int open = pc.ctx + (a.anc ? 0 : pc.p * 2 * tq + 1);
            const int look = open < pc.keys && open < pc.j1 * kBN ? v_at(max(open / kBN - pc.j0, 0), n) : 2 * n;
            // (the queries behind two positions, and not between the loop's statements: a jump over so much
            // took 200 cycles a position)
#pragma unroll 1
            for (int half = BF16 ? 0 : 1; ok && half < 2; ++half) {
                if (BF16 && half) {
#pragma unroll 1
                    for (int x = 0; x < 2; ++x) {
                        if (!takes_part(x)) continue;
                        // Q tile x to fp16 in place, a row to a thread, by a power of two that brings its largest value
                        // to 2^14 .. 2^15
                        if (!(ok = quick_wait(&qfull[x], qphase >> x & 1, s_abort, a.wait_limit))) break;
                        qphase ^= 1u << x;
                        unsigned char *row = smem + S::kQ + x * S::kTile + ci * 128;
                        uint32_t most = 0;
#pragma unroll 2
                        for (int i = 0; i < 8 * kKB; ++i) {
                            const uint4 v = *reinterpret_cast<const uint4 *>(row + (i >> 3) * 16384 + ((i + ci) & 7) * 16);
                            const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
                            for (int e = 0; e < 4; ++e) {
                                const uint32_t lo = (w[e] << 16) & 0x7fffffffu, hi = w[e] & 0x7fff0000u;
                                most = max(most, max(lo < 0x7f800000u ? lo : 0u, hi < 0x7f800000u ? hi : 0u));
                            }
                        }
                        const int shift = most ? max((int)(most >> 23) - 127 - 14, -112) : 0;
                        const float down = pow2i(-shift);
#pragma unroll 2
                        for (int i = 0; i < 8 * kKB; ++i) {
                            uint4 *p = reinterpret_cast<uint4 *>(row + (i >> 3) * 16384 + ((i + ci) & 7) * 16);
                            uint4 v = *p;
                            uint32_t *w = &v.x;
#pragma unroll
                            for (int e = 0; e < 4; ++e)
                                w[e] = pack16<false>(__uint_as_float(w[e] << 16) * down, __uint_as_float(w[e] & 0xffff0000u) * down);
                            *p = v;
                        }
                        s_shift[x * kBM + ci] = (int8_t)shift;
                        fence_async_smem();
                        warp_arrive(&qready[x]);
                    }
                    if (!ok) break;
                }
                const int end = half ? 2 * n : 2;
                // A lane's 16 codes are two words of eight: at D = 128 one of each 64 columns (of odd rows the
                // second first), at D = 64 side by side.  All go to other banks that way, there and here.
                const int from0 = row0 * D + (D == 128 ? (row0 & 1) * 64 + part * 8 : part * 16);
                const int step = D == 128 ? (row0 & 1 ? -64 : 64) : 8;
#pragma unroll 1
                for (int pos = BF16 && half ? 2 : 0; ok && pos < end;) {  // (two loops: what is rare stays out of the inner one)
                    const int stop = min(end, pos < look ? look : pos + 1);
                    if (pos >= look && (pos == 2 * n - 1 || !(pos & 1))) {  // (V: of even positions, and the last)
                        if (!(ok = quick_wait(&cfull[cst], cphase, s_abort, a.wait_limit))) break;
                        // this lane's own words, of keys open .. pc.keys - 1
                        const int key0 = (pc.j0 + tile_at(pos, n)) * kBN + row0;
                        const int i1 = min((pc.keys - key0 + kRowsStep - 1) / kRowsStep, kLoads);
                        unsigned char *codes = smem + S::kCodes + cst * (kBN * D) + from0;
#pragma unroll 1
                        for (int i = max((open - key0 + kRowsStep - 1) / kRowsStep, 0); i < i1; ++i) {
                            uint2 *p = reinterpret_cast<uint2 *>(codes + i * 2048), *q = reinterpret_cast<uint2 *>(codes + i * 2048 + step);
                            const uint2 x = *p, y = *q;
                            if (!(nan_codes(x.x) | nan_codes(x.y) | nan_codes(y.x) | nan_codes(y.y))) continue;
                            *p = make_uint2(without_nan(x.x), without_nan(x.y));
                            *q = make_uint2(without_nan(y.x), without_nan(y.y));
                            a.n_pairs[3] = 1;
                        }
                    }
#pragma unroll 1
                    for (; pos < stop; ++pos) {
                        if (!(ok = quick_wait2(&cfull[cst], cphase, &empty[st], phase ^ 1, s_abort, a.wait_limit))) break;
                        const unsigned char *codes = smem + S::kCodes + cst * (kBN * D);
                        unsigned char *tile = smem + S::kRing + st * S::kTile;
                        const unsigned char *const from = codes + from0;
                        // 128-byte swizzle: 16-byte word w of row r at w ^ (r & 7)
                        unsigned char *const to = tile + row0 * 128;
                        const int at0 = D == 128 ? (row0 & 1) * 16384 + ((part ^ (row0 & 7)) * 16) : ((2 * part) ^ (row0 & 7)) * 16;
                        const int at1 = D == 128 ? at0 ^ 16384 : ((2 * part + 1) ^ (row0 & 7)) * 16;
                        uint2 x[kLoads], y[kLoads];  // (all loads before the first store, which the compiler does not move them over)
#pragma unroll
                        for (int i = 0; i < kLoads; ++i) {
                            x[i] = *reinterpret_cast<const uint2 *>(from + i * 2048);
                            y[i] = *reinterpret_cast<const uint2 *>(from + i * 2048 + step);
                        }
#pragma unroll
                        for (int i = 0; i < kLoads; ++i) {
                            uint4 lo, hi;
                            decode4(x[i].x, lo.x, lo.y);
                            decode4(x[i].y, lo.z, lo.w);
                            decode4(y[i].x, hi.x, hi.y);
                            decode4(y[i].y, hi.z, hi.w);
                            *reinterpret_cast<uint4 *>(to + at0 + i * kRowsStep * 128) = lo;
                            *reinterpret_cast<uint4 *>(to + at1 + i * kRowsStep * 128) = hi;
                        }
                        if (tail < kBN && tile_at(pos, n) == n - 1)  // behind the last key anything was copied, NaN too
#pragma unroll 1
                            for (int i = 0; i < kLoads; ++i)
                                if (i * kRowsStep + row0 >= tail) {
                                    *reinterpret_cast<uint4 *>(to + at0 + i * kRowsStep * 128) = make_uint4(0, 0, 0, 0);
                                    *reinterpret_cast<uint4 *>(to + at1 + i * kRowsStep * 128) = make_uint4(0, 0, 0, 0);
                                }
                        fence_async_smem();
                        warp_arrive(&full[st]);
                        warp_arrive(&cempty[cst]);
                        if (++st == NR) {
                            st = 0;
                            phase ^= 1;
                        }
                        if (++cst == NC) {
                            cst = 0;
                            cphase ^= 1;
                        }
                    }
                }
            }
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

// NaN in V of new tokens, which coded_core kept out of its products, into the rows that see it: a new token and KV head to a
// warp, four codes to a lane.  Where there was none, the usual case, it returns at once.
constexpr int kNanThreads = 256;
template <int D>
__global__ void __launch_bounds__(kNanThreads)
coded_nan(FlashArgs a) {
    pdl_enter();
    if (!a.n_pairs[3]) return;
    const int lane = threadIdx.x & 31;
    const long long w0 = blockIdx.x * (kNanThreads / 32) + (threadIdx.x >> 5), warps = gridDim.x * (kNanThreads / 32);
    for (int b = 0; b < a.B; ++b) {
        const int4 rq = a.req[b];  // first row, rows, ctx
        if (a.status[b]) continue;
        for (long long w = w0; w < (long long)rq.y * a.Hkv; w += warps) {
            const int i = (int)(w / a.Hkv), h = (int)(w - (long long)i * a.Hkv), key = rq.z + i;
            const long long id = a.page_table[(long long)b * a.max_pages + (key >> a.page_log2)];
            if (id < 0 || id >= a.n_pages) continue;
            const long long slot = (id << a.page_log2) + (key & ((1 << a.page_log2) - 1));
            const uint32_t at = lane < D / 4 ? nan_codes(reinterpret_cast<const uint32_t *>(a.coded.v + (slot * a.Hkv + h) * D)[lane]) : 0;
            if (!__any_sync(0xffffffffu, at)) continue;
            for (int r = i; r < rq.y; ++r) {
                if (a.anc && !(a.anc[(long long)(rq.x + r) * kAncWords + (i >> 5)] >> (i & 31) & 1u)) continue;
                uint16_t *o = a.out + ((long long)(rq.x + r) * a.Hq + h * a.G) * D + 4 * lane;
                for (int k = 0; k < a.G; ++k, o += D)
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        if (at >> (8 * e + 7) & 1u) o[e] = 0x7fff;
            }
        }
    }
}

}  // namespace rs
