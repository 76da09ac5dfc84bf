// flash_run.cuh -- launches of the attention core for one 16-bit type
// (included by one source file per type, so that they compile side by side).
#pragma once

#include <algorithm>
#include <atomic>

#include "common.cuh"
#include "flash.cuh"

namespace rs {

// flash_combine: joins the pieces of the segments that the shares' ends cut.
// Block (c, y) looks at where CTA c + 1's share of each phase starts; if that is
// inside a segment, and the first cut of it, the block joins every gridDim.y-th
// eight of its rows, a row to a warp, its lanes the pieces' (m, l) first and then
// the columns:
//     M = max m_p, L = sum 2^(m_p - M) l_p, O = sum 2^(m_p - M) O_p / L
// It also empties the rows of rejected requests (after the pieces' writers).
// Bound: latency, of a handful of dependent loads and of the instructions, which
// are fetched anew for every launch: the loop over the rows is not unrolled (four
// rows at once in 600 instructions took 8 us for single tokens, this 6), and the
// bounds and the status are read before they are needed (one request's single
// token as a whole 21.2 -> 19.4 us).  With few rows in all a warp takes one of a
// segment (a tree of 65 nodes 34 -> 27 us), else four (16 such trees 124 us, with
// one 136), by the average request: single tokens have a block, not eight.
constexpr int kFlCombThreads = 256;

template <int D, bool BF16>
__global__ void __launch_bounds__(kFlCombThreads)
flash_combine(FlashArgs a) {
    pdl_enter();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    constexpr int kWarps = kFlCombThreads / 32;
    const int c = min((int)blockIdx.x + 1, a.grid);
    const int blocks = gridDim.x * gridDim.y;
    for (int b = blockIdx.y * gridDim.x + blockIdx.x; b < a.B; b += blocks) {
        if (!(a.status[b] & ~RS_ST_TIMEOUT)) continue;
        const int4 rq = a.req[b];
        const long long rows = (long long)rq.w * a.Hq;  // none where another request may have them
        uint4 *o = reinterpret_cast<uint4 *>(a.out + (long long)rq.x * a.Hq * D);
        for (long long i = threadIdx.x; i < rows * (D / 8); i += kFlCombThreads) o[i] = make_uint4(0, 0, 0, 0);
        for (long long i = threadIdx.x; i < rows; i += kFlCombThreads) a.lse[(long long)rq.x * a.Hq + i] = 0.f;
    }
    if (c >= a.grid) return;
#pragma unroll 1
    for (int f = 0; f < a.max_phases && (f == 0 || f < a.n_pairs[2]); ++f) {
        const int4 *bound = a.bound + f * (a.grid + 1);
        const int4 start = bound[c], before = bound[c - 1];
        const int4 p0 = bound[min(c - 1 + lane, a.grid)], q0 = bound[min(c + lane, a.grid)];
        auto same = [&](int4 r) { return r.x == start.x && r.y == start.y && r.z > 0; };
        if (start.z == 0 || same(before)) continue;  // between segments, or not the first cut
        const int4 e = a.ent[start.y];  // request, pair, first row, rows
        const int bad = a.status[e.x] & ~RS_ST_TIMEOUT;
        const int kvh = (f > 0 ? f * a.Hkv / a.n_pairs[2] : 0) + start.x;
        constexpr int kC = D / 32;  // columns of a lane
#pragma unroll 1
        for (int k = blockIdx.y * kWarps + warp; k < kFlRows; k += gridDim.y * kWarps) {
            const int x = k / kBM, r = k & (kBM - 1), t = r / a.G, tok = (e.y * 2 + x) * a.tq + t;
            if (t >= a.tq) continue;
            if (tok >= e.w) break;
            const long long row = k;
            float M = -INFINITY, L = 0.f, acc[kC] = {};
#pragma unroll 1
            for (int c0 = c - 1;; c0 += 32) {  // 32 shares at a time; the first piece is the end of share c - 1
                const int c1 = c0 + lane;
                int4 p = p0, q = q0;
                if (c0 >= c) {
                    p = bound[min(c1, a.grid)];
                    q = bound[min(c1 + 1, a.grid)];
                }
                const bool head = c1 == c - 1;
                const bool in = head || (c1 < a.grid && same(p)), have = head || (in && !(same(q) && q.z == p.z));  // not an empty share
                const long long at = (long long)(2 * (f * a.grid + c1) + (head ? 1 : 0)) * kFlRows + row;
                const float m = have ? a.part_m[at] : -INFINITY, l = have ? a.part_l[at] : 0.f;
                const float Mn = fmaxf(M, warp_max(m));
                const float old = Mn == -INFINITY ? 1.f : sm100::ex2(M - Mn);
                const float w = Mn == -INFINITY ? (have ? 1.f : 0.f) : sm100::ex2(m - Mn);
                L = L * old + warp_sum(have ? w * l : 0.f);
#pragma unroll
                for (int j = 0; j < kC; ++j) acc[j] *= old;
                M = Mn;
                const unsigned pieces = __ballot_sync(0xffffffffu, have);
                const int cnt = 32 - __clz(pieces);  // 0 where the run ended with the last 32
                const float *o = a.part_o + ((long long)(2 * (f * a.grid + c0)) * kFlRows + row) * D + lane * kC;
#pragma unroll 4
                for (int k1 = 0; k1 < cnt; ++k1) {
                    const float wp = __shfl_sync(0xffffffffu, w, k1);
                    if (!((pieces >> k1) & 1u)) continue;
                    const float *src = o + (long long)(2 * k1 + (c0 + k1 == c - 1 ? 1 : 0)) * kFlRows * D;
                    float v[kC];
                    if constexpr (kC == 4) *reinterpret_cast<float4 *>(v) = *reinterpret_cast<const float4 *>(src);
                    else *reinterpret_cast<float2 *>(v) = *reinterpret_cast<const float2 *>(src);
#pragma unroll
                    for (int j = 0; j < kC; ++j) acc[j] = fmaf(wp, v[j], acc[j]);
                }
                if (!__all_sync(0xffffffffu, in)) break;
            }
            if (bad) break;
            const float fr = L > 0.f ? 1.f / L : L;  // no key with weight: 0; NaN stays
            const long long orow = (long long)(e.z + tok) * a.Hq + kvh * a.G + (r - t * a.G);
            uint32_t *d = reinterpret_cast<uint32_t *>(a.out + orow * D + lane * kC);
            if constexpr (kC == 4)
                *reinterpret_cast<uint2 *>(d) = make_uint2(pack16<BF16>(acc[0] * fr, acc[1] * fr), pack16<BF16>(acc[2] * fr, acc[3] * fr));
            else
                *d = pack16<BF16>(acc[0] * fr, acc[1] * fr);
            if (lane == 0) a.lse[orow] = L > 0.f ? (M + log2f(L)) * 0.6931471805599453f : (L == 0.f ? -INFINITY : L);
        }
    }
}

template <int D, bool BF16>
rs_status flash_launch_d(const FlashArgs &a, const CUtensorMap &tmq, const CUtensorMap &tmk, const CUtensorMap &tmv,
                         const char *what, cudaStream_t st) {
    // per device: 0 not asked, 1 ready, -1 built with too few registers for the
    // warpgroups' split (a raise that cannot be granted would wait for ever)
    static std::atomic<int> ready[64];
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) {
        set_error("%s: no current device", what);
        return RS_ERR_CUDA;
    }
    if (ready[dev].load() == 0) {
        cudaFuncAttributes fa;
        const cudaError_t e1 = cudaFuncGetAttributes(&fa, flash_kernel<D, BF16>);
        const cudaError_t e2 = cudaFuncSetAttribute(flash_kernel<D, BF16>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                                    FlSmem<D>::kTotal);
        if (e1 != cudaSuccess || e2 != cudaSuccess) {
            set_error("%s: kernel attributes: %s", what, cudaGetErrorString(e1 != cudaSuccess ? e1 : e2));
            return RS_ERR_CUDA;
        }
        const int need = (int)(2 * 128 * kFlRegsSoft + 128 * kFlRegsProd);
        ready[dev].store(fa.numRegs * kFlThreads >= need ? 1 : -1);
    }
    if (ready[dev].load() != 1) {
        set_error("%s: attention kernel built with too few registers per thread", what);
        return RS_ERR_CUDA;
    }
    launch_pdl(flash_kernel<D, BF16>, dim3(a.grid), dim3(kFlThreads), FlSmem<D>::kTotal, st, a, tmq, tmk, tmv);
    RS_CHECK_LAUNCH(what);
    launch_full(flash_combine<D, BF16>, dim3(std::max(a.grid - 1, 1), a.comb_blocks), dim3(kFlCombThreads), 0, st, a);
    RS_CHECK_LAUNCH(what);
    return RS_OK;
}

template <bool BF16>
rs_status flash_launch(const FlashArgs &a, int D, const CUtensorMap &tmq, const CUtensorMap &tmk, const CUtensorMap &tmv,
                       const char *what, cudaStream_t st) {
    return D == 128 ? flash_launch_d<128, BF16>(a, tmq, tmk, tmv, what, st)
                    : flash_launch_d<64, BF16>(a, tmq, tmk, tmv, what, st);
}

}  // namespace rs
