// flash_run.cuh -- launches of the attention core for one 16-bit type
// (included by one source file per type, so that they compile side by side).
#pragma once

#include <algorithm>
#include <atomic>

#include "common.cuh"
#include "flash.cuh"

namespace rs {

// flash_combine: joins the pieces of the segments that the shares' ends cut.
// Block (c, y) looks at where CTA c + 1's share of phase y / 8 starts; if that
// is inside a segment, and the first cut of it, the block joins 32 of its rows,
// four to a warp, all loads of a step under way together:
//     M = max m_p, L = sum 2^(m_p - M) l_p, O = sum 2^(m_p - M) O_p / L
// It also empties the rows of rejected requests (after the pieces' writers).
// Bound: latency (a handful of dependent loads), and the pieces, read once
// from L2, where every share's end cuts a pair of full row tiles.
constexpr int kFlCombThreads = 256;
constexpr int kFlCombRows = 32;  // of a block
constexpr int kFlCombPar = kFlCombRows / (kFlCombThreads / 32);  // rows of a warp

template <int D, bool BF16>
__global__ void __launch_bounds__(kFlCombThreads)
flash_combine(FlashArgs a) {
    pdl_enter();
    __shared__ int s_slot[kAttnMaxGrid + 2];
    __shared__ int s_np;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int f = blockIdx.y / (kFlRows / kFlCombRows), y = blockIdx.y % (kFlRows / kFlCombRows);
    const int4 *bound = a.bound + f * (a.grid + 1);
    const int c = min((int)blockIdx.x + 1, a.grid);
    const int4 at = bound[c], before = bound[c - 1];
    const int blocks = gridDim.x * gridDim.y;
    for (int b = blockIdx.y * gridDim.x + blockIdx.x; b < a.B; b += blocks) {
        if (!(a.status[b] & ~RS_ST_TIMEOUT)) continue;
        const int4 rq = a.req[b];
        const long long rows = (long long)rq.w * a.Hq;  // none where another request may have them
        uint4 *o = reinterpret_cast<uint4 *>(a.out + (long long)rq.x * a.Hq * D);
        for (long long i = threadIdx.x; i < rows * (D / 8); i += kFlCombThreads) o[i] = make_uint4(0, 0, 0, 0);
        for (long long i = threadIdx.x; i < rows; i += kFlCombThreads) a.lse[(long long)rq.x * a.Hq + i] = 0.f;
    }
    auto same = [&](int4 p) { return p.x == at.x && p.y == at.y && p.z > 0; };
    if (c >= a.grid || at.z == 0 || same(before)) return;  // between segments, or not the first cut
    const int4 e = a.ent[at.y];  // request, pair, first row, rows
    const int x = y * kFlCombRows / kBM;  // row tile of the block's rows
    const int first = (e.y * 2 + x) * a.tq, r0 = y * kFlCombRows - x * kBM;
    if (r0 / a.G >= a.tq || first + r0 / a.G >= e.w) return;
    const bool rejected = a.status[e.x] & ~RS_ST_TIMEOUT;
    if (warp == 0) {  // the pieces' slots, in order
        if (lane == 0) s_slot[0] = 2 * (f * a.grid + c - 1) + 1;
        int np = 1;
        for (int c0 = c; c0 < a.grid; c0 += 32) {
            const int c1 = c0 + lane;
            const int4 p = bound[min(c1, a.grid)], q = bound[min(c1 + 1, a.grid)];
            const bool in = c1 < a.grid && same(p), has = in && !(same(q) && q.z == p.z);  // not an empty share
            const unsigned m = __ballot_sync(0xffffffffu, has);
            if (has) s_slot[np + __popc(m & ((1u << lane) - 1u))] = 2 * (f * a.grid + c1);
            np += __popc(m);
            if (__ballot_sync(0xffffffffu, in) != 0xffffffffu) break;
        }
        if (lane == 0) s_np = np;
    }
    __syncthreads();
    if (rejected) return;
    const int np = s_np, kvh = f * a.Hkv / a.phases + at.x;
    constexpr int kC = D / 32;  // columns of a lane
    long long row[kFlCombPar];
    int tok[kFlCombPar], hg[kFlCombPar];
    bool on[kFlCombPar];
    float M[kFlCombPar], L[kFlCombPar], acc[kFlCombPar][kC];
#pragma unroll
    for (int i = 0; i < kFlCombPar; ++i) {
        const int r = r0 + warp + i * (kFlCombThreads / 32), t = r / a.G;
        tok[i] = first + t;
        hg[i] = r - t * a.G;
        on[i] = t < a.tq && tok[i] < e.w;
        row[i] = x * kBM + r;
        M[i] = -INFINITY;
        L[i] = 0.f;
#pragma unroll
        for (int j = 0; j < kC; ++j) acc[i][j] = 0.f;
    }
    for (int p0 = 0; p0 < np; p0 += 32) {
        const bool have = p0 + lane < np;
        const long long slot = have ? (long long)s_slot[p0 + lane] * kFlRows : 0;
        float m[kFlCombPar], l[kFlCombPar], w[kFlCombPar];
#pragma unroll
        for (int i = 0; i < kFlCombPar; ++i) {
            m[i] = have && on[i] ? a.part_m[slot + row[i]] : -INFINITY;
            l[i] = have && on[i] ? a.part_l[slot + row[i]] : 0.f;
        }
#pragma unroll
        for (int i = 0; i < kFlCombPar; ++i) {
            const float Mn = fmaxf(M[i], warp_max(m[i]));
            const float old = Mn == -INFINITY ? 1.f : sm100::ex2(M[i] - Mn);
            w[i] = Mn == -INFINITY ? (have ? 1.f : 0.f) : sm100::ex2(m[i] - Mn);
            L[i] = L[i] * old + warp_sum(have ? w[i] * l[i] : 0.f);
#pragma unroll
            for (int j = 0; j < kC; ++j) acc[i][j] *= old;
            M[i] = Mn;
        }
        const int cnt = min(32, np - p0);
#pragma unroll 4
        for (int p = 0; p < cnt; ++p) {
            const long long at_slot = (long long)s_slot[p0 + p] * kFlRows;
#pragma unroll
            for (int i = 0; i < kFlCombPar; ++i) {
                const float wp = __shfl_sync(0xffffffffu, w[i], p);
                if (!on[i]) continue;
                const float *o = a.part_o + (at_slot + row[i]) * D + lane * kC;
                float v[kC];
                if constexpr (kC == 4) *reinterpret_cast<float4 *>(v) = *reinterpret_cast<const float4 *>(o);
                else *reinterpret_cast<float2 *>(v) = *reinterpret_cast<const float2 *>(o);
#pragma unroll
                for (int j = 0; j < kC; ++j) acc[i][j] = fmaf(wp, v[j], acc[i][j]);
            }
        }
    }
#pragma unroll
    for (int i = 0; i < kFlCombPar; ++i) {
        if (!on[i]) continue;
        const float fr = L[i] > 0.f ? 1.f / L[i] : L[i];  // no key with weight: 0; NaN stays
        const long long orow = (long long)(e.z + tok[i]) * a.Hq + kvh * a.G + hg[i];
        uint32_t *d = reinterpret_cast<uint32_t *>(a.out + orow * D + lane * kC);
        if constexpr (kC == 4)
            *reinterpret_cast<uint2 *>(d) = make_uint2(pack16<BF16>(acc[i][0] * fr, acc[i][1] * fr), pack16<BF16>(acc[i][2] * fr, acc[i][3] * fr));
        else
            *d = pack16<BF16>(acc[i][0] * fr, acc[i][1] * fr);
        if (lane == 0) a.lse[orow] = L[i] > 0.f ? (M[i] + log2f(L[i])) * 0.6931471805599453f : (L[i] == 0.f ? -INFINITY : L[i]);
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
    launch_full(flash_combine<D, BF16>, dim3(std::max(a.grid - 1, 1), a.phases * (kFlRows / kFlCombRows)), dim3(kFlCombThreads), 0, st, a);
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
