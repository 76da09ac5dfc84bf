// flash_run.cuh -- launches of the attention core for one 16-bit type
// (included by one source file per type, so that they compile side by side).
#pragma once

#include <atomic>

#include "common.cuh"
#include "flash.cuh"

namespace rs {

// flash_combine: joins the pieces of the segments that the shares' ends cut.
// Block (c, y) looks at where CTA c's share of phase y / 8 starts; if that is
// inside a segment, and the first cut of it, the block joins 32 of its rows: a
// warp takes a row at a time, its lanes the pieces' (m, l) first and then the
// columns, so that the loads of all pieces are under way together.
//     M = max m_p, L = sum 2^(m_p - M) l_p, O = sum 2^(m_p - M) O_p / L
// It also empties the rows of rejected requests (after the pieces' writers).
constexpr int kFlCombThreads = 256;
constexpr int kFlCombRows = 32;

template <int D, bool BF16>
__global__ void __launch_bounds__(kFlCombThreads)
flash_combine(FlashArgs a) {
    pdl_enter();
    __shared__ int s_slot[kAttnMaxGrid + 2];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int blocks = gridDim.x * gridDim.y;
    for (int b = blockIdx.y * gridDim.x + blockIdx.x; b < a.B; b += blocks) {
        if (!(a.status[b] & ~RS_ST_TIMEOUT)) continue;
        const int n0 = a.off[b], n = a.off[b + 1] - n0;
        if (n0 < 0 || n < 0 || (long long)n0 + n > a.T) continue;
        const long long rows = (long long)n * a.Hq;
        uint4 *o = reinterpret_cast<uint4 *>(a.out + (long long)n0 * a.Hq * D);
        for (long long i = threadIdx.x; i < rows * (D / 8); i += kFlCombThreads) o[i] = make_uint4(0, 0, 0, 0);
        for (long long i = threadIdx.x; i < rows; i += kFlCombThreads) a.lse[(long long)n0 * a.Hq + i] = 0.f;
    }
    const int f = blockIdx.y / (kFlRows / kFlCombRows), y = blockIdx.y % (kFlRows / kFlCombRows);
    const int4 *bound = a.bound + f * (a.grid + 1);
    const int c = blockIdx.x + 1;
    if (c >= a.grid) return;
    const int4 at = bound[c], before = bound[c - 1];
    auto same = [&](int4 p) { return p.x == at.x && p.y == at.y && p.z > 0; };
    if (at.z == 0 || same(before)) return;  // between segments, or not the first cut
    const int2 e = a.ent[at.y];
    const int4 rq = a.req[e.x];
    if (a.status[e.x] & ~RS_ST_TIMEOUT) return;
    const int x = y * kFlCombRows / kBM;  // row tile of the block's rows
    const int first = (e.y * 2 + x) * a.tq, r0 = y * kFlCombRows - x * kBM;
    if (r0 / a.G >= a.tq || first + r0 / a.G >= rq.y) return;
    int np = 1;
    for (int c1 = c; c1 < a.grid; ++c1) {  // every thread counts; thread 0 writes
        const int4 p = bound[c1], q = bound[c1 + 1];
        if (!same(p)) break;
        if (same(q) && q.z == p.z) continue;  // an empty share
        if (threadIdx.x == 0) s_slot[np] = 2 * (f * a.grid + c1);
        ++np;
    }
    if (threadIdx.x == 0) s_slot[0] = 2 * (f * a.grid + c - 1) + 1;
    __syncthreads();
    const int kvh = f * a.Hkv / a.phases + at.x;
    constexpr int kC = D / 32;  // columns of a lane
    for (int k = warp; k < kFlCombRows; k += kFlCombThreads / 32) {
        const int r = r0 + k, t = r / a.G, tok = first + t;
        if (t >= a.tq || tok >= rq.y) break;
        const long long row = x * kBM + r;
        float M = -INFINITY, L = 0.f, acc[kC] = {};
        for (int p0 = 0; p0 < np; p0 += 32) {
            const bool have = p0 + lane < np;
            const long long prow = have ? (long long)s_slot[p0 + lane] * kFlRows + row : 0;
            const float m = have ? a.part_m[prow] : -INFINITY, l = have ? a.part_l[prow] : 0.f;
            const float Mn = fmaxf(M, warp_max(m));
            const float old = Mn == -INFINITY ? 1.f : sm100::ex2(M - Mn);
            const float w = Mn == -INFINITY ? (have ? 1.f : 0.f) : sm100::ex2(m - Mn);
            L = L * old + warp_sum(have ? w * l : 0.f);
#pragma unroll
            for (int i = 0; i < kC; ++i) acc[i] *= old;
            M = Mn;
            const int cnt = min(32, np - p0);
#pragma unroll 8
            for (int p = 0; p < cnt; ++p) {
                const float wp = __shfl_sync(0xffffffffu, w, p);
                const float *o = a.part_o + ((long long)s_slot[p0 + p] * kFlRows + row) * D + lane * kC;
                if (kC == 4) {
                    const float4 v = *reinterpret_cast<const float4 *>(o);
                    acc[0] = fmaf(wp, v.x, acc[0]);
                    acc[1] = fmaf(wp, v.y, acc[1]);
                    acc[kC - 2] = fmaf(wp, v.z, acc[kC - 2]);
                    acc[kC - 1] = fmaf(wp, v.w, acc[kC - 1]);
                } else {
                    const float2 v = *reinterpret_cast<const float2 *>(o);
                    acc[0] = fmaf(wp, v.x, acc[0]);
                    acc[1] = fmaf(wp, v.y, acc[1]);
                }
            }
        }
        const float fr = L > 0.f ? 1.f / L : L;  // no key with weight: 0; NaN stays
        const long long orow = (long long)(rq.x + tok) * a.Hq + kvh * a.G + (r - t * a.G);
        uint32_t *d = reinterpret_cast<uint32_t *>(a.out + orow * D + lane * kC);
#pragma unroll
        for (int i = 0; i < kC / 2; ++i) d[i] = pack16<BF16>(acc[2 * i] * fr, acc[2 * i + 1] * fr);
        if (lane == 0) a.lse[orow] = L > 0.f ? (M + log2f(L)) * 0.6931471805599453f : (L == 0.f ? -INFINITY : L);
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
    launch_full(flash_combine<D, BF16>, dim3(a.grid, a.phases * (kFlRows / kFlCombRows)), dim3(kFlCombThreads), 0, st, a);
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
