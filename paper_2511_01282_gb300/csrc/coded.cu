// coded.cu -- rs_coded_append: keys and values of new tokens into the pages of
// an 8-bit cache.
#include "coded.cuh"
#include "tmap.cuh"

namespace rs {
namespace {

struct CodedAppendArgs {
    const uint16_t *k, *v;
    long long k_stride, v_stride;
    const int32_t *off;
    CodedPool c;
    int32_t *status;
    int B, T, Hkv;
};

template <bool BF16>
__device__ __forceinline__ float2 unpack16(uint32_t x) {
    if (BF16) return make_float2(__uint_as_float(x << 16), __uint_as_float(x & 0xffff0000u));
    return __half22float2(*reinterpret_cast<const __half2 *>(&x));
}

__device__ __forceinline__ uint32_t max2(uint32_t a, uint32_t b) {
    uint32_t r;
    asm("max.u16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
}
__device__ __forceinline__ uint32_t pick(const uint4 &v, int i) { return i == 0 ? v.x : i == 1 ? v.y : i == 2 ? v.z : v.w; }

// Two values times 2^k as codes.  fp16 multiplies in its own type: what loses bits among
// its subnormals is below 2^-14, far from the smallest code's half, 2^-10.
template <bool BF16>
struct Scaled {
    uint32_t two_k;
    __device__ __forceinline__ explicit Scaled(int k) : two_k(BF16 ? (uint32_t)(k + 127) << 23 : (uint32_t)(k + 15) * 0x04000400u) {}
    __device__ __forceinline__ uint32_t operator()(uint32_t x) const {
        uint32_t c;
        if (BF16) {
            const float2 v = mul2(unpack16<true>(x), make_float2(__uint_as_float(two_k), __uint_as_float(two_k)));
            return encode2(v.x, v.y);
        }
        asm("{\n\t.reg .b16 c;\n\t.reg .b32 h;\n\tmul.rn.f16x2 h, %1, %2;\n\tcvt.rn.satfinite.e4m3x2.f16x2 c, h;\n\tcvt.u32.u16 %0, c;\n\t}"
            : "=r"(c)
            : "r"(x), "r"(two_k));
        return c;
    }
};

// One block of 16 slots, one head, one of K and V: x holds the new tokens' values,
// 8 of a token's D in each lane (lanes' tokens: kTok a step).  A warp.
//   e = least exponent with max |x| <= 448 2^e over the new finite values, within the
//       type's range, and at least the old one where tokens before `lo` stay
//   code = e4m3(x 2^-e); the old tokens' codes shift by the difference
template <int D, bool BF16, int kSteps>
__device__ __forceinline__ void code_block(const uint4 (&x)[kSteps], uint8_t *codes, int8_t *exp, int row_bytes, int old_tokens,
                                           int lo, int hi) {
    constexpr int kLanes = D / 8, kTok = 32 / kLanes;
    const int lane = threadIdx.x & 31, part = lane % kLanes, tok = lane / kLanes;
    // |x| as 15-bit integers, two at a time, are ordered as the values; infinities and NaN come last
    constexpr uint32_t kInf = BF16 ? 0x7f80u : 0x7c00u;
    uint32_t most2 = 0;
#pragma unroll
    for (int u = 0; u < kSteps; ++u) {
        most2 = max2(most2, x[u].x & 0x7fff7fffu);
        most2 = max2(most2, x[u].y & 0x7fff7fffu);
        most2 = max2(most2, x[u].z & 0x7fff7fffu);
        most2 = max2(most2, x[u].w & 0x7fff7fffu);
    }
    uint32_t most16 = __reduce_max_sync(0xffffffffu, max(most2 & 0xffffu, most2 >> 16));
    const bool odd = most16 >= kInf;  // some are not finite
    if (odd) {
        most16 = 0;
#pragma unroll
        for (int u = 0; u < kSteps; ++u) {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const uint32_t v = pick(x[u], i >> 1) >> (i & 1 ? 16 : 0) & 0x7fffu;
                most16 = max(most16, v < kInf ? v : 0u);
            }
        }
        most16 = __reduce_max_sync(0xffffffffu, most16);
    }
    const uint32_t most = __float_as_uint(unpack16<BF16>(most16).x);
    // 448 = 1.75 x 2^8
    int e = code_exp((int)(most >> 23) - 127 - 8 + ((most & 0x7fffffu) > 0x600000u), BF16);
    if (old_tokens > 0) {
        const int before = code_exp(*exp, BF16);
        __syncwarp();  // all have read it
        if (e > before) {
            const float f = pow2i(-min(e - before, 100));  // smaller ones are 0 either way
            for (int t = tok; t < old_tokens; t += kTok) {
                uint2 *p = reinterpret_cast<uint2 *>(codes + (long long)t * row_bytes) + part;
                uint2 c = *p;
                uint32_t *w = &c.x;
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    uint32_t a, b;
                    decode4(w[i], a, b);
                    const float2 g = unpack16<false>(a), h = unpack16<false>(b);
                    w[i] = encode2(g.x * f, g.y * f) | encode2(h.x * f, h.y * f) << 16;
                }
                *p = c;
            }
        } else {
            e = before;
        }
    }
    if (odd || e == code_exp_max(BF16)) {  // not finite: NaN; at the largest exponent: no code above 240
        const float f = pow2i(-e);
#pragma unroll
        for (int u = 0; u < kSteps; ++u) {
            const int t = u * kTok + tok;
            if (t < lo || t >= hi) continue;
            uint32_t c[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                float2 g = unpack16<BF16>(pick(x[u], i));
                g.x = fabsf(g.x) == INFINITY ? NAN : g.x * f;
                g.y = fabsf(g.y) == INFINITY ? NAN : g.y * f;
                if (e == code_exp_max(BF16)) {
                    if (fabsf(g.x) > 240.f) g.x = copysignf(240.f, g.x);
                    if (fabsf(g.y) > 240.f) g.y = copysignf(240.f, g.y);
                }
                c[i] = encode2(g.x, g.y);
            }
            *(reinterpret_cast<uint2 *>(codes + (long long)t * row_bytes) + part) = make_uint2(c[0] | c[1] << 16, c[2] | c[3] << 16);
        }
    } else {
        const Scaled<BF16> scaled(-e);
#pragma unroll
        for (int u = 0; u < kSteps; ++u) {
            const int t = u * kTok + tok;
            if (t < lo || t >= hi) continue;
            *(reinterpret_cast<uint2 *>(codes + (long long)t * row_bytes) + part) =
                make_uint2(scaled(x[u].x) | scaled(x[u].y) << 16, scaled(x[u].z) | scaled(x[u].w) << 16);
        }
    }
    if (lane == 0) *exp = (int8_t)e;
}

// A warp per (block of 16 slots that gets new tokens, K or V, head; several heads one after
// the other where there are blocks enough for all SMs).  Blocks are numbered
// without a prefix over the requests: request b's start at off[b] / 16 + 2 b, which
// leaves room for the n / 16 + 2 that its n tokens fall into at most.
// Bound: 6 Hkv D bytes a token, read in 16 and written in 8 bits: 34000 tokens of 8 heads, 209 MB, in
// 33 us, 6.3 TB/s (with the maximum and the products value by value in fp32 72 us, instructions); single
// tokens of 16 requests 3.6 us in a graph, the launch and four dependent reads (10.5 called from Python).
constexpr int kCodeThreads = 256;

template <int D, bool BF16>
__global__ void __launch_bounds__(kCodeThreads, 4)
coded_append(CodedAppendArgs a) {
    pdl_enter();
    constexpr int kLanes = D / 8, kTok = 32 / kLanes, kSteps = kCodeBlock / kTok;
    const CodedPool &c = a.c;
    const int lane = threadIdx.x & 31;
    const int w0 = blockIdx.x * (kCodeThreads / 32) + (threadIdx.x >> 5), warps = gridDim.x * (kCodeThreads / 32);
    const long long room = (long long)c.max_pages << c.page_log2;
    // offsets that decrease anywhere belong to no batch: every request is rejected
    int bad = 0;
    for (int b = lane; b < a.B; b += 32) bad |= a.off[b] > a.off[b + 1];
    const bool ordered = !__any_sync(0xffffffffu, bad) && a.off[0] >= 0 && a.off[a.B] <= a.T;
    if (blockIdx.y == 0 && blockIdx.z == 0) {
        for (int b = w0; b < a.B; b += warps) {  // a warp per request: its slots and their pages
            const int n = a.off[b + 1] - a.off[b], ctx = c.ctx[b];
            int st = 0;
            if (!ordered || ctx < 0 || (long long)ctx + n > room) {
                st = RS_ST_BAD_OFFSET;
            } else if (n > 0) {
                for (int p = (ctx >> c.page_log2) + lane; p <= (ctx + n - 1) >> c.page_log2; p += 32) {
                    const int id = c.table[(long long)b * c.max_pages + p];
                    if (id < 0 || id >= c.n_pages) st = RS_ST_BAD_PAGE;
                }
            }
            st = __reduce_or_sync(0xffffffffu, st);
            if (lane == 0) a.status[b] = st;
        }
    }
    if (!ordered) return;
    const int items = (a.T >> kCodeBlockLog2) + 2 * a.B;
    for (int j = w0; j < items; j += warps) {
        int lo = 0, hi = a.B;  // last b with off[b] / 16 + 2 b <= j
        while (hi - lo > 1) {
            const int step = (hi - lo + 31) / 32, at = lo + lane * step;
            const unsigned m = __ballot_sync(0xffffffffu, at < hi && (a.off[at] >> kCodeBlockLog2) + 2 * at <= j) | 1u;
            lo += (31 - __clz(m)) * step;
            hi = min(lo + step, hi);
        }
        const int n0 = a.off[lo], n = a.off[lo + 1] - n0, ctx = c.ctx[lo];
        if (n <= 0 || ctx < 0 || (long long)ctx + n > room) continue;
        const int i = j - ((n0 >> kCodeBlockLog2) + 2 * lo);
        const int s0 = ((ctx >> kCodeBlockLog2) + i) << kCodeBlockLog2;  // the block's first slot
        if (i < 0 || i > ((ctx + n - 1) >> kCodeBlockLog2) - (ctx >> kCodeBlockLog2)) continue;
        const int id = c.table[(long long)lo * c.max_pages + (s0 >> c.page_log2)];
        if (id < 0 || id >= c.n_pages) continue;
        const int first = max(ctx - s0, 0), last = min(ctx + n - s0, kCodeBlock);  // new tokens of the block
        const long long slot = ((long long)id << c.page_log2) + (s0 & ((1 << c.page_log2) - 1));
        const long long row0 = n0 + (long long)s0 - ctx;  // row of the block's slot 0 (which may not be there)
        const bool is_v = blockIdx.z;
        const uint16_t *rows = is_v ? a.v : a.k;
        const long long stride = is_v ? a.v_stride : a.k_stride;
        uint8_t *codes = is_v ? c.v : c.k;
        int8_t *exps = is_v ? c.ve : c.ke;
        for (int h = blockIdx.y; h < a.Hkv; h += gridDim.y) {
            uint4 x[kSteps];
            const uint16_t *src = rows + (row0 + lane / kLanes) * stride + (long long)h * D + lane % kLanes * 8;
#pragma unroll
            for (int u = 0; u < kSteps; ++u) {
                const int t = u * kTok + lane / kLanes;
                x[u] = make_uint4(0, 0, 0, 0);
                if (t >= first && t < last) x[u] = *reinterpret_cast<const uint4 *>(src + u * kTok * stride);
            }
            code_block<D, BF16>(x, codes + (slot * a.Hkv + h) * D, exps + (slot >> kCodeBlockLog2) * a.Hkv + h, a.Hkv * D, first, first, last);
        }
    }
}

}  // namespace
}  // namespace rs

using namespace rs;

extern "C" rs_status rs_coded_append(const uint16_t *k, int64_t k_stride, const uint16_t *v, int64_t v_stride, int dtype,
                                     const int32_t *new_off, int B, int T, int Hkv, int D, uint8_t *k_codes, uint8_t *v_codes,
                                     int8_t *k_exps, int8_t *v_exps, int n_pages, int page_size, const int32_t *page_table,
                                     int max_pages, const int32_t *ctx_len, int32_t *status, void *stream) {
    clear_error();
    const char *what = "rs_coded_append";
    RS_CHECK_ARG(B >= 0 && T >= 0, "%s: negative size", what);
    RS_CHECK_ARG(dtype == RS_BF16 || dtype == RS_F16, "%s: dtype %d is neither RS_BF16 nor RS_F16", what, dtype);
    RS_CHECK_ARG(T <= 1 << 30, "%s: T=%d above 2^30", what, T);
    RS_CHECK_ARG(B <= 1 << 28, "%s: B=%d above 2^28", what, B);  // block numbers stay an int
    if (D != 64 && D != 128) {
        set_error("%s: head dim %d unsupported (64 or 128)", what, D);
        return RS_ERR_UNSUPPORTED;
    }
    RS_CHECK_ARG(Hkv >= 1 && Hkv <= 65535, "%s: Hkv=%d out of range", what, Hkv);
    const rs_status st = check_coded_pages(what, n_pages, page_size, max_pages);
    if (st != RS_OK) return st;
    RS_CHECK_ARG(B == 0 || (new_off && ctx_len && status && (page_table || max_pages == 0)), "%s: null request pointer", what);
    RS_CHECK_ARG(T == 0 || (k && v), "%s: null row pointer", what);
    RS_CHECK_ARG(n_pages == 0 || (k_codes && v_codes && k_exps && v_exps), "%s: null page pointer", what);
    RS_CHECK_ARG((((uintptr_t)k | (uintptr_t)v | (uintptr_t)k_codes | (uintptr_t)v_codes) & 15) == 0,
                 "%s: k, v and pages must be 16-byte aligned", what);
    RS_CHECK_ARG(k_stride >= (int64_t)Hkv * D && v_stride >= (int64_t)Hkv * D && k_stride % 8 == 0 && v_stride % 8 == 0,
                 "%s: rows of k and v: at least Hkv x D elements, a multiple of 8", what);
    if (B == 0) return RS_OK;
    CodedAppendArgs a{k, v, k_stride, v_stride, new_off,
                      CodedPool{k_codes, v_codes, k_exps, v_exps, page_table, ctx_len, n_pages, page_log2(page_size), n_pages ? max_pages : 0},
                      status, B, T, Hkv};
    const long long items = (T >> kCodeBlockLog2) + 2ll * B, blocks = (items + kCodeThreads / 32 - 1) / (kCodeThreads / 32);
    // Several times the warps that the SMs hold at a time (32 each), by heads where the blocks are few; as many
    // as they hold where those would be all: a second wave costs more than a second head (44 requests of a
    // token or two, 40 heads: 9.0 us in two)
    const long long most = 2 * blocks * Hkv <= 12ll * num_sms() ? 4ll * num_sms() : 12ll * num_sms();
    const unsigned x = (unsigned)std::min(blocks, most), y = (unsigned)std::min(std::max(most / (2ll * x), 1ll), (long long)Hkv);
    const dim3 grid(x, y, 2);
    const cudaStream_t s = (cudaStream_t)stream;
    if (dtype == RS_BF16) launch_pdl(D == 128 ? coded_append<128, true> : coded_append<64, true>, grid, dim3(kCodeThreads), 0, s, a);
    else launch_pdl(D == 128 ? coded_append<128, false> : coded_append<64, false>, grid, dim3(kCodeThreads), 0, s, a);
    RS_CHECK_LAUNCH(what);
    return RS_OK;
}
