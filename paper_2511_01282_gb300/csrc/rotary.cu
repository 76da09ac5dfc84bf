// rotary.cu -- rs_rotary: queries and keys turned by their positions.
#include <math.h>

#include <algorithm>

#include "common.cuh"

namespace rs {
namespace {

constexpr int kRotThreads = 256;
constexpr int kRotTokens = 8;      // tokens of a block at most
constexpr int kRotMaxHalf = 256;   // pairs of a head at most

struct RotaryArgs {
    const uint16_t *in[2];  // queries, keys
    uint16_t *out[2];
    long long in_stride[2], out_stride[2];
    int heads[2];
    const int32_t *pos;
    const unsigned long long *turns;
    int T, D, half, interleaved, tokens, copy;  // copy: some output is not its input
    float scale, sign;
};

template <bool BF16>
__device__ __forceinline__ float2 unpack16(uint32_t x) {
    if (BF16) return make_float2(__uint_as_float(x << 16), __uint_as_float(x & 0xffff0000u));
    float lo, hi;
    asm("{\n\t.reg .b16 a, b;\n\tmov.b32 {a, b}, %2;\n\tcvt.f32.f16 %0, a;\n\tcvt.f32.f16 %1, b;\n\t}" : "=f"(lo), "=f"(hi) : "r"(x));
    return make_float2(lo, hi);
}
template <bool BF16>
__device__ __forceinline__ uint32_t pack16(float lo, float hi) {
    uint32_t r;
    if (BF16) asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    else asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}

// (cos, sin) of pos x freq, times the magnitude.  turns is freq / 2 pi as a 64-bit
// fraction: the product's low 64 bits are the angle's fraction of a turn, exactly,
// for every 32-bit position.  Its upper half as a signed number is within half a
// turn, so that fp32 is off by 2^-24 of at most pi before the sine.
__device__ __forceinline__ float2 turn(const RotaryArgs &a, int pos, int pair) {
    const unsigned long long f = (unsigned long long)(long long)pos * a.turns[pair];
    float s, c;
    sincospif((float)(int)(f >> 32) * 0x1p-31f, &s, &c);
    return make_float2(c * a.scale, s * a.scale * a.sign);
}

// Row r of a block's tokens: token by token, the query heads and then the key heads.
struct RotaryRow {
    const uint16_t *in;
    uint16_t *out;
    int token;  // of the block
};
__device__ __forceinline__ RotaryRow row_of(const RotaryArgs &a, int t0, int r) {
    const int H = a.heads[0] + a.heads[1];
    RotaryRow w;
    w.token = r / H;
    int h = r - w.token * H;
    const int x = h >= a.heads[0];
    if (x) h -= a.heads[0];
    w.in = (x ? a.in[1] : a.in[0]) + (t0 + w.token) * (x ? a.in_stride[1] : a.in_stride[0]) + (long long)h * a.D;
    w.out = (x ? a.out[1] : a.out[0]) + (t0 + w.token) * (x ? a.out_stride[1] : a.out_stride[0]) + (long long)h * a.D;
    return w;
}

// Pairs (x, y) become (x c - y s, y c + x s).  A block takes a few tokens: their
// cosines and sines once into shared memory, then a thread turns a 16-byte word of a
// head (four pairs side by side) or two half a turned part apart (eight pairs), or
// copies a word of the part that is not turned.  blockDim.x: the words of one head; the
// rows (token, head) run along blockDim.y, several to a thread at once.
// kKind 0: halves, their size a multiple of 8; 1: interleaved; 2: halves of other sizes,
// whose pairs lie in different places of their words: rows go through shared memory.
// Bound: 4 (Hq + Hkv) D bytes a token: 16384 tokens of 32 + 8 heads of 128, 336 MB, in 52
// (halves) and 54 us (interleaved), 6.4 TB/s; 64 tokens 2.0 us, the launch.
template <bool BF16, int kKind>
__global__ void __launch_bounds__(kRotThreads, 5)
rotary_kernel(RotaryArgs a) {
    pdl_enter();
    // kinds 0 and 1: word q of unit c at [token][q C + c], (cos, sin) of pairs 2 q and 2 q + 1 of its own
    __shared__ float4 s_turn[kRotTokens * kRotMaxHalf / 2];
    constexpr int kPairs = kKind == 0 ? 8 : 4;  // of a unit
    const int tid = threadIdx.y * blockDim.x + threadIdx.x, threads = blockDim.x * blockDim.y;
    const int t0 = blockIdx.x * a.tokens, tokens = min(a.tokens, a.T - t0);
    const int C = (a.half + kPairs - 1) / kPairs;  // (kind 1: the last one may be turned in part)
    const int pitch = kKind < 2 ? C * kPairs : a.half;
    for (int i = tid; i < tokens * a.half; i += threads) {
        const int t = i / a.half, p = i - t * a.half;
        const float2 v = turn(a, a.pos[t0 + t], p);
        float2 *row = reinterpret_cast<float2 *>(s_turn) + t * pitch;
        row[kKind < 2 ? (p % kPairs / 2 * C + p / kPairs) * 2 + (p & 1) : p] = v;
    }
    __syncthreads();
    const int rows = tokens * (a.heads[0] + a.heads[1]);
    const int first = blockIdx.y * blockDim.y + threadIdx.y, step = gridDim.y * blockDim.y;
    if constexpr (kKind < 2) {
        constexpr int kWords = kKind == 0 ? 2 : 1, kRows = 4 / kWords;  // words of a unit, rows at a time
        const int unit = threadIdx.x;
        const bool turned = unit < C;
        // the unit's words in a row (the part that is not turned has one each)
        const int at0 = turned || kKind == 1 ? unit : unit + C, at1 = C + unit;
        for (int r = first; r < rows; r += kRows * step) {
            uint4 x[kRows][kWords];
            RotaryRow w[kRows];
#pragma unroll
            for (int k = 0; k < kRows; ++k)
                if (r + k * step < rows) {
                    w[k] = row_of(a, t0, r + k * step);
                    const uint4 *in = reinterpret_cast<const uint4 *>(w[k].in);
                    x[k][0] = in[at0];
                    if (kKind == 0 && turned) x[k][kWords - 1] = in[at1];
                }
#pragma unroll
            for (int k = 0; k < kRows; ++k)
                if (r + k * step < rows) {
                    uint4 *out = reinterpret_cast<uint4 *>(w[k].out);
                    if (!turned) {
                        out[at0] = x[k][0];
                        continue;
                    }
                    const float4 *cs = s_turn + w[k].token * (pitch / 2) + unit;
                    uint32_t u[4] = {x[k][0].x, x[k][0].y, x[k][0].z, x[k][0].w};
                    if constexpr (kKind == 1) {
#pragma unroll
                        for (int q = 0; q < 2; ++q) {
                            const float4 c = cs[q * C];
                            const float2 p0 = unpack16<BF16>(u[2 * q]), p1 = unpack16<BF16>(u[2 * q + 1]);
                            const int pair = 4 * unit + 2 * q;
                            if (pair < a.half) u[2 * q] = pack16<BF16>(fmaf(p0.x, c.x, -p0.y * c.y), fmaf(p0.y, c.x, p0.x * c.y));
                            if (pair + 1 < a.half) u[2 * q + 1] = pack16<BF16>(fmaf(p1.x, c.z, -p1.y * c.w), fmaf(p1.y, c.z, p1.x * c.w));
                        }
                    } else {
                        uint32_t v[4] = {x[k][kWords - 1].x, x[k][kWords - 1].y, x[k][kWords - 1].z, x[k][kWords - 1].w};
#pragma unroll
                        for (int q = 0; q < 4; ++q) {
                            const float4 c = cs[q * C];
                            const float2 p = unpack16<BF16>(u[q]), o = unpack16<BF16>(v[q]);
                            u[q] = pack16<BF16>(fmaf(p.x, c.x, -o.x * c.y), fmaf(p.y, c.z, -o.y * c.w));
                            v[q] = pack16<BF16>(fmaf(o.x, c.x, p.x * c.y), fmaf(o.y, c.z, p.y * c.w));
                        }
                        out[at1] = make_uint4(v[0], v[1], v[2], v[3]);
                    }
                    out[at0] = make_uint4(u[0], u[1], u[2], u[3]);
                }
        }
    } else {
        __shared__ uint4 s_row[kRotThreads];
        const float2 *s_pair = reinterpret_cast<const float2 *>(s_turn);
        const int unit = threadIdx.x, rot = 2 * a.half;
        for (int base = blockIdx.y * blockDim.y; base < rows; base += step) {
            const bool on = base + (int)threadIdx.y < rows;
            RotaryRow w;
            uint4 x = make_uint4(0, 0, 0, 0);
            if (on) {
                w = row_of(a, t0, base + threadIdx.y);
                x = reinterpret_cast<const uint4 *>(w.in)[unit];
                s_row[tid] = x;
            }
            __syncthreads();  // all of the rows is there before any of it is written
            if (on) {
                const uint16_t *row = reinterpret_cast<const uint16_t *>(s_row + threadIdx.y * blockDim.x);
                uint32_t u[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const float2 p = unpack16<BF16>(u[q]);
                    float y[2] = {p.x, p.y};
                    bool turned[2];
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        const int i = 8 * unit + 2 * q + e;
                        turned[e] = i < rot;
                        if (!turned[e]) continue;
                        const int pair = i < a.half ? i : i - a.half;
                        const float2 cs = s_pair[w.token * a.half + pair];
                        const float o = unpack16<BF16>(row[i < a.half ? i + a.half : pair]).x;
                        y[e] = i < a.half ? fmaf(y[e], cs.x, -o * cs.y) : fmaf(y[e], cs.x, o * cs.y);
                    }
                    const uint32_t v = pack16<BF16>(y[0], y[1]);
                    u[q] = __byte_perm(u[q], v, (turned[0] ? 0x54 : 0x10) | (turned[1] ? 0x7600 : 0x3200));
                }
                reinterpret_cast<uint4 *>(w.out)[unit] = make_uint4(u[0], u[1], u[2], u[3]);
            }
            __syncthreads();
        }
    }
}

template <bool BF16>
void launch_rotary(const RotaryArgs &a, int kind, dim3 grid, dim3 block, cudaStream_t s) {
    if (kind == 0) launch_pdl(rotary_kernel<BF16, 0>, grid, block, 0, s, a);
    else if (kind == 1) launch_pdl(rotary_kernel<BF16, 1>, grid, block, 0, s, a);
    else launch_pdl(rotary_kernel<BF16, 2>, grid, block, 0, s, a);
}

rs_status check_rows(const char *what, const char *name, const void *p, int64_t stride, int heads, int D) {
    RS_CHECK_ARG((reinterpret_cast<uintptr_t>(p) & 15) == 0, "%s: %s must be 16-byte aligned", what, name);
    RS_CHECK_ARG(stride >= (int64_t)heads * D && stride % 8 == 0 && stride < (1ll << 38),
                 "%s: %s rows of %lld elements: at least heads x D, a multiple of 8", what, name, (long long)stride);
    return RS_OK;
}

}  // namespace
}  // namespace rs

using namespace rs;

extern "C" rs_status rs_rotary(const uint16_t *q, int64_t q_stride, uint16_t *q_out, int64_t q_out_stride, const uint16_t *k,
                               int64_t k_stride, uint16_t *k_out, int64_t k_out_stride, int dtype, const int32_t *pos, int T,
                               int Hq, int Hkv, int D, int rot, int layout, const uint64_t *turns, float scale, int inverse,
                               void *stream) {
    clear_error();
    const char *what = "rs_rotary";
    RS_CHECK_ARG(T >= 0 && T <= 1 << 30, "%s: T=%d out of range (0 to 2^30)", what, T);
    RS_CHECK_ARG(dtype == RS_BF16 || dtype == RS_F16, "%s: dtype %d is neither RS_BF16 nor RS_F16", what, dtype);
    RS_CHECK_ARG(Hq >= 0 && Hkv >= 0 && Hq <= 65536 && Hkv <= 65536, "%s: Hq=%d, Hkv=%d out of range", what, Hq, Hkv);
    if (D < 8 || D > 2 * kRotMaxHalf || D % 8) {
        set_error("%s: head dim %d unsupported (a multiple of 8, up to %d)", what, D, 2 * kRotMaxHalf);
        return RS_ERR_UNSUPPORTED;
    }
    RS_CHECK_ARG(rot >= 2 && rot <= D && rot % 2 == 0, "%s: rot=%d: an even number from 2 to %d", what, rot, D);
    RS_CHECK_ARG(layout == RS_ROTARY_HALF || layout == RS_ROTARY_INTERLEAVED, "%s: layout %d unknown", what, layout);
    RS_CHECK_ARG(isfinite(scale), "%s: scale must be finite", what);
    RS_CHECK_ARG(T == 0 || (pos && turns), "%s: null pointer", what);
    RS_CHECK_ARG(T == 0 || Hq == 0 || (q && q_out), "%s: null row pointer (q)", what);
    RS_CHECK_ARG(T == 0 || Hkv == 0 || (k && k_out), "%s: null row pointer (k)", what);
    rs_status st;
    if (Hq > 0) {
        if ((st = check_rows(what, "q", q, q_stride, Hq, D)) != RS_OK) return st;
        if ((st = check_rows(what, "q_out", q_out, q_out_stride, Hq, D)) != RS_OK) return st;
        RS_CHECK_ARG(q != q_out || q_stride == q_out_stride, "%s: q in place with another distance between rows", what);
    }
    if (Hkv > 0) {
        if ((st = check_rows(what, "k", k, k_stride, Hkv, D)) != RS_OK) return st;
        if ((st = check_rows(what, "k_out", k_out, k_out_stride, Hkv, D)) != RS_OK) return st;
        RS_CHECK_ARG(k != k_out || k_stride == k_out_stride, "%s: k in place with another distance between rows", what);
    }
    if (T == 0 || Hq + Hkv == 0) return RS_OK;
    RotaryArgs a{};
    a.in[0] = q;
    a.in[1] = k;
    a.out[0] = q_out;
    a.out[1] = k_out;
    a.in_stride[0] = q_stride;
    a.in_stride[1] = k_stride;
    a.out_stride[0] = q_out_stride;
    a.out_stride[1] = k_out_stride;
    a.heads[0] = Hq;
    a.heads[1] = Hkv;
    a.pos = pos;
    a.turns = reinterpret_cast<const unsigned long long *>(turns);
    a.T = T;
    a.D = D;
    a.half = rot / 2;
    a.interleaved = layout == RS_ROTARY_INTERLEAVED;
    a.copy = (Hq > 0 && q != q_out) || (Hkv > 0 && k != k_out);
    a.scale = scale;
    a.sign = inverse ? -1.f : 1.f;
    // a few tokens to a block where there are enough for all SMs, one and several blocks
    // along its heads where there are not
    const int sms = num_sms(), H = Hq + Hkv;
    a.tokens = std::min(std::max(T / (4 * sms), 1), kRotTokens);
    const long long blocks = ((long long)T + a.tokens - 1) / a.tokens;
    // words of a head that a row needs: half as many units where they come in twos
    const int kind = a.interleaved ? 1 : a.half % 8 ? 2 : 0, turned = kind == 0 ? a.half / 8 : (rot + 7) / 8;
    const int x = turned + (a.copy ? D / 8 - (kind == 0 ? 2 : 1) * turned : 0);
    const dim3 block((unsigned)x, (unsigned)std::max(kRotThreads / x, 1));
    const long long rows = (long long)a.tokens * H;
    const long long most = (rows + block.y - 1) / block.y;
    const dim3 grid((unsigned)blocks, (unsigned)std::max(1ll, std::min(most, 2ll * sms / blocks)));
    const cudaStream_t s = (cudaStream_t)stream;
    if (dtype == RS_BF16) launch_rotary<true>(a, kind, grid, block, s);
    else launch_rotary<false>(a, kind, grid, block, s);
    RS_CHECK_LAUNCH(what);
    return RS_OK;
}
