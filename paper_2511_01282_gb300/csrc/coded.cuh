// coded.cuh -- the 8-bit KV cache's number format: e4m3 codes with an exponent
// of two for each block of 16 tokens and KV head, value = code 2^e.
//
// A power of two and not any scale: codes of a floating type lose nothing by it
// (their step is relative to the value), code 2^e is exact in bf16 and, within the
// exponents that an fp16 cache has, in fp16, so that products take the values as
// they are; and when a later token raises a block's exponent the codes that are
// there shift without rounding, but for those that fall among the subnormals.
#pragma once

#include <cuda_fp16.h>
#include <stdint.h>

#include "common.cuh"

namespace rs {

constexpr int kCodeBlock = 16, kCodeBlockLog2 = 4;  // tokens that share an exponent

// Exponents that values of a type get: 2^e x code has to be representable, from the
// smallest step (2^-9 x 2^e) on.  At the largest exponent the codes stop at 240: the
// next one, 256 x 2^e, is above the type's largest value (2^16 and 2^128).
__host__ __device__ constexpr int code_exp_min(bool bf16) { return bf16 ? -117 : -15; }
__host__ __device__ constexpr int code_exp_max(bool bf16) { return bf16 ? 120 : 8; }
__device__ __forceinline__ int code_exp(int e, bool bf16) { return min(max(e, code_exp_min(bf16)), code_exp_max(bf16)); }

// 2^e for -126 <= e <= 127
__device__ __forceinline__ float pow2i(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }

// Factors of scores: towards 0, so that a product above fp32's largest number becomes it and not infinity, of which a
// score of 0 would be no number (with a minimum behind it the chunks took 450 us and not 438)
__device__ __forceinline__ float finite_mul(float a, float b) { return __fmul_rz(a, b); }

// four codes -> fp16, exact (NaN stays NaN): the low and the high two
__device__ __forceinline__ void decode4(uint32_t four, uint32_t &lo, uint32_t &hi) {
    asm("{\n\t.reg .b16 a, b;\n\tmov.b32 {a, b}, %2;\n\tcvt.rn.f16x2.e4m3x2 %0, a;\n\tcvt.rn.f16x2.e4m3x2 %1, b;\n\t}"
        : "=r"(lo), "=r"(hi)
        : "r"(four));
}
// bit 7 of every code that is NaN (0x7f and 0xff)
__device__ __forceinline__ uint32_t nan_codes(uint32_t four) { return ((four & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u; }
// the codes that are not NaN, 0 in the place of those that are
__device__ __forceinline__ uint32_t without_nan(uint32_t four) { return four & ~((nan_codes(four) >> 7) * 0xffu); }
// (lo, hi) -> two codes, to nearest even; NaN -> NaN
__device__ __forceinline__ uint32_t encode2(float lo, float hi) {
    uint32_t c;
    asm("{\n\t.reg .b16 c;\n\tcvt.rn.satfinite.e4m3x2.f32 c, %1, %2;\n\tcvt.u32.u16 %0, c;\n\t}" : "=r"(c) : "f"(hi), "f"(lo));
    return c;
}

// The pool and its page table.  Codes [n_pages, page_size, Hkv, D]; exponents
// [n_pages, page_size / 16, Hkv].
struct CodedPool {
    uint8_t *k, *v;
    int8_t *ke, *ve;
    const int32_t *table, *ctx;
    int n_pages, page_log2, max_pages;
};

}  // namespace rs
