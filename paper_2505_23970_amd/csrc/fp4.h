// Elements of 4-bit pools (device code shared by the append, the read and the attention over them).
//
// The 32 consecutive elements of a block (of one token's head) share the scale s = 2^(c - 127), held as its
// exponent code c in one byte, and are E2M1 codes in units of s: sign, two exponent bits, one mantissa bit,
// magnitudes 0, 0.5, 1, 1.5, 2, 3, 4, 6. Element 2i of a row is the low half of byte i. s is the least power
// of two with A < 7 s for the block's largest magnitude A: A / s lies in [3.5, 7), so that the largest
// element, which rounds to 4 or 6, is off by at most s (a half step there), and no other rule keeps that
// with a smaller s. With s rounded down (A / s up to 8) the largest is off by up to 2 s; with A <= 6 s a
// block of A / s just above 6 gives half of its resolution away. A block that is read and appended again
// keeps its codes, since its largest is 4 s or 6 s then.
// c lies in [3, 252]: every code's value is a normal bf16 number, which widening gives exactly. c = 255: the
// block held a NaN, and its elements are NaN.
#pragma once
#include "gc_internal.h"

namespace gc {
namespace {

typedef __bf16 fp4_bf16x2 __attribute__((ext_vector_type(2)));

constexpr int kFp4Block = 32;
constexpr uint32_t kFp4Nan = 255;

// Scale code of a block by its largest magnitude's bits (fp32; a NaN's are above infinity's).
__device__ __forceinline__ uint32_t fp4_scale_code(uint32_t top) {
    // (a quarter of the mantissa's range carries from 1.75 on: floor(log2(top)) - 2, one more from 7 s on)
    const int c = (int)((top + 0x00200000u) >> 23) - 2;
    return top > 0x7F800000u ? kFp4Nan : (uint32_t)min(max(c, 3), 252);
}
// The scale as a float; NaN blocks: infinity, which the conversions below take for a NaN.
__device__ __forceinline__ float fp4_scale(uint32_t code) { return __uint_as_float(code << 23); }

// Eight elements of a block as eight codes.
__device__ __forceinline__ uint32_t fp4_quantise8(const float (&x)[8], uint32_t code) {
    const float s = fp4_scale(code);
    uint32_t w = 0;
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[0], x[1], s, 0);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[2], x[3], s, 1);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[4], x[5], s, 2);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[6], x[7], s, 3);
    return code == kFp4Nan ? 0u : w;
}

// Eight codes (one word) as eight bf16 values (four words).
__device__ __forceinline__ void fp4_widen8(uint32_t w, float s, uint32_t (&to)[4]) {
    to[0] = __builtin_bit_cast(uint32_t, (fp4_bf16x2)__builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, s, 0));
    to[1] = __builtin_bit_cast(uint32_t, (fp4_bf16x2)__builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, s, 1));
    to[2] = __builtin_bit_cast(uint32_t, (fp4_bf16x2)__builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, s, 2));
    to[3] = __builtin_bit_cast(uint32_t, (fp4_bf16x2)__builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, s, 3));
}

// Maximum of x over the four lanes of a quad.
__device__ __forceinline__ uint32_t quad_max(uint32_t x) {
    x = max(x, (uint32_t)__builtin_amdgcn_mov_dpp((int)x, 0xB1, 0xF, 0xF, true));  // lanes 1 0 3 2
    return max(x, (uint32_t)__builtin_amdgcn_mov_dpp((int)x, 0x4E, 0xF, 0xF, true));  // lanes 2 3 0 1
}

// Eight elements of a token's key and of its value, chunk c of the row (four lanes hold a block), into its slot: codes, and by
// the first of the four lanes the block's scales. All lanes of a wavefront call it, those that store nothing with ok false.
template <int D>
__device__ __forceinline__ void fp4_store(uint8_t* k_pool, uint8_t* v_pool, uint8_t* scales, int64_t slot, int c,
                                          const float (&k)[8], const float (&v)[8], bool ok) {
    uint32_t kt = 0, vt = 0;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        kt = max(kt, __float_as_uint(k[j]) & 0x7FFFFFFFu);
        vt = max(vt, __float_as_uint(v[j]) & 0x7FFFFFFFu);
    }
    const uint32_t ks = fp4_scale_code(quad_max(kt)), vs = fp4_scale_code(quad_max(vt));
    if (!ok) return;
    *reinterpret_cast<uint32_t*>(k_pool + slot * (D / 2) + c * 4) = fp4_quantise8(k, ks);
    *reinterpret_cast<uint32_t*>(v_pool + slot * (D / 2) + c * 4) = fp4_quantise8(v, vs);
    if (c % 4 == 0) *reinterpret_cast<uint16_t*>(scales + (slot * (D / kFp4Block) + c / 4) * 2) = (uint16_t)(ks | vs << 8);
}

}  // namespace
}  // namespace gc
