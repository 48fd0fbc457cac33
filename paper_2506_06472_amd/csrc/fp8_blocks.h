// Matrices stored in 8-bit floating point with a power of two for each block of 128 neighbours of a row: their layout, and the
// arithmetic of a block.
//
// A block with the largest magnitude a has the exponent e = max(min{e : a <= M 2^e}, -110), with M = 448 (e4m3) or 57344 (e5m2), both
// 1.75 times a power of two 2^k (k = 8, 15): e = floor(log2 a) - k, and one more where a's fraction is above 1.75.  An element x becomes the
// nearest code of x 2^-e, ties to even, and stands for code 2^e: |x 2^-e| <= M, so nothing is clamped.  The smallest code, 2^-16, times 2^-110 is
// the smallest normal number of 32 bits.  Blocks with an infinity or a NaN hold codes that are NaN.
//
// Layout of [rows, cols]: groups of 16 rows, ceil(rows / 16) of them, each KB = ceil(cols / 128) fragments of 2 KiB: what a wavefront's lanes
// hand to a product of 16 rows over 128 neighbours, as two 16-byte pieces of each lane, half 0 of all lanes before half 1.  Lane l has row
// l % 16; neighbour k of a block is byte k % 16 of lane (k / 16 % 4) * 16 + row in half k / 64.  (Which of its 128 slots a neighbour fills is of no
// matter to a product as long as both operands agree.)  So a fragment is read, from memory or from LDS, as 1 KiB of consecutive bytes twice,
// whatever the matrix's strides were.  Behind the fragments, for each 64 rows and each block, 64 bytes e + 127: row r at 4 (r % 16) + r / 16 % 4,
// a lane's bytes of four row groups as one word, whose byte the product instruction picks.  Rows past the last and neighbours past the last
// column hold zeros (or NaN in a block that is not finite).
#pragma once
#include "device_common.h"

namespace tio {
namespace k {

constexpr int F8_BLOCK = 128;
constexpr int F8_LEAST = 127 - 110;              // exponent byte of the smallest block
constexpr int F8_FRAG = 2048;                    // bytes of a fragment

// a stored matrix; host and device
struct Fp8Shape {
    int64_t rows, cols;
    __host__ __device__ int64_t kb() const { return (cols + F8_BLOCK - 1) / F8_BLOCK; }
    __host__ __device__ int64_t groups() const { return (rows + 15) / 16; }
    __host__ __device__ int64_t code_bytes() const { return groups() * kb() * F8_FRAG; }
    __host__ __device__ int64_t bytes() const { return code_bytes() + (rows + 63) / 64 * kb() * 64; }
};

typedef short f8_s16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 f8_bf16x2 __attribute__((ext_vector_type(2)));
typedef float f8_f32x2 __attribute__((ext_vector_type(2)));

// FORM: 0 e4m3, 1 e5m2.  A block's power of two, as the bits of an fp32, from the bits of its largest magnitude: the sum carries into the exponent where the
// fraction is above 1.75.
template <int FORM> __device__ __forceinline__ uint32_t f8_power(uint32_t top) {
    const int e = (int)(top + 0x1fffffu - ((FORM ? 15u : 8u) << 23)) & (int)0xff800000u;
    return (uint32_t)(e < (F8_LEAST << 23) ? F8_LEAST << 23 : e);
}
__device__ __forceinline__ bool f8_finite(uint32_t top) { return top < 0x7f800000u; }

// codes of four neighbours, each divided by `scale`, a power of two: the instructions round to nearest even
template <int FORM> __device__ __forceinline__ uint32_t f8_codes(uint32_t ab, uint32_t cd, float scale) {          // pairs of bf16
    f8_s16x2 w = __builtin_nondeterministic_value(w);           // both halves are written
    const f8_bf16x2 lo = __builtin_bit_cast(f8_bf16x2, ab), hi = __builtin_bit_cast(f8_bf16x2, cd);
    if (FORM) {
        w = __builtin_amdgcn_cvt_scalef32_pk_bf8_bf16(w, lo, scale, false);
        w = __builtin_amdgcn_cvt_scalef32_pk_bf8_bf16(w, hi, scale, true);
    } else {
        w = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(w, lo, scale, false);
        w = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(w, hi, scale, true);
    }
    return __builtin_bit_cast(uint32_t, w);
}
template <int FORM> __device__ __forceinline__ uint32_t f8_codes(float a, float b, float c, float d, float scale) {
    f8_s16x2 w = __builtin_nondeterministic_value(w);
    if (FORM) {
        w = __builtin_amdgcn_cvt_scalef32_pk_bf8_f32(w, a, b, scale, false);
        w = __builtin_amdgcn_cvt_scalef32_pk_bf8_f32(w, c, d, scale, true);
    } else {
        w = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(w, a, b, scale, false);
        w = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(w, c, d, scale, true);
    }
    return __builtin_bit_cast(uint32_t, w);
}
// the values of codes 2 H and 2 H + 1 of a word; exact in bf16 and in fp32
template <int FORM, int H> __device__ __forceinline__ uint32_t f8_pair_bf16(uint32_t w, float scale) {
    if (FORM) return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_bf8(w, scale, H != 0));
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, scale, H != 0));
}
template <int FORM, int H> __device__ __forceinline__ f8_f32x2 f8_pair_f32(uint32_t w, float scale) {
    if (FORM) return __builtin_amdgcn_cvt_scalef32_pk_f32_bf8(w, scale, H != 0);
    return __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(w, scale, H != 0);
}

}  // namespace k
}  // namespace tio
