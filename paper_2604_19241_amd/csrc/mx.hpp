// Blocks of 32 values that share an exponent.
//
// With m the largest magnitude of a block and e = floor(log2 m):
//   4 bits   value = 2^(e - 2) * {0, 0.5, 1, 1.5, 2, 3, 4, 6} with a sign (e2m1), nearest, ties to even, magnitudes beyond 6 become 6
//   8 bits   value = 2^(e - 6) * q, q whole from -127 to 127, nearest, ties to even, 128 becomes 127
// The exponent is kept as a byte with a bias of 127; 255 stands for a block that holds an infinity or NaN, and all of it is NaN then.  Both kinds of
// values are exact in bf16: two and seven significant bits, and nothing below 2^-132.
#pragma once
#include "common.hpp"

namespace uniep {

constexpr int kMxBlock = 32;
constexpr int kMxPad = 128;   // values a row is filled up to a multiple of: one stage of the products, 64 bytes of codes and 4 of exponents
__host__ __device__ constexpr int mx_padded(int K) { return (K + kMxPad - 1) / kMxPad * kMxPad; }
constexpr uint32_t kMxNan = 255;

// Magnitudes are compared as bit patterns: a NaN is larger than every number.
__device__ __forceinline__ uint32_t mag(float v) { return __float_as_uint(v) & 0x7fffffffu; }
// floor(log2 m) of a magnitude m > 0; subnormal ones count as the smallest normal (their blocks' exponents are at the lower end anyway).
__device__ __forceinline__ int exponent_of(uint32_t m) { return max((int)(m >> 23), 1) - 127; }
// The shared byte: of 2^(e - 2), and of 2^(e - 6) + 6.  Blocks whose scale would be below 2^-127 (in 8 bits 2^-132) have that; in 8 bits a byte of 0 is a block of zeros.
__device__ __forceinline__ uint32_t mx4_byte(uint32_t m) { return m >= 0x7f800000u ? kMxNan : (uint32_t)max(exponent_of(m) + 125, 0); }
__device__ __forceinline__ uint32_t mx8_byte(uint32_t m) { return m >= 0x7f800000u ? kMxNan : (uint32_t)(m == 0u ? 0 : exponent_of(m) + 127); }
// 2^(byte - 127)
__device__ __forceinline__ float scale_of(uint32_t byte) { return __uint_as_float(byte == 0u ? 0x00400000u : byte << 23); }

// The larger of the two halves' lanes' values, and of the four lanes' of a quad, in each of them.
__device__ __forceinline__ uint32_t max_halves(uint32_t v) {
    const auto r = __builtin_amdgcn_permlane32_swap(v, v, false, false);
    return max(r[0], r[1]);
}
__device__ __forceinline__ uint32_t max_quad(uint32_t v) {
    v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, v, 0xb1, 0xf, 0xf, true));
    return max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, v, 0x4e, 0xf, 0xf, true));
}
// Eight values in 4 bits each, the first in the lowest.  (The hardware's conversion rounds to nearest even and saturates; a block's scale of 255 makes the codes 0.)
__device__ __forceinline__ uint32_t mx4_codes(const float (&v)[8], uint32_t byte) {
    const float s = scale_of(byte);
    uint32_t c = 0;
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[0], v[1], s, 0);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[2], v[3], s, 1);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[4], v[5], s, 2);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[6], v[7], s, 3);
    return byte == kMxNan ? 0u : c;
}
__device__ __forceinline__ void mx4_values(float (&v)[8], uint32_t codes, uint32_t byte) {
    const float s = scale_of(byte);
    const f32x2_t a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, s, 0), b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, s, 1),
                  c = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, s, 2), d = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, s, 3);
    const float all[8] = {a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = byte == kMxNan ? __uint_as_float(0x7fc00000u) : all[i];
}

}  // namespace uniep
