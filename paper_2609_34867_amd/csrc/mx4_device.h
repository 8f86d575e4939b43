// Device-side pieces of the microscaled 4-bit floating point format (MXFP4 of
// the OCP Microscaling specification): 32 consecutive values of a row share
// one power of two X, each is an E2M1 number times X.
//
//   X = 2^(floor(log2 max|v|) - 2), at least 2^-127; held as byte log2 X + 127
//   code = the E2M1 number (0, 0.5, 1, 1.5, 2, 3, 4, 6 and a sign) nearest to
//          v / X, ties to the even code, saturating at 6
//
// Since X is a power of two, v / X is exact in fp32 wherever it decides a code
// (the smallest border, 0.25, lies far above what 2^-149 can round), so the
// codes follow the definition bit for bit.  A block with an infinity or a NaN
// has byte 255, which stands for NaN, and codes 0.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "wave_ops.h"

namespace p4q {

typedef float mx_f2 __attribute__((ext_vector_type(2)));
typedef __bf16 mx_b2 __attribute__((ext_vector_type(2)));

// X of a scale byte, in fp32 (255: infinity, which makes 0 * X the NaN it stands for)
__device__ __forceinline__ float mx4_scale(uint32_t byte) {
    return __uint_as_float(byte == 0 ? 0x00400000u : byte << 23);
}

// the scale byte of a block whose largest magnitude has these bits (255: not finite)
__device__ __forceinline__ uint32_t mx4_byte(uint32_t top) {
    const uint32_t e = top >> 23;
    return e == 255u ? 255u : max(e, 2u) - 2u;
}

// 1 / X of a scale byte below 255
__device__ __forceinline__ float mx4_inverse(uint32_t byte) { return __uint_as_float((254u - byte) << 23); }

// four codes (value i in nibble i) of values already divided by X
__device__ __forceinline__ uint32_t mx4_codes4(float a, float b, float c, float d) {
    uint32_t w = 0;
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, a, b, 1.0f, 0);
    return __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, c, d, 1.0f, 1);
}

// Quantizes a block that lanes l and l + 32 hold, 16 values each: lane l the
// values 8 g + 0..3, lane l + 32 the values 8 g + 4..7, in v[4 g ..].  Returns 8
// bytes of codes, lane l the block's first half, lane l + 32 its second.
__device__ __forceinline__ uint2 mx4_quantize_halves(const float (&v)[16], uint32_t &byte) {
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < 16; ++i) top = max(top, __float_as_uint(v[i]) & 0x7FFFFFFFu);
    top = max(top, (uint32_t)__shfl_xor((int)top, 32));
    byte = mx4_byte(top);
    const float inv = byte == 255u ? 0.0f : mx4_inverse(byte);
    uint32_t c[4];
#pragma unroll
    for (int g = 0; g < 4; ++g)
        c[g] = byte == 255u ? 0u : mx4_codes4(v[4 * g] * inv, v[4 * g + 1] * inv, v[4 * g + 2] * inv, v[4 * g + 3] * inv);
    // the upper lanes' groups 0 and 1 against the lower lanes' 2 and 3
    const auto s = __builtin_amdgcn_permlane32_swap(c[0] | (c[1] << 16), c[2] | (c[3] << 16), false, false);
    return make_uint2((s[0] & 0xFFFFu) | (s[1] << 16), (s[0] >> 16) | (s[1] & 0xFFFF0000u));
}

// Quantizes a block that the four lanes of a quad hold, 8 consecutive values
// each.  Returns this lane's 8 codes (value i in nibble i) and, in every lane,
// the block's scale byte.
__device__ __forceinline__ uint32_t mx4_quantize(const float (&v)[8], uint32_t &byte) {
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) top = max(top, __float_as_uint(v[i]) & 0x7FFFFFFFu);
    top = max(top, lane_xor<1>(top));
    top = max(top, lane_xor<2>(top));
    byte = mx4_byte(top);
    if (byte == 255u) return 0;
    const float inv = mx4_inverse(byte);
    return mx4_codes4(v[0] * inv, v[1] * inv, v[2] * inv, v[3] * inv) |
           (mx4_codes4(v[4] * inv, v[5] * inv, v[6] * inv, v[7] * inv) << 16);
}

// The 8 values that codes and a scale byte stand for.
__device__ __forceinline__ void mx4_values(uint32_t c, uint32_t byte, float (&v)[8]) {
    const float X = mx4_scale(byte);
    const mx_f2 p0 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, 1.0f, 0);
    const mx_f2 p1 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, 1.0f, 1);
    const mx_f2 p2 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, 1.0f, 2);
    const mx_f2 p3 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, 1.0f, 3);
    v[0] = p0[0] * X;
    v[1] = p0[1] * X;
    v[2] = p1[0] * X;
    v[3] = p1[1] * X;
    v[4] = p2[0] * X;
    v[5] = p2[1] * X;
    v[6] = p3[0] * X;
    v[7] = p3[1] * X;
}

// two fp32 values rounded to a word of two 16-bit floats (nearest, ties to even)
template <bool BF16>
__device__ __forceinline__ uint32_t round16x2(float a, float b) {
    if constexpr (BF16) {
        return __builtin_bit_cast(uint32_t, __builtin_convertvector(mx_f2{a, b}, mx_b2));
    } else {
        // (as asm operands: a product before it must round to fp32 first)
        asm("" : "+v"(a), "+v"(b));
        return (uint32_t)__builtin_bit_cast(uint16_t, (_Float16)a) |
               ((uint32_t)__builtin_bit_cast(uint16_t, (_Float16)b) << 16);
    }
}

template <bool BF16>
__device__ __forceinline__ uint4 round16x8(const float (&v)[8]) {
    return make_uint4(round16x2<BF16>(v[0], v[1]), round16x2<BF16>(v[2], v[3]), round16x2<BF16>(v[4], v[5]),
                      round16x2<BF16>(v[6], v[7]));
}

}  // namespace p4q
