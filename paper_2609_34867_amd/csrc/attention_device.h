// Device helpers shared by the attention kernels: 16-bit matrix instructions,
// packing of fp32 pairs, exchanges between the halves of a wavefront.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace p4q {
namespace {

typedef _Float16 v8h __attribute__((ext_vector_type(8)));
typedef __bf16 v8bf __attribute__((ext_vector_type(8)));
typedef _Float16 v2h __attribute__((ext_vector_type(2)));
typedef __bf16 v2bf __attribute__((ext_vector_type(2)));
typedef float v2f __attribute__((ext_vector_type(2)));
typedef int v2i __attribute__((ext_vector_type(2)));
typedef unsigned short v2u __attribute__((ext_vector_type(2)));
typedef float v4f __attribute__((ext_vector_type(4)));
typedef float v16f __attribute__((ext_vector_type(16)));
typedef short v4s __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) v4s *lds_v4s_t;

template <bool BF16>
__device__ __forceinline__ v16f mfma(uint4 a, uint4 b, v16f c) {
    if constexpr (BF16)
        return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(v8bf, a), __builtin_bit_cast(v8bf, b), c, 0, 0, 0);
    else
        return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(v8h, a), __builtin_bit_cast(v8h, b), c, 0, 0, 0);
}

template <bool BF16>
__device__ __forceinline__ v4f mfma16(uint4 a, uint4 b, v4f c) {
    if constexpr (BF16)
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(v8bf, a), __builtin_bit_cast(v8bf, b), c, 0, 0, 0);
    else
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(v8h, a), __builtin_bit_cast(v8h, b), c, 0, 0, 0);
}

// two fp32 -> two 16-bit values (nearest, ties to even), low half first
template <bool BF16>
__device__ __forceinline__ uint32_t pack2(float lo, float hi) {
    if constexpr (BF16) return __builtin_bit_cast(uint32_t, __builtin_convertvector(v2f{lo, hi}, v2bf));
    else return __builtin_bit_cast(uint32_t, __builtin_convertvector(v2f{lo, hi}, v2h));
}

// two fp32 >= 0 -> the 16-bit values one step below what cutting them off gives (0: 0)
template <bool BF16>
__device__ __forceinline__ uint32_t pack2_below(float lo, float hi) {
    uint32_t cut;
    if constexpr (BF16) cut = __builtin_amdgcn_perm(__float_as_uint(hi), __float_as_uint(lo), 0x07060302u);
    else cut = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_pkrtz(lo, hi));
    return __builtin_bit_cast(uint32_t, __builtin_elementwise_sub_sat(__builtin_bit_cast(v2u, cut), v2u{1, 1}));
}

// 16-bit values -> fp32
template <bool BF16>
__device__ __forceinline__ v2f unpack2(uint32_t x) {
    if constexpr (BF16) return v2f{__uint_as_float(x << 16), __uint_as_float(x & 0xFFFF0000u)};
    else return __builtin_convertvector(__builtin_bit_cast(v2h, x), v2f);
}

// pack2 of lo * c and hi * c.  In fp16 the product is rounded once, straight
// to 16 bits (v_fma_mixlo_f16), which takes a conversion of its own for each: the
// packed one is handed products that are already rounded to fp32.
template <bool BF16>
__device__ __forceinline__ uint32_t pack2_scaled(float lo, float hi, float c) {
    if constexpr (BF16) return pack2<true>(lo * c, hi * c);
    else {
        const _Float16 a = (_Float16)(lo * c), b = (_Float16)(hi * c);
        return (uint32_t)__builtin_bit_cast(uint16_t, a) | ((uint32_t)__builtin_bit_cast(uint16_t, b) << 16);
    }
}

// lanes l and l ^ 32 hold the two halves of a query's keys: their
// combination through a permlane swap (no LDS round trip)
__device__ __forceinline__ float xmax32(float x) {
    const auto p = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return __builtin_fmaxf(__uint_as_float(p[0]), __uint_as_float(p[1]));
}
__device__ __forceinline__ float xsum32(float x) {
    const auto p = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return __uint_as_float(p[0]) + __uint_as_float(p[1]);
}
// the same of lanes l and l ^ 16
__device__ __forceinline__ float xmax16(float x) {
    const auto p = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return __builtin_fmaxf(__uint_as_float(p[0]), __uint_as_float(p[1]));
}
__device__ __forceinline__ float xsum16(float x) {
    const auto p = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return __uint_as_float(p[0]) + __uint_as_float(p[1]);
}

// p[i], i the same in all lanes, by a scalar load: for lists that nobody writes
// while the kernel runs (lengths, block tables).  A vector load would queue in
// order with the loads of keys and values, and so would the wait for it.
__device__ __forceinline__ int32_t uniform_load(const int32_t *p, int64_t i) {
    typedef const __attribute__((address_space(4))) int32_t *constant_t;
    return reinterpret_cast<constant_t>(reinterpret_cast<uint64_t>(p))[i];
}

}  // namespace
}  // namespace p4q
