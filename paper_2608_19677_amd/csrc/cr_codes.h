// Element types and 8-bit codes of the serving kernels (cr_kvq.hip, cr_attn.hip). Not part of the ABI.
#pragma once

#include "cr_kv.h"

namespace cr {

typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));

// Rows of 16-bit elements, which go by pairs.
struct Bf16Rows {
    typedef bf16x2 Pair;
    static constexpr uint32_t kInf = 0x7F80u, kBits = 7;  // infinity, bits behind the point
    static __device__ __forceinline__ float first(uint32_t two) { return __uint_as_float(two << 16); }
    static __device__ __forceinline__ float second(uint32_t two) { return __uint_as_float(two & 0xFFFF0000u); }
};

struct F16Rows {
    typedef f16x2 Pair;
    static constexpr uint32_t kInf = 0x7C00u, kBits = 10;
    static __device__ __forceinline__ float first(uint32_t two) { return (float)__builtin_bit_cast(f16x2, two)[0]; }
    static __device__ __forceinline__ float second(uint32_t two) { return (float)__builtin_bit_cast(f16x2, two)[1]; }
};

template <typename T>
__device__ __forceinline__ uint32_t pack_pair(float x, float y)
{
    return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{x, y}), typename T::Pair));
}

// The scale 2^(b - 127) of a stored exponent b in 1 .. 254, as a float: its exponent bits.
__device__ __forceinline__ float scale_of(uint32_t b) { return __uint_as_float(b << 23); }

// An 8-bit float. wide(): codes 2 kHi and 2 kHi + 1 of four, times a power of two, as a pair of elements (exact wherever
// the element type has the value, rounded to the nearest else); floats(): the same two as they are; code(): two floats
// rounded to the nearest into bytes 2 kHi and 2 kHi + 1 of `into`. kTop: scales are chosen so that no element passes
// 1.75 * 2^kTop.
struct E4m3 {
    static constexpr int kTop = 8;
    static constexpr uint32_t kBits = 3;  // behind the point
    template <bool kHi>
    static __device__ __forceinline__ bf16x2 wide(uint32_t four, float scale, bf16x2)
    {
        return __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(four, scale, kHi);
    }
    template <bool kHi>
    static __device__ __forceinline__ f16x2 wide(uint32_t four, float scale, f16x2)
    {
        return __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(four, scale, kHi);
    }
    template <bool kHi>
    static __device__ __forceinline__ f32x2 floats(uint32_t four)
    {
        return __builtin_amdgcn_cvt_pk_f32_fp8((int)four, kHi);
    }
    template <bool kHi>
    static __device__ __forceinline__ uint32_t code(float x, float y, uint32_t into)
    {
        return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(x, y, (int)into, kHi);
    }
};

struct E5m2 {
    static constexpr int kTop = 15;
    static constexpr uint32_t kBits = 2;
    template <bool kHi>
    static __device__ __forceinline__ bf16x2 wide(uint32_t four, float scale, bf16x2)
    {
        return __builtin_amdgcn_cvt_scalef32_pk_bf16_bf8(four, scale, kHi);
    }
    template <bool kHi>
    static __device__ __forceinline__ f16x2 wide(uint32_t four, float scale, f16x2)
    {
        return __builtin_amdgcn_cvt_scalef32_pk_f16_bf8(four, scale, kHi);
    }
    template <bool kHi>
    static __device__ __forceinline__ f32x2 floats(uint32_t four)
    {
        return __builtin_amdgcn_cvt_pk_f32_bf8((int)four, kHi);
    }
    template <bool kHi>
    static __device__ __forceinline__ uint32_t code(float x, float y, uint32_t into)
    {
        return (uint32_t)__builtin_amdgcn_cvt_pk_bf8_f32(x, y, (int)into, kHi);
    }
};

// Eight codes times a scale as eight elements of type P (a pair of bf16 or f16).
template <typename C, typename P>
__device__ __forceinline__ u32x4 wide_of(u32x2 codes, float scale)
{
    u32x4 r;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        r[2 * i] = __builtin_bit_cast(uint32_t, C::template wide<false>(codes[i], scale, P{}));
        r[2 * i + 1] = __builtin_bit_cast(uint32_t, C::template wide<true>(codes[i], scale, P{}));
    }
    return r;
}

}  // namespace cr
