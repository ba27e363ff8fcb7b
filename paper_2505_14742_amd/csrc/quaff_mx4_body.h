// Device arithmetic of 4-bit microscaled values (quaff_mx4.hip), for the kernels that quantize.
#pragma once
#include "quaff_internal.h"

namespace quaff {

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

// scale byte of a block whose largest magnitude has the biased exponent e
__device__ __forceinline__ uint32_t mx4_scale_byte(uint32_t e) { return e == 255 ? 255u : e > 2 ? e - 2 : 0u; }
// 2^(byte - 127) as a float (byte 0: 2^-127, a subnormal)
__device__ __forceinline__ float mx4_scale_value(uint32_t byte) { return __uint_as_float(byte == 0 ? 0x00400000u : byte << 23); }

// the largest magnitude among eight bf16 values and m, as bits
template <class V>
__device__ __forceinline__ uint32_t mx4_max_bits(uint32_t m, const V& x) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const uint32_t lo = (uint32_t)x[j] & 0x7fffu, hi = ((uint32_t)x[j] >> 16) & 0x7fffu;
        m = m > lo ? m : lo;
        m = m > hi ? m : hi;
    }
    return m;
}

// eight bf16 values (a bit cast of a vector's element itself reads the first one's bits: copied out first)
template <class V>
__device__ __forceinline__ uint32_t mx4_code8_bf16(const V& x, float s) {
    const uint32_t x0 = x[0], x1 = x[1], x2 = x[2], x3 = x[3];
    uint32_t c = 0;
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(bf16x2, x0), s, 0);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(bf16x2, x1), s, 1);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(bf16x2, x2), s, 2);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(bf16x2, x3), s, 3);
    return c;
}

}  // namespace quaff
