// kv_format.hpp -- rows of an 8-bit generated cache (splice_tree.h): e4m3
// codes with one power of two a row, every value exact in bf16.
#pragma once

#include "device_common.hpp"

namespace splice_dev {

// Eight codes as eight bf16 values of a row with this exponent byte.
__device__ __forceinline__ u32x4_t e4m3_to_bf16(uint2 codes, uint32_t exponent) {
    const float f = __uint_as_float(exponent << 23);
    return u32x4_t{__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes.x, f, false)),
                   __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes.x, f, true)),
                   __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes.y, f, false)),
                   __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes.y, f, true))};
}

}  // namespace splice_dev
