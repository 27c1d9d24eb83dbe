// Rows of the pool in 4 bits (gfx950 only; the format is stated in esp.h): a head of a slot is 64 bytes of E2M1 codes and four E8M0 scales, one to
// 32 elements.  The chip converts pairs of codes to bf16 with their scale in one instruction, exactly.
#pragma once
#include "esp_common.h"

namespace esp {

constexpr int kQ4Head = ESP_Q4_HEAD_BYTES;
constexpr int kQ4Codes = 64;                      // bytes of them that are codes; the scales follow

// The conversions take a scale from the exponent's bits of a float and go by those alone (255: NaN), so a byte of a word of four scales needs no more than to
// be turned to their place.
__device__ __forceinline__ float q4_scale(uint32_t scales, int byte) {
    return __builtin_bit_cast(float, __builtin_amdgcn_alignbit(scales, scales, 9 + 8 * byte));
}

// eight codes to bf16
__device__ __forceinline__ uint4 q4_to_bf16(uint32_t codes, float scale) {
    return make_uint4(__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 0)),
                      __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 1)),
                      __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 2)),
                      __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 3)));
}

// A block's scale from its largest magnitude, as a bf16 pattern: the power of two with which no element is off by more than half a step (up to 7 of them
// round to the largest code's 6; from there on, the next one; at most 2^125, with which all codes are finite numbers).  A block with an infinity or a
// NaN is NaN.
__device__ __forceinline__ uint32_t q4_scale_byte(uint32_t largest) {
    const int e = (int)((largest + 0x20) >> 7) - 2;
    return largest >= 0x7f80 ? 255u : (uint32_t)min(max(e, 2), 252);
}

}  // namespace esp
