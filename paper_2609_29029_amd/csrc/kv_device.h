// Device-side helpers of the paged key-value cache: storage types, pages, scales.
#pragma once

#include "kv.h"
#include "rift_common.h"

namespace rift {

// Round to nearest even, NaN kept (one instruction on gfx950).
__device__ __forceinline__ bf16_t round_bf16(float f) { return __builtin_bit_cast(bf16_t, static_cast<__bf16>(f)); }

// 2^(b - 127) of a scale byte; infinity for 255, whose codes are 0: their product is NaN.
__device__ __forceinline__ float scale_of(uint32_t b) { return __uint_as_float(b << 23); }

// Scale byte of a row whose largest magnitude has the bits `most` (of a finite
// value): the smallest power of two that brings it to at most 448 = 1.75 2^8
// (e4m3) or 127 = 1.984375 2^6 (int8).
template <riftkv_dtype DT>
__device__ __forceinline__ uint32_t scale_byte(uint32_t most) {
    const int e = (int)(most >> 23);
    const uint32_t m = most & 0x7FFFFFu;
    const int b = DT == RIFTKV_FP8 ? e - 8 + (m > 0x600000u) : e - 6 + (m > 0x7E0000u);
    return (uint32_t)max(b, 1);
}

constexpr uint32_t kNotFinite = 0x7F800000u;   // magnitude bits from here on: infinity and NaN

}  // namespace rift
