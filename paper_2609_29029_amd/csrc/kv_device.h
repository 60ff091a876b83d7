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

// Sums over the wave's lanes up to each.
__device__ __forceinline__ int wave_scan(int x) {
    x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xf, 0xf, false);   // row_shr 1, 2, 4, 8
    x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xf, 0xf, false);
    x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xf, 0xf, false);
    x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xf, 0xf, false);
    x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xa, 0xf, false);   // row_bcast 15 into rows 1 and 3
    x += __builtin_amdgcn_update_dpp(0, x, 0x143, 0xc, 0xf, false);   // row_bcast 31 into rows 2 and 3
    return x;
}

// The largest of the wave, in every lane.
__device__ __forceinline__ uint32_t wave_most(uint32_t x) {
    x = max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x111, 0xf, 0xf, false));   // as above; 0 where there is no lane
    x = max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x112, 0xf, 0xf, false));
    x = max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x114, 0xf, 0xf, false));
    x = max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x118, 0xf, 0xf, false));
    x = max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x142, 0xa, 0xf, false));
    x = max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x143, 0xc, 0xf, false));
    return (uint32_t)__builtin_amdgcn_readlane((int)x, 63);
}

constexpr uint32_t kNotFinite = 0x7F800000u;   // magnitude bits from here on: infinity and NaN

}  // namespace rift
