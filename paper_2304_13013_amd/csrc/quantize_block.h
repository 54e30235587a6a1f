// The scale of a block of 128 (quantize_block.hip says how it is defined).
#pragma once
#include "quantize_common.h"

namespace sb {
namespace {

// Scale byte for a block's absmax (15 bits of a bf16 pattern).  As a binary32 pattern the magnitude is 1.f * 2^k, and MAX is
// 1.75 * 2^8 or 1.75 * 2^15: the exponent goes up by one where 1.f > 1.75.  A block with an infinity or a NaN takes the exponent of
// their patterns, 247 at most (NaNs above 1.75 would carry to 248): their codes are not finite, its other values scaled by it.
template <int CODE>
__device__ __forceinline__ unsigned int block_scale_byte(unsigned int bits15) {
    const int s = (int)(((bits15 << 16) + 0x1fffffu) >> 23) - (CODE == CODE_E4M3 ? 8 : 15);
    return (unsigned int)min(max(s, 0), 247);
}
__device__ __forceinline__ float inverse_of_scale_byte(unsigned int s) { return __uint_as_float((254u - s) << 23); }  // s <= 247

}  // namespace
}  // namespace sb
