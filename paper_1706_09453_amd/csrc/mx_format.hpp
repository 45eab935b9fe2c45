// Numbers of 4 and 8 bits that share a power of two in blocks of 32: the scale bytes, the rounding, the random bits.  What the
// 4-bit layers (mx4_kernels.hpp) and the 8-bit states of AdamW (adamw_kernels.hpp) have in common.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace bnn {

// 32 bits mixed: two rounds of shift and multiply.  The multipliers are the leading fraction bits of sqrt(2) and sqrt(3); with these
// shifts flipping any input bit flips every output bit with probability 0.5 +- 0.004.
__host__ __device__ __forceinline__ uint32_t mix32(uint32_t x) {
    x ^= x >> 16;
    x *= 0x6A09E667u;
    x ^= x >> 15;
    x *= 0xBB67AE85u;
    return x ^ (x >> 16);
}
__host__ __device__ __forceinline__ uint32_t seed_key(uint64_t seed) { return mix32(mix32((uint32_t)seed) + (uint32_t)(seed >> 32)); }

// The largest magnitudes of the element formats as what is added to a float's bits so that its exponent field goes up by one
// exactly where its fraction is above the magnitude's, and the magnitude's own exponent: 6 = 1.5 * 2^2, 127 = 1.984375 * 2^6,
// 255 = 1.9921875 * 2^7.
struct MxE2M1 { static constexpr uint32_t add = 0x7FFFFFu - 0x400000u; static constexpr int exponent = 2; };
struct MxInt8 { static constexpr uint32_t add = 0x7FFFFFu - 0x7E0000u; static constexpr int exponent = 6; };
struct MxUint8 { static constexpr uint32_t add = 0x7FFFFFu - 0x7F0000u; static constexpr int exponent = 7; };

// Scale byte e of a block whose largest magnitude has the float bits `top` (a maximum of bits, so that Inf and NaN win): the smallest
// e >= 0 with magnitude <= largest * 2^(e - 127), or 255, the format's NaN, if a number of the block is none.
template <class F>
__device__ __forceinline__ uint32_t mx_scale(uint32_t top) {
    const int e = (int)((top + F::add) >> 23) - F::exponent;
    return top >= 0x7F800000u ? 255u : (uint32_t)(e < 0 ? 0 : e);
}
// 2^(e - 127), NaN for 255
__device__ __forceinline__ float mx_scale_value(uint32_t e) { return __uint_as_float(e == 0 ? 0x00400000u : e == 255 ? 0x7FC00000u : e << 23); }
// 2^(127 - e) for a scale byte from mx_scale; 0 for 255, which with finite numbers gives codes of 0 (the caller keeps Inf and NaN out)
__device__ __forceinline__ float mx_inverse_scale(uint32_t e) { return __uint_as_float(e == 255 ? 0u : (254u - e) << 23); }

// the larger of the lane's value and another lane's (CTRL: a DPP control)
template <int CTRL>
__device__ __forceinline__ uint32_t max_dpp(uint32_t v) {
    return max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, 0xF, 0xF, false));
}
// the largest of 4 and of 8 neighbouring lanes' values, in all of them
__device__ __forceinline__ uint32_t max_of_4_lanes(uint32_t v) { return max_dpp<0x4E>(max_dpp<0xB1>(v)); }   // quad_perm [1, 0, 3, 2], [2, 3, 0, 1]
__device__ __forceinline__ uint32_t max_of_8_lanes(uint32_t v) { return max_dpp<0x141>(max_of_4_lanes(v)); }   // row_half_mirror: lane i and 7 - i of every 8

}  // namespace bnn
