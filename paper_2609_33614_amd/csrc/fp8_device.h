// Numbers in 8 bits with a power of two per block of 128 (gfx950).
//
// A block is held as e4m3 numbers q (4 significant bits, largest 448) and one
// byte b that stands for 2^(b - 127): the smallest power of two under which the
// block's largest finite magnitude is at most 448.  A power of two, not the
// quotient by 448: e4m3 floats, so a factor below 2 in the scale leaves the
// relative rounding (2^-4 at most) of every normal number as it is and moves only the
// end of the range, 2^-15 of the block's largest, by that factor; the division is
// exact, and the matrix instructions apply such scales themselves.  Numbers
// that are not finite are held as NaN and leave the scale alone; a block of
// zeros has the scale 1.
//
// Rows are padded with zeros to whole blocks, the bytes of their scales to
// whole words.
#pragma once
#include "eat_device.h"

namespace eat {

constexpr int kBlk = 128;

__device__ __forceinline__ bool is_finite(float v) { return (__float_as_uint(v) & 0x7fffffffu) < 0x7f800000u; }
__device__ __forceinline__ float finite_abs(float v) { return is_finite(v) ? fabsf(v) : 0.f; }

// The scale's byte for a largest magnitude amax = 1.m 2^(E - 127): 448 is 1.75
// 2^8, so 2^(E - 127 - 8) does where 1.m <= 1.75, and twice that otherwise.
__device__ __forceinline__ uint32_t scale_byte(float amax) {
    const uint32_t u = __float_as_uint(amax);
    const int b = static_cast<int>(u >> 23) - 8 + ((u & 0x7fffffu) > 0x600000u ? 1 : 0);
    return u == 0 ? 127u : static_cast<uint32_t>(max(b, 1));
}
// 2^-(b - 127), 1 <= b <= 253.
__device__ __forceinline__ float scale_inverse(uint32_t b) { return __uint_as_float((254u - b) << 23); }

// Four numbers, already divided, to e4m3 (round to nearest even; NaN for NaN and, as
// the format has no infinities, for them).
__device__ __forceinline__ uint32_t pack_e4m3(float a, float b, float c, float d) {
    int w = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
    return static_cast<uint32_t>(__builtin_amdgcn_cvt_pk_fp8_f32(c, d, w, true));
}

// The largest over the 16 lanes of a row of lanes.
__device__ __forceinline__ float row_max(float v) {
    v = fmaxf(v, dpp_f<kDppXor1>(v));
    v = fmaxf(v, dpp_f<kDppXor2>(v));
    v = fmaxf(v, dpp_f<kDppHalfMirror>(v));
    return fmaxf(v, dpp_f<kDppMirror>(v));
}

// Eight numbers of a block that 16 lanes hold side by side: its scale's byte, and
// the lane's eight in 8 bits.
__device__ __forceinline__ uint32_t quantize_lane(const float (&v)[8], uint2& q) {
    float m = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) m = fmaxf(m, finite_abs(v[i]));
    const uint32_t b = scale_byte(row_max(m));
    const float s = scale_inverse(b);
    float o[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) o[i] = v[i] * s;
    q = uint2{pack_e4m3(o[0], o[1], o[2], o[3]), pack_e4m3(o[4], o[5], o[6], o[7])};
    return b;
}

}  // namespace eat
