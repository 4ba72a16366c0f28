// mx4.hpp -- keys and values in 4 bits: blocks of 32 neighbouring elements of a head, each element the product of a power of two
// that the block shares and one of 0, 0.5, 1, 1.5, 2, 3, 4, 6 with a sign (one bit of sign, two of exponent, one of fraction: the
// element that the matrix units of gfx950 know, and the block of the open microscaling formats).  The scale is a byte s for
// 2^(s - 127).
//
// Which scale: that of the block's largest magnitude, rounded to two significant bits (up where it lies halfway), divided by 4.  The largest element then
// lies in [3.5, 7) and is held as 4 or 6, off by half a step of the grid at most; dividing by 4 without the rounding would cut
// [7, 8) down to 6, and a scale twice as large where 6 is passed would halve the resolution of the whole block for it.
// Limits: with bf16 rows 2^-125 .. 2^125, with fp16 rows 2^-23 .. 2^13, so that every product is a number of the rows' type, exactly
// (the smallest magnitude is 2^-24, fp16's own step).  A block with an infinity or a NaN has the scale 255: all of it is NaN.
#pragma once
#include "attn_plan.hpp"

namespace stand {

constexpr int kMx4Block = 32;
constexpr int kMx4Nan = 255;

// Scale of a block whose largest magnitude has these bits as a binary32 number.
STAND_BOTH int mx4_scale(uint32_t top, bool f16)
{
    const int low = f16 ? 127 - 23 : 127 - 125, high = f16 ? 127 + 13 : 127 + 125;
    if (top >= 0x7F800000u) return kMx4Nan;
    const int s = (int)((top + 0x200000u) >> 23) - 2;
    return s < low ? low : s > high ? high : s;
}

#if defined(__HIPCC__)
typedef __bf16 mx4_bf16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 mx4_f16x2 __attribute__((ext_vector_type(2)));

// (a scale as the conversions take it: the byte is the exponent of a binary32 number, 255 gives NaN)
__device__ __forceinline__ float mx4_factor(uint32_t s) { return __uint_as_float(s << 23); }

// Elements 2 I and 2 I + 1 of a word of eight, in the rows' type: exact.
template <bool F16, int I>
__device__ __forceinline__ uint32_t mx4_two(uint32_t w, float factor)
{
    if constexpr (F16) return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, factor, I));
    else return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, factor, I));
}
template <bool F16>
__device__ __forceinline__ uint4 mx4_eight(uint32_t w, float factor)
{
    return uint4{mx4_two<F16, 0>(w, factor), mx4_two<F16, 1>(w, factor), mx4_two<F16, 2>(w, factor), mx4_two<F16, 3>(w, factor)};
}

// Eight elements into a word: nearest, ties to the even code, magnitudes above 6 become 6.
__device__ __forceinline__ uint32_t mx4_pack(const float *x, float factor)
{
    uint32_t w = 0;
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[0], x[1], factor, 0);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[2], x[3], factor, 1);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[4], x[5], factor, 2);
    return __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[6], x[7], factor, 3);
}

__device__ __forceinline__ uint32_t mx4_magnitude(float x) { return __float_as_uint(x) & 0x7FFFFFFFu; }

// Half a block, 16 elements, of every lane; a lane and its neighbour have a block.  -> its words, and the block's scale.
template <bool F16>
__device__ __forceinline__ uint2 mx4_half_block(const float *x, uint32_t &scale)
{
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < 16; ++i) top = max(top, mx4_magnitude(x[i]));
    top = max(top, (uint32_t)__shfl_xor((int)top, 1));
    scale = (uint32_t)mx4_scale(top, F16);
    const float factor = mx4_factor(scale);
    return uint2{mx4_pack(x, factor), mx4_pack(x + 8, factor)};
}

// A quarter of a block, 8 elements, of every lane; four neighbours have a block.
template <bool F16>
__device__ __forceinline__ uint32_t mx4_quarter_block(const float *x, uint32_t &scale)
{
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) top = max(top, mx4_magnitude(x[i]));
    top = max(top, (uint32_t)__shfl_xor((int)top, 1));
    top = max(top, (uint32_t)__shfl_xor((int)top, 2));
    scale = (uint32_t)mx4_scale(top, F16);
    return mx4_pack(x, mx4_factor(scale));
}

// Two 16-bit elements of a word as fp32.
template <bool F16> __device__ __forceinline__ float row_low(uint32_t w)
{
    if constexpr (F16) return (float)__builtin_bit_cast(mx4_f16x2, w)[0];
    else return __uint_as_float(w << 16);
}
template <bool F16> __device__ __forceinline__ float row_high(uint32_t w)
{
    if constexpr (F16) return (float)__builtin_bit_cast(mx4_f16x2, w)[1];
    else return __uint_as_float(w & 0xFFFF0000u);
}
template <bool F16> __device__ __forceinline__ uint32_t row_two(float a, float b)
{
    if constexpr (F16) return __builtin_bit_cast(uint32_t, mx4_f16x2{(_Float16)a, (_Float16)b});
    else return __builtin_bit_cast(uint32_t, mx4_bf16x2{(__bf16)a, (__bf16)b});
}
template <bool F16>
__device__ __forceinline__ void row_eight(const uint4 &w, float *x)
{
    const uint32_t v[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        x[2 * i] = row_low<F16>(v[i]);
        x[2 * i + 1] = row_high<F16>(v[i]);
    }
}
#endif

}  // namespace stand
