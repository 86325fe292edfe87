// MX8: 8-bit floats (e4m3) with one scale 2^e for every 32 neighbours of a row.
//
// e is the smallest integer >= -127 for which the largest magnitude of the block is at most 448 * 2^e (448 is the largest e4m3
// value), so nothing saturates; a value v is held as v / 2^e rounded to e4m3, to nearest even: at most 2^-4 of v off, or 2^-10 * 2^e
// below the smallest normal value.  The scale is held as the byte e + 127.  A block with a NaN or an infinity has the scale
// byte 255 (NaN) and NaN values.
// The scales of a matrix [rows][cols] lie as [ceil(cols / 128)][rows][4]: the four bytes that a row brings into a product's
// step of 128 indices are one word, and the words of neighbouring rows are neighbours.  Bytes past cols are 127.
#pragma once
#include "kernels.h"
#include "route_select.h"

namespace unipool {

namespace {

constexpr int kMxBlock = 32;              // values that share a scale
constexpr int kMxStep = 128;              // columns of one word of scales
constexpr int kMxBias = 127;
constexpr int kMxNan = 255;               // scale byte of a block that holds a NaN or an infinity

// Larger magnitude of two values; NaN if one of them is (fmaxf would drop it).  Chains of it become v_maximum3_f32 with |.| on its operands.
__device__ __forceinline__ float mx8_max(float a, float b) { return __builtin_elementwise_maximum(__builtin_fabsf(a), __builtin_fabsf(b)); }

// Largest magnitude over LPB neighbouring lanes, the same in all of them (every lane of the wavefront is active).
template <int LPB> __device__ __forceinline__ float mx8_lanes_max(float v) {
    static_assert(LPB == 4 || LPB == 8 || LPB == 32, "8, 4 or 1 values a lane");
    v = mx8_max(v, dpp_f<kDppQuadXor1>(v));
    v = mx8_max(v, dpp_f<kDppQuadXor2>(v));
    if constexpr (LPB >= 8) v = mx8_max(v, dpp_f<kDppRowHalfMirror>(v));
    if constexpr (LPB == 32) {
        v = mx8_max(v, dpp_f<kDppRowMirror>(v));
        const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
        v = mx8_max(__uint_as_float(r[0]), __uint_as_float(r[1]));
    }
    return v;
}

// Scale byte of a block from its largest magnitude: amax = 2^(E - 127) (1 + m / 2^23) and 448 = 2^8 * 1.75, so e = E - 135, one more if
// the fraction is over 0.75.
__device__ __forceinline__ int mx8_scale_byte(float amax) {
    const unsigned b = __float_as_uint(amax) & 0x7fffffffu;
    if (b >= 0x7f800000u) return kMxNan;
    const int e = (int)(b >> 23) - 135 + ((b & 0x7fffffu) > 0x600000u ? 1 : 0);
    return max(e, -127) + kMxBias;
}
// Four values to four e4m3 bytes, the first lowest.  The instruction divides by the power of two whose exponent bits it is given, and
// |v| <= 448 after that, so it never overflows.
__device__ __forceinline__ unsigned mx8_pack4(float a, float b, float c, float d, int byte) {
    typedef short s16x2 __attribute__((ext_vector_type(2)));
    if (byte == kMxNan) return 0x7f7f7f7fu;
    const float scale = __uint_as_float((unsigned)byte << 23);
    s16x2 r = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(s16x2{0, 0}, a, b, scale, false);
    r = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(r, c, d, scale, true);
    return __builtin_bit_cast(unsigned, r);
}
__device__ __forceinline__ unsigned char mx8_pack1(float a, int byte) { return (unsigned char)(mx8_pack4(a, a, a, a, byte) & 0xffu); }

// place of the scale byte of block b of a row
__device__ __forceinline__ size_t mx8_scale_at(size_t rows, size_t row, int b) { return ((size_t)(b >> 2) * rows + row) * 4 + (b & 3); }

}  // namespace

}  // namespace unipool
