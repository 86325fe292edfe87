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

namespace unipool {

namespace {

constexpr int kMxBlock = 32;              // values that share a scale
constexpr int kMxStep = 128;              // columns of one word of scales
constexpr int kMxBias = 127;
constexpr int kMxNan = 255;               // scale byte of a block that holds a NaN or an infinity

// Magnitudes as integers: they order as the floats do, with infinity and NaN on top (fmaxf would drop a NaN).
__device__ __forceinline__ unsigned mx8_mag(float v) { return __float_as_uint(v) & 0x7fffffffu; }

// Scale byte of a block from the largest magnitude: amax = 2^(E - 127) (1 + m / 2^23) and 448 = 2^8 * 1.75, so e = E - 135, one more
// if the fraction is over 0.75.
__device__ __forceinline__ int mx8_scale_byte(unsigned amax) {
    if (amax >= 0x7f800000u) return kMxNan;
    const int e = (int)(amax >> 23) - 135 + ((amax & 0x7fffffu) > 0x600000u ? 1 : 0);
    return max(e, -127) + kMxBias;
}
// 2^-e, exact: e lies between -127 and 120
__device__ __forceinline__ float mx8_inverse(int byte) { return __uint_as_float((unsigned)(254 - byte) << 23); }

// Four values to four e4m3 bytes, the first lowest.  |v| <= 448 after the scale, so the conversion never overflows.
__device__ __forceinline__ unsigned mx8_pack4(float a, float b, float c, float d, int byte) {
    if (byte == kMxNan) return 0x7f7f7f7fu;
    const float s = mx8_inverse(byte);
    int r = __builtin_amdgcn_cvt_pk_fp8_f32(a * s, b * s, 0, false);
    r = __builtin_amdgcn_cvt_pk_fp8_f32(c * s, d * s, r, true);
    return (unsigned)r;
}
__device__ __forceinline__ unsigned char mx8_pack1(float a, int byte) { return (unsigned char)(mx8_pack4(a, a, a, a, byte) & 0xffu); }

// place of the scale byte of block b of a row
__device__ __forceinline__ size_t mx8_scale_at(size_t rows, size_t row, int b) { return ((size_t)(b >> 2) * rows + row) * 4 + (b & 3); }

}  // namespace

constexpr int kMx8Rows = 64;       // rows of a workgroup of the conversion

}  // namespace unipool
