// MXFP4 (OCP microscaling formats, version 1.0): E2M1 elements, one power of two 2^(byte - 127) as the scale of 32
// channels, byte 255 = NaN.  Arithmetic and operand layout shared by the quantizers and the products of this format.
#pragma once
#include "pq_device.h"

namespace pq {

constexpr int kMxBlock = 32;

// ---------------------------------------------------------------- quantizer
// Scale byte of a group from the largest of its bf16 magnitudes as bits: floor(log2 amax) is the exponent field less 127, the
// element format's largest exponent is 2, so byte = field - 2, cut at 0 (2^-127; groups of subnormals and of zeros land there).
// A group with an infinity or a NaN is NaN as a whole: what it feeds becomes NaN, not some finite number.
__device__ __forceinline__ uint32_t mx_scale_byte(uint32_t amax_bits) {
  const uint32_t field = amax_bits >> 7;
  return field == 255u ? 255u : field > 2u ? field - 2u : 0u;
}
// 2^(byte - 127) as a binary32 value; byte 0 is a subnormal there, byte 255 (NaN) gives a quiet NaN
__device__ __forceinline__ float mx_scale_value(uint32_t byte) {
  return as_f32(byte == 0u ? 0x00400000u : byte == 255u ? 0x7FC00000u : byte << 23);
}

typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
// Eight codes, element j in bits 4j.  The conversion unit divides by the scale, rounds to nearest even and saturates at 6
// (checked against the definition for all 2^16 bf16 values under scales 2^-127 .. 2^125).
__device__ __forceinline__ uint32_t mx_codes8(const uint4& x, float scale) {
  uint32_t c = 0;
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(bf16x2_t, x.x), scale, 0);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(bf16x2_t, x.y), scale, 1);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(bf16x2_t, x.z), scale, 2);
  return __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(bf16x2_t, x.w), scale, 3);
}
// largest of eight bf16 magnitudes, as bits (finite magnitudes order like their bits, infinities and NaN above them)
__device__ __forceinline__ uint32_t mx_amax8(const uint4& x) {
  const uint32_t m = 0x7FFFu;
  uint32_t a = max(max(x.x & m, x.x >> 16 & m), max(x.y & m, x.y >> 16 & m));
  return max(a, max(max(x.z & m, x.z >> 16 & m), max(x.w & m, x.w >> 16 & m)));
}
// four lanes hold the 32 channels of a group: its scale byte in each of them, and the codes of this lane's eight
__device__ __forceinline__ uint32_t mx_quantize8(const uint4& x, uint32_t& byte) {
  uint32_t a = mx_amax8(x);
  a = max(a, dpp_u32<0xB1>(a));                              // quad_perm [1,0,3,2]
  a = max(a, dpp_u32<0x4E>(a));                              // quad_perm [2,3,0,1]
  byte = mx_scale_byte(a);
  return mx_codes8(x, byte == 255u ? 1.0f : mx_scale_value(byte));
}

// two values rounded to bf16, nearest even, a in the low half
__device__ __forceinline__ uint32_t pack_bf16(float a, float b) {
  return (uint32_t)__builtin_bit_cast(uint16_t, (__bf16)a) | (uint32_t)__builtin_bit_cast(uint16_t, (__bf16)b) << 16;
}

// ---------------------------------------------------------------- operand of the product
// Panels of 128 channels: codes[panel][row][64 bytes], scales[panel][row][4 bytes], channels from K on zero (codes and scales).
// The rows of a tile lie next to each other whatever K is: whole lines are read (rows K / 2 bytes apart would meet in few channels of
// the caches where K is a power of two), and a gathered row's piece is still half a line.
constexpr int kMxPanel = 128;
constexpr int kMxRowBytes = kMxPanel / 2, kMxRowScales = kMxPanel / kMxBlock;
__host__ __device__ __forceinline__ int64_t mx_panels(int64_t K) { return (K + kMxPanel - 1) / kMxPanel; }
__host__ __device__ __forceinline__ size_t mx_scales_at(int64_t rows, int64_t K) {
  return ((size_t)mx_panels(K) * rows * kMxRowBytes + 255) / 256 * 256;
}

}  // namespace pq
