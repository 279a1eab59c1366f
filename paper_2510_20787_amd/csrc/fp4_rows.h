// Kept rows in 4 bits: how a row is encoded and where its bytes lie.
//
// Thirty-two channels of a row share a power of two 2^E (a byte E + 127) and hold one of +-{0, 0.5, 1, 1.5, 2, 3, 4, 6} each.  With
// the largest magnitude m * 2^k (1 <= m < 2): E = k - 2 for m <= 1.75 (its quotient, up to 7, is then at most 1 above the largest
// value) and for k = 127 (4 * 2^126 is no number any more), else k - 1.  A quotient goes to the nearest value, halfway cases to the even code, above 6 to 6.  A largest magnitude
// below 2^-120 makes a group of zeros (all values are normal numbers then), an infinity or NaN in it a group of NaN (byte 255).
// Decoding is exact in bf16 and fp32, and encoding what was decoded gives the same bytes.
//
// The rows of a head are stored in blocks of 32 (the rows that one wave of the decode step takes at a time), 34 * D bytes:
//   K codes   16 D bytes    V codes   16 D bytes    K exponents   D bytes    V exponents   D bytes
// in the order in which the lanes load them (lane = 16 * kg + c), row r of the block:
//   K  row r = 8 * (c / 4) + 4 * j + c % 4 is row c of the j-th tile of 16; kg takes a quarter of its channels.
//      D = 128: [j][lane][16 bytes]   D = 64: [lane][j][8 bytes]      exponents [c][group][j]
//   V  rows 8 * kg + u; c takes D / 16 channels of each.
//      D = 128: [u / 4][lane][u % 4][4 bytes]   D = 64: [lane][u][2 bytes]      exponents [kg][group][u]
// A byte holds channel 2 i in its low half and 2 i + 1 in its high half.
#pragma once
#include "ltea_common.h"

namespace ltea {

template <int D> struct PackGeo {
  static constexpr int kBlock = 34 * D;                     // bytes of a block
  static constexpr int kV = 16 * D, kKe = 32 * D, kVe = 33 * D;   // offsets of its parts (K codes at 0)
  static constexpr int NG = D / 32;                         // groups of a row
};

// Byte offset in its block of the codes of channels d, d + 1 (d even) of row r.
template <int D> __device__ __forceinline__ int k_code_at(int r, int d) {
  const int j = (r >> 2) & 1, c = 4 * (r >> 3) + (r & 3);
  return D == 128 ? ((j * 4 + d / 32) * 16 + c) * 16 + (d % 32) / 2 : (((d / 16) * 16 + c) * 2 + j) * 8 + (d % 16) / 2;
}
template <int D> __device__ __forceinline__ int v_code_at(int r, int d) {
  const int kg = r >> 3, u = r & 7;
  return PackGeo<D>::kV + (D == 128 ? (((u >> 2) * 64 + kg * 16 + d / 8) * 4 + (u & 3)) * 4 + (d % 8) / 2
                                    : ((kg * 16 + d / 4) * 8 + u) * 2 + (d % 4) / 2);
}
template <int D> __device__ __forceinline__ int k_exp_at(int r, int g) {
  const int j = (r >> 2) & 1, c = 4 * (r >> 3) + (r & 3);
  return PackGeo<D>::kKe + (c * PackGeo<D>::NG + g) * 2 + j;
}
template <int D> __device__ __forceinline__ int v_exp_at(int r, int g) {
  return PackGeo<D>::kVe + ((r >> 3) * PackGeo<D>::NG + g) * 8 + (r & 7);
}

// Exponent byte of a group from the largest of its magnitudes' bit patterns (as integers: a NaN is the largest of all).
__device__ __forceinline__ uint32_t group_exponent(uint32_t top) {
  if (top >= 0x7F800000u) return 255u;
  if (top < 0x03800000u) return 127u;                       // below 2^-120
  const uint32_t k = top >> 23;                             // biased
  return (top & 0x7FFFFFu) > 0x600000u && k < 254u ? k - 1 : k - 2;
}
// Code of a value of a group with that exponent byte and largest magnitude.
__device__ __forceinline__ uint32_t value_code(uint32_t bits, uint32_t exponent, uint32_t top) {
  if (exponent == 255u) return 7u;
  const uint32_t sign = bits >> 31 << 3;
  if (top < 0x03800000u) return sign;
  const float a = __uint_as_float(bits & 0x7FFFFFFFu) * __uint_as_float((254u - exponent) << 23);
  return sign | (uint32_t)((a > 0.25f) + (a >= 0.75f) + (a > 1.25f) + (a >= 1.75f) + (a > 2.5f) + (a >= 3.5f) + (a > 5.0f));
}
// 2^E from its byte; NaN from 255.
__device__ __forceinline__ float group_scale(uint32_t exponent) {
  return exponent == 255u ? __builtin_nanf("") : __uint_as_float(exponent << 23);
}
__device__ __forceinline__ float code_value(uint32_t code, float scale) {
  // 0, 0.5, 1, 1.5, 2, 3, 4, 6: doubled, they are 0 1 2 3 4 6 8 12
  const float a = (float)((0xC8643210u >> (4 * (code & 7u))) & 15u) * 0.5f;
  return (code & 8u ? -a : a) * scale;
}

// The same by the chip's conversions, two values at a time: byte `byte` of codes.  2^E is given as group_scale() has it; they read its
// exponent bits, and give NaN for 255.
__device__ __forceinline__ uint32_t bf16_pair(uint32_t codes, float scale, int byte) {
  bf16x2 r;
  switch (byte) {          // an immediate of the instruction
    case 0: r = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 0); break;
    case 1: r = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 1); break;
    case 2: r = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 2); break;
    default: r = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 3); break;
  }
  return __builtin_bit_cast(uint32_t, r);
}

// The same as two fp32 values.
__device__ __forceinline__ void f32_pair(uint32_t codes, float scale, int byte, float& a, float& b) {
  typedef float f32x2 __attribute__((ext_vector_type(2)));
  f32x2 r;
  switch (byte) {
    case 0: r = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, scale, 0); break;
    case 1: r = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, scale, 1); break;
    case 2: r = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, scale, 2); break;
    default: r = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, scale, 3); break;
  }
  a = r[0];
  b = r[1];
}

// Codes of two values into byte `byte` of codes; the quotient by 2^E rounded as value_code does.
__device__ __forceinline__ uint32_t pair_codes(uint32_t codes, float a, float b, float scale, int byte) {
  switch (byte) {
    case 0: return __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, a, b, scale, 0);
    case 1: return __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, a, b, scale, 1);
    case 2: return __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, a, b, scale, 2);
    default: return __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, a, b, scale, 3);
  }
}
__device__ __forceinline__ uint32_t pair_codes(uint32_t codes, uint32_t two_bf16, float scale, int byte) {
  const bf16x2 x = __builtin_bit_cast(bf16x2, two_bf16);
  switch (byte) {
    case 0: return __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(codes, x, scale, 0);
    case 1: return __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(codes, x, scale, 1);
    case 2: return __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(codes, x, scale, 2);
    default: return __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(codes, x, scale, 3);
  }
}

// `bytes` bytes at p, the same in all lanes; what lies past them reads as zeros and is not written.
__device__ __forceinline__ auto bytes_at(const void* p, uint32_t bytes) {
  const uint64_t a = reinterpret_cast<uint64_t>(p);        // (the compiler does not see that this is the same in all lanes)
  void* same = reinterpret_cast<void*>((uint64_t)__builtin_amdgcn_readfirstlane((uint32_t)(a >> 32)) << 32 |
                                       (uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((uint32_t)a));
  return __builtin_amdgcn_make_buffer_rsrc(same, 0, __builtin_amdgcn_readfirstlane(bytes), 0x00020000);
}
constexpr int kNonTemporal = 2;              // of buffer instructions

}  // namespace ltea
