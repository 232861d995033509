// Numbers of 8 or 4 bits with a power of two for every 32 channels of a head (pf_mx_format): value = code * 2^(byte - 127).
//
// The powers of two are bounded so that every value is a normal bf16 number: decoding is exact, in both types of rows.  gfx950 decodes two
// codes to an instruction, the power of two included (byte 255 gives NaN), and encodes two numbers to one, ties to even: both looked at over all
// codes, all bf16 numbers and all powers in use.
#pragma once
#include "../../include/pfstage.h"
#include "common.h"

namespace pf {

template <int FMT> struct Mx;
template <> struct Mx<PF_MX_E4M3> {
  static constexpr int BITS = 8;
  static constexpr unsigned kTop = 0x43e00000;                // 448 as a float
  static constexpr int kLeast = -117, kMost = 119;            // exponents of blocks
};
template <> struct Mx<PF_MX_E2M1> {
  static constexpr int BITS = 4;
  static constexpr unsigned kTop = 0x40c00000;                // 6
  static constexpr int kLeast = -125, kMost = 125;
};

inline int mx_row_bytes(int format, int head_dim) { return format == PF_MX_E4M3 ? (head_dim + 15) / 16 * 16 : (head_dim + 31) / 32 * 16; }
inline int mx_blocks(int head_dim) { return (head_dim + PF_MX_BLOCK - 1) / PF_MX_BLOCK; }

// Codes 2 i and 2 i + 1 of a word, times 2^(e - 127) for the float with exponent bits e.
#if defined(__HIP_DEVICE_COMPILE__)
typedef __bf16 mx_bf16x2 __attribute__((ext_vector_type(2)));
typedef float mx_f32x2 __attribute__((ext_vector_type(2)));
typedef short mx_s16x2 __attribute__((ext_vector_type(2)));
template <int FMT, int I>
__device__ __forceinline__ unsigned mx_decode_bf16(unsigned word, float power) {
  if constexpr (FMT == PF_MX_E4M3) return __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(word, power, I != 0));
  else return __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(word, power, I));
}
template <int FMT, int I>
__device__ __forceinline__ float2 mx_decode_f32(unsigned word, float power) {
  mx_f32x2 x;
  if constexpr (FMT == PF_MX_E4M3) x = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(word, power, I != 0);
  else x = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(word, power, I);
  return make_float2(x[0], x[1]);
}
#else   // the host pass only parses the kernels
template <int FMT, int I> __device__ unsigned mx_decode_bf16(unsigned, float) { return 0; }
template <int FMT, int I> __device__ float2 mx_decode_f32(unsigned, float) { return float2{}; }
#endif
__device__ __forceinline__ float mx_power(unsigned byte) { return __uint_as_float(byte << 23); }

// Codes of eight numbers of a block, as they are in a row, whose largest magnitude has the bits `most` of a float; returns the block's byte.
// Past the largest number e4m3 gives NaN for what is at most that times the largest power: there the numbers are bounded first.
template <int FMT, typename W>
__device__ __forceinline__ unsigned mx_encode(W row, unsigned most, unsigned (&code)[2]) {
  using M = Mx<FMT>;
  constexpr unsigned top_mant = M::kTop & 0x7fffffu, kLast = M::kTop + ((unsigned)M::kMost << 23);
  int e = (int)((most + 0x7fffffu - top_mant) >> 23) - (int)(M::kTop >> 23);   // the least with most <= top 2^e
  e = e < M::kLeast ? M::kLeast : e > M::kMost ? M::kMost : e;
  const float power = __uint_as_float((unsigned)(e + 127) << 23);
  code[0] = code[1] = 0;
#if defined(__HIP_DEVICE_COMPILE__)
  if constexpr (FMT == PF_MX_E4M3) {
    if (__builtin_amdgcn_ballot_w64(most > kLast) != 0) row.bound(kLast);
  }
  if constexpr (W::N == 1) {
    const auto at = [&](int i) __attribute__((always_inline)) { return __builtin_bit_cast(mx_bf16x2, (unsigned)row.w[0][i]); };
    if constexpr (FMT == PF_MX_E4M3) {
      mx_s16x2 c = {0, 0};
      c = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(c, at(0), power, false);
      c = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(c, at(1), power, true);
      code[0] = __builtin_bit_cast(unsigned, c);
      c = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(c, at(2), power, false);
      c = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(c, at(3), power, true);
      code[1] = __builtin_bit_cast(unsigned, c);
    } else {
      code[0] = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(code[0], at(0), power, 0);
      code[0] = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(code[0], at(1), power, 1);
      code[0] = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(code[0], at(2), power, 2);
      code[0] = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(code[0], at(3), power, 3);
    }
  } else {
    if constexpr (FMT == PF_MX_E4M3) {
      mx_s16x2 c = {0, 0};
      c = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(c, row[0], row[1], power, false);
      c = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(c, row[2], row[3], power, true);
      code[0] = __builtin_bit_cast(unsigned, c);
      c = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(c, row[4], row[5], power, false);
      c = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(c, row[6], row[7], power, true);
      code[1] = __builtin_bit_cast(unsigned, c);
    } else {
      code[0] = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(code[0], row[0], row[1], power, 0);
      code[0] = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(code[0], row[2], row[3], power, 1);
      code[0] = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(code[0], row[4], row[5], power, 2);
      code[0] = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(code[0], row[6], row[7], power, 3);
    }
  }
#endif
  const bool none = most >= 0x7f800000u;
  code[0] = none ? 0 : code[0];
  code[1] = none ? 0 : code[1];
  return none ? 255u : (unsigned)(e + 127);
}

// Eight codes of a block (one or two words) as bf16 or floats, four to a quadruple.
typedef unsigned mx_u32x4 __attribute__((ext_vector_type(4)));
template <int FMT>
__device__ __forceinline__ void mx_unit(const unsigned (&code)[2], float power, mx_u32x4 (&out)[1]) {
  if constexpr (FMT == PF_MX_E4M3)
    out[0] = mx_u32x4{mx_decode_bf16<FMT, 0>(code[0], power), mx_decode_bf16<FMT, 1>(code[0], power), mx_decode_bf16<FMT, 0>(code[1], power),
                      mx_decode_bf16<FMT, 1>(code[1], power)};
  else
    out[0] = mx_u32x4{mx_decode_bf16<FMT, 0>(code[0], power), mx_decode_bf16<FMT, 1>(code[0], power), mx_decode_bf16<FMT, 2>(code[0], power),
                      mx_decode_bf16<FMT, 3>(code[0], power)};
}
template <int FMT>
__device__ __forceinline__ void mx_unit(const unsigned (&code)[2], float power, mx_u32x4 (&out)[2]) {
  constexpr bool WIDE = FMT == PF_MX_E4M3;
  const float2 a = mx_decode_f32<FMT, 0>(code[0], power), b = mx_decode_f32<FMT, 1>(code[0], power);
  const float2 c = mx_decode_f32<FMT, WIDE ? 0 : 2>(code[WIDE], power), d = mx_decode_f32<FMT, WIDE ? 1 : 3>(code[WIDE], power);
  out[0] = mx_u32x4{__float_as_uint(a.x), __float_as_uint(a.y), __float_as_uint(b.x), __float_as_uint(b.y)};
  out[1] = mx_u32x4{__float_as_uint(c.x), __float_as_uint(c.y), __float_as_uint(d.x), __float_as_uint(d.y)};
}

}  // namespace pf
