// Numbers of 8 or 4 bits with a power of two for every 32 channels of a head (pf_mx_format): value = code * 2^(byte - 127).
//
// The powers of two are bounded so that every value is a normal bf16 number: decoding is exact, in both types of rows.  gfx950 decodes two
// codes to an instruction, the power of two included (byte 255 gives NaN), and encodes with ties to even.
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
