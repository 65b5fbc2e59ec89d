// Microscaled (MX) rows: blocks of 32 values, one E8M0 scale and a code per value.
//
// A row of `cols` values has B = ceil(cols / 32) blocks. Block scale byte s: 2^(s - 127), 255 NaN.
// Codes: E2M1 (kMx4: magnitudes 0, 0.5, 1, 1.5, 2, 3, 4, 6; 16 bytes a block, value i in nibble
// i % 2 of byte i / 2) or E4M3 (kMx8: 32 bytes a block); values past `cols` are zero codes.
// Quantisation of a block with largest magnitude a: s = max(floor(log2 a) - e + 127, 0) with e the
// exponent of the largest code (2 or 8), s = 0 for a zero block; code = round(x / 2^(s - 127)), nearest
// even, saturating at 6 / 448. A block that holds an infinity or a NaN gets s = 255 and zero codes: it
// reads back as NaN.
// A buffer of `rows` rows: the codes of all rows, then their scales [rows][B], then 16 to 31
// spare bytes that make up a multiple of 16 (reads of a row's scales go by 16).
#pragma once

#include "kernels.h"

namespace dn {

constexpr int kMxBlock = 32;

// code bytes of a block
constexpr int mx_block_bytes(int fmt) { return fmt == kMx4 ? 16 : 32; }
inline long long mx_blocks(long long cols) { return (cols + kMxBlock - 1) / kMxBlock; }

// Exponent of the largest code.
constexpr int mx_emax(int fmt) { return fmt == kMx4 ? 2 : 8; }

__device__ __forceinline__ unsigned mx_abs_bits(float x) { return __float_as_uint(x) & 0x7fffffffu; }

// Scale byte of a block from the largest |x| as bits (an infinity or a NaN has the largest).
template <int FMT> __device__ __forceinline__ unsigned mx_scale(unsigned amax_bits) {
  const int e = (int)(amax_bits >> 23);
  return e == 255 ? 255u : (unsigned)max(e - mx_emax(FMT), 0);
}

// The scale as the conversion instructions take it: they use the exponent field (0 stands for 2^-127).
__device__ __forceinline__ float mx_scale_f(unsigned s) { return __uint_as_float(s << 23); }

// Eight values -> eight E2M1 codes (nearest even, saturating: both are the instruction's).
__device__ __forceinline__ unsigned mx4_codes8(const float* v, unsigned s) {
  const float sc = mx_scale_f(s);
  unsigned w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(0u, v[0], v[1], sc, 0);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[2], v[3], sc, 1);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[4], v[5], sc, 2);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[6], v[7], sc, 3);
  return s == 255u ? 0u : w;
}

typedef short short2v __attribute__((ext_vector_type(2)));

// Four values -> four E4M3 codes. The instruction turns magnitudes past the format into NaN codes,
// so values are clamped to 448 scales first.
__device__ __forceinline__ unsigned mx8_codes4(const float* v, unsigned s) {
  const float sc = mx_scale_f(s), top = __uint_as_float(((s + 8u) << 23) | 0x600000u);  // 1.75 2^8 2^(s - 127)
  float c[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) c[e] = __builtin_amdgcn_fmed3f(v[e], -top, top);
  short2v w = {0, 0};
  w = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(w, c[0], c[1], sc, false);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(w, c[2], c[3], sc, true);
  return s == 255u ? 0u : __builtin_bit_cast(unsigned, w);
}

typedef float f32x2 __attribute__((ext_vector_type(2)));

// Eight E2M1 codes / four E4M3 codes -> values (exact; scale byte 255 gives NaN).
__device__ __forceinline__ void mx4_values8(unsigned w, unsigned s, float* v) {
  const float sc = mx_scale_f(s);
  const f32x2 a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, sc, 0), b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, sc, 1);
  const f32x2 c = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, sc, 2), d = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, sc, 3);
  v[0] = a[0], v[1] = a[1], v[2] = b[0], v[3] = b[1], v[4] = c[0], v[5] = c[1], v[6] = d[0], v[7] = d[1];
}
__device__ __forceinline__ void mx8_values4(unsigned w, unsigned s, float* v) {
  const float sc = mx_scale_f(s);
  const f32x2 a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(w, sc, false), b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(w, sc, true);
  v[0] = a[0], v[1] = a[1], v[2] = b[0], v[3] = b[1];
}

// Largest of the lanes of a quad / of a group of eight lanes, in every lane of it.
template <int CTRL> __device__ __forceinline__ unsigned dpp_umax(unsigned v) {
  return max(v, (unsigned)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, 0xf, 0xf, true));
}
__device__ __forceinline__ unsigned quad_umax(unsigned v) { return dpp_umax<0x4e>(dpp_umax<0xb1>(v)); }
__device__ __forceinline__ unsigned oct_umax(unsigned v) { return dpp_umax<0x141>(quad_umax(v)); }

}  // namespace dn
