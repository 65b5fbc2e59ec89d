// Register layout of a 32 x 32 accumulator block <-> rows as they are stored.
#pragma once

#include "common.h"

namespace dn {

__device__ __forceinline__ unsigned pack_bf16(float a, float b) {
  const bf16x2 v = {static_cast<bf16>(a), static_cast<bf16>(b)};
  return __builtin_bit_cast(unsigned, v);
}

// v_permlane32_swap: lanes 32 - 63 of a and lanes 0 - 31 of b trade places.
struct Pair {
  unsigned a, b;
};
__device__ __forceinline__ Pair swap32(unsigned a, unsigned b) {
  const auto r = __builtin_amdgcn_permlane32_swap(a, b, false, false);
  return Pair{r[0], r[1]};
}

// v_permlane16_swap: the odd 16-lane rows of a and the even ones of b trade places.
__device__ __forceinline__ Pair swap16(unsigned a, unsigned b) {
  const auto r = __builtin_amdgcn_permlane16_swap(a, b, false, false);
  return Pair{r[0], r[1]};
}

// Register layout (lane: row l % 32) <-> store layout (lane: row l % 16, a later column group
// in the odd 16-lane rows): a, b hold two column groups of 32 rows on one side, 16-row
// halves of both groups on the other. Self-inverse.
__device__ __forceinline__ void rows16(uint4& a, uint4& b) {
  const Pair x = swap16(a.x, b.x), y = swap16(a.y, b.y), z = swap16(a.z, b.z), w = swap16(a.w, b.w);
  a = make_uint4(x.a, y.a, z.a, w.a);
  b = make_uint4(x.b, y.b, z.b, w.b);
}
__device__ __forceinline__ void rows16(f32x4& a, f32x4& b) {
  uint4 u = __builtin_bit_cast(uint4, a), v = __builtin_bit_cast(uint4, b);
  rows16(u, v);
  a = __builtin_bit_cast(f32x4, u);
  b = __builtin_bit_cast(f32x4, v);
}

// Two groups of four columns, v0 of g and v1 of g + 1 (g even) -> 8 consecutive columns of the
// row in 16 bytes: columns 8 g .. in lanes 0 - 31, 8 g + 8 .. in lanes 32 - 63.
__device__ __forceinline__ uint4 bf16_row8(const float* v0, const float* v1) {
  const Pair x = swap32(pack_bf16(v0[0], v0[1]), pack_bf16(v1[0], v1[1]));
  const Pair y = swap32(pack_bf16(v0[2], v0[3]), pack_bf16(v1[2], v1[3]));
  return make_uint4(x.a, y.a, x.b, y.b);
}

}  // namespace dn
