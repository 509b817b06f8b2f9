// The codes of a group of 32 columns (8 bits with a shared exponent): four
// neighbouring lanes hold eight columns each.
#pragma once

#include "seq_common.h"

namespace emb {

constexpr int kCodeCols = 8;                              // columns a lane takes
constexpr int kCodeLanes = EMB_SAVED_GROUP / kCodeCols;   // lanes a group
static_assert(kCodeLanes == 4, "the group's exchange is one within a quad");

// largest of a quad's values, NaN and infinity being larger than any number as their bits
__device__ __forceinline__ uint32_t quad_max(uint32_t v) {
  v = max(v, (uint32_t)__builtin_amdgcn_mov_dpp((int)v, 0xb1, 0xf, 0xf, true));  // quad_perm:[1,0,3,2]
  return max(v, (uint32_t)__builtin_amdgcn_mov_dpp((int)v, 0x4e, 0xf, 0xf, true));  // [2,3,0,1]
}

// This lane's eight codes; returns the group's exponent as it is kept.  All
// four lanes of a quad take part (zeros for columns that are not there).
__device__ __forceinline__ uint8_t group_codes(const float (&x)[kCodeCols], u32x2& codes) {
  uint32_t top = 0;
#pragma unroll
  for (int i = 0; i < kCodeCols; ++i) top = max(top, __float_as_uint(x[i]) & 0x7fffffffu);
  top = quad_max(top);
  const bool fine = top < 0x7f800000u;
  // 127 * 2^e has the mantissa 0x7e0000: one more step of the exponent above it
  int e = (int)((top + 0x1ffffu) >> 23) - 133;
  e = min(max(e, -120), 121);
  const float inverse = __uint_as_float((uint32_t)(127 - e) << 23);
  uint32_t w[2] = {0u, 0u};
#pragma unroll
  for (int i = 0; i < kCodeCols; ++i) {
    float r = __builtin_rintf(x[i] * inverse);
    r = fminf(fmaxf(r, -127.f), 127.f);
    const uint32_t code = fine ? (uint32_t)(int)r & 0xffu : 0u;
    w[i / 4] |= code << (8 * (i % 4));
  }
  codes = u32x2{w[0], w[1]};
  return fine ? (uint8_t)(e + 127) : (uint8_t)255;
}

}  // namespace emb
