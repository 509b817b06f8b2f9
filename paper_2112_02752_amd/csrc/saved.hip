// Activations in 8 bits and back (gfx950).  A group of 32 columns shares the
// exponent e, the smallest with max |v| <= 127 * 2^e; scaling by a power of two
// is exact, so a code is one rounding of the value and a restored value is
// exact in bf16.  A lane takes 8 columns of a row, four lanes a group: the
// group's largest magnitude needs two exchanges within a quad.  One pass over
// the data: bound by its bytes.  16384 x 3840 bf16 to 8 bits: 31 us, 6.1 TB/s; 1000 x
// 200 fp32: 2.9 us each way, a launch and one load.
#include "seq_common.h"

namespace emb {

namespace {

constexpr int kCols = 8;                          // columns a lane takes
constexpr int kLanes = EMB_SAVED_GROUP / kCols;   // lanes a group
static_assert(kLanes == 4, "the group's exchange is one within a quad");

// largest of a quad's values, NaN and infinity being larger than any number as their bits
__device__ __forceinline__ uint32_t quad_max(uint32_t v) {
  v = max(v, (uint32_t)__builtin_amdgcn_mov_dpp((int)v, 0xb1, 0xf, 0xf, true));  // quad_perm:[1,0,3,2]
  return max(v, (uint32_t)__builtin_amdgcn_mov_dpp((int)v, 0x4e, 0xf, 0xf, true));  // [2,3,0,1]
}

template <typename T>
__global__ __launch_bounds__(256) void k_save(SaveLaunch a) {
  const int per = (a.D + EMB_SAVED_GROUP - 1) / EMB_SAVED_GROUP * kLanes;  // lanes a row
  const int64_t at = (int64_t)blockIdx.x * 256 + threadIdx.x;
  const int64_t row = at / per;
  if (row >= a.N) return;  // (a row's lanes are whole quads)
  const int lane = (int)(at - row * per), col = lane * kCols;
  const char* src = a.full.p + row * a.full.ld + (int64_t)col * (int64_t)(Vec<T, kCols>::kBytes / kCols);
  float x[kCols];
  if (a.aligned && col + kCols <= a.D) {
    Vec<T, kCols> v;
    v.load(src);
#pragma unroll
    for (int i = 0; i < kCols; ++i) x[i] = v.get(i);
  } else {
#pragma unroll
    for (int i = 0; i < kCols; ++i) {
      Vec<T, 1> v;
      v.zero();
      if (col + i < a.D) v.load(src + i * Vec<T, 1>::kBytes);
      x[i] = v.get(0);
    }
  }
  uint32_t top = 0;
#pragma unroll
  for (int i = 0; i < kCols; ++i) top = max(top, __float_as_uint(x[i]) & 0x7fffffffu);
  top = quad_max(top);
  const bool fine = top < 0x7f800000u;
  // 127 * 2^e has the mantissa 0x7e0000: one more step of the exponent above it
  int e = (int)((top + 0x1ffffu) >> 23) - 133;
  e = min(max(e, -120), 121);
  const float inverse = __uint_as_float((uint32_t)(127 - e) << 23);
  uint32_t w[2] = {0u, 0u};
#pragma unroll
  for (int i = 0; i < kCols; ++i) {
    float r = __builtin_rintf(x[i] * inverse);
    r = fminf(fmaxf(r, -127.f), 127.f);
    const uint32_t code = fine ? (uint32_t)(int)r & 0xffu : 0u;
    w[i / 4] |= code << (8 * (i % 4));
  }
  *reinterpret_cast<u32x2*>(a.saved.p + row * a.saved.ld + col) = u32x2{w[0], w[1]};
  if (lane % kLanes == 0)
    const_cast<uint8_t*>(a.saved.exps)[row * a.saved.ld_exps + col / EMB_SAVED_GROUP] = fine ? (uint8_t)(e + 127) : 255;
}

template <typename T>
__global__ __launch_bounds__(256) void k_restore(SaveLaunch a) {
  const int per = (a.D + kCols - 1) / kCols;
  const int64_t at = (int64_t)blockIdx.x * 256 + threadIdx.x;
  const int64_t row = at / per;
  if (row >= a.N) return;
  const int col = (int)(at - row * per) * kCols;
  const u32x2 w = *reinterpret_cast<const u32x2*>(a.saved.p + row * a.saved.ld + col);
  // (255: infinity, and the codes are zeros)
  const float unit = __uint_as_float((uint32_t)a.saved.exps[row * a.saved.ld_exps + col / EMB_SAVED_GROUP] << 23);
  float x[kCols];
#pragma unroll
  for (int i = 0; i < kCols; ++i) x[i] = (float)(int8_t)((i < 4 ? w.x : w.y) >> (8 * (i % 4))) * unit;
  char* dst = a.full.p + row * a.full.ld + (int64_t)col * (int64_t)(Vec<T, kCols>::kBytes / kCols);
  if (a.aligned && col + kCols <= a.D) {
    Vec<T, kCols>::store(dst, x);
  } else {
#pragma unroll
    for (int i = 0; i < kCols; ++i) {
      const float v[1] = {x[i]};
      if (col + i < a.D) Vec<T, 1>::store(dst + i * Vec<T, 1>::kBytes, v);
    }
  }
}

}  // namespace

hipError_t launch_save(const SaveLaunch& p, hipStream_t s) {
  const int64_t lanes = (int64_t)((p.D + EMB_SAVED_GROUP - 1) / EMB_SAVED_GROUP) * kLanes * p.N;
  if (!launchable((lanes + 255) / 256, 256)) return hipErrorNotSupported;
  const unsigned blocks = (unsigned)((lanes + 255) / 256);
  if (p.dtype == EMB_BF16) k_save<bf16><<<blocks, 256, 0, s>>>(p);
  else k_save<float><<<blocks, 256, 0, s>>>(p);
  return hipGetLastError();
}

hipError_t launch_restore(const SaveLaunch& p, hipStream_t s) {
  const int64_t lanes = (int64_t)((p.D + kCols - 1) / kCols) * p.N;
  if (!launchable((lanes + 255) / 256, 256)) return hipErrorNotSupported;
  const unsigned blocks = (unsigned)((lanes + 255) / 256);
  if (p.dtype == EMB_BF16) k_restore<bf16><<<blocks, 256, 0, s>>>(p);
  else k_restore<float><<<blocks, 256, 0, s>>>(p);
  return hipGetLastError();
}

}  // namespace emb
