// What the kernels over sequences of tokens share: launch descriptors, vectors
// of activations in their types, the logistic function.
#pragma once

#include "emb_common.h"
#include "kernels.h"

namespace emb {

// ------------------------------------------------------------ launches
// (each enqueues nothing and returns hipErrorNotSupported where a kernel's grid
// would be too large)

// HIP takes fewer than 2^32 work-items in a dimension of a grid
inline bool launchable(int64_t blocks, int threads) { return blocks < ((int64_t)1 << 32) / threads; }

struct TokenFwdLaunch {
  const void* W;
  const void* idx;
  const int32_t* offsets;
  int32_t idx64;
  TableOffsets ro;
  int32_t T, B, D, dtype, out_dtype;
  uint32_t rows;  // R
  int64_t N, ld;
  uint32_t pad;   // its row, or kNoRow
  float scale;
  void* out;
};
constexpr uint32_t kNoRow = 0xffffffffu;  // (R < 2^32, so no row has this number)
hipError_t launch_token_fwd(const TokenFwdLaunch& p, hipStream_t s);

struct TokenGradLaunch {
  const void* dy;
  int32_t dy_dtype;
  int64_t ld;
  const int32_t* perm;
  const int32_t* seg;
  const uint32_t* ukeys;
  const int32_t* num_unique;
  int32_t N, D;
  uint32_t rows, pad;
  float scale;
  float* grad;
  int32_t layout;
  void* ws;
  WsLayout lay;
  int32_t fuse, opt, dtype;
  float lr, eps;
  int32_t rounding;
  uint64_t seed;
  void* W;
  float* state;
};
hipError_t launch_token_grad(const TokenGradLaunch& p, hipStream_t s);
constexpr int kTokenMaxDim = 8192;

// 32-bit rows of one matrix of activations
struct Rows {
  char* p;
  int64_t ld;           // bytes from one row to the next
  const uint8_t* exps;  // 8-bit checkpoints
  int64_t ld_exps;
};

constexpr int kSpan = EMB_SCAN_SPAN;
// In the header of the recurrence's own workspace: error bit of a wait for the spans before that ran out, and the
// wait's site (the dedup's and the combine's bits are 1, 2 and 4, their sites below 0x400)
constexpr uint32_t kScanError = 8u, kSiteScan = 0x400u;

struct ScanLaunch {
  int64_t N;
  int32_t M, D, dtype, grad_dtype, gated;
  const int32_t* offsets;
  Rows x, f, o, y, dy, dx, df, dO;
  const float* bias;
  const float* h0;
  float* h_last;
  float* states;
  const float* dh_last;
  float* dbias;
  float* dh0;
  int32_t vector;  // columns a lane may take from a row at once, by alignment (1 or 2 of 16 bits)
  char* ws;
};
size_t scan_ws_bytes(int64_t N, int32_t D);
hipError_t launch_scan_fwd(const ScanLaunch& p, hipStream_t s);
hipError_t launch_scan_bwd(const ScanLaunch& p, hipStream_t s);

struct StepLaunch {
  int64_t N;
  int32_t D, dtype, gated, vector;
  Rows x, f, o, y;
  const float* bias;
  float* state;
  int64_t num_slots;
  const int32_t* slots;
};
hipError_t launch_scan_step(const StepLaunch& p, hipStream_t s);

struct SaveLaunch {
  int64_t N;
  int32_t D, dtype, aligned;
  Rows full, saved;
};
hipError_t launch_save(const SaveLaunch& p, hipStream_t s);
hipError_t launch_restore(const SaveLaunch& p, hipStream_t s);

struct WeightGradLaunch {
  int64_t N;
  int32_t K, F, dtype, add, aligned;
  Rows x, dy;
  float* dw;
  float* ws;
};
size_t weight_grad_ws_bytes(int64_t N, int32_t K, int32_t F);
hipError_t launch_weight_grad(const WeightGradLaunch& p, hipStream_t s);

// Outputs of more bytes than the L2 caches hold together are stored past them
// (nontemporal): nothing of them would be found there, and a stored line then
// takes no line's place.  65536 rows of 2048 bf16 values looked up: 81 -> 55 us;
// a table gradient of 205 MB: 117 -> 86; the recurrence forward and backward,
// 32768 x 2048: 393 -> 374.  Smaller outputs stay, for what reads them next.
constexpr int64_t kStreamBytes = (int64_t)32 << 20;

// ------------------------------------------------------------ device helpers

// bf16 as it lies in memory
struct bf16 {
  uint16_t b;
};

// fp32 to bf16, nearest even, two at a time (one instruction on gfx950; NaN stays NaN)
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
  const bf16x2 v = __builtin_convertvector(f32x2{lo, hi}, bf16x2);
  return __builtin_bit_cast(uint32_t, v);
}
__device__ __forceinline__ float bf16_lo(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float bf16_hi(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }

// Words of V values of type T: what one lane loads or stores of a row.
template <typename T, int V>
struct Vec;
template <int V>
struct Vec<float, V> {
  static constexpr int kBytes = 4 * V;
  float x[V];
  __device__ __forceinline__ void load(const void* p) {
    if constexpr (V == 1) {
      x[0] = *static_cast<const float*>(p);
    } else if constexpr (V == 2) {
      const f32x2 t = *static_cast<const f32x2*>(p);
      x[0] = t.x, x[1] = t.y;
    } else {
#pragma unroll
      for (int i = 0; i < V / 4; ++i) {
        const f32x4 t = static_cast<const f32x4*>(p)[i];
        x[4 * i] = t.x, x[4 * i + 1] = t.y, x[4 * i + 2] = t.z, x[4 * i + 3] = t.w;
      }
    }
  }
  // V values one by one, where the address is aligned to a value alone
  __device__ __forceinline__ void load_each(const void* p) {
#pragma unroll
    for (int i = 0; i < V; ++i) x[i] = static_cast<const float*>(p)[i];
  }
  __device__ __forceinline__ void zero() {
#pragma unroll
    for (int i = 0; i < V; ++i) x[i] = 0.f;
  }
  __device__ __forceinline__ float get(int i) const { return x[i]; }
  __device__ __forceinline__ static void store(void* p, const float (&v)[V]) {
    if constexpr (V == 1) {
      *static_cast<float*>(p) = v[0];
    } else if constexpr (V == 2) {
      *static_cast<f32x2*>(p) = f32x2{v[0], v[1]};
    } else {
#pragma unroll
      for (int i = 0; i < V / 4; ++i)
        static_cast<f32x4*>(p)[i] = f32x4{v[4 * i], v[4 * i + 1], v[4 * i + 2], v[4 * i + 3]};
    }
  }
  // past the caches
  __device__ __forceinline__ static void stream(void* p, const float (&v)[V]) {
    if constexpr (V == 1) {
      __builtin_nontemporal_store(v[0], static_cast<float*>(p));
    } else if constexpr (V == 2) {
      __builtin_nontemporal_store(f32x2{v[0], v[1]}, static_cast<f32x2*>(p));
    } else {
#pragma unroll
      for (int i = 0; i < V / 4; ++i)
        __builtin_nontemporal_store(f32x4{v[4 * i], v[4 * i + 1], v[4 * i + 2], v[4 * i + 3]}, static_cast<f32x4*>(p) + i);
    }
  }
  __device__ __forceinline__ static void store_each(void* p, const float (&v)[V]) {
#pragma unroll
    for (int i = 0; i < V; ++i) static_cast<float*>(p)[i] = v[i];
  }
};
template <int V>
struct Vec<bf16, V> {
  static constexpr int kBytes = 2 * V;
  static constexpr int kWords = (V + 1) / 2;
  uint32_t w[kWords];
  __device__ __forceinline__ void load(const void* p) {
    if constexpr (V == 1) {
      w[0] = *static_cast<const uint16_t*>(p);
    } else if constexpr (V == 2) {
      w[0] = *static_cast<const uint32_t*>(p);
    } else if constexpr (V == 4) {
      const u32x2 t = *static_cast<const u32x2*>(p);
      w[0] = t.x, w[1] = t.y;
    } else {
#pragma unroll
      for (int i = 0; i < V / 8; ++i) {
        const u32x4 t = static_cast<const u32x4*>(p)[i];
        w[4 * i] = t.x, w[4 * i + 1] = t.y, w[4 * i + 2] = t.z, w[4 * i + 3] = t.w;
      }
    }
  }
  __device__ __forceinline__ void load_each(const void* p) {
    const uint16_t* q = static_cast<const uint16_t*>(p);
#pragma unroll
    for (int i = 0; i < kWords; ++i) w[i] = q[2 * i] | (2 * i + 1 < V ? (uint32_t)q[2 * i + 1] << 16 : 0u);
  }
  __device__ __forceinline__ void zero() {
#pragma unroll
    for (int i = 0; i < kWords; ++i) w[i] = 0u;
  }
  __device__ __forceinline__ float get(int i) const { return i % 2 ? bf16_hi(w[i / 2]) : bf16_lo(w[i / 2]); }
  __device__ __forceinline__ static void store(void* p, const float (&v)[V]) {
    if constexpr (V == 1) {
      *static_cast<uint16_t*>(p) = (uint16_t)pack_bf16(v[0], 0.f);
    } else if constexpr (V == 2) {
      *static_cast<uint32_t*>(p) = pack_bf16(v[0], v[1]);
    } else if constexpr (V == 4) {
      *static_cast<u32x2*>(p) = u32x2{pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3])};
    } else {
#pragma unroll
      for (int i = 0; i < V / 8; ++i)
        static_cast<u32x4*>(p)[i] = u32x4{pack_bf16(v[8 * i], v[8 * i + 1]), pack_bf16(v[8 * i + 2], v[8 * i + 3]),
                                          pack_bf16(v[8 * i + 4], v[8 * i + 5]), pack_bf16(v[8 * i + 6], v[8 * i + 7])};
    }
  }
  __device__ __forceinline__ static void stream(void* p, const float (&v)[V]) {
    if constexpr (V == 1) {
      __builtin_nontemporal_store((uint16_t)pack_bf16(v[0], 0.f), static_cast<uint16_t*>(p));
    } else if constexpr (V == 2) {
      __builtin_nontemporal_store(pack_bf16(v[0], v[1]), static_cast<uint32_t*>(p));
    } else if constexpr (V == 4) {
      __builtin_nontemporal_store(u32x2{pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3])}, static_cast<u32x2*>(p));
    } else {
#pragma unroll
      for (int i = 0; i < V / 8; ++i)
        __builtin_nontemporal_store(u32x4{pack_bf16(v[8 * i], v[8 * i + 1]), pack_bf16(v[8 * i + 2], v[8 * i + 3]),
                                          pack_bf16(v[8 * i + 4], v[8 * i + 5]), pack_bf16(v[8 * i + 6], v[8 * i + 7])},
                                    static_cast<u32x4*>(p) + i);
    }
  }
  __device__ __forceinline__ static void store_each(void* p, const float (&v)[V]) {
#pragma unroll
    for (int i = 0; i < V; ++i) static_cast<uint16_t*>(p)[i] = (uint16_t)pack_bf16(v[i], 0.f);
  }
};

__device__ __forceinline__ int uniform(int v) { return __builtin_amdgcn_readfirstlane(v); }
__device__ __forceinline__ uint32_t lane_at(uint32_t v, int l) {
  return (uint32_t)__builtin_amdgcn_readlane((int)v, l);
}
__device__ __forceinline__ int lane_at(int v, int l) { return __builtin_amdgcn_readlane(v, l); }

// Number of values below or equal to `v` among the sorted p[0 .. n-1], found by
// the whole wavefront: 64 probes a round, so two rounds up to 4096 values.
template <typename T>
__device__ __forceinline__ int wave_upper_bound(const T* p, int n, T v, int lane) {
  int lo = 0, len = n;  // the answer lies in lo .. lo + len
  while (len > 0) {
    const int step = (len + kWave - 1) / kWave;
    const int at = lane * step + step - 1;  // last value of this lane's part
    const bool le = at < len ? p[lo + at] <= v : false;
    const int parts = __popcll(__ballot(le));  // whole parts at or below v
    lo += parts * step;
    len = min(len - parts * step, step - 1);
    if (step == 1) break;
  }
  return uniform(lo);
}

}  // namespace emb
