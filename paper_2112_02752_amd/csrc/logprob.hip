// Log probabilities of given tokens, entropy, top alternatives, the logits'
// gradient (gfx950).
//
//   z = scale x,  m = max x,  e_v = exp(scale (x_v - m)),  s = sum e
//   logp = scale (x_id - m) - log s
//   H = log s - (sum over v of e_v scale (x_v - m)) / s
//   dx_v = scale (dlogp (1[v = id] - p_v) - dH p_v (log p_v + H)),  p_v = e_v / s
//
// A row stays in the registers of one, four or sixteen wavefronts, as it lies
// in memory, between the largest value, the sums and the gradient, so it is
// read once and its gradient written once.  Rows that registers do not hold
// are read again for each.
#include "block_common.h"

namespace emb {

namespace {

constexpr float kLog2e = 1.44269504088896340736f;
constexpr float kLowest = -1e30f;  // in place of minus infinity where a probability of zero multiplies it

// The vectors of 16 bytes that a row lies in: the first and the last may be shared with its neighbours.
template <typename T>
struct Row {
  static constexpr int kSize = Vec<T, 1>::kBytes, kEach = 16 / kSize;
  const char* p;  // of the first vector
  int head;       // columns of it that come before the row's
  int cols, count;
  __device__ __forceinline__ Row(const char* at, int D) {
    head = (int)(((uintptr_t)at & 15u) / kSize);
    p = at - head * kSize;
    cols = D;
    count = (head + D + kEach - 1) / kEach;
  }
  // first column of a vector (negative in the first)
  __device__ __forceinline__ int column(int v) const { return v * kEach - head; }
  __device__ __forceinline__ bool whole(int v) const { return column(v) >= 0 && column(v) + kEach <= cols; }
  // minus infinity where there are no columns
  __device__ __forceinline__ Vec<T, kEach> load(int v) const {
    Vec<T, kEach> x;
    if (v < count && whole(v)) {
      x.load(p + (int64_t)v * 16);
    } else {
      float t[kEach];
#pragma unroll
      for (int i = 0; i < kEach; ++i) {
        const int c = column(v) + i;
        Vec<T, 1> one;
        t[i] = -INFINITY;
        if (v < count && c >= 0 && c < cols) {
          one.load(p + (int64_t)v * 16 + i * kSize);
          t[i] = one.get(0);
        }
      }
      Vec<T, kEach>::store(&x, t);
    }
    return x;
  }
  __device__ __forceinline__ void store(char* to, int v, const float (&t)[kEach]) const {
    if (whole(v)) {
      Vec<T, kEach>::store(to + (int64_t)v * 16, t);
    } else {
#pragma unroll
      for (int i = 0; i < kEach; ++i) {
        const float one[1] = {t[i]};
        if (column(v) + i >= 0 && column(v) + i < cols) Vec<T, 1>::store(to + (int64_t)v * 16 + i * kSize, one);
      }
    }
  }
};

__device__ __forceinline__ float wave_max(float v) {
#pragma unroll
  for (int k = 1; k < kWave; k *= 2) v = fmaxf(v, __shfl_xor(v, k, kWave));
  return v;
}
__device__ __forceinline__ float wave_sum(float v) {
#pragma unroll
  for (int k = 1; k < kWave; k *= 2) v += __shfl_xor(v, k, kWave);
  return v;
}

// Order of the alternatives: greater values first (NaN before all, both zeros alike), then lower columns.
__device__ __forceinline__ uint64_t order_key(float x, int col) {
  uint32_t u = __float_as_uint(x + 0.f);
  if (x != x) u = 0x7fffffffu;
  u = (u & 0x80000000u) != 0 ? ~u : u | 0x80000000u;
  return (uint64_t)u << 32 | (uint32_t)~col;
}
__device__ __forceinline__ float key_value(uint64_t key) {
  const uint32_t u = (uint32_t)(key >> 32);
  return __uint_as_float((u & 0x80000000u) != 0 ? u & 0x7fffffffu : ~u);
}
__device__ __forceinline__ uint64_t wave_max_key(uint64_t v) {
#pragma unroll
  for (int k = 1; k < kWave; k *= 2) {
    const uint64_t o = __shfl_xor((unsigned long long)v, k, kWave);
    v = o > v ? o : v;
  }
  return v;
}

__device__ __forceinline__ int64_t id_of(const LogpLaunch& a, int64_t row) {
  if (a.ids == nullptr) return -1;
  return a.id_bytes == 8 ? static_cast<const int64_t*>(a.ids)[row] : (int64_t) static_cast<const int32_t*>(a.ids)[row];
}

// What a row's gradient is made of: dx_v = p_v (all + slope (z_v - m)) + at the id's column `hot`
struct Slope {
  float top, c, inv, all, slope, hot;
  int64_t id;
  __device__ __forceinline__ Slope(const LogpLaunch& a, int64_t row, float top_, float sum, float entropy) {
    id = id_of(a, row);
    const bool real = id >= 0 && id < a.D, none = top_ == -INFINITY;
    const float dl = real && !none && a.dlogp != nullptr ? a.dlogp[row] : 0.f;
    const float dh = !none && a.dentropy != nullptr ? a.dentropy[row] : 0.f;
    // (no token can be: every factor is zero)
    top = none ? 0.f : top_;
    c = a.scale;
    inv = none ? 0.f : 1.f / sum;
    slope = -a.scale * dh;
    all = dh != 0.f ? a.scale * (-dl - dh * (entropy - logf(sum))) : -a.scale * dl;
    hot = a.scale * dl;
    if (!real) id = -1;
  }
  __device__ __forceinline__ float operator()(float x, int col) const {
    const float z = c * (x - top), e = __builtin_amdgcn_exp2f(z * kLog2e);
    const float d = e * inv * (all + slope * fmaxf(z, kLowest));
    return col == id ? d + hot : d;
  }
};

// W wavefronts a row, R vectors a lane in registers (0: none, the row is read again).
template <int W>
constexpr int kBlock = W <= 4 ? 256 : 64 * W;

template <typename T, int W, int R>
__global__ __launch_bounds__(kBlock<W>) void k_logp(LogpLaunch a) {
  constexpr int kTeam = 64 * W, kRows = kBlock<W> / kTeam, kEach = Row<T>::kEach;
  __shared__ float s_part[3][kBlock<W> / kWave];
  __shared__ uint64_t s_top[kBlock<W> / kWave][EMB_MAX_TOP];
  const int lane = threadIdx.x % kWave, wave = uniform(threadIdx.x / kWave), t = threadIdx.x % kTeam;
  const int64_t row = (int64_t)blockIdx.x * kRows + wave / W;
  if (row >= a.N) return;  // (W > 1: a row a block)
  const Row<T> r(a.logits.p + row * a.logits.ld, a.D);
  Vec<T, kEach> x[R > 0 ? R : 1];
  if constexpr (R > 0) {
#pragma unroll
    for (int i = 0; i < R; ++i) x[i] = r.load(t + i * kTeam);
  }
  auto each = [&](auto f) {
    if constexpr (R > 0) {
#pragma unroll
      for (int i = 0; i < R; ++i) f(x[i], t + i * kTeam);
    } else {
      for (int v = t; v < r.count; v += kTeam) f(r.load(v), v);
    }
  };
  float top = -INFINITY;
  each([&](const Vec<T, kEach>& v, int) {
#pragma unroll
    for (int k = 0; k < kEach; ++k) top = fmaxf(top, v.get(k));
  });
  top = wave_max(top);
  if constexpr (W > 1) {
    if (lane == 0) s_part[0][wave] = top;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < W; ++w) top = fmaxf(top, s_part[0][w]);
  }
  // (where no token can be, every difference would be NaN)
  const float base = top == -INFINITY ? 0.f : top;
  float sum = 0.f, along = 0.f;
  each([&](const Vec<T, kEach>& v, int) {
#pragma unroll
    for (int k = 0; k < kEach; ++k) {
      const float z = a.scale * (v.get(k) - base), e = __builtin_amdgcn_exp2f(z * kLog2e);
      sum += e;
      along += e * fmaxf(z, kLowest);
    }
  });
  sum = wave_sum(sum);
  along = wave_sum(along);
  if constexpr (W > 1) {
    if (lane == 0) s_part[1][wave] = sum, s_part[2][wave] = along;
    __syncthreads();
    sum = along = 0.f;
#pragma unroll
    for (int w = 0; w < W; ++w) sum += s_part[1][w], along += s_part[2][w];
  }
  if (sum != sum) top = NAN;  // (a largest value passes NaN over)
  const bool none = top == -INFINITY;
  const float log_sum = logf(sum), entropy = none ? 0.f : log_sum - along / sum;
  if (t == 0) {
    const int64_t id = id_of(a, row);
    if (a.logp != nullptr) {
      float l = 0.f;
      if (id >= 0 && id < a.D) {
        Vec<T, 1> v;
        v.load(a.logits.p + row * a.logits.ld + id * Row<T>::kSize);
        l = none ? -INFINITY : a.scale * (v.get(0) - base) - log_sum;
      }
      a.logp[row] = l;
    }
    if (a.entropy != nullptr) a.entropy[row] = entropy;
    if (a.stats != nullptr) Vec<float, 4>::store(a.stats + row * kStats, {top, sum, entropy, 0.f});
  }
  if (a.dlogits.p != nullptr) {
    // in place: the id's logit is read before it is overwritten
    if constexpr (W > 1) {
      if (a.dlogits.p == a.logits.p) __syncthreads();
    } else {
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    }
    const Slope d(a, row, top, sum, entropy);
    char* to = a.dlogits.p + row * a.dlogits.ld;
    const bool same = (((uintptr_t)to ^ (uintptr_t)(a.logits.p + row * a.logits.ld)) & 15u) == 0;
    each([&](const Vec<T, kEach>& v, int at) {
      if (at >= r.count) return;
      float g[kEach];
#pragma unroll
      for (int k = 0; k < kEach; ++k) g[k] = d(v.get(k), r.column(at) + k);
      if (same) {
        r.store(to - r.head * Row<T>::kSize, at, g);
      } else {
#pragma unroll
        for (int k = 0; k < kEach; ++k) {
          const float one[1] = {g[k]};
          const int c = r.column(at) + k;
          if (c >= 0 && c < a.D) Vec<T, 1>::store(to + (int64_t)c * Row<T>::kSize, one);
        }
      }
    });
  }
  if (a.top == 0) return;
  // Every wavefront's best, one after another; a lane looks through its columns again when its best has been taken.
  auto best_below = [&](uint64_t limit) {
    uint64_t best = 0;
    each([&](const Vec<T, kEach>& v, int at) {
#pragma unroll
      for (int k = 0; k < kEach; ++k) {
        const int c = r.column(at) + k;
        if (c < 0 || c >= a.D) continue;
        const uint64_t key = order_key(v.get(k), c);
        if (key < limit && key > best) best = key;
      }
    });
    return best;
  };
  uint64_t mine = best_below(~0ull);
  for (int i = 0; i < a.top; ++i) {
    const uint64_t best = wave_max_key(mine);  // (0: no column is left)
    if (lane == 0) s_top[wave][i] = best;
    if (best != 0 && mine == best) mine = best_below(best);
  }
  auto put = [&](int i, uint64_t key) {
    a.top_ids[row * a.top + i] = (int32_t)~(uint32_t)key;
    a.top_logp[row * a.top + i] = none ? -INFINITY : a.scale * (key_value(key) - base) - log_sum;
  };
  if constexpr (W > 1) {
    __syncthreads();
    if (wave > 0) return;
    // the wavefronts' lists, merged
    int taken = 0;
    uint64_t next = lane < W ? s_top[lane][0] : 0;
    for (int i = 0; i < a.top; ++i) {
      const uint64_t best = wave_max_key(next);
      if (lane == 0) put(i, best);
      if (next == best && lane < W) {
        ++taken;
        next = taken < a.top ? s_top[lane][taken] : 0;
      }
    }
  } else {
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
    if (lane < a.top) put(lane, s_top[wave][lane]);
  }
}

// The gradient from the forward's statistics: each row's vectors by blocks.
constexpr int kGradVecs = 4;
template <typename T>
__global__ __launch_bounds__(256) void k_logp_bwd(LogpLaunch a, int per) {
  constexpr int kEach = Row<T>::kEach;
  const int64_t row = blockIdx.x / per;
  const int part = (int)(blockIdx.x % per);
  const Row<T> r(a.logits.p + row * a.logits.ld, a.D);
  const float* st = a.stats + row * kStats;
  const Slope d(a, row, st[0], st[1], st[2]);
  char* to = a.dlogits.p + row * a.dlogits.ld;
  const bool same = (((uintptr_t)to ^ (uintptr_t)(a.logits.p + row * a.logits.ld)) & 15u) == 0;
  Vec<T, kEach> x[kGradVecs];
  const int at = part * 256 * kGradVecs + threadIdx.x;
#pragma unroll
  for (int i = 0; i < kGradVecs; ++i) x[i] = r.load(at + i * 256);
#pragma unroll
  for (int i = 0; i < kGradVecs; ++i) {
    const int v = at + i * 256;
    if (v >= r.count) break;
    float g[kEach];
#pragma unroll
    for (int k = 0; k < kEach; ++k) g[k] = d(x[i].get(k), r.column(v) + k);
    if (same) {
      r.store(to - r.head * Row<T>::kSize, v, g);
    } else {
#pragma unroll
      for (int k = 0; k < kEach; ++k) {
        const float one[1] = {g[k]};
        const int c = r.column(v) + k;
        if (c >= 0 && c < a.D) Vec<T, 1>::store(to + (int64_t)c * Row<T>::kSize, one);
      }
    }
  }
}

template <typename T, int W, int R>
hipError_t go(const LogpLaunch& p, hipStream_t s) {
  constexpr int kRows = kBlock<W> / (64 * W);
  const int64_t blocks = (p.N + kRows - 1) / kRows;
  if (!launchable(blocks, kBlock<W>)) return hipErrorNotSupported;
  k_logp<T, W, R><<<(unsigned)blocks, kBlock<W>, 0, s>>>(p);
  return hipGetLastError();
}

// most vectors a row of D columns lies in
template <typename T>
int64_t vectors_of(int32_t D) {
  constexpr int kEach = Row<T>::kEach;
  return ((int64_t)D + 2 * (kEach - 1)) / kEach;
}

template <typename T>
hipError_t by_width(const LogpLaunch& p, hipStream_t s) {
  const int64_t n = vectors_of<T>(p.D);
  if (n <= 64 * 2) return go<T, 1, 2>(p, s);
  if (n <= 64 * 8) return go<T, 1, 8>(p, s);
  if (n <= 256 * 8) return go<T, 4, 8>(p, s);
  if (n <= 1024 * 4) return go<T, 16, 4>(p, s);
  if (n <= 1024 * 8) return go<T, 16, 8>(p, s);
  if (n <= 1024 * 16) return go<T, 16, 16>(p, s);
  return go<T, 16, 0>(p, s);
}

}  // namespace

hipError_t launch_logp(const LogpLaunch& p, hipStream_t s) {
  return p.dtype == EMB_FP32 ? by_width<float>(p, s) : by_width<bf16>(p, s);
}

hipError_t launch_logp_bwd(const LogpLaunch& p, hipStream_t s) {
  const int64_t n = p.dtype == EMB_FP32 ? vectors_of<float>(p.D) : vectors_of<bf16>(p.D);
  const int64_t per = (n + 256 * kGradVecs - 1) / (256 * kGradVecs);
  if (!launchable(per * p.N, 256)) return hipErrorNotSupported;
  const unsigned blocks = (unsigned)(per * p.N);
  if (p.dtype == EMB_FP32) k_logp_bwd<float><<<blocks, 256, 0, s>>>(p, (int)per);
  else k_logp_bwd<bf16><<<blocks, 256, 0, s>>>(p, (int)per);
  return hipGetLastError();
}

}  // namespace emb
