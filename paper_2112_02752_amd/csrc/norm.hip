// Residual addition, dropout and root-mean-square norm (gfx950).
//
//   t = r + m x / (1 - p)                      (m: kept or not)
//   y = w n,  n = t / sqrt(mean(t^2) + eps)
//   dt = a + (w dy - n mean(w dy n)) / sqrt(mean(t^2) + eps)
//   dx = m dt / (1 - p),  dw = sum over rows of dy n
//
// A row stays in the registers of one to eight wavefronts between the sum of
// its squares and its norm, so every matrix is read or written once.  The
// backward sums the squares again (the row is there anyhow), so nothing is kept
// of the forward but t.  A mask is never stored: a draw is a function of the
// seed, the row and the column; 16 bits a value, so a share is held to 2^-16.
//
// Bound by the bytes.  32768 x 2048 bf16 with dropout: forward with the output in 8 bits
// 105 us (608 MB, 5.8 TB/s), backward 140 (671 MB, 4.8 TB/s) and 5 for the weight
// gradient's last sum.  Dropout alone, 65536 x 2048: 90 us, 6.0 TB/s.  64 x 1536: 3.4 us, one
// load and one exchange.
#include "block_common.h"
#include "saved_codes.h"

namespace emb {

namespace {

constexpr int kCols = 8;  // consecutive columns a lane takes at once

// splitmix64 (Steele, Lea and Flood 2014)
__host__ __device__ __forceinline__ uint64_t mix64(uint64_t z) {
  z = (z ^ (z >> 30)) * 0xbf58476d1ce4e5b9ull;
  z = (z ^ (z >> 27)) * 0x94d049bb133111ebull;
  return z ^ (z >> 31);
}
constexpr uint64_t kGolden = 0x9e3779b97f4a7c15ull;

// The eight columns from col on (a multiple of 8) of a row, kept and scaled or
// dropped.  `per` draws a row, four columns each.
__device__ __forceinline__ void drop_cols(const Drop& d, int64_t row, int32_t per, int col, float (&x)[kCols]) {
  const uint64_t c = (uint64_t)(d.first_row + row) * (uint64_t)(uint32_t)per + (uint64_t)(uint32_t)(col / 4) + 1u;
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const uint64_t z = mix64(d.key + (c + h) * kGolden);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t bits = (uint32_t)(z >> (16 * i)) & 0xffffu;
      x[4 * h + i] = bits < d.below ? 0.f : x[4 * h + i] * d.scale;
    }
  }
}

// `left` columns of a row from p on, zeros past them
template <typename T>
__device__ __forceinline__ void load_cols(const char* p, int left, bool aligned, float (&x)[kCols]) {
  if (aligned && left >= kCols) {
    Vec<T, kCols> v;
    v.load(p);
#pragma unroll
    for (int i = 0; i < kCols; ++i) x[i] = v.get(i);
  } else {
#pragma unroll
    for (int i = 0; i < kCols; ++i) {
      Vec<T, 1> v;
      v.zero();
      if (i < left) v.load(p + i * Vec<T, 1>::kBytes);
      x[i] = v.get(0);
    }
  }
}
template <typename T>
__device__ __forceinline__ void store_cols(char* p, int left, bool aligned, const float (&x)[kCols]) {
  if (aligned && left >= kCols) {
    Vec<T, kCols>::store(p, x);
  } else {
#pragma unroll
    for (int i = 0; i < kCols; ++i) {
      const float v[1] = {x[i]};
      if (i < left) Vec<T, 1>::store(p + i * Vec<T, 1>::kBytes, v);
    }
  }
}
// the same as it lies in memory
template <typename T>
__device__ __forceinline__ void load_vec(const char* p, int left, bool aligned, Vec<T, kCols>& x) {
  if (aligned && left >= kCols) {
    x.load(p);
  } else {
    float t[kCols];
    load_cols<T>(p, left, false, t);
    Vec<T, kCols>::store(&x, t);
  }
}
template <typename T>
constexpr int64_t kSize = Vec<T, 1>::kBytes;

// a value as type T holds it
template <typename T>
__device__ __forceinline__ float held(float v) {
  if constexpr (kSize<T> == 4) return v;
  else return bf16_lo(pack_bf16(v, 0.f));
}

// W wavefronts a row, K times eight columns a lane; a block has one row, or four of a wavefront each.
template <int W>
struct Block {
  static constexpr int kThreads = W == 1 ? 256 : 64 * W, kRows = kThreads / (64 * W);
};

// sums over a row's wavefronts (W > 1: by the whole block)
template <int W, int V>
__device__ __forceinline__ void row_sums(float (&v)[V], float* s_part) {
#pragma unroll
  for (int i = 0; i < V; ++i) v[i] = wave_sum(v[i]);
  if constexpr (W > 1) {
    const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
    __syncthreads();
    if (lane == 0) {
#pragma unroll
      for (int i = 0; i < V; ++i) s_part[wave * V + i] = v[i];
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < V; ++i) {
      v[i] = 0.f;
#pragma unroll
      for (int w = 0; w < W; ++w) v[i] += s_part[w * V + i];
    }
  }
}

template <typename T, typename R, int W, int K>
__global__ __launch_bounds__(Block<W>::kThreads) void k_norm_fwd(NormLaunch a) {
  __shared__ float s_part[W];
  const int lane = threadIdx.x % kWave, wave = uniform(threadIdx.x / kWave);
  const int64_t row = (int64_t)blockIdx.x * Block<W>::kRows + wave / W;
  if (row >= a.N) return;  // (W > 1: a row a block)
  const int32_t per = (a.D + 3) / 4;
  float t[K][kCols], ss[1] = {0.f};
#pragma unroll
  for (int k = 0; k < K; ++k) {
    const int col = ((k * W + wave % W) * kWave + lane) * kCols, left = a.D - col;
    load_cols<T>(a.x.p + row * a.x.ld + col * kSize<T>, left, a.aligned, t[k]);
    if (a.drop.below != 0 && left > 0) drop_cols(a.drop, row, per, col, t[k]);
    if (a.residual.p != nullptr) {
      float r[kCols];
      load_cols<R>(a.residual.p + row * a.residual.ld + col * kSize<R>, left, a.aligned, r);
#pragma unroll
      for (int i = 0; i < kCols; ++i) t[k][i] += r[i];
    }
    // the norm is that of the sum as its type holds it, which is what a backward pass reads
#pragma unroll
    for (int i = 0; i < kCols; ++i) {
      t[k][i] = held<R>(t[k][i]);
      ss[0] += t[k][i] * t[k][i];
    }
  }
  row_sums<W, 1>(ss, s_part);
  const float inv = 1.f / sqrtf(ss[0] / (float)a.D + a.eps);
#pragma unroll
  for (int k = 0; k < K; ++k) {
    const int col = ((k * W + wave % W) * kWave + lane) * kCols, left = a.D - col;
    if (a.total.p != nullptr) store_cols<R>(a.total.p + row * a.total.ld + col * kSize<R>, left, a.aligned, t[k]);
    float w[kCols];
    if (a.weight != nullptr) load_cols<float>(reinterpret_cast<const char*>(a.weight + col), left, a.aligned, w);
#pragma unroll
    for (int i = 0; i < kCols; ++i) {
      t[k][i] *= inv;
      if (a.weight != nullptr) t[k][i] *= w[i];
    }
    if (a.y.p != nullptr) store_cols<T>(a.y.p + row * a.y.ld + col * kSize<T>, left, a.aligned, t[k]);
    if (a.saved.p != nullptr) {
      // (columns past the row's end are zeros: so are their codes)
      float v[kCols];
#pragma unroll
      for (int i = 0; i < kCols; ++i) v[i] = i < left ? held<T>(t[k][i]) : 0.f;
      u32x2 codes;
      const uint8_t e = group_codes(v, codes);
      if (col / EMB_SAVED_GROUP * EMB_SAVED_GROUP < a.D) {
        *reinterpret_cast<u32x2*>(a.saved.p + row * a.saved.ld + col) = codes;
        if (lane % kCodeLanes == 0) const_cast<uint8_t*>(a.saved.exps)[row * a.saved.ld_exps + col / EMB_SAVED_GROUP] = e;
      }
    }
  }
}

// Rows are dealt to the blocks in turn; a lane sums its columns of dw over the
// rows of its wavefront, the block those of its wavefronts, k_norm_dw the blocks'.
// AHEAD: the next row's values are on their way while a row is worked on, as
// they lie in memory (of 16 bits each: registers do not hold more).
template <typename T, typename R, int W, int K, bool AHEAD>
__global__ __launch_bounds__(Block<W>::kThreads) void k_norm_bwd(NormLaunch a) {
  constexpr int kRows = Block<W>::kRows;
  __shared__ float s_part[2 * W];
  __shared__ float s_dw[kRows > 1 ? (kRows - 1) * K * kWave * kCols : 1];
  const int lane = threadIdx.x % kWave, wave = uniform(threadIdx.x / kWave);
  const int32_t per = (a.D + 3) / 4;
  const int64_t step = (int64_t)gridDim.x * kRows;
  auto column = [&](int k) { return ((k * W + wave % W) * kWave + lane) * kCols; };
  float dw[K][kCols] = {}, w[K][kCols];
#pragma unroll
  for (int k = 0; k < K; ++k) {
    if (a.weight != nullptr) {
      load_cols<float>(reinterpret_cast<const char*>(a.weight + column(k)), a.D - column(k), a.aligned, w[k]);
    } else {
#pragma unroll
      for (int i = 0; i < kCols; ++i) w[k][i] = 1.f;
    }
  }
  struct Loaded {
    Vec<R, kCols> t[K], arriving[K];
    Vec<T, kCols> g[K];
  };
  auto load = [&](int64_t row, Loaded& x) {
#pragma unroll
    for (int k = 0; k < K; ++k) {
      const int col = column(k), left = a.D - col;
      load_vec<R>(a.total.p + row * a.total.ld + col * kSize<R>, left, a.aligned, x.t[k]);
      load_vec<T>(a.dy.p + row * a.dy.ld + col * kSize<T>, left, a.aligned, x.g[k]);
      if (a.arriving.p != nullptr)
        load_vec<R>(a.arriving.p + row * a.arriving.ld + col * kSize<R>, left, a.aligned, x.arriving[k]);
    }
  };
  int64_t row = (int64_t)blockIdx.x * kRows + wave / W;
  Loaded x;
  if constexpr (AHEAD) {
    if (row < a.N) load(row, x);
  }
  for (; row < a.N; row += step) {
    Loaded next;
    if constexpr (AHEAD) {
      if (row + step < a.N) load(row + step, next);
    } else {
      load(row, x);
    }
    float sum[2] = {0.f, 0.f};
#pragma unroll
    for (int k = 0; k < K; ++k)
#pragma unroll
      for (int i = 0; i < kCols; ++i) {
        const float t = x.t[k].get(i);
        sum[0] += t * t;
        sum[1] += t * x.g[k].get(i) * w[k][i];
      }
    row_sums<W, 2>(sum, s_part);
    const float inv = 1.f / sqrtf(sum[0] / (float)a.D + a.eps);
    const float along = sum[1] * inv / (float)a.D;  // mean(w dy n)
#pragma unroll
    for (int k = 0; k < K; ++k) {
      const int col = column(k), left = a.D - col;
      float d[kCols];
#pragma unroll
      for (int i = 0; i < kCols; ++i) {
        const float n = x.t[k].get(i) * inv, g = x.g[k].get(i);
        dw[k][i] += g * n;
        d[i] = inv * (g * w[k][i] - n * along);
        if (a.arriving.p != nullptr) d[i] += x.arriving[k].get(i);
      }
      if (a.dtotal.p != nullptr) store_cols<R>(a.dtotal.p + row * a.dtotal.ld + col * kSize<R>, left, a.aligned, d);
      if (a.dbranch.p != nullptr) {
        if (a.drop.below != 0 && left > 0) drop_cols(a.drop, row, per, col, d);
        store_cols<T>(a.dbranch.p + row * a.dbranch.ld + col * kSize<T>, left, a.aligned, d);
      }
    }
    if constexpr (AHEAD) x = next;
  }
  if (a.dweight == nullptr) return;
  if constexpr (kRows > 1) {
    if (wave > 0) {
#pragma unroll
      for (int k = 0; k < K; ++k)
#pragma unroll
        for (int i = 0; i < kCols; ++i) s_dw[(((wave - 1) * K + k) * kCols + i) * kWave + lane] = dw[k][i];
    }
    __syncthreads();
    if (wave > 0) return;
#pragma unroll
    for (int r = 0; r < kRows - 1; ++r)
#pragma unroll
      for (int k = 0; k < K; ++k)
#pragma unroll
        for (int i = 0; i < kCols; ++i) dw[k][i] += s_dw[((r * K + k) * kCols + i) * kWave + lane];
  }
#pragma unroll
  for (int k = 0; k < K; ++k) {
    const int col = ((k * W + wave % W) * kWave + lane) * kCols, left = a.D - col;
    store_cols<float>(reinterpret_cast<char*>(a.ws + (int64_t)blockIdx.x * a.D + col), left, a.D % 4 == 0, dw[k]);
  }
}

// Sums of the blocks' rows of dw: 64 columns a block, 16 wavefronts take every 16th row.
__global__ __launch_bounds__(1024) void k_norm_dw(const float* parts, int count, int D, float* dw, int add) {
  __shared__ float s_sum[16][kWave];
  const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave, col = blockIdx.x * kWave + lane;
  float v = 0.f;
  constexpr int kAhead = 8;  // loads in flight
  if (col < D) {
    for (int r = wave; r < count; r += 16 * kAhead) {
      float x[kAhead];
#pragma unroll
      for (int i = 0; i < kAhead; ++i) x[i] = r + 16 * i < count ? parts[(int64_t)(r + 16 * i) * D + col] : 0.f;
#pragma unroll
      for (int i = 0; i < kAhead; ++i) v += x[i];
    }
  }
  s_sum[wave][lane] = v;
  __syncthreads();
  if (wave > 0 || col >= D) return;
#pragma unroll
  for (int w = 1; w < 16; ++w) v += s_sum[w][lane];
  dw[col] = add ? dw[col] + v : v;
}

template <typename T>
__global__ __launch_bounds__(256) void k_dropout(DropLaunch a) {
  const int per = (a.D + kCols - 1) / kCols;
  const int64_t at = (int64_t)blockIdx.x * 256 + threadIdx.x;
  const int64_t row = at / per;
  if (row >= a.N) return;
  const int col = (int)(at - row * per) * kCols, left = a.D - col;
  float x[kCols];
  load_cols<T>(a.x.p + row * a.x.ld + col * kSize<T>, left, a.aligned, x);
  drop_cols(a.drop, row, (a.D + 3) / 4, col, x);
  store_cols<T>(a.y.p + row * a.y.ld + col * kSize<T>, left, a.aligned, x);
}

// Blocks of the backward: as many rows of dw are left to add.  32768 x 2048 bf16: 140 us with 256, 512 or 1024, and
// 7, 11 and 26 more for adding them; narrow rows want more wavefronts to have as much in flight.
int64_t bwd_blocks(int64_t N, int32_t D, int rows) {
  const int64_t need = (N + rows - 1) / rows, most = D > 2 * kWave * kCols ? 256 : 512;
  return need < most ? need : most;
}

template <typename T, typename R, int W, int K>
hipError_t fwd(const NormLaunch& p, hipStream_t s) {
  const int64_t blocks = (p.N + Block<W>::kRows - 1) / Block<W>::kRows;
  if (!launchable(blocks, Block<W>::kThreads)) return hipErrorNotSupported;
  k_norm_fwd<T, R, W, K><<<(unsigned)blocks, Block<W>::kThreads, 0, s>>>(p);
  return hipGetLastError();
}
template <typename T, typename R, int W, int K>
hipError_t bwd(const NormLaunch& p, hipStream_t s) {
  const int64_t blocks = bwd_blocks(p.N, p.D, Block<W>::kRows);
  constexpr bool kAhead = kSize<T> == 2 && kSize<R> == 2;
  if (blocks > 0) k_norm_bwd<T, R, W, K, kAhead><<<(unsigned)blocks, Block<W>::kThreads, 0, s>>>(p);
  if (p.dweight != nullptr)
    k_norm_dw<<<(unsigned)((p.D + kWave - 1) / kWave), 1024, 0, s>>>(p.ws, (int)blocks, p.D, p.dweight, p.add);
  return hipGetLastError();
}

template <bool BACK, typename T, typename R>
hipError_t by_width(const NormLaunch& p, hipStream_t s) {
  auto go = [&](auto w, auto k) {
    if constexpr (BACK) return bwd<T, R, decltype(w)::value, decltype(k)::value>(p, s);
    else return fwd<T, R, decltype(w)::value, decltype(k)::value>(p, s);
  };
  using std::integral_constant;
  constexpr int kOne = kWave * kCols;
  if (p.D <= kOne) return go(integral_constant<int, 1>{}, integral_constant<int, 1>{});
  // (forward: more wavefronts with less each, 32768 x 2048 104 us instead of 115; the backward exchanges two
  // sums between them in every row: 140 either way)
  if (p.D <= 2 * kOne) return go(integral_constant<int, BACK ? 1 : 2>{}, integral_constant<int, BACK ? 2 : 1>{});
  if (p.D <= 4 * kOne) return go(integral_constant<int, BACK ? 1 : 4>{}, integral_constant<int, BACK ? 4 : 1>{});
  if (p.D <= 8 * kOne) return go(integral_constant<int, 4>{}, integral_constant<int, 2>{});
  if (p.D <= 16 * kOne) return go(integral_constant<int, 4>{}, integral_constant<int, 4>{});
  return go(integral_constant<int, 8>{}, integral_constant<int, 4>{});
}
template <bool BACK>
hipError_t by_type(const NormLaunch& p, hipStream_t s) {
  if (p.dtype == EMB_FP32) return by_width<BACK, float, float>(p, s);
  if (p.stream_dtype == EMB_FP32) return by_width<BACK, bf16, float>(p, s);
  return by_width<BACK, bf16, bf16>(p, s);
}

}  // namespace

Drop make_drop(float p, uint64_t seed, int64_t first_row) {
  Drop d{};
  d.below = (uint32_t)__builtin_rint((double)p * 65536.0);
  d.key = mix64(seed + kGolden);
  d.scale = (float)(65536.0 / (65536.0 - (double)d.below));
  d.first_row = first_row;
  return d;
}

size_t norm_ws_bytes(int64_t N, int32_t D) {
  return align256(sizeof(float) * (size_t)bwd_blocks(N, D, 1) * (size_t)D);
}

hipError_t launch_norm_fwd(const NormLaunch& p, hipStream_t s) { return by_type<false>(p, s); }
hipError_t launch_norm_bwd(const NormLaunch& p, hipStream_t s) { return by_type<true>(p, s); }

hipError_t launch_dropout(const DropLaunch& p, hipStream_t s) {
  const int64_t lanes = (int64_t)((p.D + kCols - 1) / kCols) * p.N;
  if (!launchable((lanes + 255) / 256, 256)) return hipErrorNotSupported;
  const unsigned blocks = (unsigned)((lanes + 255) / 256);
  if (p.dtype == EMB_BF16) k_dropout<bf16><<<blocks, 256, 0, s>>>(p);
  else k_dropout<float><<<blocks, 256, 0, s>>>(p);
  return hipGetLastError();
}

}  // namespace emb
