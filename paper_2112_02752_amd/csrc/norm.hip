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

template <typename T>
constexpr int64_t kSize = Vec<T, 1>::kBytes;

// Eight values at an address that is a multiple of one value's bytes: memory takes 16 bytes at any.  32769 x 233 bf16,
// forward: 12.7 us, with a load a value 44.
template <typename T>
struct __attribute__((packed, aligned(Vec<T, 1>::kBytes))) Eight {
  u32x4 w[Vec<T, kCols>::kBytes / 16];
};
// Columns col .. col + 7 of a row of D as they lie in memory, zeros past its end.  WHOLE: D is a multiple of eight, and a
// lane past the end gets the row's last columns (the caller's to leave out), so that no branch parts loads in flight:
// 32768 x 2048 bf16, backward: 138 us, with such branches 160.
template <typename T, bool WHOLE>
__device__ __forceinline__ void load_vec(const char* row, int col, int D, Vec<T, kCols>& x) {
  typedef Vec<T, kCols> V;
  static_assert(sizeof(Eight<T>) == sizeof(V), "eight values");
  if constexpr (WHOLE) {
    x = __builtin_bit_cast(V, *reinterpret_cast<const Eight<T>*>(row + min(col, D - kCols) * kSize<T>));
  } else if (D - col >= kCols) {
    x = __builtin_bit_cast(V, *reinterpret_cast<const Eight<T>*>(row + col * kSize<T>));
  } else {
    const char* const p = row + col * kSize<T>;
    const int left = D - col;
    float t[kCols];
#pragma unroll
    for (int i = 0; i < kCols; ++i) {
      Vec<T, 1> v;
      v.zero();
      if (i < left) v.load(p + i * kSize<T>);
      t[i] = v.get(0);
    }
    V::store(&x, t);
  }
}
template <typename T, bool WHOLE>
__device__ __forceinline__ void load_cols(const char* row, int col, int D, float (&x)[kCols]) {
  Vec<T, kCols> v;
  load_vec<T, WHOLE>(row, col, D, v);
#pragma unroll
  for (int i = 0; i < kCols; ++i) x[i] = v.get(i);
}
template <typename T, bool WHOLE>
__device__ __forceinline__ void store_cols(char* row, int col, int D, const float (&x)[kCols]) {
  if (WHOLE ? col < D : D - col >= kCols) {
    Vec<T, kCols> v;
    Vec<T, kCols>::store(&v, x);
    *reinterpret_cast<Eight<T>*>(row + col * kSize<T>) = __builtin_bit_cast(Eight<T>, v);
  } else if constexpr (!WHOLE) {
    char* const p = row + col * kSize<T>;
    const int left = D - col;
#pragma unroll
    for (int i = 0; i < kCols; ++i) {
      const float v[1] = {x[i]};
      if (i < left) Vec<T, 1>::store(p + i * kSize<T>, v);
    }
  }
}

// a value as type T holds it
template <typename T>
__device__ __forceinline__ float held(float v) {
  if constexpr (kSize<T> == 4) return v;
  else return bf16_lo(pack_bf16(v, 0.f));
}

// W wavefronts a row, K times eight columns a lane; or (W = K = 1) L lanes a row, so that narrow rows fill a wavefront.
// A block has one row, or those of four wavefronts.  Forward and backward in bf16, 30001 x 40: 17 us with 8 lanes a row, 42
// with 64; 32769 x 248: 31 with 32, 50 with 64.
template <int W>
constexpr int kBlock = W == 1 ? 256 : 64 * W;
template <int W, int L>
struct Block {
  static_assert(W == 1 || L == kWave, "whole wavefronts");
  static constexpr int kThreads = kBlock<W>, kWaves = kThreads / (64 * W), kEach = kWave / L;
  static constexpr int kRows = kWaves * kEach;
  // the row of a block, and the lane of the row, that a thread has
  static __device__ __forceinline__ int row(int wave) {
    return wave / W * kEach + (L == kWave ? 0 : (int)(threadIdx.x % kWave / L));
  }
};

// sum over L neighbouring lanes
template <int L>
__device__ __forceinline__ float lanes_sum(float v) {
  if constexpr (L == kWave) {
    return wave_sum(v);
  } else {
    static_assert(L == 8 || L == 16 || L == 32, "halves of a wavefront");
    v += lane_move<0xb1>(v);   // quad_perm:[1,0,3,2]
    v += lane_move<0x4e>(v);   // quad_perm:[2,3,0,1]
    v += lane_move<0x141>(v);  // row_half_mirror
    if constexpr (L > 8) v += lane_move<0x140>(v);  // row_mirror
    if constexpr (L > 16) v += __shfl_xor(v, 16);
    return v;
  }
}

// sums over a row's lanes (W > 1: by the whole block)
template <int W, int L, int V>
__device__ __forceinline__ void row_sums(float (&v)[V], float* s_part) {
#pragma unroll
  for (int i = 0; i < V; ++i) v[i] = lanes_sum<L>(v[i]);
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

template <typename T, typename R, int W, int K, int L, bool WHOLE>
__global__ __launch_bounds__(kBlock<W>) void k_norm_fwd(NormLaunch a) {
  __shared__ float s_part[W];
  const int lane = threadIdx.x % L, wave = uniform(threadIdx.x / kWave);
  const int64_t row = (int64_t)blockIdx.x * Block<W, L>::kRows + Block<W, L>::row(wave);
  if (row >= a.N) return;  // (W > 1: a row a block)
  const int32_t per = (a.D + 3) / 4;
  float t[K][kCols], ss[1] = {0.f};
#pragma unroll
  for (int k = 0; k < K; ++k) {
    const int col = ((k * W + wave % W) * kWave + lane) * kCols, left = a.D - col;
    load_cols<T, WHOLE>(a.x.p + row * a.x.ld, col, a.D, t[k]);
    if (a.drop.below != 0 && left > 0) drop_cols(a.drop, row, per, col, t[k]);
    if (a.residual.p != nullptr) {
      float r[kCols];
      load_cols<R, WHOLE>(a.residual.p + row * a.residual.ld, col, a.D, r);
#pragma unroll
      for (int i = 0; i < kCols; ++i) t[k][i] += r[i];
    }
    // the norm is that of the sum as its type holds it, which is what a backward pass reads
#pragma unroll
    for (int i = 0; i < kCols; ++i) {
      t[k][i] = !WHOLE || left > 0 ? held<R>(t[k][i]) : 0.f;
      ss[0] += t[k][i] * t[k][i];
    }
  }
  row_sums<W, L, 1>(ss, s_part);
  const float inv = 1.f / sqrtf(ss[0] / (float)a.D + a.eps);
#pragma unroll
  for (int k = 0; k < K; ++k) {
    const int col = ((k * W + wave % W) * kWave + lane) * kCols, left = a.D - col;
    if (a.total.p != nullptr) store_cols<R, WHOLE>(a.total.p + row * a.total.ld, col, a.D, t[k]);
    float w[kCols];
    if (a.weight != nullptr) load_cols<float, WHOLE>(reinterpret_cast<const char*>(a.weight), col, a.D, w);
#pragma unroll
    for (int i = 0; i < kCols; ++i) {
      t[k][i] *= inv;
      if (a.weight != nullptr) t[k][i] *= w[i];
    }
    if (a.y.p != nullptr) store_cols<T, WHOLE>(a.y.p + row * a.y.ld, col, a.D, t[k]);
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
template <typename T, typename R, int W, int K, int L, bool WHOLE, bool AHEAD>
__global__ __launch_bounds__(kBlock<W>) void k_norm_bwd(NormLaunch a) {
  constexpr int kRows = Block<W, L>::kRows, kWaves = Block<W, L>::kWaves;
  __shared__ float s_part[2 * W];
  __shared__ float s_dw[kWaves > 1 ? (kWaves - 1) * K * kWave * kCols : 1];
  const int lane = threadIdx.x % L, wave = uniform(threadIdx.x / kWave);
  const int32_t per = (a.D + 3) / 4;
  const int64_t step = (int64_t)gridDim.x * kRows;
  auto column = [&](int k) { return ((k * W + wave % W) * kWave + lane) * kCols; };
  float dw[K][kCols] = {}, w[K][kCols];
#pragma unroll
  for (int k = 0; k < K; ++k) {
    if (a.weight != nullptr) {
      load_cols<float, WHOLE>(reinterpret_cast<const char*>(a.weight), column(k), a.D, w[k]);
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
      const int col = column(k);
      load_vec<R, WHOLE>(a.total.p + row * a.total.ld, col, a.D, x.t[k]);
      load_vec<T, WHOLE>(a.dy.p + row * a.dy.ld, col, a.D, x.g[k]);
      if (a.arriving.p != nullptr)
        load_vec<R, WHOLE>(a.arriving.p + row * a.arriving.ld, col, a.D, x.arriving[k]);
    }
  };
  int64_t row = (int64_t)blockIdx.x * kRows + Block<W, L>::row(wave);
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
        const float t = x.t[k].get(i), along = t * x.g[k].get(i) * w[k][i];
        const bool there = !WHOLE || column(k) < a.D;
        sum[0] += there ? t * t : 0.f;
        sum[1] += there ? along : 0.f;
      }
    row_sums<W, L, 2>(sum, s_part);
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
      if (a.dtotal.p != nullptr) store_cols<R, WHOLE>(a.dtotal.p + row * a.dtotal.ld, col, a.D, d);
      if (a.dbranch.p != nullptr) {
        if (a.drop.below != 0 && left > 0) drop_cols(a.drop, row, per, col, d);
        store_cols<T, WHOLE>(a.dbranch.p + row * a.dbranch.ld, col, a.D, d);
      }
    }
    if constexpr (AHEAD) x = next;
  }
  if (a.dweight == nullptr) return;  // (by the arguments: all)
  // the rows of a wavefront
#pragma unroll
  for (int other = L; other < kWave; other *= 2)
#pragma unroll
    for (int i = 0; i < kCols; ++i) dw[0][i] += __shfl_xor(dw[0][i], other);
  if constexpr (kWaves > 1) {
    if (wave > 0) {
#pragma unroll
      for (int k = 0; k < K; ++k)
#pragma unroll
        for (int i = 0; i < kCols; ++i) s_dw[(((wave - 1) * K + k) * kCols + i) * kWave + lane] = dw[k][i];
    }
    __syncthreads();
    if (wave > 0) return;
#pragma unroll
    for (int r = 0; r < kWaves - 1; ++r)
#pragma unroll
      for (int k = 0; k < K; ++k)
#pragma unroll
        for (int i = 0; i < kCols; ++i) dw[k][i] += s_dw[((r * K + k) * kCols + i) * kWave + lane];
  }
#pragma unroll
  for (int k = 0; k < K; ++k) {
    if (L < kWave && threadIdx.x % kWave >= L) return;
    store_cols<float, WHOLE>(reinterpret_cast<char*>(a.ws + (int64_t)blockIdx.x * a.D), column(k), a.D, dw[k]);
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
  // (no grid has 2^32 threads)
  const uint32_t at = blockIdx.x * 256u + threadIdx.x, line = at / (uint32_t)per;
  const int64_t row = line;
  if (row >= a.N) return;
  const int col = (int)(at - line * (uint32_t)per) * kCols;
  float x[kCols];
  load_cols<T, false>(a.x.p + row * a.x.ld, col, a.D, x);
  drop_cols(a.drop, row, (a.D + 3) / 4, col, x);
  store_cols<T, false>(a.y.p + row * a.y.ld, col, a.D, x);
}

// Blocks of the backward: as many rows of dw are left to add.  32768 x 2048 bf16: 140 us with 256, 512 or 1024, and
// 7, 11 and 26 more for adding them; narrow rows want more wavefronts to have as much in flight.
int64_t bwd_blocks(int64_t N, int32_t D, int rows) {
  const int64_t need = (N + rows - 1) / rows, most = D > 2 * kWave * kCols ? 256 : 512;
  return need < most ? need : most;
}

template <typename T, typename R, int W, int K, int L>
hipError_t fwd(const NormLaunch& p, hipStream_t s) {
  typedef Block<W, L> B;
  const int64_t blocks = (p.N + B::kRows - 1) / B::kRows;
  if (!launchable(blocks, B::kThreads)) return hipErrorNotSupported;
  if (p.D % kCols == 0) k_norm_fwd<T, R, W, K, L, true><<<(unsigned)blocks, B::kThreads, 0, s>>>(p);
  else k_norm_fwd<T, R, W, K, L, false><<<(unsigned)blocks, B::kThreads, 0, s>>>(p);
  return hipGetLastError();
}
template <typename T, typename R, int W, int K, int L>
hipError_t bwd(const NormLaunch& p, hipStream_t s) {
  typedef Block<W, L> B;
  const int64_t blocks = bwd_blocks(p.N, p.D, B::kRows);
  constexpr bool kAhead = kSize<T> == 2 && kSize<R> == 2;
  if (blocks > 0) {
    if (p.D % kCols == 0) k_norm_bwd<T, R, W, K, L, true, kAhead><<<(unsigned)blocks, B::kThreads, 0, s>>>(p);
    else k_norm_bwd<T, R, W, K, L, false, kAhead><<<(unsigned)blocks, B::kThreads, 0, s>>>(p);
  }
  if (p.dweight != nullptr)
    k_norm_dw<<<(unsigned)((p.D + kWave - 1) / kWave), 1024, 0, s>>>(p.ws, (int)blocks, p.D, p.dweight, p.add);
  return hipGetLastError();
}

template <bool BACK, typename T, typename R>
hipError_t by_width(const NormLaunch& p, hipStream_t s) {
  auto go = [&](auto w, auto k, auto l) {
    if constexpr (BACK) return bwd<T, R, decltype(w)::value, decltype(k)::value, decltype(l)::value>(p, s);
    else return fwd<T, R, decltype(w)::value, decltype(k)::value, decltype(l)::value>(p, s);
  };
  using std::integral_constant;
  typedef integral_constant<int, 1> One;
  typedef integral_constant<int, kWave> All;
  if (p.D <= 8 * kCols) return go(One{}, One{}, integral_constant<int, 8>{});
  if (p.D <= 16 * kCols) return go(One{}, One{}, integral_constant<int, 16>{});
  if (p.D <= 32 * kCols) return go(One{}, One{}, integral_constant<int, 32>{});
  constexpr int kOne = kWave * kCols;
  if (p.D <= kOne) return go(One{}, One{}, All{});
  // (forward: more wavefronts with less each, 32768 x 2048 104 us instead of 115; the backward exchanges two
  // sums between them in every row: 140 either way)
  if (p.D <= 2 * kOne) return go(integral_constant<int, BACK ? 1 : 2>{}, integral_constant<int, BACK ? 2 : 1>{}, All{});
  if (p.D <= 4 * kOne) return go(integral_constant<int, BACK ? 1 : 4>{}, integral_constant<int, BACK ? 4 : 1>{}, All{});
  if (p.D <= 8 * kOne) return go(integral_constant<int, 4>{}, integral_constant<int, 2>{}, All{});
  if (p.D <= 16 * kOne) return go(integral_constant<int, 4>{}, integral_constant<int, 4>{}, All{});
  return go(integral_constant<int, 8>{}, integral_constant<int, 4>{}, All{});
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
