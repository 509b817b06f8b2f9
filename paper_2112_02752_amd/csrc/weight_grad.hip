// Weight gradient of a projection from its input's 8-bit checkpoint (gfx950):
//
//   dw[k][c] = sum over rows r of x[r][k] * dy[r][c]
//
// on the matrix units, in bf16: a restored x has 7 significant bits and is exact
// in bf16; an fp32 dy is split into three bf16 parts that hold all of its 24
// bits.  Sums are fp32.
//
// Both operands lie with the summed index (the rows) slowest, while a matrix
// instruction wants eight consecutive rows of a column in a lane.  So a lane
// loads four columns of eight rows and turns them in registers (two permutes
// for two columns of two rows; codes become bf16 on the way) into LDS, where a
// column's eight rows are 16 bytes.  Columns 4 q + j of a group of 128 lie by j,
// then q: lanes write and read consecutive 16 bytes, and the instruction of
// slice j gives a lane column 4 q + j, so the four slices of a lane are four
// consecutive columns of dw.
//
// Few tiles of dw: the rows are cut into parts whose sums are added in order.
//
// Bound: 2 N K F operations on the matrix units.  32768 x 2048 x 6144 (bf16 dy):
// 808 us, 1020 TFLOP/s, of 1216 that a library product of 8192^3 reaches; adding
// its four parts is 39 us of it.  2048 x 512 x 1536: 17.7 us, of which the products
// take 14 (what is read and the parts are 44 MB; small tiles with four wavefronts a
// block 15.5) and the parts' sums 4.  An fp32 dy makes three products of one and has
// one LDS buffer: 3160 us there, of 2035 at the library's rate.  Times that compare
// two ways below are of repeated calls on one set of inputs.
#include "seq_common.h"
#include "weight_plan.h"

namespace emb {

namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x16 __attribute__((ext_vector_type(16)));

constexpr int kOct = kStep / 8;
constexpr int kBand = 8;  // tiles

struct WArgs {
  const char* x;
  const uint8_t* exps;
  const char* dy;
  float* out;        // dw, or [parts][K][F]
  int64_t ld_x, ld_e, ld_dy;  // bytes
  int32_t N, K, F, steps_per_part, parts, tiles_k, tiles_f, add;
};

// unsigned halves of two words: lo | hi << 16
__device__ __forceinline__ uint32_t halves_lo(uint32_t a, uint32_t b) { return __builtin_amdgcn_perm(b, a, 0x05040100u); }
__device__ __forceinline__ uint32_t halves_hi(uint32_t a, uint32_t b) { return __builtin_amdgcn_perm(b, a, 0x07060302u); }

// The rows of a step from p on, `left` of them in the matrix, ld bytes apart,
// `row` bytes of a row readable: what lies beyond reads as zero, so neither the
// last rows nor the last tile's columns need a branch (columns beyond the
// matrix only reach sums that are not stored).
__device__ __forceinline__ __amdgpu_buffer_rsrc_t rows_at(const char* p, int left, int ld, int row) {
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(p), 0, rows_bytes(left, ld, row), 0x00020000);
}
__device__ __forceinline__ int rows_left(const WArgs& a, int64_t r0) {
  return step_rows(a.N, r0);
}

// One group of 128 columns of x: four columns of eight rows a lane.
struct XLoad {
  uint32_t w[8], e[8];
  __device__ __forceinline__ void load(const WArgs& a, int64_t r0, int k0, int quad, int oct) {
    // (a row of codes is whole groups)
    const int left = rows_left(a, r0), groups = groups_left(a.K, k0);
    const auto rx = rows_at(a.x + r0 * a.ld_x + k0, left, (int)a.ld_x, groups * EMB_SAVED_GROUP);
    const auto re = rows_at(reinterpret_cast<const char*>(a.exps) + r0 * a.ld_e + k0 / EMB_SAVED_GROUP, left, (int)a.ld_e,
                            groups);
    const int at = 8 * oct * (int)a.ld_x + 4 * quad, ae = 8 * oct * (int)a.ld_e + 4 * quad / EMB_SAVED_GROUP;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      w[i] = __builtin_amdgcn_raw_buffer_load_b32(rx, at + i * (int)a.ld_x, 0, 0);
      e[i] = __builtin_amdgcn_raw_buffer_load_b8(re, ae + i * (int)a.ld_e, 0, 0);
    }
  }
  __device__ __forceinline__ void put(u32x4* lds, int quad) const {
    uint32_t o[4][4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      // (exponent 255: the codes are zeros, and zero times infinity is NaN)
      const float u0 = __uint_as_float((e[2 * i] & 0xffu) << 23), u1 = __uint_as_float((e[2 * i + 1] & 0xffu) << 23);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const float v0 = (float)(int8_t)(w[2 * i] >> (8 * j)) * u0, v1 = (float)(int8_t)(w[2 * i + 1] >> (8 * j)) * u1;
        o[j][i] = halves_hi(__float_as_uint(v0), __float_as_uint(v1));
      }
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) lds[32 * j + quad] = u32x4{o[j][0], o[j][1], o[j][2], o[j][3]};
  }
};

// One group of 128 columns of dy.  SPLIT 1: bf16; 3: fp32 in three parts, whose
// groups lie `apart` 16-byte words from one another.
template <int SPLIT, bool PAIRS>
struct YLoad {
  static constexpr int kWords = SPLIT == 1 ? 2 : 4;
  uint32_t w[8][kWords];
  __device__ __forceinline__ void load(const WArgs& a, int64_t r0, int c0, int quad, int oct) {
    constexpr int kSize = SPLIT == 1 ? 2 : 4;
    const auto ry = rows_at(a.dy + r0 * a.ld_dy + (int64_t)c0 * kSize, rows_left(a, r0), (int)a.ld_dy,
                            dy_row_bytes(a.F, c0, kSize, PAIRS));
    const int at = 8 * oct * (int)a.ld_dy + 4 * kSize * quad;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int row = at + i * (int)a.ld_dy;
      if constexpr (SPLIT == 3) {
        const u32x4 t = __builtin_amdgcn_raw_buffer_load_b128(ry, row, 0, 0);
        w[i][0] = t.x, w[i][1] = t.y, w[i][2] = t.z, w[i][3] = t.w;
      } else if constexpr (PAIRS) {
        const u32x2 t = __builtin_amdgcn_raw_buffer_load_b64(ry, row, 0, 0);
        w[i][0] = t.x, w[i][1] = t.y;
      } else {
        // rows or values that are not aligned to words
#pragma unroll
        for (int j = 0; j < 2; ++j)
          w[i][j] = (uint32_t)(uint16_t)__builtin_amdgcn_raw_buffer_load_b16(ry, row + 4 * j, 0, 0) |
                    (uint32_t)(uint16_t)__builtin_amdgcn_raw_buffer_load_b16(ry, row + 4 * j + 2, 0, 0) << 16;
      }
    }
  }
  __device__ __forceinline__ void put(u32x4* lds, int apart, int quad) const {
    if constexpr (SPLIT == 1) {
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        uint32_t o[4];
#pragma unroll
        for (int i = 0; i < 4; ++i)
          o[i] = j % 2 ? halves_hi(w[2 * i][j / 2], w[2 * i + 1][j / 2]) : halves_lo(w[2 * i][j / 2], w[2 * i + 1][j / 2]);
        lds[32 * j + quad] = u32x4{o[0], o[1], o[2], o[3]};
      }
    } else {
      // v = p0 + p1 + p2: each part the leading 8 bits of what the parts before it leave (cut off, so every
      // difference is exact); an infinity or NaN is all in p0 (a signalling NaN, whose bits may all be among those cut
      // off, as the quiet one)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        float v[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = __builtin_canonicalizef(__uint_as_float(w[i][j]));
#pragma unroll
        for (int p = 0; p < SPLIT; ++p) {
          uint32_t o[4];
#pragma unroll
          for (int i = 0; i < 4; ++i) o[i] = halves_hi(__float_as_uint(v[2 * i]), __float_as_uint(v[2 * i + 1]));
          lds[p * apart + 32 * j + quad] = u32x4{o[0], o[1], o[2], o[3]};
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            const uint32_t u = __float_as_uint(v[i]);
            v[i] = (u & 0x7f800000u) == 0x7f800000u ? 0.f : v[i] - __uint_as_float(u & 0xffff0000u);
          }
        }
      }
    }
  }
};

// G groups of 128 columns each way a block.  G 2: four wavefronts as 2 x 2, each
// a group by a group (4 x 4 slices), every thread bringing in x and dy.  G 1: eight
// as 4 x 2, each 1 x 2 slices, four bringing in x and four dy (few steps a block:
// two wavefronts a SIMD, of which one converts while the other multiplies).
template <int G>
struct Shape;
template <>
struct Shape<2> {
  static constexpr int kThreads = 256, kSx = 4, kSy = 4, kWavesK = 2;
};
template <>
struct Shape<1> {
  static constexpr int kThreads = 512, kSx = 1, kSy = 2, kWavesK = 4;
};

template <int G, int SPLIT, bool PAIRS>
__global__ __launch_bounds__(Shape<G>::kThreads, G == 2 ? 1 : PAIRS ? 4 : 2) void k_weight_grad(WArgs a) {
  constexpr int SX = Shape<G>::kSx, SY = Shape<G>::kSy, kTile = kGroup * G, kBufs = SPLIT == 1 ? 2 : 1;
  constexpr int kApart = kOct * G * kGroup;
  __shared__ u32x4 s_x[kBufs][kOct][G * kGroup], s_y[kBufs][SPLIT][kOct][G * kGroup];
  const int lane = threadIdx.x & (kWave - 1), wave = uniform(threadIdx.x / kWave);
  const int tiles = a.tiles_k * a.tiles_f;
  int at = (int)blockIdx.x;
  if constexpr (G == 2) {
    // Blocks go to the eight XCDs in turn: an XCD takes neighbouring tiles, which read the same columns
    // (32768 x 2048 x 6144 811 us, 846 with every XCD reading all of dy;
    // small tiles gain nothing, and 2048 x 512 x 1536 takes 21.4 us instead of 18.6)
    const int each = (int)gridDim.x / 8;
    if (at < 8 * each) at = at % 8 * each + at / 8;
  }
  const int tile = at % tiles, part = at / tiles;
  // (tiles in bands of eight down the columns of x: 32 neighbours read some eight column groups of x and four of dy)
  const int band = tile / (kBand * a.tiles_f), in_band = tile - band * kBand * a.tiles_f;
  const int high = min(kBand, a.tiles_k - band * kBand);
  const int k0 = (band * kBand + in_band % high) * kTile, c0 = in_band / high * kTile;
  const int quad = threadIdx.x % 32, oct = threadIdx.x / 32 % kOct;
  const bool takes_x = G == 2 || wave < 4, takes_y = G == 2 || wave >= 4;
  const int64_t r_begin = (int64_t)part * a.steps_per_part * kStep;
  const int64_t r_end = min((int64_t)a.N, r_begin + (int64_t)a.steps_per_part * kStep);
  f32x16 acc[SX][SY] = {};
  const int wk = wave % Shape<G>::kWavesK * 32 * SX, wc = wave / Shape<G>::kWavesK * 32 * SY;
  XLoad x[G];
  YLoad<SPLIT, PAIRS> y[G];
  auto load = [&](int64_t r0) {
#pragma unroll
    for (int g = 0; g < G; ++g) {
      if (takes_x) x[g].load(a, r0, k0 + g * kGroup, quad, oct);
      if (takes_y) y[g].load(a, r0, c0 + g * kGroup, quad, oct);
    }
  };
  auto put = [&](int buf) {
#pragma unroll
    for (int g = 0; g < G; ++g) {
      if (takes_x) x[g].put(&s_x[buf][oct][g * kGroup], quad);
      if (takes_y) y[g].put(&s_y[buf][0][oct][g * kGroup], kApart, quad);
    }
  };
  // a quarter of a step: 16 rows, of which lane l holds 8 * (l / 32) ..
  bf16x8 fx[2][SX], fy[2][SY];
  auto fetch = [&](int buf, int n, int p, int to) {
    const int o = 2 * n + lane / 32, c = lane % 32;
    if (p == 0) {
#pragma unroll
      for (int i = 0; i < SX; ++i) fx[to][i] = __builtin_bit_cast(bf16x8, s_x[buf][o][wk + 32 * i + c]);
    }
#pragma unroll
    for (int i = 0; i < SY; ++i) fy[to][i] = __builtin_bit_cast(bf16x8, s_y[buf][p][o][wc + 32 * i + c]);
  };
  auto sum = [&](int xs, int ys) {
#pragma unroll
    for (int i = 0; i < SX; ++i)
#pragma unroll
      for (int j = 0; j < SY; ++j)
        acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fx[xs][i], fy[ys][j], acc[i][j], 0, 0, 0);
  };
  if (r_begin < r_end) {
    load(r_begin);
    if constexpr (kBufs == 1) {
      for (int64_t r0 = r_begin; r0 < r_end; r0 += kStep) {
        __syncthreads();
        put(0);
        __syncthreads();
        if (r0 + kStep < r_end) load(r0 + kStep);
#pragma unroll
        for (int n = 0; n < 4; ++n) {
#pragma unroll
          for (int p = 0; p < SPLIT; ++p) {
            fetch(0, n, p, 0);
            sum(0, 0);
          }
        }
      }
    } else {
      // two buffers: a step's values go to LDS while the step before them is summed, and are loaded a step earlier
      put(0);
      load(r_begin + kStep);  // (rows past the end read as zeros)
      __syncthreads();
      int buf = 0;
      for (int64_t r0 = r_begin; r0 < r_end; r0 += kStep) {
        fetch(buf, 0, 0, 0);
        if constexpr (G == 1) {
#pragma unroll
          for (int n = 0; n < 4; ++n) {
            if (n < 3) fetch(buf, n + 1, 0, (n + 1) & 1);
            sum(n & 1, n & 1);
            if (n == 1) {
              put(buf ^ 1);
              load(r0 + 2 * kStep);
            }
          }
        } else {
#pragma unroll
          for (int n = 0; n < 4; ++n) {
            if (n < 3) fetch(buf, n + 1, 0, (n + 1) & 1);
            sum(n & 1, n & 1);
            const int g = n / 2;
            if (n % 2 == 0) {
              x[g].put(&s_x[buf ^ 1][oct][g * kGroup], quad);
              x[g].load(a, r0 + 2 * kStep, k0 + g * kGroup, quad, oct);
            } else {
              y[g].put(&s_y[buf ^ 1][0][oct][g * kGroup], kApart, quad);
              y[g].load(a, r0 + 2 * kStep, c0 + g * kGroup, quad, oct);
            }
            // the matrix unit takes 32 cycles an instruction: what else there is to do goes between
            __builtin_amdgcn_sched_group_barrier(0x100, 8, 0);  // LDS reads
#pragma unroll
            for (int i = 0; i < 16; ++i) {
              __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);  // one product
              __builtin_amdgcn_sched_group_barrier(0x002, 6, 0);  // vector instructions
              if (i % 3 == 2) __builtin_amdgcn_sched_group_barrier(0x200, 1, 0);  // an LDS write
              __builtin_amdgcn_sched_group_barrier(0x020, 1, 0);  // a load
            }
            __builtin_amdgcn_sched_barrier(0);
          }
        }
        __syncthreads();
        buf ^= 1;
      }
    }
  }
  // slice i of a group holds columns 4 q + i: a wavefront's slices begin at slice (wk / 32) % 4 of group wk / 128
  float* out = a.out + (a.parts > 1 ? (int64_t)part * a.K * a.F : 0);
  const int kb = k0 + wk / kGroup * kGroup + wk / 32 % 4, cb = c0 + wc / kGroup * kGroup + wc / 32 % 4 + 4 * (lane % 32);
  const bool add = a.parts == 1 && a.add;
#pragma unroll
  for (int v = 0; v < 16; ++v) {
    const int q = 8 * (v / 4) + 4 * (lane / 32) + v % 4;
#pragma unroll
    for (int i = 0; i < SX; ++i) {
      const int k = kb + 4 * q + i;
      if (k >= a.K) continue;
      float* d = out + (int64_t)k * a.F + cb;
      float t[SY];
#pragma unroll
      for (int j = 0; j < SY; ++j) t[j] = acc[i][j][v];
      if (!add && cb + SY <= a.F && a.F % SY == 0) {
        Vec<float, SY>::store(d, t);
      } else {
#pragma unroll
        for (int j = 0; j < SY; ++j)
          if (cb + j < a.F) d[j] = add ? d[j] + t[j] : t[j];
      }
    }
  }
}

// The parts' sums, in order; four values a lane where the rows of dw allow it.
// Bound by latency: eight parts' values are in flight together.
template <int V>
__global__ __launch_bounds__(256) void k_weight_parts(const float* parts, float* dw, int64_t n, int count, int add) {
  for (int64_t i = ((int64_t)blockIdx.x * 256 + threadIdx.x) * V; i < n; i += (int64_t)gridDim.x * 256 * V) {
    float t[V] = {};
    constexpr int kAhead = 8;
    for (int p = 0; p < count; p += kAhead) {
      Vec<float, V> x[kAhead];
#pragma unroll
      for (int k = 0; k < kAhead; ++k) {
        if (p + k < count) x[k].load(parts + (int64_t)(p + k) * n + i);
        else x[k].zero();
      }
#pragma unroll
      for (int k = 0; k < kAhead; ++k)
#pragma unroll
        for (int v = 0; v < V; ++v) t[v] += x[k].get(v);
    }
    if (add) {
      Vec<float, V> old;
      old.load(dw + i);
#pragma unroll
      for (int v = 0; v < V; ++v) t[v] += old.get(v);
    }
    Vec<float, V>::store(dw + i, t);
  }
}

}  // namespace

size_t weight_grad_ws_bytes(int64_t N, int32_t K, int32_t F) {
  const int a = plan_for(N, K, F, false).parts, b = plan_for(N, K, F, true).parts, p = a > b ? a : b;
  return p > 1 ? align256(sizeof(float) * (size_t)p * (size_t)K * (size_t)F) : 0;
}

hipError_t launch_weight_grad(const WeightGradLaunch& p, hipStream_t s) {
  WArgs a{};
  a.x = p.x.p;
  a.exps = p.x.exps;
  a.dy = p.dy.p;
  a.ld_x = p.x.ld;
  a.ld_e = p.x.ld_exps;
  a.ld_dy = p.dy.ld;
  a.N = (int32_t)p.N;
  a.K = p.K;
  a.F = p.F;
  a.add = p.add;
  const Plan pl = plan_for(p.N, p.K, p.F, p.dtype == EMB_FP32 || !p.aligned);
  const int tile = pl.groups * kGroup;
  a.parts = pl.parts;
  a.steps_per_part = pl.steps;
  const int64_t tiles_k = ((int64_t)p.K + tile - 1) / tile, tiles_f = ((int64_t)p.F + tile - 1) / tile;
  const int64_t all = tiles_k * tiles_f * pl.parts;
  if (!launchable(all, Shape<1>::kThreads)) return hipErrorNotSupported;
  a.tiles_k = (int32_t)tiles_k;
  a.tiles_f = (int32_t)tiles_f;
  a.out = a.parts > 1 ? p.ws : p.dw;
  const unsigned blocks = (unsigned)all;
  if (p.dtype == EMB_FP32) k_weight_grad<1, 3, true><<<blocks, Shape<1>::kThreads, 0, s>>>(a);
  else if (!p.aligned) k_weight_grad<1, 1, false><<<blocks, Shape<1>::kThreads, 0, s>>>(a);
  else if (pl.groups == 2) k_weight_grad<2, 1, true><<<blocks, Shape<2>::kThreads, 0, s>>>(a);
  else k_weight_grad<1, 1, true><<<blocks, Shape<1>::kThreads, 0, s>>>(a);
  if (a.parts > 1) {
    const int64_t n = (int64_t)p.K * p.F;
    const bool four = n % 4 == 0 && (reinterpret_cast<uintptr_t>(p.dw) & 15u) == 0;
    const int64_t want = (four ? n / 4 + 255 : n + 255) / 256;
    const unsigned grid = (unsigned)(want < 8192 ? want : 8192);
    if (four) k_weight_parts<4><<<grid, 256, 0, s>>>(p.ws, p.dw, n, a.parts, p.add);
    else k_weight_parts<1><<<grid, 256, 0, s>>>(p.ws, p.dw, n, a.parts, p.add);
  }
  return hipGetLastError();
}

}  // namespace emb
