// Weight gradient of a projection from its input's 8-bit checkpoint (gfx950):
//
//   dw[k][c] = sum over rows r of x[r][k] * dy[r][c]
//
// on the matrix units, in bf16: a restored x has 7 significant bits and is exact
// in bf16; an fp32 dy is split into three bf16 parts that hold all of its 24
// bits.  Sums are fp32.  Both operands lie with the summed index (the rows)
// slowest, while a matrix instruction wants eight consecutive rows of a column
// in a lane, so a lane loads four columns of eight rows and turns them in
// registers on their way to LDS, where a column's eight rows are 16 bytes.  Few
// tiles of dw: the rows are cut into parts whose sums are added in order.
#include "seq_common.h"

namespace emb {

namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x16 __attribute__((ext_vector_type(16)));

constexpr int kTile = 128;  // columns of x, and of dy, a block's tile has
constexpr int kStep = 64;   // rows a step takes
constexpr int kOct = kStep / 8;
constexpr int kThreads = 256;

struct WArgs {
  const char* x;
  const uint8_t* exps;
  const char* dy;
  float* out;        // dw, or [parts][K][F]
  int64_t ld_x, ld_e, ld_dy;  // bytes
  int32_t N, K, F, steps_per_part, parts, tiles_k, tiles_f, add, aligned;
};

// unsigned halves of two words: lo | hi << 16
__device__ __forceinline__ uint32_t halves_lo(uint32_t a, uint32_t b) { return __builtin_amdgcn_perm(b, a, 0x05040100u); }
__device__ __forceinline__ uint32_t halves_hi(uint32_t a, uint32_t b) { return __builtin_amdgcn_perm(b, a, 0x07060302u); }

template <int SPLIT>  // 1: dy is bf16; 3: fp32 in three parts
__global__ __launch_bounds__(kThreads) void k_weight_grad(WArgs a) {
  __shared__ u32x4 s_x[kOct][kTile], s_y[SPLIT][kOct][kTile];
  const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x / kWave;
  const int tile = blockIdx.x % (a.tiles_k * a.tiles_f), part = blockIdx.x / (a.tiles_k * a.tiles_f);
  const int k0 = tile % a.tiles_k * kTile, c0 = tile / a.tiles_k * kTile;
  // this thread loads columns 4 * (t % 32) .. of rows 8 * (t / 32) .. of a step
  const int quad = threadIdx.x % 32, oct = threadIdx.x / 32;
  const int kx = k0 + 4 * quad, cy = c0 + 4 * quad;
  const bool k_in = kx < a.K;  // (a row of codes is padded to whole groups)
  const int64_t r_begin = (int64_t)part * a.steps_per_part * kStep;
  const int64_t r_end = min((int64_t)a.N, r_begin + (int64_t)a.steps_per_part * kStep);
  f32x16 acc[2][2] = {};
  const int wk = (wave & 1) * 64, wc = (wave >> 1) * 64;
  uint32_t xr[8], er[8], yr[8][SPLIT == 1 ? 2 : 4];
  auto load = [&](int64_t r0) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int64_t r = r0 + 8 * oct + i;
      const bool ok = r < r_end;
      xr[i] = ok && k_in ? *reinterpret_cast<const uint32_t*>(a.x + r * a.ld_x + kx) : 0u;
      er[i] = ok && k_in ? a.exps[r * a.ld_e + kx / EMB_SAVED_GROUP] : 0u;
      const char* q = a.dy + r * a.ld_dy + (int64_t)cy * (SPLIT == 1 ? 2 : 4);
      if constexpr (SPLIT == 1) {
        yr[i][0] = yr[i][1] = 0u;
        if (ok && a.aligned && cy + 4 <= a.F) {
          const u32x2 t = *reinterpret_cast<const u32x2*>(q);
          yr[i][0] = t.x, yr[i][1] = t.y;
        } else if (ok) {
          const uint16_t* h = reinterpret_cast<const uint16_t*>(q);
#pragma unroll
          for (int j = 0; j < 4; ++j)
            if (cy + j < a.F) yr[i][j / 2] |= (uint32_t)h[j] << (16 * (j % 2));
        }
      } else {
#pragma unroll
        for (int j = 0; j < 4; ++j) yr[i][j] = 0u;
        if (ok && a.aligned && cy + 4 <= a.F) {
          const u32x4 t = *reinterpret_cast<const u32x4*>(q);
          yr[i][0] = t.x, yr[i][1] = t.y, yr[i][2] = t.z, yr[i][3] = t.w;
        } else if (ok) {
#pragma unroll
          for (int j = 0; j < 4; ++j)
            if (cy + j < a.F) yr[i][j] = reinterpret_cast<const uint32_t*>(q)[j];
        }
      }
    }
  };
  auto put = [&]() {
    // x: columns j of rows 2i and 2i + 1 to one word each
    uint32_t o[4][4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float u0 = __uint_as_float(er[2 * i] << 23), u1 = __uint_as_float(er[2 * i + 1] << 23);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const float v0 = (float)(int8_t)(xr[2 * i] >> (8 * j)) * u0, v1 = (float)(int8_t)(xr[2 * i + 1] >> (8 * j)) * u1;
        o[j][i] = halves_hi(__float_as_uint(v0), __float_as_uint(v1));
      }
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) s_x[oct][4 * quad + j] = u32x4{o[j][0], o[j][1], o[j][2], o[j][3]};
    if constexpr (SPLIT == 1) {
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i)
          w[i] = j % 2 ? halves_hi(yr[2 * i][j / 2], yr[2 * i + 1][j / 2]) : halves_lo(yr[2 * i][j / 2], yr[2 * i + 1][j / 2]);
        s_y[0][oct][4 * quad + j] = u32x4{w[0], w[1], w[2], w[3]};
      }
    } else {
      // v = p0 + p1 + p2: each part the leading 8 bits of what the parts before it leave (cut off, so every
      // difference is exact); an infinity or NaN is all in p0
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        float v[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = __uint_as_float(yr[i][j]);
#pragma unroll
        for (int p = 0; p < SPLIT; ++p) {
          uint32_t w[4];
#pragma unroll
          for (int i = 0; i < 4; ++i) w[i] = halves_hi(__float_as_uint(v[2 * i]), __float_as_uint(v[2 * i + 1]));
          s_y[p][oct][4 * quad + j] = u32x4{w[0], w[1], w[2], w[3]};
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            const uint32_t u = __float_as_uint(v[i]);
            v[i] = (u & 0x7f800000u) == 0x7f800000u ? 0.f : v[i] - __uint_as_float(u & 0xffff0000u);
          }
        }
      }
    }
  };
  if (r_begin < r_end) load(r_begin);
  for (int64_t r0 = r_begin; r0 < r_end; r0 += kStep) {
    __syncthreads();
    put();
    __syncthreads();
    if (r0 + kStep < r_end) load(r0 + kStep);
    // 16 rows an instruction: lane l holds column l % 32, rows 8 * (l / 32) .. of the 16
#pragma unroll
    for (int g = 0; g < kOct / 2; ++g) {
      const int o = 2 * g + lane / 32, c = lane % 32;
      bf16x8 fx[2], fy[2];
#pragma unroll
      for (int i = 0; i < 2; ++i) fx[i] = __builtin_bit_cast(bf16x8, s_x[o][wk + 32 * i + c]);
#pragma unroll
      for (int p = 0; p < SPLIT; ++p) {
#pragma unroll
        for (int i = 0; i < 2; ++i) fy[i] = __builtin_bit_cast(bf16x8, s_y[p][o][wc + 32 * i + c]);
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
          for (int j = 0; j < 2; ++j)
            acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fx[i], fy[j], acc[i][j], 0, 0, 0);
      }
    }
  }
  float* out = a.out + (a.parts > 1 ? (int64_t)part * a.K * a.F : 0);
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
      for (int v = 0; v < 16; ++v) {
        const int k = k0 + wk + 32 * i + 8 * (v / 4) + 4 * (lane / 32) + v % 4, c = c0 + wc + 32 * j + lane % 32;
        if (k >= a.K || c >= a.F) continue;
        float* d = out + (int64_t)k * a.F + c;
        *d = a.parts == 1 && a.add ? *d + acc[i][j][v] : acc[i][j][v];
      }
}

__global__ __launch_bounds__(256) void k_weight_parts(const float* parts, float* dw, int64_t n, int count, int add) {
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (int64_t)gridDim.x * 256) {
    float t = 0.f;
    for (int p = 0; p < count; ++p) t += parts[(int64_t)p * n + i];
    dw[i] = add ? dw[i] + t : t;
  }
}

// Parts the rows are cut into: as many as give each compute unit a block or
// two, of at least four steps each.
int part_count(int64_t N, int32_t K, int32_t F) {
  const int64_t tiles = (int64_t)((K + kTile - 1) / kTile) * ((F + kTile - 1) / kTile);
  const int64_t steps = (N + kStep - 1) / kStep;
  int64_t p = 512 / tiles;
  if (p > steps / 4) p = steps / 4;
  return (int)(p < 1 ? 1 : p);
}

}  // namespace

size_t weight_grad_ws_bytes(int64_t N, int32_t K, int32_t F) {
  const int p = part_count(N, K, F);
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
  a.aligned = p.aligned;
  a.parts = part_count(p.N, p.K, p.F);
  const int64_t steps = (p.N + kStep - 1) / kStep;
  a.steps_per_part = (int32_t)((steps + a.parts - 1) / a.parts);
  a.tiles_k = (p.K + kTile - 1) / kTile;
  a.tiles_f = (p.F + kTile - 1) / kTile;
  a.out = a.parts > 1 ? p.ws : p.dw;
  const unsigned blocks = (unsigned)(a.tiles_k * a.tiles_f * a.parts);
  if (p.dtype == EMB_BF16) k_weight_grad<1><<<blocks, kThreads, 0, s>>>(a);
  else k_weight_grad<3><<<blocks, kThreads, 0, s>>>(a);
  if (a.parts > 1) {
    const int64_t n = (int64_t)p.K * p.F;
    k_weight_parts<<<(unsigned)((n + 255) / 256 < 4096 ? (n + 255) / 256 : 4096), 256, 0, s>>>(p.ws, p.dw, n, a.parts,
                                                                                               p.add);
  }
  return hipGetLastError();
}

}  // namespace emb
