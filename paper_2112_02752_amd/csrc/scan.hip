// Gated linear recurrence over ragged sequences (gfx950), one state a column:
//
//   a_t = sigmoid(f_t + bias),  h_t = a_t h_{t-1} + (1 - a_t) x_t,  y_t = sigmoid(o_t) h_t
//
// Steps h -> a h + b compose: (A1, B1) then (A2, B2) is (A1 A2, A2 B1 + B2), so
// the positions are cut into spans of 64, whatever sequences they belong to (a
// sequence's first position discards what came before it).  A block takes one
// span of 64 or 128 columns: each wavefront holds a part of the span's
// positions in registers, a lane one or two columns, and the parts are joined
// through LDS.  With more than one span:
//   k_scan_sums   each span's (A, B) from zero
//   k_scan_carry  the state before each span (16 wavefronts share the spans of
//                 64 columns)
//   k_scan_fwd    the span again, from its state
// The backward is the same scan from the last position to the first on
// dh_t = sigmoid(o_t) dy_t + a_{t+1} dh_{t+1}, with h recomputed inside each
// span from the state the forward kept.
//
// A span that holds a first position passes nothing on of what it receives:
// its A is kResets, not a product with zero, which would carry an infinity or
// NaN of one sequence into the next.
#include "seq_common.h"

namespace emb {

namespace {

constexpr float kResets = -1.0f;  // (products of a's are never negative)
constexpr int kP = 16;            // positions a wavefront holds
constexpr int kW = kSpan / kP;    // wavefronts of a block
constexpr int kThreads = kW * kWave;

struct Saved8 {};

// V columns of a matrix as they lie in memory
template <typename T, int V>
struct In {
  Vec<T, V> v;
  __device__ __forceinline__ void load(const Rows& m, int64_t row, int col) {
    v.load(m.p + row * m.ld + (int64_t)col * (Vec<T, V>::kBytes / V));
  }
  __device__ __forceinline__ float get(int i) const { return v.get(i); }
};
template <int V>
struct In<Saved8, V> {
  uint32_t codes, e;
  __device__ __forceinline__ void load(const Rows& m, int64_t row, int col) {
    const char* p = m.p + row * m.ld + col;
    if constexpr (V == 1) codes = *reinterpret_cast<const uint8_t*>(p);
    else codes = *reinterpret_cast<const uint16_t*>(p);
    e = m.exps[row * m.ld_exps + col / EMB_SAVED_GROUP];
  }
  // (exponent 255: the codes are zeros, and zero times infinity is NaN)
  __device__ __forceinline__ float get(int i) const {
    return (float)(int8_t)(codes >> (8 * i)) * __uint_as_float(e << 23);
  }
};

// sigmoid(z) and sigmoid(-z), the latter without cancellation; NaN stays NaN
__device__ __forceinline__ void forget(float z, float& a, float& q) {
  float t = -1.44269504f * z;
  t = t > 126.f ? 126.f : t;
  const float e = __builtin_amdgcn_exp2f(t);
  a = __builtin_amdgcn_rcpf(1.f + e);
  q = e * a;
}
__device__ __forceinline__ float gate(float z) {
  return __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(-1.44269504f * z));
}

// (A, B) applied to a state
__device__ __forceinline__ float through(float A, float B, float h) {
  return A < 0.f ? B : __builtin_fmaf(A, h, B);
}

struct Scan {
  const int32_t* offsets;
  Rows x, f, o, y, dy, dx, df, dO;
  const float *bias, *h0, *states, *dh_last;
  float *h_last, *dh0, *dbias;  // dbias: [spans][D], one row a span
  float *A, *B;                 // [spans][D]
  float* carry;                 // [spans][D]: what enters each span
  int32_t N, M, D, spans, slices;
};

// First and last positions of sequences among a wavefront's kP positions from
// q0 on, and the sequence of each.
struct Marks {
  uint32_t starts;  // bit t: position q0 + t is its sequence's first
  uint32_t ends;    // bit t: position q0 + t is its sequence's last
  int seq;          // lane t: the sequence of position q0 + t
  __device__ __forceinline__ Marks(const Scan& a, int q0, int lane) {
    const int m = min(max(wave_upper_bound<int32_t>(a.offsets, a.M + 1, q0, lane) - 1, 0), a.M - 1);
    // the next 64 offsets, one a lane; more only where sequences of no positions fill them
    int v = a.offsets[min(m + 1 + lane, a.M)], at = m + 1;
    uint32_t s = uniform(a.offsets[m]) == q0 ? 1u : 0u;
    seq = m;
    for (;;) {
#pragma unroll
      for (int t = 0; t <= kP; ++t) {
        const uint64_t upto = __ballot(v <= q0 + t && at + lane < a.M);
        seq += lane == t ? __popcll(upto) : 0;
        if (t > 0) s |= __ballot(v == q0 + t) ? 1u << t : 0u;
      }
      if (at + kWave > a.M || lane_at(v, kWave - 1) > q0 + kP) break;
      at += kWave;
      v = a.offsets[min(at + lane, a.M)];
    }
    starts = s & ((1u << kP) - 1u);
    ends = s >> 1;
    if (a.N - q0 <= kP) ends |= 1u << (a.N - q0 - 1);
  }
  __device__ __forceinline__ bool start(int t) const { return (starts >> t) & 1u; }
  __device__ __forceinline__ bool end(int t) const { return (ends >> t) & 1u; }
  __device__ __forceinline__ int of(int t) const { return lane_at(seq, t); }
};

template <int V>
__device__ __forceinline__ void load_f32(const float* p, int col, float (&v)[V]) {
#pragma unroll
  for (int i = 0; i < V; ++i) v[i] = p ? p[col + i] : 0.f;
}

// ---------------------------------------------------------------- forward

// FULL: from the span's state, with outputs; else the span's sums alone
template <typename T, int V, bool GATED, bool FULL>
__global__ __launch_bounds__(kThreads) void k_scan_fwd(Scan a) {
  const int lane = threadIdx.x & (kWave - 1), wave = uniform(threadIdx.x / kWave);
  const int main_blocks = a.spans * a.slices;
  if (FULL && (int)blockIdx.x >= main_blocks) {
    // sequences of no positions keep their first state
    const int m0 = ((int)blockIdx.x - main_blocks) * kWave;
    for (int m = m0 + wave; m < min(a.M, m0 + kWave); m += kW) {
      if (a.offsets[m] != a.offsets[m + 1]) continue;
      for (int d = lane; d < a.D; d += kWave)
        a.h_last[(int64_t)m * a.D + d] = a.h0 ? a.h0[(int64_t)m * a.D + d] : 0.f;
    }
    return;
  }
  const int c = blockIdx.x / a.slices, col0 = ((int)blockIdx.x % a.slices * kWave + lane) * V;
  const bool in = col0 < a.D;
  const int col = in ? col0 : 0;
  const int q0 = c * kSpan + wave * kP;
  const int n = min(kP, a.N - q0);  // (0 or less: this wavefront has no positions)
  __shared__ float s_A[kW][V * kWave], s_B[kW][V * kWave];
  float A[V], B[V], fa[kP][V], fb[kP][V];
  In<T, V> go[GATED ? kP : 1];
#pragma unroll
  for (int i = 0; i < V; ++i) A[i] = 1.f, B[i] = 0.f;
  Marks mk(a, min(q0, a.N - 1), lane);
  if (n > 0) {
    In<T, V> gx[kP], gf[kP];
#pragma unroll
    for (int t = 0; t < kP; ++t) {
      const int64_t row = min(q0 + t, a.N - 1);
      gx[t].load(a.x, row, col);
      gf[t].load(a.f, row, col);
      if constexpr (FULL && GATED) go[t].load(a.o, row, col);
    }
    float bias[V];
    load_f32<V>(a.bias, col, bias);
#pragma unroll
    for (int t = 0; t < kP; ++t) {
#pragma unroll
      for (int i = 0; i < V; ++i) {
        float q;
        forget(gf[t].get(i) + bias[i], fa[t][i], q);
        fb[t][i] = q * gx[t].get(i);
      }
    }
#pragma unroll
    for (int t = 0; t < kP; ++t) {
      if (t >= n) continue;
      if (mk.start(t)) {
        float h0[V] = {};
        if (a.h0) load_f32<V>(a.h0 + (int64_t)mk.of(t) * a.D, col, h0);
#pragma unroll
        for (int i = 0; i < V; ++i) B[i] = h0[i];
      }
#pragma unroll
      for (int i = 0; i < V; ++i) {
        A[i] *= fa[t][i];
        B[i] = __builtin_fmaf(fa[t][i], B[i], fb[t][i]);
      }
    }
    if (mk.starts) {
#pragma unroll
      for (int i = 0; i < V; ++i) A[i] = kResets;
    }
  }
#pragma unroll
  for (int i = 0; i < V; ++i) {
    s_A[wave][i * kWave + lane] = A[i];
    s_B[wave][i * kWave + lane] = B[i];
  }
  __syncthreads();
  if constexpr (!FULL) {
    if (wave != 0) return;
#pragma unroll
    for (int i = 0; i < V; ++i) {
#pragma unroll
      for (int w = 1; w < kW; ++w) {
        const float A2 = s_A[w][i * kWave + lane], B2 = s_B[w][i * kWave + lane];
        B[i] = through(A2, B2, B[i]);
        A[i] = A2 < 0.f || A[i] < 0.f ? kResets : A[i] * A2;
      }
      if (in) {
        a.A[(int64_t)c * a.D + col + i] = A[i];
        a.B[(int64_t)c * a.D + col + i] = B[i];
      }
    }
  } else {
    if (n <= 0) return;
    float h[V];
    load_f32<V>(c > 0 ? a.carry + (int64_t)c * a.D : nullptr, col, h);
    for (int w = 0; w < wave; ++w) {
#pragma unroll
      for (int i = 0; i < V; ++i) h[i] = through(s_A[w][i * kWave + lane], s_B[w][i * kWave + lane], h[i]);
    }
#pragma unroll
    for (int t = 0; t < kP; ++t) {
      if (t >= n) continue;
      if (mk.start(t)) {
        float h0[V] = {};
        if (a.h0) load_f32<V>(a.h0 + (int64_t)mk.of(t) * a.D, col, h0);
#pragma unroll
        for (int i = 0; i < V; ++i) h[i] = h0[i];
      }
      float y[V];
#pragma unroll
      for (int i = 0; i < V; ++i) {
        h[i] = __builtin_fmaf(fa[t][i], h[i], fb[t][i]);
        y[i] = GATED ? gate(go[t].get(i)) * h[i] : h[i];
      }
      if (in) Vec<T, V>::store(a.y.p + (int64_t)(q0 + t) * a.y.ld + (int64_t)col * (Vec<T, V>::kBytes / V), y);
      if (a.h_last && mk.end(t)) {
        float* dst = a.h_last + (int64_t)mk.of(t) * a.D + col;
        if (in) {
#pragma unroll
          for (int i = 0; i < V; ++i) dst[i] = h[i];
        }
      }
    }
  }
}

// What enters each span, from the spans' sums: carry[c] = through(A, B of c - 1,
// carry[c - 1]), or from the last span to the first.  A lane has one column;
// 16 wavefronts share the spans: each joins its part, the parts are joined
// through LDS, each goes over its part again.
constexpr int kCarryWaves = 16;
template <bool BACK>
__global__ __launch_bounds__(kCarryWaves * kWave) void k_scan_carry(const float* A, const float* B, float* carry,
                                                                    int spans, int D) {
  const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x / kWave;
  const int col0 = blockIdx.x * kWave + lane;
  const bool in = col0 < D;
  const int64_t col = in ? col0 : 0;
  __shared__ float s_A[kCarryWaves][kWave], s_B[kCarryWaves][kWave];
  const int per = (spans + kCarryWaves - 1) / kCarryWaves;
  const int first = wave * per, last = min(spans, first + per);
  constexpr int kAhead = 8;
  auto place = [&](int k) { return (int64_t)(BACK ? spans - 1 - k : k) * D + col; };
  float a1 = 1.f, b1 = 0.f;
  for (int k = first; k < last; k += kAhead) {
    float x[kAhead], y[kAhead];
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
      const int64_t at = place(min(k + i, last - 1));
      x[i] = A[at], y[i] = B[at];
    }
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
      if (k + i >= last) break;
      b1 = through(x[i], y[i], b1);
      a1 = x[i] < 0.f || a1 < 0.f ? kResets : a1 * x[i];
    }
  }
  s_A[wave][lane] = a1;
  s_B[wave][lane] = b1;
  __syncthreads();
  float h = 0.f;
  for (int w = 0; w < wave; ++w) h = through(s_A[w][lane], s_B[w][lane], h);
  for (int k = first; k < last; k += kAhead) {
    float x[kAhead], y[kAhead];
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
      const int64_t at = place(min(k + i, last - 1));
      x[i] = A[at], y[i] = B[at];
    }
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
      if (k + i >= last) break;
      if (in) carry[place(k + i)] = h;
      h = through(x[i], y[i], h);
    }
  }
}

// ---------------------------------------------------------------- backward

// The span's sums from its last position to its first: what position p0 - 1
// receives, a_p0 dh_p0, as (A, B) of what position p1 - 1 receives.
template <typename T, typename TG, int V, bool GATED>
__global__ __launch_bounds__(kThreads) void k_scan_back_sums(Scan a) {
  const int lane = threadIdx.x & (kWave - 1), wave = uniform(threadIdx.x / kWave);
  const int c = blockIdx.x / a.slices, col0 = ((int)blockIdx.x % a.slices * kWave + lane) * V;
  const bool in = col0 < a.D;
  const int col = in ? col0 : 0;
  const int q0 = c * kSpan + wave * kP;
  const int n = min(kP, a.N - q0);
  __shared__ float s_A[kW][V * kWave], s_B[kW][V * kWave];
  float A[V], B[V];
#pragma unroll
  for (int i = 0; i < V; ++i) A[i] = 1.f, B[i] = 0.f;
  Marks mk(a, min(q0, a.N - 1), lane);
  if (n > 0) {
    In<T, V> gf[kP], go[GATED ? kP : 1];
    In<TG, V> gy[kP];
#pragma unroll
    for (int t = 0; t < kP; ++t) {
      const int64_t row = min(q0 + t, a.N - 1);
      gf[t].load(a.f, row, col);
      gy[t].load(a.dy, row, col);
      if constexpr (GATED) go[t].load(a.o, row, col);
    }
    float bias[V];
    load_f32<V>(a.bias, col, bias);
#pragma unroll
    for (int t = kP - 1; t >= 0; --t) {
      if (t >= n) continue;
      if (mk.end(t)) {
        float g[V] = {};
        if (a.dh_last) load_f32<V>(a.dh_last + (int64_t)mk.of(t) * a.D, col, g);
#pragma unroll
        for (int i = 0; i < V; ++i) B[i] = g[i];
      }
#pragma unroll
      for (int i = 0; i < V; ++i) {
        float fa, fq;
        forget(gf[t].get(i) + bias[i], fa, fq);
        const float u = GATED ? gate(go[t].get(i)) * gy[t].get(i) : gy[t].get(i);
        A[i] *= fa;
        B[i] = fa * (u + B[i]);
      }
    }
    if (mk.ends) {
#pragma unroll
      for (int i = 0; i < V; ++i) A[i] = kResets;
    }
  }
#pragma unroll
  for (int i = 0; i < V; ++i) {
    s_A[wave][i * kWave + lane] = A[i];
    s_B[wave][i * kWave + lane] = B[i];
  }
  __syncthreads();
  if (wave != kW - 1) return;
#pragma unroll
  for (int i = 0; i < V; ++i) {
#pragma unroll
    for (int w = kW - 2; w >= 0; --w) {
      const float A2 = s_A[w][i * kWave + lane], B2 = s_B[w][i * kWave + lane];
      B[i] = through(A2, B2, B[i]);
      A[i] = A2 < 0.f || A[i] < 0.f ? kResets : A[i] * A2;
    }
    if (in) {
      a.A[(int64_t)c * a.D + col + i] = A[i];
      a.B[(int64_t)c * a.D + col + i] = B[i];
    }
  }
}

template <typename T, typename TG, int V, bool GATED>
__global__ __launch_bounds__(kThreads) void k_scan_bwd(Scan a) {
  const int lane = threadIdx.x & (kWave - 1), wave = uniform(threadIdx.x / kWave);
  const int main_blocks = a.spans * a.slices;
  if ((int)blockIdx.x >= main_blocks) {
    // sequences of no positions hand their last state's gradient to their first
    const int m0 = ((int)blockIdx.x - main_blocks) * kWave;
    for (int m = m0 + wave; m < min(a.M, m0 + kWave); m += kW) {
      if (a.offsets[m] != a.offsets[m + 1]) continue;
      for (int d = lane; d < a.D; d += kWave)
        a.dh0[(int64_t)m * a.D + d] = a.dh_last ? a.dh_last[(int64_t)m * a.D + d] : 0.f;
    }
    return;
  }
  const int c = blockIdx.x / a.slices, col0 = ((int)blockIdx.x % a.slices * kWave + lane) * V;
  const bool in = col0 < a.D;
  const int col = in ? col0 : 0;
  const int q0 = c * kSpan + wave * kP;
  const int n = min(kP, a.N - q0);
  __shared__ float s_A[2][kW][V * kWave], s_B[2][kW][V * kWave];
  float A[V], B[V], A2[V], B2[V], fa[kP][V], fq[kP][V];
  In<T, V> gx[kP], go[GATED ? kP : 1];
  In<TG, V> gy[kP];
#pragma unroll
  for (int i = 0; i < V; ++i) A[i] = A2[i] = 1.f, B[i] = B2[i] = 0.f;
  Marks mk(a, min(q0, a.N - 1), lane);
  if (n > 0) {
    In<T, V> gf[kP];
#pragma unroll
    for (int t = 0; t < kP; ++t) {
      const int64_t row = min(q0 + t, a.N - 1);
      gx[t].load(a.x, row, col);
      gf[t].load(a.f, row, col);
      gy[t].load(a.dy, row, col);
      if constexpr (GATED) go[t].load(a.o, row, col);
    }
    float bias[V];
    load_f32<V>(a.bias, col, bias);
#pragma unroll
    for (int t = 0; t < kP; ++t) {
#pragma unroll
      for (int i = 0; i < V; ++i) forget(gf[t].get(i) + bias[i], fa[t][i], fq[t][i]);
      if (t >= n) continue;
      if (mk.start(t)) {
        float h0[V] = {};
        if (a.h0) load_f32<V>(a.h0 + (int64_t)mk.of(t) * a.D, col, h0);
#pragma unroll
        for (int i = 0; i < V; ++i) B[i] = h0[i];
      }
#pragma unroll
      for (int i = 0; i < V; ++i) {
        A[i] *= fa[t][i];
        B[i] = __builtin_fmaf(fa[t][i], B[i], fq[t][i] * gx[t].get(i));
      }
    }
#pragma unroll
    for (int t = kP - 1; t >= 0; --t) {
      if (t >= n) continue;
      if (mk.end(t)) {
        float g[V] = {};
        if (a.dh_last) load_f32<V>(a.dh_last + (int64_t)mk.of(t) * a.D, col, g);
#pragma unroll
        for (int i = 0; i < V; ++i) B2[i] = g[i];
      }
#pragma unroll
      for (int i = 0; i < V; ++i) {
        const float u = GATED ? gate(go[t].get(i)) * gy[t].get(i) : gy[t].get(i);
        A2[i] *= fa[t][i];
        B2[i] = fa[t][i] * (u + B2[i]);
      }
    }
#pragma unroll
    for (int i = 0; i < V; ++i) {
      if (mk.starts) A[i] = kResets;
      if (mk.ends) A2[i] = kResets;
    }
  }
#pragma unroll
  for (int i = 0; i < V; ++i) {
    s_A[0][wave][i * kWave + lane] = A[i];
    s_B[0][wave][i * kWave + lane] = B[i];
    s_A[1][wave][i * kWave + lane] = A2[i];
    s_B[1][wave][i * kWave + lane] = B2[i];
  }
  __syncthreads();
  float sum[V] = {};
  if (n > 0) {
    float h[V], g[V], hs[kP][V];
    load_f32<V>(c > 0 ? a.states + (int64_t)c * a.D : nullptr, col, h);
    for (int w = 0; w < wave; ++w) {
#pragma unroll
      for (int i = 0; i < V; ++i) h[i] = through(s_A[0][w][i * kWave + lane], s_B[0][w][i * kWave + lane], h[i]);
    }
    load_f32<V>(c + 1 < a.spans ? a.carry + (int64_t)c * a.D : nullptr, col, g);
    for (int w = kW - 1; w > wave; --w) {
#pragma unroll
      for (int i = 0; i < V; ++i) g[i] = through(s_A[1][w][i * kWave + lane], s_B[1][w][i * kWave + lane], g[i]);
    }
    // hs[t]: the state before position t
#pragma unroll
    for (int t = 0; t < kP; ++t) {
      if (t < n && mk.start(t)) {
        float h0[V] = {};
        if (a.h0) load_f32<V>(a.h0 + (int64_t)mk.of(t) * a.D, col, h0);
#pragma unroll
        for (int i = 0; i < V; ++i) h[i] = h0[i];
      }
#pragma unroll
      for (int i = 0; i < V; ++i) {
        hs[t][i] = h[i];
        h[i] = __builtin_fmaf(fa[t][i], h[i], fq[t][i] * gx[t].get(i));
      }
    }
#pragma unroll
    for (int t = kP - 1; t >= 0; --t) {
      if (t >= n) continue;
      if (mk.end(t)) {
        float last[V] = {};
        if (a.dh_last) load_f32<V>(a.dh_last + (int64_t)mk.of(t) * a.D, col, last);
#pragma unroll
        for (int i = 0; i < V; ++i) g[i] = last[i];
      }
      float dx[V], df[V], dO[V];
#pragma unroll
      for (int i = 0; i < V; ++i) {
        const float dy = gy[t].get(i), x = gx[t].get(i);
        float u = dy;
        if constexpr (GATED) {
          const float s = gate(go[t].get(i));
          const float ht = __builtin_fmaf(fa[t][i], hs[t][i], fq[t][i] * x);
          u = s * dy;
          dO[i] = u * ht * (1.f - s);
        }
        const float dh = u + g[i];
        dx[i] = fq[t][i] * dh;
        df[i] = dx[i] * (hs[t][i] - x) * fa[t][i];
        sum[i] += df[i];
        g[i] = fa[t][i] * dh;
      }
      if (in) {
        constexpr int kB = Vec<TG, V>::kBytes / V;
        const int64_t row = q0 + t;
        Vec<TG, V>::store(a.dx.p + row * a.dx.ld + (int64_t)col * kB, dx);
        Vec<TG, V>::store(a.df.p + row * a.df.ld + (int64_t)col * kB, df);
        if constexpr (GATED) Vec<TG, V>::store(a.dO.p + row * a.dO.ld + (int64_t)col * kB, dO);
      }
      if (a.dh0 && mk.start(t)) {
        float* dst = a.dh0 + (int64_t)mk.of(t) * a.D + col;
        if (in) {
#pragma unroll
          for (int i = 0; i < V; ++i) dst[i] = g[i];
        }
      }
    }
  }
  if (a.dbias) {
    __syncthreads();
#pragma unroll
    for (int i = 0; i < V; ++i) s_A[0][wave][i * kWave + lane] = sum[i];
    __syncthreads();
    if (wave == 0 && in) {
#pragma unroll
      for (int i = 0; i < V; ++i) {
        float t = 0.f;
#pragma unroll
        for (int w = 0; w < kW; ++w) t += s_A[0][w][i * kWave + lane];
        a.dbias[(int64_t)c * a.D + col + i] = t;
      }
    }
  }
}

// The spans' rows of the bias gradient, added in double: 16 wavefronts share
// the spans of 64 columns.
__global__ __launch_bounds__(kCarryWaves * kWave) void k_scan_dbias(const float* rows, float* dbias, int spans, int D) {
  const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x / kWave;
  const int col = blockIdx.x * kWave + lane;
  __shared__ double s_sum[kCarryWaves][kWave];
  double t = 0.;
  if (col < D) {
    constexpr int kAhead = 8;
    for (int k = wave; k < spans; k += kCarryWaves * kAhead) {
      float x[kAhead];
#pragma unroll
      for (int i = 0; i < kAhead; ++i) {
        const int at = k + i * kCarryWaves;
        x[i] = at < spans ? rows[(int64_t)at * D + col] : 0.f;
      }
#pragma unroll
      for (int i = 0; i < kAhead; ++i) t += (double)x[i];
    }
  }
  s_sum[wave][lane] = t;
  __syncthreads();
  if (wave == 0 && col < D) {
    for (int w = 1; w < kCarryWaves; ++w) t += s_sum[w][lane];
    dbias[col] = (float)t;
  }
}

// no positions at all: empty sequences' states and gradients, a zero dbias
__global__ void k_scan_nothing(const float* from, float* to, int64_t n) {
  for (int64_t i = (int64_t)blockIdx.x * blockDim.x + threadIdx.x; i < n; i += (int64_t)gridDim.x * blockDim.x)
    to[i] = from ? from[i] : 0.f;
}
void nothing(const float* from, float* to, int64_t n, hipStream_t s) {
  if (n == 0 || to == nullptr) return;
  k_scan_nothing<<<(unsigned)((n + 255) / 256 < 1024 ? (n + 255) / 256 : 1024), 256, 0, s>>>(from, to, n);
}

// ---------------------------------------------------------------- one token

template <typename T, int V, bool GATED>
__global__ __launch_bounds__(256) void k_scan_step(StepLaunch a) {
  const int per = (a.D + V - 1) / V;  // lanes a token
  const int64_t at = (int64_t)blockIdx.x * 256 + threadIdx.x;
  const int64_t row = at / per;
  if (row >= a.N) return;
  const int col = (int)(at - row * per) * V;
  constexpr int kB = Vec<T, V>::kBytes / V;
  const int64_t slot = a.slots ? (int64_t)a.slots[row] : row;
  float y[V] = {};
  if (slot >= 0 && slot < a.num_slots) {
    In<T, V> x, f, o;
    x.load(a.x, row, col);
    f.load(a.f, row, col);
    if constexpr (GATED) o.load(a.o, row, col);
    float* hp = a.state + slot * a.D + col;
#pragma unroll
    for (int i = 0; i < V; ++i) {
      float fa, fq;
      forget(f.get(i) + (a.bias ? a.bias[col + i] : 0.f), fa, fq);
      const float h = __builtin_fmaf(fa, hp[i], fq * x.get(i));
      hp[i] = h;
      y[i] = GATED ? gate(o.get(i)) * h : h;
    }
  }
  Vec<T, V>::store(a.y.p + row * a.y.ld + (int64_t)col * kB, y);
}

// ---------------------------------------------------------------- launches

size_t span_rows(int64_t N, int32_t D) {
  return align256(sizeof(float) * (size_t)((N + kSpan - 1) / kSpan) * (size_t)D);
}

Scan arguments(const ScanLaunch& p) {
  Scan a{};
  a.offsets = p.offsets;
  a.x = p.x, a.f = p.f, a.o = p.o, a.y = p.y;
  a.dy = p.dy, a.dx = p.dx, a.df = p.df, a.dO = p.dO;
  a.bias = p.bias, a.h0 = p.h0, a.h_last = p.h_last;
  a.states = p.states, a.dh_last = p.dh_last, a.dh0 = p.dh0;
  a.N = (int32_t)p.N, a.M = p.M, a.D = p.D;
  a.spans = (int32_t)((p.N + kSpan - 1) / kSpan);
  const size_t rows = span_rows(p.N, p.D);
  a.A = reinterpret_cast<float*>(p.ws);
  a.B = reinterpret_cast<float*>(p.ws + rows);
  a.carry = reinterpret_cast<float*>(p.ws + 2 * rows);
  a.dbias = p.dbias ? reinterpret_cast<float*>(p.ws + 3 * rows) : nullptr;
  return a;
}
int empties(const Scan& a, const float* out) { return out ? (a.M + kWave - 1) / kWave : 0; }

template <typename T, int V, bool GATED>
hipError_t fwd(Scan a, float* states, hipStream_t s) {
  a.slices = (a.D + kWave * V - 1) / (kWave * V);
  const unsigned main = (unsigned)(a.spans * a.slices);
  if (states) a.carry = states;
  if (a.spans > 1) {
    k_scan_fwd<T, V, GATED, false><<<main, kThreads, 0, s>>>(a);
  }
  if (a.spans == 1) nothing(nullptr, states, a.D, s);
  else
    k_scan_carry<false><<<(a.D + kWave - 1) / kWave, kCarryWaves * kWave, 0, s>>>(a.A, a.B, a.carry, a.spans, a.D);
  k_scan_fwd<T, V, GATED, true><<<main + empties(a, a.h_last), kThreads, 0, s>>>(a);
  return hipGetLastError();
}
template <typename T, int V>
hipError_t fwd_gated(const ScanLaunch& p, hipStream_t s) {
  return p.gated ? fwd<T, V, true>(arguments(p), p.states, s) : fwd<T, V, false>(arguments(p), p.states, s);
}

template <typename T, typename TG, int V, bool GATED>
hipError_t bwd(Scan a, float* dbias, hipStream_t s) {
  a.slices = (a.D + kWave * V - 1) / (kWave * V);
  const unsigned main = (unsigned)(a.spans * a.slices);
  const unsigned cols = (unsigned)(a.D + kWave - 1) / kWave;
  if (a.spans > 1) {
    k_scan_back_sums<T, TG, V, GATED><<<main, kThreads, 0, s>>>(a);
    k_scan_carry<true><<<cols, kCarryWaves * kWave, 0, s>>>(a.A, a.B, a.carry, a.spans, a.D);
  }
  k_scan_bwd<T, TG, V, GATED><<<main + empties(a, a.dh0), kThreads, 0, s>>>(a);
  if (dbias) k_scan_dbias<<<cols, kCarryWaves * kWave, 0, s>>>(a.dbias, dbias, a.spans, a.D);
  return hipGetLastError();
}
template <typename T, typename TG, int V>
hipError_t bwd_gated(const ScanLaunch& p, hipStream_t s) {
  return p.gated ? bwd<T, TG, V, true>(arguments(p), p.dbias, s) : bwd<T, TG, V, false>(arguments(p), p.dbias, s);
}

template <typename T, int V>
hipError_t step(const StepLaunch& p, hipStream_t s) {
  const int64_t per = (p.D + V - 1) / V, blocks = (p.N * per + 255) / 256;
  if (p.gated) k_scan_step<T, V, true><<<(unsigned)blocks, 256, 0, s>>>(p);
  else k_scan_step<T, V, false><<<(unsigned)blocks, 256, 0, s>>>(p);
  return hipGetLastError();
}

}  // namespace

size_t scan_ws_bytes(int64_t N, int32_t D) { return 4 * span_rows(N > 0 ? N : 1, D); }

hipError_t launch_scan_fwd(const ScanLaunch& p, hipStream_t s) {
  if (p.N == 0) {
    nothing(p.h0, p.h_last, (int64_t)p.M * p.D, s);
    return hipGetLastError();
  }
  if (p.dtype == EMB_FP32) return fwd_gated<float, 1>(p, s);
  return p.vector == 2 ? fwd_gated<bf16, 2>(p, s) : fwd_gated<bf16, 1>(p, s);
}

hipError_t launch_scan_bwd(const ScanLaunch& p, hipStream_t s) {
  if (p.N == 0) {
    nothing(p.dh_last, p.dh0, (int64_t)p.M * p.D, s);
    nothing(nullptr, p.dbias, p.D, s);
    return hipGetLastError();
  }
  if (p.dtype == EMB_FP32) return bwd_gated<float, float, 1>(p, s);
  if (p.dtype == EMB_BF16) return p.vector == 2 ? bwd_gated<bf16, bf16, 2>(p, s) : bwd_gated<bf16, bf16, 1>(p, s);
  if (p.grad_dtype == EMB_FP32) return bwd_gated<Saved8, float, 1>(p, s);
  return p.vector == 2 ? bwd_gated<Saved8, bf16, 2>(p, s) : bwd_gated<Saved8, bf16, 1>(p, s);
}

hipError_t launch_scan_step(const StepLaunch& p, hipStream_t s) {
  if (p.dtype == EMB_FP32) return step<float, 1>(p, s);
  return p.vector == 2 ? step<bf16, 2>(p, s) : step<bf16, 1>(p, s);
}

}  // namespace emb
