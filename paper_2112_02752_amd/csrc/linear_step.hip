// Linear attention of one token of each running sequence (gfx950):
//
//   S = g S + k^T v,   y = scale q S
//
// A block takes a token's key head: its state, dk x dv, is read and written
// once, V columns a lane, and the sums over dk of up to R query heads are taken
// on the way.  Bound by the states' bytes: 128 tokens x 12 heads of 128 x 128, 201 MB
// read and written, 38 us, 5.3 TB/s.
#include "block_common.h"

namespace emb {

namespace {

constexpr int kThreads = 256;

// The lanes: `wide` (a power of two) across the columns, the rest down the rows.
template <typename T, int V, int R>
__global__ __launch_bounds__(kThreads) void k_linear_step(LinStepLaunch a, int wide) {
  __shared__ float s_q[R][kLinMaxDim], s_k[kLinMaxDim];
  __shared__ float s_sum[R][kThreads * V];
  const int64_t token = blockIdx.x / a.groups;
  const int group = (int)(blockIdx.x % a.groups), per = a.heads / a.groups;
  const int64_t slot = a.slots != nullptr ? a.slots[token] : token;
  const bool there = slot >= 0 && slot < a.num_slots;
  const int c = threadIdx.x % wide * V, down = kThreads / wide, r0 = threadIdx.x / wide;
  const float g = a.decay[group];
  const char* kp = a.k.p + token * a.k.ld;
  const char* vp = a.v.p + token * a.v.ld;
  const char* qp = a.q.p + token * a.q.ld;
  char* yp = a.y.p + token * a.y.ld;
  constexpr int size = Vec<T, 1>::kBytes;
  auto value = [](const char* p) {
    Vec<T, 1> v;
    v.load(p);
    return v.get(0);
  };
  float v[V];
#pragma unroll
  for (int i = 0; i < V; ++i) v[i] = c + i < a.dv ? value(vp + ((int64_t)group * a.dv + c + i) * size) : 0.f;
  float* st = there ? a.state + (slot * a.groups + group) * (int64_t)a.dk * a.dv : nullptr;
  for (int d = threadIdx.x; d < a.dk; d += kThreads) s_k[d] = value(kp + ((int64_t)group * a.dk + d) * size);
  for (int h0 = 0; h0 < per; h0 += R) {
    const int heads = min(R, per - h0);
    __syncthreads();
    for (int x = threadIdx.x; x < heads * a.dk; x += kThreads)
      s_q[x / a.dk][x % a.dk] = value(qp + (((int64_t)group * per + h0) * a.dk + x) * size);
    __syncthreads();
    float y[R][V] = {};
    if (there && c < a.dv) {
#pragma unroll 8
      for (int d = r0; d < a.dk; d += down) {
        Vec<float, V> s;
        s.load(st + (int64_t)d * a.dv + c);
        float n[V];
        const float k = s_k[d];
#pragma unroll
        for (int i = 0; i < V; ++i) n[i] = h0 == 0 ? g * s.get(i) + k * v[i] : s.get(i);
        if (h0 == 0) Vec<float, V>::store(st + (int64_t)d * a.dv + c, n);
#pragma unroll
        for (int h = 0; h < R; ++h)
#pragma unroll
          for (int i = 0; i < V; ++i) y[h][i] += (h < heads ? s_q[h][d] : 0.f) * n[i];
      }
    }
#pragma unroll
    for (int h = 0; h < R; ++h)
#pragma unroll
      for (int i = 0; i < V; ++i) s_sum[h][threadIdx.x * V + i] = y[h][i];
    __syncthreads();
    for (int x = threadIdx.x; x < heads * a.dv; x += kThreads) {
      const int h = x / a.dv, col = x % a.dv;
      float sum = 0.f;
      for (int r = 0; r < down; ++r) sum += s_sum[h][r * wide * V + col];
      const float out[1] = {there ? a.scale * sum : 0.f};
      Vec<T, 1>::store(yp + (((int64_t)group * per + h0) * a.dv + x) * size, out);
    }
  }
}

template <typename T, int V>
hipError_t by_heads(const LinStepLaunch& p, hipStream_t s) {
  const unsigned blocks = (unsigned)(p.N * p.groups);
  int wide = 1;
  while (wide * V < p.dv) wide *= 2;
  const int per = p.heads / p.groups;
  if (per == 1) k_linear_step<T, V, 1><<<blocks, kThreads, 0, s>>>(p, wide);
  else if (per == 2) k_linear_step<T, V, 2><<<blocks, kThreads, 0, s>>>(p, wide);
  else k_linear_step<T, V, 4><<<blocks, kThreads, 0, s>>>(p, wide);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_lin_step(const LinStepLaunch& p, hipStream_t s) {
  if (!launchable(p.N * p.groups, kThreads)) return hipErrorNotSupported;
  const bool four = p.dv % 4 == 0 && ((uintptr_t)p.state & 15u) == 0;
  if (p.dtype == EMB_FP32) return four ? by_heads<float, 4>(p, s) : by_heads<float, 1>(p, s);
  return four ? by_heads<bf16, 4>(p, s) : by_heads<bf16, 1>(p, s);
}

}  // namespace emb
