// Launch descriptors of the operators of a model's block (norm and dropout,
// linear attention, log probabilities).  A launch enqueues nothing and returns
// hipErrorNotSupported where a kernel's grid would be too large.
#pragma once

#include "seq_common.h"

namespace emb {

// A draw's key, and what it drops: values whose 16 bits are below `below`.
struct Drop {
  uint64_t key;
  uint32_t below;  // 0: nothing
  float scale;     // of kept values
  int64_t first_row;
};

constexpr int kNormMaxDim = 16384;
struct NormLaunch {
  int64_t N;
  int32_t D, dtype, stream_dtype;
  float eps;
  const float* weight;
  Drop drop;
  // forward: x, residual (or none), total, y, saved (each may be none)
  // backward: total, dy, arriving (or none), dtotal, dbranch (each may be none)
  Rows x, residual, total, y, saved, dy, arriving, dtotal, dbranch;
  float* dweight;
  int32_t add;
  float* ws;
};
size_t norm_ws_bytes(int64_t N, int32_t D);
hipError_t launch_norm_fwd(const NormLaunch& p, hipStream_t s);
hipError_t launch_norm_bwd(const NormLaunch& p, hipStream_t s);

struct DropLaunch {
  int64_t N;
  int32_t D, dtype;
  Drop drop;
  Rows x, y;
};
Drop make_drop(float p, uint64_t seed, int64_t first_row);  // p below 1
hipError_t launch_dropout(const DropLaunch& p, hipStream_t s);

// Heads of linear attention are at most this wide.
constexpr int kLinMaxDim = 256;
struct LinLaunch {
  int64_t N;
  int32_t M, heads, groups, dk, dv, dtype;
  int32_t aligned;  // every matrix, row and head begins at a multiple of 16 bytes
  float scale;
  const int32_t* offsets;
  const float* decay;
  Rows q, k, v, y;         // forward
  Rows dy, dq, dkey, dval; // backward
  const float* first;      // [M][groups][dk][dv] or none, as are the next three
  float* last;
  const float* dlast;
  float* dfirst;
  float* states;  // at the boundaries between segments: the forward's, read by the backward
  float* grads;   // the backward's
};
size_t lin_states_bytes(int64_t N, int32_t groups, int32_t dk, int32_t dv);
hipError_t launch_lin_fwd(const LinLaunch& p, hipStream_t s);
hipError_t launch_lin_bwd(const LinLaunch& p, hipStream_t s);

struct LinStepLaunch {
  int64_t N, num_slots;
  int32_t heads, groups, dk, dv, dtype;
  float scale;
  const float* decay;
  Rows q, k, v, y;
  float* state;
  const int32_t* slots;
};
hipError_t launch_lin_step(const LinStepLaunch& p, hipStream_t s);

// Statistics of a row of logits that its gradient needs: the largest logit m (zero where no token can be), sum of
// 2^(scale log2(e) (logit - m)), entropy, one value unused.
constexpr int kStats = 4;
constexpr int32_t kLogpMaxCols = 1 << 30;
struct LogpLaunch {
  int64_t N;
  int32_t D, dtype, id_bytes, top;
  float scale;
  Rows logits, dlogits;
  const void* ids;  // or none
  float *logp, *entropy;  // each may be none
  int32_t* top_ids;
  float* top_logp;
  float* stats;  // forward: or none
  const float *dlogp, *dentropy;  // each may be none
};
hipError_t launch_logp(const LogpLaunch& p, hipStream_t s);       // dlogits: with the gradient
hipError_t launch_logp_bwd(const LogpLaunch& p, hipStream_t s);

// ------------------------------------------------------------ device helpers

// A reduction over the wavefront: within rows of 16 lanes by lane moves that
// cost no more than the sum itself, then the four rows' (an exchange through
// LDS would take its latency six times).  Every lane gets the result, the same
// to the last bit.
template <int CTRL>
__device__ __forceinline__ float lane_move(float v) {
  return __uint_as_float((uint32_t)__builtin_amdgcn_mov_dpp((int)__float_as_uint(v), CTRL, 0xf, 0xf, true));
}
__device__ __forceinline__ float lane_at(float v, int l) { return __uint_as_float(lane_at(__float_as_uint(v), l)); }
template <typename F>
__device__ __forceinline__ float wave_reduce(float v, F op) {
  v = op(v, lane_move<0xb1>(v));   // quad_perm:[1,0,3,2]
  v = op(v, lane_move<0x4e>(v));   // quad_perm:[2,3,0,1]
  v = op(v, lane_move<0x141>(v));  // row_half_mirror
  v = op(v, lane_move<0x140>(v));  // row_mirror
  return op(op(lane_at(v, 0), lane_at(v, 16)), op(lane_at(v, 32), lane_at(v, 48)));
}
__device__ __forceinline__ float wave_sum(float v) {
  return wave_reduce(v, [](float a, float b) { return a + b; });
}
__device__ __forceinline__ float wave_max(float v) {
  return wave_reduce(v, [](float a, float b) { return fmaxf(a, b); });
}

}  // namespace emb
