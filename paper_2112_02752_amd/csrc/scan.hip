// Gated linear recurrence over ragged sequences (gfx950), one state a column:
//
//   a_t = sigmoid(f_t + bias),  h_t = a_t h_{t-1} + (1 - a_t) x_t,  y_t = sigmoid(o_t) h_t
//
// Steps h -> a h + b compose: (A1, B1) then (A2, B2) is (A1 A2, A2 B1 + B2), so
// the positions are cut into spans, whatever sequences they belong to (a
// sequence's first position discards what came before it).  A block takes one
// span of 64 or 128 columns (a slice): each wavefront holds its part of the
// span's positions in registers, a lane one or two columns, and the parts are
// joined through LDS.  Every value is read and written once: a block publishes
// its span's (A, B), then takes what enters the span from the spans before it,
// and publishes what leaves it:
//  - blocks take their span's number from a counter of the slice, so a span's
//    block waits for blocks that have started before it, and every wait ends;
//  - it looks at the 32 spans before it at once, and starts from the nearest
//    whose outgoing state is known, through the (A, B) of those after that one:
//    the same steps in the same order wherever it starts, so results do not
//    depend on timing;
//  - published words are stored and read at device scope, a flag after the
//    words it announces; flags and counters are cleared by a kernel before.
// 32768 positions x 2048 in bf16 (gated): 145 us forward, 3.8 TB/s; the same loads
// and stores without the recurrence take 105 us (93 with 8-byte lanes).  What is
// between is the chain: of the 19 us that a block lived when it was traced, 8 were
// its loads and sums, 6.5 the wait for the spans before it and 3.5 the stores, and
// two blocks (126 registers a lane) share a compute unit.  There, spans of 64 take
// 206 us, 16 wavefronts of 16 positions 152 and of 8 positions 154; looking at 64
// spans 152; all eight wavefronts polling 20 us more; the next span's x and f loaded
// during the wait 190 (spans of 112); gates computed twice, for three blocks a
// compute unit, 166; three passes over the data (the spans' steps, the states
// between them, the outputs) 190.
//
// The backward is the same from the last position to the first on
// dh_t = sigmoid(o_t) dy_t + a_{t+1} dh_{t+1}, with h recomputed inside each
// span of 64 from the state the forward kept: 238 us there, 4.1 TB/s (its loads and
// stores are 939 MB), bound likewise; from 8-bit checkpoints at 16384 x 1280, 75 us,
// 3.4 TB/s, its vector instructions half of the cycles.
//
// Gates are the hardware's exponential and reciprocal on fp32's product of z and
// log2(e), whose rounding moves the smaller of a gate and its rest by about |z| 2^-24
// of its size, twice what the rounding of z itself does; the others add a few units.
//
// A span that holds a first position passes nothing on of what it receives:
// its A is kResets, not a product with zero, which would carry an infinity or
// NaN of one sequence into the next.
#include "seq_common.h"

namespace emb {

namespace {

constexpr float kResets = -1.0f;  // (products of a's are never negative)
constexpr int kW = 8;             // wavefronts of a block
constexpr int kThreads = kW * kWave;
// Positions a wavefront holds: spans of 128 forward (of 64 where those would be
// at most 96 blocks), of 64 (the kept states') backward.
constexpr int kFwdP = 16, kFwdFewP = 8, kFwdFewBlocks = 96;
constexpr int kBackP = kSpan / kW;
constexpr int kLook = 32;         // spans a block looks back at

struct Saved8 {};

// V columns of a matrix as they lie in memory
template <typename T, int V>
struct In {
  Vec<T, V> v;
  __device__ __forceinline__ void load(const Rows& m, int64_t row, int col) {
    // (the row is the wavefront's, the column a lane's 32-bit offset)
    v.load(m.p + row * m.ld + (uint32_t)col * (uint32_t)(Vec<T, V>::kBytes / V));
  }
  __device__ __forceinline__ float get(int i) const { return v.get(i); }
};
template <int V>
struct In<Saved8, V> {
  uint32_t codes, e;
  __device__ __forceinline__ void load(const Rows& m, int64_t row, int col) {
    const char* p = m.p + row * m.ld + (uint32_t)col;
    if constexpr (V == 1) codes = *reinterpret_cast<const uint8_t*>(p);
    else codes = *reinterpret_cast<const uint16_t*>(p);
    e = (m.exps + row * m.ld_exps)[(uint32_t)col / EMB_SAVED_GROUP];
  }
  // (exponent 255: the codes are zeros, and zero times infinity is NaN)
  __device__ __forceinline__ float get(int i) const {
    return (float)(int8_t)(codes >> (8 * i)) * __uint_as_float(e << 23);
  }
};

// sigmoid(z) and sigmoid(-z), the latter without cancellation; NaN stays NaN
__device__ __forceinline__ void forget(float z, float& a, float& q) {
  float t = -1.44269504f * z;
  t = __builtin_elementwise_minimum(t, 126.f);
  const float e = __builtin_amdgcn_exp2f(t);
  a = __builtin_amdgcn_rcpf(1.f + e);
  q = e * a;
}
__device__ __forceinline__ float gate(float z) {
  return __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(-1.44269504f * z));
}

// with 1 - sigmoid(z), without cancellation; times sigmoid(z), as here, it may be anything finite where that is zero
__device__ __forceinline__ float gate(float z, float& rest) {
  const float e = __builtin_amdgcn_exp2f(-1.44269504f * z), s = __builtin_amdgcn_rcpf(1.f + e);
  rest = __builtin_elementwise_minimum(e, 0x1p126f) * s;
  return s;
}

// (kernels of their own for the two kinds of stores: behind a branch they become one)
template <typename T, int V, bool STREAM>
__device__ __forceinline__ void put(void* p, const float (&v)[V]) {
  if constexpr (STREAM) Vec<T, V>::stream(p, v);
  else Vec<T, V>::store(p, v);
}

// (A, B) applied to a state
__device__ __forceinline__ float through(float A, float B, float h) {
  return A < 0.f ? B : __builtin_fmaf(A, h, B);
}
// A product of gates is above zero, however many: where it has underflowed, the least number stands for it, so that
// an infinite state stays one.  (NaN stays NaN.)
__device__ __forceinline__ float above_zero(float A) { return __builtin_elementwise_maximum(A, 0x1p-149f); }
// the product of two that may be kResets
__device__ __forceinline__ float join(float A, float A2) { return A2 < 0.f || A < 0.f ? kResets : above_zero(A * A2); }
// whether a state of the wavefront is infinite: rare, and only then the products for single positions matter so
template <int V>
__device__ __forceinline__ bool any_infinite(const float (&h)[V]) {
  bool some = false;
#pragma unroll
  for (int i = 0; i < V; ++i) some |= __builtin_isinf(h[i]);
  return __ballot(some) != 0u;
}
template <int V>
__device__ __forceinline__ void above_zero(float (&A)[V], const float (&h)[V]) {
#pragma unroll
  for (int i = 0; i < V; ++i) A[i] = __builtin_isinf(h[i]) ? above_zero(A[i]) : A[i];
}

struct Scan {
  const int32_t* offsets;
  Rows x, f, o, y, dy, dx, df, dO;
  const float *bias, *h0, *dh_last;
  float *states, *h_last, *dh0, *dbias;  // dbias: [spans][D], one row a span
  int32_t N, M, D, spans, slices;
  WsHeader* hdr;  // of the workspace: the record of waits that ran out
  // what spans publish, by (span in the order they are taken, slice)
  uint32_t* taken;  // [slices]
  uint32_t* flags;  // [slices][spans]
  uint64_t* steps;  // [spans][slices][V * 64]: A and B
  uint32_t* out;    // [spans][slices][V * 64]: the state that leaves the span
};
enum Flag : uint32_t { kNothing = 0, kSteps = 1, kOut = 2 };

// First and last positions of sequences among a wavefront's P positions from
// q0 on, and the sequence of each.  Offsets are read by scalar loads, which do
// not wait behind the vector loads of the positions' values.
template <int P>
struct Marks {
  uint32_t starts;  // bit t: position q0 + t is its sequence's first
  uint32_t ends;    // bit t: position q0 + t is its sequence's last
  int seq;          // lane t: the sequence of position q0 + t
  __device__ __forceinline__ Marks(const Scan& a, int q0, int lane) {
    const auto* off = (const __attribute__((address_space(4))) int32_t*)(uintptr_t)a.offsets;
    // the last sequence that begins at or before q0
    int m = 0, n = a.M;
    while (n > 1) {
      const int half = n / 2;
      const bool up = off[m + half] <= q0;
      m = up ? m + half : m;
      n = up ? n - half : half;
    }
    seq = m;
    uint32_t s = off[m] == q0 ? 1u : 0u;
    int k = m + 1, at = k <= a.M ? off[k] : INT32_MAX;
    while (at - q0 <= P) {
      int next = k < a.M ? off[k + 1] : INT32_MAX;
      if (next == at) {
        // Of the sequences that begin there the last is the one with positions, and there may be millions: from k on
        // by doubling steps, then by halving ones (80 ns each one by one: 10000 of them took a call from 20 us to 820)
        int d = 1;
        for (; d <= a.M - k && off[k + d] == at; d *= 2) k += d;
        for (d /= 2; d > 0; d /= 2) {
          if (d <= a.M - k && off[k + d] == at) k += d;
        }
        next = k < a.M ? off[k + 1] : INT32_MAX;
      }
      const int t = at - q0;
      s |= 1u << t;
      if (k < a.M && lane >= t) seq = k;
      ++k;
      at = next;
    }
    starts = s & ((1u << P) - 1u);
    ends = s >> 1;
    if (a.N - q0 <= P) ends |= 1u << (a.N - q0 - 1);
  }
  __device__ __forceinline__ bool start(int t) const { return (starts >> t) & 1u; }
  __device__ __forceinline__ bool end(int t) const { return (ends >> t) & 1u; }
  // whether a sequence begins at or before t, or ends at or after it, within the wavefront's positions
  __device__ __forceinline__ bool begun(int t) const { return (starts & ((2u << t) - 1u)) != 0u; }
  __device__ __forceinline__ bool closed(int t) const { return (ends >> t) != 0u; }
  __device__ __forceinline__ int of(int t) const { return lane_at(seq, t); }
};

// V values of a row of the sequences' states
template <int V>
__device__ __forceinline__ void store_f32(float* p, bool in, const float (&v)[V]) {
  if (in) {
#pragma unroll
    for (int i = 0; i < V; ++i) p[i] = v[i];
  }
}

// ---------------------------------------------------------------- the spans' chain

__device__ __forceinline__ void publish_flag(uint32_t* flag, Flag value, int lane) {
  // the words before it have reached the device's memory
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  if (lane == 0) __hip_atomic_store(flag, (uint32_t)value, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ uint32_t ld_u32(const uint32_t* p) {
  return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

template <int V>
struct Chain {
  static constexpr int kCols = V * kWave;
  WsHeader* hdr;
  uint32_t* flags;  // of the slice
  uint64_t* steps;
  uint32_t* out;
  int64_t apart;    // words from one span's to the next's
  int idx;          // this block's place among the slice's spans
  __device__ __forceinline__ Chain(const Scan& a, int slice, int span) {
    hdr = a.hdr;
    flags = a.flags + (int64_t)slice * a.spans;
    apart = (int64_t)a.slices * kCols;
    steps = a.steps + (int64_t)slice * kCols;
    out = a.out + (int64_t)slice * kCols;
    idx = span;
  }
  __device__ __forceinline__ void publish_steps(const float (&A)[V], const float (&B)[V], int lane) const {
#pragma unroll
    for (int i = 0; i < V; ++i)
      st_u64(steps + idx * apart + i * kWave + lane, ((uint64_t)__float_as_uint(A[i]) << 32) | __float_as_uint(B[i]));
    publish_flag(flags + idx, kSteps, lane);
  }
  __device__ __forceinline__ void publish_out(const float (&h)[V], int lane) const {
#pragma unroll
    for (int i = 0; i < V; ++i)
      __hip_atomic_store(out + idx * apart + i * kWave + lane, __float_as_uint(h[i]), __ATOMIC_RELAXED,
                         __HIP_MEMORY_SCOPE_AGENT);
    publish_flag(flags + idx, kOut, lane);
  }
};

// What a block gathers of the spans before its own.
template <int V>
struct Look {
  uint64_t steps[kLook][V * kWave];
  float out[V * kWave];
  int from;  // the span whose outgoing state is known, counted back
};

// The state that enters span idx.  One wavefront waits until the outgoing state
// of one of the 32 spans before it and the steps of those after that one are
// published (a span before the first counts as one whose state is zero); then
// all fetch a share of the steps, and apply them in order.
template <int V>
__device__ __forceinline__ void look_back(const Chain<V>& ch, Look<V>& lk, float (&h)[V], int wave, int lane) {
  if (wave == kW - 1) {
    const uint64_t t0 = wait_clock();
    int j;
    for (;;) {
      const int at = ch.idx - 1 - lane;
      const uint32_t flag = lane >= kLook ? (uint32_t)kNothing : (at >= 0 ? ld_u32(ch.flags + at) : (uint32_t)kOut);
      const uint32_t known = (uint32_t)__ballot(flag == kOut), some = (uint32_t)__ballot(flag != kNothing);
      j = known ? __builtin_ctz(known) : kLook;
      if (known && (~some & ((1u << j) - 1u)) == 0u) break;
      // (not reached: the blocks waited for are running.  Two seconds, not the dedup's 20 ms: what a block would go on
      // with is wrong values, not a call that it can still undo, and a device shared with others may stop it for longer)
      if (wait_clock() - t0 > 200000000ull) {
        if (lane == 0) {
          // (the header's generation is 0: no dedup has used it)
          __hip_atomic_fetch_or(&ch.hdr->err, (uint64_t)kScanError, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
          atomic_add_u32(&ch.hdr->timeouts, 1u);
          ch.hdr->timeout_site = kSiteScan;
          ch.hdr->timeout_block = blockIdx.x;
        }
        j = -1;
        break;
      }
      __builtin_amdgcn_s_sleep(1);
    }
    if (lane == 0) lk.from = j;
  }
  __syncthreads();
  const int j = uniform(lk.from);
#pragma unroll
  for (int r = 0; r < kLook / kW; ++r) {
    const int k = wave + r * kW;
    if (k < j) {
#pragma unroll
      for (int i = 0; i < V; ++i)
        lk.steps[k][i * kWave + lane] = ld_relaxed_u64(ch.steps + (ch.idx - 1 - k) * ch.apart + i * kWave + lane);
    }
  }
  if (wave == kW - 1) {
#pragma unroll
    for (int i = 0; i < V; ++i) {
      uint32_t w = j < 0 ? 0x7fc00000u : 0u;
      if (j >= 0 && ch.idx - 1 - j >= 0) w = ld_u32(ch.out + (ch.idx - 1 - j) * ch.apart + i * kWave + lane);
      lk.out[i * kWave + lane] = __uint_as_float(w);
    }
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < V; ++i) h[i] = lk.out[i * kWave + lane];
#pragma unroll 4
  for (int k = j - 1; k >= 0; --k) {
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const uint64_t w = lk.steps[k][i * kWave + lane];
      h[i] = through(__uint_as_float((uint32_t)(w >> 32)), __uint_as_float((uint32_t)w), h[i]);
    }
  }
}

// this block's span among its slice's, in the order the blocks start
__device__ __forceinline__ int take(uint32_t* counter, int* s) {
  if (threadIdx.x == 0) *s = (int)atomic_add_u32(counter, 1u);
  __syncthreads();
  return uniform(*s);
}

template <int V>
__device__ __forceinline__ void load_f32(const float* p, int col, float (&v)[V]) {
#pragma unroll
  for (int i = 0; i < V; ++i) v[i] = p ? p[col + i] : 0.f;
}
// The same where few positions need it: the values are waited for here, in the
// branch that needs them, not by all that comes after it (whose wait would be
// for every load in flight).
template <int V>
__device__ __forceinline__ void load_rare(const float* p, int col, float (&v)[V]) {
#pragma unroll
  for (int i = 0; i < V; ++i) v[i] = p ? p[col + i] : 0.f;
  if (p) {
#pragma unroll
    for (int i = 0; i < V; ++i) asm volatile("" : "+v"(v[i]));
  }
}

// ---------------------------------------------------------------- forward

template <typename T, int V, int P, bool GATED, bool STREAM>
__global__ __launch_bounds__(kThreads, 4) void k_scan_fwd(Scan a) {
  const int lane = threadIdx.x & (kWave - 1), wave = uniform(threadIdx.x / kWave);
  const int main_blocks = a.spans * a.slices;
  if ((int)blockIdx.x >= main_blocks) {
    // sequences of no positions keep their first state
    const int m0 = ((int)blockIdx.x - main_blocks) * kWave;
    for (int m = m0 + wave; m < min(a.M, m0 + kWave); m += kW) {
      if (a.offsets[m] != a.offsets[m + 1]) continue;
      for (int d = lane; d < a.D; d += kWave)
        a.h_last[(int64_t)m * a.D + d] = a.h0 ? a.h0[(int64_t)m * a.D + d] : 0.f;
    }
    return;
  }
  __shared__ float s_A[kW][V * kWave], s_B[kW][V * kWave];
  __shared__ Look<V> s_look;
  __shared__ int s_take, s_first;
  const int slice = (int)blockIdx.x % a.slices;
  const int c = a.spans > 1 ? take(a.taken + slice, &s_take) : 0;
  const int col0 = (slice * kWave + lane) * V;
  const bool in = col0 < a.D;
  const int col = in ? col0 : 0;
  const int q0 = (c * kW + wave) * P;
  const int n = min(P, a.N - q0);  // (0 or less: this wavefront has no positions)
  // the state after position t is At[t] times the one that enters the wavefront's positions plus Bt[t]
  float A[V], B[V], At[P][V], Bt[P][V], Ae[V], Be[V], bias[V];
  In<T, V> gx[P], gf[P], go[GATED ? P : 1];
#pragma unroll
  for (int i = 0; i < V; ++i) A[i] = 1.f, B[i] = Ae[i] = Be[i] = 0.f;
#pragma unroll
  for (int t = 0; t < P; ++t) {
    const int64_t row = min(q0 + t, a.N - 1);
    gx[t].load(a.x, row, col);
    gf[t].load(a.f, row, col);
  }
  if constexpr (GATED) {
#pragma unroll
    for (int t = 0; t < P; ++t) go[t].load(a.o, min(q0 + t, a.N - 1), col);
  }
  const Marks<P> mk(a, min(q0, a.N - 1), lane);
  load_f32<V>(a.bias, col, bias);
  if (n > 0) {
#pragma unroll
    for (int t = 0; t < P; ++t) {
      if (t < n && mk.start(t)) {
        float h0[V];
        load_rare<V>(a.h0 ? a.h0 + (int64_t)mk.of(t) * a.D : nullptr, col, h0);
#pragma unroll
        for (int i = 0; i < V; ++i) B[i] = h0[i];
      }
#pragma unroll
      for (int i = 0; i < V; ++i) {
        float fa, fq;
        forget(gf[t].get(i) + bias[i], fa, fq);
        A[i] *= fa;
        B[i] = __builtin_fmaf(fa, B[i], fq * gx[t].get(i));
        At[t][i] = A[i];
        Bt[t][i] = B[i];
      }
      if (a.h_last && t < n && mk.end(t)) {
        if (mk.begun(t)) {
          store_f32<V>(a.h_last + (int64_t)mk.of(t) * a.D + col, in, B);
        } else {
          // (the one sequence that came in: its state is not known yet)
#pragma unroll
          for (int i = 0; i < V; ++i) Ae[i] = A[i], Be[i] = B[i];
        }
      }
    }
#pragma unroll
    for (int i = 0; i < V; ++i) A[i] = mk.starts ? kResets : above_zero(A[i]);
  }
#pragma unroll
  for (int i = 0; i < V; ++i) {
    s_A[wave][i * kWave + lane] = A[i];
    s_B[wave][i * kWave + lane] = B[i];
  }
  if (threadIdx.x == 0) s_first = mk.start(0);
  __syncthreads();
  const Chain<V> ch(a, slice, c);
  const bool leads = a.spans > 1 && wave == 0 && c + 1 < a.spans;  // what leaves the span is to be published
  bool resets = false;
  if (leads) {
    // the span's steps; past a first position they are its outgoing state
#pragma unroll
    for (int w = 1; w < kW; ++w) {
#pragma unroll
      for (int i = 0; i < V; ++i) {
        const float A2 = s_A[w][i * kWave + lane], B2 = s_B[w][i * kWave + lane];
        B[i] = through(A2, B2, B[i]);
        A[i] = join(A[i], A2);
      }
    }
    resets = uniform(A[0] < 0.f);
    if (resets) ch.publish_out(B, lane);
    else ch.publish_steps(A, B, lane);
  }
  // the output gates, while the spans before this one publish
  if constexpr (GATED) {
#pragma unroll
    for (int t = 0; t < P; ++t) {
#pragma unroll
      for (int i = 0; i < V; ++i) {
        const float g = gate(go[t].get(i));
        At[t][i] *= g;
        Bt[t][i] *= g;
      }
    }
  }
  float h[V] = {};
  if (a.spans > 1 && !s_first) {
    look_back<V>(ch, s_look, h, wave, lane);
    if (leads && !resets) {
      float leaves[V];
#pragma unroll
      for (int i = 0; i < V; ++i) leaves[i] = through(A[i], B[i], h[i]);
      ch.publish_out(leaves, lane);
    }
  }
  if (n <= 0) return;
  for (int w = 0; w < wave; ++w) {
#pragma unroll
    for (int i = 0; i < V; ++i) h[i] = through(s_A[w][i * kWave + lane], s_B[w][i * kWave + lane], h[i]);
  }
  if (a.states && q0 % kSpan == 0) store_f32<V>(a.states + (int64_t)(q0 / kSpan) * a.D + col, in, h);
#pragma unroll
  for (int t = 0; t < P; ++t) {
    if (t >= n) continue;
    float y[V];
#pragma unroll
    for (int i = 0; i < V; ++i) y[i] = mk.begun(t) ? Bt[t][i] : __builtin_fmaf(At[t][i], h[i], Bt[t][i]);
    if (in)
      put<T, V, STREAM>(a.y.p + (int64_t)(q0 + t) * a.y.ld + (uint32_t)col * (uint32_t)(Vec<T, V>::kBytes / V), y);
    if (a.h_last && mk.end(t) && !mk.begun(t)) {
#pragma unroll
      for (int i = 0; i < V; ++i) y[i] = __builtin_fmaf(Ae[i], h[i], Be[i]);
      store_f32<V>(a.h_last + (int64_t)mk.of(t) * a.D + col, in, y);
    }
  }
  // (after the others, whose stores then do not wait for the question)
  if (any_infinite<V>(h)) {
#pragma unroll
    for (int t = 0; t < P; ++t) {
      if (t >= n || mk.begun(t)) continue;
      float y[V];
      above_zero<V>(At[t], h);
#pragma unroll
      for (int i = 0; i < V; ++i) y[i] = __builtin_fmaf(At[t][i], h[i], Bt[t][i]);
      if (in) Vec<T, V>::store(a.y.p + (int64_t)(q0 + t) * a.y.ld + (uint32_t)col * (uint32_t)(Vec<T, V>::kBytes / V), y);
      if (a.h_last && mk.end(t)) {
        above_zero<V>(Ae, h);
#pragma unroll
        for (int i = 0; i < V; ++i) y[i] = __builtin_fmaf(Ae[i], h[i], Be[i]);
        store_f32<V>(a.h_last + (int64_t)mk.of(t) * a.D + col, in, y);
      }
    }
  }
}

// ---------------------------------------------------------------- backward

template <typename T, typename TG, int V, bool GATED, bool STREAM>
__global__ __launch_bounds__(kThreads, 4) void k_scan_bwd(Scan a) {
  constexpr int P = kBackP;
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
  __shared__ float s_A[2][kW][V * kWave], s_B[2][kW][V * kWave];
  __shared__ Look<V> s_look;
  __shared__ int s_take, s_last;
  const int slice = (int)blockIdx.x % a.slices;
  const int taken = a.spans > 1 ? take(a.taken + slice, &s_take) : 0;
  const int c = a.spans - 1 - taken;
  const int col0 = (slice * kWave + lane) * V;
  const bool in = col0 < a.D;
  const int col = in ? col0 : 0;
  const int q0 = c * kSpan + wave * P;
  const int n = min(P, a.N - q0);
  // fa, fq: a and 1 - a; u: the gradient that reaches the state through y; v: that of the output gate by the state.
  // Then dh at position t is W times the gradient that enters the wavefront's positions plus U; fq and u become
  // (1 - a) W and (1 - a) U, and r = (h before - x) a.
  float A[V], B[V], A2[V], B2[V], state[V], bias[V], W0[V], U0[V];
  float fa[P][V], fq[P][V], u[P][V], v[GATED ? P : 1][V], r[P][V];
  In<T, V> gx[P];
#pragma unroll
  for (int i = 0; i < V; ++i) A[i] = A2[i] = 1.f, B[i] = B2[i] = W0[i] = U0[i] = 0.f;
  {
    In<T, V> gf[P], go[GATED ? P : 1];
    In<TG, V> gy[P];
#pragma unroll
    for (int t = 0; t < P; ++t) {
      const int64_t row = min(q0 + t, a.N - 1);
      gf[t].load(a.f, row, col);
      gx[t].load(a.x, row, col);
      gy[t].load(a.dy, row, col);
      if constexpr (GATED) go[t].load(a.o, row, col);
    }
    load_f32<V>(a.bias, col, bias);
    load_f32<V>(c > 0 ? a.states + (int64_t)c * a.D : nullptr, col, state);
#pragma unroll
    for (int t = 0; t < P; ++t) {
#pragma unroll
      for (int i = 0; i < V; ++i) {
        forget(gf[t].get(i) + bias[i], fa[t][i], fq[t][i]);
        u[t][i] = gy[t].get(i);
        if constexpr (GATED) {
          float rest;
          u[t][i] *= gate(go[t].get(i), rest);
          v[t][i] = u[t][i] * rest;
        }
      }
    }
  }
  const Marks<P> mk(a, min(q0, a.N - 1), lane);
  if (n > 0) {
#pragma unroll
    for (int t = 0; t < P; ++t) {
      if (t >= n) continue;
      if (mk.start(t)) {
        float h0[V];
        load_rare<V>(a.h0 ? a.h0 + (int64_t)mk.of(t) * a.D : nullptr, col, h0);
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
    for (int t = P - 1; t >= 0; --t) {
      if (t >= n) continue;
      if (mk.end(t)) {
        float g[V];
        load_rare<V>(a.dh_last ? a.dh_last + (int64_t)mk.of(t) * a.D : nullptr, col, g);
#pragma unroll
        for (int i = 0; i < V; ++i) B2[i] = g[i];
      }
#pragma unroll
      for (int i = 0; i < V; ++i) {
        A2[i] *= fa[t][i];
        B2[i] = fa[t][i] * (u[t][i] + B2[i]);
      }
    }
#pragma unroll
    for (int i = 0; i < V; ++i) {
      A[i] = mk.starts ? kResets : above_zero(A[i]);
      A2[i] = mk.ends ? kResets : above_zero(A2[i]);
    }
  }
#pragma unroll
  for (int i = 0; i < V; ++i) {
    s_A[0][wave][i * kWave + lane] = A[i];
    s_B[0][wave][i * kWave + lane] = B[i];
    s_A[1][wave][i * kWave + lane] = A2[i];
    s_B[1][wave][i * kWave + lane] = B2[i];
  }
  // whether the span's last position is its sequence's last
  if (wave == kW - 1 && lane == 0) s_last = n <= 0 || mk.end(P - 1);
  __syncthreads();
  const Chain<V> ch(a, slice, taken);
  const bool leads = a.spans > 1 && wave == 0 && c > 0;
  bool resets = false;
  if (leads) {
    // from the span's last wavefront to its first
#pragma unroll
    for (int i = 0; i < V; ++i) A2[i] = s_A[1][kW - 1][i * kWave + lane], B2[i] = s_B[1][kW - 1][i * kWave + lane];
#pragma unroll
    for (int w = kW - 2; w >= 0; --w) {
#pragma unroll
      for (int i = 0; i < V; ++i) {
        const float An = s_A[1][w][i * kWave + lane], Bn = s_B[1][w][i * kWave + lane];
        B2[i] = through(An, Bn, B2[i]);
        A2[i] = join(A2[i], An);
      }
    }
    resets = uniform(A2[0] < 0.f);
    if (resets) ch.publish_out(B2, lane);
    else ch.publish_steps(A2, B2, lane);
  }
  const uint32_t at = (uint32_t)col * (uint32_t)(Vec<TG, V>::kBytes / V);
  if (n > 0) {
    // the states, and what does not need the gradients of later spans, while those publish
    float h[V];
#pragma unroll
    for (int i = 0; i < V; ++i) h[i] = state[i];
    for (int w = 0; w < wave; ++w) {
#pragma unroll
      for (int i = 0; i < V; ++i) h[i] = through(s_A[0][w][i * kWave + lane], s_B[0][w][i * kWave + lane], h[i]);
    }
#pragma unroll
    for (int t = 0; t < P; ++t) {
      if (t < n && mk.start(t)) {
        float h0[V];
        load_rare<V>(a.h0 ? a.h0 + (int64_t)mk.of(t) * a.D : nullptr, col, h0);
#pragma unroll
        for (int i = 0; i < V; ++i) h[i] = h0[i];
      }
      float dO[V];
#pragma unroll
      for (int i = 0; i < V; ++i) {
        const float x = gx[t].get(i);
        r[t][i] = (h[i] - x) * fa[t][i];
        h[i] = __builtin_fmaf(fa[t][i], h[i], fq[t][i] * x);
        if constexpr (GATED) dO[i] = v[t][i] * h[i];
      }
      if constexpr (GATED) {
        if (in && t < n) put<TG, V, STREAM>(a.dO.p + (int64_t)(q0 + t) * a.dO.ld + at, dO);
      }
    }
    float W[V], U[V];
#pragma unroll
    for (int i = 0; i < V; ++i) W[i] = 1.f, U[i] = 0.f;
#pragma unroll
    for (int t = P - 1; t >= 0; --t) {
      if (t >= n) continue;
      if (mk.end(t)) {
        float g[V];
        load_rare<V>(a.dh_last ? a.dh_last + (int64_t)mk.of(t) * a.D : nullptr, col, g);
#pragma unroll
        for (int i = 0; i < V; ++i) U[i] = g[i];
      }
#pragma unroll
      for (int i = 0; i < V; ++i) {
        U[i] += u[t][i];
        u[t][i] = fq[t][i] * U[i];
        fq[t][i] *= W[i];
        U[i] *= fa[t][i];
        W[i] *= fa[t][i];
      }
      if (a.dh0 && mk.start(t)) {
        if (mk.closed(t)) {
          store_f32<V>(a.dh0 + (int64_t)mk.of(t) * a.D + col, in, U);
        } else {
          // (the one sequence that goes on: its gradient is not known yet)
#pragma unroll
          for (int i = 0; i < V; ++i) W0[i] = W[i], U0[i] = U[i];
        }
      }
    }
  }
  float g[V] = {};
  if (a.spans > 1 && !s_last) {
    look_back<V>(ch, s_look, g, wave, lane);
    if (leads && !resets) {
      float leaves[V];
#pragma unroll
      for (int i = 0; i < V; ++i) leaves[i] = through(A2[i], B2[i], g[i]);
      ch.publish_out(leaves, lane);
    }
  }
  float sum[V] = {};
  if (n > 0) {
    for (int w = kW - 1; w > wave; --w) {
#pragma unroll
      for (int i = 0; i < V; ++i) g[i] = through(s_A[1][w][i * kWave + lane], s_B[1][w][i * kWave + lane], g[i]);
    }
    if (any_infinite<V>(g)) {
      above_zero<V>(W0, g);
#pragma unroll
      for (int t = 0; t < P; ++t) above_zero<V>(fq[t], g);
    }
#pragma unroll
    for (int t = P - 1; t >= 0; --t) {
      if (t >= n) continue;
      float dx[V], df[V];
#pragma unroll
      for (int i = 0; i < V; ++i) {
        dx[i] = mk.closed(t) ? u[t][i] : __builtin_fmaf(fq[t][i], g[i], u[t][i]);
        df[i] = dx[i] * r[t][i];
        sum[i] += df[i];
      }
      if (in) {
        const int64_t row = q0 + t;
        put<TG, V, STREAM>(a.dx.p + row * a.dx.ld + at, dx);
        put<TG, V, STREAM>(a.df.p + row * a.df.ld + at, df);
      }
      if (a.dh0 && mk.start(t) && !mk.closed(t)) {
#pragma unroll
        for (int i = 0; i < V; ++i) dx[i] = __builtin_fmaf(W0[i], g[i], U0[i]);
        store_f32<V>(a.dh0 + (int64_t)mk.of(t) * a.D + col, in, dx);
      }
    }
  }
  if (a.dbias) {
    __syncthreads();
#pragma unroll
    for (int i = 0; i < V; ++i) s_A[0][wave][i * kWave + lane] = sum[i];
    __syncthreads();
    if (wave == 0) {
      float t[V] = {};
#pragma unroll
      for (int w = 0; w < kW; ++w) {
#pragma unroll
        for (int i = 0; i < V; ++i) t[i] += s_A[0][w][i * kWave + lane];
      }
      store_f32<V>(a.dbias + (int64_t)c * a.D + col, in, t);
    }
  }
}

// The spans' rows of the bias gradient, added in double: a block takes 16
// columns, 64 rows at a time.
constexpr int kBiasCols = 16, kBiasRows = 64;
__global__ __launch_bounds__(kBiasCols * kBiasRows) void k_scan_dbias(const float* rows, float* dbias, int spans, int D) {
  const int c = threadIdx.x % kBiasCols, r = threadIdx.x / kBiasCols;
  const int col = blockIdx.x * kBiasCols + c;
  __shared__ double s_sum[kBiasRows][kBiasCols];
  double t = 0.;
  if (col < D) {
    constexpr int kAhead = 8;
    for (int k = r; k < spans; k += kBiasRows * kAhead) {
      float x[kAhead];
#pragma unroll
      for (int i = 0; i < kAhead; ++i) {
        const int at = k + i * kBiasRows;
        x[i] = at < spans ? rows[(int64_t)at * D + col] : 0.f;
      }
#pragma unroll
      for (int i = 0; i < kAhead; ++i) t += (double)x[i];
    }
  }
  s_sum[r][c] = t;
  for (int half = kBiasRows / 2; half > 0; half /= 2) {
    __syncthreads();
    if (r < half) s_sum[r][c] += s_sum[r + half][c];
  }
  if (r == 0 && col < D) dbias[col] = (float)s_sum[0][c];
}

// Zeros for the chain's counters and flags: 1.3 us, 5 after a kernel that filled
// the device.
__global__ __launch_bounds__(256) void k_scan_clear(uint32_t* words, int64_t n) {
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (int64_t)gridDim.x * 256) words[i] = 0u;
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

// A lane to each column (or two) of a token: one read of every input, one read
// and write of the state.  128 tokens x 1536: 3.3 us, a launch and two dependent
// loads (the bytes take 0.6).
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

// The workspace: header, counters and flags, steps, outgoing states, rows of the bias
// gradient; for spans of 64 (the backward's; the forward's are fewer).
struct Room {
  int64_t spans, slices, cols;
  size_t flags, steps, out, dbias, total;
};
Room room(int64_t N, int32_t D) {
  Room r{};
  r.spans = (N + kSpan - 1) / kSpan;
  r.slices = ((int64_t)D + kWave - 1) / kWave;
  r.cols = ((int64_t)D + 2 * kWave - 1) / (2 * kWave) * (2 * kWave);
  size_t at = sizeof(WsHeader);
  r.flags = at;
  at = align256(at + sizeof(uint32_t) * (size_t)(r.slices * (r.spans + 1)));
  r.steps = at;
  at = align256(at + sizeof(uint64_t) * (size_t)(r.spans * r.cols));
  r.out = at;
  at = align256(at + sizeof(uint32_t) * (size_t)(r.spans * r.cols));
  r.dbias = at;
  r.total = align256(at + sizeof(float) * (size_t)r.spans * (size_t)D);
  return r;
}

Scan arguments(const ScanLaunch& p, int V, int span) {
  Scan a{};
  a.offsets = p.offsets;
  a.x = p.x, a.f = p.f, a.o = p.o, a.y = p.y;
  a.dy = p.dy, a.dx = p.dx, a.df = p.df, a.dO = p.dO;
  a.bias = p.bias, a.h0 = p.h0, a.h_last = p.h_last;
  a.states = p.states, a.dh_last = p.dh_last, a.dh0 = p.dh0;
  a.N = (int32_t)p.N, a.M = p.M, a.D = p.D;
  a.spans = (int32_t)((p.N + span - 1) / span);
  a.slices = (p.D + kWave * V - 1) / (kWave * V);
  const Room r = room(p.N, p.D);
  a.hdr = reinterpret_cast<WsHeader*>(p.ws);
  a.taken = reinterpret_cast<uint32_t*>(p.ws + r.flags);
  a.flags = a.taken + a.slices;
  a.steps = reinterpret_cast<uint64_t*>(p.ws + r.steps);
  a.out = reinterpret_cast<uint32_t*>(p.ws + r.out);
  a.dbias = p.dbias ? reinterpret_cast<float*>(p.ws + r.dbias) : nullptr;
  return a;
}
unsigned empties(const Scan& a, const float* out) { return out ? (unsigned)(a.M + kWave - 1) / kWave : 0u; }
void clear(const Scan& a, hipStream_t s) {
  const int64_t n = (int64_t)a.slices * (a.spans + 1), blocks = (n + 255) / 256;
  if (a.spans > 1) k_scan_clear<<<(unsigned)(blocks < 256 ? blocks : 256), 256, 0, s>>>(a.taken, n);
}

template <typename T, int V, int P, bool STREAM>
hipError_t fwd(const ScanLaunch& p, const Scan& a, hipStream_t s) {
  const unsigned blocks = (unsigned)(a.spans * a.slices) + empties(a, a.h_last);
  if (!launchable(blocks, kThreads)) return hipErrorNotSupported;
  clear(a, s);
  if (p.gated) k_scan_fwd<T, V, P, true, STREAM><<<blocks, kThreads, 0, s>>>(a);
  else k_scan_fwd<T, V, P, false, STREAM><<<blocks, kThreads, 0, s>>>(a);
  return hipGetLastError();
}
template <typename T, int V>
hipError_t fwd(const ScanLaunch& p, hipStream_t s) {
  const Scan a = arguments(p, V, kFwdP * kW);
  if (p.N * p.D * (int64_t)(Vec<T, V>::kBytes / V) > kStreamBytes) return fwd<T, V, kFwdP, true>(p, a, s);
  // (us, the shorter spans against the longer ones: 500 x 2000 11.5 and 13.1, 1500 x 512 11.9 and 13.1, 8000 x 100 12.8
  // and 13.9; 128 blocks of the longer ones as fast; 192, 1500 x 2000, 18.2 and 16.0; one span 7.1 and 6.4)
  if (a.spans > 1 && a.spans * a.slices <= kFwdFewBlocks)
    return fwd<T, V, kFwdFewP, false>(p, arguments(p, V, kFwdFewP * kW), s);
  return fwd<T, V, kFwdP, false>(p, a, s);
}

template <typename T, typename TG, int V, bool STREAM>
hipError_t bwd(const ScanLaunch& p, hipStream_t s) {
  Scan a = arguments(p, V, kSpan);
  if (a.spans == 1) a.dbias = p.dbias;  // (its one row is the sum)
  const unsigned blocks = (unsigned)(a.spans * a.slices) + empties(a, a.dh0);
  if (!launchable(blocks, kThreads)) return hipErrorNotSupported;
  clear(a, s);
  if (p.gated) k_scan_bwd<T, TG, V, true, STREAM><<<blocks, kThreads, 0, s>>>(a);
  else k_scan_bwd<T, TG, V, false, STREAM><<<blocks, kThreads, 0, s>>>(a);
  if (p.dbias && a.spans > 1)
    k_scan_dbias<<<(unsigned)((a.D + kBiasCols - 1) / kBiasCols), kBiasCols * kBiasRows, 0, s>>>(a.dbias, p.dbias, a.spans,
                                                                                             a.D);
  return hipGetLastError();
}
template <typename T, typename TG, int V>
hipError_t bwd(const ScanLaunch& p, hipStream_t s) {
  const bool big = p.N * p.D * (int64_t)(Vec<TG, V>::kBytes / V) > kStreamBytes;
  return big ? bwd<T, TG, V, true>(p, s) : bwd<T, TG, V, false>(p, s);
}

template <typename T, int V>
hipError_t step(const StepLaunch& p, hipStream_t s) {
  const int64_t per = (p.D + V - 1) / V, blocks = (p.N * per + 255) / 256;
  if (!launchable(blocks, 256)) return hipErrorNotSupported;
  if (p.gated) k_scan_step<T, V, true><<<(unsigned)blocks, 256, 0, s>>>(p);
  else k_scan_step<T, V, false><<<(unsigned)blocks, 256, 0, s>>>(p);
  return hipGetLastError();
}

}  // namespace

size_t scan_ws_bytes(int64_t N, int32_t D) { return room(N > 0 ? N : 1, D).total; }

hipError_t launch_scan_fwd(const ScanLaunch& p, hipStream_t s) {
  if (p.N == 0) {
    nothing(p.h0, p.h_last, (int64_t)p.M * p.D, s);
    return hipGetLastError();
  }
  if (p.dtype == EMB_FP32) return fwd<float, 1>(p, s);
  return p.vector == 2 ? fwd<bf16, 2>(p, s) : fwd<bf16, 1>(p, s);
}

hipError_t launch_scan_bwd(const ScanLaunch& p, hipStream_t s) {
  if (p.N == 0) {
    nothing(p.dh_last, p.dh0, (int64_t)p.M * p.D, s);
    nothing(nullptr, p.dbias, p.D, s);
    return hipGetLastError();
  }
  if (p.dtype == EMB_FP32) return bwd<float, float, 1>(p, s);
  if (p.dtype == EMB_BF16) return p.vector == 2 ? bwd<bf16, bf16, 2>(p, s) : bwd<bf16, bf16, 1>(p, s);
  if (p.grad_dtype == EMB_FP32) return bwd<Saved8, float, 1>(p, s);
  return p.vector == 2 ? bwd<Saved8, bf16, 2>(p, s) : bwd<Saved8, bf16, 1>(p, s);
}

hipError_t launch_scan_step(const StepLaunch& p, hipStream_t s) {
  if (p.dtype == EMB_FP32) return step<float, 1>(p, s);
  return p.vector == 2 ? step<bf16, 2>(p, s) : step<bf16, 1>(p, s);
}

}  // namespace emb
