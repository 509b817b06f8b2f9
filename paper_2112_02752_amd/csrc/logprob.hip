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
// (above 25600 vectors of 16 bytes), and gradients that lie otherwise than their
// logits, are read twice.
//
// Bound.  8192 x 50000 bf16 with its gradient: 348 us, 1.64 GB at 4.7 TB/s.  301 x 100001
// fp32: forward 28 us (4.3 TB/s), gradient from the statistics 38 (6.5 TB/s).  64 x 50000
// with 8 alternatives, a row a compute unit: 10.4 us, of which the exponentials
// and sums of 50000 values by one compute unit take about 3, their loads as long.
#include <float.h>

#include "block_common.h"

namespace emb {

namespace {

constexpr float kLog2e = 1.44269504088896340736f;
constexpr float kLowest = -1024.f;  // in place of lower powers where what they are multiplied with is zero
constexpr float kLn2 = 0.69314718055994530942f;

// A row of D values: whole vectors of 16 bytes where it lies on them, and before the first and after the last of them a
// few values (less than a vector), which the first 16 lanes take one each.
template <typename T>
struct Row {
  static constexpr int kSize = Vec<T, 1>::kBytes, kEach = 16 / kSize;
  typedef Vec<T, kEach> V;
  const char* p;  // of the first whole vector
  int cols, lead, count;  // columns before it, whole vectors
  __device__ __forceinline__ Row(const char* at, int D) {
    cols = D;
    lead = min((int)(-(intptr_t)at & 15) / kSize, D);
    count = (D - lead) / kEach;
    p = at + lead * kSize;
  }
  __device__ __forceinline__ int column(int v) const { return lead + v * kEach; }
  // minus infinity where there is no vector
  __device__ __forceinline__ V load(int v) const {
    V x;
    if (v < count) {
      x.load(p + (int64_t)v * 16);
    } else {
      constexpr uint32_t kNone = kSize == 2 ? 0xff80ff80u : 0xff800000u;
      const u32x4 none = {kNone, kNone, kNone, kNone};
      x.load(&none);
    }
    return x;
  }
  // the column of its own that lane t of those that share the row takes, or -1
  __device__ __forceinline__ int edge(int t) const {
    if (t < 8) return t < lead ? t : -1;
    const int c = column(count) + t - 8;
    return t < 16 && c < cols ? c : -1;
  }
  __device__ __forceinline__ const char* at(int c) const { return p + (int64_t)(c - lead) * kSize; }
  __device__ __forceinline__ float value(int c) const {
    Vec<T, 1> one;
    one.load(at(c));
    return one.get(0);
  }
};

// Order of the alternatives: greater values first (NaN before all, both zeros alike), then lower columns.  No key is all
// ones or zero, the limit of a first search and what finds nothing.
__device__ __forceinline__ uint64_t order_key(float x, int col) {
  uint32_t u = __float_as_uint(x + 0.f);
  if (x != x) u = 0x7fc00000u;
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

// Exponents are taken to the base of two: with t = scale log2(e) a value's power is (x - m) t, m being the largest value.
// The difference is formed first: t x - t m by one operation has the rounding of t m as its error, which for masks of
// large finite numbers is more than exponents are (some hundreds at 1e10), and a part of a row may hold nothing else.
// Sums of a part of a row, relative to its own m:
struct Sums {
  float m, s, a;  // m, sum of 2^((x - m) t), sum of 2^((x - m) t) (x - m) t
};
// the part's m from its largest value: where no token can be, every difference would be NaN
__device__ __forceinline__ float reference(float top) { return top == -INFINITY ? 0.f : top; }
// (a power of zero where x is m, whatever the scale)
__device__ __forceinline__ float base2(float scale) { return fminf(scale * kLog2e, FLT_MAX); }
// x's power, and its share of the sums
__device__ __forceinline__ void add_value(float x, float t, Sums& p) {
  const float z = (x - p.m) * t, e = __builtin_amdgcn_exp2f(z);
  p.s += e;
  p.a = __builtin_fmaf(e, fmaxf(z, kLowest), p.a);
}
__device__ __forceinline__ void refer_to(float m, float t, Sums& p) {
  const float by = (p.m - m) * t, f = __builtin_amdgcn_exp2f(by);
  p.a = f * __builtin_fmaf(p.s, fmaxf(by, kLowest), p.a);
  p.s *= f;
  p.m = m;
}

// What a row's gradient is made of: dx_v = e_v (all + slope (x_v - m) t), and at the id's column `hot` more
struct Slope {
  float t, m, all, slope, hot;
  int64_t id;
  __device__ __forceinline__ Slope(const LogpLaunch& a, int64_t row, float t_, float m_, float s, float entropy) {
    id = id_of(a, row);
    t = t_;
    m = m_;
    // (where no token can be, every e is zero)
    const float inv = s == 0.f ? 0.f : a.scale / s;
    const float dl = id >= 0 && id < a.D && s != 0.f && a.dlogp != nullptr ? a.dlogp[row] : 0.f;
    const float dh = a.dentropy != nullptr && s != 0.f ? a.dentropy[row] : 0.f;
    slope = -inv * dh * kLn2;
    all = dh != 0.f ? inv * (-dl - dh * (entropy - logf(s))) : -inv * dl;
    hot = a.scale * dl;
  }
  template <bool ENTROPY>
  __device__ __forceinline__ float value(float x) const {
    const float z = (x - m) * t, e = __builtin_amdgcn_exp2f(z);
    if constexpr (ENTROPY) return e * __builtin_fmaf(slope, fmaxf(z, kLowest), all);
    return e * all;
  }
};

// The gradient at lane t's own column
template <bool ENTROPY, typename T>
__device__ __forceinline__ void put_edge(const Row<T>& r, const Slope& d, float x, int c, char* to) {
  if (c < 0) return;
  const float one[1] = {d.template value<ENTROPY>(x) + (c == d.id ? d.hot : 0.f)};
  Vec<T, 1>::store(to + (int64_t)c * Row<T>::kSize, one);
}
// A vector's gradient; SAME: dlogits lies in vectors as the logits do
template <bool ENTROPY, bool STREAM, bool SAME, typename T>
__device__ __forceinline__ void put_grad(const Row<T>& r, const Slope& d, const typename Row<T>::V& x, int v, char* to) {
  constexpr int E = Row<T>::kEach;
  if (v >= r.count) return;
  float g[E];
#pragma unroll
  for (int k = 0; k < E; ++k) g[k] = d.template value<ENTROPY>(x.get(k));
  const int64_t mine = d.id - r.column(v);
  if (mine >= 0 && mine < E) {
#pragma unroll
    for (int k = 0; k < E; ++k) g[k] += k == (int)mine ? d.hot : 0.f;
  }
  char* p = to + (int64_t)r.column(v) * Row<T>::kSize;
  if constexpr (SAME) {
    if constexpr (STREAM) Vec<T, E>::stream(p, g);
    else Vec<T, E>::store(p, g);
  } else {
    Vec<T, E>::store_each(p, g);
  }
}

// W wavefronts a row, R vectors a lane in registers (0: none, the row is read again, and dlogits may lie otherwise).
template <int W>
constexpr int kBlock = W <= 4 ? 256 : 64 * W;
constexpr int kCandidates = 512;  // of a block, for the alternatives

template <typename T, int W, int R, bool GRAD, bool STREAM>
__global__ __launch_bounds__(kBlock<W>, R <= 8 ? 8 : 4) void k_logp(LogpLaunch a) {
  constexpr int kTeam = 64 * W, kRows = kBlock<W> / kTeam, E = Row<T>::kEach, kMost = kCandidates / kRows;
  typedef typename Row<T>::V V;
  __shared__ float s_part[3][kBlock<W> / kWave];
  __shared__ uint64_t s_list[GRAD ? 1 : kRows][GRAD ? 1 : kMost];
  __shared__ int s_count[kRows], s_before[kWave];
  __shared__ float s_group[kWave];
  const int lane = threadIdx.x % kWave, wave = uniform(threadIdx.x / kWave), t = threadIdx.x % kTeam;
  const int64_t row = (int64_t)blockIdx.x * kRows + wave / W;
  if (row >= a.N) return;  // (W > 1: a row a block)
  if (!GRAD && t < kWave) {
    if (W > 1) s_before[t] = 0;
    if (t == 0) s_count[wave / W] = 0;
  }
  const Row<T> r(a.logits.p + row * a.logits.ld, a.D);
  const float t2 = base2(a.scale);
  V x[R > 0 ? R : 1];
  if constexpr (R > 0) {
#pragma unroll
    for (int i = 0; i < R; ++i) x[i] = r.load(t + i * kTeam);
  }
  const int own = r.edge(t);
  const float own_x = own >= 0 ? r.value(own) : -INFINITY;
  // every vector of the row; values are taken apart anew by each use (kept, they would take twice the registers)
  auto each = [&](auto f) {
    if constexpr (R > 0) {
#pragma unroll
      for (int i = 0; i < R; ++i) {
        if constexpr (Row<T>::kSize == 2) asm volatile("" : "+v"(x[i].w[0]), "+v"(x[i].w[1]), "+v"(x[i].w[2]), "+v"(x[i].w[3]));
        f(x[i], t + i * kTeam);
      }
    } else {
      for (int v = t; v < r.count; v += kTeam) f(r.load(v), v);
    }
  };
  float mine = own_x, most;  // largest of the lane's, of the wavefront's
  Sums p{0.f, 0.f, 0.f};
  if constexpr (R > 0) {
    each([&](const V& v, int) {
#pragma unroll
      for (int k = 0; k < E; ++k) mine = fmaxf(mine, v.get(k));
    });
    most = wave_max(mine);
    p.m = reference(most);
    each([&](const V& v, int) {
#pragma unroll
      for (int k = 0; k < E; ++k) add_value(v.get(k), t2, p);
    });
    add_value(own_x, t2, p);
  } else {
    // one reading: the lane's sums follow its largest value
    p.m = reference(mine);
    add_value(own_x, t2, p);
    each([&](const V& v, int) {
      float top = mine;
#pragma unroll
      for (int k = 0; k < E; ++k) top = fmaxf(top, v.get(k));
      if (top > mine) {
        const float m = reference(top);
        if (mine == -INFINITY) p.m = m;
        else refer_to(m, t2, p);
        mine = top;
      }
#pragma unroll
      for (int k = 0; k < E; ++k) add_value(v.get(k), t2, p);
    });
    most = wave_max(mine);
    if (mine != -INFINITY) refer_to(reference(most), t2, p);
    p.m = reference(most);
  }
  p.s = wave_sum(p.s);
  p.a = wave_sum(p.a);
  float top = most;
  if constexpr (W > 1) {
    if (lane == 0) s_part[0][wave] = most, s_part[1][wave] = p.s, s_part[2][wave] = p.a;
    __syncthreads();
    // a lane takes a wavefront's sums (where no token can be they are zero, or NaN)
    const float part = lane < W ? s_part[0][lane] : -INFINITY;
    Sums o{reference(part), lane < W ? s_part[1][lane] : 0.f, lane < W ? s_part[2][lane] : 0.f};
    top = wave_max(part);
    p.m = reference(top);
    if (part != -INFINITY) refer_to(p.m, t2, o);
    p.s = wave_sum(o.s);
    p.a = wave_sum(o.a);
  }
  const float log_sum = logf(p.s), entropy = p.s == 0.f ? 0.f : log_sum - kLn2 * (p.a / p.s);
  auto log_prob = [&](float v) {
    return p.s == 0.f ? -INFINITY : (v - p.m) * a.scale - log_sum;
  };
  if (t == 0) {
    const int64_t id = id_of(a, row);
    if (a.logp != nullptr) a.logp[row] = id >= 0 && id < a.D ? log_prob(r.value((int)id)) : 0.f;
    if (a.entropy != nullptr) a.entropy[row] = entropy;
    if (a.stats != nullptr) Vec<float, 4>::store(a.stats + row * kStats, {p.m, p.s, entropy, 0.f});
  }
  if constexpr (GRAD) {
    // in place: the id's logit is read before it is overwritten
    if constexpr (W > 1) {
      if (a.dlogits.p == a.logits.p) __syncthreads();
    } else {
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    }
    const Slope d(a, row, t2, p.m, p.s, entropy);
    char* to = a.dlogits.p + row * a.dlogits.ld;
    each([&](const V& v, int at) { put_grad<false, STREAM, (R > 0)>(r, d, v, at, to); });
    put_edge<false>(r, d, own_x, own, to);
    return;
  }
  if (a.top == 0) return;
  // The alternatives.  The row's lanes are 64 groups, each with its largest value; the `top`-th of those is a
  // bound that at least `top` logits reach (and few more do), so only those that reach it are looked at.  64
  // x 50000 bf16: 7.6 us without alternatives, 10.4 with 8 and 11.4 with 20; when every wavefront found its
  // lanes' `top` largest one by one 13.4 and 20.9.
  static_assert(EMB_MAX_TOP <= 64, "a group for each");
  const int mate = wave / W;
  float bound = mine;
  if constexpr (W >= 4) {
    bound = fmaxf(bound, lane_move<0xb1>(bound));  // groups of four lanes
    bound = fmaxf(bound, lane_move<0x4e>(bound));
  }
  if constexpr (W == 16) {
    bound = fmaxf(bound, lane_move<0x141>(bound));  // of sixteen
    bound = fmaxf(bound, lane_move<0x140>(bound));
  }
  static_assert(W == 1 || W == 4 || W == 16, "64 groups of W lanes");
  // A group's place: the greater ones and, of those alike, the ones before it; each wavefront counts a W-th of them.
  if constexpr (W > 1) {
    if (t % W == 0) s_group[t / W] = bound;
    __syncthreads();
    bound = s_group[lane];
    int before = 0;
#pragma unroll
    for (int i = 0; i < kWave / W; ++i) {
      const int j = wave * (kWave / W) + i;
      const float other = lane_at(bound, j);
      before += other > bound || (other == bound && j < lane);
    }
    atomicAdd(&s_before[lane], before);
    __syncthreads();
    const uint64_t at = __ballot(s_before[lane] == a.top - 1);
    bound = lane_at(bound, __ffsll((unsigned long long)at) - 1);
  } else {
    int before = 0;
#pragma unroll 8
    for (int j = 0; j < kWave; ++j) {
      const float other = lane_at(bound, j);
      before += other > bound || (other == bound && j < lane);
    }
    const uint64_t at = __ballot(before == a.top - 1);
    bound = lane_at(bound, __ffsll((unsigned long long)at) - 1);
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  }
  // (with NaN in the row every logit is looked at)
  if (p.s != p.s) bound = NAN;
  auto look = [&](float v, int c) {
    if (v < bound) return;
    const int i = atomicAdd(&s_count[mate], 1);
    if (i < kMost) s_list[mate][i] = order_key(v, c);
  };
  if (!(mine < bound)) {
    each([&](const V& v, int at) {
      float best = v.get(0);
#pragma unroll
      for (int k = 1; k < E; ++k) best = fmaxf(best, v.get(k));
      if (best < bound || at >= r.count) return;
#pragma unroll
      for (int k = 0; k < E; ++k) look(v.get(k), r.column(at) + k);
    });
    if (own >= 0) look(own_x, own);
  }
  auto put = [&](int i, uint64_t key) {
    a.top_ids[row * a.top + i] = (int32_t)~(uint32_t)key;
    a.top_logp[row * a.top + i] = log_prob(key_value(key));
  };
  if constexpr (W > 1) __syncthreads();
  else __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  const int count = s_count[mate];
  if (count <= kMost) {
    // a key's place is the number of greater ones (no two are the same)
    for (int i = t; i < count; i += kTeam) {
      const uint64_t key = s_list[mate][i];
      int before = 0;
#pragma unroll 4
      for (int j = 0; j < count; ++j) before += s_list[mate][j] > key;
      if (before < a.top) put(before, key);
    }
    return;
  }
  // Too many reach it (ties, tokens that cannot be, NaN): every wavefront's best one after another; a lane
  // looks through its columns again, in memory, when its best has been taken.  Then the wavefronts' lists are
  // merged.  (The lists lie over the row's own candidates: other rows of the block are not waited for.)
  if constexpr (W > 1) __syncthreads();
  uint64_t* const list = s_list[mate] + wave % W * EMB_MAX_TOP;
  static_assert(W * EMB_MAX_TOP <= kMost, "a list for every wavefront of a row");
  auto best_below = [&](uint64_t limit) {
    uint64_t best = 0;
    if (own >= 0) {
      const uint64_t key = order_key(own_x, own);
      if (key < limit) best = key;
    }
#pragma unroll 1
    for (int v = t; v < r.count; v += kTeam) {
      const V w = r.load(v);
#pragma unroll
      for (int k = 0; k < E; ++k) {
        const uint64_t key = order_key(w.get(k), r.column(v) + k);
        if (key < limit && key > best) best = key;
      }
    }
    return best;
  };
  uint64_t next = best_below(~0ull);
  for (int i = 0; i < a.top; ++i) {
    const uint64_t best = wave_max_key(next);  // (0: no column is left)
    if (lane == 0) list[i] = best;
    if (best != 0 && next == best) next = best_below(best);
  }
  if constexpr (W > 1) {
    __syncthreads();
    if (wave > 0) return;
    int taken = 0;
    next = lane < W ? s_list[mate][lane * EMB_MAX_TOP] : 0;
    for (int i = 0; i < a.top; ++i) {
      const uint64_t best = wave_max_key(next);
      if (lane == 0) put(i, best);
      if (next == best && lane < W) {
        ++taken;
        next = taken < a.top ? s_list[mate][lane * EMB_MAX_TOP + taken] : 0;
      }
    }
  } else {
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    if (lane < a.top) put(lane, list[lane]);
  }
}

// The gradient from the forward's statistics: each row's vectors by blocks.
constexpr int kGradVecs = 4;
template <typename T, bool ENTROPY, bool STREAM, bool SAME>
__global__ __launch_bounds__(256) void k_logp_bwd(LogpLaunch a, int per) {
  const int64_t row = blockIdx.x / per;
  const int part = (int)(blockIdx.x % per);
  const Row<T> r(a.logits.p + row * a.logits.ld, a.D);
  typename Row<T>::V x[kGradVecs];
  const int at = part * 256 * kGradVecs + threadIdx.x;
#pragma unroll
  for (int i = 0; i < kGradVecs; ++i) x[i] = r.load(at + i * 256);
  const int own = part == 0 ? r.edge(threadIdx.x) : -1;
  const float own_x = own >= 0 ? r.value(own) : 0.f;
  const float* st = a.stats + row * kStats;
  const Slope d(a, row, base2(a.scale), st[0], st[1], st[2]);
  char* to = a.dlogits.p + row * a.dlogits.ld;
#pragma unroll
  for (int i = 0; i < kGradVecs; ++i) put_grad<ENTROPY, STREAM, SAME>(r, d, x[i], at + i * 256, to);
  put_edge<ENTROPY>(r, d, own_x, own, to);
}

// whether every row of the gradient lies as the logits' does
bool alike(const LogpLaunch& p) {
  return p.dlogits.p == nullptr || ((((uintptr_t)p.dlogits.p ^ (uintptr_t)p.logits.p) & 15u) == 0 &&
                                    ((p.dlogits.ld ^ p.logits.ld) & 15) == 0);
}
// gradients that the L2 caches do not hold are stored past them
bool streams(const LogpLaunch& p) {
  return p.N * (int64_t)p.D * (p.dtype == EMB_FP32 ? 4 : 2) > kStreamBytes;
}

template <typename T, int W, int R>
hipError_t go(const LogpLaunch& p, hipStream_t s) {
  constexpr int kRows = kBlock<W> / (64 * W);
  const int64_t blocks = (p.N + kRows - 1) / kRows;
  if (!launchable(blocks, kBlock<W>)) return hipErrorNotSupported;
  if (p.dlogits.p == nullptr) k_logp<T, W, R, false, false><<<(unsigned)blocks, kBlock<W>, 0, s>>>(p);
  else if (streams(p)) k_logp<T, W, R, true, true><<<(unsigned)blocks, kBlock<W>, 0, s>>>(p);
  else k_logp<T, W, R, true, false><<<(unsigned)blocks, kBlock<W>, 0, s>>>(p);
  return hipGetLastError();
}

// The fewest wavefronts and registers that hold a row.  Forward / with gradient in us, bf16, the variant that is taken
// and the next one on the same rows: 100 vectors (16384 rows) 10/17 and 21/28; 400 (16384) 32/46 and 77/89; 2040 (8224)
// 64/96 and 98/122; 4000 (4194) 63/92 and 91/115; 8000 (2097) 62/90 and 117/153; 16000 (1048) 84/129 and 104/157;
// 25500 (657) 77/131 and, without registers, 49/164.  (What reads a row once is faster without registers from 4000
// vectors on: 16000, 50 us.  With the row in 20 or 24 vectors a lane instead of 25: 20000 (838) 84/129 and 90/141 for
// 91/145.)
template <typename T>
hipError_t by_width(const LogpLaunch& p, hipStream_t s) {
  const int64_t n = p.D / Row<T>::kEach;  // whole vectors, at most
  if (!alike(p)) return n <= 512 ? go<T, 1, 0>(p, s) : go<T, 16, 0>(p, s);
  if (n <= 64 * 2) return go<T, 1, 2>(p, s);
  if (n <= 64 * 8) return go<T, 1, 8>(p, s);
  if (n <= 256 * 8) return go<T, 4, 8>(p, s);
  if (n <= 1024 * 4) return go<T, 16, 4>(p, s);
  if (n <= 1024 * 8) return go<T, 16, 8>(p, s);
  if (n <= 1024 * 16) return go<T, 16, 16>(p, s);
  if (n <= 1024 * 25) return go<T, 16, 25>(p, s);
  return go<T, 16, 0>(p, s);
}

template <typename T>
hipError_t back(const LogpLaunch& p, hipStream_t s) {
  const int64_t n = p.D / Row<T>::kEach, per = n > 0 ? (n + 256 * kGradVecs - 1) / (256 * kGradVecs) : 1;
  if (!launchable(per * p.N, 256)) return hipErrorNotSupported;
  const unsigned blocks = (unsigned)(per * p.N);
  const bool past = streams(p);
  auto go = [&](auto entropy) {
    constexpr bool H = decltype(entropy)::value;
    if (!alike(p)) k_logp_bwd<T, H, false, false><<<blocks, 256, 0, s>>>(p, (int)per);
    else if (past) k_logp_bwd<T, H, true, true><<<blocks, 256, 0, s>>>(p, (int)per);
    else k_logp_bwd<T, H, false, true><<<blocks, 256, 0, s>>>(p, (int)per);
  };
  if (p.dentropy == nullptr) go(std::false_type{});
  else go(std::true_type{});
  return hipGetLastError();
}

}  // namespace

hipError_t launch_logp(const LogpLaunch& p, hipStream_t s) {
  return p.dtype == EMB_FP32 ? by_width<float>(p, s) : by_width<bf16>(p, s);
}

hipError_t launch_logp_bwd(const LogpLaunch& p, hipStream_t s) {
  return p.dtype == EMB_FP32 ? back<float>(p, s) : back<bf16>(p, s);
}

}  // namespace emb
