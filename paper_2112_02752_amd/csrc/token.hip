// Lookup of single tokens and its gradient by sorted tokens (gfx950).
//
//   out[j] = scale * W[key(j)]                       (padding tokens: zeros)
//   g_u    = scale * sum over sorted positions k of segment u of dy[perm[k]]
//
// Forward: a row is read by G lanes (a power of two, at most a block) as
// vectors of V values; a lane has one or two rows in flight.  Bound by bytes
// where they are many: 65536 tokens of 2048 bf16 values 54 us, 7.3 TB/s of rows
// missed by the L2s and rows written past them; 64 tokens of 1024: 2.6 us, a
// launch and two dependent loads.
//
// Gradient: a wavefront walks the 64 sorted positions of one chunk for 64 * EL
// columns, in batches whose rows (and the table rows of the segments that end
// in the batch) are in flight together.  What is walked is the same for the
// whole wavefront, so rows and segment ends live in scalar registers.  A
// segment of at most 64 positions belongs to the chunk it starts in; a longer
// one leaves a partial row per chunk, which k_token_combine adds up.  Every
// sum runs in a fixed order: results are the same from run to run.  Few
// positions get a wavefront each.  32768 tokens x 1024 (bf16 in, every row of a
// table of 50000 out): 48 us, 5.7 TB/s, most of it the table's 205 MB; the combine
// 6 us.  2000 tokens x 64 by row-wise Adagrad: 7 + 4 us, chains of dependent loads.
#include "reduce_common.h"
#include "seq_common.h"

namespace emb {

namespace {

// ---------------------------------------------------------------- forward

constexpr int kFwdThreads = 256;

struct TokFwd {
  const char* W;
  const void* idx;
  const int32_t* offsets;
  char* out;
  int64_t N, row_bytes, out_bytes;  // bytes from one row to the next
  int32_t idx64, T, B, vectors, log_g, aligned;
  uint32_t rows, pad;
  float scale;
};
// (a kernel of one table does not get the table offsets)
template <bool MANY>
struct Stacked {};
template <>
struct Stacked<true> {
  TableOffsets ro;
};

// Id j in two halves, or one of 32 bits and its sign: an id whose upper half is not zero lies outside every table.
struct Id {
  uint32_t lo, hi;
};
__device__ __forceinline__ Id load_whole_id(const void* idx, int32_t idx64, int64_t j) {
  // (two loads and no branch, behind which they would be waited for before the table is searched: 65536 tokens of 1024
  // over ten tables 41.2 us, 43.5 with one)
  const uint32_t* p = static_cast<const uint32_t*>(idx) + (idx64 ? 2 * j : j);
  const uint32_t lo = p[0], hi = p[idx64 ? 1 : 0];
  return Id{lo, idx64 ? hi : (uint32_t)((int32_t)lo >> 31)};
}

template <typename TW, typename TO, int V, int AHEAD, bool STREAM, bool MANY>
__global__ __launch_bounds__(kFwdThreads) void k_token_fwd(TokFwd a, Stacked<MANY> st) {
  const int lanes = 1 << a.log_g, per = kFwdThreads >> a.log_g;
  const int c = (int)blockIdx.y * lanes + (int)(threadIdx.x & (lanes - 1));
  const int64_t j0 = (int64_t)blockIdx.x * (per * AHEAD) + (threadIdx.x >> a.log_g);
  if (c >= a.vectors) return;
  uint32_t key[AHEAD];
#pragma unroll
  for (int u = 0; u < AHEAD; ++u) {
    const int64_t j = j0 + (int64_t)u * per;
    key[u] = kNoRow;
    if (j < a.N) {
      const Id id = load_whole_id(a.idx, a.idx64, j);
      if constexpr (MANY) {
        // the table whose sequences hold position j: the last with a first position at or before it
        int t = 0, n = a.T;
        while (n > 1) {
          const int half = n / 2;
          if ((int64_t)a.offsets[(int64_t)(t + half) * a.B] <= j) t += half, n -= half;
          else n = half;
        }
        const uint32_t r0 = st.ro.off[t];
        key[u] = id.hi == 0u && id.lo < st.ro.off[t + 1] - r0 ? r0 + id.lo : kNoRow;
      } else {
        key[u] = id.hi == 0u ? id.lo : kNoRow;
      }
      if (key[u] == a.pad) key[u] = kNoRow;
    }
  }
  Vec<TW, V> v[AHEAD];
#pragma unroll
  for (int u = 0; u < AHEAD; ++u) {
    if (key[u] < a.rows) v[u].load(a.W + (int64_t)key[u] * a.row_bytes + (int64_t)c * Vec<TW, V>::kBytes);
    else v[u].zero();
  }
#pragma unroll
  for (int u = 0; u < AHEAD; ++u) {
    const int64_t j = j0 + (int64_t)u * per;
    if (j >= a.N) break;
    float x[V];
#pragma unroll
    for (int i = 0; i < V; ++i) x[i] = key[u] < a.rows ? a.scale * v[u].get(i) : 0.f;
    char* q = a.out + j * a.out_bytes + (int64_t)c * Vec<TO, V>::kBytes;
    if (!a.aligned) Vec<TO, V>::store_each(q, x);
    else if constexpr (STREAM) Vec<TO, V>::stream(q, x);
    else Vec<TO, V>::store(q, x);
  }
}

// ---------------------------------------------------------------- gradient

// what becomes of a gradient row: stored (past the caches: kStream), or applied
enum Kind { kStore, kStream, kSgd, kAdaRow, kAdaElem };
constexpr bool stores(int kind) { return kind == kStore || kind == kStream; }
constexpr int kMostSplit = 4, kSplitWaves = 8192, kZeroWaves = 1024;
constexpr int kMostParts = 16;  // wavefronts of a block that share a chunk's columns (row-wise Adagrad)

struct TokGrad {
  const char* dy;
  int64_t ld;  // bytes from one row to the next
  const int32_t* perm;
  const int32_t* seg;
  const uint32_t* ukeys;
  const int32_t* num_unique;
  const int32_t* chunk_seg;
  const void* hdr;
  float* partials;  // [nchunks][2][D]: rows of long segments, of the one that holds a chunk's first position, of another
  float* grad;
  int32_t N, D, nchunks, parts, split, blocks, zero_blocks, zero_rows, layout, aligned;  // split: 2^split wavefronts share a chunk's columns
  uint32_t rows, pad;
  float scale;
  Upd up;
};

__device__ __forceinline__ bool failed(const TokGrad& a) {
  const WsHeader* h = static_cast<const WsHeader*>(a.hdr);
  return (call_errors(h, h->gen) & kDedupErrors) != 0u;
}

// a table row's columns c .. c + EL - 1
template <typename TW, int EL>
__device__ __forceinline__ void store_row(const Upd& up, uint32_t key, int c, const float (&o)[EL]) {
  char* q = static_cast<char*>(up.W) + ((int64_t)key * up.D + c) * (int64_t)sizeof(TW);
  if constexpr (sizeof(TW) == 2) {
    if (up.rounding) {
      uint32_t b[EL];
#pragma unroll
      for (int e = 0; e < EL; ++e)
        b[e] = bf16_stochastic(o[e], up.seed, (uint64_t)key * (uint64_t)up.D + (uint64_t)(c + e));
      if constexpr (EL == 1) {
        *reinterpret_cast<uint16_t*>(q) = (uint16_t)b[0];
      } else {
#pragma unroll
        for (int e = 0; e < EL / 2; ++e) reinterpret_cast<uint32_t*>(q)[e] = b[2 * e] | (b[2 * e + 1] << 16);
      }
      return;
    }
  }
  Vec<TW, EL>::store(q, o);
}

// Optimizer on columns c .. of row `key` with gradient g; w, h: the table row's
// columns and, element-wise Adagrad, its accumulators; step: lr, or row-wise
// Adagrad's lr / (sqrt(h) + eps).
template <typename TW, int EL, int KIND>
__device__ __forceinline__ void apply(const Upd& up, uint32_t key, int c, const float (&g)[EL], const Vec<TW, EL>& w,
                                      const Vec<float, EL>& h, float step) {
#pragma clang fp contract(off)
  float o[EL];
  if constexpr (KIND == kAdaElem) {
    float hn[EL];
#pragma unroll
    for (int e = 0; e < EL; ++e) {
      hn[e] = __builtin_fmaf(g[e], g[e], h.get(e));
      o[e] = w.get(e) - up.lr * g[e] / (sqrtf(hn[e]) + up.eps);
    }
    Vec<float, EL>::store(up.state + (int64_t)key * up.D + c, hn);
  } else {
#pragma unroll
    for (int e = 0; e < EL; ++e) o[e] = __builtin_fmaf(-step, g[e], w.get(e));
  }
  store_row<TW, EL>(up, key, c, o);
}

// x summed over the wavefront, in every lane
template <int CTRL>
__device__ __forceinline__ float add_lane(float x) {
  return x + __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(x), CTRL, 0xf, 0xf, true));
}
__device__ __forceinline__ float wave_total(float x) {
  // lanes 1 and 2 apart, then the mirrors of half rows and rows (whose lanes hold equal sums), then rows and halves
  return add_across<32>(add_across<16>(add_lane<0x140>(add_lane<0x141>(add_lane<0x4e>(add_lane<0xb1>(x))))));
}

// Rows of the table that no token named: zeros.  A wavefront takes zero_rows (up
// to kZeroRows) of them as one run of values; row = value / D by a multiplication
// (exact below 2^17 values for rows of up to 2^13).
constexpr int kZeroRows = 16;
static_assert(kZeroRows * kTokenMaxDim <= 1 << 17 && kTokenMaxDim <= 1 << 13, "the quotients are exact");
template <bool STREAM>
__device__ __forceinline__ void zero_rows(const TokGrad& a, int64_t share, int lane) {
  const int64_t r0 = share * a.zero_rows;
  if (r0 >= (int64_t)a.rows) return;
  const int n = (int)min((int64_t)a.zero_rows, (int64_t)a.rows - r0);
  const int U = failed(a) ? 0 : a.num_unique[0];
  uint32_t named = 0;
  if (U > 0) {
    const int u = r0 == 0 ? 0 : wave_upper_bound<uint32_t>(a.ukeys, U, (uint32_t)r0 - 1u, lane);
    const uint32_t key = u + lane < U ? a.ukeys[u + lane] : kNoRow;
    for (int r = 0; r < n; ++r) named |= __ballot(key == (uint32_t)r0 + r) ? 1u << r : 0u;
  }
  const uint32_t by = 0xffffffffu / (uint32_t)a.D + 1u;
  const float z[4] = {0.f, 0.f, 0.f, 0.f};
  float* dst = a.grad + r0 * (int64_t)a.D;
  for (int i = lane * 4; i < n * a.D; i += kWave * 4) {
    if ((named >> __umulhi((uint32_t)i, by)) & 1u) continue;
    if constexpr (STREAM) Vec<float, 4>::stream(dst + i, z);
    else Vec<float, 4>::store(dst + i, z);
  }
}

// of the a.blocks + a.zero_blocks blocks, those of zeros among the first b
__device__ __forceinline__ int zero_blocks_before(const TokGrad& a, int b) {
  return (int)((uint64_t)(uint32_t)b * (uint32_t)a.zero_blocks / (uint32_t)(a.blocks + a.zero_blocks));
}

// a finished gradient row's columns, where `layout` wants them
template <int EL, bool STREAM>
__device__ __forceinline__ void store_grad(const TokGrad& a, int u, uint32_t key, int col, bool in, float (&g)[EL]) {
  if (!in || (a.layout != EMB_ROWS && key >= a.rows)) return;
  float* dst = a.grad + (int64_t)(a.layout == EMB_ROWS ? (uint32_t)u : key) * a.D + col;
  if (key == a.pad) {
    if (a.layout == EMB_TABLE_ADD) return;
#pragma unroll
    for (int e = 0; e < EL; ++e) g[e] = 0.f;
  }
  if (a.layout == EMB_TABLE_ADD) {
    Vec<float, EL> old;
    old.load(dst);
#pragma unroll
    for (int e = 0; e < EL; ++e) g[e] += old.get(e);
  }
  if constexpr (STREAM) Vec<float, EL>::stream(dst, g);
  else Vec<float, EL>::store(dst, g);
}

// Chunk c's positions and segments.  They come in as few dependent loads as
// there can be: the dedup's state, its counts and the positions' rows; then the
// segments.  Until the state is known to be sound the counts only index after
// being clamped.
struct Chunk {
  bool failed;
  int u0, s0;          // the segment that holds the chunk's first position, its beginning
  int ends;            // lane l: the end of segment u0 + l
  uint32_t keys;       // its key
  int row_a, row_b;    // rows of the chunk's positions and the next one's (a segment that starts here ends before those end)
  uint64_t heavy;      // segments of more than a chunk's positions
  __device__ __forceinline__ Chunk(const TokGrad& a, int c, int lane) {
    const int p0 = c * kChunk;
    const WsHeader* h = static_cast<const WsHeader*>(a.hdr);
    const uint32_t gen = h->gen;
    const uint64_t err = __hip_atomic_load(&h->err, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    int U = a.num_unique[0];
    u0 = a.chunk_seg[c];
    row_a = a.perm[min(p0 + lane, a.N - 1)], row_b = a.perm[min(p0 + kChunk + lane, a.N - 1)];
    asm volatile("" : "+v"(U), "+v"(u0) : "v"(row_a), "v"(row_b));
    U = uniform(min(max(U, 1), a.N));
    u0 = uniform(min(max(u0, 0), U - 1));
    s0 = uniform(a.seg[u0]);
    ends = a.seg[min(u0 + 1 + lane, U)];
    keys = a.ukeys[min(u0 + lane, U - 1)];
    failed = (err_bits_of(err, gen) & kDedupErrors) != 0u;
    const int before = __shfl_up(ends, 1, kWave);
    heavy = __ballot(ends - (lane == 0 ? s0 : before) > kChunk);
  }
  __device__ __forceinline__ int row(int pos) const {
    return pos < kWave ? lane_at(row_a, pos) : lane_at(row_b, pos - kWave);
  }
};

// EL columns a lane, B positions a batch.  Row-wise Adagrad's blocks are the
// `parts` wavefronts of one chunk, which add up their rows' squares through
// LDS; others are four wavefronts of any.  EMB_TABLE's zeros are written by
// blocks of their own.  Few chunks are shared: each of up to 16 wavefronts takes
// the segments that start in its share of the positions.
template <typename TG, typename TW, int EL, int B, int KIND>
__global__ __launch_bounds__(KIND == kAdaRow ? kMostParts * kWave : 4 * kWave) void k_token_reduce(TokGrad a) {
  const int lane = threadIdx.x & (kWave - 1), wave = uniform(threadIdx.x / kWave);
  int block = blockIdx.x;
  if constexpr (stores(KIND)) {
    // blocks of zeros come among the others evenly: these write while those wait for rows
    const int z = zero_blocks_before(a, block), more = zero_blocks_before(a, block + 1);
    if (more > z) {
      zero_rows<KIND == kStream>(a, (int64_t)z * 4 + wave, lane);
      return;
    }
    block -= z;
  }
  // the chunk, the share of it whose segments start here, the columns
  int at, part;
  if constexpr (KIND == kAdaRow) {
    at = block, part = wave;
  } else {
    at = block * 4 + wave;
    part = at % a.parts, at /= a.parts;
  }
  const int c = at >> a.split, sub = at & ((1 << a.split) - 1);
  __shared__ float s_sq[2][kMostParts][B];
  if (c >= a.nchunks) return;
  const int col = (part * kWave + lane) * EL;
  const bool in = col < a.D;
  const int cs = in ? col : 0;
  const int p0 = c * kChunk, p1 = min(a.N, p0 + kChunk);
  const int b0 = p0 + sub * (kChunk >> a.split), b1 = min(p1, b0 + (kChunk >> a.split));
  const Chunk ch(a, c, lane);
  if (ch.failed) {
    if (stores(KIND) && a.layout == EMB_ROWS && in) {
      float z[EL] = {};
      for (int p = b0; p < b1; ++p) Vec<float, EL>::store(a.grad + (int64_t)p * a.D + col, z);
    }
    return;
  }
  const int u0 = ch.u0, s0 = ch.s0, ends = ch.ends;
  const uint32_t keys = ch.keys;
  const uint64_t heavy = ch.heavy;
  // the segments that start in b0 .. b1 - 1, and with them a long one's piece that came in with the chunk; a light
  // segment that came in belongs to another wavefront
  const bool came_in = s0 < p0 && sub == 0 && (heavy & 1u);
  int i = s0 >= b0 || came_in ? 0 : 1 + (int)__popcll(__ballot(ends < b0));
  const int last = (int)__popcll(__ballot(ends < b1));
  if (i > last) return;
  const int fin = (heavy >> last) & 1u ? min(p1, lane_at(ends, last)) : lane_at(ends, last);
  int q = i == 0 ? p0 : lane_at(ends, i - 1);
  // the row-wise accumulators of the segments, a lane each
  float accum = 0.f;
  if constexpr (KIND == kAdaRow) {
    if (keys < a.rows) accum = a.up.state[keys];
  }
  float acc[EL] = {};
  int parity = 0;
  while (q < fin) {
    // a padding segment has no gradient: its positions are not read
    if (lane_at(keys, i) == a.pad) {
      if constexpr (stores(KIND)) {
        if (!((heavy >> i) & 1u)) {
          float z[EL] = {};
          store_grad<EL, KIND == kStream>(a, u0 + i, a.pad, col, in, z);
        }
      }
      // (a batch may have ended inside it)
#pragma unroll
      for (int e = 0; e < EL; ++e) acc[e] = 0.f;
      q = min(lane_at(ends, i), fin);
      ++i;
      continue;
    }
    Vec<TG, EL> g[B];
    const int n = min(B, fin - q);
#pragma unroll
    for (int k = 0; k < B; ++k) {
      const int pos = min(q + k, fin - 1) - p0;
      const int row = ch.row(pos);
      const char* src = a.dy + (int64_t)row * a.ld + (uint32_t)cs * (uint32_t)(Vec<TG, EL>::kBytes / EL);
      if (a.aligned) g[k].load(src);
      else g[k].load_each(src);
    }
    if constexpr (stores(KIND)) {
#pragma unroll
      for (int k = 0; k < B; ++k) {
        if (k >= n) continue;
#pragma unroll
        for (int e = 0; e < EL; ++e) acc[e] += g[k].get(e);
        if (q + k + 1 != min(lane_at(ends, i), fin)) continue;
        float done[EL];
#pragma unroll
        for (int e = 0; e < EL; ++e) done[e] = acc[e] * a.scale, acc[e] = 0.f;
        if ((heavy >> i) & 1u) {
          if (in) Vec<float, EL>::store(a.partials + ((int64_t)c * 2 + (i == 0 ? 0 : 1)) * a.D + col, done);
        } else {
          store_grad<EL, KIND == kStream>(a, u0 + i, lane_at(keys, i), col, in, done);
        }
        i = min(i + 1, kWave - 1);
      }
    } else {
      Vec<TW, EL> w[B];
      Vec<float, EL> h[KIND == kAdaElem ? B : 1];
      float done[B][EL];
      int seg_of[B];  // the segment that ends at the batch's position, or -1
#pragma unroll
      for (int k = 0; k < B; ++k) {
        seg_of[k] = -1;
        if (k < n && q + k + 1 == min(lane_at(ends, i), fin)) {
          seg_of[k] = i;
          const uint32_t key = lane_at(keys, i);
          if (!((heavy >> i) & 1u) && key < a.rows && key != a.pad) {
            w[k].load(static_cast<const char*>(a.up.W) + ((int64_t)key * a.D + cs) * (int64_t)sizeof(TW));
            if constexpr (KIND == kAdaElem) h[k].load(a.up.state + (int64_t)key * a.D + cs);
          }
          i = min(i + 1, kWave - 1);
        }
      }
#pragma unroll
      for (int k = 0; k < B; ++k) {
#pragma unroll
        for (int e = 0; e < EL; ++e) {
          acc[e] += k < n ? g[k].get(e) : 0.f;
          done[k][e] = acc[e] * a.scale;
        }
        if (seg_of[k] >= 0) {
#pragma unroll
          for (int e = 0; e < EL; ++e) acc[e] = 0.f;
          if ((heavy >> seg_of[k]) & 1u) {
            if (in)
              Vec<float, EL>::store(a.partials + ((int64_t)c * 2 + (seg_of[k] == 0 ? 0 : 1)) * a.D + col, done[k]);
            seg_of[k] = -1;
          }
        }
      }
      float total[B];
      if constexpr (KIND == kAdaRow) {
#pragma unroll
        for (int k = 0; k < B; ++k) {
          total[k] = 0.f;
          if (seg_of[k] < 0) continue;
          float sq = 0.f;
#pragma unroll
          for (int e = 0; e < EL; ++e) sq = __builtin_fmaf(done[k][e], done[k][e], sq);
          total[k] = wave_total(in ? sq : 0.f);
        }
        if (a.parts > 1) {
          // (the accumulators are here before any wavefront of the block writes one; a batch's sums are read before the
          // batch after next is summed, a barrier later)
          asm volatile("" : "+v"(accum)::"memory");
          if (lane == 0) {
#pragma unroll
            for (int k = 0; k < B; ++k) s_sq[parity][wave][k] = total[k];
          }
          __syncthreads();
#pragma unroll
          for (int k = 0; k < B; ++k) {
            total[k] = 0.f;
            for (int p = 0; p < a.parts; ++p) total[k] += s_sq[parity][p][k];
          }
          parity ^= 1;
        }
      }
#pragma unroll
      for (int k = 0; k < B; ++k) {
        if (seg_of[k] < 0) continue;
        const uint32_t key = lane_at(keys, seg_of[k]);
        if (key >= a.rows || key == a.pad) continue;
        float step = a.up.lr;
        if constexpr (KIND == kAdaRow) {
          const float hn = __int_as_float(lane_at(__float_as_int(accum), seg_of[k])) + total[k] / (float)a.D;
          step = a.up.lr / (sqrtf(hn) + a.up.eps);
          if (wave == (a.parts > 1 ? 0 : wave) && lane == 0) a.up.state[key] = hn;
        }
        if (in) apply<TW, EL, KIND>(a.up, key, col, done[k], w[k], h[KIND == kAdaElem ? k : 0], step);
      }
    }
    q += n;
  }
}

// The same for few positions, whose time is that of dependent loads and of
// fetching the code: a wavefront to each position and part of the columns, for
// the segment that starts there or the long one's piece that came in with the
// chunk, all of whose loads but those of later batches are in flight together.
template <typename TG, typename TW, int EL, int B, int KIND>
__global__ __launch_bounds__(KIND == kAdaRow ? kMostParts * kWave : 4 * kWave) void k_token_reduce_each(TokGrad a) {
  const int lane = threadIdx.x & (kWave - 1), wave = uniform(threadIdx.x / kWave);
  int block = blockIdx.x;
  if constexpr (stores(KIND)) {
    const int z = zero_blocks_before(a, block), more = zero_blocks_before(a, block + 1);
    if (more > z) {
      zero_rows<KIND == kStream>(a, (int64_t)z * 4 + wave, lane);
      return;
    }
    block -= z;
  }
  int p, part;
  if constexpr (KIND == kAdaRow) {
    p = block, part = wave;
  } else {
    p = block * 4 + wave;
    part = p % a.parts, p /= a.parts;
  }
  __shared__ float s_sq[kMostParts];
  if (p >= a.N) return;
  const int col = (part * kWave + lane) * EL;
  const bool in = col < a.D;
  const int cs = in ? col : 0;
  const int c = p / kChunk, p0 = c * kChunk;
  const Chunk ch(a, c, lane);
  if (ch.failed) {
    if (stores(KIND) && a.layout == EMB_ROWS && in) {
      float z[EL] = {};
      Vec<float, EL>::store(a.grad + (int64_t)p * a.D + col, z);
    }
    return;
  }
  int i = 0;
  if (p != p0 || (ch.s0 < p0 && !(ch.heavy & 1u))) {
    const uint64_t starts = __ballot(ch.ends == p);
    if (starts == 0u) return;
    i = (int)__builtin_ctzll(starts) + 1;
  }
  const bool longs = (ch.heavy >> i) & 1u;
  const int fin = longs ? min(min(a.N, p0 + kChunk), lane_at(ch.ends, i)) : lane_at(ch.ends, i);
  const uint32_t key = lane_at(ch.keys, i);
  float acc[EL] = {};
  if (key == a.pad) {
    if constexpr (stores(KIND)) {
      if (!longs) store_grad<EL, KIND == kStream>(a, ch.u0 + i, key, col, in, acc);
    }
    return;
  }
  const bool applies = !stores(KIND) && !longs && key < a.rows;
  Vec<TW, EL> w;
  Vec<float, EL> h;
  float accum = 0.f;
  if constexpr (!stores(KIND)) {
    if (applies) {
      w.load(static_cast<const char*>(a.up.W) + ((int64_t)key * a.D + cs) * (int64_t)sizeof(TW));
      if constexpr (KIND == kAdaElem) h.load(a.up.state + (int64_t)key * a.D + cs);
      if constexpr (KIND == kAdaRow) accum = a.up.state[key];
    }
  }
  for (int q = p; q < fin; q += B) {
    Vec<TG, EL> g[B];
#pragma unroll
    for (int k = 0; k < B; ++k) {
      const char* src = a.dy + (int64_t)ch.row(min(q + k, fin - 1) - p0) * a.ld +
                        (uint32_t)cs * (uint32_t)(Vec<TG, EL>::kBytes / EL);
      if (a.aligned) g[k].load(src);
      else g[k].load_each(src);
    }
#pragma unroll
    for (int k = 0; k < B; ++k)
#pragma unroll
      for (int e = 0; e < EL; ++e) acc[e] += q + k < fin ? g[k].get(e) : 0.f;
  }
#pragma unroll
  for (int e = 0; e < EL; ++e) acc[e] *= a.scale;
  if (longs) {
    if (in) Vec<float, EL>::store(a.partials + ((int64_t)c * 2 + (i == 0 ? 0 : 1)) * a.D + col, acc);
    return;
  }
  if constexpr (stores(KIND)) {
    store_grad<EL, KIND == kStream>(a, ch.u0 + i, key, col, in, acc);
  } else {
    float step = a.up.lr;
    if constexpr (KIND == kAdaRow) {
      float sq = 0.f;
#pragma unroll
      for (int e = 0; e < EL; ++e) sq = __builtin_fmaf(acc[e], acc[e], sq);
      float total = wave_total(in ? sq : 0.f);
      if (a.parts > 1) {
        if (lane == 0) s_sq[wave] = total;
        // (the accumulator is here before a wavefront of the block writes it)
        asm volatile("" : "+v"(accum)::"memory");
        __syncthreads();
        total = 0.f;
        for (int k = 0; k < a.parts; ++k) total += s_sq[k];
      }
      const float hn = accum + total / (float)a.D;
      step = a.up.lr / (sqrtf(hn) + a.up.eps);
      if (applies && part == 0 && lane == 0) a.up.state[key] = hn;
    }
    if (in && applies) apply<TW, EL, KIND>(a.up, key, col, acc, w, h, step);
  }
}

__global__ __launch_bounds__(256) void k_token_zero(TokGrad a) {
  zero_rows<false>(a, (int64_t)blockIdx.x * 4 + threadIdx.x / kWave, threadIdx.x & (kWave - 1));
}

// A segment of more than 64 positions: the partial rows of its chunks added in
// double by the block of the chunk it starts in.  A lane takes four columns; a
// row leaves room for blockDim / (D / 4) groups of lanes (16 for rows of 64 values,
// 4 for 1024), which take every so many-th chunk and are added up through LDS in order.  Bound
// by latency: what tells the segment is read in two rounds, eight chunks' rows a
// lane in one.
constexpr int kCombineCols = 4, kCombineLanes = 1024;
template <typename TW, int KIND>
__global__ __launch_bounds__(kCombineLanes) void k_token_combine(TokGrad a) {
  const int c = blockIdx.x, lane = threadIdx.x & (kWave - 1), wave = threadIdx.x / kWave;
  const int p0 = c * kChunk, p1 = min(a.N, p0 + kChunk);
  if (failed(a)) return;
  const int U = a.num_unique[0];
  // the segment that holds the chunk's last position, if it is long and starts here
  const int next = a.chunk_seg[c + 1];  // (U after the last chunk)
  const int here = min(next, U - 1), prior = max(next - 1, 0);
  const int s_prior = a.seg[prior], s_here = a.seg[here], e_here = a.seg[here + 1];
  const uint32_t k_prior = a.ukeys[prior], k_here = a.ukeys[here];
  const bool back = next == U || s_here >= p1;
  const int u = back ? prior : here, s = back ? s_prior : s_here;
  const int e = back && next != U ? s_here : e_here;
  if (s < p0 || e - s <= kChunk) return;
  const uint32_t key = back ? k_prior : k_here;
  const bool pad = key == a.pad;
  if (pad && !stores(KIND)) return;
  if (key >= a.rows && !(stores(KIND) && a.layout == EMB_ROWS)) return;
  const int last = (e - 1) / kChunk;
  const int vectors = a.D / kCombineCols;
  const int lanes = blockDim.x, groups = vectors >= lanes ? 1 : lanes / vectors;
  const int group = groups == 1 ? 0 : (int)threadIdx.x / vectors, v0 = groups == 1 ? (int)threadIdx.x : (int)threadIdx.x % vectors;
  const int stride = groups == 1 ? lanes : vectors;  // (a row of 4096 values or more is gone over in turns)
  __shared__ double s_part[kCombineLanes][kCombineCols];
  __shared__ float s_sq[kCombineLanes / kWave];
  const float* first = a.partials + ((int64_t)c * 2 + (s == p0 ? 0 : 1)) * a.D;
  float sq = 0.f;
  const float old = KIND == kAdaRow ? a.up.state[key] : 0.f;
  auto finish = [&](int col, float (&g)[kCombineCols], float step) {
    if constexpr (stores(KIND)) {
      store_grad<kCombineCols, false>(a, u, key, col, true, g);
    } else {
      Vec<TW, kCombineCols> w;
      Vec<float, kCombineCols> h;
      w.load(static_cast<const char*>(a.up.W) + ((int64_t)key * a.D + col) * (int64_t)sizeof(TW));
      if constexpr (KIND == kAdaElem) h.load(a.up.state + (int64_t)key * a.D + col);
      apply<TW, kCombineCols, KIND>(a.up, key, col, g, w, h, step);
    }
  };
  for (int v = v0; v - v0 < vectors; v += stride) {
    const bool in = v < vectors && group < groups;
    const int col = in ? v * kCombineCols : 0;
    double t[kCombineCols] = {};
    if (in && !pad) {
      // chunk c itself counts as the first of the list
      constexpr int kAhead = 8;
      for (int k = c + group; k <= last; k += groups * kAhead) {
        Vec<float, kCombineCols> x[kAhead];
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
          const int at = k + i * groups;
          if (at > last) x[i].zero();
          else x[i].load((at == c ? first : a.partials + (int64_t)at * 2 * a.D) + col);
        }
#pragma unroll
        for (int i = 0; i < kAhead; ++i)
#pragma unroll
          for (int j = 0; j < kCombineCols; ++j) t[j] += (double)x[i].get(j);
      }
    }
    if (groups > 1) {
#pragma unroll
      for (int j = 0; j < kCombineCols; ++j) s_part[threadIdx.x][j] = t[j];
      __syncthreads();
      if (group == 0) {
        for (int k = 1; k < groups; ++k)
#pragma unroll
          for (int j = 0; j < kCombineCols; ++j) t[j] += s_part[k * vectors + v0][j];
      }
    }
    if (!in || group != 0) continue;
    float g[kCombineCols];
#pragma unroll
    for (int j = 0; j < kCombineCols; ++j) g[j] = (float)t[j];
    if constexpr (KIND == kAdaRow) {
      // (the sums wait in the first partial row until the squares of all columns are known)
      Vec<float, kCombineCols>::store(const_cast<float*>(first) + col, g);
#pragma unroll
      for (int j = 0; j < kCombineCols; ++j) sq = __builtin_fmaf(g[j], g[j], sq);
    } else {
      finish(col, g, a.up.lr);
    }
  }
  if constexpr (KIND == kAdaRow) {
    sq = wave_total(sq);
    if (lane == 0) s_sq[wave] = sq;
    __syncthreads();
    float total = 0.f;
    for (int w = 0; w < lanes / kWave; ++w) total += s_sq[w];
    const float hn = old + total / (float)a.D;
    const float step = a.up.lr / (sqrtf(hn) + a.up.eps);
    if (threadIdx.x == 0) a.up.state[key] = hn;
    for (int v = threadIdx.x; v < vectors; v += lanes) {
      Vec<float, kCombineCols> x;
      x.load(first + v * kCombineCols);
      float g[kCombineCols];
#pragma unroll
      for (int j = 0; j < kCombineCols; ++j) g[j] = x.get(j);
      finish(v * kCombineCols, g, step);
    }
  }
}

// blocks of zeros, of four wavefronts: as many rows to one (a power of two) as leave 1024 wavefronts (9 tokens of
// 2401 rows x 1352 11.7 us, 14.2 with 16 rows always; 4096 wavefronts 49.8 us where these take 46.5, 9000 tokens of 3000
// rows x 2000)
int zero_blocks(TokGrad& a) {
  a.zero_rows = kZeroRows;
  while (a.zero_rows > 1 && (int64_t)a.rows < (int64_t)a.zero_rows * kZeroWaves) a.zero_rows /= 2;
  return (int)(((int64_t)a.rows + 4 * a.zero_rows - 1) / (4 * a.zero_rows));
}

// Up to so many wavefronts, one to a position and its columns' parts; above, a
// wavefront walks a chunk's (us with the dedup, the former against the latter).
// Row-wise Adagrad, whose chunk costs a barrier a batch: 2000 x 64 18.0 (24.6),
// 500 x 1024 20.1 (38.3), 8000 x 1024 45.4 (54.4), 30000 x 256 56.3 (54.5).  SGD:
// 500 x 64 16.5 (20.9), 8000 x 256 31.8 (36.7), 8000 x 1024 44.6 (39.3).  Stored:
// 2000 x 64 18.6 (20.6), 2000 x 256 22.9 (23.9), 2000 x 1024 31.8 (29.8).
constexpr int64_t each_waves(int kind) { return kind == kAdaRow ? 32768 : stores(kind) ? 4096 : 8192; }

template <typename TG, typename TW, int KIND>
hipError_t grad_kernels(TokGrad a, hipStream_t s) {
  // columns a lane: 1 for rows of up to 64 values, 4, or 8 above 4096
  const int el = a.D <= kWave ? 1 : (a.D <= kMostParts * kWave * 4 ? 4 : 8);
  a.parts = (a.D + kWave * el - 1) / (kWave * el);
  constexpr bool kRow = KIND == kAdaRow;
  const dim3 block(kRow ? a.parts * kWave : 4 * kWave);
  const bool each = (int64_t)a.N * a.parts <= each_waves(KIND);
  a.split = 0;
  while (a.split < kMostSplit && ((int64_t)a.nchunks * a.parts << a.split) < kSplitWaves) ++a.split;
  a.blocks = each ? (kRow ? a.N : (a.N * a.parts + 3) / 4)
                  : (kRow ? a.nchunks << a.split : ((a.nchunks * a.parts << a.split) + 3) / 4);
  a.zero_blocks = stores(KIND) && a.layout == EMB_TABLE ? zero_blocks(a) : 0;
  const unsigned grid = (unsigned)a.blocks + (unsigned)a.zero_blocks;
  const int combine = a.D <= 256 ? kCombineLanes / 4 : kCombineLanes;
  if (!launchable(grid, (int)block.x) || !launchable(a.nchunks, combine)) return hipErrorNotSupported;
  const uintptr_t at = reinterpret_cast<uintptr_t>(a.dy) | (uintptr_t)a.ld;
  const int vec = el * (int)(sizeof(TG));
  a.aligned = at % (uintptr_t)(vec < 16 ? vec : 16) == 0;
  // positions a batch: as many loads in flight as registers allow at four wavefronts a SIMD
  constexpr int kB1 = 8, kB4 = stores(KIND) ? 16 : (KIND == kAdaElem ? 4 : 8), kB8 = stores(KIND) ? 8 : (KIND == kSgd ? 4 : 2);
  if (each) {
    if (el == 1) k_token_reduce_each<TG, TW, 1, 16, KIND><<<grid, block, 0, s>>>(a);
    else if (el == 4) k_token_reduce_each<TG, TW, 4, 8, KIND><<<grid, block, 0, s>>>(a);
    else k_token_reduce_each<TG, TW, 8, 8, KIND><<<grid, block, 0, s>>>(a);
  } else if (el == 1) k_token_reduce<TG, TW, 1, kB1, KIND><<<grid, block, 0, s>>>(a);
  else if (el == 4) k_token_reduce<TG, TW, 4, kB4, KIND><<<grid, block, 0, s>>>(a);
  else k_token_reduce<TG, TW, 8, kB8, KIND><<<grid, block, 0, s>>>(a);
  // (a long segment has more than one chunk)
  if (a.nchunks > 1)
    k_token_combine<TW, KIND == kStream ? kStore : KIND><<<a.nchunks, combine, 0, s>>>(a);
  return hipGetLastError();
}

template <typename TG, typename TW>
hipError_t update_kernels(const TokGrad& a, int opt, hipStream_t s) {
  if (opt == EMB_OPT_SGD) return grad_kernels<TG, TW, kSgd>(a, s);
  if (opt == EMB_OPT_ADAGRAD_ROWWISE) return grad_kernels<TG, TW, kAdaRow>(a, s);
  return grad_kernels<TG, TW, kAdaElem>(a, s);
}

template <typename TW, typename TO, int V, bool MANY>
hipError_t fwd_kernel(TokFwd a, const Stacked<MANY>& st, hipStream_t s) {
  a.aligned = (reinterpret_cast<uintptr_t>(a.out) | (uintptr_t)a.out_bytes) % (Vec<TO, V>::kBytes < 16 ? Vec<TO, V>::kBytes : 16) == 0;
  int lg = 0;
  while (lg < 8 && (1 << lg) < a.vectors) ++lg;
  a.log_g = lg;
  const int per = kFwdThreads >> lg;
  const unsigned parts = (unsigned)((a.vectors + (1 << lg) - 1) >> lg);
  // outputs that are streamed fill the device with two rows a lane in flight (as fast as one or four there, eight are
  // 7% slower); smaller ones spread over as many lanes as they can
  if (a.N * a.vectors * Vec<TO, V>::kBytes > kStreamBytes) {
    const int64_t blocks = (a.N + per * 2 - 1) / (per * 2);
    if (!launchable(blocks, kFwdThreads)) return hipErrorNotSupported;
    const dim3 grid((unsigned)blocks, parts);
    k_token_fwd<TW, TO, V, 2, true, MANY><<<grid, kFwdThreads, 0, s>>>(a, st);
  } else {
    const dim3 grid((unsigned)((a.N + per - 1) / per), parts);
    k_token_fwd<TW, TO, V, 1, false, MANY><<<grid, kFwdThreads, 0, s>>>(a, st);
  }
  return hipGetLastError();
}

template <bool MANY>
hipError_t fwd_types(TokFwd a, const Stacked<MANY>& st, int dtype, int out, int D, hipStream_t s) {
  // 16 bytes of the table's row a lane
  a.vectors = D / (dtype == EMB_BF16 ? 8 : 4);
  if (dtype == EMB_BF16) {
    if (out == EMB_BF16) return fwd_kernel<bf16, bf16, 8, MANY>(a, st, s);
    return fwd_kernel<bf16, float, 8, MANY>(a, st, s);
  }
  if (out == EMB_BF16) return fwd_kernel<float, bf16, 4, MANY>(a, st, s);
  return fwd_kernel<float, float, 4, MANY>(a, st, s);
}

}  // namespace

hipError_t launch_token_fwd(const TokenFwdLaunch& p, hipStream_t s) {
  TokFwd a{};
  a.W = static_cast<const char*>(p.W);
  a.idx = p.idx;
  a.idx64 = p.idx64;
  a.offsets = p.offsets;
  a.out = static_cast<char*>(p.out);
  a.N = p.N;
  a.row_bytes = (int64_t)p.D * (p.dtype == EMB_BF16 ? 2 : 4);
  a.out_bytes = p.ld * (p.out_dtype == EMB_BF16 ? 2 : 4);
  a.T = p.T;
  a.B = p.B;
  a.rows = p.rows;
  a.pad = p.pad;
  a.scale = p.scale;
  if (p.T == 1) return fwd_types<false>(a, Stacked<false>{}, p.dtype, p.out_dtype, p.D, s);
  return fwd_types<true>(a, Stacked<true>{p.ro}, p.dtype, p.out_dtype, p.D, s);
}

hipError_t launch_token_grad(const TokenGradLaunch& p, hipStream_t s) {
  char* ws = static_cast<char*>(p.ws);
  TokGrad a{};
  a.dy = static_cast<const char*>(p.dy);
  a.ld = p.ld * (p.dy_dtype == EMB_BF16 ? 2 : 4);
  a.perm = p.perm;
  a.seg = p.seg;
  a.ukeys = p.ukeys;
  a.num_unique = p.num_unique;
  a.chunk_seg = reinterpret_cast<const int32_t*>(ws + p.lay.chunk_seg);
  a.hdr = ws + p.lay.hdr;
  a.partials = reinterpret_cast<float*>(ws + p.lay.partials);
  a.grad = p.grad;
  a.N = p.N;
  a.D = p.D;
  a.nchunks = (p.N + kChunk - 1) / kChunk;
  a.layout = p.layout;
  a.rows = p.rows;
  a.pad = p.pad;
  a.scale = p.scale;
  a.up.W = p.W;
  a.up.state = p.state;
  a.up.D = p.D;
  a.up.opt = p.opt;
  a.up.lr = p.lr;
  a.up.eps = p.eps;
  a.up.rounding = p.rounding;
  a.up.seed = p.seed;
  if (!p.fuse) {
    if (p.N == 0) {
      if (p.layout == EMB_TABLE && p.rows > 0) {
        const unsigned blocks = (unsigned)zero_blocks(a);
        if (!launchable(blocks, 256)) return hipErrorNotSupported;
        k_token_zero<<<blocks, 256, 0, s>>>(a);
      }
      return hipGetLastError();
    }
    if ((p.layout == EMB_TABLE ? (int64_t)p.rows : (int64_t)p.N) * p.D * 4 > kStreamBytes)
      return p.dy_dtype == EMB_BF16 ? grad_kernels<bf16, float, kStream>(a, s) : grad_kernels<float, float, kStream>(a, s);
    return p.dy_dtype == EMB_BF16 ? grad_kernels<bf16, float, kStore>(a, s) : grad_kernels<float, float, kStore>(a, s);
  }
  if (p.N == 0) return hipSuccess;
  if (p.dtype == EMB_BF16)
    return p.dy_dtype == EMB_BF16 ? update_kernels<bf16, bf16>(a, p.opt, s) : update_kernels<float, bf16>(a, p.opt, s);
  return p.dy_dtype == EMB_BF16 ? update_kernels<bf16, float>(a, p.opt, s) : update_kernels<float, float>(a, p.opt, s);
}

}  // namespace emb
