// Linear attention with a decay for each key head (gfx950).
//
//   S_t = g S_{t-1} + k_t^T v_t,   y_t = scale q_t S_t
//
// over ragged sequences, in chunks of C positions.  With S the state before a
// chunk of n positions (i, j: positions within it)
//
//   y_i = scale ( g^(i+1) q_i S + sum over j <= i of g^(i-j) (q_i . k_j) v_j )
//   S'  = g^n S + sum over j of g^(n-1-j) k_j^T v_j
//
// and all four results of the operator are this one form of rows a, b, c:
//
//   y :  a = q,  b = k,  c = v,  in order
//   dq:  a = dy, b = v,  c = k,  in order (the state is S transposed)
//   dv:  a = k,  b = q,  c = dy, backwards, the state being the gradient G that
//        arrives at the state after a position
//   dk:  a = v,  b = dy, c = q,  backwards, with G transposed
//
// Heads that share keys and values: in order a has the heads' rows, backwards b
// and c have them, and sums over the heads arise by themselves.
//
// Sequences are cut into segments of L positions from their begin.  A boundary
// at position p (a segment's begin that is not its sequence's) is number
// p / L - 1: no two have the same one, and a sequence's are consecutive.  Three
// launches: sums of every segment that a boundary follows (backwards: precedes),
// the boundaries' states from them one after another, and the form itself,
// every segment from its boundary's state.  All sums have a fixed order.
//
// A block takes a segment's key head; its four wavefronts have the columns of c
// and of the state in quarters, the state in registers from chunk to chunk, and
// the rows of a chunk in LDS, loaded a step (a head of a chunk) ahead.  Products
// a . b go through LDS once, from the wavefronts that make them to all.
//
// Bound.  One prompt of 32768 tokens, 16 heads of 128 x 128: 221 us, of which sums 75 (293 MB,
// 3.9 TB/s), boundaries 13 and the form 137 (571 MB, 4.2 TB/s).  A training batch of 48
// sequences, 32768 x 16 heads (4 key heads) of 128: forward 182 (sums 29, boundaries 17, the form
// 137), backward 406 (sums 70, boundaries 16, the three forms 320, 1.09 GB at 3.4 TB/s) where a
// profiler separates them, 492 together among calls.  There LDS is busy a third of the time (its
// reads: every wavefront takes all rows of a and b), the matrix units a quarter; the rest is the
// latency of a step's phases at two blocks a compute unit, and the last round of blocks.
// Rows or heads that do not begin at multiples of 16 bytes are loaded and stored value by value:
// 16384 tokens in 24 sequences, 16 heads of 65 x 72, forward and backward 1047 us, of 64 x 72 274.
#include "block_common.h"

namespace emb {

namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef short s16x4 __attribute__((ext_vector_type(4)));

constexpr int kThreads = 256;  // of the chain

// What a matrix instruction's operand is made of: lane l holds row (or column)
// l % 16 and, with q = l / 16, part of a block of kBlock summed indexes.
template <typename T>
struct Operand;

// v_mfma 16 x 16 x 32: eight of 32 indexes a lane, 8 q .. 8 q + 7; from a state 4 q + e and 16 + 4 q + e
template <>
struct Operand<bf16> {
  static constexpr int kChunk = 64, kBlock = 32, kPad = 8, kVec = 8, kParts = 3, kWeights = 2, kStates = 2;
  typedef uint16_t Value;
  // Distance of rows that are also read by columns: 12 (or 36) words past a multiple of 64 banks, so that 16 rows' 16
  // bytes as well as four rows' 32 bytes lie apart
  static constexpr int apart(int w) { return w == 64 ? 72 : w + 24; }
  bf16x8 v;
  // row `at` (an address in LDS), indexes 0 .. kBlock - 1 of it
  __device__ __forceinline__ void row(const Value* at, int q) { v = *reinterpret_cast<const bf16x8*>(at + 8 * q); }
  __device__ __forceinline__ void row_as_state(const Value* at, int q) {
    const u32x2 lo = *reinterpret_cast<const u32x2*>(at + 4 * q), hi = *reinterpret_cast<const u32x2*>(at + 16 + 4 * q);
    v = __builtin_bit_cast(bf16x8, u32x4{lo.x, lo.y, hi.x, hi.y});
  }
  // column APART (l / 4) + l % 4 from `at` on, rows 0 .. kBlock - 1 of LD values: the transposing load gives
  // a lane four rows of its column where the 16 lanes of a quarter point at those rows' 16 columns in order,
  // four each
  template <int LD, int APART = 4>
  __device__ __forceinline__ void column(const Value* at, int q, int l) {
    const Value* p = at + (8 * q + l / 4) * LD + APART * (l % 4);
    const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)p);
    const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)(p + 4 * LD));
    const u32x2 a = __builtin_bit_cast(u32x2, lo), b = __builtin_bit_cast(u32x2, hi);
    v = __builtin_bit_cast(bf16x8, u32x4{a.x, a.y, b.x, b.y});
  }
  // 32 indexes of a state, two tiles: the nearest to them, which are left with what that leaves of them
  __device__ __forceinline__ void state(f32x4& a, f32x4& b) {
    const u32x4 w{pack_bf16(a.x, a.y), pack_bf16(a.z, a.w), pack_bf16(b.x, b.y), pack_bf16(b.z, b.w)};
    v = __builtin_bit_cast(bf16x8, w);
    a -= f32x4{bf16_lo(w.x), bf16_hi(w.x), bf16_lo(w.y), bf16_hi(w.y)};
    b -= f32x4{bf16_lo(w.z), bf16_hi(w.z), bf16_lo(w.w), bf16_hi(w.w)};
  }
  __device__ __forceinline__ float get(int e) const {
    const uint32_t w = __builtin_bit_cast(u32x4, v)[e / 2];
    return e % 2 ? bf16_hi(w) : bf16_lo(w);
  }
  // the nearest to x, which is left with what that leaves of it (three times: nothing)
  __device__ __forceinline__ void take(float (&x)[8]) {
    u32x4 w;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      w[i] = pack_bf16(x[2 * i], x[2 * i + 1]);
      x[2 * i] -= bf16_lo(w[i]);
      x[2 * i + 1] -= bf16_hi(w[i]);
    }
    v = __builtin_bit_cast(bf16x8, w);
  }
  static __device__ __forceinline__ int index(int q, int e) { return 8 * q + e; }
  static constexpr int kEach = 8;
};

// v_mfma 16 x 16 x 4, four times: a lane's four of 16 indexes are 4 q .. 4 q + 3, one a time
template <>
struct Operand<float> {
  static constexpr int kChunk = 32, kBlock = 16, kPad = 4, kVec = 4, kParts = 1, kWeights = 1, kStates = 1;
  typedef float Value;
  static constexpr int apart(int w) { return w + kPad; }
  f32x4 v;
  __device__ __forceinline__ void row(const Value* at, int q) { v = *reinterpret_cast<const f32x4*>(at + 4 * q); }
  __device__ __forceinline__ void row_as_state(const Value* at, int q) { row(at, q); }
  template <int LD, int APART = 4>
  __device__ __forceinline__ void column(const Value* at, int q, int l) {
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = at[(4 * q + e) * LD + APART * (l / 4) + l % 4];
  }
  __device__ __forceinline__ void state(const f32x4& a, const f32x4&) { v = a; }
  __device__ __forceinline__ float get(int e) const { return v[e]; }
  __device__ __forceinline__ void take(const float (&x)[4]) { v = f32x4{x[0], x[1], x[2], x[3]}; }
  static __device__ __forceinline__ int index(int q, int e) { return 4 * q + e; }
  static constexpr int kEach = 4;
};

// D[m][n] += sum over k of A[m][k] B[n][k]; lane l holds n = l % 16, m = 4 (l / 16) .. + 3
__device__ __forceinline__ void mul(f32x4& d, const Operand<bf16>& a, const Operand<bf16>& b) {
  d = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a.v, b.v, d, 0, 0, 0);
}
__device__ __forceinline__ void mul(f32x4& d, const Operand<float>& a, const Operand<float>& b) {
#pragma unroll
  for (int e = 0; e < 4; ++e) d = __builtin_amdgcn_mfma_f32_16x16x4f32(a.v[e], b.v[e], d, 0, 0, 0);
}

struct Form {
  Rows a, b, c, out;
  const float* bounds;  // states at the boundaries
  const float* begin;   // of whole sequences: states that the sweep begins with, or none
  float* end;           // and ends with, or none
  int32_t da, dc;       // widths of a and b, of c and out
  int32_t sd, sn;       // state: distance of two indexes of b, of c
  int32_t rev;          // backwards
  float p_scale, u_scale, out_scale;  // of products a . b, of what the state gets, of out
};

struct Args {
  int64_t N, bounds;  // number of boundaries
  int32_t log;        // of the segment length L = 2^log
  int32_t M, groups, per;  // heads of a group
  int32_t aligned;
  const int32_t* offsets;
  const float* decay;
  int64_t state;  // values of a group's state
  Form f[3];
  int32_t slices[3];
  float* sums;
  int32_t cols[3];  // columns of c that a block takes
};

// g^e for a whole e >= 0, in 64 bits
__device__ __forceinline__ double power(float g, int64_t e) {
  double r = 1.0, b = (double)g;
  for (; e > 0; e >>= 1) {
    if (e & 1) r *= b;
    b *= b;
  }
  return r;
}

struct Segment {
  int64_t begin, end;
  int32_t seq;
  bool first, last;  // of its sequence
};

// the boundary of this number: the segment that begins there; false if there is none
__device__ __forceinline__ bool boundary(const Args& a, int64_t number, int lane, Segment& s) {
  const int64_t pos = (number + 1) << a.log;
  int64_t o, e;
  if (a.M < kWave) {  // every offset in a lane
    const int32_t v = lane <= a.M ? a.offsets[lane] : 0x7fffffff;
    s.seq = __popcll(__ballot(v <= (int32_t)pos)) - 1;
    if (s.seq < 0 || s.seq >= a.M) return false;
    o = lane_at(v, s.seq);
    e = lane_at(v, s.seq + 1);
  } else {
    s.seq = wave_upper_bound(a.offsets, a.M + 1, (int32_t)pos, lane) - 1;
    if (s.seq < 0 || s.seq >= a.M) return false;
    o = a.offsets[s.seq];
    e = a.offsets[s.seq + 1];
  }
  e = min(e, a.N);
  const int64_t L = (int64_t)1 << a.log;
  if (pos == o) return false;
  s.begin = o + ((pos - o + L - 1) & -L);
  if (s.begin >= e) return false;
  s.end = min(s.begin + L, e);
  s.first = false;
  s.last = s.end == e;
  return true;
}
// segments: the boundaries', then the sequences' first ones
__device__ __forceinline__ bool segment(const Args& a, int64_t number, int lane, Segment& s) {
  if (number < a.bounds) return boundary(a, number, lane, s);
  s.seq = (int32_t)(number - a.bounds);
  const int64_t e = min((int64_t)max(a.offsets[s.seq + 1], 0), a.N);
  s.begin = min((int64_t)max(a.offsets[s.seq], 0), e);
  s.end = min(s.begin + ((int64_t)1 << a.log), e);
  s.first = true;
  s.last = s.end == e;
  return true;
}

// A chunk's rows: offsets are 32 bits from the first of them in memory, and one past the last row's columns
// reads as zero and is not written, so neither a chunk's last rows nor a head's last columns need a branch
// and loads stay in flight together.  kNowhere is past any chunk, also with the distance of its rows (below
// 2^30) added or taken off.
constexpr uint32_t kNowhere = 0x80000000u;
__device__ __forceinline__ __amdgpu_buffer_rsrc_t from_base(const void* p, int bytes) {
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(p), 0, bytes, 0x00020000);
}
// `n` rows from `row` on, which a step takes in order or (rev) from the last one up; `top` is its first one's
// offset, `ld` the distance of two.
struct Chunk {
  __amdgpu_buffer_rsrc_t rsrc;
  int ld, top;
  __device__ __forceinline__ Chunk(const char* p, int stride, int64_t row, int n, int bytes, bool rev, bool wanted) {
    const int span = (n - 1) * stride;
    rsrc = from_base(p + row * stride, wanted && n > 0 ? span + bytes : 0);
    ld = rev ? -stride : stride;
    top = rev ? span : 0;
  }
};

// Rows of a chunk on their way to LDS, in 16 bytes a lane, zeros where there are none.
template <typename T, int W, int THREADS, bool ALIGNED>
struct Rowset {
  typedef typename Operand<T>::Value Value;
  static constexpr int kVec = Operand<T>::kVec, kRow = W / kVec;
  static constexpr int kEach = Operand<T>::kChunk * kRow / THREADS, kApart = THREADS / kRow;
  static_assert(Operand<T>::kChunk * kRow % THREADS == 0 && THREADS % kRow == 0, "whole rounds");
  u32x4 v[kEach];
  __device__ __forceinline__ void load(const Chunk& c, int w) {
    const int r = threadIdx.x / kRow, col = threadIdx.x % kRow * kVec;
    const uint32_t off = (uint32_t)(c.top + r * c.ld + col * (int)sizeof(Value));
    if constexpr (ALIGNED) {
      const uint32_t at = col < w ? off : kNowhere;
#pragma unroll
      for (int i = 0; i < kEach; ++i)
        v[i] = __builtin_amdgcn_raw_buffer_load_b128(c.rsrc, at + (uint32_t)(i * kApart * c.ld), 0, 0);
    } else {
#pragma unroll
      for (int i = 0; i < kEach; ++i) {
        const uint32_t row = off + (uint32_t)(i * kApart * c.ld);
        if constexpr (kVec == 8) {
#pragma unroll
          for (int k = 0; k < 8; k += 2) {
            const uint32_t lo = (uint16_t)__builtin_amdgcn_raw_buffer_load_b16(c.rsrc, col + k < w ? row + 2 * k : kNowhere, 0, 0);
            const uint32_t hi =
                (uint16_t)__builtin_amdgcn_raw_buffer_load_b16(c.rsrc, col + k + 1 < w ? row + 2 * k + 2 : kNowhere, 0, 0);
            v[i][k / 2] = lo | hi << 16;
          }
        } else {
#pragma unroll
          for (int k = 0; k < 4; ++k)
            v[i][k] = __builtin_amdgcn_raw_buffer_load_b32(c.rsrc, col + k < w ? row + 4 * k : kNowhere, 0, 0);
        }
      }
    }
  }
  __device__ __forceinline__ void put(Value* lds, int ld) const {
    Value* to = lds + threadIdx.x / kRow * ld + threadIdx.x % kRow * kVec;
#pragma unroll
    for (int i = 0; i < kEach; ++i) *reinterpret_cast<u32x4*>(to + i * kApart * ld) = v[i];
  }
};

// A block's LDS: the rows of a chunk, a step's products, powers of the decay, and what a full chunk's rows
// enter the state with, then zeros.
template <typename T, int DA, int DC, bool OUT>
struct Room {
  typedef Operand<T> Op;
  static constexpr int C = Op::kChunk, LA = DA + Op::kPad, LB = Op::apart(DA), LC = Op::apart(DC), LP = C + Op::kPad,
                       P = C * LP;
  alignas(16) typename Op::Value a[OUT ? C * LA : 8], b[C * LB], c[C * LC], p[OUT ? Op::kWeights * P : 8];
  alignas(16) float fade[2 * C], pow[C + 1];
};

// DA: widest a and b; DC: columns of c that a block takes; begin .. until - 1: of the group's heads (in
// order, a part of them may be).  OUT: the form itself, else the sums of the segment that ends (backwards:
// begins) at a boundary.
template <typename T, int DA, int DC, int W, bool OUT, bool ALIGNED, bool REV>
__device__ __forceinline__ void sweep(const Args& args, const Form& f, int64_t number, int group, int slice,
                                      int begin, int until, Room<T, DA, DC, OUT>& lds) {
  typedef Operand<T> Op;
  typedef typename Op::Value Value;
  constexpr int C = Op::kChunk, KB = Op::kBlock, TC = C / 16, TD = DA / 16, KC = C / KB, KD = DA / KB;
  constexpr int kThreads = kWave * W, TN = DC / (16 * W);
  static_assert(!OUT || W == 4, "three squares of products");
  typedef Room<T, DA, DC, OUT> Lds;
  constexpr int LA = Lds::LA, LB = Lds::LB, LC = Lds::LC, LP = Lds::LP;
  Value* const s_a = lds.a;
  Value* const s_b = lds.b;
  Value* const s_c = lds.c;
  Value* const s_p = lds.p;
  float* const s_pow = lds.pow;
  float* const s_fade = lds.fade;
  const int lane = threadIdx.x % kWave, wave = uniform(threadIdx.x / kWave), l = lane % 16, q = lane / 16;
  constexpr bool rev = REV;
  constexpr int size = sizeof(Value);
  const int c0 = slice * DC, wc = min(DC, f.dc - c0), n0 = 16 * TN * wave;
  const int64_t states = (int64_t)args.groups * args.state, mine = (int64_t)group * args.state;
  // The matrices' places stay in scalar registers (loaded again from the arguments in every step, they would
  // be waited for), from the group's columns on: heads are `apart` bytes from one another.
  struct Place {
    const char* p;
    int ld, apart;
  };
  auto place_of = [&](const Rows& m, int cols, bool per_head, int first) {
    Place x{m.p + ((int64_t)group * (per_head ? args.per : 1) * cols + first) * size, (int)m.ld, per_head ? cols * size : 0};
    asm volatile("" : "+s"(x.p), "+s"(x.ld), "+s"(x.apart));
    return x;
  };
  const Place pa = OUT ? place_of(f.a, f.da, !rev, 0) : Place{}, pb = place_of(f.b, f.da, rev, 0),
              pc = place_of(f.c, f.dc, rev, c0), po = OUT ? place_of(f.out, f.dc, !rev, c0) : Place{};
  int da = f.da;
  asm volatile("" : "+s"(da));
  // (what a block waits for at its begin, one after another: the offsets, then rows and states; the rest on the way)
  const float g = args.decay[group];
  Segment s;
  if (OUT ? !segment(args, number, lane, s) : !boundary(args, number, lane, s)) return;
  if (!OUT && !rev) {  // the segment before
    s.end = s.begin;
    s.begin -= (int64_t)1 << args.log;
  }
  const int length = (int)(s.end - s.begin);
  auto chunk = [&](const Place& m, int at, int h, int n, int w, bool wanted) {
    return Chunk(m.p + h * m.apart, m.ld, rev ? s.end - at - n : s.begin + at, n, w * size, rev, wanted);
  };
  // A step is a head of a chunk; its rows are on their way while the one before it is worked on.
  struct Step {
    int at, h;
  };
  auto after = [&](Step x) { return x.h + 1 < until ? Step{x.at, x.h + 1} : Step{x.at + C, begin}; };
  Rowset<T, DA, kThreads, ALIGNED> ra, rb;
  Rowset<T, DC, kThreads, ALIGNED> rc;
  // (rows that a step does not need are loaded from nowhere: a branch around loads would wait for them at its end)
  auto load = [&](Step x) {
    const int n = min(C, length - x.at);
    if constexpr (OUT) ra.load(chunk(pa, x.at, x.h, n, da, !rev || x.h == begin), da);
    rb.load(chunk(pb, x.at, x.h, n, da, rev || x.h == begin), da);
    rc.load(chunk(pc, x.at, x.h, n, wc, rev || x.h == begin), wc);
  };
  Step now{0, begin};
  load(now);
  // The state: lane l holds rows 16 d + 4 q .. of a column.  With two tiles of columns a wavefront, those of
  // tile t are 8 j + 4 t + (0 .. 3), so that a lane's results of both are eight values in a row.
  constexpr int kApart = 4 * TN, kTile = TN == 2 ? 4 : 16;
  // (`from_l` is l, in a register of the caller's: the offsets of the first use are not kept for the second)
  auto place = [&](int from_l, int d, int t, int e) {
    const int row = 16 * d + 4 * q + e, col = n0 + kTile * t + kApart * (from_l / 4) + from_l % 4;
    return row < f.da && col < wc ? (uint32_t)(row * f.sd + (c0 + col) * f.sn) * 4u : kNowhere;
  };
  f32x4 st[TD][TN] = {};
  const float* from = nullptr;
  if constexpr (OUT) {
    if (rev ? s.last : s.first) from = f.begin != nullptr ? f.begin + s.seq * states + mine : nullptr;
    else from = f.bounds + (((rev ? s.end : s.begin) >> args.log) - 1) * states + mine;
    if (from != nullptr) {
      const auto base = from_base(from, 4 * (int)args.state);
#pragma unroll
      for (int d = 0; d < TD; ++d)
#pragma unroll
        for (int t = 0; t < TN; ++t)
#pragma unroll
          for (int e = 0; e < 4; ++e)
            st[d][t][e] = __uint_as_float(__builtin_amdgcn_raw_buffer_load_b32(base, place(l, d, t, e), 0, 0));
    }
  }
  auto put = [&](int h) {
    if (OUT && (!rev || h == begin)) ra.put(s_a, LA);
    if (rev || h == begin) {
      rb.put(s_b, LB);
      rc.put(s_c, LC);
    }
  };
  // (a power for every exponent from C down)
  for (int i = threadIdx.x; i < 2 * C; i += kThreads) {
    const int at = i - (rev ? 0 : 1);
    const float v = i <= C ? (float)power(g, C - i) : 0.f;
    if (i <= C) s_pow[C - i] = v;
    if (at >= 0) s_fade[at] = f.u_scale * v;
    if (i == 2 * C - 1 && !rev) s_fade[i] = 0.f;
  }
  put(begin);
  __syncthreads();
  // Weights of the products that a lane makes, in row l % 16 of a tile, columns 4 q ..: in one on the
  // diagonal, in the one before it, and how much less those before that have
  constexpr int kSide = TC / 2, kSquares = 3;  // (the fourth square is above the diagonal)
  const int square = wave, ti = square >= 1 ? kSide : 0, tj = square >= 2 ? kSide : 0;
  float on[4], off[4], less[2 * kSide - 1], before[TC];
  if constexpr (OUT) {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      on[e] = f.p_scale * s_pow[max(l - 4 * q - e, 0)];
      off[e] = f.p_scale * s_pow[16 + l - 4 * q - e];
    }
#pragma unroll
    for (int i = 0; i < TC; ++i) before[i] = lane_at(s_pow[16 * max(i - wave - 1, 0)], 0);
#pragma unroll
    for (int i = 0; i < 2 * kSide - 1; ++i) less[i] = lane_at(s_pow[16 * max(ti - tj + i - kSide, 0)], 0);
  }
  // A state that is kept gets weighted rows with all of their 24 bits, in three parts; one that only
  // multiplies rows of this segment, and is rounded to 16 bits for that, gets 16 of them.
  const bool exact = f.end != nullptr && begin == 0 && (rev ? s.first : s.last);
  f32x4 o[TC][TN];
  while (now.at < length) {
    const int at = now.at, h = now.h, n = min(C, length - at);
    const bool new_a = !rev || h == begin, last = h == until - 1;
    // (addresses are made again in every step: kept across it they take the registers that loads are on their way to)
    int l = lane % 16, q = lane / 16;
    asm volatile("" : "+v"(l), "+v"(q));
    __syncthreads();
    const Step next = after(now);
    load(next);
    if constexpr (OUT) {
      auto put_products = [&](f32x4 p, int i, int j, float fade) {
        // (of tile i, j; weights of bf16 rows have two parts of bf16, 16 bits: with one alone a short sequence is off by
        // 0.0024 of y where y's own rounding is 0.0015; the second part is 4% of a form's time)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float w = i == j ? on[e] : off[e] * fade;
          p[e] = 16 * (i - j) + l - 4 * q - e >= 0 ? p[e] * w : 0.f;
        }
        Value* to = s_p + (16 * i + l) * LP + 16 * j + 4 * q;
        if constexpr (sizeof(Value) == 2) {
#pragma unroll
          for (int part = 0; part < Op::kWeights; ++part) {
            const u32x2 w{pack_bf16(p[0], p[1]), pack_bf16(p[2], p[3])};
            *reinterpret_cast<u32x2*>(to + part * Lds::P) = w;
            p -= f32x4{bf16_lo(w.x), bf16_hi(w.x), bf16_lo(w.y), bf16_hi(w.y)};
          }
        } else {
          *reinterpret_cast<f32x4*>(to) = p;
        }
      };
      if (new_a) {
        // What the state before the chunk gives (lane l: row 16 i + l % 16), and in order on the way, as the
        // rows of a are there, their products with 16 rows of b a wavefront, for LDS.  (Tiles above the
        // diagonal are zeros.)
        f32x4 p[TC];
#pragma unroll
        for (int i = 0; i < TC; ++i) {
          p[i] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int t = 0; t < TN; ++t) o[i][t] = f32x4{0.f, 0.f, 0.f, 0.f};
        }
#pragma unroll
        for (int k = 0; k < KD; ++k) {
          Op x[Op::kStates][TN], z;
          if constexpr (!rev) z.row_as_state(s_b + (16 * (wave % TC) + l) * LB + k * KB, q);
          // (of bf16 rows, the state has two parts, 16 bits: results that cancel in it, as queries across a component that
          // keys and values share have them, were off by up to a seventh of y with one; 32768 tokens, 16 heads of 128 x
          // 128: 221 us, 216 with one part; their training with 4 key heads: 492, 466 with one)
#pragma unroll
          for (int t = 0; t < TN; ++t) {
            f32x4 lo = st[k * KB / 16][t], hi = st[(k * KB / 16 + 1) % TD][t];
#pragma unroll
            for (int part = 0; part < Op::kStates; ++part) x[part][t].state(lo, hi);
          }
#pragma unroll
          for (int i = 0; i < TC; ++i) {
            Op y;
            y.row_as_state(s_a + (16 * i + l) * LA + k * KB, q);
            if constexpr (!rev) mul(p[i], z, y);
#pragma unroll
            for (int t = 0; t < TN; ++t)
#pragma unroll
              for (int part = 0; part < Op::kStates; ++part) mul(o[i][t], x[part][t], y);
          }
        }
#pragma unroll
        for (int i = 0; i < TC; ++i) {
          const float w = s_pow[16 * i + l + (rev ? 0 : 1)];
#pragma unroll
          for (int t = 0; t < TN; ++t) o[i][t] *= w;
          if (!rev && wave < TC) put_products(p[i], i, wave, before[i]);
        }
      }
      if (rev && square < kSquares) {
        // backwards, where rows of b are new in every step: kSide x kSide tiles a wavefront, of the squares
        // on and below the diagonal
        f32x4 p[kSide][kSide];
#pragma unroll
        for (int i = 0; i < kSide; ++i)
#pragma unroll
          for (int j = 0; j < kSide; ++j) p[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int k = 0; k < KD; ++k) {
          Op x[kSide], y[kSide];
#pragma unroll
          for (int i = 0; i < kSide; ++i) {
            x[i].row(s_b + (16 * (tj + i) + l) * LB + k * KB, q);
            y[i].row(s_a + (16 * (ti + i) + l) * LA + k * KB, q);
          }
#pragma unroll
          for (int i = 0; i < kSide; ++i)
#pragma unroll
            for (int j = 0; j < kSide; ++j) mul(p[i][j], x[j], y[i]);
        }
#pragma unroll
        for (int i = 0; i < kSide; ++i)
#pragma unroll
          for (int j = 0; j < kSide; ++j) put_products(p[i][j], ti + i, tj + j, less[kSide - 1 + i - j]);
      }
      __syncthreads();
    }
    Op c[KC][TN];
#pragma unroll
    for (int k = 0; k < KC; ++k)
#pragma unroll
      for (int t = 0; t < TN; ++t) c[k][t].template column<LC, kApart>(s_c + k * KB * LC + n0 + kTile * t, q, l);
    if constexpr (OUT) {
#pragma unroll
      for (int i = 0; i < TC; ++i)
#pragma unroll
        for (int k = 0; k <= 16 * i / KB; ++k) {
          Op y[Op::kWeights];
#pragma unroll
          for (int part = 0; part < Op::kWeights; ++part) y[part].row(s_p + part * Lds::P + (16 * i + l) * LP + k * KB, q);
#pragma unroll
          for (int t = 0; t < TN; ++t)
#pragma unroll
            for (int part = 0; part < Op::kWeights; ++part) mul(o[i][t], c[k][t], y[part]);
        }
      {
        // (to nowhere where nothing is to be stored yet: as many stores follow the loads in every step, so that the
        // wait for the loads does not take in the stores)
        const Chunk out = chunk(po, at, h, n, wc, !rev || last);
        const int col = n0 + kApart * q;
#pragma unroll
        for (int i = 0; i < TC; ++i) {
          const uint32_t row = (uint32_t)(out.top + (l + 16 * i) * out.ld + col * size);
          float v[4 * TN];
#pragma unroll
          for (int t = 0; t < TN; ++t)
#pragma unroll
            for (int e = 0; e < 4; ++e) v[4 * t + e] = o[i][t][e] * f.out_scale;
          if constexpr (!ALIGNED) {
#pragma unroll
            for (int e = 0; e < 4 * TN; ++e) {
              const uint32_t to = col + e < wc ? row + (uint32_t)(e * size) : kNowhere;
              if constexpr (size == 2)
                __builtin_amdgcn_raw_buffer_store_b16((uint16_t)pack_bf16(v[e], 0.f), out.rsrc, to, 0, 0);
              else __builtin_amdgcn_raw_buffer_store_b32(__float_as_uint(v[e]), out.rsrc, to, 0, 0);
            }
          } else {
            // (a head's columns end at a multiple of 16 bytes)
#pragma unroll
            for (int e = 0; e < 4 * TN; e += 16 / size) {
              const uint32_t to = col + e < wc ? row + (uint32_t)(e * size) : kNowhere;
              if constexpr (size == 4) {
                __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, f32x4{v[e], v[e + 1], v[e + 2], v[e + 3]}),
                                                       out.rsrc, to, 0, 0);
              } else if constexpr (TN == 1) {
                __builtin_amdgcn_raw_buffer_store_b64(u32x2{pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3])}, out.rsrc, to, 0, 0);
              } else {
                __builtin_amdgcn_raw_buffer_store_b128(
                    u32x4{pack_bf16(v[e], v[e + 1]), pack_bf16(v[e + 2], v[e + 3]), pack_bf16(v[e + 4], v[e + 5]),
                          pack_bf16(v[e + 6], v[e + 7])},
                    out.rsrc, to, 0, 0);
              }
            }
          }
        }
      }
    }
    __builtin_amdgcn_sched_barrier(0);
    // (what a segment's last chunk leaves is only for a state that is kept)
    if ((rev || last) && (!OUT || exact || at + C < length)) {
      const float all = rev && h > begin ? 1.f : s_pow[n];
#pragma unroll
      for (int d = 0; d < TD; ++d)
#pragma unroll
        for (int t = 0; t < TN; ++t) st[d][t] *= all;
#pragma unroll
      for (int k = 0; k < KC; ++k) {
        __builtin_amdgcn_sched_barrier(0);
        float w[Op::kEach];
        const int j = k * KB + Op::index(q, 0) + C - n;
        if (n == C) {
#pragma unroll
          for (int e = 0; e < Op::kEach; e += 4) {
            const f32x4 v = *reinterpret_cast<const f32x4*>(s_fade + j + e);
#pragma unroll
            for (int i = 0; i < 4; ++i) w[e + i] = v[i];
          }
        } else {
#pragma unroll
          for (int e = 0; e < Op::kEach; ++e) w[e] = s_fade[j + e];
        }
        // parts `from` up to `to` of the rows times their weights
        auto add = [&](auto from, auto to) {
          constexpr int F = decltype(from)::value, P = decltype(to)::value;
          Op x[TN][P];
#pragma unroll
          for (int t = 0; t < TN; ++t) {
            float v[Op::kEach];
#pragma unroll
            for (int e = 0; e < Op::kEach; ++e) v[e] = c[k][t].get(e) * w[e];
#pragma unroll
            for (int p = 0; p < P; ++p) x[t][p].take(v);
          }
#pragma unroll
          for (int d = 0; d < TD; ++d) {
            Op y;
            y.template column<LB>(s_b + k * KB * LB + 16 * d, q, l);
#pragma unroll
            for (int t = 0; t < TN; ++t)
#pragma unroll
              for (int p = F; p < P; ++p) mul(st[d][t], y, x[t][p]);
          }
        };
        using std::integral_constant;
        if constexpr (!OUT || Op::kParts == 1) {
          add(integral_constant<int, 0>{}, integral_constant<int, Op::kParts>{});
        } else {
          add(integral_constant<int, 0>{}, integral_constant<int, 2>{});
          if (exact) add(integral_constant<int, 2>{}, integral_constant<int, Op::kParts>{});
        }
      }
    }
    __syncthreads();
    put(next.h);
    now = next;
  }
  float* to = nullptr;
  if constexpr (!OUT) to = args.sums + number * states + mine;
  else if (exact) to = f.end + s.seq * states + mine;
  if (to == nullptr) return;
  int other = l;
  asm volatile("" : "+v"(other));
  const auto base = from_base(to, 4 * (int)args.state);
#pragma unroll
  for (int d = 0; d < TD; ++d)
#pragma unroll
    for (int t = 0; t < TN; ++t)
#pragma unroll
      for (int e = 0; e < 4; ++e)
        __builtin_amdgcn_raw_buffer_store_b32(__float_as_uint(st[d][t][e]), base, place(other, d, t, e), 0, 0);
}

// `forms` of the forms from `first` on, which have as many slices each, in one launch; `parts`: blocks that share a
// group's heads (in order)
template <typename T, int DA, int DC, int W, bool OUT, bool ALIGNED>
__global__ __launch_bounds__(kWave* W, DA > 128 ? 1 : 2) void k_linear(Args a, int first, int forms, int parts) {
  __shared__ Room<T, DA, DC, OUT> lds;
  uint32_t at = blockIdx.x;
  const Form& f = a.f[first + (int)(at % (uint32_t)forms)];
  at /= (uint32_t)forms;
  const uint32_t slices = (uint32_t)a.slices[first], groups = (uint32_t)a.groups;
  const int slice = (int)(at % slices);
  at /= slices;
  const int each = a.per / parts, begin = (int)(at % (uint32_t)parts) * each, until = OUT || f.rev ? begin + each : 1;
  at /= (uint32_t)parts;
  // (apart: each needs fewer registers than one body for both)
  if (f.rev) sweep<T, DA, DC, W, OUT, ALIGNED, true>(a, f, at / groups, (int)(at % groups), slice, begin, until, lds);
  else sweep<T, DA, DC, W, OUT, ALIGNED, false>(a, f, at / groups, (int)(at % groups), slice, begin, until, lds);
}

// States at a sequence's boundaries from the sums between them, in place: in order, or backwards.
template <int V, bool REV>
__global__ __launch_bounds__(kThreads) void k_linear_chain(Args a, const float* begin) {
  const int lane = threadIdx.x % kWave;
  const int64_t slices = (a.state + kThreads * V - 1) / (kThreads * V);
  int64_t at = blockIdx.x;
  const int64_t i = (at % slices * kThreads + threadIdx.x) * V;
  at /= slices;
  const int group = (int)(at % a.groups);
  const int64_t number = at / a.groups;
  Segment s;
  // one block a sequence: its first boundary's
  if (!boundary(a, number, lane, s)) return;
  const int64_t o = max(a.offsets[s.seq], 0), e = min((int64_t)a.offsets[s.seq + 1], a.N);
  if (s.begin - o != (int64_t)1 << a.log || i >= a.state) return;
  const int64_t count = (e - o - 1) >> a.log, states = (int64_t)a.groups * a.state;
  const float g = a.decay[group];
  const float whole = (float)power(g, (int64_t)1 << a.log), part = (float)power(g, e - o - (count << a.log));
  float* p = a.sums + number * states + group * a.state + i;
  float v[V] = {};
  if (begin != nullptr) {
    Vec<float, V> x;
    x.load(begin + s.seq * states + group * a.state + i);
#pragma unroll
    for (int k = 0; k < V; ++k) v[k] = x.get(k);
  }
  constexpr int kAhead = 8;
  for (int64_t b = 0; b < count; b += kAhead) {
    Vec<float, V> x[kAhead];
#pragma unroll
    for (int j = 0; j < kAhead; ++j)
      if (b + j < count) x[j].load(p + (REV ? count - 1 - b - j : b + j) * states);
#pragma unroll
    for (int j = 0; j < kAhead; ++j) {
      if (b + j >= count) break;
      const float w = REV && b + j == 0 ? part : whole;
#pragma unroll
      for (int k = 0; k < V; ++k) v[k] = w * v[k] + x[j].get(k);
      Vec<float, V>::store(p + (REV ? count - 1 - b - j : b + j) * states, v);
    }
  }
}

// ---------------------------------------------------------------- host

// Segments: a chunk of 64 positions, or twice as long until there are no more blocks of sums than the device holds at
// once (two a compute unit).
constexpr int kMinLog = 6;
constexpr int64_t kMaxBlocks = 512;
int64_t most_bounds(int groups) { return groups >= kMaxBlocks ? 1 : kMaxBlocks / groups; }
int log_length(int64_t N, int groups) {
  int log = kMinLog;
  while (N > 0 && (N - 1) >> log > most_bounds(groups)) ++log;
  return log;
}

// Columns of c that a block takes, and the widest a and b of the kernel that does (rows that are not aligned
// are for any width up to 128, or to 256).
int columns_of(const Args& a, int da, int dc, bool narrow) { return narrow || !a.aligned || da > 128 || dc <= 64 ? 64 : 128; }
int width_of(const Args& a, int da) { return da > 128 ? 256 : a.aligned && da <= 64 ? 64 : 128; }

// Blocks that the device holds at once: two a compute unit.
constexpr int64_t kResident = 512;

template <typename T, bool OUT>
hipError_t go(const Args& a, int first, int forms, hipStream_t s) {
  const Form& f = a.f[first];
  int64_t blocks = (OUT ? a.bounds + a.M : a.bounds) * a.groups * a.slices[first] * forms;
  // In order the heads of a group may be shared by blocks, each of which makes the state: what that costs
  // (about half of a head's work, and as much again for a block's begin and end) against rounds of blocks on
  // the device.  Four heads, 700 blocks of all: 137 us with one block a group, 130 with two, 148 with four;
  // three, 92 blocks (1501 tokens): 23 us with all in a block, 18 with one.
  int parts = 1;
  if (OUT && forms == 1 && !f.rev) {
    auto cost = [&](int n) { return (float)((blocks * n + kResident - 1) / kResident) * ((float)(a.per / n) + 0.9f); };
    for (int n = 2; n <= a.per; ++n)
      if (a.per % n == 0 && blocks * n < ((int64_t)1 << 22) && cost(n) < 0.95f * cost(parts)) parts = n;
  }
  blocks *= parts;
  if (blocks == 0) return hipSuccess;
  const unsigned grid = (unsigned)blocks;
  const int da = width_of(a, f.da), dc = a.cols[first];
  if (!a.aligned) {
    if (da == 128) k_linear<T, 128, 64, 4, OUT, false><<<grid, kThreads, 0, s>>>(a, first, forms, parts);
    else k_linear<T, 256, 64, 4, OUT, false><<<grid, kThreads, 0, s>>>(a, first, forms, parts);
  } else if (da == 64) {
    if (dc == 128) k_linear<T, 64, 128, 4, OUT, true><<<grid, kThreads, 0, s>>>(a, first, forms, parts);
    else k_linear<T, 64, 64, 4, OUT, true><<<grid, kThreads, 0, s>>>(a, first, forms, parts);
  } else if (da == 128) {
    if (dc == 128) k_linear<T, 128, 128, 4, OUT, true><<<grid, kThreads, 0, s>>>(a, first, forms, parts);
    else k_linear<T, 128, 64, 4, OUT, true><<<grid, kThreads, 0, s>>>(a, first, forms, parts);
  } else {
    k_linear<T, 256, 64, 4, OUT, true><<<grid, kThreads, 0, s>>>(a, first, forms, parts);
  }
  return hipGetLastError();
}
// whether two forms are taken by the same kernel
bool alike(const Args& a, int i, int j) {
  return width_of(a, a.f[i].da) == width_of(a, a.f[j].da) &&
         a.cols[i] == a.cols[j] && a.slices[i] == a.slices[j];
}

template <bool REV>
hipError_t chain(const Args& a, const float* begin, hipStream_t s) {
  if (a.bounds == 0) return hipSuccess;
  const bool four = a.state % 4 == 0 && ((uintptr_t)begin & 15u) == 0;
  const int64_t slices = (a.state + kThreads * (four ? 4 : 1) - 1) / (kThreads * (four ? 4 : 1));
  const unsigned grid = (unsigned)(a.bounds * a.groups * slices);
  if (four) k_linear_chain<4, REV><<<grid, kThreads, 0, s>>>(a, begin);
  else k_linear_chain<1, REV><<<grid, kThreads, 0, s>>>(a, begin);
  return hipGetLastError();
}

void add_form(Args& a, int which, const Form& f, bool narrow = false) {
  a.f[which] = f;
  a.cols[which] = columns_of(a, f.da, f.dc, narrow);
  a.slices[which] = (f.dc + a.cols[which] - 1) / a.cols[which];
}

void prepare(const LinLaunch& p, Args& a) {
  a.N = p.N;
  a.M = p.M;
  a.groups = p.groups;
  a.per = p.heads / p.groups;
  a.aligned = p.aligned;
  a.offsets = p.offsets;
  a.decay = p.decay;
  a.state = (int64_t)p.dk * p.dv;
  a.log = log_length(p.N, p.groups);
  a.bounds = p.N > 0 ? (p.N - 1) >> a.log : 0;
}
// whether every grid is one (states are taken in pieces of 256 values or more)
bool fits(const Args& a, int forms) {
  int slices = 1;
  for (int i = 0; i < 3; ++i) slices = a.slices[i] > slices ? a.slices[i] : slices;
  return launchable((a.bounds + a.M) * a.groups * slices * forms, kThreads) &&
         launchable(a.bounds * a.groups * ((a.state + kThreads - 1) / kThreads), kThreads);
}

// fp32 products are most of a wavefront's time (matrix units do a fraction of the bf16 ones): blocks of half the
// columns, as long as the device holds them at once.  Forward and backward of 4 heads of 128 x 128, 1001 tokens in 4
// sequences, 2 key heads: 62 us, 87 with whole ones; 2001 tokens, one key head: 83 and 114.
template <typename T>
bool narrow(const Args& a, int forms) {
  return sizeof(T) == 4 && 2 * forms * (a.bounds + a.M) * a.groups <= kResident;
}

template <typename T>
hipError_t forward(const LinLaunch& p, hipStream_t s) {
  Args a{};
  prepare(p, a);
  a.sums = p.states;
  add_form(a, 0, Form{p.q, p.k, p.v, p.y, p.states, p.first, p.last, p.dk, p.dv, p.dv, 1, 0, 1.f, 1.f, p.scale},
           narrow<T>(a, a.per));
  if (!fits(a, 1)) return hipErrorNotSupported;
  hipError_t e = go<T, false>(a, 0, 1, s);
  if (e == hipSuccess) e = chain<false>(a, p.first, s);
  if (e == hipSuccess) e = go<T, true>(a, 0, 1, s);
  return e;
}

template <typename T>
hipError_t backward(const LinLaunch& p, hipStream_t s) {
  Args a{};
  prepare(p, a);
  a.sums = p.grads;
  add_form(a, 0, Form{p.k, p.q, p.dy, p.dval, p.grads, p.dlast, p.dfirst, p.dk, p.dv, p.dv, 1, 1, p.scale, p.scale, 1.f},
           narrow<T>(a, 1));
  add_form(a, 1, Form{p.v, p.dy, p.q, p.dkey, p.grads, p.dlast, nullptr, p.dv, p.dk, 1, p.dv, 1, p.scale, p.scale, 1.f},
           narrow<T>(a, 2));
  add_form(a, 2, Form{p.dy, p.v, p.k, p.dq, p.states, p.first, nullptr, p.dv, p.dk, 1, p.dv, 0, 1.f, 1.f, p.scale},
           narrow<T>(a, 2));
  if (!fits(a, 3)) return hipErrorNotSupported;
  hipError_t e = go<T, false>(a, 0, 1, s);
  if (e == hipSuccess) e = chain<true>(a, p.dlast, s);
  // (dk and dq have the same widths; with dv's too they are one launch, whose last blocks fill the device better)
  const bool one = alike(a, 0, 1);
  if (e == hipSuccess) e = go<T, true>(a, 0, one ? 3 : 1, s);
  if (e == hipSuccess && !one) e = go<T, true>(a, 1, 2, s);
  return e;
}

}  // namespace

size_t lin_states_bytes(int64_t N, int32_t groups, int32_t dk, int32_t dv) {
  const int64_t most = most_bounds(groups), need = N > 0 ? (N - 1) >> kMinLog : 0;
  return align256(sizeof(float) * (size_t)(need < most ? need : most) * (size_t)groups * (size_t)dk * (size_t)dv);
}

hipError_t launch_lin_fwd(const LinLaunch& p, hipStream_t s) {
  return p.dtype == EMB_FP32 ? forward<float>(p, s) : forward<bf16>(p, s);
}
hipError_t launch_lin_bwd(const LinLaunch& p, hipStream_t s) {
  return p.dtype == EMB_FP32 ? backward<float>(p, s) : backward<bf16>(p, s);
}

}  // namespace emb
