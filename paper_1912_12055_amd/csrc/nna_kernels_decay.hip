// Linear attention with a decay l for each head: S_t = l S_{t-1} + k_t^T v_t, o_t = scale q_t S_t.
//
// Taken a chunk of 64 frames at a time, the sums are products of small matrices: with S the state before the chunk, i and j its frames,
//   o_i = sum_{j <= i} l^(i-j) (q_i . k_j) v_j + l^(i+1) q_i S,      S' = l^n S + sum_j l^(n-1-j) k_j^T v_j.
// The gradients are the same mix of other arrays: gq = mix(go, v, k) with S^T, and, with time reversed and the state's gradient G in
// S's place, gk = mix(v, go, q) with G^T, gv = mix(k, q, go) with G.  One kernel runs them all: out = mix(a, b, c).
//
// A workgroup of four waves (float32 heads of 128: eight; gradients in pairs: sixteen) goes through the chunks of a (sequence, head), or of a segment of one where
// there are too few of them to fill the card (the segments' own states are then summed in a launch before, and joined in order).  Its state stays in registers,
// float32, some of the columns to a wave; the chunk's a, b and c are in LDS.  Where values are float32 a chunk is 32 frames (Shape).
//
// 4 sequences of 16 heads of 128, 16,384 frames, bfloat16: states 126 us (4.3 TB/s), joined in 11, the mix 305 to 320 (3.4 TB/s; a copy as large reaches 5.1), the
// gradients' states 223, joined in 21, three mixes 855 to 930.  The conversions and scalings around the products (830 vector instructions a wave and chunk beside 162
// matrix instructions) and the barriers between a chunk's steps keep it from memory's rate.  Few heads (8 of 64, 15,504 frames): 13, 8 and 25 us, latencies of a
// segment's chunks one after the other.  float32, 16 sequences of 431 frames, 8 heads of 64: 43 and 60 us, half of the CUs, one wave a SIMD.
#include "nna_decay.h"

namespace nna {

constexpr int CHUNK = DECAY_CHUNK;

namespace {

typedef __bf16 bf16;
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef unsigned u32x4 __attribute__((ext_vector_type(4)));

// ---- operands ----------------------------------------------------------------------------------------------------------
// All products are bfloat16 matrix instructions with float32 sums, 16 x 16 x 32.  A float32 is the sum of three bfloat16, each the rounding of what the ones
// before leave; a product of two takes the six of the nine products of planes that a float32 sum can tell from zero.  An operand is
// planes of eight values a lane: lane (i, g) of (lane % 16, lane / 16) holds row (A) or column (B) i, of the 32 k either 8 g .. 8 g + 7 or, so
// that a 16 x 16 accumulator of an earlier product (rows 4 g .. 4 g + 3 of column i) is one as it lies, 4 g .. 4 g + 3 and 16 + 4 g .. 16 + 4 g + 3.
template <int NA, int NB>
__device__ __forceinline__ f32x4 mma(const bf16x8 (&a)[NA], const bf16x8 (&b)[NB], f32x4 s) {
  constexpr int most = NA > NB ? NA : NB;
#pragma unroll
  for (int t = most - 1; t >= 0; --t)  // small terms first
#pragma unroll
    for (int i = 0; i <= t; ++i)
      if (i < NA && t - i < NB) s = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a[i], b[t - i], s, 0, 0, 0);
  return s;
}
__device__ __forceinline__ bf16x8 join(bf16x4 a, bf16x4 b) { return __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7); }

// What a first plane is rounded from: the last 2^-9 of float32's range would round to an infinity, so it is bfloat16's largest there and the next planes hold the rest;
// an infinity or a NaN stays one in them.  Beside bfloat16 values (T), none of which is larger, it is left out (16,384 frames, 64 heads of 128, both directions: 1,429 us
// with it, 1,395 without): a state or weight that near to float32's end is then an infinity to the frames it meets.
template <typename T>
__device__ __forceinline__ float in_range(float v) { return sizeof(T) == 4 ? __builtin_amdgcn_fmed3f(v, -0x1.fep127f, 0x1.fep127f) : v; }
template <typename T, typename V>
__device__ __forceinline__ V all_in_range(V v) {
#pragma unroll
  for (int i = 0; i < (int)(sizeof(V) / sizeof(float)); ++i) v[i] = in_range<T>(v[i]);
  return v;
}

// two accumulators (k and 16 + k) as an operand of N planes
template <typename T, int N>
__device__ __forceinline__ void split(f32x4 v, f32x4 w, bf16x8 (&o)[N]) {
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const bf16x4 a = __builtin_convertvector(i ? v : all_in_range<T>(v), bf16x4), b = __builtin_convertvector(i ? w : all_in_range<T>(w), bf16x4);
    o[i] = join(a, b);
    if (i + 1 < N) {
      v -= __builtin_convertvector(a, f32x4);
      w -= __builtin_convertvector(b, f32x4);
    }
  }
}

// ---- tiles in LDS: planes of rows (frames), a head's values along a row ------------------------------------------------------
// Rows are an odd multiple of 32 bytes apart, and in the lower half of every 16 rows the octets of a pair change places: 16 lanes that read octets along 16 rows,
// and eight rows' pairs of octets read across, then meet all 64 banks once (64 heads of 128, 16,384 frames: 1 % faster than rows 8 or 24 values longer; a state's
// launch has no bank conflict).
__host__ __device__ constexpr int pitch_of(int d) { return d + 16; }
__device__ __forceinline__ int swap_of(int row) { return row & 8; }
template <int ROWS, int D, int N>
struct Tile {
  static constexpr int PITCH = pitch_of(D), PLANE = ROWS * PITCH, SIZE = N * PLANE;
  // k along a row: values k0 + 8 g .. of row0 + i
  static __device__ __forceinline__ void rows8(const bf16* tile, int row0, int k0, int li, int lg, bf16x8 (&o)[N]) {
#pragma unroll
    for (int p = 0; p < N; ++p) o[p] = *reinterpret_cast<const bf16x8*>(tile + p * PLANE + (row0 + li) * PITCH + k0 + (lg * 8 ^ swap_of(li)));
  }
  // ... in the order of accumulators
  static __device__ __forceinline__ void rows4(const bf16* tile, int row0, int k0, int li, int lg, bf16x8 (&o)[N]) {
#pragma unroll
    for (int p = 0; p < N; ++p) {
      const bf16* at = tile + p * PLANE + (row0 + li) * PITCH + k0 + (lg * 4 ^ swap_of(li));
      o[p] = join(*reinterpret_cast<const bf16x4*>(at), *reinterpret_cast<const bf16x4*>(at + 16));
    }
  }
  // k across rows, in the order of accumulators: rows row0 .. row0 + 31 of column0 + i
  static __device__ __forceinline__ void columns(const bf16* tile, int row0, int column0, int lane, bf16x8 (&o)[N]) {
#pragma unroll
    for (int p = 0; p < N; ++p) {
      const bf16* at = tile + p * PLANE + (row0 + (lane >> 2)) * PITCH + column0 + ((lane & 3) * 4 ^ swap_of(lane >> 2));
      bf16x4 f[2];
#pragma unroll
      for (int h = 0; h < 2; ++h)
        f[h] = __builtin_bit_cast(bf16x4, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)(at + h * 16 * PITCH)));
      o[p] = join(f[0], f[1]);
    }
  }
};

__device__ __forceinline__ float power(float log2_decay, int n) { return __builtin_amdgcn_exp2f(log2_decay * (float)n); }
// log2 of a decay; of zero, one whose first power is zero and whose zeroth is one
__device__ __forceinline__ float log2_of(float decay) { return decay == 0.f ? -1e5f : log2f(decay); }

// a value that all lanes hold, in a scalar register
__device__ __forceinline__ int uniform(int v) { return __builtin_amdgcn_readfirstlane(v); }
__device__ __forceinline__ float uniform(float v) { return __builtin_bit_cast(float, uniform(__builtin_bit_cast(int, v))); }

// What is computed of `v` after this is computed there: not ahead of a loop, to be kept in registers through it.
template <typename V>
__device__ __forceinline__ V here_only(V v) {
  asm volatile("" : "+v"(v));
  return v;
}

template <typename T>
struct Kind;
template <>
struct Kind<bf16> {
  static constexpr int planes = 1;
  typedef bf16 oct __attribute__((ext_vector_type(8), aligned(2)));
  // zero times the values: NaN where one is not finite
  static __device__ __forceinline__ float nothing(oct v, float s) {
    const bf16x8 w = v;
    const bf16x2 zero = {(bf16)0.f, (bf16)0.f};
#pragma unroll
    for (int i = 0; i < 4; ++i) s = __builtin_amdgcn_fdot2_f32_bf16(bf16x2{w[2 * i], w[2 * i + 1]}, zero, s, false);
    return s;
  }
  static __device__ __forceinline__ void put(bf16* p, int plane, oct v) { *reinterpret_cast<bf16x8*>(p) = v; }
  static __device__ __forceinline__ void put1(bf16* p, int plane, bf16 v) { *p = v; }
};
template <>
struct Kind<float> {
  static constexpr int planes = 3;
  typedef float oct __attribute__((ext_vector_type(8), aligned(4)));
  static __device__ __forceinline__ float nothing(oct v, float s) {
#pragma unroll
    for (int i = 0; i < 8; ++i) s = __builtin_fmaf(v[i], 0.f, s);
    return s;
  }
  static __device__ __forceinline__ void put(bf16* p, int plane, oct v) {
    f32x8 left = v;
#pragma unroll
    for (int i = 0; i < 3; ++i) {
      const bf16x8 w = __builtin_convertvector(i ? left : all_in_range<float>(left), bf16x8);
      *reinterpret_cast<bf16x8*>(p + i * plane) = w;
      if (i < 2) left -= __builtin_convertvector(w, f32x8);
    }
  }
  static __device__ __forceinline__ void put1(bf16* p, int plane, float v) {
#pragma unroll
    for (int i = 0; i < 3; ++i) {
      p[i * plane] = (bf16)(i ? v : in_range<float>(v));
      v -= (float)p[i * plane];
    }
  }
};

// ROWS rows of D values (d of them real) as THREADS threads hold them between memory and LDS, eight neighbours a lane at a time.  No lane reads what is not
// there: a row past the end is read as the last one, a lane past d as column 0, and the octet that d ends in is the row's last eight
// (which then also lie in LDS where they belong; where d < 8, one value after the other).
template <typename T, int ROWS, int D, int THREADS, bool FULL, bool REVERSE>
struct Rows {
  typedef Kind<T> K;
  typedef typename K::oct oct;
  typedef Tile<ROWS, D, K::planes> tile_type;
  static constexpr int PER_ROW = D / 8, OCTETS = ROWS * PER_ROW, N = OCTETS >= THREADS ? OCTETS / THREADS : 1, STEP = THREADS / PER_ROW;
  oct v[N];

  static __device__ __forceinline__ bool idle(int thread) { return OCTETS < THREADS && thread >= OCTETS; }

  // frame u (row) of `here` frames, whose first in memory is at `base`; `step` elements (below 2^24) from one to the next
  __device__ __forceinline__ void load(const T* base, int step, int here, int d, int thread) {
    thread = here_only(thread);
    const int row = idle(thread) ? 0 : thread / PER_ROW, column = thread % PER_ROW * 8;
    const int at = FULL || column + 8 <= d ? column : column < d && d >= 8 ? d - 8 : 0;
    const char* p = reinterpret_cast<const char*>(base);
    const unsigned bytes = step * (unsigned)sizeof(T);
    if (here == ROWS && (FULL || d >= 8)) {
      unsigned offset = (REVERSE ? ROWS - 1 - row : row) * bytes + at * (unsigned)sizeof(T);
#pragma unroll
      for (int i = 0; i < N; ++i, offset += REVERSE ? -STEP * bytes : STEP * bytes) v[i] = *reinterpret_cast<const oct*>(p + offset);
    } else {
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const int r = row + i * STEP < here ? row + i * STEP : here - 1;
        const T* q = reinterpret_cast<const T*>(p + (REVERSE ? here - 1 - r : r) * bytes) + at;
        if (FULL || d >= 8) {
          v[i] = *reinterpret_cast<const oct*>(q);
        } else {
#pragma unroll
          for (int e = 0; e < 8; ++e) v[i][e] = q[e < d ? e : 0];
        }
      }
    }
  }
  // the first `here` rows are real, the others and the columns past d zero
  __device__ __forceinline__ void store(bf16* tile, int here, int d, int thread) {
    if (idle(thread)) return;
    const int column = thread % PER_ROW * 8;
    if (here < ROWS) {
      const int row = here_only(thread) / PER_ROW;
#pragma unroll
      for (int i = 0; i < N; ++i)
        if (row + i * STEP >= here) v[i] = (oct)(T)0;
    }
    bf16* p = tile + thread / PER_ROW * tile_type::PITCH;
    static_assert(STEP % 16 == 0 || N == 1, "a lane's octets change places in all of its rows or in none");
    const int swap = swap_of(thread / PER_ROW);
#pragma unroll
    for (int i = 0; i < N; ++i, p += STEP * tile_type::PITCH) {
      if (FULL) {
        K::put(p + (column ^ swap), tile_type::PLANE, v[i]);
        continue;
      }
      K::put(p + (column ^ swap), tile_type::PLANE, column + 8 <= d ? v[i] : (oct)(T)0);
      if (column < d && column + 8 > d) {
        const int first = d >= 8 ? d - 8 : 0;
#pragma unroll
        for (int e = 0; e < 8; ++e)
          if (e < d) K::put1(p + (first + e ^ here_only(swap)), tile_type::PLANE, v[i][e]);
      }
    }
  }
  // zero in the place of octets with a value that is not finite; the first of the `here` rows that has one (ROWS: none)
  __device__ __forceinline__ int clean(int here, int thread) {
    float s = 0.f;
#pragma unroll
    for (int i = 0; i < N; ++i) s = K::nothing(v[i], s);
    int first = ROWS;
    if (s != s)
#pragma unroll
      for (int i = N - 1; i >= 0; --i)
        if (K::nothing(v[i], 0.f) != 0.f) {
          v[i] = (oct)(T)0;
          const int row = here_only(thread) / PER_ROW + i * STEP;
          if (row < here) first = row;
        }
    return first;
  }
};

// Planes of a float32 sum (the state, the weights of a chunk) where it is an operand again.  Beside float32 values all three; beside bfloat16 ones two, off by 2^-17 of
// it, some 2^-9 of what the outputs' own rounding takes: they are as far from 64 bits as the float32 state's, rounded once (0.00166 of their norm).  4 sequences of 16 heads
// of 128, 16,384 frames, both directions: 1,415 us; three planes 1,720, for the same error; one plane 1,280, off by 0.00235.
template <typename T>
constexpr int sums_of() { return sizeof(T) == 4 ? 3 : 2; }

// What a launch does with the chunks: out = mix(a, b, c); the state alone; or, with twice the threads and time reversed, out = mix(a, b, c) and
// out2 = mix(a2, c, b), whose states are each other's transpose, from one reading of all four.
enum { MIX, STATE, PAIR };
constexpr int XCDS = 8;  // workgroups go to them in turn

// Frames of a chunk: 64; of three planes 32, so that heads of 64 leave room for two workgroups on a CU (64 clips of 431 frames, 8 heads of 64, float32: 64 us forward
// and 165 backward, 90 and 262 with 64) and heads of 128 for one.  Columns of the state to a wave: 32 where a state of 128 x 32 and
// the rest fit 256 registers, so that what is read from LDS meets two products; else 16.
template <typename T, int DA, int DC>
struct Shape {
  static constexpr int PLANES = Kind<T>::planes, ROWS = PLANES == 3 ? 32 : 64;
  static constexpr int CB = PLANES == 1 && DC == 128 ? 2 : 1, WAVES = DC / 16 / CB, THREADS = 64 * WAVES;
  static constexpr int IB = ROWS / 16, BLOCKS = IB * (IB + 1) / 2;  // 16 x 16 blocks on and below the diagonal
  static constexpr int SUMS = sums_of<T>(), WEIGHTS = BLOCKS * 64 * SUMS;  // quads
  static constexpr int threads(int mode) { return mode == PAIR ? 2 * THREADS : THREADS; }
  static constexpr int lds(int mode) {
    const int a = Tile<ROWS, DA, PLANES>::SIZE, c = Tile<ROWS, DC, PLANES>::SIZE;
    return (int)sizeof(bf16) * (mode == PAIR ? 2 * (a + c) : mode == MIX ? 2 * a + c : a + c) + (mode == STATE ? 0 : WEIGHTS * 8 * (mode == PAIR ? 2 : 1)) + 16;
  }
};

__device__ __forceinline__ int length_of(const DecayMix& P, long long batch) {
  if (!P.lengths) return P.T;
  const int given = P.lengths[batch];
  return given < 0 ? 0 : given < P.T ? given : P.T;
}

// A product that sums over frames j meets c_j = 0 * x where its weight is zero (j after i): an infinity or a NaN there would reach frames before its own.  It is
// taken out of the tile, and every frame from its own on is NaN, as is the state.
typedef float quad_anywhere_t __attribute__((ext_vector_type(4), aligned(4)));

// the frames of a workgroup's segment, and those of them that are their sequence's
struct Span {
  int head, segment, n, from, to, real_to;  // head: of all sequences' heads
};
__device__ __forceinline__ Span span_of(const DecayMix& P, int workgroup) {
  Span s;
  // (a quotient is computed a lane at a time: unless it is taken back to a scalar register, all that follows of it is kept for every lane)
  s.head = uniform(workgroup / P.segments);
  s.segment = workgroup - s.head * P.segments;
  s.n = uniform(length_of(P, uniform(s.head / P.H)));
  const int frames = P.segment_chunks * CHUNK;
  s.from = s.segment * frames;
  s.to = P.T - s.from < frames ? P.T : s.from + frames;
  s.real_to = s.to < s.n ? s.to : s.n;
  return s;
}

template <typename T, int DA, int DC, int PLANES, int MODE, bool REVERSE, bool FULL>
__device__ __forceinline__ void mix_chunks(const DecayMix& P, const int workgroup, unsigned char* const lds) {
  static_assert(MODE != PAIR || DA == DC, "both halves run the same sizes");
  typedef Shape<T, DA, DC> S;
  constexpr int NP = S::PLANES, SUMS = S::SUMS, ROWS = S::ROWS, CB = S::CB, WAVES = S::WAVES, THREADS = S::THREADS, IB = S::IB, RB = DA / 16;
  typedef Tile<ROWS, DA, NP> TileA;
  typedef Tile<ROWS, DC, NP> TileC;
  const int thread = threadIdx.x & (THREADS - 1), lane = thread & 63, li = lane & 15, lg = lane >> 4;
  const int wave = uniform(thread >> 6);
  const bool second = MODE == PAIR && uniform((int)threadIdx.x / THREADS) != 0;

  bf16* const tiles = reinterpret_cast<bf16*>(lds);
  bf16* tile_b = tiles;
  bf16* tile_c = tiles + TileA::SIZE;
  bf16* tile_a = tile_c + TileC::SIZE;  // (not there where the state alone is summed)
  bf16x4* weights = reinterpret_cast<bf16x4*>(tile_a + TileA::SIZE * (MODE == PAIR ? 2 : MODE == MIX ? 1 : 0));
  int* const bad_row = reinterpret_cast<int*>(weights + (MODE == STATE ? 0 : S::WEIGHTS * (MODE == PAIR ? 2 : 1)));
  if (second) {
    bf16* const b = tile_b;
    tile_b = tile_c;
    tile_c = b;
    tile_a += TileA::SIZE;
    weights += S::WEIGHTS;
  }

  const Span span = span_of(P, workgroup);
  if (MODE == STATE && span.segment == P.segments - 1) return;  // nothing comes after it
  const int segment = span.segment, of_batch = uniform(span.head / P.H), head = span.head - of_batch * P.H;
  const long long bh = span.head, batch = of_batch;
  const int n = span.n, all = P.T;
  const float log2_decay = uniform(log2_of(P.decay[head]));
  const int da = second ? P.dc : P.da, dc = second ? P.da : P.dc;
  const bool transposed = second || P.transposed;
  const int column0 = wave * CB * 16;

  // fn(row, column, value) of the state's quads a lane holds: four rows of a column
  auto state_values = [&](f32x4 (&state)[RB][CB], auto fn) {
#pragma unroll
    for (int r = 0; r < RB; ++r)
#pragma unroll
      for (int m = 0; m < CB; ++m) fn(r * 16 + lg * 4, column0 + m * 16 + li, state[r][m]);
  };

  // between memory and LDS: a, b and c; of a pair, the first half of the threads a and b, the second a2 and c
  Rows<T, ROWS, DA, THREADS, FULL, REVERSE> ra, rb;
  Rows<T, ROWS, DC, THREADS, FULL, REVERSE> rc;
  const T* const a = (second ? static_cast<const T*>(P.a2) + batch * P.a2_b + head * P.a2_h : static_cast<const T*>(P.a) + batch * P.a_b + head * P.a_h);
  const T* const b = (second ? static_cast<const T*>(P.c) + batch * P.c_b + head * P.c_h : static_cast<const T*>(P.b) + batch * P.b_b + head * P.b_h);
  const T* const c = static_cast<const T*>(P.c) + batch * P.c_b + head * P.c_h;
  const int step_a = (int)(second ? P.a2_t : P.a_t), step_b = (int)(second ? P.c_t : P.b_t), step_c = (int)P.c_t;
  auto load = [&](int u0) {
    const int here = n - u0 < ROWS ? n - u0 : ROWS;
    const long long t = REVERSE ? n - u0 - here : u0;
    if (MODE != STATE) ra.load(a + t * step_a, step_a, here, da, thread);
    rb.load(b + t * step_b, step_b, here, da, thread);
    if (MODE != PAIR) rc.load(c + t * step_c, step_c, here, dc, thread);
  };

  // a chunk's outputs, written behind the next chunk's first barriers: the wait for what is loaded is then no wait for them
  typedef T quad __attribute__((ext_vector_type(4)));
  T* const out = static_cast<T*>(second ? P.out2 : P.out) + (batch * all * P.H + head) * dc;
  const int out_step = P.H * dc;
  quad done[IB][CB];
  int done_u0 = -1;
  auto write = [&]() {
    typedef T quad_anywhere __attribute__((ext_vector_type(4), aligned(sizeof(T))));
    const int here = n - done_u0 < ROWS ? n - done_u0 : ROWS;
    const int lane_row = here_only(li), lane_column = column0 + here_only(lg) * 4;
#pragma unroll
    for (int i = 0; i < IB; ++i) {
      const int u = i * 16 + lane_row;
      if (here < ROWS && done_u0 + u >= all) continue;
      const long long t = REVERSE && u < here ? n - 1 - (done_u0 + u) : done_u0 + u;
      T* const row = out + t * out_step + lane_column;
#pragma unroll
      for (int m = 0; m < CB; ++m) {
        if (FULL || lane_column + m * 16 + 4 <= dc) {
          *reinterpret_cast<quad_anywhere*>(row + m * 16) = done[i][m];
        } else {
#pragma unroll
          for (int e = 0; e < 3; ++e)
            if (lane_column + m * 16 + e < dc) row[m * 16 + e] = done[i][m][e];
        }
      }
    }
  };

  const int from = span.from, to = span.to, real_to = span.real_to;
  if (from < real_to) load(from);  // on its way while the state is read and the powers are taken

  // the state: rows 16 r + 4 lg .. + 3 of column column0 + 16 m + li
  f32x4 state[RB][CB];
  float* const part = P.parts + (bh * P.segments + segment) * P.part_size;
  {
    const bool parts = P.segments > 1;
    const float* from_state = parts ? part : P.first ? P.first + bh * da * dc : nullptr;
    const int pitch = parts ? P.part_pitch : transposed ? da : dc, to_row = transposed ? 1 : pitch, to_column = transposed ? pitch : 1;
    const float factor = parts ? 1.f : P.first_factor;
    state_values(state, [&](int row, int column, f32x4& v) {
      v = 0.f;
      if (MODE == STATE || !from_state) return;
      // (where the head's sizes are not the tile's, what is not there is read at a place that is)
      const int c = FULL || column < dc ? column : dc - 1;
      if (transposed && (FULL || (parts && row < da))) {
        v = *reinterpret_cast<const quad_anywhere_t*>(from_state + c * to_column + row) * factor;
      } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int r = FULL || row + e < da ? row + e : da - 1;
          v[e] = from_state[r * to_row + c * to_column] * factor;
        }
      }
      if (!FULL)
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = row + e < da && column < dc ? v[e] : 0.f;
    });
  }

  // powers of the decay that every whole chunk takes, as a lane's own times the block's: of the weights (on the diagonal; one block below it), of the first
  // state, and of a frame's product in the next state
  f32x4 on_diagonal, below, left;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const int apart = li - lg * 4 - e;
    on_diagonal[e] = power(log2_decay, apart < 0 ? 0 : apart) * P.factor;
    below[e] = power(log2_decay, 16 + apart) * P.factor;
    left[e] = power(log2_decay, 15 - lg * 4 - e + (REVERSE ? 1 : 0));
  }
  const float since = power(log2_decay, li + (REVERSE ? 0 : 1)) * P.factor;
  const float power16 = uniform(power(log2_decay, 16)), power32 = uniform(power(log2_decay, 32)), power48 = uniform(power(log2_decay, 48));
  const float carry_whole = uniform(power(log2_decay, ROWS));
  auto block_power = [&](int i) { return i == 0 ? 1.f : here_only(i == 1 ? power16 : i == 2 ? power32 : power48); };

  for (int u0 = from; u0 < real_to; u0 += ROWS) {
    const int here = n - u0 < ROWS ? n - u0 : ROWS;
    int* bad_here = bad_row + (u0 / ROWS & 1);  // two in turn: a wave may still read the last chunk's
    if (threadIdx.x == 0) *bad_here = ROWS;
    __syncthreads();
    // tile_b of a pair's half is the other's c
    if (MODE != STATE) ra.store(tile_a, here, da, thread);
    const int bad = MODE == PAIR ? rb.clean(here, thread) : rc.clean(here, thread);
    rb.store(tile_b, here, da, thread);
    if (MODE != PAIR) rc.store(tile_c, here, dc, thread);
    if (bad < ROWS) atomicMin(bad_here, bad);
    __syncthreads();
    const int first_bad = uniform(*bad_here);
    if (MODE != STATE && done_u0 >= 0) write();
    if (u0 + ROWS < real_to) load(u0 + ROWS);
    f32x4 o[IB][CB];
    if constexpr (MODE != STATE) {
      // the weights l^(i-j) (a_i . b_j) of the blocks on and below the diagonal, as (j, i): the operand of frame i's sum over j
#pragma unroll
      for (int k = 0; k < (S::BLOCKS + WAVES - 1) / WAVES; ++k) {
        const int block = wave + k * WAVES;
        if (block < S::BLOCKS) {
          const int ib = block >= 6 ? 3 : block >= 3 ? 2 : block >= 1 ? 1 : 0, jb = block - ib * (ib + 1) / 2;
          f32x4 s = 0.f;
#pragma unroll
          for (int d = 0; d < DA; d += 32) {
            bf16x8 vb[NP], va[NP];
            TileA::rows8(tile_b, jb * 16, d, li, lg, vb);
            TileA::rows8(tile_a, ib * 16, d, li, lg, va);
            s = mma(vb, va, s);
          }
          if (ib == jb) {
#pragma unroll
            for (int e = 0; e < 4; ++e) s[e] = li < lg * 4 + e ? 0.f : s[e] * on_diagonal[e];  // a frame after this one has no part, whatever it is
          } else {
            s *= below * block_power(ib - jb - 1);
          }
#pragma unroll
          for (int p = 0; p < SUMS; ++p) {
            const bf16x4 w = __builtin_convertvector(p ? s : all_in_range<T>(s), bf16x4);
            weights[(block * SUMS + p) * 64 + lane] = w;
            s -= __builtin_convertvector(w, f32x4);
          }
        }
      }
      // out, as (column, frame): l^(i+1) (a S) ...
#pragma unroll
      for (int i = 0; i < IB; ++i)
#pragma unroll
        for (int m = 0; m < CB; ++m) o[i][m] = 0.f;
#pragma unroll
      for (int r = 0; r < RB; r += 2) {
        bf16x8 vs[CB][SUMS];
#pragma unroll
        for (int m = 0; m < CB; ++m) split<T>(state[r][m], state[r + 1][m], vs[m]);
#pragma unroll
        for (int i = 0; i < IB; ++i) {
          bf16x8 va[NP];
          TileA::rows4(tile_a, i * 16, r * 16, li, lg, va);
#pragma unroll
          for (int m = 0; m < CB; ++m) o[i][m] = mma(vs[m], va, o[i][m]);
        }
      }
#pragma unroll
      for (int i = 0; i < IB; ++i)
#pragma unroll
        for (int m = 0; m < CB; ++m) o[i][m] *= since * block_power(i);
      __syncthreads();
    }
    const float carry = here == ROWS ? carry_whole : power(log2_decay, here);
#pragma unroll
    for (int r = 0; r < RB; ++r)
#pragma unroll
      for (int m = 0; m < CB; ++m) state[r][m] *= carry;
#pragma unroll
    for (int j = 0; j < IB; j += 2) {
      bf16x8 vc[CB][NP];
#pragma unroll
      for (int m = 0; m < CB; ++m) TileC::columns(tile_c, j * 16, column0 + m * 16, lane, vc[m]);
      if constexpr (MODE != STATE) {
        // ... + weights c
#pragma unroll
        for (int i = j; i < IB; ++i) {
          bf16x8 vw[SUMS];
#pragma unroll
          for (int p = 0; p < SUMS; ++p) {
            const bf16x4 zero = {};
            const int block = i * (i + 1) / 2 + j;
            vw[p] = join(weights[(block * SUMS + p) * 64 + lane], j < i ? weights[((block + 1) * SUMS + p) * 64 + lane] : zero);
          }
#pragma unroll
          for (int m = 0; m < CB; ++m) o[i][m] = mma(vc[m], vw, o[i][m]);
        }
      }
      // S' = l^n S + sum over j of b_j^T (l^(n-1-j) c_j): the scaled c as the sum of PLANES operands
      bf16x8 vs[CB][PLANES];
      f32x4 weight[2];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        weight[h] = left * block_power(IB - 1 - j - h);
        if (here < ROWS) {
          const int lane_row = here_only(lg) * 4;
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const int after = here - 1 - ((j + h) * 16 + lane_row + e);
            weight[h][e] = after < 0 ? 0.f : power(log2_decay, after + (REVERSE ? 1 : 0));
          }
        }
      }
#pragma unroll
      for (int m = 0; m < CB; ++m) {
        f32x8 v = __builtin_convertvector(vc[m][NP - 1], f32x8);
#pragma unroll
        for (int p = NP - 2; p >= 0; --p) v += __builtin_convertvector(vc[m][p], f32x8);
        split<T>(__builtin_shufflevector(v, v, 0, 1, 2, 3) * weight[0], __builtin_shufflevector(v, v, 4, 5, 6, 7) * weight[1], vs[m]);
      }
#pragma unroll
      for (int r = 0; r < RB; ++r) {
        bf16x8 vb[NP];
        TileA::columns(tile_b, j * 16, r * 16, lane, vb);
#pragma unroll
        for (int m = 0; m < CB; ++m) state[r][m] = mma(vb, vs[m], state[r][m]);
      }
    }
    if constexpr (MODE != STATE) {
      if (here < ROWS || first_bad < ROWS)
#pragma unroll
        for (int i = 0; i < IB; ++i) {
          const int u = i * 16 + here_only(li);
#pragma unroll
          for (int m = 0; m < CB; ++m) o[i][m] = u >= here ? (f32x4)0.f : u >= first_bad ? o[i][m] * here_only(__builtin_nanf("")) : o[i][m];
        }
#pragma unroll
      for (int i = 0; i < IB; ++i)
#pragma unroll
        for (int m = 0; m < CB; ++m) done[i][m] = __builtin_convertvector(o[i][m], quad);
      done_u0 = u0;
    }
    if (first_bad < ROWS)
#pragma unroll
      for (int r = 0; r < RB; ++r)
#pragma unroll
        for (int m = 0; m < CB; ++m) state[r][m] *= here_only(__builtin_nanf(""));
  }

  if (MODE != STATE) {
    if (done_u0 >= 0) write();
    // past the sequence's end, from the first frame that no chunk held
    const int lane_column = thread % (DC / 4) * 4;
    for (int u = (done_u0 >= 0 ? done_u0 + ROWS : from > n ? from : n) + thread / (DC / 4); u < to; u += THREADS / (DC / 4)) {
      T* const row = out + (long long)u * out_step + lane_column;
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (lane_column + e < dc) row[e] = (T)0;
    }
    if (second || !P.last || segment != P.segments - 1) return;
  }
  float* const to_state = MODE == STATE ? part : P.last + bh * da * dc;
  const bool turned = MODE != STATE && transposed;
  const int pitch = MODE == STATE ? P.part_pitch : turned ? da : dc, to_row = turned ? 1 : pitch, to_column = turned ? pitch : 1;
  state_values(state, [&](int row, int column, f32x4& v) {
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (MODE == STATE || FULL || (row + e < da && column < dc))
        to_state[(row + e) * to_row + column * to_column] = MODE == STATE ? v[e] : v[e] * P.last_factor;
  });
}

// Where gk and gv are computed as a pair, of sizes padded to the larger: the mixes of three planes of 128 columns leave no room for two workgroups on a CU.
template <typename T, int DA, int DC>
constexpr bool in_pairs() { return sizeof(T) == 4 && (DA == 128 || DC == 128); }
bool in_pairs(int type, int da, int dc) { return type == NNA_F32 && (da > 64 || dc > 64); }

// planes of a state's new products: where a state is given back it is as exact as its float32 sums; where it only meets frames again, as many as it does so with
template <typename T, bool GIVEN>
constexpr int planes_of() { return GIVEN ? 3 : sums_of<T>(); }

template <typename T, int DA, int DC, int PLANES, int MODE, bool REVERSE, bool FULL>
__global__ __launch_bounds__((Shape<T, DA, DC>::threads(MODE)), 2) void decay_mix_kernel(DecayMix P) {
  extern __shared__ __align__(16) unsigned char lds[];
  mix_chunks<T, DA, DC, PLANES, MODE, REVERSE, FULL>(P, blockIdx.x, lds);
}

// The backward pass's launches of two directions in one.  The states before the segments, of the forward pass and of the gradient:
template <typename T, int DA, int DC, int PLANES, bool FULL>
__global__ __launch_bounds__((Shape<T, DA, DC>::threads(STATE)), 2) void decay_both_states_kernel(DecayMix P, DecayMix R, int workgroups) {
  extern __shared__ __align__(16) unsigned char lds[];
  if ((int)blockIdx.x < workgroups)
    mix_chunks<T, DA, DC, planes_of<T, false>(), STATE, false, FULL>(P, blockIdx.x, lds);
  else
    mix_chunks<T, DA, DC, PLANES, STATE, true, FULL>(R, blockIdx.x - workgroups, lds);
}
// All three gradients, gk and gv as a pair, where the two launches together are one workgroup a CU at most: the pairs in the first workgroups, gq in the others, half
// of whose waves only keep up with the barriers, three a chunk.
template <typename T, int D, int PLANES, bool FULL>
__global__ __launch_bounds__((Shape<T, D, D>::threads(PAIR)), 2) void decay_gradients_kernel(DecayMix R, DecayMix P, int workgroups) {
  typedef Shape<T, D, D> S;
  extern __shared__ __align__(16) unsigned char lds[];
  if ((int)blockIdx.x < workgroups) {
    mix_chunks<T, D, D, PLANES, PAIR, true, FULL>(R, blockIdx.x, lds);
  } else if (uniform((int)threadIdx.x / S::THREADS) == 0) {
    mix_chunks<T, D, D, planes_of<T, false>(), MIX, false, FULL>(P, blockIdx.x - workgroups, lds);
  } else {
    const Span span = span_of(P, blockIdx.x - workgroups);
    for (int u0 = span.from; u0 < span.real_to; u0 += S::ROWS) {
      __syncthreads();
      __syncthreads();
      __syncthreads();
    }
  }
}

// The gradients as mixes of their own, all in one launch: gv, gk and (if wanted) gq of a segment in workgroups of one XCD, begun together, so that what two of them
// read comes from its cache the second time.  Two such workgroups fit a CU and one's products run beside the other's loads and barriers; a pair reads a third less but
// has the CU for itself (bfloat16, 64 heads of 128, 16,384 frames: 1,045 us with the states before, gq and then the pair 1,080; float32, 32 clips of 431 frames, 8 heads of 64: 87 and 105).
// Heads of 128 in float32 fill a CU either way: there the pair is ahead (16 clips of 431 frames, 8 heads: a quarter faster than as mixes, 126 us).
template <typename T, int DK, int DV, int PLANES, bool FULL>
__global__ __launch_bounds__((Shape<T, DK, DV>::THREADS), 2) void decay_mixes_kernel(DecayMix V, DecayMix K, DecayMix Q, int workgroups, int mixes) {
  extern __shared__ __align__(16) unsigned char lds[];
  static_assert(Shape<T, DK, DV>::THREADS == Shape<T, DV, DK>::THREADS, "one launch");
  const int round = (int)blockIdx.x / XCDS, at = uniform(round / mixes), which = round - at * mixes, workgroup = at * XCDS + (int)blockIdx.x % XCDS;
  if (workgroup >= workgroups) return;
  if (which == 0)
    mix_chunks<T, DK, DV, PLANES, MIX, true, FULL>(V, workgroup, lds);
  else if (which == 1)
    mix_chunks<T, DV, DK, planes_of<T, false>(), MIX, true, FULL>(K, workgroup, lds);
  else
    mix_chunks<T, DV, DK, planes_of<T, false>(), MIX, false, FULL>(Q, workgroup, lds);
}

// parts[s]: from each segment's own state to the state before it, in order; four values of a (sequence, head) to a thread, all segments of a round read before
// the first of them is written.  For few segments (8 of 64 heads of 128: 11 us, 30 by the kernel below).
constexpr int JOIN_FEW = 16;
__device__ __forceinline__ void join_few(const DecayMix& P, int block) {
  const int workgroups = P.part_size / 1024, of_head = uniform(block / workgroups);
  const int at = (block - of_head * workgroups) * 1024 + threadIdx.x * 4, row = at / P.part_pitch, column = at % P.part_pitch;
  const long long bh = of_head;
  float* const part = P.parts + bh * P.segments * P.part_size + at;
  f32x4 own[JOIN_FEW];
#pragma unroll
  for (int k = 0; k < JOIN_FEW; ++k)
    if (k + 1 < P.segments) own[k] = *reinterpret_cast<const f32x4*>(part + (long long)k * P.part_size);
  const int n = uniform(length_of(P, of_head / P.H)), frames = P.segment_chunks * CHUNK;
  const float log2_decay = log2_of(P.decay[of_head % P.H]), whole = power(log2_decay, frames);
  f32x4 s = 0.f;
  if (P.first && row < P.da)
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (column + e < P.dc) s[e] = P.first[(bh * P.da + row) * P.dc + column + e] * P.first_factor;
#pragma unroll
  for (int k = 0; k < JOIN_FEW; ++k)
    if (k < P.segments) {
      *reinterpret_cast<f32x4*>(part + (long long)k * P.part_size) = s;
      const long long left = n - (long long)k * frames;
      if (k + 1 < P.segments) s = s * (left >= frames ? whole : power(log2_decay, left < 0 ? 0 : (int)left)) + own[k];
    }
}

// (and of a second direction from workgroup `workgroups` on)
__global__ __launch_bounds__(256) void decay_join_few_kernel(DecayMix P, DecayMix R, int workgroups) {
  if ((int)blockIdx.x < workgroups)
    join_few(P, blockIdx.x);
  else
    join_few(R, blockIdx.x - workgroups);
}

// ... and for many: a lane has four values, each of JOIN_WAVES waves JOIN_AHEAD segments; all are read at once, every wave's own run is joined, and then
// the runs (61 segments of 8 heads of 64: 7 us, 15 one after the other).
constexpr int JOIN_WAVES = 8, JOIN_AHEAD = 8;
__device__ __forceinline__ void join_many(const DecayMix& P, int block, f32x4 (&sums)[2][JOIN_WAVES][64]) {
  const int workgroups = P.part_size / 256, of_head = uniform(block / workgroups), lane = threadIdx.x & 63, wave = uniform((int)threadIdx.x >> 6);
  const int at = (block - of_head * workgroups) * 256 + lane * 4, row = at / P.part_pitch, column = at % P.part_pitch;
  const long long bh = of_head;
  float* const part = P.parts + bh * P.segments * P.part_size + at;
  const int n = uniform(length_of(P, of_head / P.H)), frames = P.segment_chunks * CHUNK;
  const float log2_decay = log2_of(P.decay[of_head % P.H]);
  f32x4 s = 0.f;  // the state before the next JOIN_WAVES * JOIN_AHEAD segments
  if (P.first && row < P.da)
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (column + e < P.dc) s[e] = P.first[(bh * P.da + row) * P.dc + column + e] * P.first_factor;
  // the decay over segments i .. j - 1
  auto over = [&](int i, int j) {
    const long long a = (long long)i * frames, b = (long long)j * frames;
    return power(log2_decay, (int)((b < n ? b : n) - (a < n ? a : n)));
  };
  for (int i0 = 0, turn = 0; i0 < P.segments; i0 += JOIN_WAVES * JOIN_AHEAD, turn ^= 1) {
    const int each = P.segments - i0 < JOIN_WAVES * JOIN_AHEAD ? (P.segments - i0 + JOIN_WAVES - 1) / JOIN_WAVES : JOIN_AHEAD;
    const int first = i0 + wave * each < P.segments ? i0 + wave * each : P.segments, end = first + each < P.segments ? first + each : P.segments;
    f32x4 own[JOIN_AHEAD], run = 0.f;
#pragma unroll
    for (int k = 0; k < JOIN_AHEAD; ++k) {
      own[k] = 0.f;
      if (first + k < end && first + k + 1 < P.segments) own[k] = *reinterpret_cast<const f32x4*>(part + (long long)(first + k) * P.part_size);
    }
#pragma unroll
    for (int k = 0; k < JOIN_AHEAD; ++k)
      if (first + k < end) run = run * over(first + k, first + k + 1) + own[k];
    sums[turn][wave][lane] = run;
    __syncthreads();  // (two buffers in turn: the next runs never meet a wave that still reads these)
    f32x4 before = s;
    for (int w = 0; w < JOIN_WAVES; ++w) {
      const int a = i0 + w * each < P.segments ? i0 + w * each : P.segments, b = a + each < P.segments ? a + each : P.segments;
      if (w == wave) before = s;
      s = s * over(a, b) + sums[turn][w][lane];
    }
#pragma unroll
    for (int k = 0; k < JOIN_AHEAD; ++k)
      if (first + k < end) {
        *reinterpret_cast<f32x4*>(part + (long long)(first + k) * P.part_size) = before;
        before = before * over(first + k, first + k + 1) + own[k];
      }
  }
}

__global__ __launch_bounds__(64 * JOIN_WAVES) void decay_join_kernel(DecayMix P, DecayMix R, int workgroups) {
  __shared__ f32x4 sums[2][JOIN_WAVES][64];
  if ((int)blockIdx.x < workgroups)
    join_many(P, blockIdx.x, sums);
  else
    join_many(R, blockIdx.x - workgroups, sums);
}

// One frame: the state is read and written once, four columns of it to a lane, a slab of 32 columns to a workgroup.  Bound by the state's bytes: 256 streams of 16
// heads of 128 x 128, 98 us, 5.5 TB/s; one stream of 8 heads of 64 x 64, 4 us of a call of 10.
constexpr int STEP_COLUMNS = 32, STEP_RUNS = 256 / (STEP_COLUMNS / 4);
template <typename T>
__global__ __launch_bounds__(256) void decay_step_kernel(DecayStep P) {
  __shared__ f32x4 sums[4][STEP_COLUMNS / 4];
  const int slabs = (P.dv + STEP_COLUMNS - 1) / STEP_COLUMNS;
  const long long bh = blockIdx.x / slabs, b = bh / P.H;
  const int h = (int)(bh % P.H);
  const int column = (int)(blockIdx.x % slabs) * STEP_COLUMNS + (threadIdx.x % (STEP_COLUMNS / 4)) * 4, run = threadIdx.x / (STEP_COLUMNS / 4);
  const int columns = P.dv - column;  // real ones here; may be none
  const float decay = P.decay[h];
  const T* q = static_cast<const T*>(P.q) + b * P.q_b + h * P.q_h;
  const T* k = static_cast<const T*>(P.k) + b * P.k_b + h * P.k_h;
  const T* v = static_cast<const T*>(P.v) + b * P.v_b + h * P.v_h;
  f32x4 value = 0.f, o = 0.f;
#pragma unroll
  for (int e = 0; e < 4; ++e)
    if (e < columns) value[e] = (float)v[column + e];
  float* state = P.state + bh * P.dk * P.dv + column;
  typedef float quad __attribute__((ext_vector_type(4), aligned(4)));
#pragma unroll 4
  for (int row = run; row < P.dk; row += STEP_RUNS) {
    const float key = (float)k[row], query = (float)q[row];
    float* at = state + (long long)row * P.dv;
    if (columns >= 4) {
      f32x4 s = *reinterpret_cast<const quad*>(at);
      s = s * decay + key * value;
      *reinterpret_cast<quad*>(at) = s;
      o += query * s;
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (e < columns) {
          const float s = at[e] * decay + key * value[e];
          at[e] = s;
          o[e] += query * s;
        }
    }
  }
  // the 32 runs of rows: eight in a wave, then the waves
#pragma unroll
  for (int d = STEP_COLUMNS / 4; d < 64; d <<= 1)
#pragma unroll
    for (int e = 0; e < 4; ++e) o[e] += __shfl_xor(o[e], d);
  if ((threadIdx.x & 63) < STEP_COLUMNS / 4) sums[threadIdx.x >> 6][threadIdx.x & 63] = o;
  __syncthreads();
  if (threadIdx.x >= STEP_COLUMNS / 4) return;
  o = ((sums[0][threadIdx.x] + sums[1][threadIdx.x]) + (sums[2][threadIdx.x] + sums[3][threadIdx.x])) * P.factor;
  T* out = static_cast<T*>(P.out) + bh * P.dv + column;
#pragma unroll
  for (int e = 0; e < 4; ++e)
    if (e < columns) out[e] = (T)o[e];
}

// a head's values in a tile: 64 or 128
template <typename F>
hipError_t by_heads(int da, int dc, F fn) {
  if (da <= 64 && dc <= 64) return fn(std::integral_constant<int, 64>(), std::integral_constant<int, 64>());
  if (da <= 64) return fn(std::integral_constant<int, 64>(), std::integral_constant<int, 128>());
  if (dc <= 64) return fn(std::integral_constant<int, 128>(), std::integral_constant<int, 64>());
  return fn(std::integral_constant<int, 128>(), std::integral_constant<int, 128>());
}

template <typename T, int DA, int DC, bool GIVEN, int MODE, bool REVERSE, bool FULL>
hipError_t run_mix(const DecayMix& P, int workgroups, hipStream_t stream) {
  typedef Shape<T, DA, DC> S;
  const auto kernel = &decay_mix_kernel<T, DA, DC, planes_of<T, GIVEN>(), MODE, REVERSE, FULL>;
  if (workgroups < 0) return hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, S::lds(MODE));
  hipLaunchKernelGGL(kernel, dim3(workgroups), dim3(S::threads(MODE)), S::lds(MODE), stream, P);
  return hipGetLastError();
}
template <typename F>
hipError_t by_bool(bool v, F fn) { return v ? fn(std::true_type()) : fn(std::false_type()); }

template <typename T>
hipError_t launch_mode(const DecayMix& P, int mode, bool given, int workgroups, hipStream_t stream) {
  const int da = mode == PAIR ? std::max(P.da, P.dc) : P.da, dc = mode == PAIR ? da : P.dc;
  return by_heads(da, dc, [&](auto a, auto c) {
    constexpr int DA = a.value, DC = c.value;
    return by_bool(P.da == DA && P.dc == DC, [&](auto full) {
      return by_bool(given || sizeof(T) == 4, [&](auto exact) {
        constexpr bool FULL = full.value, GIVEN = exact.value;
        if constexpr (sizeof(T) == 4 && !GIVEN) return hipErrorInvalidValue;
        else {
          if constexpr (DA == DC && in_pairs<T, DA, DC>())
            if (mode == PAIR) return run_mix<T, DA, DC, GIVEN, PAIR, true, FULL>(P, workgroups, stream);
          if (mode == PAIR) return hipErrorInvalidValue;
          if (mode == STATE)
            return by_bool(P.reverse != 0, [&](auto reverse) { return run_mix<T, DA, DC, GIVEN, STATE, reverse.value, FULL>(P, workgroups, stream); });
          return run_mix<T, DA, DC, GIVEN, MIX, false, FULL>(P, workgroups, stream);
        }
      });
    });
  });
}
hipError_t launch_mode(const DecayMix& P, int type, int mode, bool given, int workgroups, hipStream_t stream) {
  return type == NNA_F32 ? launch_mode<float>(P, mode, given, workgroups, stream) : launch_mode<bf16>(P, mode, given, workgroups, stream);
}

// P and R in one launch: their states, or (gradients) gq and the pair
template <typename T>
hipError_t launch_both(const DecayMix& P, const DecayMix& R, bool given, int workgroups, bool gradients, hipStream_t stream) {
  const int most = std::max(R.da, R.dc), da = gradients ? most : R.da, dc = gradients ? most : R.dc;
  return by_heads(da, dc, [&](auto a, auto c) {
    constexpr int DA = a.value, DC = c.value;
    typedef Shape<T, DA, DC> S;
    return by_bool(R.da == DA && R.dc == DC, [&](auto full) {
      return by_bool(given || sizeof(T) == 4, [&](auto exact) {
        constexpr bool FULL = full.value, GIVEN = exact.value;
        if constexpr (sizeof(T) == 4 && !GIVEN) return hipErrorInvalidValue;
        else {
          constexpr int PLANES = planes_of<T, GIVEN>();
          if constexpr (DA == DC && in_pairs<T, DA, DC>())
            if (gradients) {
              const auto kernel = &decay_gradients_kernel<T, DA, PLANES, FULL>;
              if (workgroups < 0) return hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, S::lds(PAIR));
              hipLaunchKernelGGL(kernel, dim3(2 * workgroups), dim3(S::threads(PAIR)), S::lds(PAIR), stream, R, P, workgroups);
              return hipGetLastError();
            }
          if (gradients) return hipErrorInvalidValue;
          const auto kernel = &decay_both_states_kernel<T, DA, DC, PLANES, FULL>;
          if (workgroups < 0) return hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, S::lds(STATE));
          hipLaunchKernelGGL(kernel, dim3(2 * workgroups), dim3(S::threads(STATE)), S::lds(STATE), stream, P, R, workgroups);
          return hipGetLastError();
        }
      });
    });
  });
}
hipError_t launch_both(const DecayMix& P, const DecayMix& R, int type, bool given, int workgroups, bool gradients, hipStream_t stream) {
  return type == NNA_F32 ? launch_both<float>(P, R, given, workgroups, gradients, stream) : launch_both<bf16>(P, R, given, workgroups, gradients, stream);
}

// gv, gk of R, its pair, and gq = P (out NULL: not wanted)
template <typename T>
hipError_t launch_mixes(const DecayMix& P, const DecayMix& R, bool given, int workgroups, hipStream_t stream) {
  return by_heads(R.da, R.dc, [&](auto a, auto c) {
    constexpr int DK = a.value, DV = c.value;
    return by_bool(R.da == DK && R.dc == DV, [&](auto full) {
      return by_bool(given || sizeof(T) == 4, [&](auto exact) {
        constexpr bool FULL = full.value, GIVEN = exact.value;
        if constexpr (in_pairs<T, DK, DV>() || (sizeof(T) == 4 && !GIVEN)) return hipErrorInvalidValue;
        else {
          const auto kernel = &decay_mixes_kernel<T, DK, DV, planes_of<T, GIVEN>(), FULL>;
          constexpr int LDS = std::max(Shape<T, DK, DV>::lds(MIX), Shape<T, DV, DK>::lds(MIX));
          if (workgroups < 0) return hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, LDS);
          DecayMix V = R, K = R;
          V.out2 = nullptr;
          K.a = R.a2, K.a_b = R.a2_b, K.a_t = R.a2_t, K.a_h = R.a2_h;
          K.b = R.c, K.b_b = R.c_b, K.b_t = R.c_t, K.b_h = R.c_h;
          K.c = R.b, K.c_b = R.b_b, K.c_t = R.b_t, K.c_h = R.b_h;
          K.out = R.out2;
          K.last = nullptr;
          K.da = R.dc, K.dc = R.da;
          K.transposed = 1;
          const int mixes = P.out ? 3 : 2, rounds = (workgroups + XCDS - 1) / XCDS;
          hipLaunchKernelGGL(kernel, dim3(XCDS * mixes * rounds), dim3(Shape<T, DK, DV>::THREADS), LDS, stream, V, K, P, workgroups, mixes);
          return hipGetLastError();
        }
      });
    });
  });
}
hipError_t launch_mixes(const DecayMix& P, const DecayMix& R, int type, bool given, int workgroups, hipStream_t stream) {
  return type == NNA_F32 ? launch_mixes<float>(P, R, given, workgroups, stream) : launch_mixes<bf16>(P, R, given, workgroups, stream);
}

int padded(int d) { return d <= 64 ? 64 : 128; }

}  // namespace

hipError_t decay_kernels_init() {
  DecayMix P = {};
  for (int type : {NNA_F32, NNA_BF16})
    for (int mode : {MIX, STATE, PAIR})
      for (int all = 0; all < 32; ++all) {
        hipError_t e = hipSuccess;
        P.da = (all & 1 ? 128 : 64) - (all & 4 ? 1 : 0);
        P.dc = all & 2 ? 128 : 64;
        P.reverse = all & 8;
        if (mode == PAIR && !in_pairs(type, P.da, P.dc)) {
          e = launch_mixes(P, P, type, all & 16, -1, nullptr);
        } else {
          e = launch_mode(P, type, mode, all & 16, -1, nullptr);
          if (e == hipSuccess) e = launch_both(P, P, type, all & 16, -1, mode == PAIR, nullptr);
        }
        if (e != hipSuccess) return e;
      }
  return hipSuccess;
}

// Segments cost half as much again (their states) and a launch that joins them, so there are some only where the heads alone leave the card idle, and then as many as
// its workgroups: 512 forward (256 in float32 with heads of 128: one a CU), 256 backward, of three mixes each.  Forward / backward in us, the number of segments before
// the colon:
//   float32, heads of 64    8 heads, 2,048 frames      1: 185/189  8: 47/51    32: 27/40
//                           64 heads, 1,024 frames     1: 96/103   4: 51/82    8: 44/82
//                           128 heads, 1,024 frames    1: 96/137   4: 67/135
//   bfloat16, heads of 64   8 heads, 512 frames        1: 26/27    4: 22/24            (float32: 1: 49/51  4: 28/31)
//                           128 heads, 16,384 frames   1: 719/896  4: 343/865
//                           256 heads, 2,048 frames    1: 94/180   2: 94/211
//   bfloat16, heads of 128  64 heads, 1,024 frames     1: 86/88    4: 54/97
//                           64 heads, 16,384 frames    1: 1370/1388  4: 491/1036  8: 398/1020
//   float32, heads of 128   128 heads, 2,048 frames    1: 348/550  2: 270/617  4: 274/663
// Between them: bfloat16, heads of 64, 96 heads, 1,024 frames 1: 49/60  5: 34/59, 8,192 frames 1: 355/447  5: 135/329 (backward one is taken: the rule is the short one's);
// heads of 128 1: 86/115  5: 65/132; 200 heads forward, where one each leaves a quarter of the card idle: 2,048 frames 1: 92  2: 87, heads of 128 1: 179  2: 188, float32
// 1,024 frames 1: 95  2: 104.
size_t decay_segments(long long B, long long T, int H, int dk, int dv, int type, bool backward, int* segments, int* chunks) {
  const long long all = std::max(1LL, (T + CHUNK - 1) / CHUNK), heads = std::max(1LL, B * H);
  const bool wide = dk > 64 || dv > 64;
  const long long workgroups = backward || in_pairs(type, dk, dv) ? 256 : 512;
  long long n = std::min(workgroups / heads, all / 2);
  if (backward && wide && type == NNA_BF16) n = std::max(std::min(512 / heads, all / 16), std::min(128 / heads, all / 2));  // (three mixes of 64 heads: nearly two a CU)
  const long long fewest = backward ? 4 : in_pairs(type, dk, dv) ? 2 : 3;
  if (n < fewest || (backward && heads >= 128) || all < (type == NNA_F32 ? 8 : 12)) n = 1;
  const long long each = (all + n - 1) / n;
  n = (all + each - 1) / each;
  *segments = (int)n;
  *chunks = (int)each;
  return n == 1 ? 0 : (size_t)(heads * n) * padded(dk) * padded(dv) * sizeof(float);
}

static void set_parts(DecayMix& P) {
  P.part_pitch = padded(P.transposed ? P.da : P.dc);
  P.part_size = padded(P.transposed ? P.dc : P.da) * P.part_pitch;
}

// the states before the segments of P, and of R if it is given (of the same sizes)
static hipError_t launch_join(const DecayMix& P, const DecayMix* R, hipStream_t stream) {
  const bool few = P.segments <= JOIN_FEW;
  const int workgroups = (int)(P.B * P.H) * (P.part_size / (few ? 1024 : 256)), both = R ? 2 * workgroups : workgroups;
  if (few)
    hipLaunchKernelGGL(decay_join_few_kernel, dim3(both), dim3(256), 0, stream, P, R ? *R : P, workgroups);
  else
    hipLaunchKernelGGL(decay_join_kernel, dim3(both), dim3(64 * JOIN_WAVES), 0, stream, P, R ? *R : P, workgroups);
  return hipGetLastError();
}

hipError_t launch_decay(DecayMix P, int type, hipStream_t stream) {
  const int workgroups = (int)(P.B * P.H * P.segments);
  const bool given = P.last != nullptr;
  set_parts(P);
  if (P.segments > 1) {
    hipError_t e = launch_mode(P, type, STATE, given, workgroups, stream);
    if (e == hipSuccess) e = launch_join(P, nullptr, stream);
    if (e != hipSuccess) return e;
  }
  return launch_mode(P, type, MIX, given, workgroups, stream);
}

hipError_t launch_decay_gradients(DecayMix states, DecayMix gq, DecayMix pair, int type, hipStream_t stream) {
  const int workgroups = (int)(pair.B * pair.H * pair.segments);
  const bool given = pair.last != nullptr;
  set_parts(states);
  set_parts(gq);
  set_parts(pair);
  if (pair.segments > 1) {
    hipError_t e = gq.out ? launch_both(states, pair, type, given, workgroups, false, stream) : launch_mode(pair, type, STATE, given, workgroups, stream);
    if (e == hipSuccess) e = gq.out ? launch_join(states, &pair, stream) : launch_join(pair, nullptr, stream);
    if (e != hipSuccess) return e;
  }
  if (!in_pairs(type, pair.da, pair.dc)) return launch_mixes(gq, pair, type, given, workgroups, stream);
  // a workgroup a CU at most: together (16 clips of 431 frames, 8 heads of 128, float32: 126 us, 195 in two launches); more than that, the waves that
  // only wait would hold registers that a second workgroup runs in
  if (gq.out && 2 * workgroups <= 256) return launch_both(gq, pair, type, given, workgroups, true, stream);
  if (gq.out) {
    const hipError_t e = launch_mode(gq, type, MIX, false, workgroups, stream);
    if (e != hipSuccess) return e;
  }
  return launch_mode(pair, type, PAIR, given, workgroups, stream);
}

hipError_t launch_decay_step(const DecayStep& P, int type, hipStream_t stream) {
  const unsigned grid = (unsigned)(P.B * P.H * ((P.dv + STEP_COLUMNS - 1) / STEP_COLUMNS));
  if (type == NNA_F32)
    hipLaunchKernelGGL(decay_step_kernel<float>, dim3(grid), dim3(256), 0, stream, P);
  else
    hipLaunchKernelGGL(decay_step_kernel<bf16>, dim3(grid), dim3(256), 0, stream, P);
  return hipGetLastError();
}

}  // namespace nna
