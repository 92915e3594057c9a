// Linear attention with a decay l for each head: S_t = l S_{t-1} + k_t^T v_t, o_t = scale q_t S_t.
//
// Taken a chunk of 64 frames at a time, the sums are products of small matrices: with S the state before the chunk, i and j its frames,
//   o_i = sum_{j <= i} l^(i-j) (q_i . k_j) v_j + l^(i+1) q_i S,      S' = l^n S + sum_j l^(n-1-j) k_j^T v_j.
// The gradients are the same mix of other arrays: gq = mix(go, v, k) with S^T, and, with time reversed and the state's gradient G in
// S's place, gk = mix(v, go, q) with G^T, gv = mix(k, q, go) with G.  One kernel runs them all: out = mix(a, b, c).
//
// A workgroup of four waves goes through the chunks of a (sequence, head), or of a segment of one where there are too few of them to
// fill the card (the segments' own states are then summed in a launch before, and joined in order).  Its state stays in registers, float32,
// a quarter of the columns to a wave; the chunk's a, b and c are in LDS.
#include "nna_decay.h"

namespace nna {

namespace {

typedef __bf16 bf16;
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef short s16x4 __attribute__((ext_vector_type(4)));

constexpr int CHUNK = DECAY_CHUNK;
constexpr int THREADS = 256, WAVES = THREADS / 64;

// A fragment: 16 of a matrix's k, lane (i, g) of (lane % 16, lane / 16) holds k = 4 g .. 4 g + 3 of row (A) or column (B) i.  It is how the 16 x 16
// accumulator of an earlier product lies (rows 4 g .. 4 g + 3 of column i), so that a state or a block of weights is an operand as it is.
template <typename T>
struct Kind;

template <>
struct Kind<bf16> {
  typedef bf16x4 frag;
  static constexpr int pad = 16;  // elements: a row's reads along it, and four rows' across, meet every bank once
  static constexpr int planes = 3;  // a float32 as this many operands: exactly
  typedef bf16 oct __attribute__((ext_vector_type(8), aligned(2)));
  static __device__ __forceinline__ f32x4 mma(frag a0, frag a1, frag b0, frag b1, f32x4 s) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_shufflevector(a0, a1, 0, 1, 2, 3, 4, 5, 6, 7), __builtin_shufflevector(b0, b1, 0, 1, 2, 3, 4, 5, 6, 7), s, 0, 0, 0);
  }
  // 8 consecutive k of a row, at p
  static __device__ __forceinline__ void row8(const bf16* p, frag& f0, frag& f1) {
    const bf16x8 v = *reinterpret_cast<const bf16x8*>(p);
    f0 = __builtin_shufflevector(v, v, 0, 1, 2, 3);
    f1 = __builtin_shufflevector(v, v, 4, 5, 6, 7);
  }
  static __device__ __forceinline__ frag row4(const bf16* p) { return *reinterpret_cast<const bf16x4*>(p); }
  // k along the rows: the fragment of rows k0 .. k0 + 15, columns n0 .. n0 + 15 of a tile
  static __device__ __forceinline__ frag column(const bf16* tile, int pitch, int k0, int n0, int lane) {
    const bf16* p = tile + (k0 + (lane >> 2)) * pitch + n0 + (lane & 3) * 4;
    return __builtin_bit_cast(bf16x4, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)p));
  }
  static __device__ __forceinline__ frag round(f32x4 v) { return __builtin_convertvector(v, bf16x4); }
  // v exactly, as the sum of three
  static __device__ __forceinline__ void split(f32x4 v, frag (&f)[3]) {
#pragma unroll
    for (int i = 0; i < 3; ++i) {
      f[i] = __builtin_convertvector(v, bf16x4);
      v -= __builtin_convertvector(f[i], f32x4);
    }
  }
  // whether one of the eight is not finite
  static __device__ __forceinline__ bool odd(oct v) {
    typedef unsigned u32x4 __attribute__((ext_vector_type(4)));
    const bf16x8 w = v;
    const u32x4 u = (__builtin_bit_cast(u32x4, w) & 0x7f807f80u) + 0x00800080u;
    return ((u[0] | u[1] | u[2] | u[3]) & 0x80008000u) != 0;
  }
};

template <>
struct Kind<float> {
  typedef f32x4 frag;
  static constexpr int pad = 4;
  static constexpr int planes = 1;
  typedef float oct __attribute__((ext_vector_type(8), aligned(4)));
  static __device__ __forceinline__ f32x4 mma(frag a0, frag a1, frag b0, frag b1, f32x4 s) {
#pragma unroll
    for (int e = 0; e < 4; ++e) s = __builtin_amdgcn_mfma_f32_16x16x4f32(a0[e], b0[e], s, 0, 0, 0);
#pragma unroll
    for (int e = 0; e < 4; ++e) s = __builtin_amdgcn_mfma_f32_16x16x4f32(a1[e], b1[e], s, 0, 0, 0);
    return s;
  }
  static __device__ __forceinline__ void row8(const float* p, frag& f0, frag& f1) {
    f0 = *reinterpret_cast<const f32x4*>(p);
    f1 = *reinterpret_cast<const f32x4*>(p + 4);
  }
  static __device__ __forceinline__ frag row4(const float* p) { return *reinterpret_cast<const f32x4*>(p); }
  static __device__ __forceinline__ frag column(const float* tile, int pitch, int k0, int n0, int lane) {
    const float* p = tile + (k0 + (lane >> 4) * 4) * pitch + n0 + (lane & 15);
    return f32x4{p[0], p[pitch], p[2 * pitch], p[3 * pitch]};
  }
  static __device__ __forceinline__ frag round(f32x4 v) { return v; }
  static __device__ __forceinline__ void split(f32x4 v, frag (&f)[1]) { f[0] = v; }
  static __device__ __forceinline__ bool odd(oct v) {
    bool bad = false;
#pragma unroll
    for (int i = 0; i < 8; ++i) bad |= !(__builtin_fabsf(v[i]) < __builtin_inff());
    return bad;
  }
};

__device__ __forceinline__ float power(float log2_decay, int n) { return __builtin_amdgcn_exp2f(log2_decay * (float)n); }
// log2 of a decay; of zero, one whose first power is zero and whose zeroth is one
__device__ __forceinline__ float log2_of(float decay) { return decay == 0.f ? -1e5f : log2f(decay); }

// 64 rows of D values (d of them real) as the threads hold them between memory and LDS
template <typename T, int D>
struct Rows {
  static constexpr int PER_ROW = D / 8, N = CHUNK * PER_ROW / THREADS;
  typename Kind<T>::oct v[N];

  // frames u0 .. u0 + 63 of n; those past the end are zero
  __device__ __forceinline__ void load(const T* base, long long step, long long u0, long long n, bool reverse, int d) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int at = threadIdx.x + i * THREADS, column = at % PER_ROW * 8;
      const long long u = u0 + at / PER_ROW;
      v[i] = (T)0;
      if (u < n && column < d) {
        const T* p = base + (reverse ? n - 1 - u : u) * step + column;
        if (column + 8 <= d) {
          v[i] = *reinterpret_cast<const typename Kind<T>::oct*>(p);
        } else {
#pragma unroll
          for (int e = 0; e < 8; ++e)
            if (column + e < d) v[i][e] = p[e];
        }
      }
    }
  }
  __device__ __forceinline__ void store(T* tile) const {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int at = threadIdx.x + i * THREADS;
      T* p = tile + at / PER_ROW * (D + Kind<T>::pad) + at % PER_ROW * 8;
      typedef T half __attribute__((ext_vector_type(16 / sizeof(T))));
      const typename Kind<T>::oct w = v[i];
#pragma unroll
      for (int e = 0; e < 8; e += 16 / sizeof(T)) {
        half h;
#pragma unroll
        for (int k = 0; k < (int)(16 / sizeof(T)); ++k) h[k] = w[e + k];
        *reinterpret_cast<half*>(p + e) = h;
      }
    }
  }
  // zero in the place of octets with a value that is not finite; the first row that has one (64: none)
  __device__ __forceinline__ int clean() {
    int first = CHUNK;
#pragma unroll
    for (int i = 0; i < N; ++i)
      if (Kind<T>::odd(v[i])) {
        v[i] = (T)0;
        const int row = (threadIdx.x + i * THREADS) / PER_ROW;
        first = row < first ? row : first;
      }
    return first;
  }
};

template <typename T, int DA, int DC>
constexpr int mix_lds(bool state_only) {
  const int pad = Kind<T>::pad;
  return (int)sizeof(T) * CHUNK * ((state_only ? 1 : 2) * (DA + pad) + DC + pad) + (state_only ? 0 : 10 * 64 * (int)sizeof(typename Kind<T>::frag)) + 16;
}

// A product that sums over frames j meets c_j = 0 * x where its weight is zero (j after i): an infinity or a NaN there would reach frames before its own.  It is
// taken out of the tile, and every frame from its own on is NaN, as is the state.
template <typename T, int DA, int DC, bool STATE_ONLY>
__global__ __launch_bounds__(THREADS, 2) void decay_mix_kernel(DecayMix P) {
  typedef Kind<T> K;
  typedef typename K::frag frag;
  constexpr int PA = DA + K::pad, PC = DC + K::pad, RB = DA / 16, CB = DC / 16 / WAVES, IB = CHUNK / 16;
  extern __shared__ __align__(16) unsigned char lds[];
  T* tile_b = reinterpret_cast<T*>(lds);
  T* tile_c = tile_b + CHUNK * PA;
  T* tile_a = tile_c + CHUNK * PC;  // (not there where the state alone is summed)
  frag* weights = reinterpret_cast<frag*>(tile_a + CHUNK * PA);
  int* bad_row = reinterpret_cast<int*>(STATE_ONLY ? reinterpret_cast<unsigned char*>(tile_a) : reinterpret_cast<unsigned char*>(weights + 10 * 64));

  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), li = lane & 15, lg = lane >> 4;
  const int segment = blockIdx.x % P.segments;
  if (STATE_ONLY && segment == P.segments - 1) return;  // nothing comes after it
  const long long bh = blockIdx.x / P.segments;
  const long long batch = bh / P.H;
  const int head = (int)(bh % P.H);
  const bool reverse = P.reverse;
  long long n = P.T;
  if (P.lengths) {
    const long long given = P.lengths[batch];
    n = given < 0 ? 0 : given < n ? given : n;
  }
  const float log2_decay = log2_of(P.decay[head]);
  const T* a = static_cast<const T*>(P.a) + batch * P.a_b + head * P.a_h;
  const T* b = static_cast<const T*>(P.b) + batch * P.b_b + head * P.b_h;
  const T* c = static_cast<const T*>(P.c) + batch * P.c_b + head * P.c_h;
  const int column0 = wave * CB * 16;

  // the state: rows 16 r + 4 lg .. + 3 of column column0 + 16 m + li
  f32x4 state[RB][CB];
  float* part = P.parts + (bh * P.segments + segment) * (DA * DC);
#pragma unroll
  for (int r = 0; r < RB; ++r)
#pragma unroll
    for (int m = 0; m < CB; ++m) {
      state[r][m] = 0.f;
      if (STATE_ONLY) continue;
      if (P.segments > 1) {
        state[r][m] = *reinterpret_cast<const f32x4*>(part + ((r * CB + m) * THREADS + threadIdx.x) * 4);
      } else if (P.first) {
        const int column = column0 + m * 16 + li;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int row = r * 16 + lg * 4 + e;
          if (row < P.da && column < P.dc)
            state[r][m][e] = P.first[bh * P.da * P.dc + (P.transposed ? (long long)column * P.da + row : (long long)row * P.dc + column)] * P.first_factor;
        }
      }
    }

  const long long chunks = (P.T + CHUNK - 1) / CHUNK;
  const long long from = (long long)segment * P.segment_chunks;
  const long long to = from + P.segment_chunks < chunks ? from + P.segment_chunks : chunks;

  Rows<T, DA> ra, rb;
  Rows<T, DC> rc;
  if (from < to && from * CHUNK < n) {
    if (!STATE_ONLY) ra.load(a, P.a_t, from * CHUNK, n, reverse, P.da);
    rb.load(b, P.b_t, from * CHUNK, n, reverse, P.da);
    rc.load(c, P.c_t, from * CHUNK, n, reverse, P.dc);
  }
  for (long long chunk = from; chunk < to; ++chunk) {
    const long long u0 = chunk * CHUNK;
    T* out = static_cast<T*>(P.out) + (batch * P.T * P.H + head) * P.dc;
    if (u0 >= n) {  // past the sequence's end
      if (!STATE_ONLY)
        for (int at = threadIdx.x; at < CHUNK * P.dc; at += THREADS)
          if (u0 + at / P.dc < P.T) out[(u0 + at / P.dc) * P.H * P.dc + at % P.dc] = (T)0;
      continue;
    }
    const int here = (int)(n - u0 < CHUNK ? n - u0 : CHUNK);
    int* bad_here = bad_row + (chunk & 1);  // two in turn: a wave may still read the last chunk's
    if (threadIdx.x == 0) *bad_here = CHUNK;
    __syncthreads();
    if (!STATE_ONLY) ra.store(tile_a);
    rb.store(tile_b);
    const int bad = rc.clean();
    if (bad < CHUNK) atomicMin(bad_here, bad);
    rc.store(tile_c);
    __syncthreads();
    const int first_bad = *bad_here;
    if (chunk + 1 < to && u0 + CHUNK < n) {
      if (!STATE_ONLY) ra.load(a, P.a_t, u0 + CHUNK, n, reverse, P.da);
      rb.load(b, P.b_t, u0 + CHUNK, n, reverse, P.da);
      rc.load(c, P.c_t, u0 + CHUNK, n, reverse, P.dc);
    }
    if constexpr (!STATE_ONLY) {
      // the weights l^(i-j) (a_i . b_j) of the ten blocks on and below the diagonal, as (j, i): the operand of frame i's sum over j
#pragma unroll
      for (int k = 0; k < 3; ++k) {
        const int block = wave + k * WAVES;
        if (block < 10) {
          const int ib = block >= 6 ? 3 : block >= 3 ? 2 : block >= 1 ? 1 : 0, jb = block - ib * (ib + 1) / 2;
          f32x4 s = 0.f;
#pragma unroll
          for (int d = 0; d < DA; d += 32) {
            frag b0, b1, a0, a1;
            K::row8(tile_b + (jb * 16 + li) * PA + d + lg * 8, b0, b1);
            K::row8(tile_a + (ib * 16 + li) * PA + d + lg * 8, a0, a1);
            s = K::mma(b0, b1, a0, a1, s);
          }
          const int apart = (ib - jb) * 16 + li - lg * 4;
#pragma unroll
          for (int e = 0; e < 4; ++e) s[e] = apart - e < 0 ? 0.f : s[e] * power(log2_decay, apart - e);
          weights[block * 64 + lane] = K::round(s);
        }
      }
      __syncthreads();
    }
    frag cf[IB][CB];
#pragma unroll
    for (int j = 0; j < IB; ++j)
#pragma unroll
      for (int m = 0; m < CB; ++m) cf[j][m] = K::column(tile_c, PC, j * 16, column0 + m * 16, lane);
    if constexpr (!STATE_ONLY) {
      // out, as (column, frame): l^(i+1) (a S) + weights c
      f32x4 o[IB][CB];
#pragma unroll
      for (int i = 0; i < IB; ++i)
#pragma unroll
        for (int m = 0; m < CB; ++m) o[i][m] = 0.f;
#pragma unroll
      for (int r = 0; r < RB; r += 2) {
        frag s0[CB], s1[CB];
#pragma unroll
        for (int m = 0; m < CB; ++m) {
          s0[m] = K::round(state[r][m]);
          s1[m] = K::round(state[r + 1][m]);
        }
#pragma unroll
        for (int i = 0; i < IB; ++i) {
          const T* p = tile_a + (i * 16 + li) * PA + r * 16 + lg * 4;
          const frag a0 = K::row4(p), a1 = K::row4(p + 16);
#pragma unroll
          for (int m = 0; m < CB; ++m) o[i][m] = K::mma(s0[m], s1[m], a0, a1, o[i][m]);
        }
      }
      const frag zero = {};
#pragma unroll
      for (int i = 0; i < IB; ++i) {
        const float since = power(log2_decay, i * 16 + li + (reverse ? 0 : 1));
#pragma unroll
        for (int m = 0; m < CB; ++m) o[i][m] *= since;
#pragma unroll
        for (int j = 0; j <= i; j += 2) {
          const frag w0 = weights[(i * (i + 1) / 2 + j) * 64 + lane];
          const frag w1 = j + 1 <= i ? weights[(i * (i + 1) / 2 + j + 1) * 64 + lane] : zero;
#pragma unroll
          for (int m = 0; m < CB; ++m) o[i][m] = K::mma(cf[j][m], j + 1 <= i ? cf[j + 1][m] : zero, w0, w1, o[i][m]);
        }
        const int u = i * 16 + li;
        if (u0 + u < P.T) {
          T* row = out + (reverse && u < here ? n - 1 - (u0 + u) : u0 + u) * P.H * P.dc;
#pragma unroll
          for (int m = 0; m < CB; ++m) {
            const int column = column0 + m * 16 + lg * 4;
            f32x4 v = o[i][m] * P.factor;
            if (u >= here) v = 0.f;
            else if (u >= first_bad) v = __builtin_nanf("");
            typedef T quad __attribute__((ext_vector_type(4)));
            typedef T quad_anywhere __attribute__((ext_vector_type(4), aligned(sizeof(T))));
            const quad w = __builtin_convertvector(v, quad);
            if (column + 4 <= P.dc) {
              *reinterpret_cast<quad_anywhere*>(row + column) = w;
            } else {
#pragma unroll
              for (int e = 0; e < 4; ++e)
                if (column + e < P.dc) row[column + e] = w[e];
            }
          }
        }
      }
    }
    // S' = l^n S + sum over j of b_j^T (l^(n-1-j) c_j): the scaled c as the sum of three operands, so that the state is as exact as its float32 sums
    const float carry = power(log2_decay, here);
#pragma unroll
    for (int r = 0; r < RB; ++r)
#pragma unroll
      for (int m = 0; m < CB; ++m) state[r][m] *= carry;
#pragma unroll
    for (int j = 0; j < IB; j += 2) {
      frag s0[CB][K::planes], s1[CB][K::planes];
#pragma unroll
      for (int half = 0; half < 2; ++half) {
        f32x4 left;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int after = here - 1 - ((j + half) * 16 + lg * 4 + e);
          left[e] = after < 0 ? 0.f : power(log2_decay, after + (reverse ? 1 : 0));
        }
#pragma unroll
        for (int m = 0; m < CB; ++m) K::split(__builtin_convertvector(cf[j + half][m], f32x4) * left, half ? s1[m] : s0[m]);
      }
#pragma unroll
      for (int r = 0; r < RB; ++r) {
        const frag b0 = K::column(tile_b, PA, j * 16, r * 16, lane), b1 = K::column(tile_b, PA, j * 16 + 16, r * 16, lane);
#pragma unroll
        for (int m = 0; m < CB; ++m)
#pragma unroll
          for (int p = K::planes - 1; p >= 0; --p) state[r][m] = K::mma(b0, b1, s0[m][p], s1[m][p], state[r][m]);
      }
    }
    if (first_bad < CHUNK)
#pragma unroll
      for (int r = 0; r < RB; ++r)
#pragma unroll
        for (int m = 0; m < CB; ++m) state[r][m] = __builtin_nanf("");
  }

  if (STATE_ONLY) {
#pragma unroll
    for (int r = 0; r < RB; ++r)
#pragma unroll
      for (int m = 0; m < CB; ++m) *reinterpret_cast<f32x4*>(part + ((r * CB + m) * THREADS + threadIdx.x) * 4) = state[r][m];
  } else if (P.last && segment == P.segments - 1) {
#pragma unroll
    for (int r = 0; r < RB; ++r)
#pragma unroll
      for (int m = 0; m < CB; ++m) {
        const int column = column0 + m * 16 + li;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int row = r * 16 + lg * 4 + e;
          if (row < P.da && column < P.dc)
            P.last[bh * P.da * P.dc + (P.transposed ? (long long)column * P.da + row : (long long)row * P.dc + column)] = state[r][m][e] * P.last_factor;
        }
      }
  }
}

// parts[s]: from each segment's own state to the state before it, in order
template <int DA, int DC>
__global__ __launch_bounds__(256) void decay_join_kernel(DecayMix P) {
  constexpr int CB = DC / 16 / WAVES, WGS = DA * DC / 1024;
  const long long bh = blockIdx.x / WGS, batch = bh / P.H;
  const int quad = blockIdx.x % WGS, r = quad / CB, m = quad % CB;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, column = wave * CB * 16 + m * 16 + (lane & 15);
  long long n = P.T;
  if (P.lengths) {
    const long long given = P.lengths[batch];
    n = given < 0 ? 0 : given < n ? given : n;
  }
  const float log2_decay = log2_of(P.decay[bh % P.H]);
  f32x4 s = 0.f;
  if (P.first)
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int row = r * 16 + (lane >> 4) * 4 + e;
      if (row < P.da && column < P.dc)
        s[e] = P.first[bh * P.da * P.dc + (P.transposed ? (long long)column * P.da + row : (long long)row * P.dc + column)] * P.first_factor;
    }
  float* at = P.parts + bh * P.segments * (DA * DC) + (quad * THREADS + threadIdx.x) * 4;
  const long long frames = (long long)P.segment_chunks * CHUNK;
  for (int i = 0; i < P.segments; ++i, at += DA * DC) {
    f32x4 own = 0.f;
    if (i + 1 < P.segments) own = *reinterpret_cast<const f32x4*>(at);
    *reinterpret_cast<f32x4*>(at) = s;
    const long long left = n - i * frames, here = left < 0 ? 0 : left < frames ? left : frames;
    s = s * __builtin_amdgcn_exp2f(log2_decay * (float)here) + own;
  }
}

// One frame: the state is read and written once, four columns of it to a lane, a slab of 32 columns to a workgroup
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

template <typename T, int DA, int DC, bool STATE_ONLY>
hipError_t mix_init() {
  return hipFuncSetAttribute(reinterpret_cast<const void*>(&decay_mix_kernel<T, DA, DC, STATE_ONLY>), hipFuncAttributeMaxDynamicSharedMemorySize,
                             mix_lds<T, DA, DC>(STATE_ONLY));
}

template <typename T>
hipError_t launch_mix(const DecayMix& P, hipStream_t stream) {
  return by_heads(P.da, P.dc, [&](auto a, auto c) {
    constexpr int DA = a.value, DC = c.value;
    const unsigned grid = (unsigned)(P.B * P.H * P.segments);
    if (P.segments > 1) {
      hipLaunchKernelGGL((decay_mix_kernel<T, DA, DC, true>), dim3(grid), dim3(THREADS), (mix_lds<T, DA, DC>(true)), stream, P);
      hipError_t e = hipGetLastError();
      if (e != hipSuccess) return e;
      hipLaunchKernelGGL((decay_join_kernel<DA, DC>), dim3((unsigned)(P.B * P.H * (DA * DC / 1024))), dim3(256), 0, stream, P);
      e = hipGetLastError();
      if (e != hipSuccess) return e;
    }
    hipLaunchKernelGGL((decay_mix_kernel<T, DA, DC, false>), dim3(grid), dim3(THREADS), (mix_lds<T, DA, DC>(false)), stream, P);
    return hipGetLastError();
  });
}

}  // namespace

hipError_t decay_kernels_init() {
  for (int da : {64, 128})
    for (int dc : {64, 128}) {
      const hipError_t e = by_heads(da, dc, [&](auto a, auto c) {
        constexpr int A = a.value, C = c.value;
        hipError_t e = mix_init<bf16, A, C, false>();
        if (e == hipSuccess) e = mix_init<bf16, A, C, true>();
        if (e == hipSuccess) e = mix_init<float, A, C, false>();
        if (e == hipSuccess) e = mix_init<float, A, C, true>();
        return e;
      });
      if (e != hipSuccess) return e;
    }
  return hipSuccess;
}

size_t decay_segments(long long B, long long T, int H, int da, int dc, int* segments, int* chunks) {
  const long long all = std::max(1LL, (T + CHUNK - 1) / CHUNK), heads = std::max(1LL, B * H);
  // two workgroups on each of 256 CUs, segments of four chunks at least
  long long n = std::max(1LL, std::min((512 + heads - 1) / heads, all / 4));
  const long long each = (all + n - 1) / n;
  n = (all + each - 1) / each;
  *segments = (int)n;
  *chunks = (int)each;
  return n == 1 ? 0 : (size_t)(heads * n) * (da <= 64 ? 64 : 128) * (dc <= 64 ? 64 : 128) * sizeof(float);
}

hipError_t launch_decay_mix(const DecayMix& P, int type, hipStream_t stream) { return type == NNA_F32 ? launch_mix<float>(P, stream) : launch_mix<bf16>(P, stream); }

hipError_t launch_decay_step(const DecayStep& P, int type, hipStream_t stream) {
  const unsigned grid = (unsigned)(P.B * P.H * ((P.dv + STEP_COLUMNS - 1) / STEP_COLUMNS));
  if (type == NNA_F32)
    hipLaunchKernelGGL(decay_step_kernel<float>, dim3(grid), dim3(256), 0, stream, P);
  else
    hipLaunchKernelGGL(decay_step_kernel<bf16>, dim3(grid), dim3(256), 0, stream, P);
  return hipGetLastError();
}

}  // namespace nna
