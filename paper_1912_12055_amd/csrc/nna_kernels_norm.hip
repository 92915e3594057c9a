// Layer norm of rows and of frames, forward and backward, and values kept in 8 bits.
//
// A row's mean m, r = 1 / sqrt(mean((x - m)^2) + eps) and h = (x - m) r give y = h w + b; with gh = gy w,
//   gx = r (gh - mean(gh) - h mean(gh h)),   gw = sum over rows of gy h,   gb = sum over rows of gy.
// All of it is some ten operations a value: the bytes bound it.  A row is read once into registers (of 16 lanes up to a
// workgroup, eight neighbours a lane at a time), the mean is known before the squares are summed, and every sum is float32.
#include "nna_norm.h"

#include <type_traits>

namespace nna {

namespace {

typedef _Float16 f16;
typedef __bf16 bf16;

// eight neighbours wherever they start: the address need only be a multiple of the element
template <typename T>
struct Oct {
  typedef T type __attribute__((ext_vector_type(8), aligned(sizeof(T))));
};
typedef float f32x8 __attribute__((ext_vector_type(8)));

// n (at least 1) of eight values from p, the others zero
template <typename T>
__device__ __forceinline__ f32x8 load8(const T* p, int n) {
  if (n >= 8) return __builtin_convertvector(*reinterpret_cast<const typename Oct<T>::type*>(p), f32x8);
  f32x8 v;
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = i < n ? (float)p[i] : 0.f;
  return v;
}

// ... as they lie in memory, for a use further on
template <typename T>
__device__ __forceinline__ typename Oct<T>::type raw8(const T* p, int n) {
  if (n >= 8) return *reinterpret_cast<const typename Oct<T>::type*>(p);
  typename Oct<T>::type v;
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = i < n ? p[i] : (T)0;
  return v;
}
template <typename T>
__device__ __forceinline__ void store8(T* p, int n, f32x8 v) {
  typedef T plain __attribute__((ext_vector_type(8)));
  const plain u = __builtin_convertvector(v, plain);
  if (n >= 8) {
    *reinterpret_cast<typename Oct<T>::type*>(p) = u;
    return;
  }
#pragma unroll
  for (int i = 0; i < 8; ++i)
    if (i < n) p[i] = u[i];
}

// ---- 8 bits ----------------------------------------------------------------------------------------------------------
// A block's largest magnitude a gives the scale s = a fl(1/127) and the codes rint(x (127 / a)), the quotient rounded once: what a
// code stands for is c s in float32, wherever it is computed.  Blocks below 2^-100 (whose 127 / a would overflow) are zero; a block
// that holds a value that is not finite is NaN throughout, so that none is lost.
struct Scale8 {
  float up, down;
};
__device__ __forceinline__ Scale8 scale8(float most) {
  if (!(most < __builtin_inff())) return {0.f, __builtin_nanf("")};
  if (most < 0x1p-100f) return {0.f, 0.f};
  return {127.f / most, most * (1.f / 127.f)};
}
__device__ __forceinline__ float most8(f32x8 v) {
  float m = 0.f;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float a = __builtin_fabsf(v[i]);
    m = a <= m || m != m ? m : a;  // a NaN compares false: it is taken, and stays
  }
  return m;
}

typedef signed char i8x8 __attribute__((ext_vector_type(8), aligned(1)));
__device__ __forceinline__ void store_codes(signed char* p, int n, f32x8 v, float up) {
  i8x8 c;
#pragma unroll
  for (int i = 0; i < 8; ++i) c[i] = up == 0.f ? 0 : (signed char)(int)__builtin_rintf(v[i] * up);
  if (n >= 8) {
    *reinterpret_cast<i8x8*>(p) = c;
    return;
  }
#pragma unroll
  for (int i = 0; i < 8; ++i)
    if (i < n) p[i] = c[i];
}
__device__ __forceinline__ f32x8 values_of(i8x8 c, float scale) {
  f32x8 v;
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = (float)c[i] * scale;
  return v;
}
template <>
struct Oct<signed char> {
  typedef i8x8 type;
};

// ---- over lanes, without LDS: rotations within 16 lanes, then exchanges of rows of 16 and halves of the wave ------------------------
template <int N>
__device__ __forceinline__ float rotated(float v) {
  return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), 0x120 + N, 0xf, 0xf, true));
}
__device__ __forceinline__ float larger(float m, float o) { return o <= m || m != m ? m : o; }  // NaN beats all
// the largest of 16 neighbouring lanes' magnitudes
__device__ __forceinline__ float most16(float m) {
  m = larger(m, rotated<8>(m));
  m = larger(m, rotated<4>(m));
  m = larger(m, rotated<2>(m));
  return larger(m, rotated<1>(m));
}
// the sum over LANES (16, 32 or 64) neighbouring lanes, in all of them
template <int LANES>
__device__ __forceinline__ float lanes_sum(float v) {
  v += rotated<8>(v);
  v += rotated<4>(v);
  v += rotated<2>(v);
  v += rotated<1>(v);
  if (LANES > 16) {
    const auto p = __builtin_amdgcn_permlane16_swap(__builtin_bit_cast(unsigned, v), __builtin_bit_cast(unsigned, v), false, false);
    const unsigned a = p[0], b = p[1];  // (a bit cast of an element itself takes the first)
    v = __builtin_bit_cast(float, a) + __builtin_bit_cast(float, b);
  }
  if (LANES > 32) {
    const auto p = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(unsigned, v), __builtin_bit_cast(unsigned, v), false, false);
    const unsigned a = p[0], b = p[1];  // (a bit cast of an element itself takes the first)
    v = __builtin_bit_cast(float, a) + __builtin_bit_cast(float, b);
  }
  return v;
}

// over the lanes that hold a row
template <int LANES>
__device__ __forceinline__ float2 row_sum(float2 v, float2* lds, int& turn) {
  v.x = lanes_sum<(LANES < 64 ? LANES : 64)>(v.x);
  v.y = lanes_sum<(LANES < 64 ? LANES : 64)>(v.y);
  if constexpr (LANES > 64) {
    // two buffers in turn: the next sum's writes never meet a lane that still reads this one
    float2* at = lds + (turn & 1) * (LANES / 64);
    ++turn;
    if ((threadIdx.x & 63) == 0) at[threadIdx.x >> 6] = v;
    __syncthreads();
    v = at[0];
#pragma unroll
    for (int i = 1; i < LANES / 64; ++i) {
      v.x += at[i].x;
      v.y += at[i].y;
    }
  }
  return v;
}

template <int LANES>
constexpr int threads_of() { return LANES > 256 ? LANES : 256; }

// Rows in registers: LANES lanes hold a row, CHUNKS times eight values each.  The weights stay in registers over all rows of a lane.  Bound by memory: 65,536 rows of
// 2,048, bfloat16, 102 us, 5.3 TB/s; 131,072 of 1,024 with their 8 bits 141 us, 4.8 TB/s.  One row of 512: 2 us of a call of 9, the rest the host's.
template <typename TX, typename TY, int LANES, int CHUNKS, bool KEEP8>
__global__ __launch_bounds__(threads_of<LANES>()) void norm_rows_kernel(NormParams P) {
  constexpr int GROUPS = threads_of<LANES>() / LANES;
  __shared__ float2 lds[2 * (LANES > 64 ? LANES / 64 : 1)];
  const int lane = threadIdx.x % LANES;
  const int width = P.width, blocks = (width + NORM_BLOCK8 - 1) / NORM_BLOCK8;
  f32x8 w[CHUNKS], b[CHUNKS];
  int n[CHUNKS];
#pragma unroll
  for (int c = 0; c < CHUNKS; ++c) {
    const int at = (lane + c * LANES) * 8;
    n[c] = width - at;
    w[c] = b[c] = 0.f;
    if (n[c] > 0) {
      w[c] = 1.f;
      if (P.weight) w[c] = load8(P.weight + at, n[c]);
      if (P.bias) b[c] = load8(P.bias + at, n[c]);
    }
  }
  const float inv = 1.f / (float)width;
  int turn = 0;
  for (long long row = (long long)blockIdx.x * GROUPS + threadIdx.x / LANES; row < P.rows; row += (long long)gridDim.x * GROUPS) {
    const TX* x = static_cast<const TX*>(P.x) + row * P.row_stride;
    f32x8 v[CHUNKS];
    float2 s = {0.f, 0.f};
#pragma unroll
    for (int c = 0; c < CHUNKS; ++c) {
      v[c] = 0.f;
      if (n[c] > 0) v[c] = load8(x + (lane + c * LANES) * 8, n[c]);
#pragma unroll
      for (int i = 0; i < 8; ++i) s.x += v[c][i];
    }
    const float mean = row_sum<LANES>(s, lds, turn).x * inv;
    s = {0.f, 0.f};
#pragma unroll
    for (int c = 0; c < CHUNKS; ++c)
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float d = i < n[c] ? v[c][i] - mean : 0.f;
        s.x += d * d;
      }
    const float rstd = 1.f / sqrtf(row_sum<LANES>(s, lds, turn).x * inv + P.eps);
    TY* y = static_cast<TY*>(P.y) + row * width;
#pragma unroll
    for (int c = 0; c < CHUNKS; ++c) {
      const int at = (lane + c * LANES) * 8;
      if (n[c] > 0) store8(y + at, n[c], (v[c] - mean) * rstd * w[c] + b[c]);
      if constexpr (KEEP8) {
        const Scale8 q = scale8(most16(most8(v[c])));
        if (n[c] > 0) {
          store_codes(P.codes + row * width + at, n[c], v[c], q.up);
          if ((lane & 15) == 0) P.scales[row * blocks + at / NORM_BLOCK8] = q.down;
        }
      }
    }
    if (P.stats && lane == 0) {
      P.stats[2 * row] = mean;
      P.stats[2 * row + 1] = rstd;
    }
  }
}

// The gradients of a row, and of the weights over the rows of a workgroup: summed in registers, then over the workgroup's rows in
// LDS in a fixed order, one partial sum a workgroup.  65,536 rows of 2,048, bfloat16: 155 us, 5.2 TB/s; 131,072 of 1,024 from 8 bits 139 us, 4.9 TB/s.
template <typename TX, typename TY, int LANES, int CHUNKS, bool KEPT8>
__global__ __launch_bounds__(threads_of<LANES>()) void norm_rows_backward_kernel(NormParams P) {
  constexpr int GROUPS = threads_of<LANES>() / LANES;
  __shared__ float2 lds[2 * (LANES > 64 ? LANES / 64 : 1)];
  __shared__ float joined[GROUPS > 1 ? GROUPS * LANES * CHUNKS * 8 : 1];
  const int lane = threadIdx.x % LANES, group = threadIdx.x / LANES;
  const int width = P.width, blocks = (width + NORM_BLOCK8 - 1) / NORM_BLOCK8;
  f32x8 w[CHUNKS], gw[CHUNKS], gb[CHUNKS];
  int n[CHUNKS];
#pragma unroll
  for (int c = 0; c < CHUNKS; ++c) {
    const int at = (lane + c * LANES) * 8;
    n[c] = width - at;
    w[c] = gw[c] = gb[c] = 0.f;
    if (n[c] > 0) {
      w[c] = 1.f;
      if (P.weight) w[c] = load8(P.weight + at, n[c]);
    }
  }
  const float inv = 1.f / (float)width;
  // A row as it lies in memory.  Where a row is a workgroup's, whose waves all wait for its sums, the next one is requested before (65,536 rows of 2,048
  // bfloat16: 157 us, 165 without); rows within a wave have other waves beside them, and their registers hold more of those (131,072 rows of 1,024 in
  // 8 bits: 139 us, 206 with)
  constexpr bool AHEAD = LANES > 64 && LANES * CHUNKS <= 1024;
  typedef std::conditional_t<KEPT8, signed char, TX> TK;
  struct Row {
    typename Oct<TY>::type g[CHUNKS];
    typename Oct<TK>::type x[CHUNKS];
    float scale[KEPT8 ? CHUNKS : 1], mean, rstd;
  };
  auto request = [&](long long row, Row& r) {
    r.mean = P.stats[2 * row];
    r.rstd = P.stats[2 * row + 1];
#pragma unroll
    for (int c = 0; c < CHUNKS; ++c) {
      const int at = (lane + c * LANES) * 8;
      if (n[c] <= 0) continue;
      r.g[c] = raw8(static_cast<const TY*>(P.gout) + row * width + at, n[c]);
      if constexpr (KEPT8) {
        r.x[c] = raw8(P.codes + row * width + at, n[c]);
        r.scale[c] = P.scales[row * blocks + at / NORM_BLOCK8];
      } else {
        r.x[c] = raw8(static_cast<const TX*>(P.x) + row * P.row_stride + at, n[c]);
      }
    }
  };
  int turn = 0;
  const long long step = (long long)gridDim.x * GROUPS;
  long long row = (long long)blockIdx.x * GROUPS + group;
  Row next;
  if (AHEAD && row < P.rows) request(row, next);
  for (; row < P.rows; row += step) {
    if (!AHEAD) request(row, next);
    const Row now = next;
    if (AHEAD && row + step < P.rows) request(row + step, next);
    f32x8 h[CHUNKS], gh[CHUNKS];
    float2 s = {0.f, 0.f};
#pragma unroll
    for (int c = 0; c < CHUNKS; ++c) {
      h[c] = gh[c] = 0.f;
      if (n[c] > 0) {
        const f32x8 g = __builtin_convertvector(now.g[c], f32x8);
        if constexpr (KEPT8)
          h[c] = values_of(now.x[c], now.scale[c]);
        else
          h[c] = __builtin_convertvector(now.x[c], f32x8);
        h[c] = (h[c] - now.mean) * now.rstd;
        gw[c] += g * h[c];
        gb[c] += g;
        gh[c] = g * w[c];  // zero past the row's end, as g is
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          s.x += gh[c][i];
          s.y += i < n[c] ? gh[c][i] * h[c][i] : 0.f;
        }
      }
    }
    if (!P.gx) continue;
    s = row_sum<LANES>(s, lds, turn);
    s.x *= inv;
    s.y *= inv;
    TX* gx = static_cast<TX*>(P.gx) + row * width;
#pragma unroll
    for (int c = 0; c < CHUNKS; ++c)
      if (n[c] > 0) store8(gx + (lane + c * LANES) * 8, n[c], (gh[c] - s.x - h[c] * s.y) * now.rstd);
  }
  if (!P.partial) return;
  float* out = P.partial + (long long)blockIdx.x * 2 * width;
#pragma unroll
  for (int part = 0; part < 2; ++part) {
    if constexpr (GROUPS == 1) {
#pragma unroll
      for (int c = 0; c < CHUNKS; ++c)
        if (n[c] > 0) store8(out + part * width + (lane + c * LANES) * 8, n[c], part ? gb[c] : gw[c]);
    } else {  // the groups' sums side by side, then a column to a thread
#pragma unroll
      for (int c = 0; c < CHUNKS; ++c)
        if (n[c] > 0) store8(joined + group * width + (lane + c * LANES) * 8, n[c], part ? gb[c] : gw[c]);
      __syncthreads();
      for (int d = threadIdx.x; d < width; d += 256) {
        float s = joined[d];
#pragma unroll
        for (int g = 1; g < GROUPS; ++g) s += joined[g * width + d];
        out[part * width + d] = s;
      }
      __syncthreads();
    }
  }
}

// gw, gb: the sum of the workgroups' partial sums, JOIN_RUNS runs of them side by side and joined in order (4 to 5 us: a launch and two reads' latency)
constexpr int JOIN_COLUMNS = 32, JOIN_RUNS = 32;
__global__ __launch_bounds__(JOIN_COLUMNS* JOIN_RUNS) void norm_join_kernel(const float* partial, int groups, int width, float* gw, float* gb) {
  __shared__ float lds[JOIN_RUNS][JOIN_COLUMNS];
  const int column = blockIdx.x * JOIN_COLUMNS + threadIdx.x % JOIN_COLUMNS, run = threadIdx.x / JOIN_COLUMNS;
  float s = 0.f;
  if (column < 2 * width)
#pragma unroll 8
    for (int g = run; g < groups; g += JOIN_RUNS) s += partial[(long long)g * 2 * width + column];
  lds[run][threadIdx.x % JOIN_COLUMNS] = s;
  __syncthreads();
  if (run || column >= 2 * width) return;
#pragma unroll
  for (int i = 1; i < JOIN_RUNS; ++i) s += lds[i][threadIdx.x];
  float* out = column < width ? gw : gb;
  if (out) out[column < width ? column : column - width] = s;
}

// ---- frames: x[B, width, T], T fastest ---------------------------------------------------------------------------------
// A workgroup takes FRAMES neighbouring frames of a waveform: their columns are read along T, turned in LDS, and every frame is a row there, of which a
// wave holds PAIRS pairs of values a lane.  y and gout are rows [B, T, width]; gx goes back the way x came.
// 16 x 1,025 x 431, float32: 17 us forward (3.2 TB/s), 33 backward (2.6); 64 x 128 x 216 to bfloat16: 7 and 9.  Two workgroups a CU, each of which reads, turns and
// writes in turn: loads, LDS and stores have to come from different workgroups to overlap.
constexpr int FR_THREADS = 512, FR_WAVES = FR_THREADS / 64;
constexpr long long MAX_TILES = 1LL << 22;  // of a launch: its threads are counted in 32 bits
__host__ __device__ constexpr int frames_pitch(int width) { return width | 1; }  // odd: a column's frames are in different banks
// as many frames as leave two workgroups of 72 KB a CU: 128 (64, 32) consecutive bytes of every bin
constexpr int FR_WIDTH_32 = 558, FR_WIDTH_16 = 1088;
constexpr int frames_per_tile(int width) { return width <= FR_WIDTH_32 ? 32 : width <= FR_WIDTH_16 ? 16 : 8; }

// Workgroups go to the eight XCDs in turn: consecutive tiles, whose columns share cache lines, to one XCD's workgroups
__device__ __forceinline__ long long tile_of(long long i, long long tiles) {
  const long long each = tiles / 8, more = tiles % 8, xcd = i % 8, at = i / 8;
  return xcd * each + (xcd < more ? xcd : more) + at;
}

// What is computed of `v` after this is computed there: not ahead of a loop, to be kept in registers through it.
__device__ __forceinline__ int here_only(int v) {
  asm volatile("" : "+v"(v));
  return v;
}

// fn(column, frame, i) of the tile's values a thread holds between memory and LDS
template <int FRAMES, int N, typename F>
__device__ __forceinline__ void each_of_tile(int width, int frames, F fn) {
  const int thread = here_only(threadIdx.x), t = thread % FRAMES, d = thread / FRAMES;
#pragma unroll
  for (int i = 0; i < N; ++i)
    if (t < frames && d + i * (FR_THREADS / FRAMES) < width) fn(d + i * (FR_THREADS / FRAMES), t, i);
}
template <int FRAMES, int PAIRS>
constexpr int values_of_tile() { return PAIRS * 128 * FRAMES / FR_THREADS; }

template <int FRAMES, int PAIRS>
__device__ __forceinline__ void read_tile(const float* x, long long T, int width, int frames, float (&v)[values_of_tile<FRAMES, PAIRS>()]) {
  each_of_tile<FRAMES, values_of_tile<FRAMES, PAIRS>()>(width, frames, [&](int d, int t, int i) { v[i] = x[d * T + t]; });
}
template <int FRAMES, int PAIRS>
__device__ __forceinline__ void store_tile(float* tile, int width, int frames, const float (&v)[values_of_tile<FRAMES, PAIRS>()]) {
  const int pitch = frames_pitch(width);
  each_of_tile<FRAMES, values_of_tile<FRAMES, PAIRS>()>(width, frames, [&](int d, int t, int i) { tile[t * pitch + d] = v[i]; });
}

// a pair of neighbours, the second of which may be past the row's end
template <typename T>
struct Two {
  typedef T type __attribute__((ext_vector_type(2), aligned(sizeof(T))));
};
typedef float f32x2 __attribute__((ext_vector_type(2)));
template <typename T>
__device__ __forceinline__ f32x2 load2(const T* p, int n) {
  if (n >= 2) return __builtin_convertvector(*reinterpret_cast<const typename Two<T>::type*>(p), f32x2);
  return f32x2{n > 0 ? (float)p[0] : 0.f, 0.f};
}
template <typename T>
__device__ __forceinline__ void store2(T* p, int n, f32x2 v) {
  typedef T plain __attribute__((ext_vector_type(2)));
  const plain u = __builtin_convertvector(v, plain);
  if (n >= 2)
    *reinterpret_cast<typename Two<T>::type*>(p) = u;
  else if (n > 0)
    *p = u[0];
}

template <typename TY, int FRAMES, int PAIRS>
__global__ __launch_bounds__(FR_THREADS) void norm_frames_kernel(NormParams P) {
  constexpr int N = values_of_tile<FRAMES, PAIRS>();
  extern __shared__ float tile[];
  const int width = P.width, pitch = frames_pitch(width), lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const long long tiles = (P.T + FRAMES - 1) / FRAMES;
  const float inv = 1.f / (float)width;
  const long long at = P.first_tile + tile_of(blockIdx.x, gridDim.x), b = at / tiles, t0 = (at % tiles) * FRAMES;
  const int frames = (int)(P.T - t0 < FRAMES ? P.T - t0 : FRAMES);
  float read[N];
  read_tile<FRAMES, PAIRS>(static_cast<const float*>(P.x) + b * width * P.T + t0, P.T, width, frames, read);
  constexpr bool HELD = PAIRS < 9;  // the weights stay in registers where there is room, else they are read again for every frame
  f32x2 held[HELD ? PAIRS : 1], held_shift[HELD ? PAIRS : 1];
  auto weight = [&](int c) {
    const int d = c * 128 + (HELD ? lane : here_only(lane)) * 2;
    return P.weight ? load2(P.weight + d, width - d) : f32x2{1.f, 1.f};
  };
  auto shift = [&](int c) {
    const int d = c * 128 + (HELD ? lane : here_only(lane)) * 2;
    return P.bias ? load2(P.bias + d, width - d) : f32x2{0.f, 0.f};
  };
  if constexpr (HELD)
#pragma unroll
    for (int c = 0; c < PAIRS; ++c) {
      held[c] = weight(c);
      held_shift[c] = shift(c);
    }
  store_tile<FRAMES, PAIRS>(tile, width, frames, read);
  __syncthreads();
#pragma unroll 1
  for (int t = wave; t < frames; t += FR_WAVES) {
    f32x2 v[PAIRS];
    float s = 0.f;
#pragma unroll
    for (int c = 0; c < PAIRS; ++c) {
      const int d = c * 128 + lane * 2;
      v[c] = load2(tile + t * pitch + d, width - d);
      s += v[c].x + v[c].y;
    }
    const float mean = lanes_sum<64>(s) * inv;
    s = 0.f;
#pragma unroll
    for (int c = 0; c < PAIRS; ++c) {
      const int d = c * 128 + lane * 2;
      v[c] -= mean;
      s += (d < width ? v[c].x * v[c].x : 0.f) + (d + 1 < width ? v[c].y * v[c].y : 0.f);
    }
    const float rstd = 1.f / sqrtf(lanes_sum<64>(s) * inv + P.eps);
    const long long row = b * P.T + t0 + t;
    TY* y = static_cast<TY*>(P.y) + row * width;
#pragma unroll
    for (int c = 0; c < PAIRS; ++c) {
      const int d = c * 128 + lane * 2;
      store2(y + d, width - d, v[c] * rstd * (HELD ? held[HELD ? c : 0] : weight(c)) + (HELD ? held_shift[HELD ? c : 0] : shift(c)));
    }
    if (P.stats && lane == 0) {
      P.stats[2 * row] = mean;
      P.stats[2 * row + 1] = rstd;
    }
  }
}

template <typename TY, int FRAMES, int PAIRS>
__global__ __launch_bounds__(FR_THREADS) void norm_frames_backward_kernel(NormParams P) {
  constexpr int ROWS = FRAMES / FR_WAVES, N = values_of_tile<FRAMES, PAIRS>();
  extern __shared__ float tile[];
  const int width = P.width, pitch = frames_pitch(width), lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const long long tiles = (P.T + FRAMES - 1) / FRAMES, all = P.batch * tiles;
  const float inv = 1.f / (float)width;
  // the weights stay in registers where there is room, else they are read again for every frame
  constexpr bool HELD = PAIRS < 9;
  f32x2 gw[PAIRS], gb[PAIRS], held[HELD ? PAIRS : 1];
  auto weight = [&](int c) {
    const int d = c * 128 + (HELD ? lane : here_only(lane)) * 2;
    return P.weight ? load2(P.weight + d, width - d) : f32x2{1.f, 1.f};
  };
#pragma unroll
  for (int c = 0; c < PAIRS; ++c) {
    gw[c] = gb[c] = 0.f;
    if constexpr (HELD) held[c] = weight(c);
  }
  for (long long i = blockIdx.x; i < all; i += gridDim.x) {
    const long long at = tile_of(i, all), b = at / tiles, t0 = (at % tiles) * FRAMES;
    const int frames = (int)(P.T - t0 < FRAMES ? P.T - t0 : FRAMES);
    float read[N];
    read_tile<FRAMES, PAIRS>(static_cast<const float*>(P.x) + b * width * P.T + t0, P.T, width, frames, read);
    // a wave's rows of gout are on their way while the tile is turned
    f32x2 g[ROWS][PAIRS];
    float2 stats[ROWS];
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
      const int t = wave + r * FR_WAVES < frames ? wave + r * FR_WAVES : frames - 1;
      const long long row = b * P.T + t0 + t;
      const TY* gout = static_cast<const TY*>(P.gout) + row * width;
#pragma unroll
      for (int c = 0; c < PAIRS; ++c) g[r][c] = load2(gout + c * 128 + lane * 2, width - c * 128 - lane * 2);
      stats[r] = {P.stats[2 * row], P.stats[2 * row + 1]};
    }
    store_tile<FRAMES, PAIRS>(tile, width, frames, read);
    __syncthreads();
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
      const int t = wave + r * FR_WAVES;
      if (t >= frames) break;
      f32x2 h[PAIRS];
      float s0 = 0.f, s1 = 0.f;
#pragma unroll
      for (int c = 0; c < PAIRS; ++c) {
        const int d = c * 128 + lane * 2;
        h[c] = (load2(tile + t * pitch + d, width - d) - stats[r].x) * stats[r].y;
        if (d >= width) h[c].x = 0.f;
        if (d + 1 >= width) h[c].y = 0.f;
        gw[c] += g[r][c] * h[c];
        gb[c] += g[r][c];
        g[r][c] *= HELD ? held[HELD ? c : 0] : weight(c);  // zero past the row's end
        s0 += g[r][c].x + g[r][c].y;
        s1 += g[r][c].x * h[c].x + g[r][c].y * h[c].y;
      }
      s0 = lanes_sum<64>(s0) * inv;
      s1 = lanes_sum<64>(s1) * inv;
#pragma unroll
      for (int c = 0; c < PAIRS; ++c) {
        const int d = c * 128 + lane * 2;
        store2(tile + t * pitch + d, width - d, (g[r][c] - s0 - h[c] * s1) * stats[r].y);
      }
    }
    __syncthreads();
    if (P.gx) {
      float* gx = static_cast<float*>(P.gx) + b * width * P.T + t0;
      each_of_tile<FRAMES, N>(width, frames, [&](int d, int t, int) { gx[d * P.T + t] = tile[t * pitch + d]; });
    }
    __syncthreads();
  }
  if (!P.partial) return;
  float* out = P.partial + (long long)blockIdx.x * 2 * width;
#pragma unroll
  for (int part = 0; part < 2; ++part) {  // the waves' sums side by side (a tile holds at least as many rows), then a column to a thread
#pragma unroll
    for (int c = 0; c < PAIRS; ++c) {
      const int d = c * 128 + lane * 2;
      store2(tile + wave * width + d, width - d, part ? gb[c] : gw[c]);
    }
    __syncthreads();
    for (int d = threadIdx.x; d < width; d += FR_THREADS) {
      float s = tile[d];
#pragma unroll
      for (int k = 1; k < FR_WAVES; ++k) s += tile[k * width + d];
      out[part * width + d] = s;
    }
    __syncthreads();
  }
}

// ---- values to 8 bits and back -------------------------------------------------------------------------------------------
// 16 lanes take a block: 8 values each.  3,063,808 values of float32: 4.6 us to 8 bits and 6.2 back, 3.3 and 2.5 TB/s, a launch's start and end among them.
template <typename T>
__global__ __launch_bounds__(256) void pack8_kernel(const T* x, long long rows, long long width, long long row_stride, signed char* codes, float* scales) {
  const long long blocks = (width + NORM_BLOCK8 - 1) / NORM_BLOCK8;
  for (long long i = ((long long)blockIdx.x * 256 + threadIdx.x) >> 4; i < rows * blocks; i += (long long)gridDim.x * 16) {
    const long long row = rows == 1 ? 0 : i / blocks, at = (i - row * blocks) * NORM_BLOCK8 + (threadIdx.x & 15) * 8;
    const int n = width - at > 8 ? 8 : (int)(width - at);
    f32x8 v = 0.f;
    if (n > 0) v = load8(x + row * row_stride + at, n);
    const Scale8 q = scale8(most16(most8(v)));
    if (n > 0) store_codes(codes + row * width + at, n, v, q.up);
    if ((threadIdx.x & 15) == 0) scales[i] = q.down;
  }
}

template <typename T>
__global__ __launch_bounds__(256) void unpack8_kernel(const signed char* codes, const float* scales, long long rows, long long width, T* out) {
  const long long blocks = (width + NORM_BLOCK8 - 1) / NORM_BLOCK8;
  for (long long i = ((long long)blockIdx.x * 256 + threadIdx.x) >> 4; i < rows * blocks; i += (long long)gridDim.x * 16) {
    const long long row = rows == 1 ? 0 : i / blocks, at = (i - row * blocks) * NORM_BLOCK8 + (threadIdx.x & 15) * 8;
    const int n = width - at > 8 ? 8 : (int)(width - at);
    if (n > 0) store8(out + row * width + at, n, values_of(raw8(codes + row * width + at, n), scales[i]));
  }
}

// ---- which kernel --------------------------------------------------------------------------------------------------------
// fn(lanes, chunks): the fewest lanes that hold a row of `width` in one or two chunks of eight a lane
template <typename F>
auto by_width(int width, F fn) {
  if (width <= 128) return fn(std::integral_constant<int, 16>(), std::integral_constant<int, 1>());
  if (width <= 256) return fn(std::integral_constant<int, 32>(), std::integral_constant<int, 1>());
  if (width <= 512) return fn(std::integral_constant<int, 64>(), std::integral_constant<int, 1>());
  if (width <= 1024) return fn(std::integral_constant<int, 64>(), std::integral_constant<int, 2>());
  if (width <= 2048) return fn(std::integral_constant<int, 256>(), std::integral_constant<int, 1>());
  if (width <= 4096) return fn(std::integral_constant<int, 256>(), std::integral_constant<int, 2>());
  if (width <= 8192) return fn(std::integral_constant<int, 1024>(), std::integral_constant<int, 1>());
  return fn(std::integral_constant<int, 1024>(), std::integral_constant<int, 2>());
}
// fn(x's type, y's type): equal, or float32 to 16 bits
template <typename F>
hipError_t by_types(int x_type, int y_type, F fn) {
  if (x_type == NNA_F32 && y_type == NNA_F32) return fn(float(), float());
  if (x_type == NNA_F32 && y_type == NNA_BF16) return fn(float(), bf16());
  if (x_type == NNA_F32 && y_type == NNA_F16) return fn(float(), f16());
  if (x_type == NNA_BF16 && y_type == NNA_BF16) return fn(bf16(), bf16());
  if (x_type == NNA_F16 && y_type == NNA_F16) return fn(f16(), f16());
  return hipErrorInvalidValue;
}
template <typename F>
hipError_t by_type(int type, F fn) {
  return type == NNA_F32 ? fn(float()) : type == NNA_BF16 ? fn(bf16()) : type == NNA_F16 ? fn(f16()) : hipErrorInvalidValue;
}
// fn(frames, pairs)
template <typename F>
hipError_t by_frame(int width, F fn) {
  if (width <= 128) return fn(std::integral_constant<int, 32>(), std::integral_constant<int, 1>());
  if (width <= 256) return fn(std::integral_constant<int, 32>(), std::integral_constant<int, 2>());
  if (width <= FR_WIDTH_32) return fn(std::integral_constant<int, 32>(), std::integral_constant<int, 5>());
  if (width <= FR_WIDTH_16) return fn(std::integral_constant<int, 16>(), std::integral_constant<int, 9>());
  return fn(std::integral_constant<int, 8>(), std::integral_constant<int, 17>());
}
size_t frames_lds(int width, int frames) { return sizeof(float) * frames * frames_pitch(width); }

template <typename TY, int F, int C>
hipError_t frames_init() {
  hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(&norm_frames_kernel<TY, F, C>), hipFuncAttributeMaxDynamicSharedMemorySize, 72 * 1024);
  if (e != hipSuccess) return e;
  return hipFuncSetAttribute(reinterpret_cast<const void*>(&norm_frames_backward_kernel<TY, F, C>), hipFuncAttributeMaxDynamicSharedMemorySize, 72 * 1024);
}

constexpr long long MAX_GROUPS = 1024;  // four workgroups of 256 on each of 256 CUs

}  // namespace

hipError_t norm_kernels_init() {
  for (int type : {NNA_F32, NNA_BF16, NNA_F16})
    for (int width : {1, 129, 257, FR_WIDTH_32 + 1, FR_WIDTH_16 + 1}) {
      const hipError_t e = by_type(type, [&](auto y) { return by_frame(width, [&](auto f, auto pairs) { return frames_init<decltype(y), f.value, pairs.value>(); }); });
      if (e != hipSuccess) return e;
    }
  return hipSuccess;
}

int norm_backward_groups(long long rows, int width, bool frames, long long batch, long long T) {
  long long n;
  if (frames) {
    const long long f = frames_per_tile(width);
    n = batch * ((T + f - 1) / f);
  } else {
    n = by_width(width, [&](auto lanes, auto) {
      constexpr int groups = threads_of<lanes.value>() / lanes.value;
      return (rows + groups - 1) / groups;
    });
  }
  return (int)std::max(1LL, std::min(n, MAX_GROUPS));
}

hipError_t launch_norm(const NormParams& P, int x_type, int y_type, bool frames, hipStream_t stream) {
  if (frames)
    return by_type(y_type, [&](auto y) {
      return by_frame(P.width, [&](auto f, auto pairs) {
        constexpr int F = f.value, C = pairs.value;
        const size_t lds = frames_lds(P.width, F);
        const long long tiles = P.batch * ((P.T + F - 1) / F);
        NormParams Q = P;
        for (Q.first_tile = 0; Q.first_tile < tiles; Q.first_tile += MAX_TILES)
          hipLaunchKernelGGL((norm_frames_kernel<decltype(y), F, C>), dim3((unsigned)std::min(tiles - Q.first_tile, MAX_TILES)), dim3(FR_THREADS), lds, stream, Q);
        return hipGetLastError();
      });
    });
  return by_types(x_type, y_type, [&](auto x, auto y) {
    return by_width(P.width, [&](auto lanes, auto chunks) {
      constexpr int L = lanes.value, C = chunks.value, groups = threads_of<L>() / L;
      const unsigned grid = (unsigned)std::max(1LL, std::min((P.rows + groups - 1) / groups, 2 * MAX_GROUPS));
      if constexpr (std::is_same<decltype(x), decltype(y)>::value) {
        if (P.codes) {
          hipLaunchKernelGGL((norm_rows_kernel<decltype(x), decltype(y), L, C, true>), dim3(grid), dim3(threads_of<L>()), 0, stream, P);
          return hipGetLastError();
        }
      }
      hipLaunchKernelGGL((norm_rows_kernel<decltype(x), decltype(y), L, C, false>), dim3(grid), dim3(threads_of<L>()), 0, stream, P);
      return hipGetLastError();
    });
  });
}

hipError_t launch_norm_backward(const NormParams& P, int x_type, int g_type, bool frames, float* gw, float* gb, hipStream_t stream) {
  const int grid = norm_backward_groups(P.rows, P.width, frames, P.batch, P.T);
  hipError_t e;
  if (frames)
    e = by_type(g_type, [&](auto y) {
      return by_frame(P.width, [&](auto f, auto pairs) {
        constexpr int F = f.value, C = pairs.value;
        const size_t lds = frames_lds(P.width, F);
        hipLaunchKernelGGL((norm_frames_backward_kernel<decltype(y), F, C>), dim3(grid), dim3(FR_THREADS), lds, stream, P);
        return hipGetLastError();
      });
    });
  else
    e = by_types(x_type, g_type, [&](auto x, auto y) {
      return by_width(P.width, [&](auto lanes, auto chunks) {
        constexpr int L = lanes.value, C = chunks.value;
        if constexpr (std::is_same<decltype(x), decltype(y)>::value) {
          if (P.codes) {
            hipLaunchKernelGGL((norm_rows_backward_kernel<decltype(x), decltype(y), L, C, true>), dim3(grid), dim3(threads_of<L>()), 0, stream, P);
            return hipGetLastError();
          }
        }
        hipLaunchKernelGGL((norm_rows_backward_kernel<decltype(x), decltype(y), L, C, false>), dim3(grid), dim3(threads_of<L>()), 0, stream, P);
        return hipGetLastError();
      });
    });
  if (e != hipSuccess || !P.partial) return e;
  hipLaunchKernelGGL(norm_join_kernel, dim3((2 * P.width + JOIN_COLUMNS - 1) / JOIN_COLUMNS), dim3(JOIN_COLUMNS * JOIN_RUNS), 0, stream, P.partial, grid, P.width, gw, gb);
  return hipGetLastError();
}

// rows whose blocks follow one another without a gap are one row: the kernel's quotients are then none
static void one_row(long long& rows, long long& width, long long row_stride) {
  if (rows > 1 && width % NORM_BLOCK8 == 0 && row_stride == width) {
    width *= rows;
    rows = 1;
  }
}
static unsigned pack_grid(long long rows, long long width) {
  const long long blocks = rows * ((width + NORM_BLOCK8 - 1) / NORM_BLOCK8);
  return (unsigned)std::max(1LL, std::min((blocks + 15) / 16, 4 * MAX_GROUPS));
}

hipError_t launch_pack8(const void* x, int type, long long rows, long long width, long long row_stride, signed char* codes, float* scales, hipStream_t stream) {
  one_row(rows, width, row_stride);
  return by_type(type, [&](auto t) {
    hipLaunchKernelGGL((pack8_kernel<decltype(t)>), dim3(pack_grid(rows, width)), dim3(256), 0, stream, static_cast<const decltype(t)*>(x), rows, width, row_stride,
                       codes, scales);
    return hipGetLastError();
  });
}

hipError_t launch_unpack8(const signed char* codes, const float* scales, long long rows, long long width, void* out, int type, hipStream_t stream) {
  one_row(rows, width, width);
  return by_type(type, [&](auto t) {
    hipLaunchKernelGGL((unpack8_kernel<decltype(t)>), dim3(pack_grid(rows, width)), dim3(256), 0, stream, codes, scales, rows, width, static_cast<decltype(t)*>(out));
    return hipGetLastError();
  });
}

}  // namespace nna
