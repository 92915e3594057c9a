// Layer norm of rows and of frames, forward and backward, and values kept in 8 bits.
//
// A row's mean m, r = 1 / sqrt(mean((x - m)^2) + eps) and h = (x - m) r give y = h w + b; with gh = gy w,
//   gx = r (gh - mean(gh) - h mean(gh h)),   gw = sum over rows of gy h,   gb = sum over rows of gy.
// All of it is some ten operations a value: the bytes bound it.  A row is read once into registers (of 16 lanes up to a
// workgroup, eight neighbours a lane at a time), the mean is known before the squares are summed, and every sum is float32.
#include "nna_norm.h"

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
__device__ __forceinline__ f32x8 load_codes(const signed char* p, int n, float scale) {
  f32x8 v;
  if (n >= 8) {
    const i8x8 c = *reinterpret_cast<const i8x8*>(p);
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = (float)c[i] * scale;
    return v;
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = i < n ? (float)p[i] * scale : 0.f;
  return v;
}
// the largest of 16 neighbouring lanes' magnitudes: NaN beats all
__device__ __forceinline__ float most16(float m) {
#pragma unroll
  for (int d = 1; d < 16; d <<= 1) {
    const float o = __shfl_xor(m, d);
    m = o <= m || m != m ? m : o;
  }
  return m;
}

// ---- sums over the lanes that hold a row ---------------------------------------------------------------------------------
template <int LANES>
__device__ __forceinline__ float2 row_sum(float2 v, float2* lds, int& turn) {
#pragma unroll
  for (int d = (LANES < 64 ? LANES : 64) / 2; d; d >>= 1) {
    v.x += __shfl_xor(v.x, d);
    v.y += __shfl_xor(v.y, d);
  }
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

// Rows in registers: LANES lanes hold a row, CHUNKS times eight values each.  The weights stay in registers over all rows of a lane.
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
// LDS in a fixed order, one partial sum a workgroup.
template <typename TX, typename TY, int LANES, int CHUNKS, bool KEPT8>
__global__ __launch_bounds__(threads_of<LANES>()) void norm_rows_backward_kernel(NormParams P) {
  constexpr int GROUPS = threads_of<LANES>() / LANES;
  __shared__ float2 lds[2 * (LANES > 64 ? LANES / 64 : 1)];
  __shared__ float joined[GROUPS > 1 ? LANES * CHUNKS * 8 : 1];
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
  int turn = 0;
  for (long long row = (long long)blockIdx.x * GROUPS + group; row < P.rows; row += (long long)gridDim.x * GROUPS) {
    const TY* gout = static_cast<const TY*>(P.gout) + row * width;
    const float mean = P.stats[2 * row], rstd = P.stats[2 * row + 1];
    f32x8 h[CHUNKS], gh[CHUNKS];
    float2 s = {0.f, 0.f};
#pragma unroll
    for (int c = 0; c < CHUNKS; ++c) {
      const int at = (lane + c * LANES) * 8;
      h[c] = gh[c] = 0.f;
      if (n[c] > 0) {
        const f32x8 g = load8(gout + at, n[c]);
        if constexpr (KEPT8)
          h[c] = load_codes(P.codes + row * width + at, n[c], P.scales[row * blocks + at / NORM_BLOCK8]);
        else
          h[c] = load8(static_cast<const TX*>(P.x) + row * P.row_stride + at, n[c]);
        h[c] = (h[c] - mean) * rstd;
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
      if (n[c] > 0) store8(gx + (lane + c * LANES) * 8, n[c], (gh[c] - s.x - h[c] * s.y) * rstd);
  }
  if (!P.partial) return;
  float* out = P.partial + (long long)blockIdx.x * 2 * width;
#pragma unroll
  for (int part = 0; part < 2; ++part) {
#pragma unroll
    for (int g = GROUPS - 1; g > 0; --g) {
      if (group == g)
#pragma unroll
        for (int c = 0; c < CHUNKS; ++c)
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            float& at = joined[(lane + c * LANES) * 8 + i];
            const float v = (part ? gb : gw)[c][i];
            at = g == GROUPS - 1 ? v : at + v;
          }
      __syncthreads();
    }
    if (group == 0)
#pragma unroll
      for (int c = 0; c < CHUNKS; ++c) {
        f32x8 v = (part ? gb : gw)[c];
        if constexpr (GROUPS > 1)
#pragma unroll
          for (int i = 0; i < 8; ++i) v[i] += joined[(lane + c * LANES) * 8 + i];
        if (n[c] > 0) store8(out + part * width + (lane + c * LANES) * 8, n[c], v);
      }
    __syncthreads();
  }
}

// gw, gb: the sum of the workgroups' partial sums, 16 runs of them side by side and joined in order
constexpr int JOIN_COLUMNS = 64, JOIN_RUNS = 16;
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
// A workgroup takes FRAMES neighbouring frames of a waveform: their columns are read along T, turned in LDS, and every frame is a row
// there, which a wave holds COLUMNS values a lane of.  y and gout are rows [B, T, width]; gx goes back the way x came.
constexpr int FR_THREADS = 256, FR_WAVES = FR_THREADS / 64;
__host__ __device__ constexpr int frames_pitch(int width) { return width | 1; }  // odd: a column's frames are in different banks
// as many frames as leave two workgroups of 72 KB a CU: 128 (64, 32) consecutive bytes of every bin
constexpr int FR_WIDTH_32 = 558, FR_WIDTH_16 = 1088;
constexpr int frames_per_tile(int width) { return width <= FR_WIDTH_32 ? 32 : width <= FR_WIDTH_16 ? 16 : 8; }

template <int FRAMES, typename F>
__device__ __forceinline__ void each_of_tile(int width, int frames, F fn) {
  const int t = threadIdx.x % FRAMES;
  if (t < frames)
#pragma unroll 8
    for (int d = threadIdx.x / FRAMES; d < width; d += FR_THREADS / FRAMES) fn(d, t);
}
__device__ __forceinline__ float wave_sum(float v) {
#pragma unroll
  for (int d = 32; d; d >>= 1) v += __shfl_xor(v, d);
  return v;
}

template <typename TY, int FRAMES, int COLUMNS>
__global__ __launch_bounds__(FR_THREADS) void norm_frames_kernel(NormParams P) {
  extern __shared__ float tile[];
  const int width = P.width, pitch = frames_pitch(width), lane = threadIdx.x & 63;
  const long long tiles = (P.T + FRAMES - 1) / FRAMES;
  const float inv = 1.f / (float)width;
  const long long b = blockIdx.x / tiles, t0 = (blockIdx.x % tiles) * FRAMES;
  const int frames = (int)(P.T - t0 < FRAMES ? P.T - t0 : FRAMES);
  const float* x = static_cast<const float*>(P.x) + b * width * P.T + t0;
  each_of_tile<FRAMES>(width, frames, [&](int d, int t) { tile[t * pitch + d] = x[(long long)d * P.T + t]; });
  __syncthreads();
  for (int t = threadIdx.x >> 6; t < frames; t += FR_WAVES) {
    float v[COLUMNS], s = 0.f;
#pragma unroll
    for (int c = 0; c < COLUMNS; ++c) {
      const int d = lane + c * 64;
      v[c] = d < width ? tile[t * pitch + d] : 0.f;
      s += v[c];
    }
    const float mean = wave_sum(s) * inv;
    s = 0.f;
#pragma unroll
    for (int c = 0; c < COLUMNS; ++c)
      if (lane + c * 64 < width) s += (v[c] - mean) * (v[c] - mean);
    const float rstd = 1.f / sqrtf(wave_sum(s) * inv + P.eps);
    const long long row = b * P.T + t0 + t;
    TY* y = static_cast<TY*>(P.y) + row * width;
#pragma unroll
    for (int c = 0; c < COLUMNS; ++c) {
      const int d = lane + c * 64;
      if (d < width) y[d] = (TY)((v[c] - mean) * rstd * (P.weight ? P.weight[d] : 1.f) + (P.bias ? P.bias[d] : 0.f));
    }
    if (P.stats && lane == 0) {
      P.stats[2 * row] = mean;
      P.stats[2 * row + 1] = rstd;
    }
  }
}

template <typename TY, int FRAMES, int COLUMNS>
__global__ __launch_bounds__(FR_THREADS) void norm_frames_backward_kernel(NormParams P) {
  extern __shared__ float tile[];
  const int width = P.width, pitch = frames_pitch(width), lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const long long tiles = (P.T + FRAMES - 1) / FRAMES;
  const float inv = 1.f / (float)width;
  float gw[COLUMNS], gb[COLUMNS], w[COLUMNS];
#pragma unroll
  for (int c = 0; c < COLUMNS; ++c) {
    const int d = lane + c * 64;
    gw[c] = gb[c] = 0.f;
    w[c] = d >= width ? 0.f : P.weight ? P.weight[d] : 1.f;
  }
  for (long long i = blockIdx.x; i < P.batch * tiles; i += gridDim.x) {
    const long long b = i / tiles, t0 = (i % tiles) * FRAMES;
    const int frames = (int)(P.T - t0 < FRAMES ? P.T - t0 : FRAMES);
    const float* x = static_cast<const float*>(P.x) + b * width * P.T + t0;
    each_of_tile<FRAMES>(width, frames, [&](int d, int t) { tile[t * pitch + d] = x[(long long)d * P.T + t]; });
    __syncthreads();
    for (int t = wave; t < frames; t += FR_WAVES) {
      const long long row = b * P.T + t0 + t;
      const TY* gout = static_cast<const TY*>(P.gout) + row * width;
      const float mean = P.stats[2 * row], rstd = P.stats[2 * row + 1];
      float h[COLUMNS], gh[COLUMNS], s0 = 0.f, s1 = 0.f;
#pragma unroll
      for (int c = 0; c < COLUMNS; ++c) {
        const int d = lane + c * 64;
        h[c] = gh[c] = 0.f;
        if (d < width) {
          const float g = (float)gout[d];
          h[c] = (tile[t * pitch + d] - mean) * rstd;
          gw[c] += g * h[c];
          gb[c] += g;
          gh[c] = g * w[c];
          s0 += gh[c];
          s1 += gh[c] * h[c];
        }
      }
      s0 = wave_sum(s0) * inv;
      s1 = wave_sum(s1) * inv;
#pragma unroll
      for (int c = 0; c < COLUMNS; ++c) {
        const int d = lane + c * 64;
        if (d < width) tile[t * pitch + d] = (gh[c] - s0 - h[c] * s1) * rstd;
      }
    }
    __syncthreads();
    if (P.gx) {
      float* gx = static_cast<float*>(P.gx) + b * width * P.T + t0;
      each_of_tile<FRAMES>(width, frames, [&](int d, int t) { gx[(long long)d * P.T + t] = tile[t * pitch + d]; });
    }
    __syncthreads();
  }
  if (!P.partial) return;
  float* out = P.partial + (long long)blockIdx.x * 2 * width;
  for (int g = FR_WAVES - 1; g >= 0; --g) {  // the waves' sums, one after the other: tile holds at least 8 rows
    if (wave == g)
#pragma unroll
      for (int c = 0; c < COLUMNS; ++c) {
        const int d = lane + c * 64;
        if (d < width) {
          if (g < FR_WAVES - 1) {
            gw[c] += tile[d];
            gb[c] += tile[width + d];
          }
          tile[d] = gw[c];
          tile[width + d] = gb[c];
          if (g == 0) {
            out[d] = gw[c];
            out[width + d] = gb[c];
          }
        }
      }
    __syncthreads();
  }
}

// ---- values to 8 bits and back -------------------------------------------------------------------------------------------
// 16 lanes take a block: 8 values each
template <typename T>
__global__ __launch_bounds__(256) void pack8_kernel(const T* x, long long rows, long long width, long long row_stride, signed char* codes, float* scales) {
  const long long blocks = (width + NORM_BLOCK8 - 1) / NORM_BLOCK8;
  for (long long i = ((long long)blockIdx.x * 256 + threadIdx.x) >> 4; i < rows * blocks; i += (long long)gridDim.x * 16) {
    const long long row = i / blocks, at = (i % blocks) * NORM_BLOCK8 + (threadIdx.x & 15) * 8;
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
    const long long row = i / blocks, at = (i % blocks) * NORM_BLOCK8 + (threadIdx.x & 15) * 8;
    const int n = width - at > 8 ? 8 : (int)(width - at);
    if (n > 0) store8(out + row * width + at, n, load_codes(codes + row * width + at, n, scales[i]));
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
template <typename F>
hipError_t by_frame(int width, F fn) {
  if (width <= 128) return fn(std::integral_constant<int, 32>(), std::integral_constant<int, 2>());
  if (width <= 256) return fn(std::integral_constant<int, 32>(), std::integral_constant<int, 4>());
  if (width <= FR_WIDTH_32) return fn(std::integral_constant<int, 32>(), std::integral_constant<int, 9>());
  if (width <= FR_WIDTH_16) return fn(std::integral_constant<int, 16>(), std::integral_constant<int, 17>());
  return fn(std::integral_constant<int, 8>(), std::integral_constant<int, 33>());
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
      const hipError_t e = by_type(type, [&](auto y) { return by_frame(width, [&](auto f, auto columns) { return frames_init<decltype(y), f.value, columns.value>(); }); });
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
      return by_frame(P.width, [&](auto f, auto columns) {
        constexpr int F = f.value, C = columns.value;
        const size_t lds = frames_lds(P.width, F);
        hipLaunchKernelGGL((norm_frames_kernel<decltype(y), F, C>), dim3((unsigned)(P.batch * ((P.T + F - 1) / F))), dim3(FR_THREADS), lds, stream, P);
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
      return by_frame(P.width, [&](auto f, auto columns) {
        constexpr int F = f.value, C = columns.value;
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

static unsigned pack_grid(long long rows, long long width) {
  const long long blocks = rows * ((width + NORM_BLOCK8 - 1) / NORM_BLOCK8);
  return (unsigned)std::max(1LL, std::min((blocks + 15) / 16, 4 * MAX_GROUPS));
}

hipError_t launch_pack8(const void* x, int type, long long rows, long long width, long long row_stride, signed char* codes, float* scales, hipStream_t stream) {
  return by_type(type, [&](auto t) {
    hipLaunchKernelGGL((pack8_kernel<decltype(t)>), dim3(pack_grid(rows, width)), dim3(256), 0, stream, static_cast<const decltype(t)*>(x), rows, width, row_stride,
                       codes, scales);
    return hipGetLastError();
  });
}

hipError_t launch_unpack8(const signed char* codes, const float* scales, long long rows, long long width, void* out, int type, hipStream_t stream) {
  return by_type(type, [&](auto t) {
    hipLaunchKernelGGL((unpack8_kernel<decltype(t)>), dim3(pack_grid(rows, width)), dim3(256), 0, stream, codes, scales, rows, width, static_cast<decltype(t)*>(out));
    return hipGetLastError();
  });
}

}  // namespace nna
