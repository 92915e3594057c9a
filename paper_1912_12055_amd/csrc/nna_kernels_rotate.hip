// Queries and keys: the norm of each head and the rotation of its pairs by the frame's position, in one pass, and their gradients.
//
//   h = x r,  r = 1 / sqrt(mean(x^2) + eps);   v = h w;   a pair (a, b) of v at position p becomes (a cos - b sin, a sin + b cos) of the angle p f.
//   Backward: g' = the pairs of g rotated by -p f;   gw = sum over rows of g' h;   gx = r (g' w - h mean(g' w h)).
// A row (a head of a frame) is read once into the registers of a few lanes; the angles are the same for all heads of a frame and are made once for all of
// them, in LDS.  An angle is a product of 64 bits, reduced there: far positions leave nothing of one in 32.
#include "nna_norm.h"
#include "nna_rotate.h"
#include "nna_vector.h"

namespace nna {

namespace {

constexpr int THREADS = 256, TABLE = 2048, TOKENS_MAX = 64;
constexpr long long MOST_GROUPS = 1LL << 22;  // of a launch: its threads are counted in 32 bits
constexpr long long MAX_GROUPS = 1024;  // backward: workgroups that leave a partial sum

// Lanes hold V pairs each, LANES = 2^shift lanes a row: of the half layout V neighbours of either half, else 2 V neighbours.  V is the most, up to 16 bytes, that
// divides the rotated half and the head: no vector then holds rotated pairs and others, or ends behind the head.
struct Split {
  int v, shift;
};
Split split_of(int width, int pairs, int size) {
  int v = 16 / size;
  while (v > 1 && (pairs % v || width % (2 * v))) v /= 2;
  if (v == 2) v = 1;  // (two kernels fewer; such heads are short)
  const int lanes = ((width + 1) / 2 + v - 1) / v;
  int shift = 0;
  while ((1 << shift) < lanes && shift < 6) ++shift;
  return {v, shift};
}

__device__ __forceinline__ float2 turn_of(double position, double freq) {
  // cos and sin of position * freq: whole quarters taken off in 64 bits, what is left has 24 bits of its own
  const double angle = position * freq, quarter = __builtin_rint(angle * 0.63661977236758134308);
  const float rest = (float)__builtin_fma(-quarter, 6.123233995736766e-17, __builtin_fma(-quarter, 1.5707963267948966, angle));
  const float s = sinf(rest), c = cosf(rest);
  const int n = (int)(long long)quarter & 3;
  const float cs = n & 1 ? s : c, sn = n & 1 ? c : s;
  return make_float2(n == 1 || n == 2 ? -cs : cs, n >= 2 ? -sn : sn);
}

template <typename T, int V, int CHUNKS, bool INTERLEAVED>
struct Row {
  float a[CHUNKS][V], b[CHUNKS][V];  // pairs
};

// where a lane's values lie in a head: its pairs' number, and the offsets of its two vectors
struct Place {
  int pair, first, second;
  bool has, both;  // V = 1: a head of odd width ends with half a pair
};
template <int V, bool INTERLEAVED>
__device__ __forceinline__ Place place_of(int lane, int chunk, int lanes, int width, int pairs) {
  Place p;
  p.pair = (chunk * lanes + lane) * V;
  const bool halves = !INTERLEAVED && p.pair < pairs;
  p.first = halves ? p.pair : 2 * p.pair;
  p.second = halves ? p.pair + pairs : 2 * p.pair + V;
  p.has = p.first < width;
  p.both = p.second < width;
  return p;
}

template <typename T, int V, int CHUNKS, bool INTERLEAVED>
__device__ __forceinline__ void load_row(Row<T, V, CHUNKS, INTERLEAVED>& row, const T* x, const Place (&p)[CHUNKS]) {
#pragma unroll
  for (int c = 0; c < CHUNKS; ++c) {
    typename Vec<T, V>::plain u, v;
#pragma unroll
    for (int e = 0; e < V; ++e) vec_set<V>(u, e, (T)0.f), vec_set<V>(v, e, (T)0.f);
    if (p[c].has) u = vec_load<V>(x + p[c].first);
    if (V > 1 ? p[c].has : p[c].both) v = vec_load<V>(x + p[c].second);
#pragma unroll
    for (int e = 0; e < V; ++e) {
      // (behind the rotated part of the half layout any two may be called a pair)
      const float f = (float)vec_at<V>(u, e), s = (float)vec_at<V>(v, e);
      if (!INTERLEAVED || V == 1) {
        row.a[c][e] = f;
        row.b[c][e] = s;
      } else {
        const int at = e * 2;
        row.a[c][e] = (float)(at < V ? vec_at<V>(u, at) : vec_at<V>(v, at - V));
        row.b[c][e] = (float)(at < V ? vec_at<V>(u, at + 1) : vec_at<V>(v, at + 1 - V));
      }
    }
  }
}
template <typename T, int V, int CHUNKS, bool INTERLEAVED>
__device__ __forceinline__ void store_row(const Row<T, V, CHUNKS, INTERLEAVED>& row, T* y, const Place (&p)[CHUNKS]) {
#pragma unroll
  for (int c = 0; c < CHUNKS; ++c) {
    typename Vec<T, V>::plain u, v;
#pragma unroll
    for (int e = 0; e < V; ++e) {
      if (!INTERLEAVED || V == 1) {
        vec_set<V>(u, e, (T)row.a[c][e]);
        vec_set<V>(v, e, (T)row.b[c][e]);
      } else {
        const int i = e / 2;
        vec_set<V>(u, e, (T)(e & 1 ? row.b[c][i] : row.a[c][i]));
        vec_set<V>(v, e, (T)(e & 1 ? row.b[c][V / 2 + i] : row.a[c][V / 2 + i]));
      }
    }
    if (p[c].has) vec_store<V>(y + p[c].first, u);
    if (V > 1 ? p[c].has : p[c].both) vec_store<V>(y + p[c].second, v);
  }
}

// the sum over 2^shift neighbouring lanes, in all of them
__device__ __forceinline__ float row_sum(float v, int shift) {
  for (int s = 0; s < shift; ++s) v += __shfl_xor(v, 1 << s);
  return v;
}

// a workgroup's tokens: where their rows begin, and their angles
struct Tokens {
  long long q[TOKENS_MAX], k[TOKENS_MAX];
  float2 turn[TABLE];
};
__device__ __forceinline__ void make_tokens(const RotateParams& P, Tokens& at, long long first, int count) {
  const int threads = THREADS;
  for (int i = threadIdx.x; i < count; i += threads) {
    const long long n = first + i, b = n / P.T, t = n - b * P.T;
    at.q[i] = b * P.q.x_b + t * P.q.x_t;
    at.k[i] = b * P.k.x_b + t * P.k.x_t;
  }
  for (int i = threadIdx.x; i < count * P.pairs; i += threads) {
    const int token = i / P.pairs, pair = i - token * P.pairs;
    const long long n = first + token, b = n / P.T, t = n - b * P.T;
    at.turn[i] = turn_of(P.positions ? (double)P.positions[b * P.p_b + t * P.p_t] : (double)(P.offset + t), P.freqs[pair]);
  }
}

template <typename T, int V, int CHUNKS, bool INTERLEAVED>
__global__ __launch_bounds__(THREADS) void rotate_kernel(RotateParams P, int shift, int tokens) {
  __shared__ Tokens at;
  const long long first = P.first_token + (long long)blockIdx.x * tokens;
  const int count = (int)std::min((long long)tokens, P.B * P.T - first), heads = P.q.heads + P.k.heads;
  make_tokens(P, at, first, count);
  __syncthreads();
  const int lanes = 1 << shift, lane = threadIdx.x & (lanes - 1), slots = THREADS >> shift;
  Place p[CHUNKS];
#pragma unroll
  for (int c = 0; c < CHUNKS; ++c) p[c] = place_of<V, INTERLEAVED>(lane, c, lanes, P.width, P.pairs);
  // (whole waves go round together: the sum over a row's lanes needs them all)
  for (int base = 0; base < count * heads; base += slots) {
    const int r = base + (int)(threadIdx.x >> shift);
    const bool here = r < count * heads;
    const int row = here ? r : 0, token = row / heads, h = row - token * heads;
    const bool query = h < P.q.heads;
    const RotateHeads& H = query ? P.q : P.k;
    const int head = query ? h : h - P.q.heads;
    Row<T, V, CHUNKS, INTERLEAVED> v;
    load_row(v, static_cast<const T*>(H.x) + (query ? at.q[token] : at.k[token]) + head * H.x_h, p);
    float scale = 1.f;
    if (P.norm) {
      float sum = 0.f;
#pragma unroll
      for (int c = 0; c < CHUNKS; ++c)
#pragma unroll
        for (int e = 0; e < V; ++e) sum += v.a[c][e] * v.a[c][e] + v.b[c][e] * v.b[c][e];
      scale = 1.f / sqrtf(row_sum(sum, shift) / (float)P.width + P.eps);
      Row<float, V, CHUNKS, INTERLEAVED> w;
      if (H.weight) load_row(w, H.weight, p);
#pragma unroll
      for (int c = 0; c < CHUNKS; ++c)
#pragma unroll
        for (int e = 0; e < V; ++e) {
          v.a[c][e] *= scale * (H.weight ? w.a[c][e] : 1.f);
          v.b[c][e] *= scale * (H.weight ? w.b[c][e] : 1.f);
        }
    }
#pragma unroll
    for (int c = 0; c < CHUNKS; ++c)
      if (p[c].pair < P.pairs)
#pragma unroll
        for (int e = 0; e < V; ++e) {
          const float2 u = at.turn[token * P.pairs + p[c].pair + e];
          const float a = v.a[c][e], b = v.b[c][e];
          v.a[c][e] = a * u.x - b * u.y;
          v.b[c][e] = a * u.y + b * u.x;
        }
    if (here) store_row(v, static_cast<T*>(H.y) + ((first + token) * H.heads + head) * P.width, p);
  }
}

template <typename T, int V, int CHUNKS, bool INTERLEAVED>
__global__ __launch_bounds__(THREADS) void rotate_backward_kernel(RotateParams P, int shift, int tokens) {
  __shared__ Tokens at;
  __shared__ float sums[THREADS * 2 * V * CHUNKS];  // [slots][lanes][2 V]: a slot's sums
  const int heads = P.q.heads + P.k.heads;
  const int lanes = 1 << shift, lane = threadIdx.x & (lanes - 1), slots = THREADS >> shift;
  Place p[CHUNKS];
#pragma unroll
  for (int c = 0; c < CHUNKS; ++c) p[c] = place_of<V, INTERLEAVED>(lane, c, lanes, P.width, P.pairs);
  Row<float, V, CHUNKS, INTERLEAVED> gq = {}, gk = {};
  for (long long first = (long long)blockIdx.x * tokens; first < P.B * P.T; first += (long long)gridDim.x * tokens) {
    const int count = (int)std::min((long long)tokens, P.B * P.T - first);
    __syncthreads();
    make_tokens(P, at, first, count);
    __syncthreads();
    for (int base = 0; base < count * heads; base += slots) {
      const int r = base + (int)(threadIdx.x >> shift);
      const bool here = r < count * heads;
      const int row = here ? r : 0, token = row / heads, h = row - token * heads;
      const bool query = h < P.q.heads;
      const RotateHeads& H = query ? P.q : P.k;
      const int head = query ? h : h - P.q.heads;
      const long long packed = ((first + token) * H.heads + head) * P.width;
      Row<T, V, CHUNKS, INTERLEAVED> g;
      load_row(g, static_cast<const T*>(H.g) + packed, p);
#pragma unroll
      for (int c = 0; c < CHUNKS; ++c)
        if (p[c].pair < P.pairs)
#pragma unroll
          for (int e = 0; e < V; ++e) {
            const float2 u = at.turn[token * P.pairs + p[c].pair + e];
            const float a = g.a[c][e], b = g.b[c][e];
            g.a[c][e] = a * u.x + b * u.y;
            g.b[c][e] = b * u.x - a * u.y;
          }
      if (P.norm) {
        Row<T, V, CHUNKS, INTERLEAVED> v;
        load_row(v, static_cast<const T*>(H.x) + (query ? at.q[token] : at.k[token]) + head * H.x_h, p);
        Row<float, V, CHUNKS, INTERLEAVED> w;
        if (H.weight) load_row(w, H.weight, p);
        float square = 0.f;
#pragma unroll
        for (int c = 0; c < CHUNKS; ++c)
#pragma unroll
          for (int e = 0; e < V; ++e) square += v.a[c][e] * v.a[c][e] + v.b[c][e] * v.b[c][e];
        const float scale = 1.f / sqrtf(row_sum(square, shift) / (float)P.width + P.eps);
        float dot = 0.f;
#pragma unroll
        for (int c = 0; c < CHUNKS; ++c)
#pragma unroll
          for (int e = 0; e < V; ++e) {
            v.a[c][e] *= scale;
            v.b[c][e] *= scale;
            if (here && P.partial) {
              (query ? gq : gk).a[c][e] += g.a[c][e] * v.a[c][e];
              (query ? gq : gk).b[c][e] += g.b[c][e] * v.b[c][e];
            }
            g.a[c][e] *= H.weight ? w.a[c][e] : 1.f;
            g.b[c][e] *= H.weight ? w.b[c][e] : 1.f;
            dot += g.a[c][e] * v.a[c][e] + g.b[c][e] * v.b[c][e];
          }
        dot = row_sum(dot, shift) / (float)P.width;
#pragma unroll
        for (int c = 0; c < CHUNKS; ++c)
#pragma unroll
          for (int e = 0; e < V; ++e) {
            g.a[c][e] = scale * (g.a[c][e] - v.a[c][e] * dot);
            g.b[c][e] = scale * (g.b[c][e] - v.b[c][e] * dot);
          }
      }
      if (here) store_row(g, static_cast<T*>(H.y) + packed, p);
    }
  }
  if (!P.partial) return;
  // the slots' sums in order: one value of a head after the other, as they lie in it
  for (int part = 0; part < 2; ++part) {
    __syncthreads();
    const Row<float, V, CHUNKS, INTERLEAVED>& s = part ? gk : gq;
    const int pitch = 2 * V * CHUNKS * lanes;
    store_row(s, sums + (threadIdx.x >> shift) * pitch, p);
    __syncthreads();
    for (int d = threadIdx.x; d < P.width; d += THREADS) {
      float sum = sums[d];
      for (int i = 1; i < slots; ++i) sum += sums[i * pitch + d];
      P.partial[((long long)blockIdx.x * 2 + part) * P.width + d] = sum;
    }
  }
}

// tokens of a workgroup at a time: some four rows for each of its slots, no more than the table of angles holds
int tokens_of(int heads, int pairs, const Split& s) {
  int n = std::max(1, (4 * THREADS >> s.shift) / heads);
  n = std::min(n, TOKENS_MAX);
  return pairs ? std::min(n, TABLE / pairs) : n;
}

// fn(pairs of a lane, times that many, layout)
template <typename T, typename F>
hipError_t by_split(const Split& s, int width, bool interleaved, F fn) {
  const auto layout = [&](auto v, auto chunks) { return interleaved ? fn(v, chunks, std::true_type()) : fn(v, chunks, std::false_type()); };
  if constexpr (sizeof(T) == 2)
    if (s.v == 8) return layout(std::integral_constant<int, 8>(), std::integral_constant<int, 1>());
  if (s.v == 4) return layout(std::integral_constant<int, 4>(), std::integral_constant<int, 1>());
  if (width <= 128) return layout(std::integral_constant<int, 1>(), std::integral_constant<int, 1>());
  return layout(std::integral_constant<int, 1>(), std::integral_constant<int, 2>());
}

}  // namespace

int rotate_backward_groups(long long tokens, int heads, int width, int pairs, int type) {
  const int each = tokens_of(heads, pairs, split_of(width, pairs, type == NNA_F32 ? 4 : 2));
  return (int)std::max(1LL, std::min((tokens + each - 1) / each, MAX_GROUPS));
}

hipError_t launch_rotate(const RotateParams& P, int type, hipStream_t stream) {
  return by_element(type, [&](auto t) {
    typedef decltype(t) T;
    const Split s = split_of(P.width, P.pairs, sizeof(T));
    return by_split<T>(s, P.width, P.interleaved, [&](auto v, auto chunks, auto layout) {
      const int tokens = tokens_of(P.q.heads + P.k.heads, P.pairs, s);
      const long long groups = (P.B * P.T + tokens - 1) / tokens;
      RotateParams Q = P;
      for (long long g = 0; g < groups; g += MOST_GROUPS) {
        Q.first_token = g * tokens;
        hipLaunchKernelGGL((rotate_kernel<T, v.value, chunks.value, layout.value>), dim3((unsigned)std::min(groups - g, MOST_GROUPS)), dim3(THREADS), 0, stream, Q,
                           s.shift, tokens);
      }
      return hipGetLastError();
    });
  });
}

hipError_t launch_rotate_backward(const RotateParams& P, int type, float* gqw, float* gkw, hipStream_t stream) {
  const int grid = rotate_backward_groups(P.B * P.T, P.q.heads + P.k.heads, P.width, P.pairs, type);
  const hipError_t e = by_element(type, [&](auto t) {
    typedef decltype(t) T;
    const Split s = split_of(P.width, P.pairs, sizeof(T));
    return by_split<T>(s, P.width, P.interleaved, [&](auto v, auto chunks, auto layout) {
      const int tokens = tokens_of(P.q.heads + P.k.heads, P.pairs, s);
      hipLaunchKernelGGL((rotate_backward_kernel<T, v.value, chunks.value, layout.value>), dim3(grid), dim3(THREADS), 0, stream, P, s.shift, tokens);
      return hipGetLastError();
    });
  });
  if (e != hipSuccess || !P.partial) return e;
  return launch_norm_join(P.partial, grid, P.width, gqw, gkw, stream);
}

}  // namespace nna
