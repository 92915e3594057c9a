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

// cos and sin of position * freq: whole quarters taken off in 64 bits; of what is left, an eighth of a turn at most, the series to the terms that 2^-28 can tell
__device__ __forceinline__ float2 turn_of(double position, double freq) {
  const double angle = position * freq, quarter = __builtin_rint(angle * 0.63661977236758134308);
  const float x = (float)__builtin_fma(-quarter, 6.123233995736766e-17, __builtin_fma(-quarter, 1.5707963267948966, angle)), z = x * x;
  const float s = __builtin_fmaf(x * z, __builtin_fmaf(z, __builtin_fmaf(z, __builtin_fmaf(z, 1.f / 362880, -1.f / 5040), 1.f / 120), -1.f / 6), x);
  const float c = __builtin_fmaf(z * z, __builtin_fmaf(z, __builtin_fmaf(z, __builtin_fmaf(z, -1.f / 3628800, 1.f / 40320), -1.f / 720), 1.f / 24), __builtin_fmaf(z, -0.5f, 1.f));
  const int n = (int)(long long)quarter & 3;
  const float cs = n & 1 ? s : c, sn = n & 1 ? c : s;
  return make_float2(n == 1 || n == 2 ? -cs : cs, n >= 2 ? -sn : sn);
}

template <int V, int CHUNKS>
struct Row {
  float a[CHUNKS][V], b[CHUNKS][V];  // pairs
};
// ... as it lies in memory
template <typename T, int V, int CHUNKS>
struct Raw {
  typename Vec<T, V>::plain u[CHUNKS], v[CHUNKS];
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

template <typename T, int V, int CHUNKS>
__device__ __forceinline__ void load_raw(Raw<T, V, CHUNKS>& raw, const T* x, const Place (&p)[CHUNKS]) {
#pragma unroll
  for (int c = 0; c < CHUNKS; ++c) {
#pragma unroll
    for (int e = 0; e < V; ++e) vec_set<V>(raw.u[c], e, (T)0.f), vec_set<V>(raw.v[c], e, (T)0.f);
    if (p[c].has) raw.u[c] = vec_load<V>(x + p[c].first);
    if (V > 1 ? p[c].has : p[c].both) raw.v[c] = vec_load<V>(x + p[c].second);
  }
}
template <bool INTERLEAVED, typename T, int V, int CHUNKS>
__device__ __forceinline__ Row<V, CHUNKS> row_of(const Raw<T, V, CHUNKS>& raw) {
  Row<V, CHUNKS> row;
#pragma unroll
  for (int c = 0; c < CHUNKS; ++c)
#pragma unroll
    for (int e = 0; e < V; ++e) {
      // (behind the rotated part of the half layout any two may be called a pair)
      if (!INTERLEAVED || V == 1) {
        row.a[c][e] = (float)vec_at<V>(raw.u[c], e);
        row.b[c][e] = (float)vec_at<V>(raw.v[c], e);
      } else {
        const int at = e * 2;
        row.a[c][e] = (float)(at < V ? vec_at<V>(raw.u[c], at) : vec_at<V>(raw.v[c], at - V));
        row.b[c][e] = (float)(at < V ? vec_at<V>(raw.u[c], at + 1) : vec_at<V>(raw.v[c], at + 1 - V));
      }
    }
  return row;
}
template <bool INTERLEAVED, typename T, int V, int CHUNKS>
__device__ __forceinline__ void store_row(const Row<V, CHUNKS>& row, T* y, const Place (&p)[CHUNKS]) {
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

// the sum over 2^shift neighbouring lanes, in all of them: mirrored within 4, 8 and 16 lanes (whose sums so far are equal), then rows of 16 and halves of the wave
template <int CONTROL>
__device__ __forceinline__ float moved(float v) {
  return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), CONTROL, 0xf, 0xf, true));
}
__device__ __forceinline__ float row_sum(float v, int shift) {
  if (shift > 0) v += moved<0xB1>(v);   // 1 0 3 2
  if (shift > 1) v += moved<0x4E>(v);   // 2 3 0 1
  if (shift > 2) v += moved<0x141>(v);  // 7 to 0
  if (shift > 3) v += moved<0x140>(v);  // 15 to 0
  if (shift > 4) {
    const auto p = __builtin_amdgcn_permlane16_swap(__builtin_bit_cast(unsigned, v), __builtin_bit_cast(unsigned, v), false, false);
    const unsigned a = p[0], b = p[1];
    v = __builtin_bit_cast(float, a) + __builtin_bit_cast(float, b);
  }
  if (shift > 5) {
    const auto p = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(unsigned, v), __builtin_bit_cast(unsigned, v), false, false);
    const unsigned a = p[0], b = p[1];
    v = __builtin_bit_cast(float, a) + __builtin_bit_cast(float, b);
  }
  return v;
}

// A workgroup's tokens: `count` from `first` on, where their queries and keys begin, and their angles.
struct Tokens {
  long long q[TOKENS_MAX], k[TOKENS_MAX];
  float2 turns[TABLE];
};
__device__ __forceinline__ void make_tokens(const RotateParams& P, Tokens& at, long long first, int count) {
  const long long b0 = first / P.T;
  const unsigned t0 = (unsigned)(first - b0 * P.T), T = (unsigned)P.T;
  const auto place = [&](int token, long long& b, long long& t) {
    const unsigned u = t0 + token, over = u / T;
    b = b0 + over;
    t = u - over * T;
  };
  for (int i = threadIdx.x; i < count; i += THREADS) {
    long long b, t;
    place(i, b, t);
    at.q[i] = b * P.q.x_b + t * P.q.x_t;
    at.k[i] = b * P.k.x_b + t * P.k.x_t;
  }
  for (int i = threadIdx.x; i < count * P.pairs; i += THREADS) {
    const int token = i / P.pairs, pair = i - token * P.pairs;
    long long b, t;
    place(token, b, t);
    at.turns[i] = turn_of(P.positions ? (double)P.positions[b * P.p_b + t * P.p_t] : (double)(P.offset + t), P.freqs[pair]);
  }
}

// Row r of some tokens' queries or keys, and where it lies.  (r / heads by the rounded-up quotient of 2^32: r is below 2^12 where there is more than one token.)
struct Where {
  int token, r;
  long long x;
  __device__ __forceinline__ Where(const RotateHeads& H, const long long* starts, int count, int row) : r(row) {
    token = count == 1 ? 0 : (int)(((unsigned long long)row * H.inverse) >> 32);
    x = starts[token] + (row - token * H.heads) * H.x_h;
  }
};

// a pair (a, b) turned on or back
template <int V, int CHUNKS>
__device__ __forceinline__ void turn_row(Row<V, CHUNKS>& v, const float2* turns, const Place (&p)[CHUNKS], int pairs, float way) {
#pragma unroll
  for (int c = 0; c < CHUNKS; ++c)
    if (p[c].pair < pairs)
#pragma unroll
      for (int e = 0; e < V; ++e) {
        const float2 u = turns[p[c].pair + e];
        const float a = v.a[c][e], b = v.b[c][e], s = u.y * way;
        v.a[c][e] = a * u.x - b * s;
        v.b[c][e] = a * s + b * u.x;
      }
}

template <int V, int CHUNKS>
__device__ __forceinline__ float dot(const Row<V, CHUNKS>& x, const Row<V, CHUNKS>& y) {
  float sum = 0.f;
#pragma unroll
  for (int c = 0; c < CHUNKS; ++c)
#pragma unroll
    for (int e = 0; e < V; ++e) sum += x.a[c][e] * y.a[c][e] + x.b[c][e] * y.b[c][e];
  return sum;
}

template <typename F, int V, int CHUNKS>
__device__ __forceinline__ void each_value(Row<V, CHUNKS>& x, const Row<V, CHUNKS>& y, F fn) {
#pragma unroll
  for (int c = 0; c < CHUNKS; ++c)
#pragma unroll
    for (int e = 0; e < V; ++e) {
      x.a[c][e] = fn(x.a[c][e], y.a[c][e]);
      x.b[c][e] = fn(x.b[c][e], y.b[c][e]);
    }
}

template <bool INTERLEAVED, int V, int CHUNKS>
__device__ __forceinline__ Row<V, CHUNKS> weights_of(const float* weight, const Place (&p)[CHUNKS]) {
  Raw<float, V, CHUNKS> raw;
  if (weight) {
    load_raw(raw, weight, p);
    return row_of<INTERLEAVED>(raw);
  }
  Row<V, CHUNKS> ones;
#pragma unroll
  for (int c = 0; c < CHUNKS; ++c)
#pragma unroll
    for (int e = 0; e < V; ++e) ones.a[c][e] = ones.b[c][e] = 1.f;
  return ones;
}

template <typename T, int V, int CHUNKS, bool INTERLEAVED>
__global__ __launch_bounds__(THREADS) void rotate_kernel(RotateParams P, int shift, int each) {
  __shared__ Tokens at;
  const long long first = P.first_token + (long long)blockIdx.x * each;
  const int count = (int)std::min((long long)each, P.B * P.T - first);
  const int lane = threadIdx.x & ((1 << shift) - 1), slot = threadIdx.x >> shift, slots = THREADS >> shift;
  Place p[CHUNKS];
#pragma unroll
  for (int c = 0; c < CHUNKS; ++c) p[c] = place_of<V, INTERLEAVED>(lane, c, 1 << shift, P.width, P.pairs);
  make_tokens(P, at, first, count);
  __syncthreads();
  const auto run = [&](const RotateHeads& H, const long long* starts) {
    const int rows = count * H.heads;
    T* const y = static_cast<T*>(H.y) + first * H.heads * P.width;
    Row<V, CHUNKS> w;
    if (P.norm) w = weights_of<INTERLEAVED, V, CHUNKS>(H.weight, p);
    Raw<T, V, CHUNKS> next;
    // (lanes without a row do the last one again and write nothing; whole waves go round together: the sum over a row's lanes needs them all)
    const auto load = [&](int r) { load_raw(next, static_cast<const T*>(H.x) + Where(H, starts, count, r < rows ? r : rows - 1).x, p); };
    load(slot);
    for (int base = 0; base < rows; base += slots) {
      const int r = base + slot;
      Row<V, CHUNKS> v = row_of<INTERLEAVED>(next);
      if (base + slots < rows) load(r + slots);
      if (P.norm) {
        const float scale = 1.f / sqrtf(row_sum(dot(v, v), shift) / (float)P.width + P.eps);
        each_value(v, w, [&](float x, float w) { return x * scale * w; });
      }
      turn_row(v, at.turns + Where(H, starts, count, r < rows ? r : rows - 1).token * P.pairs, p, P.pairs, 1.f);
      if (r < rows) store_row<INTERLEAVED>(v, y + (long long)r * P.width, p);
    }
  };
  run(P.q, at.q);
  if (P.k.heads) run(P.k, at.k);
}

// Half of the workgroups take the queries, half the keys: the sums of one weight's gradient are all that a lane keeps.  (Both in one: 153 registers, or their overflow in memory.)
template <typename T, int V, int CHUNKS, bool INTERLEAVED>
__global__ __launch_bounds__(THREADS, 4) void rotate_backward_kernel(RotateParams P, int shift, int each) {
  __shared__ Tokens at;
  __shared__ float sums[THREADS * 2 * V * CHUNKS];  // [slots][lanes][2 V]: a slot's sums
  const int lane = threadIdx.x & ((1 << shift) - 1), slot = threadIdx.x >> shift, slots = THREADS >> shift;
  Place p[CHUNKS];
#pragma unroll
  for (int c = 0; c < CHUNKS; ++c) p[c] = place_of<V, INTERLEAVED>(lane, c, 1 << shift, P.width, P.pairs);
  const RotateHeads& H = blockIdx.y ? P.k : P.q;
  const long long* starts = blockIdx.y ? at.k : at.q;
  Row<V, CHUNKS> gw = {}, w;
  if (P.norm) w = weights_of<INTERLEAVED, V, CHUNKS>(H.weight, p);
  for (long long first = (long long)blockIdx.x * each; H.heads && first < P.B * P.T; first += (long long)gridDim.x * each) {
    const int count = (int)std::min((long long)each, P.B * P.T - first), rows = count * H.heads;
    const long long packed = first * H.heads * P.width;
    __syncthreads();  // (the last tokens' angles are read)
    make_tokens(P, at, first, count);
    __syncthreads();
    for (int base = 0; base < rows; base += slots) {
      // (lanes without a row do the last one again and write nothing; whole waves go round together: the sums over a row's lanes need them all)
      const bool here = base + slot < rows;
      const int r = here ? base + slot : rows - 1;
      const Where where(H, starts, count, r);
      Raw<T, V, CHUNKS> raw_g, raw_x;
      load_raw(raw_g, static_cast<const T*>(H.g) + packed + (long long)r * P.width, p);
      if (P.norm) load_raw(raw_x, static_cast<const T*>(H.x) + where.x, p);
      Row<V, CHUNKS> g = row_of<INTERLEAVED>(raw_g);
      turn_row(g, at.turns + where.token * P.pairs, p, P.pairs, -1.f);
      if (P.norm) {
        Row<V, CHUNKS> h = row_of<INTERLEAVED>(raw_x);
        const float scale = 1.f / sqrtf(row_sum(dot(h, h), shift) / (float)P.width + P.eps);
        each_value(h, h, [&](float x, float) { return x * scale; });
        if (here)
#pragma unroll
          for (int c = 0; c < CHUNKS; ++c)
#pragma unroll
            for (int e = 0; e < V; ++e) {
              gw.a[c][e] += g.a[c][e] * h.a[c][e];
              gw.b[c][e] += g.b[c][e] * h.b[c][e];
            }
        each_value(g, w, [](float g, float w) { return g * w; });
        const float mean = row_sum(dot(g, h), shift) / (float)P.width;
        each_value(g, h, [&](float g, float h) { return scale * (g - h * mean); });
      }
      if (here) store_row<INTERLEAVED>(g, static_cast<T*>(H.y) + packed + (long long)r * P.width, p);
    }
  }
  if (!P.partial) return;
  // the slots' sums in order: one value of a head after the other, as they lie in it
  const int pitch = 2 * V * CHUNKS << shift;
  store_row<INTERLEAVED>(gw, sums + slot * pitch, p);
  __syncthreads();
  for (int d = threadIdx.x; d < P.width; d += THREADS) {
    float sum = sums[d];
    for (int i = 1; i < slots; ++i) sum += sums[i * pitch + d];
    P.partial[((long long)blockIdx.x * 2 + blockIdx.y) * P.width + d] = sum;
  }
}

// Tokens of a workgroup at a time: two rows for each of its slots, and angles for some 96 lanes, no more than the table holds.  (16 x 431 frames of 16 heads of 64, float32: four tokens 11.2 us, eight
// 12.9; 3 x 7,001 of 16 heads of 80, 40 of them rotated, float16: two tokens 28 us, four 21; 4 x 16,384 of 32 heads of 128, bfloat16: two 174 us, four 182.)
int tokens_of(int heads, int pairs, const Split& s) {
  int n = std::max(1, (2 * THREADS >> s.shift) / heads);
  if (pairs) n = std::max(n, 96 / pairs);
  n = std::min(n, std::max(1, std::min(TOKENS_MAX, 4096 / heads)));  // (what Where's quotient is good for)
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
  return (int)std::max(1LL, std::min((tokens + each - 1) / each, (long long)ROTATE_GROUPS));
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
      hipLaunchKernelGGL((rotate_backward_kernel<T, v.value, chunks.value, layout.value>), dim3(grid, P.k.heads || P.partial ? 2 : 1), dim3(THREADS), 0, stream, P, s.shift, tokens);
      return hipGetLastError();
    });
  });
  if (e != hipSuccess || !P.partial) return e;
  return launch_norm_join(P.partial, grid, P.width, gqw, gkw, stream);
}

}  // namespace nna
