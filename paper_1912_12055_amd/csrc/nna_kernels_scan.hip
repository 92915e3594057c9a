// The gated linear recurrence: whole sequences, their gradients, one frame at a time.
//
//   h_t = a_t h_{t-1} + u_t x_t,   a = sigmoid(f),   u = sigmoid(i), or 1 - a where there is no gate of the input's own;
//   e_t = g_t + a_{t+1} e_{t+1},   gx = u e,   gf = a (1 - a) e (h_{t-1} - x, or h_{t-1}),   gi = u (1 - u) e x,   gradient of the first state = a_0 e_0.
// The steps of a run of frames are one step of the same form: h = A h' + H, A the product of the a, H what the run makes of a zero state (and backwards
// c = A c' + E for c_t = a_t e_t).  So a wave takes FRAMES frames of 64 lanes' channels into registers and makes their A and H, the waves of a workgroup exchange those
// through LDS, and each walks its frames again from its own first state: every array is read or written once.
//
// A channel that remembers for thousands of frames has a within 2^-12 of one, where a float32 holds a itself to 2^-13 of its distance from one.  So 1 - a = sigmoid(-f) is
// computed too, and a is held as the nearest float32 and what that leaves: products of thousands of them are off by their own roundings alone.
#include "nna_scan.h"
#include "nna_vector.h"

namespace nna {

namespace {

constexpr int WAVES = 8, FRAMES = SCAN_KEPT / WAVES, THREADS = WAVES * 64;

// e^-|v|: the argument of the machine's 2^y rounded in two parts, since y's rounding alone is y 2^-24 of the result
__device__ __forceinline__ float exp_down(float v) {
  const float x = -__builtin_fabsf(v), y = x * 1.44269502f;
  const float rest = __builtin_fmaf(x, 1.44269502f, -y) + x * 1.92596303e-8f;
  const float e = __builtin_amdgcn_exp2f(y);
  // (x is -inf: the rest is NaN and e zero)
  return e > 0.f ? __builtin_fmaf(e * 0.693147182f, rest, e) : e;
}
// sigmoid(v) and sigmoid(-v), both to float32's own precision
struct Gate {
  float on, off;
};
__device__ __forceinline__ Gate gate(float v) {
  const float e = exp_down(v), r = __builtin_amdgcn_rcpf(1.f + e), s = e * r;
  return v >= 0.f ? Gate{r, s} : Gate{s, r};
}

// a as a float32 and what it leaves of it
struct Stay {
  float a, rest;
  __device__ __forceinline__ Stay() {}
  __device__ __forceinline__ Stay(Gate g, bool here) {
    a = here ? g.on : 1.f;
    rest = here && g.on >= 0.5f ? (1.f - g.on) - g.off : 0.f;  // (the first difference is exact there; below a half a float32 holds a to its own 2^-24)
  }
  __device__ __forceinline__ float of(float h) const { return __builtin_fmaf(a, h, rest * h); }
  __device__ __forceinline__ float of(float h, float add) const { return __builtin_fmaf(a, h, __builtin_fmaf(rest, h, add)); }
};

// One wave's frames of a round, as they lie in memory.  Frames behind `count` are read from the last one that there is; they are masked later.
template <typename T, int V>
struct Rows {
  typename Vec<T, V>::plain v[FRAMES];
  __device__ __forceinline__ void load(const T* base, long long step, int t, int T_) {
#pragma unroll
    for (int k = 0; k < FRAMES; ++k) {
      const int at = t + k < T_ ? t + k : T_ - 1;
      v[k] = vec_load<V>(base + at * step);
    }
  }
  __device__ __forceinline__ float at(int k, int c) const { return (float)vec_at<V>(v[k], c); }
};

template <int V>
__device__ __forceinline__ void zero_rows(float* v) {
#pragma unroll
  for (int c = 0; c < V; ++c) v[c] = 0.f;
}

__device__ __forceinline__ int length_of(const int* lengths, long long b, int T) {
  if (!lengths) return T;
  const int n = lengths[b];
  return n < 0 ? 0 : n < T ? n : T;
}

template <typename T, int V, bool INPUT>
__global__ __launch_bounds__(THREADS) void scan_kernel(ScanParams P) {
  __shared__ float2 sums[2][WAVES][V][64];
  const int groups = (P.C + 64 * V - 1) / (64 * V);
  const long long b = blockIdx.x / groups;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  // lanes behind the last channel do its neighbours' work again and write nothing
  const int mine = ((int)(blockIdx.x % groups) * 64 + lane) * V, channel = mine <= P.C - V ? mine : P.C - V;
  const bool live = mine < P.C;
  const int n = length_of(P.lengths, b, P.T);
  const T* x = static_cast<const T*>(P.x) + b * P.x_b + channel;
  const T* f = static_cast<const T*>(P.f) + b * P.f_b + channel;
  const T* i = INPUT ? static_cast<const T*>(P.i) + b * P.i_b + channel : nullptr;
  T* out = static_cast<T*>(P.out) + b * P.T * P.C + channel;
  float state[V];
#pragma unroll
  for (int c = 0; c < V; ++c) state[c] = P.first ? P.first[b * P.C + channel + c] : 0.f;
  const int rounds = (P.T + SCAN_KEPT - 1) / SCAN_KEPT, used = (n + SCAN_KEPT - 1) / SCAN_KEPT;
  Rows<T, V> rx, rf, ri;
  if (used) {
    rx.load(x, P.x_t, wave * FRAMES, P.T);
    rf.load(f, P.f_t, wave * FRAMES, P.T);
    if (INPUT) ri.load(i, P.i_t, wave * FRAMES, P.T);
  }
  for (int r = 0; r < used; ++r) {
    const int t = r * SCAN_KEPT + wave * FRAMES;
    float As[FRAMES][V], Hs[FRAMES][V], A[V], H[V];  // of the wave's frames up to each
#pragma unroll
    for (int c = 0; c < V; ++c) A[c] = 1.f, H[c] = 0.f;
#pragma unroll
    for (int k = 0; k < FRAMES; ++k)
#pragma unroll
      for (int c = 0; c < V; ++c) {
        const Gate a = gate(rf.at(k, c));
        const float u = INPUT ? gate(ri.at(k, c)).on : a.off;
        const Stay stay(a, t + k < n);
        As[k][c] = A[c] = stay.of(A[c]);
        Hs[k][c] = H[c] = stay.of(H[c], t + k < n ? u * rx.at(k, c) : 0.f);
      }
    if (r + 1 < used) {
      rx.load(x, P.x_t, t + SCAN_KEPT, P.T);
      rf.load(f, P.f_t, t + SCAN_KEPT, P.T);
      if (INPUT) ri.load(i, P.i_t, t + SCAN_KEPT, P.T);
    }
    // two buffers in turn: the next round's writes never meet a wave that still reads this one
#pragma unroll
    for (int c = 0; c < V; ++c) sums[r & 1][wave][c][lane] = make_float2(A[c], H[c]);
    __syncthreads();
    if (P.kept && wave == 0 && live)
#pragma unroll
      for (int c = 0; c < V; ++c) P.kept[(b * rounds + r) * P.C + channel + c] = state[c];
    float h[V];
#pragma unroll
    for (int w = 0; w < WAVES; ++w)
#pragma unroll
      for (int c = 0; c < V; ++c) {
        if (w == wave) h[c] = state[c];
        const float2 s = sums[r & 1][w][c][lane];
        state[c] = __builtin_fmaf(s.x, state[c], s.y);
      }
#pragma unroll
    for (int k = 0; k < FRAMES; ++k) {
      typename Vec<T, V>::plain o;
#pragma unroll
      for (int c = 0; c < V; ++c) {
        const float now = __builtin_fmaf(As[k][c], h[c], Hs[k][c]);
        vec_set<V>(o, c, (T)(t + k < n ? now : 0.f));
      }
      if (t + k < P.T && live) vec_store<V>(out + (long long)(t + k) * P.C, o);
    }
  }
  if (live) {
    if (P.last && wave == 0)
#pragma unroll
      for (int c = 0; c < V; ++c) P.last[b * P.C + channel + c] = state[c];
    typename Vec<T, V>::plain zero;
#pragma unroll
    for (int c = 0; c < V; ++c) vec_set<V>(zero, c, (T)0.f);
    for (int t = used * SCAN_KEPT + wave; t < P.T; t += WAVES) vec_store<V>(out + (long long)t * P.C, zero);
  }
}

template <typename T, int V, bool INPUT>
__global__ __launch_bounds__(THREADS) void scan_backward_kernel(ScanParams P) {
  __shared__ float sums[2][WAVES][3][V][64];
  const int groups = (P.C + 64 * V - 1) / (64 * V);
  const long long b = blockIdx.x / groups;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int mine = ((int)(blockIdx.x % groups) * 64 + lane) * V, channel = mine <= P.C - V ? mine : P.C - V;
  const bool live = mine < P.C;
  const int n = length_of(P.lengths, b, P.T);
  const T* x = static_cast<const T*>(P.x) + b * P.x_b + channel;
  const T* f = static_cast<const T*>(P.f) + b * P.f_b + channel;
  const T* i = INPUT ? static_cast<const T*>(P.i) + b * P.i_b + channel : nullptr;
  const long long packed = b * P.T * P.C + channel;
  const T* g = static_cast<const T*>(P.g) + packed;
  T *gx = static_cast<T*>(P.gx) + packed, *gf = static_cast<T*>(P.gf) + packed, *gi = INPUT ? static_cast<T*>(P.gi) + packed : nullptr;
  float carry[V];  // a e of the frame behind
#pragma unroll
  for (int c = 0; c < V; ++c) carry[c] = P.glast ? P.glast[b * P.C + channel + c] : 0.f;
  const int rounds = (P.T + SCAN_KEPT - 1) / SCAN_KEPT, used = (n + SCAN_KEPT - 1) / SCAN_KEPT;
  if (live) {
    typename Vec<T, V>::plain zero;
#pragma unroll
    for (int c = 0; c < V; ++c) vec_set<V>(zero, c, (T)0.f);
    for (int t = used * SCAN_KEPT + wave; t < P.T; t += WAVES) {
      vec_store<V>(gx + (long long)t * P.C, zero);
      vec_store<V>(gf + (long long)t * P.C, zero);
      if (INPUT) vec_store<V>(gi + (long long)t * P.C, zero);
    }
  }
  Rows<T, V> rx, rf, ri, rg;
  if (used) {
    const int t = (used - 1) * SCAN_KEPT + wave * FRAMES;
    rx.load(x, P.x_t, t, P.T);
    rf.load(f, P.f_t, t, P.T);
    if (INPUT) ri.load(i, P.i_t, t, P.T);
    rg.load(g, P.C, t, P.T);
  }
  for (int r = used - 1; r >= 0; --r) {
    const int t = r * SCAN_KEPT + wave * FRAMES;
    Stay stay[FRAMES][V];
    float slope[FRAMES][V], take[FRAMES][V], take_slope[FRAMES][V], in[FRAMES][V], go[FRAMES][V];
    float A[V], H[V], E[V], h[V];
#pragma unroll
    for (int c = 0; c < V; ++c) {
      A[c] = 1.f, H[c] = 0.f, E[c] = 0.f;
      h[c] = P.kept[(b * rounds + r) * P.C + channel + c];
    }
#pragma unroll
    for (int k = 0; k < FRAMES; ++k)
#pragma unroll
      for (int c = 0; c < V; ++c) {
        const bool here = t + k < n;
        const Gate a = gate(rf.at(k, c));
        stay[k][c] = Stay(a, here);
        slope[k][c] = here ? a.on * a.off : 0.f;
        in[k][c] = here ? rx.at(k, c) : 0.f;
        go[k][c] = here ? rg.at(k, c) : 0.f;
        if (INPUT) {
          const Gate u = gate(ri.at(k, c));
          take[k][c] = here ? u.on : 0.f;
          take_slope[k][c] = here ? u.on * u.off : 0.f;
        } else {
          take[k][c] = here ? a.off : 0.f;
        }
        A[c] = stay[k][c].of(A[c]);
        H[c] = stay[k][c].of(H[c], take[k][c] * in[k][c]);
      }
#pragma unroll
    for (int k = FRAMES - 1; k >= 0; --k)
#pragma unroll
      for (int c = 0; c < V; ++c) {
        E[c] = stay[k][c].of(E[c] + go[k][c]);
      }
    if (r) {
      rx.load(x, P.x_t, t - SCAN_KEPT, P.T);
      rf.load(f, P.f_t, t - SCAN_KEPT, P.T);
      if (INPUT) ri.load(i, P.i_t, t - SCAN_KEPT, P.T);
      rg.load(g, P.C, t - SCAN_KEPT, P.T);
    }
#pragma unroll
    for (int c = 0; c < V; ++c) {
      sums[r & 1][wave][0][c][lane] = A[c];
      sums[r & 1][wave][1][c][lane] = H[c];
      sums[r & 1][wave][2][c][lane] = E[c];
    }
    __syncthreads();
    float e[V];
#pragma unroll
    for (int w = 0; w < WAVES; ++w)
      if (w < wave)
#pragma unroll
        for (int c = 0; c < V; ++c) h[c] = __builtin_fmaf(sums[r & 1][w][0][c][lane], h[c], sums[r & 1][w][1][c][lane]);
#pragma unroll
    for (int w = WAVES - 1; w >= 0; --w)
#pragma unroll
      for (int c = 0; c < V; ++c) {
        if (w == wave) e[c] = carry[c];
        carry[c] = __builtin_fmaf(sums[r & 1][w][0][c][lane], carry[c], sums[r & 1][w][2][c][lane]);
      }
    float before[FRAMES][V];
#pragma unroll
    for (int k = 0; k < FRAMES; ++k)
#pragma unroll
      for (int c = 0; c < V; ++c) {
        before[k][c] = h[c];
        h[c] = stay[k][c].of(h[c], take[k][c] * in[k][c]);
      }
#pragma unroll
    for (int k = FRAMES - 1; k >= 0; --k) {
      typename Vec<T, V>::plain ox, of, oi;
#pragma unroll
      for (int c = 0; c < V; ++c) {
        e[c] += go[k][c];
        const bool here = t + k < n;
        vec_set<V>(ox, c, (T)(here ? take[k][c] * e[c] : 0.f));
        vec_set<V>(of, c, (T)(here ? slope[k][c] * e[c] * (INPUT ? before[k][c] : before[k][c] - in[k][c]) : 0.f));
        if (INPUT) vec_set<V>(oi, c, (T)(here ? take_slope[k][c] * e[c] * in[k][c] : 0.f));
        e[c] = stay[k][c].of(e[c]);
      }
      if (t + k < P.T && live) {
        const long long at = (long long)(t + k) * P.C;
        vec_store<V>(gx + at, ox);
        vec_store<V>(gf + at, of);
        if (INPUT) vec_store<V>(gi + at, oi);
      }
    }
  }
  if (P.gfirst && live && wave == 0)
#pragma unroll
    for (int c = 0; c < V; ++c) P.gfirst[b * P.C + channel + c] = carry[c];
}

// One frame: bound by the states' bytes where there are many streams, by the launch where there are few.
constexpr int STEP = 4;  // channels of a lane
template <typename T, bool INPUT>
__global__ __launch_bounds__(256) void scan_step_kernel(ScanStep P) {
  const int quads = (P.C + STEP - 1) / STEP;
  const long long all = P.B * quads;
  for (long long at = (long long)blockIdx.x * 256 + threadIdx.x; at < all; at += (long long)gridDim.x * 256) {
    const long long b = at / quads;
    const int channel = (int)(at - b * quads) * STEP;
    const T* x = static_cast<const T*>(P.x) + b * P.x_b + channel;
    const T* f = static_cast<const T*>(P.f) + b * P.f_b + channel;
    const T* i = INPUT ? static_cast<const T*>(P.i) + b * P.i_b + channel : nullptr;
    float* state = P.state + b * P.C + channel;
    T* out = static_cast<T*>(P.out) + b * P.C + channel;
    const auto next = [](float h, float x, float f, float i) {
      const Gate a = gate(f);
      return Stay(a, true).of(h, (INPUT ? gate(i).on : a.off) * x);
    };
    if (channel + STEP <= P.C) {
      const auto vx = vec_load<STEP>(x), vf = vec_load<STEP>(f), vi = INPUT ? vec_load<STEP>(i) : vf;
      auto h = vec_load<STEP>(state);
      typename Vec<T, STEP>::plain o;
#pragma unroll
      for (int c = 0; c < STEP; ++c) {
        h[c] = next(h[c], (float)vx[c], (float)vf[c], (float)vi[c]);
        o[c] = (T)h[c];
      }
      vec_store<STEP>(state, h);
      vec_store<STEP>(out, o);
    } else {
      for (int c = 0; c < P.C - channel; ++c) {
        const float h = next(state[c], (float)x[c], (float)f[c], INPUT ? (float)i[c] : 0.f);
        state[c] = h;
        out[c] = (T)h;
      }
    }
  }
}

// channels of a lane: four bytes of them, where there are as many
template <typename T, typename F>
hipError_t by_lane(int C, F fn) {
  if constexpr (sizeof(T) == 2)
    if (C > 1) return fn(std::integral_constant<int, 2>());
  return fn(std::integral_constant<int, 1>());
}

}  // namespace

size_t scan_workspace(long long, long long, long long) { return 0; }

hipError_t launch_scan(const ScanParams& P, int type, hipStream_t stream) {
  return by_element(type, [&](auto t) {
    typedef decltype(t) T;
    return by_lane<T>(P.C, [&](auto v) {
      constexpr int V = v.value;
      const unsigned grid = (unsigned)(P.B * ((P.C + 64 * V - 1) / (64 * V)));
      if (P.i)
        hipLaunchKernelGGL((scan_kernel<T, V, true>), dim3(grid), dim3(THREADS), 0, stream, P);
      else
        hipLaunchKernelGGL((scan_kernel<T, V, false>), dim3(grid), dim3(THREADS), 0, stream, P);
      return hipGetLastError();
    });
  });
}

hipError_t launch_scan_backward(const ScanParams& P, int type, hipStream_t stream) {
  return by_element(type, [&](auto t) {
    typedef decltype(t) T;
    return by_lane<T>(P.C, [&](auto v) {
      constexpr int V = v.value;
      const unsigned grid = (unsigned)(P.B * ((P.C + 64 * V - 1) / (64 * V)));
      if (P.i)
        hipLaunchKernelGGL((scan_backward_kernel<T, V, true>), dim3(grid), dim3(THREADS), 0, stream, P);
      else
        hipLaunchKernelGGL((scan_backward_kernel<T, V, false>), dim3(grid), dim3(THREADS), 0, stream, P);
      return hipGetLastError();
    });
  });
}

hipError_t launch_scan_step(const ScanStep& P, int type, hipStream_t stream) {
  return by_element(type, [&](auto t) {
    typedef decltype(t) T;
    const long long all = P.B * ((P.C + STEP - 1) / STEP);
    const unsigned grid = (unsigned)std::min((all + 255) / 256, 8192LL);
    if (P.i)
      hipLaunchKernelGGL((scan_step_kernel<T, true>), dim3(grid), dim3(256), 0, stream, P);
    else
      hipLaunchKernelGGL((scan_step_kernel<T, false>), dim3(grid), dim3(256), 0, stream, P);
    return hipGetLastError();
  });
}

}  // namespace nna
