// The gated linear recurrence: whole sequences, their gradients, one frame at a time.
//
//   h_t = a_t h_{t-1} + u_t x_t,   a = sigmoid(f),   u = sigmoid(i), or 1 - a where there is no gate of the input's own;
//   e_t = g_t + a_{t+1} e_{t+1},   gx = u e,   gf = a (1 - a) e (h_{t-1} - x, or h_{t-1}),   gi = u (1 - u) e x,   gradient of the first state = a_0 e_0.
// The steps of a run of frames are one step of the same form: h = A h' + H, A the product of the a, H what the run makes of a zero state (and backwards
// c = A c' + E for c_t = a_t e_t).  So a wave takes FRAMES frames of 64 lanes' channels into registers and makes their A and H, the waves of a workgroup exchange those
// through LDS, and each walks its frames again from its own first state: every array is read or written once.
//
// A channel that remembers for thousands of frames has a within 2^-12 of one, where a float32 holds a to 2^-13 of its distance from one; and where its gate is steady every frame's, every run's
// and every segment's product is rounded the same way: over 16,384 frames what is left of a first state would be off by 5 10^-4 (runs' products as one float32 each), and by 10^-4 at the median.
// So 1 - a = sigmoid(-f) is computed too, and of what is passed on, a run's A, also Q = 1 - A: Q <- Q + q (1 - Q) with q = 1 - a, and the state goes through A as the nearest float32 and what that
// leaves: 5 10^-6, and 4 10^-7 at the median.  Inside of a run, whose products end there, a and A are one float32.
#include "nna_scan.h"
#include "nna_vector.h"

namespace nna {

namespace {

// sigmoid(v) and sigmoid(-v), each to float32's own precision of itself.  Of a float32 v the argument of the machine's 2^y is made in two parts, since y's rounding alone is y 2^-24 of the
// result; a 16-bit v is itself off by far more.  (minimum and maximum let a NaN through.)
struct Gate {
  float on, off;
  __device__ __forceinline__ Gate where(bool here) const { return {here ? on : 1.f, here ? off : 0.f}; }  // a frame that takes no part leaves the state as it is
};
template <typename T>
__device__ __forceinline__ float exp_of_minus(T v) {
  float e;
  if constexpr (sizeof(T) == 4) {
    const float x = __builtin_elementwise_maximum(__builtin_elementwise_minimum(-v, 87.f), -104.f), y = x * 1.44269502f;
    const float rest = __builtin_fmaf(x, 1.92596303e-8f, __builtin_fmaf(x, 1.44269502f, -y));
    e = __builtin_amdgcn_exp2f(y);
    e = __builtin_fmaf(e * 0.693147182f, rest, e);
  } else {
    e = __builtin_amdgcn_exp2f(__builtin_elementwise_minimum((float)v * -1.44269502f, 126.f));
  }
  return e;
}
template <typename T>
__device__ __forceinline__ Gate gate(T v) {
  const float e = exp_of_minus(v), r = __builtin_amdgcn_rcpf(1.f + e);
  return {r, e * r};
}

// A product A of gates and 1 - A, each to float32's own precision of itself, the second without the first's roundings: Q + q (1 - Q)
struct Product {
  float a = 1.f, q = 0.f;
  __device__ __forceinline__ void by(float on, float off) {
    q += __builtin_fmaf(-off, q, off);
    a *= on;
  }
  // what the float32 a leaves of A (the first difference is exact from a half on, and below it A is held to its own 2^-24): of a as it was rounded, so no product is fused into it
  __device__ __forceinline__ float rest() const {
#pragma clang fp contract(off)
    return a >= 0.5f ? (1.f - a) - q : 0.f;
  }
  __device__ __forceinline__ static Product of(float a, float rest) {
    Product p;
    p.a = a;
    p.q = (1.f - a) - rest;
    return p;
  }
  // the one of the two that is below a half as one number: A, or -(1 - A), with its sign set also where it is zero
  __device__ __forceinline__ float code() const { return a >= 0.5f ? -q : a; }
  __device__ __forceinline__ static Product of_code(float code) {
    Product p;
    p.a = __builtin_signbit(code) ? 1.f + code : code;
    p.q = __builtin_signbit(code) ? -code : 1.f - code;
    return p;
  }
};
// A h + add
__device__ __forceinline__ float through(float a, float rest, float h, float add) { return __builtin_fmaf(a, h, __builtin_fmaf(rest, h, add)); }

// A workgroup's lanes: CL neighbours along the channels, V channels each, 64 / CL runs of FRAMES frames in a wave, WAVES waves behind one another.
template <int CL, int FRAMES, int WAVES>
struct Shape {
  static constexpr int RUNS = 64 / CL, WAVE = RUNS * FRAMES, ROUND = WAVES * WAVE;  // runs of a wave; frames of a wave, of a round
  static constexpr int KEPT_WAVES = SCAN_KEPT / WAVE;                               // waves from one kept state to the next
};

// A lane's frames of a round, as they lie in memory
template <typename T, int V, int FRAMES>
struct Rows {
  typename Vec<T, V>::plain v[FRAMES];
  // frames from t on; those behind the last one that there is are read from it, and masked later
  template <bool FULL>
  __device__ __forceinline__ void load(const T* base, long long step, int t, int last) {
    const T* p = base + (FULL ? t : 0) * step;
#pragma unroll
    for (int k = 0; k < FRAMES; ++k) v[k] = vec_load<V>(FULL ? p + k * step : base + (t + k < last ? t + k : last) * step);
  }
  __device__ __forceinline__ T at(int k, int c) const { return vec_at<V>(v[k], c); }
};

// A run's A and H alone, for segments' ends.  With d = 1 / a = 1 + e^-f and D = 1 + M the product of the d so far the sums have no quotient in their recurrences,
//   M_t = M_{t-1} + e^-f D_{t-1},   G_t = G_{t-1} + u x D_t  (u = 1 - a: + e^-f x D_{t-1}),   A = 1 / D,   1 - A = M / D,   H = G / D   (backwards E = sum of g_t / D_t):
// 14 instructions a value in place of 30.  Where D or G comes near float32's largest value (gates that all but forget frame after frame, and what is not
// finite) the run is walked by a and 1 - a.
constexpr float ENDS_MOST = 0x1p124f;
template <bool INPUT, typename T, int V, int FRAMES>
__device__ __forceinline__ void run_ends(const Rows<T, V, FRAMES>& rx, const Rows<T, V, FRAMES>& rf, const Rows<T, V, FRAMES>& ri, int here /* frames taken */, Product (&A)[V], float (&H)[V]) {
#pragma unroll
  for (int c = 0; c < V; ++c) {
    float D = 1.f, M = 0.f, G = 0.f;
#pragma unroll
    for (int k = 0; k < FRAMES; ++k) {
      const float e = k < here ? exp_of_minus(rf.at(k, c)) : 0.f;
      if (INPUT) {
        M = __builtin_fmaf(e, D, M);
        D = 1.f + M;
        G = __builtin_fmaf(k < here ? gate(ri.at(k, c)).on * (float)rx.at(k, c) : 0.f, D, G);
      } else {
        G = __builtin_fmaf(k < here ? e * (float)rx.at(k, c) : 0.f, D, G);
        M = __builtin_fmaf(e, D, M);
        D = 1.f + M;
      }
    }
    A[c].a = __builtin_amdgcn_rcpf(D);
    A[c].q = M * A[c].a;
    H[c] = G * A[c].a;
    if (__builtin_expect(!(D + __builtin_fabsf(G) < ENDS_MOST), 0)) {
      A[c] = Product(), H[c] = 0.f;
#pragma unroll
      for (int k = 0; k < FRAMES; ++k) {
        const Gate a = gate(rf.at(k, c)).where(k < here);
        A[c].by(a.on, a.off);
        H[c] = __builtin_fmaf(a.on, H[c], k < here ? (INPUT ? gate(ri.at(k, c)).on : a.off) * (float)rx.at(k, c) : 0.f);
      }
    }
  }
}
template <typename T, int V, int FRAMES>
__device__ __forceinline__ void run_ends_back(const Rows<T, V, FRAMES>& rf, const Rows<T, V, FRAMES>& rg, int here, Product (&A)[V], float (&E)[V]) {
#pragma unroll
  for (int c = 0; c < V; ++c) {
    float D = 1.f, M = 0.f;
    E[c] = 0.f;
#pragma unroll
    for (int k = 0; k < FRAMES; ++k) {
      const float e = k < here ? exp_of_minus(rf.at(k, c)) : 0.f;
      M = __builtin_fmaf(e, D, M);
      D = 1.f + M;
      A[c].a = __builtin_amdgcn_rcpf(D);
      E[c] = __builtin_fmaf(k < here ? (float)rg.at(k, c) : 0.f, A[c].a, E[c]);
    }
    A[c].q = M * A[c].a;
    if (__builtin_expect(!(D < ENDS_MOST), 0)) {
      A[c] = Product(), E[c] = 0.f;
#pragma unroll
      for (int k = FRAMES - 1; k >= 0; --k) {
        const Gate a = gate(rf.at(k, c)).where(k < here);
        A[c].by(a.on, a.off);
        E[c] = a.on * (E[c] + (k < here ? (float)rg.at(k, c) : 0.f));
      }
    }
  }
}

__device__ __forceinline__ int length_of(const int* lengths, long long b, int T) {
  if (!lengths) return T;
  const int n = lengths[b];
  return n < 0 ? 0 : n < T ? n : T;
}

// Which part of the work is a workgroup's.  Neighbouring channels' groups follow one another on one die (workgroups go round the eight of them), whose cache then serves both
// halves of a line.
struct Part {
  long long b;
  int segment, channel;
  bool live;
};
template <int CL, int V>
__device__ __forceinline__ Part part_of(const ScanParams& P) {
  const int groups = (P.C + CL * V - 1) / (CL * V);
  const unsigned all = gridDim.x, each = all / 8, id = blockIdx.x < each * 8 ? (blockIdx.x % 8) * each + blockIdx.x / 8 : blockIdx.x;
  Part p;
  const unsigned group = id % groups, rest = id / groups;
  p.segment = (int)(rest % P.segments);
  p.b = rest / P.segments;
  // lanes behind the last channel do its neighbours' work again and write nothing
  const int mine = ((int)group * CL + (int)(threadIdx.x % CL)) * V;
  p.channel = mine <= P.C - V ? mine : P.C - V;
  p.live = mine < P.C;
  return p;
}

// A value of the lower and of the upper of two neighbouring runs, in all lanes of both: rows of 16 lanes, halves of the wave.
struct Two {
  float low, high;
};
__device__ __forceinline__ Two rows_of(float v) {
  const auto p = __builtin_amdgcn_permlane16_swap(__builtin_bit_cast(unsigned, v), __builtin_bit_cast(unsigned, v), false, false);
  const unsigned a = p[0], b = p[1];
  return {__builtin_bit_cast(float, a), __builtin_bit_cast(float, b)};
}
__device__ __forceinline__ Two halves_of(float v) {
  const auto p = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(unsigned, v), __builtin_bit_cast(unsigned, v), false, false);
  const unsigned a = p[0], b = p[1];
  return {__builtin_bit_cast(float, a), __builtin_bit_cast(float, b)};
}
// A run makes h = a h' + h of the state before it, and c = a c' + e of the carry behind it.  In a wave: what the runs before this lane's make together (before_a, before_h), those behind
// it (behind_a, behind_e), and all of them (all).
template <int CL>
struct Joined {
  float before_a, before_h, behind_a, behind_e, all_h, all_e;
  Product all;
  template <bool FORWARD, bool BACKWARD>
  __device__ __forceinline__ void join(Product a, float h, float e) {
    before_a = behind_a = 1.f;
    before_h = behind_e = 0.f;
    all = a, all_h = h, all_e = e;
    if constexpr (CL <= 16) step<FORWARD, BACKWARD>(threadIdx.x & 16, rows_of);
    if constexpr (CL <= 32) step<FORWARD, BACKWARD>(threadIdx.x & 32, halves_of);
  }
  template <bool FORWARD, bool BACKWARD, typename F>
  __device__ __forceinline__ void step(bool upper, F two) {
    const Two A = two(all.a), Q = two(all.q);
    if (FORWARD) {
      const Two H = two(all_h);
      before_h = upper ? __builtin_fmaf(before_a, H.low, before_h) : before_h;
      before_a = upper ? before_a * A.low : before_a;
      all_h = __builtin_fmaf(A.high, H.low, H.high);
    }
    if (BACKWARD) {
      const Two E = two(all_e);
      behind_e = upper ? behind_e : __builtin_fmaf(behind_a, E.high, behind_e);
      behind_a = upper ? behind_a : behind_a * A.high;
      all_e = __builtin_fmaf(A.low, E.high, E.low);
    }
    all.q = Q.low + __builtin_fmaf(-Q.high, Q.low, Q.high);
    all.a = A.low * A.high;
  }
};

// What the waves of a workgroup tell each other, a column's side by side: two buffers in turn, so that the next round's writes never meet a wave that still reads this one.
typedef float Quad __attribute__((ext_vector_type(4)));
template <int V, int CL, int WAVES>
struct alignas(16) Told {
  float at[2][V][CL][WAVES];
  __device__ __forceinline__ Quad four(int turn, int c, int column, int w) const { return *reinterpret_cast<const Quad*>(&at[turn][c][column][w]); }
  __device__ __forceinline__ void get(int turn, int c, int column, float (&to)[WAVES]) const {
#pragma unroll
    for (int w = 0; w < WAVES; w += 4) {
      const Quad q = four(turn, c, column, w);
#pragma unroll
      for (int k = 0; k < 4; ++k) to[w + k] = q[k];
    }
  }
};

// Forward.  ENDS: no outputs, but what each segment makes of the state before it, P.parts[b][segment][A (coded), h][C]; the mix composes those of the segments before its own.
// The next round's loads are asked for when this one's values have been used, half a round ahead.  16 x 4,096 frames of 2,048 channels, bfloat16: 171 us, 4.7 TB/s of the 5.1 that a copy
// reaches; 4 x 16,384 (rows of half lines): 195 us.  With D and G of run_ends here, too, it takes a third of the instructions less, 143 registers, and is no faster.
template <typename T, int V, int CL, int FRAMES, int WAVES, bool INPUT, bool ENDS>
__global__ __launch_bounds__(WAVES * 64) void scan_kernel(ScanParams P) {
  typedef Shape<CL, FRAMES, WAVES> S;
  __shared__ Told<V, CL, WAVES> told_a, told_rest, told_h;
  const Part part = part_of<CL, V>(P);
  const long long b = part.b;
  const int channel = part.channel, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), column = threadIdx.x % CL, run = (threadIdx.x & 63) / CL;
  if (ENDS && part.segment == P.segments - 1) return;  // (there is none behind the last)
  const int n = length_of(P.lengths, b, P.T);
  const T* x = static_cast<const T*>(P.x) + b * P.x_b + channel;
  const T* f = static_cast<const T*>(P.f) + b * P.f_b + channel;
  const T* i = INPUT ? static_cast<const T*>(P.i) + b * P.i_b + channel : nullptr;
  T* out = static_cast<T*>(P.out) + b * P.T * P.C + channel;
  const int begin = part.segment * P.segment_frames, end = begin + P.segment_frames < P.T ? begin + P.segment_frames : P.T;
  const int used = n < end ? n : end;  // frames up to here are taken
  const int kept_rows = (P.T + SCAN_KEPT - 1) / SCAN_KEPT;
  float state[V];
  Product factor[V];
#pragma unroll
  for (int c = 0; c < V; ++c) state[c] = !ENDS && P.first ? P.first[b * P.C + channel + c] : 0.f;
  if (!ENDS && part.segment) {
    // the segments before this one, shared out among the runs
    const int each = (part.segment + S::RUNS * WAVES - 1) / (S::RUNS * WAVES), from = (wave * S::RUNS + run) * each, to = from + each < part.segment ? from + each : part.segment;
    Product A[V];
    float H[V];
#pragma unroll
    for (int c = 0; c < V; ++c) H[c] = 0.f;
    for (int s = from; s < to; ++s) {
      const float* p = P.parts + (b * P.segments + s) * 2 * P.C + channel;
#pragma unroll
      for (int c = 0; c < V; ++c) {
        const Product of = Product::of_code(p[c]);
        H[c] = through(of.a, of.rest(), H[c], p[P.C + c]);
        A[c].by(of.a, of.q);
      }
    }
#pragma unroll
    for (int c = 0; c < V; ++c) {
      Joined<CL> joined;
      joined.template join<true, false>(A[c], H[c], 0.f);
      if (run == 0) {
        told_a.at[1][c][column][wave] = joined.all.a;
        told_rest.at[1][c][column][wave] = joined.all.rest();
        told_h.at[1][c][column][wave] = joined.all_h;
      }
    }
    __syncthreads();
#pragma unroll
    for (int c = 0; c < V; ++c) {
      float as[WAVES], rests[WAVES], hs[WAVES];
      told_a.get(1, c, column, as);
      told_rest.get(1, c, column, rests);
      told_h.get(1, c, column, hs);
#pragma unroll
      for (int w = 0; w < WAVES; ++w) state[c] = through(as[w], rests[w], state[c], hs[w]);
    }
  }
  Rows<T, V, FRAMES> rx, rf, ri;
  const auto load = [&](int t) {
    if (t + S::ROUND <= P.T) {
      const int at = t + wave * S::WAVE + run * FRAMES;
      rx.template load<true>(x, P.x_t, at, 0);
      rf.template load<true>(f, P.f_t, at, 0);
      if (INPUT) ri.template load<true>(i, P.i_t, at, 0);
    } else {
      const int at = t + wave * S::WAVE + run * FRAMES;
      rx.template load<false>(x, P.x_t, at, P.T - 1);
      rf.template load<false>(f, P.f_t, at, P.T - 1);
      if (INPUT) ri.template load<false>(i, P.i_t, at, P.T - 1);
    }
  };
  const auto round = [&](int first, int turn, auto full) {
    constexpr bool FULL = full.value;  // all frames of the round are taken
    const int t = first + wave * S::WAVE + run * FRAMES;
    float As[FRAMES][V], Hs[FRAMES][V], H[V];  // of the run's frames up to each
    Product A[V];
#pragma unroll
    for (int c = 0; c < V; ++c) H[c] = 0.f;
    if (ENDS) run_ends<INPUT>(rx, rf, ri, FULL ? FRAMES : used - t, A, H);
#pragma unroll
    for (int k = 0; k < (ENDS ? 0 : FRAMES); ++k)
#pragma unroll
      for (int c = 0; c < V; ++c) {
        const bool here = FULL || t + k < used;
        const Gate a = gate(rf.at(k, c)).where(here);
        const float u = INPUT ? gate(ri.at(k, c)).on : a.off;
        A[c].by(a.on, a.off);
        H[c] = __builtin_fmaf(a.on, H[c], here ? u * (float)rx.at(k, c) : 0.f);
        As[k][c] = A[c].a, Hs[k][c] = H[c];
      }
    if (first + S::ROUND < used) load(first + S::ROUND);
    Joined<CL> joined[V];
#pragma unroll
    for (int c = 0; c < V; ++c) {
      joined[c].template join<true, false>(A[c], H[c], 0.f);
      if (run == 0) {
        told_a.at[turn][c][column][wave] = joined[c].all.a;
        told_rest.at[turn][c][column][wave] = joined[c].all.rest();
        told_h.at[turn][c][column][wave] = joined[c].all_h;
      }
    }
    __syncthreads();
    if (ENDS && wave) return;  // (the first wave's state is the segment's)
    float h[V];
#pragma unroll
    for (int c = 0; c < V; ++c) {
      h[c] = state[c];
#pragma unroll
      for (int w = 0; w < WAVES; w += 4) {
        const Quad as = told_a.four(turn, c, column, w), rests = told_rest.four(turn, c, column, w), hs = told_h.four(turn, c, column, w);
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          state[c] = through(as[k], rests[k], state[c], hs[k]);
          if (ENDS) factor[c].by(as[k], Product::of(as[k], rests[k]).q);
          if (w + k + 1 == wave) h[c] = state[c];
        }
        if (INPUT && !ENDS) __builtin_amdgcn_sched_barrier(0);  // (the next four asked for now would take the registers that a second workgroup has its place by: 132 of 128)
      }
      h[c] = __builtin_fmaf(joined[c].before_a, h[c], joined[c].before_h);
    }
    if (ENDS) return;
    if (P.kept && t % SCAN_KEPT == 0 && t < used && part.live)
#pragma unroll
      for (int c = 0; c < V; ++c) P.kept[(b * kept_rows + t / SCAN_KEPT) * P.C + channel + c] = h[c];
#pragma unroll
    for (int k = 0; k < FRAMES; ++k) {
      typename Vec<T, V>::plain o;
#pragma unroll
      for (int c = 0; c < V; ++c) {
        const float now = __builtin_fmaf(As[k][c], h[c], Hs[k][c]);
        vec_set<V>(o, c, (T)(FULL || t + k < used ? now : 0.f));
      }
      if ((FULL || t + k < end) && part.live) vec_store<V>(out + (long long)(t + k) * P.C, o);
    }
  };
  if (begin < used) load(begin);
  int turn = 0, t = begin;
  for (; t < used; t += S::ROUND, turn ^= 1) {
    if (t + S::ROUND <= used)
      round(t, turn, std::true_type());
    else
      round(t, turn, std::false_type());
  }
  if (!part.live) return;
  if (ENDS) {
    if (threadIdx.x >= CL) return;
    float* p = P.parts + (b * P.segments + part.segment) * 2 * P.C + channel;
#pragma unroll
    for (int c = 0; c < V; ++c) p[c] = factor[c].code(), p[P.C + c] = state[c];
    return;
  }
  if (P.last && part.segment == P.segments - 1 && threadIdx.x < CL)
#pragma unroll
    for (int c = 0; c < V; ++c) P.last[b * P.C + channel + c] = state[c];
  typename Vec<T, V>::plain zero;
#pragma unroll
  for (int c = 0; c < V; ++c) vec_set<V>(zero, c, (T)0.f);
  for (t += threadIdx.x / CL; t < end; t += WAVES * 64 / CL) vec_store<V>(out + (long long)t * P.C, zero);
}

// Backward, from the last frame to the first; the states inside a round are made again from the kept one.  ENDS: what each segment makes of the carry behind it, P.parts[b][segment][A (coded), e][C].
// 16 x 4,096 frames of 2,048 channels, bfloat16: 300 us, 4.5 TB/s; 4 x 16,384: 361 us.  Rounds of eight frames a lane need 230 registers and more, half as many 156.
template <typename T, int V, int CL, int FRAMES, int WAVES, bool INPUT, bool ENDS>
__global__ __launch_bounds__(WAVES * 64) void scan_backward_kernel(ScanParams P) {
  typedef Shape<CL, FRAMES, WAVES> S;
  __shared__ Told<V, CL, WAVES> told_a, told_rest, told_h, told_e;
  const Part part = part_of<CL, V>(P);
  const long long b = part.b;
  const int channel = part.channel, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), column = threadIdx.x % CL, run = (threadIdx.x & 63) / CL;
  if (ENDS && part.segment == 0) return;  // (there is none before the first)
  const int n = length_of(P.lengths, b, P.T);
  const T* x = static_cast<const T*>(P.x) + b * P.x_b + channel;
  const T* f = static_cast<const T*>(P.f) + b * P.f_b + channel;
  const T* i = INPUT ? static_cast<const T*>(P.i) + b * P.i_b + channel : nullptr;
  const long long packed = b * P.T * P.C + channel;
  const T* g = static_cast<const T*>(P.g) + packed;
  T *gx = static_cast<T*>(P.gx) + packed, *gf = static_cast<T*>(P.gf) + packed, *gi = INPUT ? static_cast<T*>(P.gi) + packed : nullptr;
  const int begin = part.segment * P.segment_frames, end = begin + P.segment_frames < P.T ? begin + P.segment_frames : P.T;
  const int used = n < end ? n : end;
  const int kept_rows = (P.T + SCAN_KEPT - 1) / SCAN_KEPT;
  float carry[V];  // a e of the frame behind
  Product factor[V];
#pragma unroll
  for (int c = 0; c < V; ++c) carry[c] = !ENDS && P.glast ? P.glast[b * P.C + channel + c] : 0.f;
  const int behind = P.segments - 1 - part.segment;
  if (!ENDS && behind) {
    // the segments behind this one, shared out among the runs
    const int each = (behind + S::RUNS * WAVES - 1) / (S::RUNS * WAVES), from = part.segment + 1 + (wave * S::RUNS + run) * each;
    const int to = from + each < P.segments ? from + each : P.segments;
    Product A[V];
    float E[V];
#pragma unroll
    for (int c = 0; c < V; ++c) E[c] = 0.f;
    for (int s = to - 1; s >= from; --s) {
      const float* p = P.parts + (b * P.segments + s) * 2 * P.C + channel;
#pragma unroll
      for (int c = 0; c < V; ++c) {
        const Product of = Product::of_code(p[c]);
        E[c] = through(of.a, of.rest(), E[c], p[P.C + c]);
        A[c].by(of.a, of.q);
      }
    }
#pragma unroll
    for (int c = 0; c < V; ++c) {
      Joined<CL> joined;
      joined.template join<false, true>(A[c], 0.f, E[c]);
      if (run == 0) {
        told_a.at[1][c][column][wave] = joined.all.a;
        told_rest.at[1][c][column][wave] = joined.all.rest();
        told_e.at[1][c][column][wave] = joined.all_e;
      }
    }
    __syncthreads();
#pragma unroll
    for (int c = 0; c < V; ++c) {
      float as[WAVES], rests[WAVES], es[WAVES];
      told_a.get(1, c, column, as);
      told_rest.get(1, c, column, rests);
      told_e.get(1, c, column, es);
#pragma unroll
      for (int w = WAVES - 1; w >= 0; --w) carry[c] = through(as[w], rests[w], carry[c], es[w]);
    }
  }
  const int rounds = used > begin ? (used - begin + S::ROUND - 1) / S::ROUND : 0;
  if (!ENDS && part.live) {
    typename Vec<T, V>::plain zero;
#pragma unroll
    for (int c = 0; c < V; ++c) vec_set<V>(zero, c, (T)0.f);
    for (int t = begin + rounds * S::ROUND + threadIdx.x / CL; t < end; t += WAVES * 64 / CL) {
      vec_store<V>(gx + (long long)t * P.C, zero);
      vec_store<V>(gf + (long long)t * P.C, zero);
      if (INPUT) vec_store<V>(gi + (long long)t * P.C, zero);
    }
  }
  Rows<T, V, FRAMES> rx, rf, ri, rg;
  const auto load = [&](int t) {
    const int at = t + wave * S::WAVE + run * FRAMES;
    if (t + S::ROUND <= P.T) {
      rf.template load<true>(f, P.f_t, at, 0);
      rg.template load<true>(g, P.C, at, 0);
      if (!ENDS) rx.template load<true>(x, P.x_t, at, 0);
      if (INPUT && !ENDS) ri.template load<true>(i, P.i_t, at, 0);
    } else {
      rf.template load<false>(f, P.f_t, at, P.T - 1);
      rg.template load<false>(g, P.C, at, P.T - 1);
      if (!ENDS) rx.template load<false>(x, P.x_t, at, P.T - 1);
      if (INPUT && !ENDS) ri.template load<false>(i, P.i_t, at, P.T - 1);
    }
  };
  const auto round = [&](int first, int turn, auto full) {
    constexpr bool FULL = full.value;
    const int t = first + wave * S::WAVE + run * FRAMES;
    float on[FRAMES][V], off[FRAMES][V], take[FRAMES][V], take_slope[FRAMES][V], in[FRAMES][V], go[FRAMES][V], before[FRAMES][V];
    Product A[V];
    float H[V], E[V], h[V];
#pragma unroll
    for (int c = 0; c < V; ++c) {
      H[c] = 0.f, E[c] = 0.f;
      if (!ENDS) {
        const int row = (first + (wave - wave % S::KEPT_WAVES) * S::WAVE) / SCAN_KEPT;
        h[c] = FULL || row < kept_rows ? P.kept[(b * kept_rows + row) * P.C + channel + c] : 0.f;
      }
    }
    if (ENDS) run_ends_back(rf, rg, FULL ? FRAMES : used - t, A, E);
#pragma unroll
    for (int k = 0; k < (ENDS ? 0 : FRAMES); ++k)
#pragma unroll
      for (int c = 0; c < V; ++c) {
        const bool here = FULL || t + k < used;
        const Gate a = gate(rf.at(k, c)).where(here);
        on[k][c] = a.on;
        go[k][c] = here ? (float)rg.at(k, c) : 0.f;
        // (the slope a (1 - a) is made of these two where it is used)
        off[k][c] = a.off;
        in[k][c] = here ? (float)rx.at(k, c) : 0.f;
        if (INPUT) {
          const Gate u = gate(ri.at(k, c));
          take[k][c] = here ? u.on : 0.f;
          take_slope[k][c] = here ? u.on * u.off : 0.f;
        } else {
          take[k][c] = off[k][c];
        }
        A[c].by(a.on, a.off);
        H[c] = __builtin_fmaf(a.on, H[c], take[k][c] * in[k][c]);
      }
#pragma unroll
    for (int k = ENDS ? -1 : FRAMES - 1; k >= 0; --k)
#pragma unroll
      for (int c = 0; c < V; ++c) E[c] = on[k][c] * (E[c] + go[k][c]);
    if (first > begin) load(first - S::ROUND);
    Joined<CL> joined[V];
#pragma unroll
    for (int c = 0; c < V; ++c) {
      joined[c].template join<!ENDS, true>(A[c], H[c], E[c]);
      if (run == 0) {
        told_a.at[turn][c][column][wave] = joined[c].all.a;
        told_rest.at[turn][c][column][wave] = joined[c].all.rest();
        if (!ENDS) told_h.at[turn][c][column][wave] = joined[c].all_h;
        told_e.at[turn][c][column][wave] = joined[c].all_e;
      }
    }
    __syncthreads();
    if (ENDS && wave) return;  // (the first wave's carry is the segment's)
    float e[V];
#pragma unroll
    for (int c = 0; c < V; ++c) {
      float as[WAVES], rests[WAVES], es[WAVES];
      told_a.get(turn, c, column, as);
      told_rest.get(turn, c, column, rests);
      told_e.get(turn, c, column, es);
      if (!ENDS) {
        float hs[WAVES];
        told_h.get(turn, c, column, hs);
        const int from = wave - wave % S::KEPT_WAVES;
#pragma unroll
        for (int w = 0; w + 1 < WAVES; ++w)
          if (w >= from && w < wave) h[c] = through(as[w], rests[w], h[c], hs[w]);
        h[c] = __builtin_fmaf(joined[c].before_a, h[c], joined[c].before_h);
      }
      e[c] = carry[c];
#pragma unroll
      for (int w = WAVES - 1; w >= 0; --w) {
        carry[c] = through(as[w], rests[w], carry[c], es[w]);
        if (ENDS) factor[c].by(as[w], Product::of(as[w], rests[w]).q);
        if (w == wave + 1) e[c] = carry[c];
      }
      e[c] = __builtin_fmaf(joined[c].behind_a, e[c], joined[c].behind_e);
    }
    if (ENDS) return;
#pragma unroll
    for (int k = 0; k < FRAMES; ++k)
#pragma unroll
      for (int c = 0; c < V; ++c) {
        before[k][c] = h[c];
        h[c] = __builtin_fmaf(on[k][c], h[c], take[k][c] * in[k][c]);
      }
#pragma unroll
    for (int k = FRAMES - 1; k >= 0; --k) {
      typename Vec<T, V>::plain ox, of, oi;
#pragma unroll
      for (int c = 0; c < V; ++c) {
        e[c] += go[k][c];
        const bool here = FULL || t + k < used;
        vec_set<V>(ox, c, (T)(here ? take[k][c] * e[c] : 0.f));
        vec_set<V>(of, c, (T)(here ? on[k][c] * off[k][c] * e[c] * (INPUT ? before[k][c] : before[k][c] - in[k][c]) : 0.f));
        if (INPUT) vec_set<V>(oi, c, (T)(here ? take_slope[k][c] * e[c] * in[k][c] : 0.f));
        e[c] *= on[k][c];
      }
      if ((FULL || t + k < end) && part.live) {
        const long long at = (long long)(t + k) * P.C;
        vec_store<V>(gx + at, ox);
        vec_store<V>(gf + at, of);
        if (INPUT) vec_store<V>(gi + at, oi);
      }
    }
  };
  if (rounds) load(begin + (rounds - 1) * S::ROUND);
  int turn = 0;
  for (int r = rounds - 1; r >= 0; --r, turn ^= 1) {
    const int t = begin + r * S::ROUND;
    if (t + S::ROUND <= used)
      round(t, turn, std::true_type());
    else
      round(t, turn, std::false_type());
  }
  if (!part.live || threadIdx.x >= CL) return;
  if (ENDS) {
    float* p = P.parts + (b * P.segments + part.segment) * 2 * P.C + channel;
#pragma unroll
    for (int c = 0; c < V; ++c) p[c] = factor[c].code(), p[P.C + c] = carry[c];
    return;
  }
  if (P.gfirst && part.segment == 0)
#pragma unroll
    for (int c = 0; c < V; ++c) P.gfirst[b * P.C + channel + c] = carry[c];
}

// One frame: bound by the states' bytes where there are many streams, by the launch where there are few.  256 streams of 2,048 channels, bfloat16: 3 us of a call of 8.
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
    const auto next = [](float h, T x, T f, T i) {
      // (a as the nearest float32 and what that leaves of it; the first difference is exact from a half on, and below it a float32 holds a to its own 2^-24)
      const Gate a = gate(f);
      const float rest = a.on >= 0.5f ? (1.f - a.on) - a.off : 0.f;
      return __builtin_fmaf(a.on, h, __builtin_fmaf(rest, h, (INPUT ? gate(i).on : a.off) * (float)x));
    };
    if (channel + STEP <= P.C) {
      const auto vx = vec_load<STEP>(x), vf = vec_load<STEP>(f), vi = INPUT ? vec_load<STEP>(i) : vf;
      auto h = vec_load<STEP>(state);
      typename Vec<T, STEP>::plain o;
#pragma unroll
      for (int c = 0; c < STEP; ++c) {
        h[c] = next(h[c], vx[c], vf[c], vi[c]);
        o[c] = (T)h[c];
      }
      vec_store<STEP>(state, h);
      vec_store<STEP>(out, o);
    } else {
      for (int c = 0; c < P.C - channel; ++c) {
        const float h = next(state[c], x[c], f[c], INPUT ? i[c] : f[c]);
        state[c] = h;
        out[c] = (T)h;
      }
    }
  }
}

// How a call is cut up: neighbouring channels' lanes in a wave, waves, segments.  16 sequences of 4,096 frames of 2,048 channels in bfloat16, forward and backward: 32 lanes (rows of 128 bytes, a
// line) 171 and 300 us, 16 lanes 220 and 391: lines shared by workgroups cost more than waves that wait.  So 32 lanes wherever their workgroups
// fill the card: 256 of them, the same values, 167 and 304.  128 of them leave half of it idle, 272 and 527; 16 lanes' 256 take 195 and 361, segments of 32 lanes (512 workgroups) 108 + 165 and
// 110 + 311 (two readings).  With 64 workgroups of 32 lanes (half the values) 16 lanes take 162 and 309, segments 54 + 80 and 60 + 170.
struct Cut {
  int lanes, waves;
  int segments, frames;
};
Cut cut_of(long long B, long long T, long long C, int channels /* of a lane */) {
  const long long wide = std::max(1LL, B * ((C + 32 * channels - 1) / (32 * channels))), narrow = std::max(1LL, B * ((C + 16 * channels - 1) / (16 * channels)));
  Cut c = {32, 8, 1, (int)std::max(1LL, T)};
  if (T <= 64) {
    c.waves = 4;
  } else if (T > 256 && wide < 180) {
    if (narrow >= 200) {
      c.lanes = 16;
    } else {
      // 512 workgroups: one sequence of 15,504 frames of 512 channels 9 + 14 us, with 1,024 of them 9 + 18
      const long long rounds = (T + 127) / 128, want = std::min((512 + wide - 1) / wide, rounds), each = (rounds + want - 1) / want;
      c.segments = (int)((rounds + each - 1) / each);
      c.frames = (int)(each * 128);
    }
  }
  return c;
}
unsigned grid_of(const ScanParams& P, int lanes, int channels) { return (unsigned)(P.B * P.segments * ((P.C + lanes * channels - 1) / (lanes * channels))); }

// channels of a lane: four bytes of them, where there are as many
template <typename T, typename F>
hipError_t by_lane(int C, F fn) {
  if constexpr (sizeof(T) == 2)
    if (C > 1) return fn(std::integral_constant<int, 2>());
  return fn(std::integral_constant<int, 1>());
}

// fn(the type, channels of a lane, lanes along the channels, waves, whether there is a gate of the input's own)
template <typename F>
hipError_t by_cut(ScanParams& P, int type, F fn) {
  return by_element(type, [&](auto t) {
    return by_lane<decltype(t)>(P.C, [&](auto v) {
      const Cut c = cut_of(P.B, P.T, P.C, v.value);
      P.segments = c.segments;
      P.segment_frames = c.frames;
      const auto gated = [&](auto lanes, auto waves) { return P.i ? fn(t, v, lanes, waves, std::true_type()) : fn(t, v, lanes, waves, std::false_type()); };
      if (c.waves == 4) return gated(std::integral_constant<int, 32>(), std::integral_constant<int, 4>());
      if (c.lanes == 16) return gated(std::integral_constant<int, 16>(), std::integral_constant<int, 8>());
      return gated(std::integral_constant<int, 32>(), std::integral_constant<int, 8>());
    });
  });
}

}  // namespace

size_t scan_workspace(long long B, long long T, long long C) {
  size_t most = 0;
  for (int channels : {1, 2}) {
    const Cut c = cut_of(B, T, C, channels);
    if (c.segments > 1) most = std::max(most, (size_t)(B * c.segments * 2 * C) * sizeof(float));
  }
  return most;
}

hipError_t launch_scan(ScanParams P, int type, hipStream_t stream) {
  return by_cut(P, type, [&](auto t, auto v, auto lanes, auto waves, auto gated) {
    typedef decltype(t) T;
    constexpr int V = v.value, L = lanes.value, W = waves.value;
    const unsigned grid = grid_of(P, L, V);
    if constexpr (L == 32 && W == 8)
      if (P.segments > 1) hipLaunchKernelGGL((scan_kernel<T, V, L, 8, W, gated.value, true>), dim3(grid), dim3(W * 64), 0, stream, P);
    hipLaunchKernelGGL((scan_kernel<T, V, L, 8, W, gated.value, false>), dim3(grid), dim3(W * 64), 0, stream, P);
    return hipGetLastError();
  });
}

hipError_t launch_scan_backward(ScanParams P, int type, hipStream_t stream) {
  return by_cut(P, type, [&](auto t, auto v, auto lanes, auto, auto gated) {
    typedef decltype(t) T;
    constexpr int V = v.value, L = lanes.value, W = 8;  // (rounds of half as many frames: more is held of each)
    const unsigned grid = grid_of(P, L, V);
    if constexpr (L == 32)
      if (P.segments > 1) hipLaunchKernelGGL((scan_backward_kernel<T, V, L, 8, W, false, true>), dim3(grid), dim3(W * 64), 0, stream, P);
    hipLaunchKernelGGL((scan_backward_kernel<T, V, L, 4, W, gated.value, false>), dim3(grid), dim3(W * 64), 0, stream, P);
    return hipGetLastError();
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
