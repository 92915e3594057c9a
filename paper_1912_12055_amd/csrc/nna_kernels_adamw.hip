// AdamW steps over many tensors in one launch, states in 32 bits or in 8.
//
//   m <- b1 m + (1 - b1) g,   v <- b2 v + (1 - b2) g^2,   p <- (1 - lr wd) p - lr / (1 - b1^t) m / (sqrt(v / (1 - b2^t)) + eps).
// Bound by memory: a float32 weight with float32 states is 16 bytes read and 12 written, with states in 8 bits 10.1 and 6.1.
//
// 8 bits: ADAMW_BLOCK neighbours share a scale s, their largest magnitude.  A first moment's code c in -127..127 stands for s (c / 127) |c / 127|, a second moment's in
// 0..255 for s (c / 255)^4: both finer towards zero.  An update divides by sqrt(v), which goes with (c / 255)^2: down to 2^-16 of the block's largest, where the first
// moment, which ends at 2^-14 of its largest, is zero before it; and none that is not zero becomes zero.  A second moment changes by 1 - b2 of itself a step, far less than the
// distance of its codes (1.6 % at the largest): rounded to the nearest it would stay where it is for good.  So it is rounded up or down by a number in [0, 1) that
// goes with the value's place and the step, the fractions of an additive sequence, whose mean over the steps is 1/2: no state of a random generator, and the same inputs give the same bits.
// The moments' codes and scales are what 64 bits make of them: a code is then what the definition says, not what an order of roundings makes of it.  Made in 64 bits throughout that
// took 170 instructions a value, and 1,015 us for 201 million weights, half as long again as their bytes; now float32 does what it can tell, and 64 bits the few values near a border or a block's largest.  (The largest code's value is the scale itself, and no product is fused into a sum: b1 s + (1 - b1) g is often halfway between two float32, and
// which of them is the next scale has to be one answer.)  The weights and the divisions are float32.
#include "nna_adamw.h"
#include "nna_vector.h"

#include <type_traits>

namespace nna {

namespace {

constexpr int THREADS = 256, EACH = 8;  // values of a lane: 16 lanes take a block

template <typename T>
struct Values {
  T v[EACH];
};
// n (at least 1) values from p, the others zero
template <typename T>
__device__ __forceinline__ Values<T> load_some(const T* p, int n) {
  Values<T> r;
  if (n >= EACH) {
    const auto u = vec_load<EACH>(p);
#pragma unroll
    for (int i = 0; i < EACH; ++i) r.v[i] = u[i];
  } else {
#pragma unroll
    for (int i = 0; i < EACH; ++i) r.v[i] = i < n ? p[i] : (T)0;
  }
  return r;
}
template <typename T, typename S>
__device__ __forceinline__ void store_some(T* p, int n, const S (&v)[EACH]) {
  if (n >= EACH) {
    typename Vec<T, EACH>::plain u;
#pragma unroll
    for (int i = 0; i < EACH; ++i) u[i] = (T)v[i];
    vec_store<EACH>(p, u);
  } else {
#pragma unroll
    for (int i = 0; i < EACH; ++i)
      if (i < n) p[i] = (T)v[i];
  }
}

// the largest of 16 neighbouring lanes' magnitudes, in all of them; a NaN beats all
__device__ __forceinline__ float larger(float m, float o) { return o <= m || m != m ? m : o; }
template <int N>
__device__ __forceinline__ float rotated(float v) {
  return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), 0x120 + N, 0xf, 0xf, true));
}
__device__ __forceinline__ float most16(float m) {
  m = larger(m, rotated<8>(m));
  m = larger(m, rotated<4>(m));
  m = larger(m, rotated<2>(m));
  return larger(m, rotated<1>(m));
}

constexpr double FIRST = 127. * 127., SECOND = 255. * 255. * 255. * 255.;
static_assert(FIRST * (1. / FIRST) == 1. && SECOND * (1. / SECOND) == 1., "the largest codes' values");
__device__ __forceinline__ double first_value(int code, double scale) { return (double)(code * (code < 0 ? -code : code)) * (1. / FIRST) * scale; }
__device__ __forceinline__ double second_value(unsigned code, double scale) { return (double)(code * code * code * code) * (1. / SECOND) * scale; }
__device__ __forceinline__ double blend(double old, double b, double fresh) {
#pragma clang fp contract(off)
  return old * b + fresh * (1. - b);
}

// One moment of a lane's eight values in 8 bits: what was, and what is now, in float32 and in 64 bits, as the definition has it.
constexpr float TINY = 0x1p-100f;  // below it products of float32 may have lost their last bits: everything is made in 64 then
struct First {
  Values<signed char> was;
  float scale;
  double beta;
  __device__ __forceinline__ float now(int i, float g) const {
    const float c = (float)was.v[i];
    return c * __builtin_fabsf(c) * (scale * (float)(1. / FIRST)) * (float)beta + g * (float)(1. - beta);
  }
  __device__ __forceinline__ double exact(int i, float g) const { return blend(first_value(was.v[i], (double)scale), beta, (double)g); }
  // what now() may be off by: five roundings of its terms.  The sum may be far smaller than they are; with the new scale s no term is larger than s + the old one's
  __device__ __forceinline__ float off(float s) const { return s < TINY ? __builtin_inff() : 0x1p-21f * (s + 2.f * scale); }
};
struct Second {
  Values<unsigned char> was;
  float scale;
  double beta;
  __device__ __forceinline__ float now(int i, float g) const {
    const float c = (float)was.v[i], s = c * c * (float)(1. / 65025.);
    return s * s * scale * (float)beta + g * (g * (float)(1. - beta));
  }
  __device__ __forceinline__ double exact(int i, float g) const { return blend(second_value(was.v[i], (double)scale), beta, (double)g * (double)g); }
  __device__ __forceinline__ float off(float s) const { return s < TINY ? __builtin_inff() : 0x1p-20f * s; }  // (a sum of positive terms)
};

// The scale of 16 lanes' block, the largest of the 64-bit moments rounded: only those that float32 can't tell from the largest are made in 64 bits.
template <typename M>
__device__ __forceinline__ float scale_of(const M& moment, const float (&now)[EACH], const Values<float>& g, int n) {
  float most = 0.f, spoilt = 0.f;
#pragma unroll
  for (int i = 0; i < EACH; ++i) {
    const float a = i < n ? __builtin_fabsf(now[i]) : 0.f;
    most = __builtin_fmaxf(most, a);
    spoilt = __builtin_fmaf(a, 0.f, spoilt);  // NaN if one is not finite
  }
  most = most16(spoilt != spoilt ? spoilt : most);
  const float near = most - 2.f * moment.off(most);
  float exact = most != most ? most : 0.f;
#pragma unroll
  for (int i = 0; i < EACH; ++i)
    if (i < n && __builtin_fabsf(now[i]) >= near) exact = larger(exact, (float)__builtin_fabs(moment.exact(i, g.v[i])));
  return most16(exact);
}

// The code whose square is nearest to |m| (by its root) in units of the scale s.  float32's guess y is off by 127^2 / (2 y) of what m is (`per`: 127^2 off / s) and by five roundings of
// itself; where a border is as near, or y so small that this does not say it, 64 bits decide.
__device__ __forceinline__ int first_code(const First& moment, int i, float g, float now, float s, float per_scale, float per) {
  float y = 127.f * __builtin_amdgcn_sqrtf(__builtin_fabsf(now) * per_scale), c = __builtin_rintf(y);
  if (__builtin_expect(!((0.5f - __builtin_fabsf(y - c)) * y > per + y * 0x1p-13f || (y < 0.25f && per < 0.125f)), 0)) {
    const double m = moment.exact(i, g), a = __builtin_fabs(m), unit = (double)s * (1. / FIRST);
    c = __builtin_rintf(127.f * __builtin_amdgcn_sqrtf((float)a * per_scale));
    const double lower = (double)c - 0.5, upper = (double)c + 0.5;
    if (c > 0.f && a < lower * lower * unit)
      c -= 1.f;
    else if (a >= upper * upper * unit)
      c += 1.f;
    now = (float)m;
  }
  c = c < 127.f ? c : 127.f;
  return (int)__builtin_copysignf(c, now);
}
// The largest code that, `shift` (in [0, 1)) less, is no larger than v's fourth root in units of the scale.  The root leaves a quarter of v's five roundings, and of the quotient's: y is off by 2^-14.
__device__ __forceinline__ unsigned second_code(const Second& moment, int i, float g, float now, float s, float per_scale, float shift) {
  const float y = 255.f * __builtin_amdgcn_sqrtf(__builtin_amdgcn_sqrtf(now * per_scale)) + shift;
  float c = __builtin_floorf(y);
  const bool tiny = now < TINY && (g != 0.f || moment.was.v[i] != 0);
  if (__builtin_expect(__builtin_fabsf(y - c - 0.5f) > 0.5f - 0x1p-12f || tiny, 0)) {
    const double unit = (double)s * (1. / SECOND), v = moment.exact(i, g);
    c = __builtin_floorf(255.f * __builtin_amdgcn_sqrtf(__builtin_amdgcn_sqrtf((float)v * per_scale)) + shift);
    const double here = (double)c - (double)shift, next = here + 1.;
    if (here > 0. && here * here * (here * here) * unit > v)
      c -= 1.f;
    else if (next * next * (next * next) * unit <= v)
      c += 1.f;
    now = v > 0. ? 1.f : 0.f;
  }
  c = c < 255.f ? c : 255.f;
  return now > 0.f && c < 1.f ? 1u : (unsigned)c;
}

// the root to one unit, of values that have no normal float32, too
__device__ __forceinline__ float root_of(float v) {
  const bool small = v < 0x1p-60f;
  return __builtin_amdgcn_sqrtf(small ? v * 0x1p64f : v) * (small ? 0x1p-32f : 1.f);
}

struct Factors {
  float keep, rate, root;  // 1 - lr wd, lr / (1 - b1^t), 1 / sqrt(1 - b2^t)
  unsigned shift;          // the step's part of the additive sequence
};
__device__ __forceinline__ double power(double b, long long t) {
  double r = 1.;
  for (; t > 0; t >>= 1, b *= b)
    if (t & 1) r *= b;
  return r;
}

template <typename T, int BITS>
__device__ __forceinline__ void update(const AdamwParams& P, const AdamwTensor& tensor, long long from, const Factors& F) {
  // 64 lanes take four blocks
  const long long begin = from + threadIdx.x * EACH;
  const long long end = from + P.piece < tensor.n ? from + P.piece : tensor.n;
  T* const p = static_cast<T*>(tensor.p);
  const T* const g = static_cast<const T*>(tensor.g);
  constexpr bool NARROW = sizeof(T) == 2;
  const float b1 = (float)P.beta1, b2 = (float)P.beta2, n1 = (float)(1. - P.beta1), n2 = (float)(1. - P.beta2);
  for (long long base = from; base < end; base += THREADS * EACH) {
    const long long at = begin + (base - from), state = tensor.at + at;
    const int n = at < end ? (int)(end - at < EACH ? end - at : EACH) : 0;
    if (BITS == 32 && !n) continue;
    Values<T> vp = {}, vg = {};
    Values<float> copy = {};
    float m[EACH], v[EACH], weight[EACH];
    if (n) {
      vg = load_some(g + at, n);
      if (NARROW && P.master)
        copy = load_some(P.master + state, n);
      else
        vp = load_some(p + at, n);
    }
    if constexpr (BITS == 32) {
      const Values<float> om = load_some(static_cast<float*>(P.m) + state, n), ov = load_some(static_cast<float*>(P.v) + state, n);
#pragma unroll
      for (int i = 0; i < EACH; ++i) {
        const float d = (float)vg.v[i];
        m[i] = om.v[i] * b1 + d * n1;
        v[i] = ov.v[i] * b2 + d * d * n2;
      }
      store_some(static_cast<float*>(P.m) + state, n, m);
      store_some(static_cast<float*>(P.v) + state, n, v);
    } else {
      signed char* const mc = static_cast<signed char*>(P.m) + state;
      unsigned char* const vc = static_cast<unsigned char*>(P.v) + state;
      // (n is none for whole groups of 16 lanes, too, behind the tensor's last block: those have no scales)
      const long long block = state / ADAMW_BLOCK;
      const bool there = at - (threadIdx.x & 15) * EACH < end;
      First first = {{}, 0.f, P.beta1};
      Second second = {{}, 0.f, P.beta2};
      Values<float> d;
      if (n) {
        first.was = load_some(mc, n);
        second.was = load_some(vc, n);
      }
      if (there) {
        first.scale = P.m_scales[block];
        second.scale = P.v_scales[block];
      }
#pragma unroll
      for (int i = 0; i < EACH; ++i) {
        d.v[i] = (float)vg.v[i];
        m[i] = first.now(i, d.v[i]);
        v[i] = second.now(i, d.v[i]);
      }
      const float most_m = scale_of(first, m, d, n), most_v = scale_of(second, v, d, n);
      // a block with a value that is not finite stands for NaN throughout, so that none is lost; one without a normal float32 is zero
      const bool some_m = most_m >= 0x1p-126f && most_m < __builtin_inff(), some_v = most_v >= 0x1p-126f && most_v < __builtin_inff();
      if (there && (threadIdx.x & 15) == 0) {
        P.m_scales[block] = some_m ? most_m : most_m < 1.f ? 0.f : __builtin_nanf("");
        P.v_scales[block] = some_v ? most_v : most_v < 1.f ? 0.f : __builtin_nanf("");
      }
      signed char cm[EACH];
      unsigned char cv[EACH];
      const float rm = 1.f / most_m, rv = 1.f / most_v, per = 127.f * 127.f * first.off(most_m) * rm;
#pragma unroll
      for (int i = 0; i < EACH; ++i) {
        const float shift = (float)(((unsigned)(state + i) * 0x9E3779B9u + F.shift) >> 8) * 0x1p-24f;
        cm[i] = (signed char)(some_m ? first_code(first, i, d.v[i], m[i], most_m, rm, per) : 0);
        cv[i] = (unsigned char)(some_v ? second_code(second, i, d.v[i], v[i], most_v, rv, shift) : 0);
      }
      if (n) {
        store_some(mc, n, cm);
        store_some(vc, n, cv);
      }
    }
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
      const float old = NARROW && P.master ? copy.v[i] : (float)vp.v[i];
      weight[i] = old * F.keep - F.rate * (m[i] * __builtin_amdgcn_rcpf(root_of(v[i]) * F.root + P.eps));
      asm("" : "+v"(weight[i]));  // a float32 from here on: the 16-bit weight is its float32 copy rounded, not the sum behind it
    }
    if (n) {
      store_some(p + at, n, weight);
      if (NARROW && P.master) store_some(P.master + state, n, weight);
    }
  }
}

template <int BITS>
__global__ __launch_bounds__(THREADS) void adamw_kernel(AdamwParams P) {
  // the tensor of this piece: the last one whose first piece is not behind it
  int low = 0, high = P.count;
  while (high - low > 1) {
    const int middle = (low + high) / 2;
    if ((int)blockIdx.x < P.tensors[middle].first)
      high = middle;
    else
      low = middle;
  }
  const AdamwTensor tensor = P.tensors[low];
  const long long from = (long long)((int)blockIdx.x - tensor.first) * P.piece;
  const long long t = P.step_dev ? *P.step_dev : P.step;
  const double lr = P.lr_dev ? (double)*P.lr_dev : P.lr;
  Factors F;
  F.keep = (float)(1. - lr * P.weight_decay);
  F.rate = (float)(lr / (1. - power(P.beta1, t)));
  F.root = (float)(1. / sqrt(1. - power(P.beta2, t)));
  F.shift = (unsigned)t * 0xB504F333u;
  if (tensor.type == NNA_F32)
    update<float, BITS>(P, tensor, from, F);
  else if (tensor.type == NNA_BF16)
    update<bf16, BITS>(P, tensor, from, F);
  else
    update<f16, BITS>(P, tensor, from, F);
}

template <bool SECOND_ONE>
__global__ __launch_bounds__(THREADS) void moment_kernel(const void* codes, const float* scales, long long blocks, float* out) {
  for (long long at = (long long)blockIdx.x * THREADS + threadIdx.x; at < blocks * (ADAMW_BLOCK / EACH); at += (long long)gridDim.x * THREADS) {
    const double scale = scales[at / (ADAMW_BLOCK / EACH)];
    float v[EACH];
    if constexpr (SECOND_ONE) {
      const Values<unsigned char> c = load_some(static_cast<const unsigned char*>(codes) + at * EACH, EACH);
#pragma unroll
      for (int i = 0; i < EACH; ++i) v[i] = (float)second_value(c.v[i], scale);
    } else {
      const auto c = load_some(static_cast<const signed char*>(codes) + at * EACH, EACH);
#pragma unroll
      for (int i = 0; i < EACH; ++i) v[i] = (float)first_value(c.v[i], scale);
    }
    store_some(out + at * EACH, EACH, v);
  }
}

}  // namespace

int adamw_piece(long long values) { return values < 1 << 22 ? THREADS * EACH : 4 * THREADS * EACH; }

hipError_t launch_adamw(const AdamwParams& P, hipStream_t stream) {
  static_assert(sizeof(AdamwParams) <= 4096, "arguments of a launch");
  if (P.m_scales)
    hipLaunchKernelGGL(adamw_kernel<8>, dim3(P.pieces), dim3(THREADS), 0, stream, P);
  else
    hipLaunchKernelGGL(adamw_kernel<32>, dim3(P.pieces), dim3(THREADS), 0, stream, P);
  return hipGetLastError();
}

hipError_t launch_adamw_moment(const void* codes, bool second, const float* scales, long long blocks, float* out, hipStream_t stream) {
  const unsigned grid = (unsigned)std::max(1LL, std::min((blocks * (ADAMW_BLOCK / EACH) + THREADS - 1) / THREADS, 1LL << 22));
  if (second)
    hipLaunchKernelGGL(moment_kernel<true>, dim3(grid), dim3(THREADS), 0, stream, codes, scales, blocks, out);
  else
    hipLaunchKernelGGL(moment_kernel<false>, dim3(grid), dim3(THREADS), 0, stream, codes, scales, blocks, out);
  return hipGetLastError();
}

}  // namespace nna
