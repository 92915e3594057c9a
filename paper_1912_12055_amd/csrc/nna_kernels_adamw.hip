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
// The moments are made and their codes' borders met in 64 bits (additions and products there run at float32's rate): a code is then what the definition says, not
// what an order of roundings makes of it.  (The largest code's value is the scale itself, and no product is fused into a sum: b1 s + (1 - b1) g is often halfway between two float32, and
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

// the largest of 16 neighbouring lanes' magnitudes; a NaN beats all
__device__ __forceinline__ float larger(float m, float o) { return o <= m || m != m ? m : o; }
__device__ __forceinline__ float most16(float m) {
  for (int d = 1; d < 16; d <<= 1) m = larger(m, __shfl_xor(m, d));
  return m;
}

constexpr double FIRST = 127. * 127., SECOND = 255. * 255. * 255. * 255.;
static_assert(FIRST * (1. / FIRST) == 1. && SECOND * (1. / SECOND) == 1., "the largest codes' values");
__device__ __forceinline__ double first_value(int code, double scale) { return (double)(code * (code < 0 ? -code : code)) * (1. / FIRST) * scale; }
__device__ __forceinline__ double second_value(unsigned code, double scale) { return (double)(code * code * code * code) * (1. / SECOND) * scale; }
__device__ __forceinline__ double blend(double old, double b, double fresh, double n) {
#pragma clang fp contract(off)
  return old * b + fresh * n;
}

// the code whose square is nearest to a = |m| (by its root) in units of the scale: a first guess in float32, its borders in 64 bits
__device__ __forceinline__ int first_code(double m, double unit, float per_scale) {
  const double a = __builtin_fabs(m);
  float c = __builtin_rintf(127.f * __builtin_amdgcn_sqrtf((float)a * per_scale));
  c = c < 127.f ? c : 127.f;
  const double lower = (double)c - 0.5, upper = (double)c + 0.5;
  if (c > 0.f && a < lower * lower * unit)
    c -= 1.f;
  else if (c < 127.f && a >= upper * upper * unit)
    c += 1.f;
  return m < 0. ? -(int)c : (int)c;
}
// the largest code that, `shift` (in [0, 1)) less, is no larger than v's fourth root in units of the scale
__device__ __forceinline__ unsigned second_code(double v, double unit, float per_scale, float shift) {
  float c = __builtin_floorf(255.f * __builtin_amdgcn_sqrtf(__builtin_amdgcn_sqrtf((float)v * per_scale)) + shift);
  c = c < 255.f ? c : 255.f;
  const double here = (double)c - (double)shift, next = here + 1.;
  if (here > 0. && here * here * (here * here) * unit > v)
    c -= 1.f;
  else if (c < 255.f && next * next * (next * next) * unit <= v)
    c += 1.f;
  return v > 0. && c < 1.f ? 1u : (unsigned)c;
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
      Values<signed char> om = {};
      Values<unsigned char> ov = {};
      double um = 0., uv = 0.;
      // (n is none for whole groups of 16 lanes, too, behind the tensor's last block: those have no scales)
      const long long block = state / ADAMW_BLOCK;
      const bool there = at - (threadIdx.x & 15) * EACH < end;
      if (n) {
        om = load_some(mc, n);
        ov = load_some(vc, n);
      }
      if (there) {
        um = (double)P.m_scales[block];
        uv = (double)P.v_scales[block];
      }
      double dm[EACH], dv[EACH];
      float most_m = 0.f, most_v = 0.f;
#pragma unroll
      for (int i = 0; i < EACH; ++i) {
        const double d = (double)(float)vg.v[i];
        dm[i] = blend(first_value(om.v[i], um), P.beta1, d, 1. - P.beta1);
        dv[i] = blend(second_value(ov.v[i], uv), P.beta2, d * d, 1. - P.beta2);
        m[i] = (float)dm[i];
        v[i] = (float)dv[i];
        if (i < n) {
          most_m = larger(most_m, __builtin_fabsf(m[i]));
          most_v = larger(most_v, v[i]);
        }
      }
      most_m = most16(most_m);
      most_v = most16(most_v);
      // a block with a value that is not finite stands for NaN throughout, so that none is lost; one without a normal float32 is zero
      const bool some_m = most_m >= 0x1p-126f && most_m < __builtin_inff(), some_v = most_v >= 0x1p-126f && most_v < __builtin_inff();
      if (there && (threadIdx.x & 15) == 0) {
        P.m_scales[block] = some_m ? most_m : most_m < 1.f ? 0.f : __builtin_nanf("");
        P.v_scales[block] = some_v ? most_v : most_v < 1.f ? 0.f : __builtin_nanf("");
      }
      signed char cm[EACH];
      unsigned char cv[EACH];
      um = (double)most_m * (1. / FIRST);
      uv = (double)most_v * (1. / SECOND);
      const float rm = 1.f / most_m, rv = 1.f / most_v;
#pragma unroll
      for (int i = 0; i < EACH; ++i) {
        const unsigned place = (unsigned)(state + i) * 0x9E3779B9u + F.shift;
        cm[i] = (signed char)(some_m ? first_code(dm[i], um, rm) : 0);
        cv[i] = (unsigned char)(some_v ? second_code(dv[i], uv, rv, (float)(place >> 8) * 0x1p-24f) : 0);
      }
      if (n) {
        store_some(mc, n, cm);
        store_some(vc, n, cv);
      }
    }
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
      const float old = NARROW && P.master ? copy.v[i] : (float)vp.v[i];
      weight[i] = old * F.keep - F.rate * (m[i] / (sqrtf(v[i]) * F.root + P.eps));
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
      const auto c = load_some(static_cast<const unsigned char*>(codes) + at * EACH, EACH);
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
  const unsigned grid = (unsigned)std::max(1LL, std::min((blocks * (ADAMW_BLOCK / EACH) + THREADS - 1) / THREADS, 8192LL));
  if (second)
    hipLaunchKernelGGL(moment_kernel<true>, dim3(grid), dim3(THREADS), 0, stream, codes, scales, blocks, out);
  else
    hipLaunchKernelGGL(moment_kernel<false>, dim3(grid), dim3(THREADS), 0, stream, codes, scales, blocks, out);
  return hipGetLastError();
}

}  // namespace nna
