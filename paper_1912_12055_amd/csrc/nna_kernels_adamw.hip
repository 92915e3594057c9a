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
// The moments' codes and scales are what 64 bits make of them, so that a code is what the definition says and not what an order of roundings makes of it.  (The largest code's value is the
// scale itself, and no product is fused into a sum: b1 s + (1 - b1) g is often halfway between two float32, and which of them is the next scale has to be one answer.)  Float32 does what it
// can tell, and 64 bits the few values near a border or a block's largest: in 64 bits throughout, 126 to 170 instructions a value, 201 million bfloat16 weights with their float32 copies took
// 890 to 1,025 us; now 642, 5.1 TB/s.  With states in 32 bits 1,092 us, 5.2 TB/s.  A table of a launch's tensors goes with its arguments; 28 small tensors, 1.6 million values: 10 us.
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
template <bool FULL, typename T>
__device__ __forceinline__ Values<T> load_some(const T* p, int n) {
  Values<T> r;
  if (FULL || n >= EACH) {
    const auto u = vec_load<EACH>(p);
#pragma unroll
    for (int i = 0; i < EACH; ++i) r.v[i] = u[i];
  } else {
#pragma unroll
    for (int i = 0; i < EACH; ++i) r.v[i] = i < n ? p[i] : (T)0;
  }
  return r;
}
template <bool FULL, typename T, typename S>
__device__ __forceinline__ void store_some(T* p, int n, const S (&v)[EACH]) {
  if (FULL || n >= EACH) {
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

// Eight codes, as two words.
struct Codes {
  unsigned w[2];
  __device__ __forceinline__ unsigned at(int i) const { return (w[i / 4] >> (i % 4 * 8)) & 255u; }
  // the next code, a float32 that is a whole number from 0 to 255
  __device__ __forceinline__ void put(int i, float c) { w[i / 4] = __builtin_amdgcn_cvt_pk_u8_f32(c, i % 4, w[i / 4]); }
};
typedef unsigned Pair __attribute__((ext_vector_type(2), aligned(1)));
template <bool FULL>
__device__ __forceinline__ Codes load_codes(const unsigned char* p, int n) {
  if (FULL || n >= EACH) {
    const Pair u = *reinterpret_cast<const Pair*>(p);
    return {{u[0], u[1]}};
  }
  Codes c = {{0u, 0u}};
#pragma unroll
  for (int i = 0; i < EACH; ++i)
    if (i < n) c.w[i / 4] |= (unsigned)p[i] << (i % 4 * 8);
  return c;
}
template <bool FULL>
__device__ __forceinline__ void store_codes(unsigned char* p, int n, const Codes& c) {
  if (FULL || n >= EACH) {
    *reinterpret_cast<Pair*>(p) = Pair{c.w[0], c.w[1]};
    return;
  }
#pragma unroll
  for (int i = 0; i < EACH; ++i)
    if (i < n) p[i] = (unsigned char)c.at(i);
}

// One moment of a lane's eight values in 8 bits: what was, and what is now, in float32 and in 64 bits, as the definition has it.
constexpr float TINY = 0x1p-80f;  // below it products of float32 may have lost their last bits: everything is made in 64 then
// Whether a factor of the codes' powers has no normal float32, though what it makes of the larger codes has one: what was is then read in 64 bits (else a block's history, scales below 2^-94
// of second moments and 2^-112 of first ones, fades out of its weights: steps up to 1 / sqrt(1 - b2) too long where eps is as small)
__device__ __forceinline__ bool faded(float factor, float scale, double beta) { return factor < 0x1p-126f && scale > 0.f && beta > 0.; }
struct First {
  Codes was;  // their highest bits turned: 0..255 for -128..127
  float scale, old, fresh;
  double beta;
  __device__ __forceinline__ First(Codes c, float s, double b) : was(c), scale(s), old(s * (float)(b * (1. / FIRST))), fresh((float)(1. - b)), beta(b) {
    was.w[0] ^= 0x80808080u;
    was.w[1] ^= 0x80808080u;
  }
  __device__ __forceinline__ float now(int i, float g) const {
    const float c = (float)was.at(i) - 128.f;
    return __builtin_fmaf(c * __builtin_fabsf(c), old, g * fresh);
  }
  __device__ __forceinline__ double exact(int i, float g) const { return blend(first_value((int)was.at(i) - 128, (double)scale), beta, (double)g); }
  // what now() may be off by: five roundings of its terms.  The sum may be far smaller than they are; with the new scale s no term is larger than s + the old one's
  __device__ __forceinline__ float off(float s) const { return s < TINY ? __builtin_inff() : 0x1p-21f * (s + 2.f * scale); }
};
struct Second {
  Codes was;
  float scale, old, fresh;
  double beta;
  __device__ __forceinline__ Second(Codes c, float s, double b) : was(c), scale(s), old(s * (float)(b * (1. / SECOND))), fresh((float)(1. - b)), beta(b) {}
  __device__ __forceinline__ float now(int i, float g) const {
    const float c = (float)was.at(i), s = c * c;
    return __builtin_fmaf(s * s, old, g * (g * fresh));
  }
  __device__ __forceinline__ double exact(int i, float g) const { return blend(second_value(was.at(i), (double)scale), beta, (double)g * (double)g); }
  __device__ __forceinline__ float off(float s) const { return s < TINY ? __builtin_inff() : 0x1p-20f * s; }  // (a sum of positive terms)
};

// The scale of 16 lanes' block, the largest of the 64-bit moments rounded: only those that float32 can't tell from the largest are made in 64 bits.
template <bool FULL, typename M>
__device__ __forceinline__ float scale_of(const M& moment, const float (&now)[EACH], const Values<float>& g, int n) {
  float most = 0.f, spoilt = 0.f;
#pragma unroll
  for (int i = 0; i < EACH; ++i) {
    const float a = FULL || i < n ? __builtin_fabsf(now[i]) : 0.f;
    most = __builtin_fmaxf(most, a);
    spoilt = __builtin_fmaf(a, 0.f, spoilt);  // NaN if one is not finite
  }
  most = most16(spoilt != spoilt ? spoilt : most);
  const float near = most - 2.f * moment.off(most);
  float exact = most != most ? most : 0.f;
#pragma unroll
  for (int i = 0; i < EACH; ++i)
    if ((FULL || i < n) && __builtin_fabsf(now[i]) >= near) exact = larger(exact, (float)__builtin_fabs(moment.exact(i, g.v[i])));
  return most16(exact);
}

// The code whose square is nearest to |m| (by its root) in units of the scale s (`each` = 1 / s).  float32's guess y is off by 127^2 / (2 y) of what m is (`per` = 127^2 off / s) and by
// five roundings of itself; where a border is as near 64 bits decide.  (Below a quarter y is held to be one there: the code is 0 if y^2 + 2 per is below a quarter.)
__device__ __forceinline__ float first_code(const First& moment, int i, float g, float now, float s, float each, float per) {
  const float y = 127.f * __builtin_amdgcn_sqrtf(__builtin_fabsf(now) * each);
  float c = __builtin_rintf(y);
  if (__builtin_expect(!(((0.5f - 0x1p-13f) - __builtin_fabsf(y - c)) * __builtin_fmaxf(y, 0.25f) > per), 0)) {
    const double m = moment.exact(i, g), a = __builtin_fabs(m), unit = (double)s * (1. / FIRST);
    c = __builtin_rintf(127.f * __builtin_amdgcn_sqrtf((float)a * each));
    const double lower = (double)c - 0.5, upper = (double)c + 0.5;
    if (c > 0.f && a < lower * lower * unit)
      c -= 1.f;
    else if (a >= upper * upper * unit)
      c += 1.f;
    c = c < 127.f ? c : 127.f;
    now = (float)m;
  }
  return __builtin_copysignf(c, now);
}
// The largest code that, `shift` (in [0, 1)) less, is no larger than v's fourth root in units of the scale s (`each` = 1 / s).  The root leaves a quarter of v's five roundings and of
// the quotient's: y is off by less than 2^-13.
__device__ __forceinline__ float second_code(const Second& moment, int i, float g, float now, float s, float each, float shift) {
  const float y = __builtin_fmaf(255.f, __builtin_amdgcn_sqrtf(__builtin_amdgcn_sqrtf(now * each)), shift);
  float c = __builtin_floorf(y);
  bool some = now > 0.f;
  if (__builtin_expect(!(__builtin_fabsf(y - c - 0.5f) < 0.5f - 0x1p-12f) || now < TINY, 0)) {
    const double unit = (double)s * (1. / SECOND), v = moment.exact(i, g);
    c = __builtin_floorf(__builtin_fmaf(255.f, __builtin_amdgcn_sqrtf(__builtin_amdgcn_sqrtf((float)v * each)), shift));
    const double here = (double)c - (double)shift, next = here + 1.;
    if (here > 0. && here * here * (here * here) * unit > v)
      c -= 1.f;
    else if (next * next * (next * next) * unit <= v)
      c += 1.f;
    c = c < 255.f ? c : 255.f;
    some = v > 0.;
  }
  return __builtin_fmaxf(c, some ? 1.f : 0.f);
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

// n (FULL: all of them) of a lane's values from `at` on, the tensor's own count
template <typename T, int BITS, bool FULL>
__device__ __forceinline__ void update(const AdamwParams& P, const AdamwTensor& tensor, long long at, int n, bool there, const Factors& F) {
  T* const p = static_cast<T*>(tensor.p) + at;
  const T* const g = static_cast<const T*>(tensor.g) + at;
  const long long state = tensor.at + at;
  const bool copied = sizeof(T) == 2 && P.master;
  float m[EACH], v[EACH], old[EACH] = {}, root[EACH];
  Values<float> d = {};
  if (FULL || n) {
    const Values<T> fresh = load_some<FULL>(g, n);
#pragma unroll
    for (int i = 0; i < EACH; ++i) d.v[i] = (float)fresh.v[i];
    if (copied) {
      const Values<float> w = load_some<FULL>(P.master + state, n);
#pragma unroll
      for (int i = 0; i < EACH; ++i) old[i] = w.v[i];
    } else {
      const Values<T> w = load_some<FULL>(p, n);
#pragma unroll
      for (int i = 0; i < EACH; ++i) old[i] = (float)w.v[i];
    }
  }
  if constexpr (BITS == 32) {
    float *const pm = static_cast<float*>(P.m) + state, *const pv = static_cast<float*>(P.v) + state;
    const float b1 = (float)P.beta1, b2 = (float)P.beta2, n1 = (float)(1. - P.beta1), n2 = (float)(1. - P.beta2);
    if (!FULL && !n) return;
    const Values<float> om = load_some<FULL>(pm, n), ov = load_some<FULL>(pv, n);
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
      m[i] = om.v[i] * b1 + d.v[i] * n1;
      v[i] = ov.v[i] * b2 + d.v[i] * (d.v[i] * n2);
    }
    store_some<FULL>(pm, n, m);
    store_some<FULL>(pv, n, v);
  } else {
    unsigned char *const pm = static_cast<unsigned char*>(P.m) + state, *const pv = static_cast<unsigned char*>(P.v) + state;
    const long long block = state / ADAMW_BLOCK;
    const First first(load_codes<FULL>(pm, n), FULL || there ? P.m_scales[block] : 0.f, P.beta1);
    const Second second(load_codes<FULL>(pv, n), FULL || there ? P.v_scales[block] : 0.f, P.beta2);
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
      m[i] = first.now(i, d.v[i]);
      v[i] = second.now(i, d.v[i]);
    }
    if (__builtin_expect(faded(first.old, first.scale, P.beta1), 0))
#pragma unroll
      for (int i = 0; i < EACH; ++i) m[i] = (float)first.exact(i, d.v[i]);
    if (__builtin_expect(faded(second.old, second.scale, P.beta2), 0))
#pragma unroll
      for (int i = 0; i < EACH; ++i) v[i] = (float)second.exact(i, d.v[i]);
    const float most_m = scale_of<FULL>(first, m, d, n), most_v = scale_of<FULL>(second, v, d, n);
    // a block with a value that is not finite stands for NaN throughout, so that none is lost; one without a normal float32 is zero
    const bool some_m = most_m >= 0x1p-126f && most_m < __builtin_inff(), some_v = most_v >= 0x1p-126f && most_v < __builtin_inff();
    if ((FULL || there) && (threadIdx.x & 15) == 0) {
      P.m_scales[block] = some_m ? most_m : most_m < 1.f ? 0.f : __builtin_nanf("");
      P.v_scales[block] = some_v ? most_v : most_v < 1.f ? 0.f : __builtin_nanf("");
    }
    Codes cm = {}, cv = {};
    if (some_m) {
      const float each = 1.f / most_m, per = (float)FIRST * (first.off(most_m) * each);
#pragma unroll
      for (int i = 0; i < EACH; ++i) cm.put(i, first_code(first, i, d.v[i], m[i], most_m, each, per) + 128.f);
      cm.w[0] ^= 0x80808080u;
      cm.w[1] ^= 0x80808080u;
    }
    if (some_v) {
      const float each = 1.f / most_v;
      const unsigned place = (unsigned)state * 0x9E3779B9u + F.shift;
#pragma unroll
      for (int i = 0; i < EACH; ++i) {
        const float shift = (float)((place + i * 0x9E3779B9u) >> 8) * 0x1p-24f;
        cv.put(i, second_code(second, i, d.v[i], v[i], most_v, each, shift));
      }
    }
    if (FULL || n) {
      store_codes<FULL>(pm, n, cm);
      store_codes<FULL>(pv, n, cv);
    }
  }
  // (a root that has lost its last bits is one of a v below 2^-126: nothing beside any eps but the smallest)
#pragma unroll
  for (int i = 0; i < EACH; ++i) root[i] = __builtin_amdgcn_sqrtf(v[i]);
  if (P.eps < 0x1p-40f)
#pragma unroll
    for (int i = 0; i < EACH; ++i) root[i] = root_of(v[i]);
#pragma unroll
  for (int i = 0; i < EACH; ++i) {
    old[i] = old[i] * F.keep - F.rate * (m[i] * __builtin_amdgcn_rcpf(__builtin_fmaf(root[i], F.root, P.eps)));
    asm("" : "+v"(old[i]));  // a float32 from here on: the 16-bit weight is its float32 copy rounded, not the sum behind it
  }
  if (FULL || n) {
    store_some<FULL>(p, n, old);
    if (copied) store_some<FULL>(P.master + state, n, old);
  }
}

template <typename T, int BITS>
__device__ __forceinline__ void update_piece(const AdamwParams& P, const AdamwTensor& tensor, long long from, const Factors& F) {
  const long long end = from + P.piece < tensor.n ? from + P.piece : tensor.n;
  for (long long base = from; base < end; base += THREADS * EACH) {
    const long long at = base + threadIdx.x * EACH;
    if (base + THREADS * EACH <= end)
      update<T, BITS, true>(P, tensor, at, EACH, true, F);
    else  // (16 lanes behind the tensor's last block have no scales)
      update<T, BITS, false>(P, tensor, at, at < end ? (int)(end - at < EACH ? end - at : EACH) : 0, at - (threadIdx.x & 15) * EACH < end, F);
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
  const long long t = P.step_dev ? P.step_dev[tensor.step] : tensor.step;
  const double lr = P.lr_dev ? (double)*P.lr_dev : P.lr;
  Factors F;
  F.keep = (float)(1. - lr * P.weight_decay);
  F.rate = (float)(lr / (1. - power(P.beta1, t)));
  F.root = (float)(1. / sqrt(1. - power(P.beta2, t)));
  F.shift = (unsigned)t * 0xB504F333u;
  if (tensor.type == NNA_F32)
    update_piece<float, BITS>(P, tensor, from, F);
  else if (tensor.type == NNA_BF16)
    update_piece<bf16, BITS>(P, tensor, from, F);
  else
    update_piece<f16, BITS>(P, tensor, from, F);
}

template <bool SECOND_ONE>
__global__ __launch_bounds__(THREADS) void moment_kernel(const void* codes, const float* scales, long long blocks, float* out) {
  for (long long at = (long long)blockIdx.x * THREADS + threadIdx.x; at < blocks * (ADAMW_BLOCK / EACH); at += (long long)gridDim.x * THREADS) {
    const double scale = scales[at / (ADAMW_BLOCK / EACH)];
    float v[EACH];
    if constexpr (SECOND_ONE) {
      const Values<unsigned char> c = load_some<true>(static_cast<const unsigned char*>(codes) + at * EACH, EACH);
#pragma unroll
      for (int i = 0; i < EACH; ++i) v[i] = (float)second_value(c.v[i], scale);
    } else {
      const auto c = load_some<true>(static_cast<const signed char*>(codes) + at * EACH, EACH);
#pragma unroll
      for (int i = 0; i < EACH; ++i) v[i] = (float)first_value(c.v[i], scale);
    }
    store_some<true>(out + at * EACH, EACH, v);
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
