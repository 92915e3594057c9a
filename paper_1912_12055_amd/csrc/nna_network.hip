// Further operators of networks on the frames (C ABI): heads normalised and rotated, the gated recurrence, the optimiser's step.  Argument checks, shapes, launches.
#include "nna_adamw.h"
#include "nna_host.h"
#include "nna_rotate.h"
#include "nna_scan.h"

using namespace nna;
using namespace nna::host;

namespace {

bool known_type(int t) { return t == NNA_F32 || t == NNA_BF16 || t == NNA_F16; }

nna_status enter_device(DeviceGuard& guard, int device) {
  if (device < 0) return fail(NNA_ERR_INVALID_ARG, "device must be the HIP device of the arrays");
  const hipError_t e = guard.enter(device);  // (refuses a device that there is not)
  return e == hipSuccess ? NNA_OK : fail_hip(e, "hipSetDevice");
}

// An output over an input is written while other workgroups still read: refused where the pointers are equal (what overlaps otherwise is the caller's to see to).
nna_status refuse_same(std::initializer_list<const void*> outputs, std::initializer_list<const void*> inputs) {
  for (const void* o : outputs)
    for (const void* i : inputs)
      if (o && o == i) return fail(NNA_ERR_INVALID_ARG, "an output must not be an input of the call");
  return NNA_OK;
}

// ---- heads normalised and rotated ----

nna_status check_rotate(int type, long long B, long long T, long long q_heads, long long k_heads, long long width, long long pairs) {
  if (!known_type(type)) return fail(NNA_ERR_INVALID_ARG, "unknown nna_dtype");
  if (B < 0 || T < 0 || q_heads < 1 || k_heads < 0 || width < 1) return fail(NNA_ERR_SHAPE, "B, T and k_heads must not be negative, q_heads and width at least 1");
  if (width > ROTATE_HEAD_MAX) return fail(NNA_ERR_UNSUPPORTED, "heads of more than " + std::to_string(ROTATE_HEAD_MAX) + " values");
  if (pairs < 0 || 2 * pairs > width) return fail(NNA_ERR_SHAPE, "pairs must not be negative, nor more than a head holds");
  if (q_heads > 65536 || k_heads > 65536 || T > INT_MAX - 65536 || (T && B > (1LL << 40) / T)) return fail(NNA_ERR_SHAPE, "too many heads or frames");
  return NNA_OK;
}

nna_status check_rotate_args(const double* freqs, long long pairs, const int* positions, const long long* positions_strides, long long offset, int norm, double eps,
                             const void* q_weight, const void* k_weight) {
  if (pairs && !freqs) return fail(NNA_ERR_INVALID_ARG, "freqs_dev is NULL");
  if (positions && !positions_strides) return fail(NNA_ERR_INVALID_ARG, "positions_strides is NULL");
  if (offset > (1LL << 52) || offset < -(1LL << 52)) return fail(NNA_ERR_INVALID_ARG, "offset is too large");
  if (norm && (!(eps >= 0.0) || eps > 3.0e38)) return fail(NNA_ERR_INVALID_ARG, "eps must be finite and not negative");
  if (!norm && (q_weight || k_weight)) return fail(NNA_ERR_INVALID_ARG, "weights are the norm's: there is none");
  return NNA_OK;
}

RotateParams rotate_params(long long B, long long T, long long width, long long pairs, const double* freqs, const int* positions, const long long* positions_strides,
                           long long offset, int interleaved, int norm, double eps) {
  RotateParams P = {};
  P.freqs = freqs;
  P.positions = positions;
  if (positions) {
    P.p_b = positions_strides[0];
    P.p_t = positions_strides[1];
  }
  P.offset = offset;
  P.B = B;
  P.T = T;
  P.width = (int)width;
  P.pairs = (int)pairs;
  P.interleaved = interleaved != 0;
  P.norm = norm != 0;
  P.eps = (float)eps;
  return P;
}

RotateHeads rotate_heads(const void* x, const long long* strides, long long heads, const float* weight, void* y, const void* g) {
  RotateHeads H = {};
  H.heads = (int)heads;
  if (!heads) return H;
  H.inverse = ((1ULL << 32) + heads - 1) / heads;
  H.x = x;
  if (strides) {
    H.x_b = strides[0];
    H.x_t = strides[1];
    H.x_h = strides[2];
  }
  H.weight = weight;
  H.y = y;
  H.g = g;
  return H;
}

size_t rotate_workspace(long long B, long long T, long long width) { return (size_t)std::max(1LL, std::min(B * T, (long long)ROTATE_GROUPS)) * 2 * width * sizeof(float); }

// ---- the gated recurrence ----

nna_status check_scan(int type, long long B, long long T, long long C) {
  if (!known_type(type)) return fail(NNA_ERR_INVALID_ARG, "unknown nna_dtype");
  if (B < 0 || T < 0 || C < 1) return fail(NNA_ERR_SHAPE, "B and T must not be negative, C at least 1");
  // (groups of 32 channels times the 512 lanes of their workgroups are less than 2^32 in a launch)
  if (C > (1 << 27) || B > (1LL << 21) / ((C + 63) / 64)) return fail(NNA_ERR_SHAPE, "B C is too large");
  if (T > INT_MAX - 65536) return fail(NNA_ERR_SHAPE, "T is too large");
  return NNA_OK;
}

nna_status check_scan_strides(std::initializer_list<const long long*> strides) {
  for (const long long* s : strides)
    if (!s) return fail(NNA_ERR_INVALID_ARG, "strides are NULL");
  return NNA_OK;
}

nna_status check_scan_workspace(const void* workspace, size_t bytes, size_t need) {
  if (need && (!workspace || (reinterpret_cast<uintptr_t>(workspace) & 255) || bytes < need))
    return fail(NNA_ERR_INVALID_ARG, "workspace_dev is NULL, misaligned or smaller than the call's _workspace function asks for");
  return NNA_OK;
}

// ---- the optimiser's step ----

struct Span {
  uintptr_t from, to;
  bool operator<(const Span& o) const { return from < o.from; }
};
Span span_of(const void* p, long long bytes) { return {reinterpret_cast<uintptr_t>(p), reinterpret_cast<uintptr_t>(p) + (uintptr_t)bytes}; }
// sorts them
bool disjoint(std::vector<Span>& spans) {
  if (!std::is_sorted(spans.begin(), spans.end())) std::sort(spans.begin(), spans.end());
  for (size_t i = 1; i < spans.size(); ++i)
    if (spans[i].from < spans[i - 1].to) return false;
  return true;
}
// whether one shares memory with a span of `others`, which disjoint() has sorted
bool meets(const Span& s, const std::vector<Span>& others) {
  const auto behind = std::lower_bound(others.begin(), others.end(), Span{s.to, s.to});
  return behind != others.begin() && (behind - 1)->to > s.from;
}

struct AdamwCall {
  void* const* p;
  const void* const* g;
  const long long* n;
  const int* types;
  long long count;
  void *m, *v;
  float *m_scales, *v_scales, *master;
  long long state_size;
  const long long *steps, *steps_dev;
  int apart;
  double lr;
  const float* lr_dev;
  double beta1, beta2, eps, weight_decay;
};

// What a workgroup writes no other one may read or write: weights, states, and (states_too, of gradients) what is read beside them.  The states are taken whole first, `size` values of each,
// and if that fails (`closely`) tensor by tensor, as they are written: those without a gradient are not, nor copies of float32 tensors, whose weights may lie there.
nna_status refuse_shared(const AdamwCall& c, long long size, bool states_too, bool closely) {
  std::vector<Span> weights, all, grads;
  weights.reserve((size_t)c.count);
  grads.reserve((size_t)c.count);
  for (long long i = 0; i < c.count; ++i) {
    if (!c.n[i] || !c.g[i]) continue;
    const long long bytes = c.n[i] * (c.types[i] == NNA_F32 ? 4 : 2);
    weights.push_back(span_of(c.p[i], bytes));
    grads.push_back(span_of(c.g[i], bytes));
  }
  if (!disjoint(weights)) return fail(NNA_ERR_INVALID_ARG, "two tensors share memory");
  if (weights.empty()) return NNA_OK;
  all.reserve(weights.size() * (closely ? 6 : 1) + 5);
  all = weights;
  const long long value = c.m_scales ? 1 : 4;
  const auto states = [&](long long at, long long n, bool copied) {
    const long long block = at / ADAMW_BLOCK, blocks = (n + ADAMW_BLOCK - 1) / ADAMW_BLOCK;
    for (void* p : {c.m, c.v}) all.push_back(span_of(static_cast<char*>(p) + at * value, n * value));
    for (float* p : {c.m_scales, c.v_scales})
      if (p) all.push_back(span_of(p + block, blocks * 4));
    if (c.master && copied) all.push_back(span_of(c.master + at, n * 4));
  };
  if (closely) {
    long long at = 0;
    for (long long i = 0; i < c.count; ++i) {
      if (c.n[i] && c.g[i]) states(at, c.n[i], c.types[i] != NNA_F32);
      at += (c.n[i] + ADAMW_BLOCK - 1) / ADAMW_BLOCK * ADAMW_BLOCK;
    }
  } else {
    states(0, size, true);
  }
  if (!disjoint(all)) return fail(NNA_ERR_INVALID_ARG, "two of the states, or a state and a tensor, share memory");
  for (const Span& g : grads)
    if (meets(g, states_too ? all : weights)) return fail(NNA_ERR_INVALID_ARG, "a gradient shares memory with what the step writes");
  if (c.lr_dev && meets(span_of(c.lr_dev, 4), all)) return fail(NNA_ERR_INVALID_ARG, "lr_dev is in what the step writes");
  if (c.steps_dev && meets(span_of(c.steps_dev, (c.apart ? c.count : 1) * 8), all)) return fail(NNA_ERR_INVALID_ARG, "the numbers of steps are in what the step writes");
  return NNA_OK;
}

nna_status adamw(const AdamwCall& c, bool states_too, int device, void* hip_stream) {
  if (c.count < 0 || c.state_size < 0 || (c.count && (!c.p || !c.g || !c.n || !c.types))) return fail(NNA_ERR_INVALID_ARG, "count or state_size is negative, or an array is NULL");
  if (!c.m_scales != !c.v_scales) return fail(NNA_ERR_INVALID_ARG, "m_scales_dev and v_scales_dev come together");
  if (c.apart != 0 && c.apart != 1) return fail(NNA_ERR_INVALID_ARG, "apart is 0 (one number of steps for all tensors) or 1 (each its own)");
  if (!c.steps && !c.steps_dev && (c.count || !c.apart)) return fail(NNA_ERR_INVALID_ARG, "steps is NULL");
  const auto step_of = [&](long long i) { return c.steps_dev ? i * c.apart : c.steps[i * c.apart]; };  // ... or where it is
  if (!c.steps_dev && !c.apart && c.steps[0] < 1) return fail(NNA_ERR_INVALID_ARG, "steps count from 1");
  if (!(c.beta1 >= 0.0 && c.beta1 < 1.0 && c.beta2 >= 0.0 && c.beta2 < 1.0)) return fail(NNA_ERR_INVALID_ARG, "beta1 and beta2 must be in [0, 1)");
  if (!(c.eps >= 0.0) || c.eps > 3.0e38) return fail(NNA_ERR_INVALID_ARG, "eps must be finite and not negative");
  if ((!c.lr_dev && !(std::fabs(c.lr) < 1e30)) || !(std::fabs(c.weight_decay) < 1e30)) return fail(NNA_ERR_INVALID_ARG, "lr and weight_decay must be finite");
  long long size = 0, values = 0;
  for (long long i = 0; i < c.count; ++i) {
    if (!known_type(c.types[i])) return fail(NNA_ERR_INVALID_ARG, "unknown nna_dtype");
    if (c.n[i] < 0 || c.n[i] > (1LL << 36)) return fail(NNA_ERR_SHAPE, "a tensor's number of values is negative or too large");
    size += (c.n[i] + ADAMW_BLOCK - 1) / ADAMW_BLOCK * ADAMW_BLOCK;
    if (size > c.state_size) return fail(NNA_ERR_INVALID_ARG, "a tensor's state ends behind state_size");
    if (!c.n[i] || !c.g[i]) continue;
    if (!c.steps_dev && step_of(i) < 1) return fail(NNA_ERR_INVALID_ARG, "steps count from 1");
    if (!c.p[i] || c.p[i] == c.g[i]) return fail(NNA_ERR_INVALID_ARG, "a tensor is NULL, or its own gradient");
    values += c.n[i];
  }
  if (values && (!c.m || !c.v)) return fail(NNA_ERR_INVALID_ARG, "m_dev or v_dev is NULL");
  const void* states[] = {c.m, c.v, c.m_scales, c.v_scales, c.master};
  for (const void*& a : states)
    for (const void*& b : states)
      if (values && a && &a != &b && a == b) return fail(NNA_ERR_INVALID_ARG, "two of the states are the same");
  try {
    if (refuse_shared(c, size, states_too, false) != NNA_OK) {
      const nna_status shared = refuse_shared(c, size, states_too, true);
      if (shared != NNA_OK) return shared;
    }
  } catch (const std::exception&) {
    return fail(NNA_ERR_ALLOC, "out of host memory");
  }
  DeviceGuard guard;
  const nna_status s = enter_device(guard, device);
  if (s != NNA_OK || !values) return s;
  AdamwParams P;
  P.m = c.m;
  P.v = c.v;
  P.m_scales = c.m_scales;
  P.v_scales = c.v_scales;
  P.master = c.master;
  P.beta1 = c.beta1;
  P.beta2 = c.beta2;
  P.step_dev = c.steps_dev;
  P.lr_dev = c.lr_dev;
  P.lr = c.lr;
  P.weight_decay = c.weight_decay;
  // (the quotient's reciprocal takes no float32 below the normal ones: beside a root that is not zero an eps as small is nothing, and beside one that is, nothing over it stays nothing)
  P.eps = c.eps > 0.0 ? std::max((float)c.eps, 0x1p-126f) : 0.f;
  P.piece = adamw_piece(values);
  P.count = P.pieces = 0;
  long long at = 0;
  for (long long i = 0; i < c.count; ++i) {
    const long long pieces = c.g[i] ? (c.n[i] + P.piece - 1) / P.piece : 0;
    if (pieces) {
      // (threads of a launch are counted in 32 bits)
      if (P.count == ADAMW_TENSORS || (P.count && P.pieces + pieces >= 1LL << 24)) {
        const hipError_t e = launch_adamw(P, static_cast<hipStream_t>(hip_stream));
        if (e != hipSuccess) return fail_hip(e, "nna_adamw");
        P.count = P.pieces = 0;
      }
      P.tensors[P.count++] = {c.p[i], c.g[i], c.n[i], at, step_of(i), P.pieces, c.types[i]};
      P.pieces += (int)pieces;
    }
    at += (c.n[i] + ADAMW_BLOCK - 1) / ADAMW_BLOCK * ADAMW_BLOCK;
  }
  const hipError_t e = launch_adamw(P, static_cast<hipStream_t>(hip_stream));  // (there is a tensor: a launch is left to do, since one before it made room for the next)
  return e == hipSuccess ? NNA_OK : fail_hip(e, "nna_adamw");
}

}  // namespace

extern "C" {

nna_status nna_rotate_heads(const void* q_dev, const long long* q_strides, long long q_heads, const void* k_dev, const long long* k_strides, long long k_heads,
                            nna_dtype type, long long B, long long T, long long width, const double* freqs_dev, long long pairs, int interleaved,
                            const int* positions_dev, const long long* positions_strides, long long offset, int norm, double eps, const float* q_weight_dev,
                            const float* k_weight_dev, void* q_out_dev, void* k_out_dev, int device, void* hip_stream) {
  nna_status s = check_rotate(type, B, T, q_heads, k_heads, width, pairs);
  if (s == NNA_OK) s = check_rotate_args(freqs_dev, pairs, positions_dev, positions_strides, offset, norm, eps, q_weight_dev, k_weight_dev);
  if (s != NNA_OK) return s;
  if (!q_strides || (k_heads && !k_strides)) return fail(NNA_ERR_INVALID_ARG, "strides are NULL");
  const bool some = B && T;
  if (some && (!q_dev || !q_out_dev)) return fail(NNA_ERR_INVALID_ARG, "q_dev / q_out_dev is NULL");
  if (some && k_heads && (!k_dev || !k_out_dev)) return fail(NNA_ERR_INVALID_ARG, "k_dev / k_out_dev is NULL");
  if (q_out_dev && k_heads && q_out_dev == k_out_dev) return fail(NNA_ERR_INVALID_ARG, "q_out_dev and k_out_dev are the same");
  RotateParams P = rotate_params(B, T, width, pairs, freqs_dev, positions_dev, positions_strides, offset, interleaved, norm, eps);
  P.q = rotate_heads(q_dev, q_strides, q_heads, q_weight_dev, q_out_dev, nullptr);
  P.k = rotate_heads(k_dev, k_strides, k_heads, k_weight_dev, k_out_dev, nullptr);
  DeviceGuard guard;
  s = enter_device(guard, device);
  if (s == NNA_OK) s = refuse_same({P.q.y, P.k.y}, {P.q.x, P.k.x, freqs_dev, positions_dev, q_weight_dev, k_weight_dev});
  if (s != NNA_OK || !some) return s;
  const hipError_t e = launch_rotate(P, type, static_cast<hipStream_t>(hip_stream));
  return e == hipSuccess ? NNA_OK : fail_hip(e, "nna_rotate_heads");
}

nna_status nna_rotate_heads_backward_workspace(long long B, long long T, long long width, size_t* bytes) {
  if (!bytes) return fail(NNA_ERR_INVALID_ARG, "bytes is NULL");
  const nna_status s = check_rotate(NNA_F32, B, T, 1, 0, width, 0);
  if (s == NNA_OK) *bytes = rotate_workspace(B, T, width);
  return s;
}

nna_status nna_rotate_heads_backward(const void* gq_out_dev, const void* gk_out_dev, const void* q_dev, const long long* q_strides, long long q_heads, const void* k_dev,
                                     const long long* k_strides, long long k_heads, nna_dtype type, long long B, long long T, long long width, const double* freqs_dev,
                                     long long pairs, int interleaved, const int* positions_dev, const long long* positions_strides, long long offset, int norm,
                                     double eps, const float* q_weight_dev, const float* k_weight_dev, void* gq_dev, void* gk_dev, float* gq_weight_dev,
                                     float* gk_weight_dev, void* workspace_dev, size_t workspace_bytes, int device, void* hip_stream) {
  nna_status s = check_rotate(type, B, T, q_heads, k_heads, width, pairs);
  if (s == NNA_OK) s = check_rotate_args(freqs_dev, pairs, positions_dev, positions_strides, offset, norm, eps, q_weight_dev, k_weight_dev);
  if (s != NNA_OK) return s;
  const bool some = B && T;
  if (norm && (!q_strides || (k_heads && !k_strides))) return fail(NNA_ERR_INVALID_ARG, "strides are NULL");
  if (some && (!gq_out_dev || !gq_dev || (norm && !q_dev))) return fail(NNA_ERR_INVALID_ARG, "gq_out_dev / gq_dev / q_dev is NULL");
  if (some && k_heads && (!gk_out_dev || !gk_dev || (norm && !k_dev))) return fail(NNA_ERR_INVALID_ARG, "gk_out_dev / gk_dev / k_dev is NULL");
  if (!norm && (gq_weight_dev || gk_weight_dev)) return fail(NNA_ERR_INVALID_ARG, "weights are the norm's: there is none");
  if (gk_weight_dev && !k_heads) return fail(NNA_ERR_INVALID_ARG, "gk_weight_dev without keys");
  if (k_heads && gq_dev && gq_dev == gk_dev) return fail(NNA_ERR_INVALID_ARG, "gq_dev and gk_dev are the same");
  RotateParams P = rotate_params(B, T, width, pairs, freqs_dev, positions_dev, positions_strides, offset, interleaved, norm, eps);
  P.q = rotate_heads(q_dev, q_strides, q_heads, q_weight_dev, gq_dev, gq_out_dev);
  P.k = rotate_heads(k_dev, k_strides, k_heads, k_weight_dev, gk_dev, gk_out_dev);
  if (gq_weight_dev || gk_weight_dev) {
    if (!workspace_dev || (reinterpret_cast<uintptr_t>(workspace_dev) & 15) || workspace_bytes < rotate_workspace(B, T, width))
      return fail(NNA_ERR_INVALID_ARG, "workspace_dev is NULL, misaligned or smaller than nna_rotate_heads_backward_workspace asks for");
    P.partial = static_cast<float*>(workspace_dev);
  }
  DeviceGuard guard;
  s = enter_device(guard, device);
  if (s == NNA_OK) s = refuse_same({P.q.y, P.k.y}, {P.q.x, P.k.x, P.q.g, P.k.g, freqs_dev, positions_dev, q_weight_dev, k_weight_dev});
  if (s != NNA_OK || (!some && !P.partial)) return s;
  const hipError_t e = launch_rotate_backward(P, type, gq_weight_dev, gk_weight_dev, static_cast<hipStream_t>(hip_stream));
  return e == hipSuccess ? NNA_OK : fail_hip(e, "nna_rotate_heads_backward");
}

nna_status nna_gated_scan_workspace(long long B, long long T, long long C, size_t* bytes) {
  if (!bytes) return fail(NNA_ERR_INVALID_ARG, "bytes is NULL");
  const nna_status s = check_scan(NNA_F32, B, T, C);
  if (s == NNA_OK) *bytes = scan_workspace(B, T, C);
  return s;
}

nna_status nna_gated_scan(const void* x_dev, const long long* x_strides, const void* forget_dev, const long long* forget_strides, const void* input_dev,
                          const long long* input_strides, nna_dtype type, long long B, long long T, long long C, const int* lengths_dev, const float* first_dev,
                          float* last_dev, void* out_dev, float* kept_dev, void* workspace_dev, size_t workspace_bytes, int device, void* hip_stream) {
  nna_status s = check_scan(type, B, T, C);
  if (s == NNA_OK) s = check_scan_strides({x_strides, forget_strides, input_dev ? input_strides : x_strides});
  if (s != NNA_OK) return s;
  if (B && T && (!x_dev || !forget_dev || !out_dev)) return fail(NNA_ERR_INVALID_ARG, "x_dev / forget_dev / out_dev is NULL");
  s = check_scan_workspace(workspace_dev, workspace_bytes, scan_workspace(B, T, C));
  if (s != NNA_OK) return s;
  ScanParams P = {};
  P.x = x_dev;
  P.x_b = x_strides[0];
  P.x_t = x_strides[1];
  P.f = forget_dev;
  P.f_b = forget_strides[0];
  P.f_t = forget_strides[1];
  if (input_dev) {
    P.i = input_dev;
    P.i_b = input_strides[0];
    P.i_t = input_strides[1];
  }
  P.lengths = lengths_dev;
  P.first = first_dev;
  P.last = last_dev;
  P.kept = kept_dev;
  P.out = out_dev;
  P.parts = static_cast<float*>(workspace_dev);
  P.B = B;
  P.T = (int)T;
  P.C = (int)C;
  DeviceGuard guard;
  s = enter_device(guard, device);
  if (s == NNA_OK) s = refuse_same({out_dev, last_dev, kept_dev}, {x_dev, forget_dev, input_dev, first_dev, lengths_dev});
  if (s != NNA_OK || !B || (!T && !last_dev)) return s;
  const hipError_t e = launch_scan(P, type, static_cast<hipStream_t>(hip_stream));
  return e == hipSuccess ? NNA_OK : fail_hip(e, "nna_gated_scan");
}

nna_status nna_gated_scan_backward(const void* gout_dev, const float* kept_dev, const void* x_dev, const long long* x_strides, const void* forget_dev,
                                   const long long* forget_strides, const void* input_dev, const long long* input_strides, nna_dtype type, long long B, long long T,
                                   long long C, const int* lengths_dev, const float* glast_dev, void* gx_dev, void* gforget_dev, void* ginput_dev, float* gfirst_dev,
                                   void* workspace_dev, size_t workspace_bytes, int device, void* hip_stream) {
  nna_status s = check_scan(type, B, T, C);
  if (s == NNA_OK) s = check_scan_strides({x_strides, forget_strides, input_dev ? input_strides : x_strides});
  if (s != NNA_OK) return s;
  if (B && T && (!gout_dev || !kept_dev || !x_dev || !forget_dev)) return fail(NNA_ERR_INVALID_ARG, "gout_dev / kept_dev / x_dev / forget_dev is NULL");
  if (B && T && (!gx_dev || !gforget_dev || !ginput_dev != !input_dev))
    return fail(NNA_ERR_INVALID_ARG, "gx_dev / gforget_dev is NULL, or ginput_dev and input_dev do not come together");
  s = check_scan_workspace(workspace_dev, workspace_bytes, scan_workspace(B, T, C));
  if (s != NNA_OK) return s;
  ScanParams P = {};
  P.x = x_dev;
  P.x_b = x_strides[0];
  P.x_t = x_strides[1];
  P.f = forget_dev;
  P.f_b = forget_strides[0];
  P.f_t = forget_strides[1];
  if (input_dev) {
    P.i = input_dev;
    P.i_b = input_strides[0];
    P.i_t = input_strides[1];
  }
  P.lengths = lengths_dev;
  P.kept = const_cast<float*>(kept_dev);
  P.g = gout_dev;
  P.glast = glast_dev;
  P.gx = gx_dev;
  P.gf = gforget_dev;
  P.gi = ginput_dev;
  P.gfirst = gfirst_dev;
  P.parts = static_cast<float*>(workspace_dev);
  P.B = B;
  P.T = (int)T;
  P.C = (int)C;
  DeviceGuard guard;
  s = enter_device(guard, device);
  if (s == NNA_OK) s = refuse_same({gx_dev, gforget_dev, ginput_dev, gfirst_dev}, {gout_dev, kept_dev, x_dev, forget_dev, input_dev, glast_dev, lengths_dev});
  if (s != NNA_OK || !B || (!T && !gfirst_dev)) return s;
  if (gx_dev && (gx_dev == gforget_dev || gx_dev == ginput_dev || (ginput_dev && ginput_dev == gforget_dev)))
    return fail(NNA_ERR_INVALID_ARG, "two outputs are the same");
  const hipError_t e = launch_scan_backward(P, type, static_cast<hipStream_t>(hip_stream));
  return e == hipSuccess ? NNA_OK : fail_hip(e, "nna_gated_scan_backward");
}

nna_status nna_gated_scan_step(const void* x_dev, long long x_stride, const void* forget_dev, long long forget_stride, const void* input_dev, long long input_stride,
                               nna_dtype type, long long B, long long C, float* state_dev, void* out_dev, int device, void* hip_stream) {
  nna_status s = check_scan(type, B, 1, C);
  if (s != NNA_OK) return s;
  if (B && (!x_dev || !forget_dev || !state_dev || !out_dev)) return fail(NNA_ERR_INVALID_ARG, "x_dev / forget_dev / state_dev / out_dev is NULL");
  ScanStep P = {x_dev, forget_dev, input_dev, x_stride, forget_stride, input_stride, state_dev, out_dev, B, (int)C};
  DeviceGuard guard;
  s = enter_device(guard, device);
  if (s == NNA_OK) s = refuse_same({out_dev, state_dev}, {x_dev, forget_dev, input_dev});
  if (s == NNA_OK) s = refuse_same({out_dev}, {state_dev});
  if (s != NNA_OK || !B) return s;
  const hipError_t e = launch_scan_step(P, type, static_cast<hipStream_t>(hip_stream));
  return e == hipSuccess ? NNA_OK : fail_hip(e, "nna_gated_scan_step");
}

nna_status nna_adamw(void* const* p_dev, const void* const* g_dev, const long long* n, const int* types, long long count, void* m_dev, void* v_dev, float* m_scales_dev,
                     float* v_scales_dev, float* master_dev, long long state_size, long long step, const long long* step_dev, double lr, const float* lr_dev, double beta1,
                     double beta2, double eps, double weight_decay, int device, void* hip_stream) {
  return adamw({p_dev, g_dev, n, types, count, m_dev, v_dev, m_scales_dev, v_scales_dev, master_dev, state_size, &step, step_dev, 0, lr, lr_dev, beta1, beta2, eps, weight_decay}, false,
               device, hip_stream);
}

nna_status nna_adamw_steps(void* const* p_dev, const void* const* g_dev, const long long* n, const int* types, long long count, void* m_dev, void* v_dev, float* m_scales_dev,
                           float* v_scales_dev, float* master_dev, long long state_size, const long long* steps, const long long* steps_dev, int apart, double lr,
                           const float* lr_dev, double beta1, double beta2, double eps, double weight_decay, int device, void* hip_stream) {
  return adamw({p_dev, g_dev, n, types, count, m_dev, v_dev, m_scales_dev, v_scales_dev, master_dev, state_size, steps, steps_dev, apart, lr, lr_dev, beta1, beta2, eps, weight_decay}, true,
               device, hip_stream);
}

nna_status nna_adamw_moment(const void* codes_dev, int second, const float* scales_dev, long long size, float* out_dev, int device, void* hip_stream) {
  if (size < 0 || size % ADAMW_BLOCK) return fail(NNA_ERR_SHAPE, "size must be a multiple of 128");
  if (size && (!codes_dev || !scales_dev || !out_dev)) return fail(NNA_ERR_INVALID_ARG, "codes_dev / scales_dev / out_dev is NULL");
  DeviceGuard guard;
  nna_status s = enter_device(guard, device);
  if (s == NNA_OK) s = refuse_same({out_dev}, {codes_dev, scales_dev});
  if (s != NNA_OK || !size) return s;
  const hipError_t e = launch_adamw_moment(codes_dev, second != 0, scales_dev, size / ADAMW_BLOCK, out_dev, static_cast<hipStream_t>(hip_stream));
  return e == hipSuccess ? NNA_OK : fail_hip(e, "nna_adamw_moment");
}

}  // extern "C"
