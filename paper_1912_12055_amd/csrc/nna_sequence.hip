// The operators of networks on top of the transforms (C ABI): argument checks, shapes, launches.
#include "nna_decay.h"
#include "nna_host.h"
#include "nna_norm.h"

using namespace nna;
using namespace nna::host;

namespace {

// Kernels' set-up, once per device and at the first call that needs it: the transforms' users do not wait for it, nor those of one operator for the other's.
struct Setup {
  hipError_t (*const init)();
  std::mutex mutex;
  std::vector<char> done;
};
Setup norm_setup{nna::norm_kernels_init}, decay_setup{nna::decay_kernels_init};

// enters the device for a call without a plan, its kernels set up (pack and unpack: there is nothing to)
nna_status enter_device(DeviceGuard& guard, int device, Setup* setup) {
  if (device < 0) return fail(NNA_ERR_INVALID_ARG, "device must be the HIP device of the arrays");
  hipError_t e = guard.enter(device);  // (refuses a device that there is not)
  if (e != hipSuccess) return fail_hip(e, "hipSetDevice");
  if (!setup) return NNA_OK;
  try {
    std::lock_guard<std::mutex> lock(setup->mutex);
    if ((int)setup->done.size() <= device) setup->done.resize(device + 1, 0);
    if (setup->done[device]) return NNA_OK;
    e = setup->init();
    setup->done[device] = e == hipSuccess;
  } catch (const std::exception&) {
    return fail(NNA_ERR_ALLOC, "out of host memory while setting kernels up");
  }
  return e == hipSuccess ? NNA_OK : fail_hip(e, "kernel set-up");
}

// An output over an input is written while other workgroups still read: refused where the pointers are equal (what overlaps otherwise is the caller's to see to).
nna_status refuse_same(std::initializer_list<const void*> outputs, std::initializer_list<const void*> inputs) {
  for (const void* o : outputs)
    for (const void* i : inputs)
      if (o && o == i) return fail(NNA_ERR_INVALID_ARG, "an output must not be an input of the call");
  return NNA_OK;
}

bool known_type(int t) { return t == NNA_F32 || t == NNA_BF16 || t == NNA_F16; }

// rows (B x T frames) of `width` values
nna_status check_rows(long long rows, long long width, long long width_max) {
  if (rows < 0 || width < 1) return fail(NNA_ERR_SHAPE, "rows must not be negative, and width at least 1");
  if (width > width_max) return fail(NNA_ERR_UNSUPPORTED, "width " + std::to_string(width) + " is above " + std::to_string(width_max));
  if (rows > (1LL << 60) / width) return fail(NNA_ERR_SHAPE, "too many values");
  return NNA_OK;
}

nna_status check_frames(long long B, long long width, long long T) {
  if (B < 0 || T < 0) return fail(NNA_ERR_SHAPE, "B and T must not be negative");
  if (T && B > INT_MAX / ((T + 7) / 8)) return fail(NNA_ERR_SHAPE, "B T is too large");
  return check_rows(B * T, width, NORM_FRAMES_WIDTH_MAX);
}

nna_status check_norm_types(int x_type, int y_type) {
  if (!known_type(x_type) || !known_type(y_type)) return fail(NNA_ERR_INVALID_ARG, "unknown nna_dtype");
  if (x_type != y_type && x_type != NNA_F32) return fail(NNA_ERR_INVALID_ARG, "the outputs' type must be the inputs', or narrower than float32");
  return NNA_OK;
}

size_t norm_workspace(long long rows, int width, bool frames, long long B, long long T) {
  return (size_t)norm_backward_groups(rows, width, frames, B, T) * 2 * width * sizeof(float);
}

nna_status run_norm(NormParams& P, int x_type, int y_type, double eps, bool frames, int device, void* stream) {
  if (!(eps >= 0.0) || eps > 3.0e38) return fail(NNA_ERR_INVALID_ARG, "eps must be finite and not negative");
  if (P.rows && (!P.x || !P.y)) return fail(NNA_ERR_INVALID_ARG, "x_dev / y_dev is NULL");
  if (P.rows && !P.codes != !P.scales) return fail(NNA_ERR_INVALID_ARG, "codes_dev and scales_dev come together");
  if (P.codes && x_type != y_type) return fail(NNA_ERR_UNSUPPORTED, "8-bit codes need outputs of the inputs' type");
  P.eps = (float)eps;
  DeviceGuard guard;
  nna_status s = enter_device(guard, device, &norm_setup);
  // (every row where it was read, by the lanes that read it: y may be x)
  if (s == NNA_OK && (frames || x_type != y_type || (P.rows > 1 && P.row_stride != P.width))) s = refuse_same({P.y}, {P.x});
  if (s != NNA_OK || !P.rows) return s;
  const hipError_t e = launch_norm(P, x_type, y_type, frames, static_cast<hipStream_t>(stream));
  return e == hipSuccess ? NNA_OK : fail_hip(e, "layer norm");
}

nna_status run_norm_backward(NormParams& P, int x_type, int g_type, bool frames, float* gw, float* gb, void* workspace, size_t bytes, int device, void* stream) {
  if (!P.gx && !gw && !gb) return fail(NNA_ERR_INVALID_ARG, "no gradient is asked for");
  if (P.rows && (!P.gout || !P.stats)) return fail(NNA_ERR_INVALID_ARG, "gout_dev / stats_dev is NULL");
  if (P.rows && !P.codes != !P.scales) return fail(NNA_ERR_INVALID_ARG, "codes_dev and scales_dev come together");
  if (P.rows && !P.x == !P.codes) return fail(NNA_ERR_INVALID_ARG, "either x_dev or its codes");
  if (P.rows && P.gx && P.gx == P.x) return fail(NNA_ERR_INVALID_ARG, "gx_dev must not be x_dev");
  if (P.codes && x_type != g_type) return fail(NNA_ERR_UNSUPPORTED, "8-bit codes need outputs of the inputs' type");
  if (gw || gb) {
    if (!workspace || (reinterpret_cast<uintptr_t>(workspace) & 15) || bytes < norm_workspace(P.rows, P.width, frames, P.batch, P.T))
      return fail(NNA_ERR_INVALID_ARG, "workspace_dev is NULL, misaligned or smaller than nna_layer_norm_backward_workspace asks for");
    P.partial = static_cast<float*>(workspace);
  }
  DeviceGuard guard;
  nna_status s = enter_device(guard, device, &norm_setup);
  if (s == NNA_OK && (frames || x_type != g_type)) s = refuse_same({P.gx}, {P.gout});
  if (s != NNA_OK || (!P.rows && !P.partial)) return s;
  const hipError_t e = launch_norm_backward(P, x_type, g_type, frames, gw, gb, static_cast<hipStream_t>(stream));
  return e == hipSuccess ? NNA_OK : fail_hip(e, "layer norm, backward");
}

nna_status check_pack(int type, long long rows, long long width) {
  if (!known_type(type)) return fail(NNA_ERR_INVALID_ARG, "unknown nna_dtype");
  return check_rows(rows, width, 1LL << 60);
}

nna_status check_heads(int type, long long B, long long T, long long H, long long dk, long long dv) {
  if (!known_type(type)) return fail(NNA_ERR_INVALID_ARG, "unknown nna_dtype");
  if (type == NNA_F16) return fail(NNA_ERR_UNSUPPORTED, "float16 is not implemented here: float32 or bfloat16");
  if (B < 0 || T < 0 || H < 1 || dk < 1 || dv < 1) return fail(NNA_ERR_SHAPE, "B and T must not be negative, H, dk and dv at least 1");
  if (dk > DECAY_HEAD_MAX || dv > DECAY_HEAD_MAX) return fail(NNA_ERR_UNSUPPORTED, "heads of more than " + std::to_string(DECAY_HEAD_MAX) + " values");
  // (sequence, head)s times the lanes of their workgroups, up to four of 256 or one of 1,024, are less than 2^32 in a launch
  if (H > 65536 || B > (1LL << 21) / H) return fail(NNA_ERR_SHAPE, "H or B H is too large");
  if (T > INT_MAX - 4 * DECAY_CHUNK) return fail(NNA_ERR_SHAPE, "T is too large");
  return NNA_OK;
}

// bytes of the states before all segments, of either type
nna_status states_size(long long B, long long T, long long H, long long dk, long long dv, bool backward, size_t* bytes) {
  if (!bytes) return fail(NNA_ERR_INVALID_ARG, "bytes is NULL");
  const nna_status s = check_heads(NNA_F32, B, T, H, dk, dv);
  if (s != NNA_OK) return s;
  int segments, chunks;
  *bytes = 0;
  if (!B) return NNA_OK;
  *bytes = std::max(decay_segments(B, T, (int)H, (int)dk, (int)dv, NNA_F32, backward, &segments, &chunks),
                    decay_segments(B, T, (int)H, (int)dk, (int)dv, NNA_BF16, backward, &segments, &chunks));
  return NNA_OK;
}

nna_status check_decay_args(const void* decay, double scale, const void* workspace, size_t bytes, size_t need) {
  if (!decay) return fail(NNA_ERR_INVALID_ARG, "decay_dev is NULL");
  if (!(scale != 0.0) || !(std::fabs(scale) < 1e30) || !(std::fabs(scale) > 1e-30)) return fail(NNA_ERR_INVALID_ARG, "scale must be finite and not 0");
  if (need && (!workspace || (reinterpret_cast<uintptr_t>(workspace) & 255) || bytes < need))
    return fail(NNA_ERR_INVALID_ARG, "workspace_dev is NULL, misaligned or smaller than the call's _workspace function asks for");
  return NNA_OK;
}

nna_status check_strides(const long long* const (&strides)[3], long long T) {
  for (const long long* s : strides) {
    if (!s) return fail(NNA_ERR_INVALID_ARG, "strides are NULL");
    if (T <= 1) continue;  // (of one frame there is no next: the step is not taken, whatever it is)
    if (s[1] < 0 || s[1] > DECAY_STEP_MAX) return fail(NNA_ERR_SHAPE, "more than " + std::to_string(DECAY_STEP_MAX) + " elements from one frame to the next");
  }
  return NNA_OK;
}

// which array a mix reads in which place
struct Heads {
  const void* at;
  long long strides[3];
  int width;
};
Heads heads_of(const void* at, const long long* strides, long long width, long long T) { return {at, {strides[0], T > 1 ? strides[1] : 0, strides[2]}, (int)width}; }

void set_mix(DecayMix& P, const Heads& a, const Heads& b, const Heads& c) {
  P.a = a.at;
  P.a_b = a.strides[0];
  P.a_t = a.strides[1];
  P.a_h = a.strides[2];
  P.b = b.at;
  P.b_b = b.strides[0];
  P.b_t = b.strides[1];
  P.b_h = b.strides[2];
  P.c = c.at;
  P.c_b = c.strides[0];
  P.c_t = c.strides[1];
  P.c_h = c.strides[2];
  P.da = a.width;
  P.dc = c.width;
}
void set_pair(DecayMix& P, const Heads& a2, void* out2) {
  P.a2 = a2.at;
  P.a2_b = a2.strides[0];
  P.a2_t = a2.strides[1];
  P.a2_h = a2.strides[2];
  P.out2 = out2;
}

}  // namespace

extern "C" {

nna_status nna_layer_norm(const void* x_dev, nna_dtype x_type, long long rows, long long width, long long row_stride, const float* weight_dev,
                          const float* bias_dev, double eps, void* y_dev, nna_dtype y_type, float* stats_dev, signed char* codes_dev,
                          float* scales_dev, int device, void* hip_stream) {
  nna_status s = check_norm_types(x_type, y_type);
  if (s == NNA_OK) s = check_rows(rows, width, NORM_WIDTH_MAX);
  if (s != NNA_OK) return s;
  NormParams P = {};
  P.x = x_dev;
  P.rows = rows;
  P.row_stride = row_stride;
  P.width = (int)width;
  P.weight = weight_dev;
  P.bias = bias_dev;
  P.y = y_dev;
  P.stats = stats_dev;
  P.codes = codes_dev;
  P.scales = scales_dev;
  return run_norm(P, x_type, y_type, eps, false, device, hip_stream);
}

nna_status nna_layer_norm_frames(const float* x_dev, long long B, long long width, long long T, const float* weight_dev, const float* bias_dev,
                                 double eps, void* y_dev, nna_dtype y_type, float* stats_dev, int device, void* hip_stream) {
  nna_status s = check_norm_types(NNA_F32, y_type);
  if (s == NNA_OK) s = check_frames(B, width, T);
  if (s != NNA_OK) return s;
  NormParams P = {};
  P.x = x_dev;
  P.rows = B * T;
  P.batch = B;
  P.T = T;
  P.width = (int)width;
  P.weight = weight_dev;
  P.bias = bias_dev;
  P.y = y_dev;
  P.stats = stats_dev;
  return run_norm(P, NNA_F32, y_type, eps, true, device, hip_stream);
}

nna_status nna_layer_norm_backward_workspace(long long rows, long long width, long long B, long long T, size_t* bytes) {
  if (!bytes) return fail(NNA_ERR_INVALID_ARG, "bytes is NULL");
  nna_status s = B ? check_frames(B, width, T) : check_rows(rows, width, NORM_WIDTH_MAX);
  if (s != NNA_OK) return s;
  *bytes = norm_workspace(rows, (int)width, B != 0, B, T);
  return NNA_OK;
}

nna_status nna_layer_norm_backward(const void* gout_dev, nna_dtype gout_type, const void* x_dev, nna_dtype x_type, long long rows, long long width,
                                   long long row_stride, const signed char* codes_dev, const float* scales_dev, const float* stats_dev,
                                   const float* weight_dev, void* gx_dev, float* gw_dev, float* gb_dev, void* workspace_dev,
                                   size_t workspace_bytes, int device, void* hip_stream) {
  nna_status s = check_norm_types(x_type, gout_type);
  if (s == NNA_OK) s = check_rows(rows, width, NORM_WIDTH_MAX);
  if (s != NNA_OK) return s;
  NormParams P = {};
  P.x = x_dev;
  P.gout = gout_dev;
  P.rows = rows;
  P.row_stride = row_stride;
  P.width = (int)width;
  P.weight = weight_dev;
  P.gx = gx_dev;
  P.stats = const_cast<float*>(stats_dev);
  P.codes = const_cast<signed char*>(codes_dev);
  P.scales = const_cast<float*>(scales_dev);
  return run_norm_backward(P, x_type, gout_type, false, gw_dev, gb_dev, workspace_dev, workspace_bytes, device, hip_stream);
}

nna_status nna_layer_norm_frames_backward(const void* gout_dev, nna_dtype gout_type, const float* x_dev, long long B, long long width, long long T,
                                          const float* stats_dev, const float* weight_dev, float* gx_dev, float* gw_dev, float* gb_dev,
                                          void* workspace_dev, size_t workspace_bytes, int device, void* hip_stream) {
  nna_status s = check_norm_types(NNA_F32, gout_type);
  if (s == NNA_OK) s = check_frames(B, width, T);
  if (s != NNA_OK) return s;
  NormParams P = {};
  P.x = x_dev;
  P.gout = gout_dev;
  P.rows = B * T;
  P.batch = B;
  P.T = T;
  P.width = (int)width;
  P.weight = weight_dev;
  P.gx = gx_dev;
  P.stats = const_cast<float*>(stats_dev);
  return run_norm_backward(P, NNA_F32, gout_type, true, gw_dev, gb_dev, workspace_dev, workspace_bytes, device, hip_stream);
}

nna_status nna_pack8(const void* x_dev, nna_dtype type, long long rows, long long width, long long row_stride, signed char* codes_dev,
                     float* scales_dev, int device, void* hip_stream) {
  nna_status s = check_pack(type, rows, width);
  if (s != NNA_OK) return s;
  if (rows && (!x_dev || !codes_dev || !scales_dev)) return fail(NNA_ERR_INVALID_ARG, "x_dev / codes_dev / scales_dev is NULL");
  DeviceGuard guard;
  s = enter_device(guard, device, nullptr);
  if (s != NNA_OK || !rows) return s;
  const hipError_t e = launch_pack8(x_dev, type, rows, width, row_stride, codes_dev, scales_dev, static_cast<hipStream_t>(hip_stream));
  return e == hipSuccess ? NNA_OK : fail_hip(e, "nna_pack8");
}

nna_status nna_unpack8(const signed char* codes_dev, const float* scales_dev, long long rows, long long width, void* out_dev, nna_dtype type,
                       int device, void* hip_stream) {
  nna_status s = check_pack(type, rows, width);
  if (s != NNA_OK) return s;
  if (rows && (!out_dev || !codes_dev || !scales_dev)) return fail(NNA_ERR_INVALID_ARG, "out_dev / codes_dev / scales_dev is NULL");
  DeviceGuard guard;
  s = enter_device(guard, device, nullptr);
  if (s != NNA_OK || !rows) return s;
  const hipError_t e = launch_unpack8(codes_dev, scales_dev, rows, width, out_dev, type, static_cast<hipStream_t>(hip_stream));
  return e == hipSuccess ? NNA_OK : fail_hip(e, "nna_unpack8");
}

nna_status nna_decay_attention_workspace(long long B, long long T, long long H, long long dk, long long dv, size_t* bytes) {
  return states_size(B, T, H, dk, dv, false, bytes);
}

nna_status nna_decay_attention_backward_workspace(long long B, long long T, long long H, long long dk, long long dv, size_t* bytes) {
  const nna_status s = states_size(B, T, H, dk, dv, true, bytes);
  if (s == NNA_OK) *bytes *= 2;  // both directions' states
  return s;
}

nna_status nna_decay_attention(const void* q_dev, const long long* q_strides, const void* k_dev, const long long* k_strides, const void* v_dev,
                               const long long* v_strides, nna_dtype type, long long B, long long T, long long H, long long dk, long long dv,
                               const float* decay_dev, double scale, const int* lengths_dev, const float* first_dev, float* last_dev,
                               void* out_dev, void* workspace_dev, size_t workspace_bytes, int device, void* hip_stream) {
  nna_status s = check_heads(type, B, T, H, dk, dv);
  if (s != NNA_OK) return s;
  s = check_strides({q_strides, k_strides, v_strides}, T);
  if (s != NNA_OK) return s;
  if (B && T && (!q_dev || !k_dev || !v_dev || !out_dev)) return fail(NNA_ERR_INVALID_ARG, "q_dev / k_dev / v_dev / out_dev is NULL");
  DecayMix P = {};
  size_t need = 0;
  s = nna_decay_attention_workspace(B, T, H, dk, dv, &need);
  if (s == NNA_OK) s = check_decay_args(decay_dev, scale, workspace_dev, workspace_bytes, need);
  if (s != NNA_OK) return s;
  decay_segments(B, T, (int)H, (int)dk, (int)dv, type, false, &P.segments, &P.segment_chunks);
  set_mix(P, heads_of(q_dev, q_strides, dk, T), heads_of(k_dev, k_strides, dk, T), heads_of(v_dev, v_strides, dv, T));
  P.out = out_dev;
  P.decay = decay_dev;
  P.lengths = lengths_dev;
  P.first = first_dev;
  P.last = last_dev;
  P.parts = static_cast<float*>(workspace_dev);
  P.factor = (float)scale;
  P.first_factor = P.last_factor = 1.f;
  P.B = B;
  P.T = (int)T;
  P.H = (int)H;
  DeviceGuard guard;
  s = enter_device(guard, device, &decay_setup);
  if (s == NNA_OK) s = refuse_same({out_dev}, {q_dev, k_dev, v_dev, first_dev});
  if (s != NNA_OK || !B) return s;
  const hipStream_t stream = static_cast<hipStream_t>(hip_stream);
  const hipError_t e = launch_decay(P, type, stream);
  return e == hipSuccess ? NNA_OK : fail_hip(e, "linear attention");
}

nna_status nna_decay_attention_backward(const void* gout_dev, const void* q_dev, const long long* q_strides, const void* k_dev,
                                        const long long* k_strides, const void* v_dev, const long long* v_strides, nna_dtype type, long long B,
                                        long long T, long long H, long long dk, long long dv, const float* decay_dev, double scale,
                                        const int* lengths_dev, const float* first_dev, const float* glast_dev, void* gq_dev, void* gk_dev,
                                        void* gv_dev, float* gfirst_dev, void* workspace_dev, size_t workspace_bytes, int device, void* hip_stream) {
  nna_status s = check_heads(type, B, T, H, dk, dv);
  if (s != NNA_OK) return s;
  s = check_strides({q_strides, k_strides, v_strides}, T);
  if (s != NNA_OK) return s;
  if (B && T && (!gout_dev || !q_dev || !k_dev || !v_dev)) return fail(NNA_ERR_INVALID_ARG, "gout_dev / q_dev / k_dev / v_dev is NULL");
  if (B && T && (!gk_dev || !gv_dev)) return fail(NNA_ERR_INVALID_ARG, "gk_dev / gv_dev is NULL");
  DecayMix P = {};
  size_t need = 0;
  s = nna_decay_attention_backward_workspace(B, T, H, dk, dv, &need);
  if (s == NNA_OK) s = check_decay_args(decay_dev, scale, workspace_dev, workspace_bytes, need);
  if (s != NNA_OK) return s;
  decay_segments(B, T, (int)H, (int)dk, (int)dv, type, true, &P.segments, &P.segment_chunks);
  const long long packed[3] = {T * H * dv, H * dv, dv};
  const Heads q = heads_of(q_dev, q_strides, dk, T), k = heads_of(k_dev, k_strides, dk, T), v = heads_of(v_dev, v_strides, dv, T), g = heads_of(gout_dev, packed, dv, T);
  P.decay = decay_dev;
  P.lengths = lengths_dev;
  P.parts = static_cast<float*>(workspace_dev);
  P.factor = (float)scale;
  P.B = B;
  P.T = (int)T;
  P.H = (int)H;
  DeviceGuard guard;
  s = enter_device(guard, device, &decay_setup);
  if (s == NNA_OK) s = refuse_same({gq_dev, gk_dev, gv_dev, gfirst_dev}, {gout_dev, q_dev, k_dev, v_dev, first_dev, glast_dev});
  if (s != NNA_OK || !B) return s;
  const hipStream_t stream = static_cast<hipStream_t>(hip_stream);
  DecayMix states = P, gq = P, pair = P;
  set_mix(states, q, k, v);
  states.first = first_dev;
  states.first_factor = 1.f;
  set_mix(gq, g, v, k);  // on those states, transposed
  gq.first = first_dev;
  gq.first_factor = 1.f;
  gq.transposed = 1;
  gq.out = gq_dev;
  // the state's gradient, without q's scale: the outputs get it at the end, as gfirst does
  set_mix(pair, k, q, g);
  set_pair(pair, v, gk_dev);
  pair.out = gv_dev;
  pair.reverse = 1;
  pair.first = glast_dev;
  pair.first_factor = (float)(1.0 / scale);
  pair.last = gfirst_dev;
  pair.last_factor = (float)scale;
  pair.parts = P.parts + need / 2 / sizeof(float);
  if (!gq_dev && !gk_dev && !gfirst_dev) return NNA_OK;  // (no frames)
  const hipError_t e = launch_decay_gradients(states, gq, pair, type, stream);
  return e == hipSuccess ? NNA_OK : fail_hip(e, "linear attention, backward");
}

nna_status nna_decay_attention_step(const void* q_dev, const long long* q_strides, const void* k_dev, const long long* k_strides, const void* v_dev,
                                    const long long* v_strides, nna_dtype type, long long B, long long H, long long dk, long long dv,
                                    const float* decay_dev, double scale, float* state_dev, void* out_dev, int device, void* hip_stream) {
  nna_status s = check_heads(type, B, 1, H, dk, dv);
  if (s == NNA_OK) s = check_decay_args(decay_dev, scale, nullptr, 0, 0);
  if (s != NNA_OK) return s;
  if (!q_strides || !k_strides || !v_strides) return fail(NNA_ERR_INVALID_ARG, "strides are NULL");
  if (B && (!q_dev || !k_dev || !v_dev || !state_dev || !out_dev)) return fail(NNA_ERR_INVALID_ARG, "q_dev / k_dev / v_dev / state_dev / out_dev is NULL");
  DecayStep P = {};
  P.q = q_dev;
  P.k = k_dev;
  P.v = v_dev;
  P.q_b = q_strides[0];
  P.q_h = q_strides[1];
  P.k_b = k_strides[0];
  P.k_h = k_strides[1];
  P.v_b = v_strides[0];
  P.v_h = v_strides[1];
  P.out = out_dev;
  P.decay = decay_dev;
  P.state = state_dev;
  P.factor = (float)scale;
  P.B = B;
  P.H = (int)H;
  P.dk = (int)dk;
  P.dv = (int)dv;
  DeviceGuard guard;
  s = enter_device(guard, device, &decay_setup);
  if (s == NNA_OK) s = refuse_same({out_dev}, {q_dev, k_dev, v_dev, state_dev});
  if (s != NNA_OK || !B) return s;
  const hipError_t e = launch_decay_step(P, type, static_cast<hipStream_t>(hip_stream));
  return e == hipSuccess ? NNA_OK : fail_hip(e, "linear attention, one frame");
}

}  // extern "C"
