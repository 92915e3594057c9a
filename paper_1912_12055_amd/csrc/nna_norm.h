// Parameters of the layer-norm and 8-bit kernels (nna_kernels_norm.hip), and their launches.
#pragma once

#include "nna_internal.h"

namespace nna {

constexpr int NORM_BLOCK8 = 128;          // neighbours of a row that share a scale
constexpr int NORM_WIDTH_MAX = 16384;     // values of a row that a workgroup holds in registers
constexpr int NORM_FRAMES_WIDTH_MAX = 2112;  // ... of a frame, eight of which fit half a CU's LDS

struct NormParams {
  // forward: x -> y; backward: gout (and x or its codes) -> gx.  Rows of `width`; frames: x and gx are [batch, width, T]
  const void* x;
  const void* gout;
  long long rows, row_stride;  // elements between rows of x
  long long batch, T;          // frames only: rows = batch * T
  long long first_tile;        // frames, forward: of this launch
  int width;
  float eps;
  const float* weight;  // or NULL: ones
  const float* bias;    // or NULL: zeros
  void* y;
  void* gx;             // or NULL
  float* stats;         // [rows][2]: mean, 1 / sqrt(variance + eps); forward: or NULL
  signed char* codes;   // [rows][width], or NULL
  float* scales;        // [rows][ceil(width / NORM_BLOCK8)]
  float* partial;       // backward: [workgroups][2][width] or NULL
};

hipError_t norm_kernels_init();  // per device, before the first launch
// workgroups of the backward launch: each leaves one partial sum of the weight's and the bias's gradient
int norm_backward_groups(long long rows, int width, bool frames, long long batch, long long T);
hipError_t launch_norm(const NormParams& P, int x_type, int y_type, bool frames, hipStream_t stream);
hipError_t launch_norm_backward(const NormParams& P, int x_type, int g_type, bool frames, float* gw, float* gb, hipStream_t stream);
hipError_t launch_pack8(const void* x, int type, long long rows, long long width, long long row_stride, signed char* codes, float* scales, hipStream_t stream);
hipError_t launch_unpack8(const signed char* codes, const float* scales, long long rows, long long width, void* out, int type, hipStream_t stream);

}  // namespace nna
