// Parameters of the kernels that normalise and rotate heads (nna_kernels_rotate.hip), and their launches.
#pragma once

#include "nna_internal.h"

namespace nna {

constexpr int ROTATE_HEAD_MAX = 256;  // values of a head
constexpr int ROTATE_GROUPS = 512;    // backward: workgroups, at most, that leave a partial sum of each weight's gradient

struct RotateHeads {
  const void* x;                 // [B, T, heads, width], a head's values next to each other
  long long x_b, x_t, x_h;       // elements between batches, frames, heads
  const float* weight;           // [width] or NULL: ones
  void* y;                       // [B, T, heads, width]; backward: the gradient of x
  const void* g;                 // backward: [B, T, heads, width]
  int heads;                     // 0: none
  unsigned long long inverse;    // 2^32 / heads, rounded up
};

struct RotateParams {
  RotateHeads q, k;
  const double* freqs;           // [pairs] radians a position
  const int* positions;          // [B, T], p_b and p_t between them, or NULL: offset + t
  long long p_b, p_t, offset;
  long long B, T;
  long long first_token;         // of this launch
  int width, pairs;              // the first 2 * pairs values of a head are rotated
  int interleaved, norm;
  float eps;
  float* partial;                // backward: [workgroups][2][width] or NULL
};

int rotate_backward_groups(long long tokens, int heads, int width, int pairs, int type);
hipError_t launch_rotate(const RotateParams& P, int type, hipStream_t stream);
hipError_t launch_rotate_backward(const RotateParams& P, int type, float* gqw, float* gkw, hipStream_t stream);

}  // namespace nna
