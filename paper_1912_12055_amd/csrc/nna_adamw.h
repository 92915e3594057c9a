// Parameters of the optimiser's kernels (nna_kernels_adamw.hip), and their launches.
#pragma once

#include "nna_internal.h"

namespace nna {

constexpr int ADAMW_BLOCK = NNA_BLOCK8;  // values of a tensor that share a scale; tensors' states begin at multiples of it
constexpr int ADAMW_TENSORS = 80;        // of a launch: their table is among its arguments, which are 4 KB at most

struct AdamwTensor {
  void* p;
  const void* g;
  long long n, at;  // values, and where their states begin
  long long step;   // its number of steps with this one; with step_dev, where that is in it
  int first, type;  // the first of its pieces in the launch
};

struct AdamwParams {
  AdamwTensor tensors[ADAMW_TENSORS];
  int count, pieces;
  int piece;                     // values of a piece
  void *m, *v;                   // float32, or 8-bit codes with their scales
  float *m_scales, *v_scales;
  float* master;                 // float32 copies of 16-bit tensors, or NULL
  double beta1, beta2;
  const long long* step_dev;     // or NULL: the tensors' step
  const float* lr_dev;           // or NULL: lr
  double lr, weight_decay;
  float eps;
};

int adamw_piece(long long values);  // of a call's tensors together: values of a workgroup
hipError_t launch_adamw(const AdamwParams& P, hipStream_t stream);
hipError_t launch_adamw_moment(const void* codes, bool second, const float* scales, long long blocks, float* out, hipStream_t stream);

}  // namespace nna
