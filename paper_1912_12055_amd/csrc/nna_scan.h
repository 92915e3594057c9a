// Parameters of the gated recurrence's kernels (nna_kernels_scan.hip), and their launches.
#pragma once

#include "nna_internal.h"

namespace nna {

constexpr int SCAN_KEPT = 64;  // frames from one kept state to the next

// h_t = a_t h_{t-1} + u_t x_t along the frames, a = sigmoid(f), u = sigmoid(i), without i: u = 1 - a
struct ScanParams {
  const void *x, *f, *i;           // [B, T, C], a frame's channels next to each other; i or NULL
  long long x_b, x_t, f_b, f_t, i_b, i_t;
  const int* lengths;              // [B] or NULL: T
  const float* first;              // [B, C] or NULL: zero
  float* last;                     // [B, C] or NULL
  float* kept;                     // [B][ceil(T / SCAN_KEPT)][C]: the states before those frames (forward: or NULL)
  void* out;                       // [B, T, C]
  // backward
  const void* g;                   // [B, T, C]
  const float* glast;              // [B, C] or NULL: zero
  void *gx, *gf, *gi;              // [B, T, C]; gi with i
  float* gfirst;                   // [B, C] or NULL
  float* parts;                    // scan_workspace bytes
  long long B;
  int T, C;
  int segments, segment_frames;    // the launch's
};

struct ScanStep {
  const void *x, *f, *i;           // [B, C]
  long long x_b, f_b, i_b;
  float* state;                    // [B, C], updated
  void* out;                       // [B, C]
  long long B;
  int C;
};

// bytes of `parts`: none where a workgroup takes a sequence from its first frame to its last
size_t scan_workspace(long long B, long long T, long long C);
hipError_t launch_scan(ScanParams P, int type, hipStream_t stream);
hipError_t launch_scan_backward(ScanParams P, int type, hipStream_t stream);
hipError_t launch_scan_step(const ScanStep& P, int type, hipStream_t stream);

}  // namespace nna
