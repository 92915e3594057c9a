// Parameters of the linear-attention kernels (nna_kernels_decay.hip), and their launches.
#pragma once

#include "nna_internal.h"

namespace nna {

constexpr int DECAY_HEAD_MAX = 128;  // values of a head
constexpr int DECAY_CHUNK = 64;      // frames a workgroup takes at a time

// One mix of the frames: out_u = factor (sum over w <= u of decay^(u-w) (a_u . b_w) c_w + decay^(u+1) a_u S), S the state before the first;
// u counts the frames from the first, or (reverse) from the last one back, where the state's own exponent is one less.
struct DecayMix {
  const void *a, *b, *c;                 // [B, T, H, da], [.., da], [.., dc], a head's values next to each other
  long long a_b, a_t, a_h;               // elements between batches, frames, heads
  long long b_b, b_t, b_h;
  long long c_b, c_t, c_h;
  void* out;                             // [B, T, H, dc]
  const float* decay;                    // [H]
  const int* lengths;                    // [B] or NULL: T
  const float* first;                    // [B, H, da, dc] (transposed: [B, H, dc, da]) or NULL: zero
  float* last;                           // likewise, or NULL
  float* parts;                          // [B H][segments][padded da x dc]: each segment's own state, then the state before it
  float factor, first_factor, last_factor;
  int transposed;                        // first and last are [B, H, dc, da]
  long long B, T;
  int H, da, dc;
  int reverse;
  int segments, segment_chunks;
};

struct DecayStep {
  const void *q, *k, *v;                 // [B, H, dk], [B, H, dk], [B, H, dv]
  long long q_b, q_h, k_b, k_h, v_b, v_h;
  void* out;                             // [B, H, dv]
  const float* decay;
  float* state;                          // [B, H, dk, dv], updated
  float factor;
  long long B;
  int H, dk, dv;
};

// segments of a mix, chunks in each, and the bytes of `parts` (0 for one segment)
size_t decay_segments(long long B, long long T, int H, int da, int dc, int* segments, int* chunks);
hipError_t decay_kernels_init();  // per device, before the first launch
hipError_t launch_decay_mix(const DecayMix& P, int type, hipStream_t stream);
hipError_t launch_decay_step(const DecayStep& P, int type, hipStream_t stream);

}  // namespace nna
