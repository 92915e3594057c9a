// Parameters of the linear-attention kernels (nna_kernels_decay.hip), and their launches.
#pragma once

#include "nna_internal.h"

namespace nna {

constexpr int DECAY_HEAD_MAX = 128;  // values of a head
constexpr int DECAY_CHUNK = 64;      // a segment's frames are a multiple of it
constexpr long long DECAY_STEP_MAX = 1LL << 24;  // elements between frames: 64 of them are 32-bit offsets in bytes

// One mix of the frames: out_u = factor (sum over w <= u of decay^(u-w) (a_u . b_w) c_w + decay^(u+1) a_u S), S the state before the first;
// u counts the frames from the first, or (reverse) from the last one back, where the state's own exponent is one less.
// With out2, a pair: out2 = mix(a2, c, b) beside it, whose state is the transpose of out's.
struct DecayMix {
  const void *a, *b, *c, *a2;            // [B, T, H, da], [.., da], [.., dc], [.., dc], a head's values next to each other
  long long a_b, a_t, a_h;               // elements between batches, frames, heads
  long long b_b, b_t, b_h;
  long long c_b, c_t, c_h;
  long long a2_b, a2_t, a2_h;
  void *out, *out2;                      // [B, T, H, dc], [B, T, H, da]
  const float* decay;                    // [H]
  const int* lengths;                    // [B] or NULL: T
  const float* first;                    // [B, H, da, dc] (transposed: [B, H, dc, da]) or NULL: zero
  float* last;                           // likewise, or NULL
  float* parts;                          // [B H][segments][part_size]: each segment's own state, then the state before it, part_pitch between its rows
  float factor, first_factor, last_factor;
  int transposed;                        // first, last and parts are [dc, da]
  long long B;
  int T, H, da, dc;
  int reverse;
  int segments, segment_chunks, part_size, part_pitch;
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
size_t decay_segments(long long B, long long T, int H, int dk, int dv, int type, bool backward, int* segments, int* chunks);
hipError_t decay_kernels_init();  // per device, before the first launch
// out, and its states before (parts is as large as decay_segments says)
hipError_t launch_decay(DecayMix P, int type, hipStream_t stream);
// gq (out NULL: not wanted) with the states that `states` = (q, k, v) has, parts the same, and the pair gv, gk with its own parts
hipError_t launch_decay_gradients(DecayMix states, DecayMix gq, DecayMix pair, int type, hipStream_t stream);
hipError_t launch_decay_step(const DecayStep& P, int type, hipStream_t stream);

}  // namespace nna
