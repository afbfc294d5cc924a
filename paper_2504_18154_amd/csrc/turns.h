// Angles of the position rotation, for the kernels that turn rows on their way into the cache (kv_rope.hip says how they are formed).
#pragma once

#include "common.h"

namespace eco {

// What the kernels need of the rotation (by value: the axes of the pairs travel with the launch).
struct Turns {
  const double* inv_freq;
  const int32_t* positions;  // [num_axes][T] or NULL
  int32_t T, rotary, num_axes;
  uint8_t axis[128];
};
inline Turns make_turns(const ecoserve_rope& rope, const double* inv_freq, const int32_t* positions, int32_t T) {
  Turns t;
  t.inv_freq = inv_freq;
  t.positions = positions;
  t.T = T;
  t.rotary = rope.rotary_dim;
  t.num_axes = rope.num_axes;
  for (int i = 0; i < 128; ++i) t.axis[i] = rope.axis[i];
  return t;
}

#if defined(__HIPCC__)
struct Angle {
  float c, s;
};
__device__ __forceinline__ Angle angle_of(int32_t position, double inv_freq) {
  const double t = (double)position * (inv_freq * 0.15915494309189535);  // turns
  const double q4 = (t - rint(t)) * 4.0, k = rint(q4);
  const float a = (float)((q4 - k) * 1.5707963267948966), a2 = a * a;
  const float s = a + a * a2 * (-1.f / 6 + a2 * (1.f / 120 + a2 * (-1.f / 5040 + a2 * (1.f / 362880))));
  const float c = 1.f + a2 * (-0.5f + a2 * (1.f / 24 + a2 * (-1.f / 720 + a2 * (1.f / 40320 - a2 * (1.f / 3628800)))));
  const int quarter = (int)k & 3;
  const float x = quarter & 1 ? s : c, y = quarter & 1 ? c : s;
  return {quarter == 1 || quarter == 2 ? -x : x, quarter >= 2 ? -y : y};
}
// The angle of pair i of packed token `tok`, at `place` in its sequence.
__device__ __forceinline__ Angle angle_of_pair(const Turns& r, int i, int tok, int place) {
  const int32_t p = r.positions ? r.positions[(size_t)(r.num_axes > 1 ? r.axis[i] : 0) * r.T + tok] : place;
  return angle_of(p, r.inv_freq[i]);
}
#endif

}  // namespace eco
