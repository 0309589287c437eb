// Positions of items turned into queries and keys: arguments after validation, and the launchers.
#pragma once

#include "laser_internal.h"

namespace laser {

struct RotaryArgs {
  const void* x[2];        // queries [T,H,D], keys [T,Hkv,D] (or nullptr)
  void* y[2];              // may be x itself
  long long xp[2], yp[2];  // elements from one token's row to the next
  int heads[2];
  const int32_t* pos;      // [T]
  const double* freq;      // [R / 2], radians a position
  int T, D, R;
  bool interleaved, back;
  float scale;
  laser_dtype dt;
  hipStream_t stream;
};
laser_status rotary_launch(const RotaryArgs& a);

struct RotaryFrequencies {
  double* freq;
  int R;
  double base, factor;     // of the slow pairs: factor > 1 stretches
  laser_rotary_scaling scaling;
  double length, low, high;
  hipStream_t stream;
};
laser_status rotary_frequencies_launch(const RotaryFrequencies& a);

}  // namespace laser
