// Rotary position embedding: the angles every rotating kernel uses.
#pragma once
#include <hip/hip_runtime.h>

#include "flexco.h"

namespace flexco {

// Rotation angles.  Pair i of a head turns by pos * theta^(-2 i / d).  The host hands over the frequencies in
// revolutions, theta^(-2 i / d) / (2 pi), as doubles (a kernel argument: pow and a double-precision sincos per
// (token, i) on the device were a third of these kernels' run time).  The device takes the fractional part of
// pos * rev in double precision (exact to 1e-10 of a turn at any position) and the sine and cosine of that
// fraction of a turn in single precision (angle in [0, 2 pi): about 5e-7 absolute).
constexpr int ROPE_MAX_HALF = 128;   // head_dim <= 256
struct RopeFreq {
  double rev[ROPE_MAX_HALF];
};
__device__ inline void rope_cos_sin(const RopeFreq& f, int i, int pos, float* c, float* sn) {
  const double r = (double)pos * f.rev[i];
  const float turn = (float)(r - floor(r));
  sincosf(turn * 6.283185307179586f, sn, c);
}
// The frequencies of a configuration's (rope_theta, head_dim).
int32_t rope_freq(const flexco_layer_cfg& c, RopeFreq* out);

}  // namespace flexco
