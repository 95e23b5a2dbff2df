// Internal launcher of the delta rule's recurrent form (arguments validated).
#pragma once

#include "vda_common.h"

namespace vda {

struct StepArgs {
  const void *q, *k, *v;
  const float *g, *beta;
  float* state;
  const int* slots;
  void* out;
  int n, tokens, n_slots, Hk, Hv, group, d_v;
  float scale;
};
hipError_t launch_delta_step(bool f32, int d_k, const StepArgs& a, hipStream_t stream);

}  // namespace vda
