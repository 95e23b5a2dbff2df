// Internal launcher of the rotary positions (arguments validated).
#pragma once

#include "vda_common.h"

namespace vda {

struct RopeArgs {
  const void* x;      // [B * L][x_stride]; backward: the forward input (l2) or null
  const void* dout;   // backward: the output's gradient, in the output's layout
  const float* inv_freq;
  const int* positions;  // [B * L][3] or null (grid)
  void* out;             // forward: the output; backward: dx [B * L][out_stride]
  size_t x_stride, out_stride;  // elements between token rows of x and of dx
  int B, L, H, d;
  int pairs[3];
  int grid_h, grid_w, frame_offset;
  bool interleaved, l2, heads;  // heads: the output is [B * H][L][d], else [B * L][H * d]
};
hipError_t launch_rope(bool f32, bool backward, const RopeArgs& a, hipStream_t stream);

}  // namespace vda
