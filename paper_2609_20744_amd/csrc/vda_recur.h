// Internal definitions of the channel-wise gated recurrence (vda.h, vda_recur_*).
#pragma once

#include "vda_common.h"

namespace vda {

constexpr int kRecurChans = 128;  // channels of a workgroup: 16 lanes of eight
constexpr int kRecurRuns = 16;    // runs of consecutive tokens that it takes side by side
constexpr int kRecurRun = 4;      // tokens of a run of the backward pass
constexpr int kRecurTile = kRecurRuns * kRecurRun;
constexpr int kRecurUnit = 128;   // the forward pass's segments are multiples of it

struct RecurArgs {
  const void *x, *g, *dout;
  const float *S_in, *dS_out;
  void *out, *dx, *dg;
  float *S_out, *dS_in;
  size_t xs, gs, dxs, dgs;  // elements between token rows (out and dout: C)
  const int* cu;
  int n, T, L, C;           // L: tokens of a sequence, equal lengths
  int gate, reverse;
  int seg;                  // forward: tokens of a segment
  int tiles;                // places of all sequences' segments (backward: of their tiles)
  bool carried;             // there may be sequences of more than one
  float *A, *H, *G;         // [tiles][C] a part's decay, and what it adds to the state and to the state's gradient
};

struct RecurStepArgs {
  const void *x, *g;
  const int* slots;
  float* state;
  void* out;
  int n, tokens, C, gate, n_slots;
};

hipError_t launch_recur(bool f32, bool backward, const RecurArgs& a, hipStream_t stream);
hipError_t launch_recur_step(bool f32, const RecurStepArgs& a, hipStream_t stream);

}  // namespace vda
