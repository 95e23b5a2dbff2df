// C ABI of the channel-wise gated recurrence: argument validation, workspace
// layout, launch order.  Declarations and contracts are in include/vda.h.
#include <algorithm>
#include <initializer_list>

#include "../../include/vda.h"
#include "vda_host.h"
#include "vda_recur.h"

namespace {

using vda::aligned;
using vda::hip_status;
using vda::overlaps;
using vda::Range;
using vda::range_of;
using vda::RecurArgs;
using vda::round_up;

constexpr long long kMaxThreads = 0xffffffffLL;  // of a launch
constexpr int kMaxGridY = 65535;

size_t gate_size(int gate, int is_f32) { return is_f32 || gate == VDA_GATE_LOG ? 4 : 2; }

int check_channels(int C, int gate) {
  if (C < 1) return VDA_ERR_SIZE;
  if (C % 8 || (gate != VDA_GATE_LOG && gate != VDA_GATE_LOGIT && gate != VDA_GATE_NORM)) return VDA_ERR_UNSUPPORTED;
  return C > 128 * kMaxGridY ? VDA_ERR_SIZE : VDA_OK;
}

// Tokens of a part of a sequence: a tile backward; forward a segment, so long that about
// three workgroups of 128 channels are there for each compute unit (40320 tokens of 896 channels
// 63 us, 66 us with one and with six a unit, inputs in the last-level cache; 100000 of 128
// channels 34, 35 and 38 us).
int part_of(const vda_recur_problem* p, bool backward) {
  if (backward) return vda::kRecurTile;
  const long long slabs = (p->C + vda::kRecurChans - 1) / vda::kRecurChans;
  const long long share = (long long)p->T * slabs / (3LL * vda::current_device_cus());
  return (int)std::min(2048LL, std::max(1LL, (share + vda::kRecurUnit - 1) / vda::kRecurUnit) * vda::kRecurUnit);
}

long long parts_of(const vda_recur_problem* p, int part) {
  const long long n = p->n_seqs, T = p->T;
  return p->cu_seqlens ? T / part + n : n * ((T / n + part - 1) / part);
}

bool carried(const vda_recur_problem* p, int part) { return (p->cu_seqlens ? p->T : p->T / p->n_seqs) > part; }

int check_stride(int stride, int C, size_t es) {
  if (stride != 0 && stride < C) return VDA_ERR_SIZE;
  return stride * es % 16 ? VDA_ERR_ALIGN : VDA_OK;
}

int check_problem(const vda_recur_problem* p, bool backward) {
  if (!p) return VDA_ERR_NULL;
  if (p->T < 1 || p->n_seqs < 1) return VDA_ERR_SIZE;
  if (!p->cu_seqlens && p->T % p->n_seqs) return VDA_ERR_SIZE;
  int st = check_channels(p->C, p->gate);
  if (st != VDA_OK) return st;
  const size_t es = p->is_f32 ? 4 : 2, ge = gate_size(p->gate, p->is_f32);
  if ((st = check_stride(p->x_row_stride, p->C, es)) != VDA_OK || (st = check_stride(p->g_row_stride, p->C, ge)) != VDA_OK)
    return st;
  if (backward && ((st = check_stride(p->dx_row_stride, p->C, es)) != VDA_OK ||
                   (st = check_stride(p->dg_row_stride, p->C, ge)) != VDA_OK))
    return st;
  if (!aligned(p->cu_seqlens, 4)) return VDA_ERR_ALIGN;
  // A workgroup of 256 threads per tile, one of 1024 per sequence; tokens are counted in 32 bits.
  const long long slabs = (p->C + vda::kRecurChans - 1) / vda::kRecurChans;
  if (parts_of(p, vda::kRecurTile) * slabs > kMaxThreads / 256 || (long long)p->n_seqs * 1024 > kMaxThreads ||
      (long long)p->T + vda::kRecurTile > 0x7fffffffLL)
    return VDA_ERR_SIZE;
  // Backward, the kernel that carries states from tile to tile has 64 channels a workgroup in the grid's y.
  if (backward && carried(p, vda::kRecurTile) && ((long long)p->C + 63) / 64 > kMaxGridY) return VDA_ERR_SIZE;
  return VDA_OK;
}

size_t workspace(const vda_recur_problem* p, bool backward) {
  const int part = part_of(p, backward);
  if (!carried(p, part)) return 0;
  return (backward ? 3 : 2) * round_up((size_t)parts_of(p, part) * p->C * 4, 256);
}

RecurArgs args_of(const vda_recur_problem* p, bool backward, void* work) {
  RecurArgs a = {};
  a.cu = p->cu_seqlens, a.n = p->n_seqs, a.T = p->T, a.L = p->T / p->n_seqs, a.C = p->C;
  a.xs = p->x_row_stride ? p->x_row_stride : p->C, a.gs = p->g_row_stride ? p->g_row_stride : p->C;
  a.dxs = p->dx_row_stride ? p->dx_row_stride : p->C, a.dgs = p->dg_row_stride ? p->dg_row_stride : p->C;
  a.gate = p->gate, a.reverse = p->reverse != 0;
  a.seg = part_of(p, backward);
  a.tiles = (int)parts_of(p, a.seg), a.carried = carried(p, a.seg);
  const size_t each = round_up((size_t)a.tiles * p->C * 4, 256) / 4;
  a.A = static_cast<float*>(work), a.H = a.A + each, a.G = a.H + each;
  return a;
}

bool any_overlap(std::initializer_list<Range> outs, std::initializer_list<Range> ins) {
  for (const Range* o = outs.begin(); o != outs.end(); ++o) {
    for (const Range& i : ins)
      if (overlaps(*o, i)) return true;
    for (const Range* q = o + 1; q != outs.end(); ++q)
      if (overlaps(*o, *q)) return true;
  }
  return false;
}

Range opt_range(const void* p, size_t bytes) { return range_of(p, p ? bytes : 0); }

Range rows_range(const void* p, const vda_recur_problem* q, int stride, size_t es) {
  return range_of(p, ((size_t)(q->T - 1) * (stride ? stride : q->C) + q->C) * es);
}

}  // namespace

extern "C" {

size_t vda_recur_forward_workspace(const vda_recur_problem* p) {
  return check_problem(p, false) == VDA_OK ? workspace(p, false) : 0;
}

size_t vda_recur_backward_workspace(const vda_recur_problem* p) {
  return check_problem(p, true) == VDA_OK ? workspace(p, true) : 0;
}

int vda_recur_forward(const vda_recur_problem* p, const void* x, const void* g, const float* S_in, void* out, float* S_out,
                      void* work, hipStream_t stream) {
  if (!p || !x || !g || !out) return VDA_ERR_NULL;
  const int st = check_problem(p, false);
  if (st != VDA_OK) return st;
  const size_t need = workspace(p, false);
  if (need && !work) return VDA_ERR_NULL;
  if (!need) work = nullptr;
  for (const void* t : {x, g, (const void*)S_in, (const void*)out, (const void*)S_out, (const void*)work})
    if (!aligned(t, 16)) return VDA_ERR_ALIGN;
  const size_t es = p->is_f32 ? 4 : 2, ge = gate_size(p->gate, p->is_f32), state = (size_t)p->n_seqs * p->C * 4;
  if (any_overlap({rows_range(out, p, 0, es), opt_range(S_out, state), opt_range(work, need)},
                  {rows_range(x, p, p->x_row_stride, es), rows_range(g, p, p->g_row_stride, ge), opt_range(S_in, state),
                   opt_range(p->cu_seqlens, (size_t)(p->n_seqs + 1) * 4)}))
    return VDA_ERR_OVERLAP;
  RecurArgs a = args_of(p, false, work);
  a.x = x, a.g = g, a.S_in = S_in, a.out = out, a.S_out = S_out;
  return hip_status(vda::launch_recur(p->is_f32 != 0, false, a, stream));
}

int vda_recur_backward(const vda_recur_problem* p, const void* dout, const void* x, const void* g, const float* S_in,
                       const float* dS_out, void* dx, void* dg, float* dS_in, void* work, hipStream_t stream) {
  if (!p || !dout || !x || !g || !dx || !dg) return VDA_ERR_NULL;
  const int st = check_problem(p, true);
  if (st != VDA_OK) return st;
  const size_t need = workspace(p, true);
  if (need && !work) return VDA_ERR_NULL;
  if (!need) work = nullptr;
  for (const void* t : {dout, x, g, (const void*)S_in, (const void*)dS_out, (const void*)dx, (const void*)dg, (const void*)dS_in,
                        (const void*)work})
    if (!aligned(t, 16)) return VDA_ERR_ALIGN;
  const size_t es = p->is_f32 ? 4 : 2, ge = gate_size(p->gate, p->is_f32), state = (size_t)p->n_seqs * p->C * 4;
  const Range rdx = rows_range(dx, p, p->dx_row_stride, es), rdg = rows_range(dg, p, p->dg_row_stride, ge);
  const Range both = Range{std::min(rdx.lo, rdg.lo), std::max(rdx.hi, rdg.hi)};
  const bool meet = overlaps(rdx, rdg);
  if (meet && (es != ge || !vda::slices_apart(dx, p->dx_row_stride, dg, p->dg_row_stride, (size_t)p->C * es, es)))
    return VDA_ERR_OVERLAP;
  const std::initializer_list<Range> ins = {rows_range(dout, p, 0, es), rows_range(x, p, p->x_row_stride, es),
                                            rows_range(g, p, p->g_row_stride, ge), opt_range(S_in, state),
                                            opt_range(dS_out, state), opt_range(p->cu_seqlens, (size_t)(p->n_seqs + 1) * 4)};
  const Range rs = opt_range(dS_in, state), rw = opt_range(work, need);
  if (meet ? any_overlap({both, rs, rw}, ins) : any_overlap({rdx, rdg, rs, rw}, ins)) return VDA_ERR_OVERLAP;
  RecurArgs a = args_of(p, true, work);
  a.x = x, a.g = g, a.dout = dout, a.S_in = S_in, a.dS_out = dS_out, a.dx = dx, a.dg = dg, a.dS_in = dS_in;
  return hip_status(vda::launch_recur(p->is_f32 != 0, true, a, stream));
}

int vda_recur_step(const void* x, const void* g, int n, int tokens, int C, int gate, int is_f32, const int* slots, int n_slots,
                   float* state, void* out, hipStream_t stream) {
  if (!x || !g || !state || !out) return VDA_ERR_NULL;
  if (n < 1 || tokens < 1 || n_slots < 1 || (!slots && n > n_slots)) return VDA_ERR_SIZE;
  const int st = check_channels(C, gate);
  if (st != VDA_OK) return st;
  if ((long long)n * (C / 4) + 256 > kMaxThreads || (long long)n * tokens > 0x7fffffffLL) return VDA_ERR_SIZE;
  if (!aligned(x, 16) || !aligned(g, 16) || !aligned(out, 16) || !aligned(state, 16) || !aligned(slots, 4)) return VDA_ERR_ALIGN;
  const size_t es = is_f32 ? 4 : 2, rows = (size_t)n * tokens * C;
  if (any_overlap({range_of(out, rows * es), range_of(state, (size_t)n_slots * C * 4)},
                  {range_of(x, rows * es), range_of(g, rows * gate_size(gate, is_f32)), opt_range(slots, (size_t)n * 4)}))
    return VDA_ERR_OVERLAP;
  vda::RecurStepArgs a = {};
  a.x = x, a.g = g, a.slots = slots, a.state = state, a.out = out;
  a.n = n, a.tokens = tokens, a.C = C, a.gate = gate, a.n_slots = n_slots;
  return hip_status(vda::launch_recur_step(is_f32 != 0, a, stream));
}

}  // extern "C"
