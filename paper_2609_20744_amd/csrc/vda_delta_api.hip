// C ABI of the token-wise gated delta rule and of the rotary positions:
// argument validation, workspace layout, launch order.  Declarations and
// contracts are in include/vda.h.
#include <algorithm>
#include <initializer_list>

#include "../../include/vda.h"
#include "vda_delta.h"
#include "vda_delta_step.h"
#include "vda_host.h"
#include "vda_rope.h"

namespace {

using vda::aligned;
using vda::hip_status;
using vda::overlaps;
using vda::Range;
using vda::range_of;
using vda::round_up;
using vda::supported_dim;

// A launch holds fewer than 2^32 threads.
constexpr long long kMaxThreads = 0xffffffffLL;

int check_heads(int H_k, int H_v, int d_k, int d_v) {
  if (H_k < 1 || H_v < 1 || H_v % H_k) return VDA_ERR_SIZE;
  if (!supported_dim(d_k) || !supported_dim(d_v)) return VDA_ERR_UNSUPPORTED;
  return VDA_OK;
}

int check_problem(const vda_delta_problem* p) {
  if (!p) return VDA_ERR_NULL;
  if (p->T < 1 || p->n_seqs < 1) return VDA_ERR_SIZE;
  if (!p->cu_seqlens && p->T % p->n_seqs) return VDA_ERR_SIZE;
  const int st = check_heads(p->H_k, p->H_v, p->d_k, p->d_v);
  if (st != VDA_OK) return st;
  if (p->layout != VDA_LAYOUT_HEADS && p->layout != VDA_LAYOUT_TOKENS) return VDA_ERR_UNSUPPORTED;
  if (!aligned(p->cu_seqlens, 4)) return VDA_ERR_ALIGN;
  // A token's row is addressed in 24 bits, a chunk's in 32, and a launch has one
  // workgroup of up to 512 threads per chunk (or two per segment) and head.
  const long long es = p->is_f32 ? 4 : 2;
  const long long row = p->layout == VDA_LAYOUT_TOKENS
                            ? es * std::max((long long)p->H_k * p->d_k, (long long)p->H_v * p->d_v)
                            : es * std::max(p->d_k, p->d_v);
  if (row >= 1 << 24) return VDA_ERR_SIZE;
  const long long items = ((long long)p->T / vda::kChunk + p->n_seqs + 1) * p->H_v;
  const long long joined = ((long long)p->n_seqs * p->H_v + 7) / 8 * 8 * (p->d_v / 16);
  if (items * 1024 > kMaxThreads || joined * 256 > kMaxThreads ||
      (long long)p->T + vda::kChunk > 0x7fffffffLL)
    return VDA_ERR_SIZE;
  return VDA_OK;
}

vda::DeltaPlan plan_of(const vda_delta_problem* p, bool backward) {
  vda::DeltaPlan d;
  const bool table = p->cu_seqlens != nullptr;
  const long long n = p->n_seqs, T = p->T;
  const long long per = (T / n + vda::kChunk - 1) / vda::kChunk;  // chunks of a sequence (equal lengths)
  const long long longest = table ? (T + vda::kChunk - 1) / vda::kChunk : per;
  d.max_chunks = (int)(table ? (T + (vda::kChunk - 1) * n) / vda::kChunk : per * n);
  // Segments.  A sequence that is cut costs each of its chunks a second scan
  // (5.9 us beside an output's 3.4, 128 x 128, bf16) and a step of the join per
  // segment (1.1 us).  Figures: us of a forward and a backward call, bf16,
  // 128 x 128 where not said.
  //  - Where sequences and heads alone fill the compute units, only one that is
  //    far longer than the rest is cut, into segments of four times the mean.  24
  //    uneven sequences of 16411 tokens, 16 heads: 158 and 722 whole (166 and 738
  //    as here, with maps and a join that find nothing to do), 184 and 755 in
  //    segments of 16 chunks.  40 sequences of 4 chunks in the mean, 8 heads, one of
  //    them 12 times as long: 198 and 522 as here, 184 and 559 whole, 139 and 410
  //    in segments of twice the mean; one 6 times as long: 161 and 434, 109 and
  //    383, 116 and 393.  So four is right for what it leaves whole, and too long
  //    for what it cuts.
  //  - Where they do not, every unit gets a segment: 9 uneven sequences of 16401
  //    tokens, 16 heads, 218 and 786 cut, 389 and 1308 whole; 1560 tokens of 24
  //    heads 64 and 173 cut, 95 and 250 whole.
  //  - Shorter segments make the scans shorter and the join longer: the least time
  //    is at about the square root of an eighth of the sequence's chunks.  8 heads
  //    of 1088 tokens in segments of 2, 3 and 4 chunks 45, 48 and 55 (100, 108 and
  //    120); 2 heads of 38400 tokens of 5, 7, 9 and 12 chunks 205, 179, 172 and 175
  //    (569, 495, 473 and 473).
  //  - Short sequences stay whole.  8 heads of eight chunks: 36 and 84 whole, 38 and
  //    83 in segments of two chunks (nine: 39 and 92, 39 and 87; 24 heads of nine: 39
  //    and 99, 43 and 97; 64 channels, nine: 25 and 51, 24 and 50).  fp32, six chunks:
  //    64 channels 47 and 94 whole, 43 and 91 cut, in two more launches and four
  //    (seven: 52 and 104, 43 and 92); 128 channels 115 and 225, 97 and 212 (five: 98
  //    and 196, 97 and 211).
  //  - Segments that the compute units make longer than two chunks pay from the
  //    fourth on, or later: of three chunks, 32 heads of 24 chunks 67 and 202 cut, 93
  //    and 261 whole, but 64 heads of 12 chunks 65 and 194 cut, 55 and 175 whole; of
  //    six chunks, 64 heads of 24 chunks 99 and 357 cut, 102 and 374 whole.
  const long long cus = vda::current_device_cus();
  long long share = std::max(2LL, (d.max_chunks * (long long)p->H_v + cus - 1) / cus);
  while (8 * share * share < longest) ++share;
  if (n * p->H_v >= cus) share = std::max(share, 4 * ((d.max_chunks + n - 1) / n));
  const int whole = p->is_f32 ? 6 : 8;
  d.split = longest > whole && (share == 2 || longest > 4 * share);
  d.seg_chunks = (int)(d.split ? share : std::max(longest, 1LL));
  d.whole = std::max(d.seg_chunks, whole);
  d.max_segs =
      (int)(table ? d.max_chunks / d.seg_chunks + n : n * ((per + d.seg_chunks - 1) / d.seg_chunks));
  // Workspace.
  size_t at = 0;
  auto take = [&](size_t bytes) {
    const size_t from = at;
    at = round_up(at + bytes, 1024);
    return from;
  };
  const size_t mat = (size_t)p->d_v * p->d_k * 4, km = (size_t)p->d_k * p->d_k * 4;
  const size_t segs = (size_t)d.max_segs * p->H_v, chunks = (size_t)d.max_chunks * p->H_v;
  const size_t entries = (size_t)d.max_chunks * 16 + (size_t)d.max_segs * (16 + 4);
  d.tabs = take(table ? round_up((4 + 2 * (n + 1)) * 4, 16) + entries : 0);
  d.rec = take(chunks * vda::ChunkRecord::bytes(p->is_f32 != 0, backward));
  d.segs = take(d.split ? segs * (mat * (backward ? 2 : 1) + 2 * km) : 0);
  d.keep = take(backward ? chunks * 2 * (mat + (size_t)p->d_v * vda::kChunk * 4) : 0);
  d.total = at;
  return d;
}

vda::DeltaArgs args_of(const vda_delta_problem* p, const vda::DeltaPlan& d, bool backward, void* work) {
  vda::DeltaArgs a = {};
  a.Hk = p->H_k, a.Hv = p->H_v, a.group = p->H_v / p->H_k, a.d_v = p->d_v;
  if (p->layout == VDA_LAYOUT_HEADS) {
    a.qk_tok = p->d_k, a.qk_head = (size_t)p->T * p->d_k;
    a.v_tok = p->d_v, a.v_head = (size_t)p->T * p->d_v;
    a.gate_tok = 1, a.gate_head = p->T;
  } else {
    a.qk_tok = (size_t)p->H_k * p->d_k, a.qk_head = p->d_k;
    a.v_tok = (size_t)p->H_v * p->d_v, a.v_head = p->d_v;
    a.gate_tok = p->H_v, a.gate_head = 1;
  }
  a.scale = p->scale;
  a.n_seqs = p->n_seqs, a.L = p->T / p->n_seqs;
  a.seg_chunks = d.seg_chunks, a.max_chunks = d.max_chunks, a.max_segs = d.max_segs;
  char* w = static_cast<char*>(work);
  if (p->cu_seqlens) {
    int* tabs = reinterpret_cast<int*>(w + d.tabs);
    a.counts = tabs;
    a.chunk_tab = reinterpret_cast<int4*>(tabs + (4 + 2 * (p->n_seqs + 1) + 3) / 4 * 4);
    a.seg_tab = a.chunk_tab + d.max_chunks;
    a.seg_id = reinterpret_cast<const int*>(a.seg_tab + d.max_segs);
  }
  a.rec = w + d.rec;
  const size_t mat = (size_t)p->d_v * p->d_k, km = (size_t)p->d_k * p->d_k;
  const size_t segs = (size_t)d.max_segs * p->H_v, chunks = (size_t)d.max_chunks * p->H_v;
  if (d.split) {
    a.segJ = reinterpret_cast<float*>(w + d.segs);
    a.segM = w + d.segs + segs * mat * 4;
    if (backward) a.segdJ = reinterpret_cast<float*>(a.segM + segs * 2 * km * 4);
  }
  if (backward) {
    a.keepS = w + d.keep;
    a.keepdS = a.keepS + chunks * mat * 4;
    a.keepE = a.keepdS + chunks * mat * 4;
    a.keepdv = a.keepE + chunks * p->d_v * vda::kChunk * 4;
  }
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

struct Sizes {
  size_t qk, v, gate, state, cu;
};
Sizes sizes_of(const vda_delta_problem* p) {
  const size_t es = p->is_f32 ? 4 : 2, T = p->T;
  return Sizes{T * p->H_k * p->d_k * es, T * p->H_v * p->d_v * es, T * p->H_v * 4,
               (size_t)p->n_seqs * p->H_v * p->d_v * p->d_k * 4, (size_t)(p->n_seqs + 1) * 4};
}

hipError_t plan_and_prepare(const vda_delta_problem* p, const vda::DeltaPlan& d, const vda::DeltaArgs& a,
                            bool backward, hipStream_t stream) {
  if (p->cu_seqlens) {
    const hipError_t e = vda::launch_delta_plan(p->cu_seqlens, p->n_seqs, p->T, d, const_cast<int*>(a.counts),
                                                stream);
    if (e != hipSuccess) return e;
  }
  hipError_t e = vda::launch_delta_prepare(p->is_f32 != 0, p->d_k, backward, a, stream);
  if (e != hipSuccess || !d.split) return e;
  if ((e = vda::launch_delta_scan(p->is_f32 != 0, p->d_k, 0, a, stream)) != hipSuccess) return e;
  return vda::launch_delta_join(p->is_f32 != 0, p->d_k, false, a, stream);
}

}  // namespace

extern "C" {

size_t vda_delta_forward_workspace(const vda_delta_problem* p) {
  return check_problem(p) == VDA_OK ? plan_of(p, false).total : 0;
}

size_t vda_delta_backward_workspace(const vda_delta_problem* p) {
  return check_problem(p) == VDA_OK ? plan_of(p, true).total : 0;
}

int vda_delta_forward(const vda_delta_problem* p, const void* q, const void* k, const void* v,
                      const float* g, const float* beta, const float* S_in, void* out, float* S_out,
                      void* work, hipStream_t stream) {
  if (!p || !q || !k || !v || !g || !beta || !out || !work) return VDA_ERR_NULL;
  const int st = check_problem(p);
  if (st != VDA_OK) return st;
  if (!aligned(q, 16) || !aligned(k, 16) || !aligned(v, 16) || !aligned(out, 16) || !aligned(work, 16) ||
      !aligned(S_in, 16) || !aligned(S_out, 16) || !aligned(g, 4) || !aligned(beta, 4))
    return VDA_ERR_ALIGN;
  const vda::DeltaPlan d = plan_of(p, false);
  const Sizes z = sizes_of(p);
  if (any_overlap({range_of(out, z.v), opt_range(S_out, z.state), range_of(work, d.total)},
                  {range_of(q, z.qk), range_of(k, z.qk), range_of(v, z.v), range_of(g, z.gate),
                   range_of(beta, z.gate), opt_range(S_in, z.state), opt_range(p->cu_seqlens, z.cu)}))
    return VDA_ERR_OVERLAP;
  vda::DeltaArgs a = args_of(p, d, false, work);
  a.q = q, a.k = k, a.v = v, a.g = g, a.beta = beta;
  a.S_in = S_in, a.S_out = S_out, a.out = out;
  const hipError_t e = plan_and_prepare(p, d, a, false, stream);
  if (e != hipSuccess) return hip_status(e);
  return hip_status(vda::launch_delta_scan(p->is_f32 != 0, p->d_k, 1, a, stream));
}

int vda_delta_backward(const vda_delta_problem* p, const void* dout, const void* q, const void* k,
                       const void* v, const float* g, const float* beta, const float* S_in,
                       const float* dS_out, void* dq, void* dk, void* dv, float* dg, float* dbeta,
                       float* dS_in, void* work, hipStream_t stream) {
  if (!p || !dout || !q || !k || !v || !g || !beta || !dq || !dk || !dv || !dg || !dbeta || !work)
    return VDA_ERR_NULL;
  const int st = check_problem(p);
  if (st != VDA_OK) return st;
  if (!aligned(dout, 16) || !aligned(q, 16) || !aligned(k, 16) || !aligned(v, 16) || !aligned(dq, 16) ||
      !aligned(dk, 16) || !aligned(dv, 16) || !aligned(work, 16) || !aligned(S_in, 16) ||
      !aligned(dS_out, 16) || !aligned(dS_in, 16) || !aligned(g, 4) || !aligned(beta, 4) ||
      !aligned(dg, 4) || !aligned(dbeta, 4))
    return VDA_ERR_ALIGN;
  const vda::DeltaPlan d = plan_of(p, true);
  const Sizes z = sizes_of(p);
  if (any_overlap({range_of(dq, z.qk), range_of(dk, z.qk), range_of(dv, z.v), range_of(dg, z.gate),
                   range_of(dbeta, z.gate), opt_range(dS_in, z.state), range_of(work, d.total)},
                  {range_of(dout, z.v), range_of(q, z.qk), range_of(k, z.qk), range_of(v, z.v),
                   range_of(g, z.gate), range_of(beta, z.gate), opt_range(S_in, z.state),
                   opt_range(dS_out, z.state), opt_range(p->cu_seqlens, z.cu)}))
    return VDA_ERR_OVERLAP;
  vda::DeltaArgs a = args_of(p, d, true, work);
  a.q = q, a.k = k, a.v = v, a.dout = dout, a.g = g, a.beta = beta;
  a.S_in = S_in, a.dS_out = dS_out, a.dS_in = dS_in;
  a.dq = dq, a.dk = dk, a.dv = dv, a.dg = dg, a.dbeta = dbeta;
  const bool f32 = p->is_f32 != 0;
  hipError_t e = plan_and_prepare(p, d, a, true, stream);
  if (e == hipSuccess) e = vda::launch_delta_scan(f32, p->d_k, 2, a, stream);
  if (e == hipSuccess && d.split) {
    e = vda::launch_delta_reverse(f32, p->d_k, true, a, stream);
    if (e == hipSuccess) e = vda::launch_delta_join(f32, p->d_k, true, a, stream);
  }
  if (e == hipSuccess) e = vda::launch_delta_reverse(f32, p->d_k, false, a, stream);
  if (e == hipSuccess) e = vda::launch_delta_grad(f32, p->d_k, a, stream);
  return hip_status(e);
}

int vda_delta_step(const void* q, const void* k, const void* v, const float* g, const float* beta, int n,
                   int tokens, int H_k, int H_v, int d_k, int d_v, int is_f32, float scale,
                   const int* slots, int n_slots, float* state, void* out, hipStream_t stream) {
  if (!q || !k || !v || !g || !beta || !state || !out) return VDA_ERR_NULL;
  if (n < 1 || tokens < 1 || n_slots < 1 || (!slots && n > n_slots)) return VDA_ERR_SIZE;
  const int st = check_heads(H_k, H_v, d_k, d_v);
  if (st != VDA_OK) return st;
  if ((long long)n * H_v > kMaxThreads / (d_v * 16LL) || (long long)n * tokens > 0x7fffffffLL)
    return VDA_ERR_SIZE;
  if (!aligned(q, 16) || !aligned(k, 16) || !aligned(v, 16) || !aligned(out, 16) || !aligned(state, 16) ||
      !aligned(g, 4) || !aligned(beta, 4) || !aligned(slots, 4))
    return VDA_ERR_ALIGN;
  const size_t es = is_f32 ? 4 : 2, rows = (size_t)n * tokens;
  const size_t qk = rows * H_k * d_k * es, vb = rows * H_v * d_v * es, gate = rows * H_v * 4;
  if (any_overlap({range_of(out, vb), range_of(state, (size_t)n_slots * H_v * d_v * d_k * 4)},
                  {range_of(q, qk), range_of(k, qk), range_of(v, vb), range_of(g, gate), range_of(beta, gate),
                   opt_range(slots, (size_t)n * 4)}))
    return VDA_ERR_OVERLAP;
  vda::StepArgs a = {};
  a.q = q, a.k = k, a.v = v, a.g = g, a.beta = beta, a.state = state, a.slots = slots, a.out = out;
  a.n = n, a.tokens = tokens, a.n_slots = n_slots;
  a.Hk = H_k, a.Hv = H_v, a.group = H_v / H_k, a.d_v = d_v, a.scale = scale;
  return hip_status(vda::launch_delta_step(is_f32 != 0, d_k, a, stream));
}

}  // extern "C"

namespace {

int rope_impl(bool backward, const void* x, const void* dout, const float* inv_freq, const int* positions, int B,
              int L, int H, int d, const vda_rope_options* o, int is_f32, void* out, hipStream_t stream) {
  if (!o || !inv_freq || !out || (backward && !dout)) return VDA_ERR_NULL;
  const bool reads_x = !backward || o->l2;  // otherwise x may be anything
  if (!reads_x) x = nullptr;
  if (reads_x && !x) return VDA_ERR_NULL;
  if (B < 1 || L < 1 || H < 1) return VDA_ERR_SIZE;
  if (d != 16 && !supported_dim(d)) return VDA_ERR_UNSUPPORTED;
  if (o->pairs_t < 0 || o->pairs_h < 0 || o->pairs_w < 0) return VDA_ERR_SIZE;
  const long long pairs = (long long)o->pairs_t + o->pairs_h + o->pairs_w;
  if (pairs < 1 || pairs > d / 2) return VDA_ERR_SIZE;
  if (pairs % 8) return VDA_ERR_UNSUPPORTED;
  if (o->layout != VDA_LAYOUT_HEADS && o->layout != VDA_LAYOUT_TOKENS) return VDA_ERR_UNSUPPORTED;
  if (!positions && (o->grid_h < 1 || o->grid_w < 1 || o->frame_offset < 0 ||
                     (long long)o->frame_offset + L > 0x7fffffffLL))
    return VDA_ERR_SIZE;
  const long long row = (long long)H * d;
  const size_t es = is_f32 ? 4 : 2;
  const long long xs = reads_x && o->x_row_stride ? o->x_row_stride : row;
  const long long ds = backward && o->dx_row_stride ? o->dx_row_stride : row;
  // One workgroup of 256 threads per four tokens; a workgroup's items are 32-bit.
  if (row > 0x7fffffffLL / 64 || xs < row || ds < row || (long long)B * L > (kMaxThreads / 256) * 4 ||
      (long long)B * L > 0x7fffffffLL)
    return VDA_ERR_SIZE;
  if (xs * es % 16 || ds * es % 16) return VDA_ERR_ALIGN;
  if (!aligned(x, 16) || !aligned(dout, 16) || !aligned(out, 16) || !aligned(inv_freq, 4) ||
      !aligned(positions, 4))
    return VDA_ERR_ALIGN;
  const size_t rows = (size_t)B * L;
  auto bytes = [&](long long stride) { return ((rows - 1) * stride + row) * es; };
  if (any_overlap({range_of(out, bytes(ds))},
                  {opt_range(x, bytes(xs)), opt_range(dout, bytes(row)),
                   range_of(inv_freq, (size_t)pairs * 4), opt_range(positions, rows * 12)}))
    return VDA_ERR_OVERLAP;
  vda::RopeArgs a = {};
  a.x = x, a.dout = dout, a.inv_freq = inv_freq, a.positions = positions, a.out = out;
  a.x_stride = xs, a.out_stride = ds;
  a.B = B, a.L = L, a.H = H, a.d = d;
  a.pairs[0] = o->pairs_t, a.pairs[1] = o->pairs_h, a.pairs[2] = o->pairs_w;
  a.grid_h = o->grid_h, a.grid_w = o->grid_w, a.frame_offset = o->frame_offset;
  a.interleaved = o->interleaved != 0, a.l2 = o->l2 != 0, a.heads = o->layout == VDA_LAYOUT_HEADS;
  return hip_status(vda::launch_rope(is_f32 != 0, backward, a, stream));
}

}  // namespace

extern "C" {

int vda_rope(const void* x, const float* inv_freq, const int* positions, int B, int L, int H, int d,
             const vda_rope_options* opts, int is_f32, void* out, hipStream_t stream) {
  return rope_impl(false, x, nullptr, inv_freq, positions, B, L, H, d, opts, is_f32, out, stream);
}

int vda_rope_backward(const void* dout, const void* x, const float* inv_freq, const int* positions, int B, int L,
                      int H, int d, const vda_rope_options* opts, int is_f32, void* dx, hipStream_t stream) {
  return rope_impl(true, x, dout, inv_freq, positions, B, L, H, d, opts, is_f32, dx, stream);
}

}  // extern "C"
