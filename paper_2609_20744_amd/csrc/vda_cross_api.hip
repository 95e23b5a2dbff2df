// C ABI of the cross attention to an encoder's states: argument validation,
// workspace layout, launch order.  Declarations and contracts are in
// include/vda.h.
#include <algorithm>
#include <initializer_list>

#include "../../include/vda.h"
#include "vda_cross.h"
#include "vda_host.h"

namespace {

using vda::aligned;
using vda::CrossArgs;
using vda::CrossStrides;
using vda::hip_status;
using vda::overlaps;
using vda::Range;
using vda::range_of;
using vda::round_up;

constexpr long long kMaxThreads = 0xffffffffLL;  // of a launch
constexpr long long kMaxInt = 0x7fffffffLL;

bool is_layout(int l) { return l == VDA_LAYOUT_HEADS || l == VDA_LAYOUT_TOKENS; }

int check_stride(int stride, int layout, long long row, size_t es) {
  if (layout == VDA_LAYOUT_HEADS) return stride == 0 ? VDA_OK : VDA_ERR_UNSUPPORTED;
  const long long s = stride == 0 ? row : stride;
  if (s < row || s * (long long)es >= 1 << 24) return VDA_ERR_SIZE;
  return s * es % 16 ? VDA_ERR_ALIGN : VDA_OK;
}

// slots: n_slots of states where it is > 0.
int check_problem(const vda_cross_problem* p, int n_slots, bool backward) {
  if (!p) return VDA_ERR_NULL;
  const int n_kv = n_slots > 0 ? n_slots : p->n_seqs;
  if (p->T < 1 || p->S < 1 || p->n_seqs < 1 || p->H_q < 1 || p->H_k < 1 || p->H_q % p->H_k) return VDA_ERR_SIZE;
  if ((!p->cu_q && p->T % p->n_seqs) || (!p->cu_k && p->S % n_kv)) return VDA_ERR_SIZE;
  if (!vda::supported_dim(p->d)) return VDA_ERR_UNSUPPORTED;
  if (!is_layout(p->layout) || !is_layout(p->kv_layout) || !is_layout(p->out_layout)) return VDA_ERR_UNSUPPORTED;
  const long long group = p->H_q / p->H_k;
  if (group > 1024) return VDA_ERR_UNSUPPORTED;
  const size_t es = p->is_f32 ? 4 : 2;
  const long long row_q = (long long)p->H_q * p->d, row_k = (long long)p->H_k * p->d;
  // Rows and tiles are counted in 32 bits; a launch has 256 threads a tile, those of dkv_waves() a tile
  // of states backward, and a thread for four channels of a row.
  const long long threads_k = 64 * vda::dkv_waves(p->is_f32 != 0);
  const long long rows = (long long)p->T * group;
  if (rows + 256 > kMaxInt || (long long)p->S + 256 > kMaxInt || row_q * (long long)es >= 1 << 24) return VDA_ERR_SIZE;
  if ((rows / 32 + p->n_seqs + 1) * p->H_k + 8 > kMaxThreads / 256 ||
      ((long long)p->S / 128 + p->n_seqs + 1) * p->H_k + 8 > kMaxThreads / (backward ? threads_k : 256) ||
      ((long long)p->T * p->H_q + 64) * (p->d / 4) > kMaxThreads || ((long long)p->S * p->H_k + 64) * (p->d / 4) > kMaxThreads)
    return VDA_ERR_SIZE;
  for (int st : {check_stride(p->q_row_stride, p->layout, row_q, es), check_stride(p->k_row_stride, p->kv_layout, row_k, es),
                 check_stride(p->v_row_stride, p->kv_layout, row_k, es)})
    if (st != VDA_OK) return st;
  if (backward)
    for (int st : {check_stride(p->dq_row_stride, p->layout, row_q, es), check_stride(p->dk_row_stride, p->kv_layout, row_k, es),
                   check_stride(p->dv_row_stride, p->kv_layout, row_k, es)})
      if (st != VDA_OK) return st;
  if (!aligned(p->cu_q, 4) || !aligned(p->cu_k, 4) || !aligned(p->k_lens, 4)) return VDA_ERR_ALIGN;
  return VDA_OK;
}

// Strides of a tensor of H heads whose sequences are packed, or n of equal length.
CrossStrides strides_of(int layout, bool packed, int total, int n, int H, int d, int row_stride) {
  const size_t row = row_stride ? (size_t)row_stride : (size_t)H * d;
  if (layout == VDA_LAYOUT_TOKENS) return CrossStrides{row, (size_t)d, packed ? 0 : (size_t)(total / n) * row};
  if (packed) return CrossStrides{(size_t)d, (size_t)total * d, 0};
  return CrossStrides{(size_t)d, (size_t)(total / n) * d, (size_t)H * (total / n) * d};
}

struct CrossPlan {
  int few;              // waves of a workgroup of few rows, which share them; 0: many rows
  int tiles, splits;    // of the rows; ranges of the states
  int tiles_k, splits_k, range;  // backward: of the states; ranges of the rows at most, and their rows
  size_t part, part2, stats, counts, total;  // workspace offsets
};

long long tiles_of(bool packed, long long total, int n, long long per_token, int tile) {
  return packed ? total * per_token / tile + n : n * ((total / n * per_token + tile - 1) / tile);
}

CrossPlan plan_of(const vda_cross_problem* p, int n_slots, bool backward) {
  CrossPlan c = {};
  const long long cus = vda::current_device_cus(), group = p->H_q / p->H_k, n = p->n_seqs;
  const long long n_kv = n_slots > 0 ? n_slots : n;
  const long long rows = (long long)p->T * group / n, states = (p->S + n_kv - 1) / n_kv;  // of a sequence, in the mean
  c.few = !backward && rows <= vda::kFewRows;
  const int tile = c.few ? vda::kFewRows : vda::kCrossRows;
  c.tiles = (int)tiles_of(p->cu_q != nullptr, p->T, p->n_seqs, group, tile);
  // Ranges of the states, of two tiles at least, that make two workgroups a CU where there is
  // less than one (64 rows of 40320 states of 16 heads, D = 64: 38 us, 46 us with one a CU, 40 us with
  // four; 200 rows of 8 heads, D = 128: 59, 67 and 67 us; up to 8% behind one a CU where that fits
  // better).  From one a CU on a join costs more than it gives (1560 x 512 of 24 heads 21 and 44 us).
  auto ranges = [&](long long groups, long long units) {
    if (groups >= cus) return 1LL;
    return std::max(1LL, std::min({(2 * cus + groups - 1) / groups, (units + 1) / 2, 64LL}));
  };
  const long long groups_q = (long long)c.tiles * p->H_k;
  const int waves = vda::few_waves(p->is_f32 != 0, p->d);
  if (c.few && groups_q <= cus && states <= 128 * waves) {
    // A workgroup a CU, 128 states a wave: no join to launch.  One sequence of 16 heads and 512
    // states, D = 128: 11.6 us where ranges of single waves and a join took 15.5 us (captured,
    // 9.6 and 9.8 us).  Of 768 states the one launch still takes 12.6 us for 14.3, but captured 17.0
    // for 14.7 (640: 11.6 and 14.4, captured 16.0 and 14.8; 1024: 14.8 and 14.3, captured 19.0 and 14.9;
    // 2048: 23 and 14), and in fp32, two waves, 33 us for 25 at 384 states: so the limit is where it
    // loses in neither.
    c.few = waves;
    c.splits = 1;
  } else if (c.few) {
    // Two waves a CU, of 128 states at least: three a CU unsplit measured 75 us where six and
    // a join took 78 us and twelve 81 us (96 sequences of 8 key heads, 1500 states, D = 128).
    c.splits = (int)std::max(1LL, std::min({(2 * cus + groups_q - 1) / groups_q, (states + 127) / 128, 64LL}));
  } else {
    c.splits = (int)ranges(groups_q, (states + vda::kCrossTile - 1) / vda::kCrossTile);
  }
  const size_t q_rows = (size_t)p->T * p->H_q, k_rows = (size_t)p->S * p->H_k;
  size_t at = 0;
  auto take = [&](size_t bytes) {
    const size_t from = at;
    at = round_up(at + bytes, 256);
    return from;
  };
  if (!backward) {
    if (c.splits > 1) {
      c.part = take(c.splits * q_rows * p->d * 4);
      c.part2 = take(c.splits * q_rows * 8);
    }
  } else {
    c.tiles_k = (int)tiles_of(p->cu_k != nullptr, p->S, p->n_seqs, 1, vda::kCrossRows);
    const long long most = p->cu_q ? (long long)p->T * group : rows;
    const long long groups = (long long)c.tiles_k * p->H_k;
    // Rows of a workgroup of the gradient of k and v.  Fewer groups than CUs: as many ranges as
    // make one workgroup a CU (1560 rows of 512 states of 24 heads 74 us, 100 us with the three a
    // CU of below; 16384 of 16 heads 277 and 310 us).  Otherwise about three a CU, so that
    // sequences of uneven length even out (16401 rows over 9 sequences 386 us, 410 us with one a
    // CU, 420 us with six), of 512 rows at least, as each range's sums are written and added up.
    // Eight ranges at most bound the workspace; where the groups are fewer than an eighth of the CUs these
    // do not fill the device.
    const long long each = groups < cus ? (rows + cus / groups - 1) / (cus / groups) : std::max(512LL, rows * groups / (3 * cus));
    // No longer than the rows that there are, so that a range is an int where they are.
    const long long range = (std::clamp(each, 1LL, std::max(most, 1LL)) + 63) / 64 * 64;
    c.range = (int)range;
    c.splits_k = (int)std::clamp((most + range - 1) / range, 1LL, 8LL);
    c.stats = take(q_rows * 8);
    c.counts = take((size_t)p->S * 4);
    const size_t a = c.splits > 1 ? c.splits * q_rows * p->d * 4 : 0;
    const size_t b = c.splits_k > 1 ? round_up(c.splits_k * k_rows * p->d * 4, 256) : 0;
    c.part = take(std::max(a, 2 * b));
    c.part2 = c.part + b;
  }
  c.total = at;
  return c;
}

CrossArgs args_of(const vda_cross_problem* p, const CrossPlan& c, int n_slots, void* work) {
  CrossArgs a = {};
  const bool pq = p->cu_q != nullptr, pk = p->cu_k != nullptr;
  const int n_kv = n_slots > 0 ? n_slots : p->n_seqs;
  a.sq = strides_of(p->layout, pq, p->T, p->n_seqs, p->H_q, p->d, p->q_row_stride);
  a.sdq = strides_of(p->layout, pq, p->T, p->n_seqs, p->H_q, p->d, p->dq_row_stride);
  a.so = strides_of(p->out_layout, pq, p->T, p->n_seqs, p->H_q, p->d, 0);
  a.sk = strides_of(p->kv_layout, pk, p->S, n_kv, p->H_k, p->d, p->k_row_stride);
  a.sv = strides_of(p->kv_layout, pk, p->S, n_kv, p->H_k, p->d, p->v_row_stride);
  a.sdk = strides_of(p->kv_layout, pk, p->S, n_kv, p->H_k, p->d, p->dk_row_stride);
  a.sdv = strides_of(p->kv_layout, pk, p->S, n_kv, p->H_k, p->d, p->dv_row_stride);
  a.cu_q = p->cu_q, a.cu_k = p->cu_k, a.k_lens = p->k_lens, a.k_mask = p->k_mask;
  a.n = p->n_seqs, a.n_slots = n_kv, a.T = p->T, a.S = p->S;
  a.Lq = pq ? 0 : p->T / p->n_seqs, a.Lk = pk ? 0 : p->S / n_kv;
  a.Hq = p->H_q, a.Hk = p->H_k, a.group = p->H_q / p->H_k;
  a.group_magic = (uint32_t)(((1u << 24) + a.group - 1) / a.group);
  a.scale = p->scale, a.flip = p->scale < 0.f;
  // Above 0, so that a score of -inf has no weight; a scale of 0 is 1e-37, below what fp32 tells from it.
  a.s = std::max(a.flip ? -p->scale : p->scale, 1e-37f), a.c = std::max(a.s * vda::kLog2e, 1e-37f);
  auto near = [&](const CrossStrides& s) { return (64 * s.tok + a.group * s.head) * (p->is_f32 ? 4 : 2) < (size_t)1 << 31; };
  a.near = near(a.sq) && near(a.so);
  // With heads that share out evenly over the 8 XCDs: of 5 heads, 24 sequences of 1000 x 600 took 64 us sorted, 53 us not,
  // and uneven ones between 0.92 and 1.09 of the time; of 12 heads nothing gained.
  a.sorted = pq && pk && p->n_seqs < 64 && !c.few && (p->H_k % 8 == 0 || 8 % p->H_k == 0);
  // Less than a workgroup a CU in the gradient of q: products are cheap then, and what roundings leave does not average out.
  a.fine = !p->is_f32 && (long long)c.tiles * p->H_k < vda::current_device_cus();
  a.tiles = c.tiles, a.splits = c.splits;
  char* w = static_cast<char*>(work);
  a.part = reinterpret_cast<float*>(w + c.part);
  a.part2 = reinterpret_cast<float*>(w + c.part2);
  a.stats = reinterpret_cast<float2*>(w + c.stats);
  a.counts = reinterpret_cast<int*>(w + c.counts);
  a.range = c.range;
  return a;
}

Range opt_range(const void* p, size_t bytes) { return range_of(p, p ? bytes : 0); }

// From the first to the last byte of a tensor of `rows` tokens.
Range tensor_range(const void* p, int layout, size_t tokens, int H, int d, int stride, size_t es) {
  const size_t row = (size_t)H * d;
  if (layout == VDA_LAYOUT_HEADS || stride == 0) return range_of(p, tokens * row * es);
  return range_of(p, ((tokens - 1) * stride + row) * es);
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

int forward(const vda_cross_problem* p, const void* q, const void* k, const void* v, const int* slots, int n_slots, void* out,
            float* lse, void* work, hipStream_t stream) {
  const int st = check_problem(p, n_slots, false);
  if (st != VDA_OK) return st;
  const CrossPlan c = plan_of(p, n_slots, false);
  if (c.total && !work) return VDA_ERR_NULL;
  if (!c.total) work = nullptr;
  if (!aligned(q, 16) || !aligned(k, 16) || !aligned(v, 16) || !aligned(out, 16) || !aligned(work, 16) || !aligned(lse, 4) ||
      !aligned(slots, 4))
    return VDA_ERR_ALIGN;
  const size_t es = p->is_f32 ? 4 : 2;
  const int n_kv = n_slots > 0 ? n_slots : p->n_seqs;
  if (any_overlap({tensor_range(out, p->out_layout, p->T, p->H_q, p->d, 0, es), opt_range(lse, (size_t)p->T * p->H_q * 4),
                   opt_range(work, c.total)},
                  {tensor_range(q, p->layout, p->T, p->H_q, p->d, p->q_row_stride, es),
                   tensor_range(k, p->kv_layout, p->S, p->H_k, p->d, p->k_row_stride, es),
                   tensor_range(v, p->kv_layout, p->S, p->H_k, p->d, p->v_row_stride, es),
                   opt_range(p->cu_q, (size_t)(p->n_seqs + 1) * 4), opt_range(p->cu_k, (size_t)(p->n_seqs + 1) * 4),
                   opt_range(p->k_lens, (size_t)n_kv * 4), opt_range(p->k_mask, p->S),
                   opt_range(slots, (size_t)p->n_seqs * 4)}))
    return VDA_ERR_OVERLAP;
  CrossArgs a = args_of(p, c, n_slots, work);
  a.q = q, a.k = k, a.v = v, a.out = out, a.lse = lse, a.slots = slots;
  hipError_t e = vda::launch_cross_forward(p->is_f32 != 0, p->d, c.few, a, stream);
  if (e == hipSuccess && c.splits > 1) e = vda::launch_cross_join(p->is_f32 != 0, p->d, a, stream);
  return hip_status(e);
}

int check_step(const vda_cross_problem* p, int n_slots) {
  if (!p) return VDA_ERR_NULL;
  if (n_slots < 1 || p->cu_q || p->cu_k) return VDA_ERR_SIZE;
  return VDA_OK;
}

}  // namespace

extern "C" {

size_t vda_cross_forward_workspace(const vda_cross_problem* p) {
  return check_problem(p, 0, false) == VDA_OK ? plan_of(p, 0, false).total : 0;
}

size_t vda_cross_backward_workspace(const vda_cross_problem* p) {
  return check_problem(p, 0, true) == VDA_OK ? plan_of(p, 0, true).total : 0;
}

size_t vda_cross_step_workspace(const vda_cross_problem* p, int n_slots) {
  if (check_step(p, n_slots) != VDA_OK || check_problem(p, n_slots, false) != VDA_OK) return 0;
  return plan_of(p, n_slots, false).total;
}

int vda_cross_forward(const vda_cross_problem* p, const void* q, const void* k, const void* v, void* out, float* lse, void* work,
                      hipStream_t stream) {
  if (!p || !q || !k || !v || !out) return VDA_ERR_NULL;
  return forward(p, q, k, v, nullptr, 0, out, lse, work, stream);
}

int vda_cross_step(const vda_cross_problem* p, const void* q, const void* k, const void* v, const int* slots, int n_slots,
                   void* out, void* work, hipStream_t stream) {
  if (!p || !q || !k || !v || !out) return VDA_ERR_NULL;
  const int st = check_step(p, n_slots);
  if (st != VDA_OK) return st;
  if (!slots && p->n_seqs > n_slots) return VDA_ERR_SIZE;
  return forward(p, q, k, v, slots, n_slots, out, nullptr, work, stream);
}

int vda_cross_backward(const vda_cross_problem* p, const void* dout, const void* q, const void* k, const void* v, const void* out,
                       const float* lse, void* dq, void* dk, void* dv, void* work, hipStream_t stream) {
  if (!p || !dout || !q || !k || !v || !out || !lse || !dq || !dk || !dv || !work) return VDA_ERR_NULL;
  const int st = check_problem(p, 0, true);
  if (st != VDA_OK) return st;
  for (const void* t : {dout, q, k, v, out, (const void*)dq, (const void*)dk, (const void*)dv, (const void*)work})
    if (!aligned(t, 16)) return VDA_ERR_ALIGN;
  if (!aligned(lse, 4)) return VDA_ERR_ALIGN;
  const CrossPlan c = plan_of(p, 0, true);
  const size_t es = p->is_f32 ? 4 : 2;
  const Range rdk = tensor_range(dk, p->kv_layout, p->S, p->H_k, p->d, p->dk_row_stride, es);
  const Range rdv = tensor_range(dv, p->kv_layout, p->S, p->H_k, p->d, p->dv_row_stride, es);
  const Range both = Range{std::min(rdk.lo, rdv.lo), std::max(rdk.hi, rdv.hi)};
  const bool meet = overlaps(rdk, rdv);
  if (meet && !vda::slices_apart(dk, p->dk_row_stride, dv, p->dv_row_stride, (size_t)p->H_k * p->d * es, es)) return VDA_ERR_OVERLAP;
  const std::initializer_list<Range> ins = {
      tensor_range(dout, p->out_layout, p->T, p->H_q, p->d, 0, es), tensor_range(out, p->out_layout, p->T, p->H_q, p->d, 0, es),
      tensor_range(q, p->layout, p->T, p->H_q, p->d, p->q_row_stride, es),
      tensor_range(k, p->kv_layout, p->S, p->H_k, p->d, p->k_row_stride, es),
      tensor_range(v, p->kv_layout, p->S, p->H_k, p->d, p->v_row_stride, es), range_of(lse, (size_t)p->T * p->H_q * 4),
      opt_range(p->cu_q, (size_t)(p->n_seqs + 1) * 4), opt_range(p->cu_k, (size_t)(p->n_seqs + 1) * 4),
      opt_range(p->k_lens, (size_t)p->n_seqs * 4), opt_range(p->k_mask, p->S)};
  const Range rdq = tensor_range(dq, p->layout, p->T, p->H_q, p->d, p->dq_row_stride, es), rw = range_of(work, c.total);
  if (meet ? any_overlap({rdq, both, rw}, ins) : any_overlap({rdq, rdk, rdv, rw}, ins)) return VDA_ERR_OVERLAP;
  CrossArgs a = args_of(p, c, 0, work);
  a.q = q, a.k = k, a.v = v, a.o = out, a.dout = dout, a.lse_in = lse;
  a.dq = dq, a.dk = dk, a.dv = dv;
  const bool f32 = p->is_f32 != 0;
  hipError_t e = vda::launch_cross_dq(f32, p->d, a, stream);
  if (e == hipSuccess && c.splits > 1)
    e = vda::launch_cross_sum(
        f32, p->d, vda::CrossSum{{a.part}, nullptr, {dq}, {a.sdq}, a.cu_q, a.n, a.Lq, a.Hq, a.splits, (long long)a.T * a.Hq}, stream);
  // Most of these workgroups have no range and end at once: for them the order's search would cost more than it gives.
  a.tiles = c.tiles_k, a.splits = c.splits_k, a.sorted = 0;
  if (e == hipSuccess) e = vda::launch_cross_dkv(f32, p->d, a, stream);
  if (e == hipSuccess && c.splits_k > 1)
    e = vda::launch_cross_sum(f32, p->d, vda::CrossSum{{a.part, a.part2}, a.counts, {dk, dv}, {a.sdk, a.sdv}, a.cu_k, a.n, a.Lk, a.Hk,
                                                       a.splits, (long long)a.S * a.Hk}, stream);
  return hip_status(e);
}

}  // extern "C"
