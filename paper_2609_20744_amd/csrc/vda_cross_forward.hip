// Cross attention to an encoder's states: the forward pass, for whole sequences
// and for a few tokens of each (vda.h, vda_cross_forward, vda_cross_step), and
// the join of states that several workgroups shared.
//
// One pass over the states with the running maximum and sum of the softmax
// (vda_cross.h has the operands).  Per 64 states and 32 rows a wave makes
//     S^T = K Q^T -> p = 2^(c s - m) -> O^T += V^T P^T,
// all in registers: a lane has one row's column of S^T and of O^T, so the
// maximum, the sum and the scaling of O are its own, and the rounded p are the
// next product's operand as they stand.  The maximum is taken up where it grew by
// more than 2^8 only: p stays below 2^8 then, where a rounding to bf16 is as good.
//
// Many rows: a wave has 32 rows, the four waves of a workgroup share the states'
// tiles.  Few rows (a step): a wave by itself, bound by the copies that it has on the way.
// Where workgroups would not fill the device, each takes a range of the states
// and the join kernel adds their parts.
#include "vda_cross.h"

namespace vda {
namespace {

constexpr float kGrow = 8.f;  // in powers of two

// The softmax's part of a tile of 32 NB states, and its product with V.  FINE: p in two parts,
// rounded and rest (bf16).
template <bool F32, int D, int NB, bool FINE>
__device__ __forceinline__ void attend(const lds_char* kt, const lds_char* vt, const typename Frag<F32>::X (&q)[D / 16], uint64_t bits,
                                       bool all, float c, floatx16 (&o)[D / 32], float& m, float& l,
                                       const typename CrossTile<F32, D>::Lane& at) {
  typedef Frag<F32> Fr;
  typedef CrossTile<F32, D> Tile;
  floatx16 s[NB];
#pragma unroll
  for (int b = 0; b < NB; ++b) s[b] = floatx16{};
#pragma unroll
  for (int e = 0; e < D / 16; ++e)
#pragma unroll
    for (int b = 0; b < NB; ++b) s[b] = Fr::mma(Tile::row_frag(kt + 32 * b * Tile::kRow, e, at), q[e], s[b]);
  if (!all) {
#pragma unroll
    for (int b = 0; b < NB; ++b) {
      const uint32_t w = (uint32_t)(bits >> 32 * b) >> (threadIdx.x & 32) / 8;
#pragma unroll
      for (int i = 0; i < 16; ++i) s[b][i] = row_or(s[b][i], w, i, -INFINITY);
    }
  }
  float top = s[0][0];
#pragma unroll
  for (int b = 0; b < NB; ++b)
#pragma unroll
    for (int i = 0; i < 16; ++i) top = fmaxf(top, s[b][i]);
  top = fmaxf(top, other_half(top));
  top *= c;
  if (__any(top > m + kGrow)) {
    const float to = top > m + kGrow ? top : m;
    const float f = to == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m - to);
    m = to;
    l *= f;
#pragma unroll
    for (int b = 0; b < D / 32; ++b) o[b] *= f;
  }
  const float from = m == -INFINITY ? 0.f : m;
#pragma unroll
  for (int b = 0; b < NB; ++b) {
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      s[b][i] = __builtin_amdgcn_exp2f(fmaf(s[b][i], c, -from));  // c > 0: 0 where s is -inf
      l += s[b][i];
    }
  }
#pragma unroll
  for (int b = 0; b < NB; ++b)
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const typename Fr::X p = Fr::of(s[b], t);
#pragma unroll
      for (int e = 0; e < D / 32; ++e) o[e] = Fr::mma(Tile::col_frag(vt + (32 * b + 16 * t) * Tile::kRow, e, at), p, o[e]);
      if constexpr (FINE && !F32) {
        const typename Fr::X y = Fr::rest(s[b], t);
#pragma unroll
        for (int e = 0; e < D / 32; ++e) o[e] = Fr::mma(Tile::col_frag(vt + (32 * b + 16 * t) * Tile::kRow, e, at), y, o[e]);
      }
    }
}

// In 64 bits, the sum's power of two apart: rounded once, where it is stored.
__device__ __forceinline__ float lse_of(float m, float l) {
  if (l == 0.f) return -INFINITY;
  const double power = (double)m + __builtin_amdgcn_frexp_expf(l);
  return (float)((power + __builtin_amdgcn_logf(__builtin_amdgcn_frexp_mantf(l))) * 0.69314718055994530942);
}

// Where a lane's row goes: to the output, or (not divided by the sum) to its split's part.
template <bool F32, int D>
struct Put {
  const CrossArgs& a;
  const Row& row;
  float m, l, r;
  size_t part;
  __device__ __forceinline__ Put(const CrossArgs& a, const Row& row, float m, float l)
      : a(a), row(row), m(m), l(l), r(l == 0.f ? 0.f : 1.f / l), part((size_t)blockIdx.y * ((size_t)a.T * a.Hq) + row.part) {}
  __device__ __forceinline__ void channels(int first, floatx4 x) const {
    if (a.splits > 1)
      *reinterpret_cast<floatx4*>(a.part + part * D + first) = x;
    else
      store4<F32>(a.out, row.out + first, x * r);
  }
  __device__ __forceinline__ void stats() const {
    if (a.splits > 1)
      *reinterpret_cast<float2*>(a.part2 + part * 2) = make_float2(m, l);
    else if (a.lse != nullptr)
      a.lse[row.lse] = lse_of(m, l);
  }
};

template <bool F32, int D>
__device__ __forceinline__ void put_rows(const CrossArgs& a, const Row& row, const floatx16 (&o)[D / 32], float m, float l,
                                         int lane) {
  const Put<F32, D> put(a, row, m, l);
#pragma unroll
  for (int e = 0; e < D / 32; ++e)
#pragma unroll
    for (int i = 0; i < 4; ++i)
      put.channels(32 * e + 8 * i + 4 * (lane >> 5), floatx4{o[e][4 * i], o[e][4 * i + 1], o[e][4 * i + 2], o[e][4 * i + 3]});
  if (lane < 32) put.stats();
}

// Many rows: 128 of them, 32 a wave, and tiles of 64 states in two places of LDS, the next one
// copied while one is used.  q and the output go through LDS too, so that memory is asked
// for whole rows (with 16 bytes of each of 32 rows to an instruction 264 us instead of 251).  Two
// workgroups a CU: 229 registers a wave.  Bound by the products and the exponentials beside
// them, in sequences of few tiles by memory too, which is hardly overlapped: 32760 x 4096 of 24
// heads, D = 128, 1086 TFLOP/s (8192^3 by the library: 1115), 32760 x 512 247 to 257 us, 835 to 800 TFLOP/s,
// of which about 80 us are q and the output; fp32 108 to 115 TFLOP/s (139).  Several tiles of rows
// a workgroup, without or with q loaded ahead, and first workgroups that start at other times
// changed nothing or spilled.
template <bool F32, int D>
__global__ __launch_bounds__(kThreads, F32 ? 1 : 2) void cross_forward_kernel(CrossArgs a) {
  typedef Frag<F32> Fr;
  typedef CrossTile<F32, D> Tile;
  constexpr int kTileBytes = kCrossTile * Tile::kRow;
  __shared__ __align__(16) char k0[kTileBytes], v0[kTileBytes], k1[kTileBytes], v1[kTileBytes];
  const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6);
  CrossSeq s;
  int hk, place, tile;
  if (!place_of(a, hk, place)) return;
  if (!seq_of_tile<false>(a, kCrossRows, place, s, tile)) return;
  const int r0 = tile * kCrossRows;
  if (r0 >= s.lq * a.group) return;
  const int rows = s.lq * a.group, w0 = r0 + wave * 32;

  // The range of states of this split, in tiles.
  const int tiles = (s.seen + kCrossTile - 1) / kCrossTile, per = (tiles + a.splits - 1) / a.splits;
  const int from = per * (int)blockIdx.y, to = from + per < tiles ? from + per : tiles;
  const char* kb = (const char*)a.k + (seq_base(a.sk, a.cu_k, s.k0, s.kv) + (size_t)hk * a.sk.head) * Tile::kEs;
  const char* vb = (const char*)a.v + (seq_base(a.sv, a.cu_k, s.k0, s.kv) + (size_t)hk * a.sv.head) * Tile::kEs;
  const uint8_t* mask = a.k_mask == nullptr ? nullptr : a.k_mask + (a.cu_k != nullptr ? (size_t)s.k0 : (size_t)s.kv * a.Lk);

  typename Fr::X q[D / 16];
  floatx16 o[D / 32];
#pragma unroll
  for (int e = 0; e < D / 32; ++e) o[e] = floatx16{};
  float m = -INFINITY, l = 0.f;
  uint8_t byte = 1;
  const typename Tile::Lane offs = Tile::lane_of(lane);

  auto copy = [&](int t, lds_char* kt, lds_char* vt) {
    const int first = t * kCrossTile, last = s.seen - 1 - first;
    copy_states<F32, D, kCrossTile, 4>(kb + (size_t)first * a.sk.tok * Tile::kEs, a.sk.tok, last, kt, wave, lane);
    copy_states<F32, D, kCrossTile, 4>(vb + (size_t)first * a.sv.tok * Tile::kEs, a.sv.tok, last, vt, wave, lane);
    if (mask != nullptr) byte = mask[first + (lane < last ? lane : last)];
  };
  // Tile t, whose copies are there when it begins; the next one's begin behind the barrier.
  auto step = [&](int t, lds_char* kt, lds_char* vt, lds_char* next_k, lds_char* next_v) {
    copies_landed();
    const uint64_t bits = seen_bits(s.seen - t * kCrossTile, mask != nullptr, byte, lane);
    if (mask != nullptr && ~bits != 0) clear_copied<F32, D, kCrossTile, 4>(bits, wave, lane, vt);
    lds_barrier();
    if (t + 1 < to) copy(t + 1, next_k, next_v);
    if (bits != 0) attend<F32, D, 2, false>(kt, vt, q, bits, ~bits == 0, a.c, o, m, l, offs);
  };
  // A wave's part of two tiles' places: its q comes and its output goes through it.
  auto part = [&](lds_char* kt, lds_char* vt) { return (wave < 2 ? kt : vt) + (wave & 1) * 32 * Tile::kRow; };
  if (from < to) {
    lds_char* mine = part((lds_char*)k1, (lds_char*)v1);
    const int r = w0 < rows ? w0 : rows - 1;
    const size_t qb = seq_base(a.sq, a.cu_q, s.q0, s.i) + (size_t)hk * a.group * a.sq.head;
    copy_rows<F32, D, 32, 1>(a, (const char*)a.q + qb * Tile::kEs, a.sq, r, rows - 1 - r, mine, 0, lane);
    copy(from, (lds_char*)k0, (lds_char*)v0);
    copies_landed();
#pragma unroll
    for (int e = 0; e < D / 16; ++e) {
      q[e] = Tile::row_frag(mine, e, offs);
      if (a.flip) q[e] = Fr::flip(q[e]);
    }
    for (int t = from; t < to; t += 2) {
      step(t, (lds_char*)k0, (lds_char*)v0, (lds_char*)k1, (lds_char*)v1);
      if (t + 1 < to) step(t + 1, (lds_char*)k1, (lds_char*)v1, (lds_char*)k0, (lds_char*)v0);
    }
  }
  l += other_half(l);
  if (w0 >= rows) return;
  const Row row = row_of(a, s, hk, w0 + (lane & 31));
  if (a.splits > 1) {
    if (row.real) put_rows<F32, D>(a, row, o, m, l, lane);
    return;
  }
  const bool odd = (to - from) & 1;  // the last tile's places were k0 and v0
  lds_char* mine = from < to && !odd ? part((lds_char*)k0, (lds_char*)v0) : part((lds_char*)k1, (lds_char*)v1);
  const size_t ob = seq_base(a.so, a.cu_q, s.q0, s.i) + (size_t)hk * a.group * a.so.head;
  store_rows<F32, D>(a, (uint16_t*)a.out + ob * (Tile::kEs / 2), a.so, w0, rows, o, l == 0.f ? 0.f : 1.f / l, mine, lane);
  if (a.lse != nullptr && row.real && lane < 32) a.lse[row.lse] = lse_of(m, l);
}

// Few rows: a wave with 32 rows takes tiles of 32 states through two places in LDS, one on
// the way while the other is used, with no barrier.  WAVES of them share a workgroup's
// rows, take a part of its range each and add their parts behind a barrier; of the few states
// that these have p enters the product in two parts (out 1.7e-3 of its norm off instead of
// 2.3e-3, 11.7 and 11.8 us for 512 states of 16 heads; of the long ones it would be 78 us for 76).  Bound by
// the states' bytes: 96 sequences of 8 key heads and 1130 states in the mean, D = 128, 76 us, 300 MB
// at 3.95 TB/s (two waves that share a place and a barrier 83 us, four places of one wave 98).
constexpr int kFewStates = 32;

template <bool F32, int D, bool MASKED, int WAVES>
__global__ __launch_bounds__(64 * WAVES, 1) void cross_few_kernel(CrossArgs a) {
  typedef Frag<F32> Fr;
  typedef CrossTile<F32, D> Tile;
  constexpr int kBytes = kFewStates * Tile::kRow, kCopies = 2 * kBytes / 1024;
  __shared__ __align__(16) char ks0[WAVES * kBytes], vs0[WAVES * kBytes], ks1[WAVES * kBytes], vs1[WAVES * kBytes];
  const int lane = threadIdx.x & 63, wave = WAVES == 1 ? 0 : uniform(threadIdx.x >> 6);
  lds_char* const k0 = (lds_char*)ks0 + wave * kBytes;
  lds_char* const v0 = (lds_char*)vs0 + wave * kBytes;
  lds_char* const k1 = (lds_char*)ks1 + wave * kBytes;
  lds_char* const v1 = (lds_char*)vs1 + wave * kBytes;
  const int hk = uniform(blockIdx.x % (unsigned)a.Hk);
  CrossSeq s;
  int tile;
  if (!seq_of_tile<false>(a, kFewRows, blockIdx.x / (unsigned)a.Hk, s, tile)) return;
  const int r0 = tile * kFewRows;
  if (r0 >= s.lq * a.group) return;
  const Row row = row_of(a, s, hk, r0 + (lane & 31));

  const int tiles = (s.seen + kFewStates - 1) / kFewStates, per = (tiles + a.splits - 1) / a.splits;
  const int first = per * (int)blockIdx.y, behind = first + per < tiles ? first + per : tiles;
  const int each = (behind - first + WAVES - 1) / WAVES, from = first + wave * each;
  const int to = WAVES == 1 || from + each > behind ? behind : from + each;
  const char* kb = (const char*)a.k + (seq_base(a.sk, a.cu_k, s.k0, s.kv) + (size_t)hk * a.sk.head) * Tile::kEs;
  const char* vb = (const char*)a.v + (seq_base(a.sv, a.cu_k, s.k0, s.kv) + (size_t)hk * a.sv.head) * Tile::kEs;
  const uint8_t* mask = !MASKED ? nullptr : a.k_mask + (a.cu_k != nullptr ? (size_t)s.k0 : (size_t)s.kv * a.Lk);

  typename Fr::X q[D / 16];
#pragma unroll
  for (int e = 0; e < D / 16; ++e) {
    q[e] = Fr::load(a.q, row.q + 16 * e + 8 * (lane >> 5));
    if (a.flip) q[e] = Fr::flip(q[e]);
  }
  floatx16 o[D / 32];
#pragma unroll
  for (int e = 0; e < D / 32; ++e) o[e] = floatx16{};
  float m = -INFINITY, l = 0.f;
  uint8_t b0 = 0, b1 = 0;  // the mask's bytes of the tiles
  const typename Tile::Lane offs = Tile::lane_of(lane);

  auto copy = [&](int t, lds_char* kt, lds_char* vt, uint8_t& byte) {
    const int first = (t < to ? t : to - 1) * kFewStates, last = s.seen - 1 - first;
    if (MASKED) byte = mask[first + (lane < last ? lane : last)];
    copy_states<F32, D, kFewStates, 1>(kb + (size_t)first * a.sk.tok * Tile::kEs, a.sk.tok, last, kt, 0, lane);
    copy_states<F32, D, kFewStates, 1>(vb + (size_t)first * a.sv.tok * Tile::kEs, a.sv.tok, last, vt, 0, lane);
  };
  auto step = [&](int t, lds_char* kt, lds_char* vt, uint8_t byte) {
    __builtin_amdgcn_sched_barrier(0);
    // All copies but those of the next tile, the newest ones, have landed.
    __builtin_amdgcn_s_waitcnt((kCopies & 15) | 0x0f70 | (kCopies >> 4 << 14));
    __builtin_amdgcn_sched_barrier(0);
    const uint64_t bits = seen_bits(s.seen - t * kFewStates, MASKED, byte, lane) & 0xffffffffull;
    const bool all = bits == 0xffffffffull;
    if (bits != 0) {
      if (MASKED && !all) clear_copied<F32, D, kFewStates, 1>(bits, 0, lane, vt);
      attend<F32, D, 1, (WAVES > 1)>(kt, vt, q, bits, all, a.c, o, m, l, offs);
    }
    __builtin_amdgcn_sched_barrier(0);
  };
  if (from < to) {
    // Each step has the copies of one more tile on the way, behind the last one that one's
    // again: where not every way through had them, the compiler could not count them and
    // would wait for all before each read.
    copy(from, k0, v0, b0);
    for (int t = from;; t += 2) {
      copy(t + 1, k1, v1, b1);
      step(t, k0, v0, b0);
      if (t + 1 >= to) break;
      copy(t + 2, k0, v0, b0);
      step(t + 1, k1, v1, b1);
      if (t + 2 >= to) break;
    }
    copies_landed();
  }
  l += other_half(l);
  if constexpr (WAVES == 1) {
    if (row.real) put_rows<F32, D>(a, row, o, m, l, lane);
  } else {
    // o goes to the wave's own places, 16 bytes a lane in the lanes' order; then each wave
    // adds a share of the channels up, in the waves' order.
    __shared__ float2 stats[WAVES][32];
    auto place = [&](int w, int block) -> Lds<floatx4>* {  // 4 channels of 32 rows
      const int byte = block * 512;
      return (Lds<floatx4>*)((byte < kBytes ? (lds_char*)ks0 + w * kBytes + byte : (lds_char*)vs0 + w * kBytes + byte - kBytes) +
                             (lane & 31) * 16);
    };
#pragma unroll
    for (int e = 0; e < D / 32; ++e)
#pragma unroll
      for (int i = 0; i < 4; ++i)
        *place(wave, 8 * e + 2 * i + (lane >> 5)) = floatx4{o[e][4 * i], o[e][4 * i + 1], o[e][4 * i + 2], o[e][4 * i + 3]};
    if (lane < 32) stats[wave][lane] = make_float2(m, l);
    lds_barrier();
    float2 each_of[WAVES];
    float top = -INFINITY, sum = 0.f;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) each_of[w] = stats[w][lane & 31], top = fmaxf(top, each_of[w].x);
#pragma unroll
    for (int w = 0; w < WAVES; ++w) {
      each_of[w].x = each_of[w].x == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(each_of[w].x - top);
      sum += each_of[w].x * each_of[w].y;
    }
    if (!row.real) return;
    const Put<F32, D> put(a, row, top, sum);
    for (int b = 2 * wave + (lane >> 5); b < D / 4; b += 2 * WAVES) {
      floatx4 x = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int w = 0; w < WAVES; ++w) x += each_of[w].x * *place(w, b);
      put.channels(4 * b, x);
    }
    if (wave == 0 && lane < 32) put.stats();
  }
}

// Adds the parts of a row's splits: a wave per row, whose lanes have a split's maximum
// and sum each, and then four channels of every 256 / D-th split; the order is fixed.  A
// launch and two waits for memory: 5 us for 2048 rows of 16 splits, D = 64 (a thread per
// four channels 8 us).
template <bool F32, int D>
__global__ __launch_bounds__(kThreads) void cross_join_kernel(CrossArgs a) {
  constexpr int LANES = D / 4, SIDE = 64 / LANES;  // splits side by side
  const int lane = threadIdx.x & 63;
  const size_t rows = (size_t)a.T * a.Hq, R = (size_t)blockIdx.x * 4 + uniform(threadIdx.x >> 6);
  if (R >= rows) return;
  const int tok = uniform((int)(R / (unsigned)a.Hq)), h = uniform((int)(R - (size_t)tok * a.Hq));
  size_t out, lse;
  if (a.cu_q != nullptr) {
    if (tok < clamp_to(a.cu_q[0], 0, a.T) || tok >= clamp_to(a.cu_q[a.n], 0, a.T)) return;
    out = (size_t)tok * a.so.tok + (size_t)h * a.so.head;
    lse = (size_t)h * a.T + tok;
  } else {
    const int i = uniform(tok / a.Lq), t = tok - i * a.Lq;
    if (a.slots != nullptr && (a.slots[i] < 0 || a.slots[i] >= a.n_slots)) return;
    out = (size_t)i * a.so.seq + (size_t)t * a.so.tok + (size_t)h * a.so.head;
    lse = ((size_t)i * a.Hq + h) * a.Lq + t;
  }
  const float2* ml = reinterpret_cast<const float2*>(a.part2);
  const float2 mine = lane < a.splits ? ml[lane * rows + R] : make_float2(-INFINITY, 0.f);
  float top = mine.x;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) top = fmaxf(top, __shfl_xor(top, d));
  const float f = mine.x == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(mine.x - top);
  float sum = mine.x == -INFINITY ? mine.y : f * mine.y;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) sum += __shfl_xor(sum, d);
  const int chan = lane % LANES * 4, side = lane / LANES;
  floatx4 x = {0.f, 0.f, 0.f, 0.f};
  for (int b = side; b - side < a.splits; b += 4 * SIDE) {
    floatx4 z[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const int p = b + u * SIDE < a.splits ? b + u * SIDE : a.splits - 1;
      z[u] = *reinterpret_cast<const floatx4*>(a.part + (p * rows + R) * D + chan);
    }
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const float w = __shfl(f, b + u * SIDE & 63);
      x += (b + u * SIDE < a.splits ? w : 0.f) * z[u];
    }
  }
#pragma unroll
  for (int d = LANES; d < 64; d <<= 1)
#pragma unroll
    for (int e = 0; e < 4; ++e) x[e] += __shfl_xor(x[e], d);
  if (side == 0) store4<F32>(a.out, out + chan, x * (sum == 0.f ? 0.f : 1.f / sum));
  if (a.lse != nullptr && lane == 0) a.lse[lse] = lse_of(top, sum);
}

template <bool F32, int D, int WAVES>
void few_rows(const CrossArgs& a, hipStream_t stream) {
  const dim3 grid((unsigned)a.tiles * a.Hk, a.splits);
  if (a.k_mask != nullptr)
    cross_few_kernel<F32, D, true, WAVES><<<grid, 64 * WAVES, 0, stream>>>(a);
  else
    cross_few_kernel<F32, D, false, WAVES><<<grid, 64 * WAVES, 0, stream>>>(a);
}

template <bool F32, int D>
hipError_t forward(int few, const CrossArgs& a, hipStream_t stream) {
  if (few == 1) {
    few_rows<F32, D, 1>(a, stream);
  } else if (few != 0) {
    few_rows<F32, D, few_waves(F32, D)>(a, stream);
  } else {
    const unsigned grid = ((unsigned)a.tiles * a.Hk + 7) / 8 * 8;
    cross_forward_kernel<F32, D><<<dim3(grid, a.splits), kThreads, 0, stream>>>(a);
  }
  return hipGetLastError();
}

template <bool F32, int D>
hipError_t join(const CrossArgs& a, hipStream_t stream) {
  cross_join_kernel<F32, D><<<(unsigned)(((size_t)a.T * a.Hq + 3) / 4), kThreads, 0, stream>>>(a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_cross_forward(bool f32, int d, int few, const CrossArgs& a, hipStream_t stream) {
  switch (d) {
    case 32: return f32 ? forward<true, 32>(few, a, stream) : forward<false, 32>(few, a, stream);
    case 64: return f32 ? forward<true, 64>(few, a, stream) : forward<false, 64>(few, a, stream);
    default: return f32 ? forward<true, 128>(few, a, stream) : forward<false, 128>(few, a, stream);
  }
}

hipError_t launch_cross_join(bool f32, int d, const CrossArgs& a, hipStream_t stream) {
  switch (d) {
    case 32: return f32 ? join<true, 32>(a, stream) : join<false, 32>(a, stream);
    case 64: return f32 ? join<true, 64>(a, stream) : join<false, 64>(a, stream);
    default: return f32 ? join<true, 128>(a, stream) : join<false, 128>(a, stream);
  }
}

}  // namespace vda
