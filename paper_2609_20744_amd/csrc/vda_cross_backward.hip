// Cross attention to an encoder's states: the gradients (vda.h,
// vda_cross_backward).  With p_j = 2^(c s_j - lse) made again from q, k and the
// kept lse, and D = sum dout o over a row's channels,
//     dP_j = dout . v_j,  dS_j = p_j (dP_j - D),
//     dq = scale sum_j dS_j k_j,  dk_j = scale sum_r dS_j q_r,  dv_j = sum_r p_j dout_r.
//
// Two kernels, each with its own sums in registers and no atomics: one goes along
// the states for 128 rows (dq, and D and lse of each row for the other), one along
// the rows for 128 states (dk and dv).  Scores and dP are made in both, seven
// products where one kernel would need five, and a sum over the other side's
// workgroups.  The rows of all query heads of a key head are one sequence of rows
// (vda_cross.h), so the gradients of shared heads are ordinary sums.  Where a
// side's tiles are too few to fill the device, the other side is cut into ranges,
// whose fp32 sums are added in their order.
#include "vda_cross.h"

namespace vda {
namespace {

// A score's weight.  lse in powers of two; in fp32 as it is kept, as its rounding in other units would
// be one more in every weight of a row (dk and dv of 60000 states: 9e-7 of their norm off).
template <bool F32>
__device__ __forceinline__ float weight_of(const CrossArgs& a, float score, float lse) {
  return __builtin_amdgcn_exp2f(F32 ? fmaf(score, a.s, -lse) * kLog2e : fmaf(score, a.c, -lse));
}

// D is summed from p dP in a pass before, in fp32, where at most kExactTiles tiles have a state that is
// seen, and of at most kExactStates wherever a mask leaves them.  As dout out it has
// the rounding of out, whose part in dS is as large as the others where a few states share
// the weight: of 2, 5, 30 and 60 states that are seen dq and dk were 4.5, 3.1, 2.6 and 2.5e-3 of their norm
// off (bf16, D = 128), 2.4e-3 with this pass; of 65 to 200 scattered ones 2.5e-3, of 500 and more 2.4e-3
// without it.
// It is two products more: 1560 rows x 128 states of 24 heads 42 -> 47 us, 32760 x 226 488 -> 592 us
// for the whole backward pass.  A state that is seen alone leaves dS = 0, not a remainder; in fp32,
// whose error the rounding does not show in, that is all the pass is for.
// Where the rows do not fill the device either (`fine`), p and dS of sequences of up to kExactTiles
// tiles enter their products in two parts, rounded and rest: 1.7e-3, the results' own rounding (300
// rows x 77 states of 16 heads 30 -> 32 us, 2 x 500 x 200 54 -> 58 us).
constexpr int kExactTiles = 4, kExactStates = 64;

// dq: as the forward kernel, with dP beside the scores.  9 uneven sequences of 16401 tokens, 4607
// states and 8 key heads of 2, D = 128: 152 us, 610 TFLOP/s of its three products; fp32, 2 x 333
// rows x 77 states of 4 heads, D = 64: 14 us, two tiles of dependent fp32 products.
template <bool F32, int D>
__global__ __launch_bounds__(kThreads, F32 ? 1 : 2) void cross_dq_kernel(CrossArgs a) {
  typedef Frag<F32> Fr;
  typedef CrossTile<F32, D> Tile;
  constexpr int kTileBytes = kCrossTile * Tile::kRow;
  __shared__ __align__(16) char k0[kTileBytes], v0[kTileBytes], k1[kTileBytes], v1[kTileBytes];
  __shared__ __align__(16) float starts[4][64];
  const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6);
  Lds<float>* const start = (Lds<float>*)starts[wave];
  CrossSeq s;
  int hk, place, tile;
  if (!place_of(a, hk, place)) return;
  if (!seq_of_tile<false>(a, kCrossRows, place, s, tile)) return;
  const int r0 = tile * kCrossRows;
  if (r0 >= s.lq * a.group) return;
  const int rows = s.lq * a.group, w0 = r0 + wave * 32;

  const int tiles = (s.seen + kCrossTile - 1) / kCrossTile;
  const int per = tiles <= kExactTiles ? kExactTiles : (tiles + a.splits - 1) / a.splits;
  const int from = per * (int)blockIdx.y, to = from + per < tiles ? from + per : tiles;
  const char* kb = (const char*)a.k + (seq_base(a.sk, a.cu_k, s.k0, s.kv) + (size_t)hk * a.sk.head) * Tile::kEs;
  const char* vb = (const char*)a.v + (seq_base(a.sv, a.cu_k, s.k0, s.kv) + (size_t)hk * a.sv.head) * Tile::kEs;
  const uint8_t* mask = a.k_mask == nullptr ? nullptr : a.k_mask + (a.cu_k != nullptr ? (size_t)s.k0 : (size_t)s.kv * a.Lk);

  // q, dout and the output come through a wave's part of the tiles' places, memory's rows
  // whole; the output in registers until q's place is free.
  auto part = [&](lds_char* kt, lds_char* vt) { return (wave < 2 ? kt : vt) + (wave & 1) * 32 * Tile::kRow; };
  const typename Tile::Lane offs = Tile::lane_of(lane);
  typename Fr::X q[D / 16], g[D / 16];
  float dot = 0.f, lse = a.lse_in[row_of(a, s, hk, w0 + (lane & 31)).lse] * (F32 ? 1.f : kLog2e);
  // States that are seen, and tiles that have some: of a mask counted until D is not summed from the weights.
  constexpr int kAtOnce = 8;
  int count = s.seen, used = tiles;
  auto summed = [&] { return F32 ? count <= 1 : count <= kExactStates || used <= kExactTiles; };
  {
    lds_char* const q_part = part((lds_char*)k1, (lds_char*)v1);
    lds_char* const g_part = part((lds_char*)k0, (lds_char*)v0);
    const int r = w0 < rows ? w0 : rows - 1;
    const size_t qb = seq_base(a.sq, a.cu_q, s.q0, s.i) + (size_t)hk * a.group * a.sq.head;
    const size_t ob = seq_base(a.so, a.cu_q, s.q0, s.i) + (size_t)hk * a.group * a.so.head;
    copy_rows<F32, D, 32, 1>(a, (const char*)a.q + qb * Tile::kEs, a.sq, r, rows - 1 - r, q_part, 0, lane);
    copy_rows<F32, D, 32, 1>(a, (const char*)a.dout + ob * Tile::kEs, a.so, r, rows - 1 - r, g_part, 0, lane);
    u32x4 o[32 * Tile::kPieces / 64];
    load_rows<F32, D>(a, (const char*)a.o + ob * Tile::kEs, a.so, r, rows - 1 - r, o, lane);
    if (mask != nullptr) count = used = 0;
    for (int t = 0; mask != nullptr && t < tiles && summed(); t += kAtOnce) {
      uint8_t bytes[kAtOnce];
#pragma unroll
      for (int u = 0; u < kAtOnce; ++u) bytes[u] = mask[min((t + u) * kCrossTile + lane, s.seen - 1)];
#pragma unroll
      for (int u = 0; u < kAtOnce; ++u) {
        const uint64_t bits = seen_bits(s.seen - (t + u) * kCrossTile, true, bytes[u], lane);
        count += __popcll(bits), used += bits != 0;
      }
    }
    copies_landed();
#pragma unroll
    for (int e = 0; e < D / 16; ++e) {
      q[e] = Tile::row_frag(q_part, e, offs);
      if (a.flip) q[e] = Fr::flip(q[e]);
      g[e] = Tile::row_frag(g_part, e, offs);
    }
#pragma unroll
    for (int i = 0; i < 32 * Tile::kPieces / 64; ++i) *(Lds<u32x4>*)(q_part + (64 * i + lane) * 16) = o[i];
#pragma unroll
    for (int e = 0; e < D / 16; ++e) {
      const typename Fr::X x = Tile::row_frag(q_part, e, offs);
#pragma unroll
      for (int i = 0; i < 8; ++i) dot = fmaf(Fr::value(g[e], i), Fr::value(x, i), dot);
    }
    lds_barrier();  // the first tile is copied over all of them
  }
  dot += other_half(dot);
  // A row that sees no state has an lse of -inf: as +inf it leaves no p.
  lse = lse == -INFINITY ? INFINITY : lse;
  uint8_t byte = 1;
  auto copy = [&](int t, lds_char* kt, lds_char* vt) {
    const int first = t * kCrossTile, last = s.seen - 1 - first, here = again(lane);
    copy_states<F32, D, kCrossTile, 4>(kb + (size_t)first * a.sk.tok * Tile::kEs, a.sk.tok, last, kt, wave, here);
    copy_states<F32, D, kCrossTile, 4>(vb + (size_t)first * a.sv.tok * Tile::kEs, a.sv.tok, last, vt, wave, here);
    if (mask != nullptr) byte = mask[first + (here < last ? here : last)];
  };
  // Which of the states of tile t, whose copies it waits for, are seen.
  auto arrived = [&](int t, lds_char* kt, lds_char* vt) {
    copies_landed();
    const uint64_t bits = seen_bits(s.seen - t * kCrossTile, mask != nullptr, byte, lane);
    if (~bits != 0) {
      const int here = again(lane);
      if (mask != nullptr) clear_copied<F32, D, kCrossTile, 4>(bits, wave, here, kt, vt);
      put_start(start, bits, here);
    }
    lds_barrier();
    return bits;
  };
  // p and dP of half a tile.
  auto weights = [&](const lds_char* kt, const lds_char* vt, int b, bool all, const typename Tile::Lane& here, floatx16& p,
                     floatx16& dp) __attribute__((always_inline)) {
    if (all)
      p = Fr::mma(Tile::row_frag(kt + 32 * b * Tile::kRow, 0, here), q[0], floatx16{});
    else  // a score of -inf leaves no p
      p = Fr::mma(Tile::row_frag(kt + 32 * b * Tile::kRow, 0, here), q[0], start_of(start + 32 * b, lane));
    dp = floatx16{};
#pragma unroll
    for (int e = 0; e < D / 16; ++e) {
      if (e > 0) p = Fr::mma(Tile::row_frag(kt + 32 * b * Tile::kRow, e, here), q[e], p);
      dp = Fr::mma(Tile::row_frag(vt + 32 * b * Tile::kRow, e, here), g[e], dp);
    }
#pragma unroll
    for (int i = 0; i < 16; ++i) p[i] = weight_of<F32>(a, p[i], lse);
  };
  if (from < to && count > 0 && summed()) {
    float sum = 0.f, one = 0.f;
    for (int t = 0; t < tiles; ++t) {
      if (mask != nullptr) {
        const int first = t * kCrossTile;
        if (seen_bits(s.seen - first, true, mask[min(first + lane, s.seen - 1)], lane) == 0) continue;
      }
      copy(t, (lds_char*)k0, (lds_char*)v0);
      const uint64_t bits = arrived(t, (lds_char*)k0, (lds_char*)v0);
      for (int b = 0; b < 2; ++b) {
        floatx16 p, dp;
        weights((lds_char*)k0, (lds_char*)v0, b, ~bits == 0, Tile::again(offs), p, dp);
#pragma unroll
        for (int i = 0; i < 16; ++i) sum = fmaf(p[i], dp[i], sum), one += p[i] > 0.f ? dp[i] : 0.f;
      }
      lds_barrier();
    }
    dot = count == 1 ? one : sum;
    dot += other_half(dot);
  }
  const bool fine = a.fine && tiles <= kExactTiles;
  floatx16 dq[D / 32];
#pragma unroll
  for (int e = 0; e < D / 32; ++e) dq[e] = floatx16{};

  auto step = [&](int t, lds_char* kt, lds_char* vt, lds_char* next_k, lds_char* next_v) {
    const uint64_t bits = arrived(t, kt, vt);
    if (t + 1 < to) copy(t + 1, next_k, next_v);
    if (bits == 0) return;
#pragma unroll
    for (int b = 0; b < 2; ++b) {
      const typename Tile::Lane here = Tile::again(offs);
      floatx16 p, dp;
      weights(kt, vt, b, ~bits == 0, here, p, dp);
#pragma unroll
      for (int i = 0; i < 16; ++i) p[i] *= dp[i] - dot;
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const typename Fr::X x = Fr::of(p, h);
#pragma unroll
        for (int e = 0; e < D / 32; ++e)
          dq[e] = Fr::mma(Tile::col_frag(kt + (32 * b + 16 * h) * Tile::kRow, e, here), x, dq[e]);
        if (!F32 && fine) {
          const typename Fr::X y = Fr::rest(p, h);
#pragma unroll
          for (int e = 0; e < D / 32; ++e)
            dq[e] = Fr::mma(Tile::col_frag(kt + (32 * b + 16 * h) * Tile::kRow, e, here), y, dq[e]);
        }
      }
    }
  };
  if (from < to) {
    copy(from, (lds_char*)k0, (lds_char*)v0);
    for (int t = from; t < to; t += 2) {
      step(t, (lds_char*)k0, (lds_char*)v0, (lds_char*)k1, (lds_char*)v1);
      if (t + 1 < to) step(t + 1, (lds_char*)k1, (lds_char*)v1, (lds_char*)k0, (lds_char*)v0);
    }
  }
  if (w0 >= rows) return;
  const Row row = row_of(a, s, hk, w0 + (again(lane) & 31));
  if (blockIdx.y == 0 && row.real && lane < 32) a.stats[row.part] = make_float2(lse, dot);
  if (a.splits == 1) {
    const bool odd = (to - from) & 1;  // the last tile's places were k0 and v0
    lds_char* mine = from < to && !odd ? part((lds_char*)k0, (lds_char*)v0) : part((lds_char*)k1, (lds_char*)v1);
    const size_t at = seq_base(a.sdq, a.cu_q, s.q0, s.i) + (size_t)hk * a.group * a.sdq.head;
    store_rows<F32, D>(a, (uint16_t*)a.dq + at * (Tile::kEs / 2), a.sdq, w0, rows, dq, a.scale, mine, lane);
    return;
  }
  if (!row.real) return;
#pragma unroll
  for (int e = 0; e < D / 32; ++e)
#pragma unroll
    for (int i = 0; i < 4; ++i)
      *reinterpret_cast<floatx4*>(a.part + ((size_t)blockIdx.y * ((size_t)a.T * a.Hq) + row.part) * D + 32 * e + 8 * i +
                                  4 * (lane >> 5)) =
          floatx4{dq[e][4 * i], dq[e][4 * i + 1], dq[e][4 * i + 2], dq[e][4 * i + 3]} * a.scale;
}

// Shape of the kernel of dk and dv: 128 states a workgroup, 32 a wave.  In bf16
// two waves have the same states and every other 32 rows, so that each SIMD has two
// waves whose products and exponentials overlap; to leave them 256 registers, v
// comes from LDS and k alone is held.  That is not quite enough: D = 128 spills 9 registers (22 of 512
// in fp32), D = 32 10 of the 128 that its launch bound leaves.  With four waves and both held the batch of
// above took 735 us in all where it took 407 then.  Now 260 us beside 152 for dq and 18 for the sums,
// 485 TFLOP/s of its four products: sequences
// end inside tiles of 128 states, and 3.7 rounds of workgroups of uneven work stand
// where 4096 x 4096 of 16 heads, 4 sequences, keeps 1000 TFLOP/s of both kernels' products.
template <bool F32>
struct DkvShape {
  static constexpr int kWaves = dkv_waves(F32), kHalves = kWaves / 4, kRows = 32 * kHalves;  // rows of a tile
};

template <bool F32, int D>
__global__ __launch_bounds__((64 * DkvShape<F32>::kWaves), (F32 ? 1 : D == 32 ? 4 : 2)) void cross_dkv_kernel(CrossArgs a) {
  typedef Frag<F32> Fr;
  typedef CrossTile<F32, D> Tile;
  typedef DkvShape<F32> Shape;
  constexpr int kRows = Shape::kRows, kTileBytes = kRows * Tile::kRow;
  __shared__ __align__(16) char q0[kTileBytes], g0[kTileBytes], q1[kTileBytes], g1[kTileBytes], vt[kCrossRows * Tile::kRow];
  __shared__ __align__(16) float lse0[kRows], dot0[kRows], lse1[kRows], dot1[kRows];
  const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6);
  const int part_of = wave & 3, half = wave >> 2;  // which 32 states, which rows
  CrossSeq s;
  int hk, place, tile;
  if (!place_of(a, hk, place)) return;
  if (!seq_of_tile<true>(a, kCrossRows, place, s, tile)) return;
  const int j0 = tile * kCrossRows;
  if (j0 >= s.lk) return;

  // The sequence's rows in ranges of about a.range, this workgroup's in tiles; none where no state is seen.
  const int rows = s.lq * a.group;
  int ranges = (int)(((unsigned)rows + (unsigned)a.range - 1u) / (unsigned)a.range);
  ranges = ranges < 1 ? 1 : ranges > a.splits ? a.splits : ranges;
  if ((int)blockIdx.y >= ranges) return;
  const int tiles = j0 < s.seen ? (rows + kRows - 1) / kRows : 0, per = (tiles + ranges - 1) / ranges;
  const int from = per * (int)blockIdx.y, to = from + per < tiles ? from + per : tiles;

  // The lane's state.
  const int j = j0 + part_of * 32 + (lane & 31), jc = j < s.lk ? j : s.lk - 1;
  bool seen = j < s.seen;
  if (seen && a.k_mask != nullptr)
    seen = a.k_mask[(a.cu_k != nullptr ? (size_t)s.k0 : (size_t)s.kv * a.Lk) + jc] != 0;
  const size_t token = (a.cu_k != nullptr ? (size_t)s.k0 : (size_t)s.kv * a.Lk) + jc;
  if (blockIdx.y == 0 && hk == 0 && half == 0 && lane < 32 && j < s.lk) a.counts[token] = ranges;
  typename Fr::X k[D / 16];
  const size_t kat = seq_base(a.sk, a.cu_k, s.k0, s.kv) + (size_t)hk * a.sk.head;
  const size_t vat = seq_base(a.sv, a.cu_k, s.k0, s.kv) + (size_t)hk * a.sv.head + (size_t)j0 * a.sv.tok;
  copy_states<F32, D, kCrossRows, Shape::kWaves>((const char*)a.v + vat * Tile::kEs, a.sv.tok, s.lk - 1 - j0, (lds_char*)vt, wave, lane);
  // k comes through the tiles' places, a place 32 states, memory's rows whole.
  lds_char* const room = (lds_char*)(part_of == 0 ? q0 : part_of == 1 ? g0 : part_of == 2 ? q1 : g1);
  const int w0 = j0 + part_of * 32, k0 = w0 < s.lk ? w0 : s.lk - 1;
  copy_states<F32, D, 32, Shape::kHalves>((const char*)a.k + (kat + (size_t)k0 * a.sk.tok) * Tile::kEs, a.sk.tok, s.lk - 1 - k0, room,
                                          half, lane);
  const typename Tile::Lane offs = Tile::lane_of(lane);
  cross_barrier();
#pragma unroll
  for (int e = 0; e < D / 16; ++e) {
    k[e] = Tile::row_frag(room, e, offs);
    if (a.flip) k[e] = Fr::flip(k[e]);
    // What stands in a masked place may be anything.
    if (!seen) k[e] = Fr::zero();
  }
  if (!seen && half == 0) {
    constexpr int kEach = Tile::kPieces / 2;
    for (int e = 0; e < kEach; ++e)
      *reinterpret_cast<uint4*>(vt + ((part_of * 32 + (lane & 31)) * Tile::kRow + ((lane >> 5) * kEach + e) * 16)) =
          make_uint4(0u, 0u, 0u, 0u);
  }
  lds_barrier();  // the first tile is copied over k
  const bool fine = a.fine && s.seen <= kExactTiles * kCrossTile;
  floatx16 dk[D / 32], dv[D / 32];
#pragma unroll
  for (int e = 0; e < D / 32; ++e) dk[e] = floatx16{}, dv[e] = floatx16{};

  const char* qb = (const char*)a.q +
                   (seq_base(a.sq, a.cu_q, s.q0, s.i) + (size_t)hk * a.group * a.sq.head) * Tile::kEs;
  const char* gb = (const char*)a.dout +
                   (seq_base(a.so, a.cu_q, s.q0, s.i) + (size_t)hk * a.group * a.so.head) * Tile::kEs;
  const float2* stats = a.stats + (a.cu_q != nullptr ? (size_t)s.q0 : (size_t)s.i * a.Lq) * a.Hq + hk * a.group;
  float2 mine = make_float2(0.f, 0.f);
  const bool all = __all(seen);
  const lds_char* vmine = (const lds_char*)vt + part_of * 32 * Tile::kRow;

  auto copy = [&](int t, lds_char* qt, lds_char* gt) {
    const int first = t * kRows, last = rows - 1 - first;
    copy_rows<F32, D, kRows, Shape::kWaves>(a, qb, a.sq, first, last, qt, wave, lane);
    copy_rows<F32, D, kRows, Shape::kWaves>(a, gb, a.so, first, last, gt, wave, lane);
    if (wave == 0) {
      const int r = first + (lane < last ? lane : last), tok = r / a.group;
      mine = stats[(size_t)tok * a.Hq + r - tok * a.group];
    }
  };
  auto keep = [&](int t, float* lse, float* dot) {
    // A row behind the last leaves no p.
    if (wave == 0 && lane < kRows) lse[lane] = t * kRows + lane < rows ? mine.x : INFINITY, dot[lane] = mine.y;
  };
  auto step = [&](const lds_char* qt, const lds_char* gt, const float* lse, const float* dot) {
    const typename Tile::Lane here = Tile::again(offs);
    const int h32 = half * 32 * Tile::kRow;
    floatx16 p = {}, dp = {};
#pragma unroll
    for (int e = 0; e < D / 16; ++e) {
      p = Fr::mma(Tile::row_frag(qt + h32, e, here), k[e], p);
      dp = Fr::mma(Tile::row_frag(gt + h32, e, here), Tile::row_frag(vmine, e, here), dp);
    }
    if (!all)
#pragma unroll
      for (int i = 0; i < 16; ++i) p[i] = seen ? p[i] : -INFINITY;  // no weight
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const floatx4 z = *reinterpret_cast<const floatx4*>(lse + 32 * half + 8 * i + 4 * (lane >> 5));
      const floatx4 y = *reinterpret_cast<const floatx4*>(dot + 32 * half + 8 * i + 4 * (lane >> 5));
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float x = weight_of<F32>(a, p[4 * i + e], z[e]);
        p[4 * i + e] = x;
        dp[4 * i + e] = x * (dp[4 * i + e] - y[e]);
      }
    }
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const typename Fr::X x = Fr::of(p, h), y = Fr::of(dp, h);
#pragma unroll
      for (int e = 0; e < D / 32; ++e) {
        dv[e] = Fr::mma(Tile::col_frag(gt + h32 + 16 * h * Tile::kRow, e, here), x, dv[e]);
        dk[e] = Fr::mma(Tile::col_frag(qt + h32 + 16 * h * Tile::kRow, e, here), y, dk[e]);
      }
      if (!F32 && fine) {
        const typename Fr::X z = Fr::rest(p, h), w = Fr::rest(dp, h);
#pragma unroll
        for (int e = 0; e < D / 32; ++e) {
          dv[e] = Fr::mma(Tile::col_frag(gt + h32 + 16 * h * Tile::kRow, e, here), z, dv[e]);
          dk[e] = Fr::mma(Tile::col_frag(qt + h32 + 16 * h * Tile::kRow, e, here), w, dk[e]);
        }
      }
    }
  };
  if (from < to) {
    copy(from, (lds_char*)q0, (lds_char*)g0);
    for (int t = from;;) {
      keep(t, lse0, dot0);
      cross_barrier();
      if (t + 1 < to) copy(t + 1, (lds_char*)q1, (lds_char*)g1);
      step((lds_char*)q0, (lds_char*)g0, lse0, dot0);
      if (++t >= to) break;
      keep(t, lse1, dot1);
      cross_barrier();
      if (t + 1 < to) copy(t + 1, (lds_char*)q0, (lds_char*)g0);
      step((lds_char*)q1, (lds_char*)g1, lse1, dot1);
      if (++t >= to) break;
    }
  }
  if constexpr (Shape::kHalves == 2) {
    // The second half's sums, through the four tiles.
#pragma unroll
    for (int w = 0; w < 2; ++w) {
      floatx16(&x)[D / 32] = w == 0 ? dk : dv;
      lds_barrier();
      if (half == 1)
#pragma unroll
        for (int e = 0; e < D / 32; ++e)
#pragma unroll
          for (int i = 0; i < 4; ++i)
            *(Lds<floatx4>*)(room + (4 * e + i) * 1024 + lane * 16) =
                floatx4{x[e][4 * i], x[e][4 * i + 1], x[e][4 * i + 2], x[e][4 * i + 3]};
      lds_barrier();
      if (half == 0)
#pragma unroll
        for (int e = 0; e < D / 32; ++e)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const floatx4 y = *(const Lds<floatx4>*)(room + (4 * e + i) * 1024 + lane * 16);
#pragma unroll
            for (int u = 0; u < 4; ++u) x[e][4 * i + u] += y[u];
          }
    }
    if (half == 1) return;
  } else {
    lds_barrier();
  }
  const int count = s.lk - w0;  // the wave's states
  if (count <= 0) return;
  if (!seen)  // a weight of 0 is not enough where a query or its gradient is not finite
#pragma unroll
    for (int e = 0; e < D / 32; ++e) dk[e] = dv[e] = floatx16{};
  if (ranges > 1) {
    const size_t first = (a.cu_k != nullptr ? (size_t)s.k0 : (size_t)s.kv * a.Lk) + w0;
    const size_t part = ((size_t)blockIdx.y * ((size_t)a.S * a.Hk) + first * a.Hk + hk) * D;
    store_states<true, D>(a.part + part, (size_t)a.Hk * D * 4, count, dk, a.scale, room, lane);
    store_states<true, D>(a.part2 + part, (size_t)a.Hk * D * 4, count, dv, 1.f, room, lane);
  } else {
    const size_t dkat = seq_base(a.sdk, a.cu_k, s.k0, s.kv) + (size_t)hk * a.sdk.head + (size_t)w0 * a.sdk.tok;
    const size_t dvat = seq_base(a.sdv, a.cu_k, s.k0, s.kv) + (size_t)hk * a.sdv.head + (size_t)w0 * a.sdv.tok;
    store_states<F32, D>((uint16_t*)a.dk + dkat * (Tile::kEs / 2), a.sdk.tok * Tile::kEs, count, dk, a.scale, room, lane);
    store_states<F32, D>((uint16_t*)a.dv + dvat * (Tile::kEs / 2), a.sdv.tok * Tile::kEs, count, dv, 1.f, room, lane);
  }
}

// Adds the parts of a row's (token x head) ranges, in their order: D / 4 lanes a row, two gradients
// a launch.  Bound by the parts' bytes: 18 us in the batch of above.
template <bool F32, int D>
__global__ __launch_bounds__(kThreads) void cross_sum_kernel(CrossSum a) {
  constexpr int LANES = D / 4, ROWS = kThreads / LANES;
  const size_t R = (size_t)blockIdx.x * ROWS + threadIdx.x / LANES;
  const bool second = blockIdx.y != 0;
  const CrossStrides& s = a.s[second];
  if (R >= (size_t)a.rows) return;
  const int tok = (int)(R / (unsigned)a.H), h = (int)(R - (size_t)tok * a.H), chan = threadIdx.x % LANES * 4;
  size_t out;
  if (a.cu != nullptr) {
    const int total = (int)(a.rows / a.H);
    if (tok < clamp_to(a.cu[0], 0, total) || tok >= clamp_to(a.cu[a.n], 0, total)) return;
    out = (size_t)tok * s.tok + (size_t)h * s.head;
  } else {
    const int i = tok / a.L, t = tok - i * a.L;
    out = (size_t)i * s.seq + (size_t)t * s.tok + (size_t)h * s.head;
  }
  const int count = a.counts != nullptr ? clamp_to(a.counts[tok], 1, a.splits) : a.splits;
  if (count == 1) return;  // there already
  floatx4 x = {0.f, 0.f, 0.f, 0.f};
  for (int p = 0; p < count; ++p) x += *reinterpret_cast<const floatx4*>(a.part[second] + (p * (size_t)a.rows + R) * D + chan);
  store4<F32>(a.out[second], out + chan, x);
}

template <bool F32, int D>
hipError_t dq(const CrossArgs& a, hipStream_t stream) {
  const unsigned grid = ((unsigned)a.tiles * a.Hk + 7) / 8 * 8;
  cross_dq_kernel<F32, D><<<dim3(grid, a.splits), kThreads, 0, stream>>>(a);
  return hipGetLastError();
}
template <bool F32, int D>
hipError_t dkv(const CrossArgs& a, hipStream_t stream) {
  const unsigned grid = ((unsigned)a.tiles * a.Hk + 7) / 8 * 8;
  cross_dkv_kernel<F32, D><<<dim3(grid, a.splits), 64 * DkvShape<F32>::kWaves, 0, stream>>>(a);
  return hipGetLastError();
}
template <bool F32, int D>
hipError_t sum(const CrossSum& a, hipStream_t stream) {
  constexpr int ROWS = kThreads / (D / 4);
  const dim3 grid((unsigned)(((size_t)a.rows + ROWS - 1) / ROWS), a.out[1] != nullptr ? 2 : 1);
  cross_sum_kernel<F32, D><<<grid, kThreads, 0, stream>>>(a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_cross_dq(bool f32, int d, const CrossArgs& a, hipStream_t stream) {
  switch (d) {
    case 32: return f32 ? dq<true, 32>(a, stream) : dq<false, 32>(a, stream);
    case 64: return f32 ? dq<true, 64>(a, stream) : dq<false, 64>(a, stream);
    default: return f32 ? dq<true, 128>(a, stream) : dq<false, 128>(a, stream);
  }
}

hipError_t launch_cross_dkv(bool f32, int d, const CrossArgs& a, hipStream_t stream) {
  switch (d) {
    case 32: return f32 ? dkv<true, 32>(a, stream) : dkv<false, 32>(a, stream);
    case 64: return f32 ? dkv<true, 64>(a, stream) : dkv<false, 64>(a, stream);
    default: return f32 ? dkv<true, 128>(a, stream) : dkv<false, 128>(a, stream);
  }
}

hipError_t launch_cross_sum(bool f32, int d, const CrossSum& a, hipStream_t stream) {
  switch (d) {
    case 32: return f32 ? sum<true, 32>(a, stream) : sum<false, 32>(a, stream);
    case 64: return f32 ? sum<true, 64>(a, stream) : sum<false, 64>(a, stream);
    default: return f32 ? sum<true, 128>(a, stream) : sum<false, 128>(a, stream);
  }
}

}  // namespace vda
