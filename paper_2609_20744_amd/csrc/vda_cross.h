// Internal definitions of the cross attention to an encoder's states (vda.h,
// vda_cross_*), shared by its kernels and its host code.
//
// The query heads that share a key head are taken together: a sequence of lq
// tokens has lq * group rows per key head, row r being token r / group of query
// head key_head * group + r % group.  So states are read once for all of them, and
// the gradients of a shared key head are one sum over rows.
//
// Every product runs on 32 x 32 results of which a lane holds one column: column
// li = lane % 32, rows 8 (i / 4) + 4 lh + i % 4 (lh = lane / 32).  Scores are taken
// transposed (states x queries) where a softmax runs along the states, so its
// maximum and sum are a lane's own; and the 16 rows of a result that a lane half
// holds are what the next product contracts, in the order of col_frag.
#pragma once

#include "vda_common.h"

namespace vda {

typedef float floatx16 __attribute__((ext_vector_type(16)));
typedef float floatx8 __attribute__((ext_vector_type(8)));
typedef short shortx4 __attribute__((ext_vector_type(4)));
typedef short shortx8 __attribute__((ext_vector_type(8)));
typedef __attribute__((address_space(3))) void lds_void;
typedef __attribute__((address_space(3))) char lds_char;  // tiles: never through a generic pointer
template <typename T>
using Lds = __attribute__((address_space(3))) T;
typedef __attribute__((address_space(3))) shortx4 lds_shortx4;
typedef __attribute__((address_space(1))) const void global_void;

constexpr float kLog2e = 1.4426950408889634f;
constexpr int kCrossTile = 64;   // states (or rows) of a tile in LDS
constexpr int kCrossRows = 128;  // rows (or states) of a workgroup, 32 a wave
constexpr int kFewRows = 32;     // rows of a workgroup whose waves share them

// Where a tensor's tokens are: element strides.
struct CrossStrides {
  size_t tok, head, seq;  // seq: equal lengths only; a packed sequence starts tok * its first token in
};

struct CrossArgs {
  const void *q, *k, *v, *o, *dout;
  void *out, *dq, *dk, *dv;
  const float* lse_in;
  float* lse;
  CrossStrides sq, sk, sv, so, sdq, sdk, sdv;  // so: out, its gradient and what the backward pass reads of it
  const int *cu_q, *cu_k, *k_lens, *slots;
  const uint8_t* k_mask;
  int n, n_slots, T, S, Lq, Lk;
  int Hq, Hk, group;
  uint32_t group_magic;  // x / group = x * group_magic >> 24 for x < group + 64
  float scale, c, s;     // c = |scale| log2 e, s = |scale|, above 0
  int fine;              // backward, bf16: two parts of what a short sequence's products take
  int sorted;            // tiles of packed sequences in the order of what they have to do
  int near;              // a tile's rows are within 2^31 bytes of its first, whichever their heads
  int flip;              // scale < 0: the sign of one factor of each score is changed
  int tiles, splits;     // tiles of rows (of states in the gradient of k and v) of a head
  int range;             // gradient of k and v: rows that a workgroup takes, about; at most `splits` ranges
  float *part, *part2;  // workspace: what splits leave
  int* counts;          // [S] ranges of a state's sequence
  float2* stats;        // [T * Hq] backward: lse in powers of two, and D = sum of dout o
};

// One sequence's queries and states.
struct CrossSeq {
  int i, kv;        // its index, and that of its states (the slot)
  int q0, lq;       // packed: first token; tokens
  int k0, lk, seen; // packed: first state; states; of which the length leaves `seen`
};

__device__ __forceinline__ int clamp_to(int x, int lo, int hi) { return x < lo ? lo : x > hi ? hi : x; }

// Offsets of sequence i of a packed tensor, from those of a wave's lanes (b + lane) where
// it has both.  Offsets outside [0, total] are taken as the nearest bound, and a length
// below 0 as 0.
__device__ __forceinline__ void packed_range(const int* cu, int lanes, int b, int i, int total, int& first, int& len) {
  const int at = i - b;
  const int c = at < 64 ? __builtin_amdgcn_readlane(lanes, at) : cu[i];
  const int d = at < 63 ? __builtin_amdgcn_readlane(lanes, at + 1) : cu[i + 1];
  first = uniform(clamp_to(c, 0, total));
  const int end = uniform(clamp_to(d, 0, total));
  len = end > first ? end - first : 0;
}

__device__ __forceinline__ size_t seq_base(const CrossStrides& s, const int* cu, int first, int i) {
  return cu != nullptr ? (size_t)first * s.tok : (size_t)i * s.seq;
}

// A workgroup's key head and tile, all tiles of a head after each other: heads go to
// the XCDs in turn, so that each has tiles of every length, and their states stay in one
// L2.  (All heads of a tile first: 118 -> 177 us for 24 uneven sequences of 16411 tokens,
// and 2 to 6% more where they are equal.)  Sorted tiles (see below) of all heads are taken
// in their order.
__device__ __forceinline__ bool place_of(const CrossArgs& a, int& hk, int& t) {
  if (a.sorted) {
    t = uniform(blockIdx.x / (unsigned)a.Hk), hk = uniform(blockIdx.x - t * (unsigned)a.Hk);
    return t < a.tiles;
  }
  const unsigned id = xcd_grouped_id(blockIdx.x, gridDim.x);
  hk = uniform(id / (unsigned)a.tiles), t = uniform(id - hk * (unsigned)a.tiles);
  return hk < a.Hk;
}

// The sequence that tile `t` of a head belongs to, and which of its tiles it is; false: none.
// Tiles of `per` rows of the queries' side, or (KEYS) of the states'.  A packed
// sequence i has the tiles from first_i / per + i on, first_i being its first row: as many
// places as it needs or one more, so no table is made and every place is found from the
// offsets alone.  Both lists are loaded before either is waited for.
// Sorted (the queries' side): up to 63 sequences packed on both sides, those with most states
// first, so that none of their tiles is left for the end.  24 uneven sequences of 16411 tokens and
// 9601 states, D = 128, eight draws of lengths: with 4 key heads of 2 63 -> 49 us in the mean (0.58 to
// 0.97 of the time), with 8 106 -> 95 (0.81 to 0.98), with 16 182 -> 178 (0.94 to 1.02); of one length the
// search costs 6 to 11% with up to 8 heads and up to 6% with more.  A lane
// has a sequence; its tiles begin behind those of all with more states.
template <bool KEYS>
__device__ __forceinline__ bool seq_of_tile(const CrossArgs& a, int per, int t, CrossSeq& s, int& tile) {
  const int* cu = KEYS ? a.cu_k : a.cu_q;
  const int total = KEYS ? a.S : a.T, group = KEYS ? 1 : a.group, lane = threadIdx.x & 63;
  if (!KEYS && a.sorted) {
    const int at = lane < a.n ? lane : a.n - 1;
    const int q0 = a.cu_q[at], q1 = a.cu_q[at + 1], k0 = a.cu_k[at], k1 = a.cu_k[at + 1];
    const int fq = clamp_to(q0, 0, a.T), fk = clamp_to(k0, 0, a.S);
    const int lq = max(clamp_to(q1, 0, a.T) - fq, 0), lk = max(clamp_to(k1, 0, a.S) - fk, 0);
    const int tiles = lane < a.n ? (lq * group + per - 1) / per : 0;
    const int key = min(lk, (1 << 25) - 1) << 6 | (63 - lane);
    int first = 0;
    for (int j = 0; j < a.n; ++j)
      first += __builtin_amdgcn_readlane(key, j) > key ? __builtin_amdgcn_readlane(tiles, j) : 0;
    const uint64_t is = __ballot(t >= first && t - first < tiles);
    if (is == 0) return false;
    s.i = s.kv = __builtin_ctzll(is);
    tile = t - __builtin_amdgcn_readlane(first, s.i);
    s.q0 = __builtin_amdgcn_readlane(fq, s.i), s.lq = __builtin_amdgcn_readlane(lq, s.i);
    s.k0 = __builtin_amdgcn_readlane(fk, s.i), s.lk = __builtin_amdgcn_readlane(lk, s.i);
    s.seen = s.lk;
    if (a.k_lens != nullptr) s.seen = uniform(clamp_to(a.k_lens[s.kv], 0, s.lk));
    return true;
  }
  s.q0 = s.k0 = 0;
  s.lq = a.Lq, s.lk = a.Lk;
  int lanes_q = 0, lanes_k = 0, base = 0;
  if (cu == nullptr) {
    const int each = ((KEYS ? a.Lk : a.Lq) * group + per - 1) / per;
    s.i = uniform(t / each);
    if (s.i >= a.n) return false;
    tile = t - s.i * each;
    base = s.i;  // one lane's worth
    const int at = s.i + lane < a.n + 1 ? s.i + lane : a.n;
    if (a.cu_q != nullptr) lanes_q = a.cu_q[at];
    if (a.cu_k != nullptr) lanes_k = a.cu_k[at];
  } else {
    int before = 0;
    for (int b = 0; b < a.n; b += 64) {
      const int at = b + lane < a.n + 1 ? b + lane : a.n;
      int x = 0, y = 0;
      if (a.cu_q != nullptr) x = a.cu_q[at];
      if (a.cu_k != nullptr) y = a.cu_k[at];
      const uint64_t is = __ballot(b + lane < a.n && clamp_to(KEYS ? y : x, 0, total) * group / per + b + lane <= t);
      if (is == 0) break;  // in order, so that no later one starts before t
      before += __popcll(is);
      lanes_q = x, lanes_k = y, base = b;
    }
    s.i = uniform(before) - 1;
    if (s.i < base) return false;  // none; or offsets out of order
  }
  if (a.cu_q != nullptr) packed_range(a.cu_q, lanes_q, base, s.i, a.T, s.q0, s.lq);
  if (a.cu_k != nullptr) packed_range(a.cu_k, lanes_k, base, s.i, a.S, s.k0, s.lk);
  if (cu != nullptr) {
    tile = t - (uniform((KEYS ? s.k0 : s.q0) * group / per) + s.i);
    if (tile < 0) return false;  // out of order
  }
  s.kv = s.i;
  if (a.slots != nullptr) {
    s.kv = uniform(a.slots[s.i]);
    if (s.kv < 0 || s.kv >= a.n_slots) return false;  // a row of padding
  }
  s.seen = s.lk;
  if (a.k_lens != nullptr) s.seen = uniform(clamp_to(a.k_lens[s.kv], 0, s.lk));
  return true;
}

// ---------------------------------------------------------------------------
// Operands: eight elements a lane.
// ---------------------------------------------------------------------------
template <bool F32>
struct Frag;

template <>
struct Frag<false> {
  typedef bf16x8 X;
  static __device__ __forceinline__ floatx16 mma(X a, X b, floatx16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
  }
  // Elements 8 t .. of a result, rounded: the first factor of a product that has two roundings at most.
  static __device__ __forceinline__ X of(const floatx16& s, int t) {
    u32x4 w;
#pragma unroll
    for (int e = 0; e < 4; ++e) w[e] = pack_bf16x2(s[8 * t + 2 * e], s[8 * t + 2 * e + 1]);
    return __builtin_bit_cast(X, w);
  }
  // What of() leaves of them.
  static __device__ __forceinline__ X rest(const floatx16& s, int t) {
    const u32x4 w = __builtin_bit_cast(u32x4, of(s, t));
    u32x4 r;
#pragma unroll
    for (int e = 0; e < 4; ++e) r[e] = pack_bf16x2(s[8 * t + 2 * e] - bf16_lo(w[e]), s[8 * t + 2 * e + 1] - bf16_hi(w[e]));
    return __builtin_bit_cast(X, r);
  }
  static __device__ __forceinline__ X load(const void* p, size_t at) {
    return *reinterpret_cast<const bf16x8*>((const uint16_t*)p + at);
  }
  static __device__ __forceinline__ X flip(X x) { return __builtin_bit_cast(X, __builtin_bit_cast(u32x4, x) ^ 0x80008000u); }
  static __device__ __forceinline__ X zero() { return __builtin_bit_cast(X, u32x4{0u, 0u, 0u, 0u}); }
  static __device__ __forceinline__ float value(X x, int e) { return (float)x[e]; }
};

template <>
struct Frag<true> {
  typedef floatx8 X;
  static __device__ __forceinline__ floatx16 mma(X a, X b, floatx16 c) {
#pragma unroll
    for (int e = 0; e < 8; ++e) c = __builtin_amdgcn_mfma_f32_32x32x2f32(a[e], b[e], c, 0, 0, 0);
    return c;
  }
  static __device__ __forceinline__ X of(const floatx16& s, int t) {
    X x;
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = s[8 * t + e];
    return x;
  }
  static __device__ __forceinline__ X rest(const floatx16&, int) { return zero(); }
  static __device__ __forceinline__ X load(const void* p, size_t at) {
    const floatx4* f = reinterpret_cast<const floatx4*>((const float*)p + at);
    const floatx4 a = f[0], b = f[1];
    return X{a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]};
  }
  static __device__ __forceinline__ X flip(X x) { return -x; }
  static __device__ __forceinline__ X zero() { return X{0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f}; }
  static __device__ __forceinline__ float value(X x, int e) { return x[e]; }
};

// ---------------------------------------------------------------------------
// Tiles in LDS: rows of D channels, as they are in memory but for the order of a
// row's 16-byte pieces: piece c of row r stands at place c ^ swizzle(r).  With it
// the 16 lanes whose 16 bytes of one column LDS serves together (rows that differ
// modulo 16) meet all banks, and so do the four rows by 64 bytes that a transposing
// read takes.  A copy of 1 KB fills consecutive places, and reads whole rows.
// ---------------------------------------------------------------------------
template <bool F32, int D>
struct CrossTile {
  typedef typename Frag<F32>::X X;
  static constexpr int kEs = F32 ? 4 : 2, kRow = D * kEs, kPieces = kRow / 16;
  static __device__ __forceinline__ int swizzle(int r) {
    if constexpr (kPieces >= 16) return (r & 3) << 2 | (r >> 2 & 3);
    if constexpr (kPieces == 8) return (r >> 1 & 1) << 2 | (r >> 2 & 3);
    return r >> 2 & 3;
  }
  // A lane's offsets in a tile `from` bytes behind an array's begin, opaque: the
  // others are these with constant bits changed, so that an address is one instruction
  // and one register, not one of its own for each of a tile's reads.
  static constexpr int kColOffs = F32 ? 8 : 2;
  struct Lane {
    int row, col[kColOffs];
  };
  static __device__ __forceinline__ Lane lane_of(int lane, int from = 0) {
    Lane l;
    const int li = lane & 31, lh = lane >> 5;
    l.row = from + li * kRow + ((F32 ? 2 * lh : lh) ^ swizzle(li)) * 16;
#pragma unroll
    for (int s = 0; s < kColOffs; ++s) {
      if constexpr (F32) {
        const int r = (s >> 2) * 8 + 4 * lh + (s & 3);
        l.col[s] = from + r * kRow + ((li >> 2) ^ swizzle(r)) * 16 + (li & 3) * 4;
      } else {
        // ds_read_b64_tr_b16: lane i of 16 receives element i % 4 of the 8 bytes that lanes i / 4 + 4 e address.
        const int r = 8 * s + 4 * lh + (lane >> 2 & 3);
        const int piece = 2 * (lane >> 4 & 1) + (lane >> 1 & 1);
        l.col[s] = from + r * kRow + (piece ^ swizzle(r)) * 16 + (lane & 1) * 8;
      }
    }
    return again(l);
  }
  // Offsets that the compiler takes for new: used in a loop's body, they keep the
  // others from being computed before the loop and held through it.
  static __device__ __forceinline__ Lane again(Lane l) {
    asm volatile("" : "+v"(l.row));
#pragma unroll
    for (int s = 0; s < kColOffs; ++s) asm volatile("" : "+v"(l.col[s]));
    return l;
  }
  // Channels 16 s + 8 lh .. + 7 of row li of the rows behind `tile` (a multiple of 16 rows in).
  // An address is one addition to a named array: of a longer chain the compiler
  // does not see which array it is in, and waits for copies into the others.
  static __device__ __forceinline__ X row_frag(const lds_char* tile, int s, const Lane& l) {
    if constexpr (F32) {
      const floatx4 a = *(const Lds<floatx4>*)(tile + (l.row ^ 64 * s));
      const floatx4 b = *(const Lds<floatx4>*)(tile + (l.row ^ (64 * s + 16)));
      return X{a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]};
    } else {
      return *(const Lds<bf16x8>*)(tile + (l.row ^ 32 * s));
    }
  }
  // Channel 32 b + li of the rows 4 lh + e and 8 + 4 lh + e, e < 4, behind `tile`.
  static __device__ __forceinline__ X col_frag(const lds_char* tile, int b, const Lane& l) {
    if constexpr (F32) {
      X x;
#pragma unroll
      for (int e = 0; e < 8; ++e) x[e] = *(const Lds<float>*)(tile + (l.col[e] ^ 128 * b));
      return x;
    } else {
      const shortx4 v = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_shortx4*)(tile + (l.col[0] ^ 64 * b)));
      const shortx4 w = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_shortx4*)(tile + (l.col[1] ^ 64 * b)));
      return __builtin_bit_cast(bf16x8, shortx8{v[0], v[1], v[2], v[3], w[0], w[1], w[2], w[3]});
    }
  }
};

// Copies ROWS rows of consecutive tokens into a tile; rows behind `last` repeat
// it.  base: the tile's first row.  One way for whole tiles and others: of copies that only
// one way to a read has, the compiler does not see where they go, and waits for all.
template <bool F32, int D, int ROWS, int WAVES>
__device__ __forceinline__ void copy_states(const void* base, size_t row_elems, int last, lds_char* tile, int wave, int lane) {
#if defined(__HIP_DEVICE_COMPILE__)  // the compiler's host pass refuses the builtin in some kernels
  typedef CrossTile<F32, D> Tile;
  constexpr int kPieces = ROWS * Tile::kRow / 1024, kStep = 64 * WAVES / Tile::kPieces;
  const __amdgpu_buffer_rsrc_t src = make_rsrc(base, 0xfffffff0u);
  const uint32_t row_bytes = (uint32_t)row_elems * Tile::kEs;  // below 2^24
  const int r0 = (wave * 64 + lane) / Tile::kPieces, piece0 = lane % Tile::kPieces ^ Tile::swizzle(r0);
#pragma unroll
  for (int i = 0; i < (kPieces + WAVES - 1) / WAVES; ++i) {
    const int p = wave + i * WAVES, r = r0 + i * kStep;
    if (kPieces % WAVES != 0 && p >= kPieces) break;
    __builtin_amdgcn_raw_ptr_buffer_load_lds(
        src, (lds_void*)(tile + p * 1024), 16,
        __umul24(min(r, last), row_bytes) + (piece0 ^ Tile::swizzle(i * kStep)) * 16u, 0, 0, 0);
  }
#endif
}

// Writes zeros over the rows of tiles whose bit is not set, each wave over what it copied
// itself, once that is there: what stands in a masked place may be anything, and 0 times it
// has to be 0.  A copy's 1024 bytes whose rows are all seen cost no more than a scalar look.
template <bool F32, int D, int ROWS, int WAVES, typename... Tiles>
__device__ __forceinline__ void clear_copied(uint64_t bits, int wave, int lane, Tiles... tiles) {
  typedef CrossTile<F32, D> Tile;
  constexpr int kPieces = ROWS * Tile::kRow / 1024, kRows = 64 / Tile::kPieces;
#pragma unroll
  for (int i = 0; i < (kPieces + WAVES - 1) / WAVES; ++i) {
    const int p = wave + i * WAVES;
    if (kPieces % WAVES != 0 && p >= kPieces) break;
    const uint32_t w = (uint32_t)(bits >> p * kRows) & ((1u << kRows) - 1);
    if (w != (1u << kRows) - 1 && !(w >> lane / Tile::kPieces & 1))
      ((*(Lds<u32x4>*)(tiles + (p * 64 + lane) * 16) = u32x4{0u, 0u, 0u, 0u}), ...);
  }
}

// Copies ROWS rows of queries (token x head) into a tile; rows behind `last` repeat it.
// base: the sequence's first token of the key head's first query head.  Where the
// query heads of a key head divide what a wave's copies step by, one offset again.
template <bool F32, int D, int ROWS, int WAVES>
__device__ __forceinline__ void copy_rows(const CrossArgs& a, const void* base, const CrossStrides& s, int r0, int last,
                                          lds_char* tile, int wave, int lane) {
  typedef CrossTile<F32, D> Tile;
  constexpr int kPieces = ROWS * Tile::kRow / 1024, kStep = 64 * WAVES / Tile::kPieces;
  const int t0 = uniform(r0 / a.group), g0 = r0 - t0 * a.group;
  const char* from = (const char*)base + (size_t)t0 * s.tok * Tile::kEs;
  const int first = (wave * 64 + lane) / Tile::kPieces, piece0 = lane % Tile::kPieces ^ Tile::swizzle(first);
  if (a.near && g0 == 0 && kStep % a.group == 0 && last >= ROWS - 1) {
    const __amdgpu_buffer_rsrc_t src = make_rsrc(from, 0xfffffff0u);
    const uint32_t t = first * a.group_magic >> 24, g = first - t * a.group;
    const uint32_t at = (t * (uint32_t)s.tok + g * (uint32_t)s.head) * Tile::kEs;
    const uint32_t step = kStep / a.group * (uint32_t)s.tok * Tile::kEs;
#pragma unroll
    for (int i = 0; i < (kPieces + WAVES - 1) / WAVES; ++i) {
      const int p = wave + i * WAVES;
      if (kPieces % WAVES != 0 && p >= kPieces) break;
      __builtin_amdgcn_raw_ptr_buffer_load_lds(src, (lds_void*)(tile + p * 1024), 16,
                                               at + (piece0 ^ Tile::swizzle(i * kStep)) * 16u, i * step, 0, 0);
    }
    return;
  }
#pragma unroll
  for (int i = 0; i < (kPieces + WAVES - 1) / WAVES; ++i) {
    const int p = wave + i * WAVES, r = first + i * kStep;
    if (kPieces % WAVES != 0 && p >= kPieces) break;
    const uint32_t x = g0 + (r < last ? r : last);
    const uint32_t t = x * a.group_magic >> 24, g = x - t * a.group;
    __builtin_amdgcn_global_load_lds(
        (global_void*)(from + (t * s.tok + g * s.head) * Tile::kEs + (piece0 ^ Tile::swizzle(i * kStep)) * 16),
        (lds_void*)(tile + p * 1024), 16, 0, 0);
  }
}

// x where the lane's bit of a result's row i is set, else `otherwise` (a constant), whatever
// x is; two operations.  w: the bits of the 32 rows, from the lane's first row on.
__device__ __forceinline__ float row_or(float x, uint32_t w, int i, float otherwise) {
  const int m = __builtin_amdgcn_sbfe((int)w, 8 * (i >> 2) + (i & 3), 1);
  return __int_as_float((m & __float_as_int(x)) | (~m & __float_as_int(otherwise)));
}

// What the scores of a tile's states start from where not all are seen, a wave's own in LDS:
// -inf stays in the sum of finite products (the rows that are not seen are zeros, or the
// last one again), so that no score has to be looked at by itself.
__device__ __forceinline__ void put_start(Lds<float>* start, uint64_t bits, int lane) {
  start[lane] = __builtin_amdgcn_inverse_ballot_w64(bits) ? 0.f : -INFINITY;
}
__device__ __forceinline__ floatx16 start_of(const Lds<float>* start, int lane) {
  floatx16 x;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const floatx4 y = *(const Lds<floatx4>*)(start + 8 * i + 4 * (lane >> 5));
#pragma unroll
    for (int e = 0; e < 4; ++e) x[4 * i + e] = y[e];
  }
  return x;
}

// The wave's copies into LDS are there.
__device__ __forceinline__ void copies_landed() {
  __builtin_amdgcn_sched_barrier(0);
  __builtin_amdgcn_s_waitcnt(0x0f70);  // vmcnt 0
  __builtin_amdgcn_sched_barrier(0);
}

// Barrier behind which the copies into LDS that any wave issued before it are there.
__device__ __forceinline__ void cross_barrier() {
  __builtin_amdgcn_sched_barrier(0);
  __builtin_amdgcn_s_waitcnt(0x0070);  // vmcnt 0, lgkmcnt 0
  __syncthreads();
}

// A lane's row: where its query, output and lse are, and its part of a workspace.
struct Row {
  bool real;
  size_t q, out, lse, part;
};
__device__ __forceinline__ Row row_of(const CrossArgs& a, const CrossSeq& s, int hk, int r) {
  Row w;
  const int rows = s.lq * a.group;
  w.real = r < rows;
  if (!w.real) r = rows - 1;
  const int t = r / a.group, h = hk * a.group + r - t * a.group;
  w.q = seq_base(a.sq, a.cu_q, s.q0, s.i) + (size_t)t * a.sq.tok + (size_t)h * a.sq.head;
  w.out = seq_base(a.so, a.cu_q, s.q0, s.i) + (size_t)t * a.so.tok + (size_t)h * a.so.head;
  w.lse = a.cu_q != nullptr ? (size_t)h * a.T + s.q0 + t : ((size_t)s.i * a.Hq + h) * a.Lq + t;
  w.part = ((a.cu_q != nullptr ? (size_t)s.q0 : (size_t)s.i * a.Lq) + t) * a.Hq + h;
  return w;
}

// Which of the 64 states from one on are seen: `left` of them are the sequence's,
// byte is the mask's of the lane's.
__device__ __forceinline__ uint64_t seen_bits(int left, bool masked, uint8_t byte, int lane) {
  uint64_t bits = left >= 64 ? ~0ull : left <= 0 ? 0 : (1ull << left) - 1;
  if (masked) bits &= __ballot(byte != 0 && lane < left);
  return bits;
}

// A value that the compiler takes for new: what is made of it is not held through a loop.
__device__ __forceinline__ int again(int x) {
  asm volatile("" : "+v"(x));
  return x;
}

// The other lane half's value.
__device__ __forceinline__ float other_half(float x) { return __shfl_xor(x, 32); }

// Four channels to memory.
template <bool F32>
__device__ __forceinline__ void store4(void* p, size_t at, floatx4 x) {
  if constexpr (F32)
    *reinterpret_cast<floatx4*>((float*)p + at) = x;
  else
    *reinterpret_cast<uint2*>((uint16_t*)p + at) = make_uint2(pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3]));
}

// What copy_rows would copy of 32 rows with one wave, in registers.
template <bool F32, int D>
__device__ __forceinline__ void load_rows(const CrossArgs& a, const void* base, const CrossStrides& s, int r0, int last,
                                          u32x4 (&x)[CrossTile<F32, D>::kPieces / 2], int lane) {
  typedef CrossTile<F32, D> Tile;
  const int t0 = uniform(r0 / a.group), g0 = r0 - t0 * a.group;
  const char* from = (const char*)base + (size_t)t0 * s.tok * Tile::kEs;
#pragma unroll
  for (int i = 0; i < Tile::kPieces / 2; ++i) {
    const int r = lane / Tile::kPieces + i * (64 / Tile::kPieces);
    const uint32_t y = g0 + (r < last ? r : last), t = y * a.group_magic >> 24, g = y - t * a.group;
    x[i] = *reinterpret_cast<const u32x4*>(from + (t * s.tok + g * s.head) * Tile::kEs +
                                           (lane % Tile::kPieces ^ Tile::swizzle(r)) * 16);
  }
}

// A wave's 32 rows of D channels, as a product leaves them, times `by`, through its own part
// of LDS (32 rows of a tile): put(r, piece, 16 bytes) then has rows' bytes next to one another
// in the lanes.
template <bool F32, int D, typename Put>
__device__ __forceinline__ void rows_through(const floatx16 (&x)[D / 32], float by, lds_char* tile, int lane, Put put) {
  typedef CrossTile<F32, D> Tile;
  const int li = lane & 31, lh = lane >> 5;
  const int at = li * Tile::kRow + (F32 ? lh ^ Tile::swizzle(li) : Tile::swizzle(li)) * 16 + (F32 ? 0 : lh * 8);
#pragma unroll
  for (int e = 0; e < D / 32; ++e)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const floatx4 z = floatx4{x[e][4 * i], x[e][4 * i + 1], x[e][4 * i + 2], x[e][4 * i + 3]} * by;
      if constexpr (F32)
        *(Lds<floatx4>*)(tile + (at ^ (8 * e + 2 * i) * 16)) = z;
      else
        *(Lds<u32x2>*)(tile + (at ^ (4 * e + i) * 16)) = u32x2{pack_bf16x2(z[0], z[1]), pack_bf16x2(z[2], z[3])};
    }
  const int piece = lane % Tile::kPieces;
#pragma unroll
  for (int i = 0; i < Tile::kPieces / 2; ++i) {
    const int r = lane / Tile::kPieces + i * (64 / Tile::kPieces);
    put(r, piece, *(const Lds<u32x4>*)(tile + r * Tile::kRow + (piece ^ Tile::swizzle(r)) * 16));
  }
}

// The rows (token x head) from r0 on of `rows` to memory.  base: as for copy_rows.
template <bool F32, int D>
__device__ __forceinline__ void store_rows(const CrossArgs& a, void* base, const CrossStrides& s, int r0, int rows,
                                           const floatx16 (&x)[D / 32], float by, lds_char* tile, int lane) {
  const int t0 = uniform(r0 / a.group), g0 = r0 - t0 * a.group;
  char* to = (char*)base + (size_t)t0 * s.tok * CrossTile<F32, D>::kEs;
  rows_through<F32, D>(x, by, tile, lane, [&](int r, int piece, u32x4 z) {
    const uint32_t y = g0 + r, t = y * a.group_magic >> 24, g = y - t * a.group;
    if (r0 + r < rows) *reinterpret_cast<u32x4*>(to + (t * s.tok + g * s.head) * CrossTile<F32, D>::kEs + piece * 16) = z;
  });
}

// `rows` rows (at most 32) that are row_bytes apart to memory, in the type of F32.
template <bool F32, int D>
__device__ __forceinline__ void store_states(void* to, size_t row_bytes, int rows, const floatx16 (&x)[D / 32], float by,
                                             lds_char* tile, int lane) {
  rows_through<F32, D>(x, by, tile, lane, [&](int r, int piece, u32x4 z) {
    if (r < rows) *reinterpret_cast<u32x4*>((char*)to + r * row_bytes + piece * 16) = z;
  });
}

// Host-side launchers (arguments validated).
// Waves of a workgroup of few rows that share its range of the states; their tiles have to fit LDS.
constexpr int few_waves(bool f32, int d) { return f32 && d == 128 ? 2 : 4; }

// Waves of a workgroup of the gradients of k and v.
constexpr int dkv_waves(bool f32) { return f32 ? 4 : 8; }

// few: waves of a workgroup of few rows, 1 or few_waves(); 0: many rows
hipError_t launch_cross_forward(bool f32, int d, int few, const CrossArgs& a, hipStream_t stream);
hipError_t launch_cross_join(bool f32, int d, const CrossArgs& a, hipStream_t stream);
hipError_t launch_cross_dq(bool f32, int d, const CrossArgs& a, hipStream_t stream);
hipError_t launch_cross_dkv(bool f32, int d, const CrossArgs& a, hipStream_t stream);
// Sums of part [splits][rows][d] to the rows of a tensor of H heads; counts: of how many each token's are, or null (all).
struct CrossSum {
  const float* part[2];  // of one gradient, or of two at once
  const int* counts;
  void* out[2];
  CrossStrides s[2];
  const int* cu;
  int n, L, H, splits;
  long long rows;  // tokens * H
};
hipError_t launch_cross_sum(bool f32, int d, const CrossSum& a, hipStream_t stream);

}  // namespace vda
