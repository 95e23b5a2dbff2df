// Internal definitions of the token-wise gated delta rule (Eq. 2), shared by
// its kernels and its host code.
//
// Tokens are taken in chunks of 64.  With S the state entering a chunk
// (d_v x d_k), G_i the sum of the chunk's log decays up to token i,
// D_ij = e^(G_i - G_j), gam_i = e^(G_i), eta_i = e^(G_63 - G_i):
//     L_ij = D_ij k_i.k_j (i > j),   T = (I + L diag(beta))^-1,
//     P_ij = scale D_ij q_i.k_j (i >= j),
//     E = T (V - diag(gam) K S^T),   N = diag(beta) E, what the tokens write
//     O = scale diag(gam) Q S^T + P N
//     S <- gam_63 S + N^T diag(eta) K
// T and P do not depend on the state; the chunk-preparation kernel makes them
// for all chunks at once, and the scans carry the state.  With the strengths on
// the right of L, a token of strength 0 has zeros in its column of T (but the
// diagonal) and its row of N, whatever its key and value are, and beta's gradient,
// E times that of N, needs no division by a strength.
#pragma once

#include "vda_common.h"

namespace vda {

constexpr int kChunk = 64;  // tokens of a chunk
constexpr int kLds = 160 * 1024;  // bytes of LDS of a workgroup

typedef float floatx8 __attribute__((ext_vector_type(8)));
typedef short shortx4 __attribute__((ext_vector_type(4)));

// ---------------------------------------------------------------------------
// Matrix operands.  A product contracts 32 indices a step; lane (li, lg) =
// (lane % 16, lane / 16) holds, of the operand's row (or column) li, the
// indices 4 lg + e and 16 + 4 lg + e, e < 4.  That is the order in which a
// lane holds the rows of two 16 x 16 results, so a result whose rows are the
// next product's contraction goes into it from registers.
//
// bf16 storage: an exact operand X is one bf16 vector (inputs, which are
// bf16); a wide operand W is two, hi = bf16(x) and lo = bf16(x - hi), about
// 16 mantissa bits, for values that exist in fp32 only: states, writes and
// the triangular inverse go through such products (lo * lo is left out), so
// that the state and the gates' gradients keep fp32-like accuracy (2^-17 a
// factor); products that only reach a bf16 output take `head`, one rounding.
// fp32 storage: both are fp32 vectors, on the fp32 matrix cores.
// ---------------------------------------------------------------------------
template <bool F32>
struct Op;

// What the pair x, y leaves of itself beside its rounding `hi`, rounded: each
// remainder in one instruction, a dot product of hi with (-1, 0) or (0, -1)
// added to the value, exact (1 M values over all exponents compared with the
// subtraction).  The constants pass through registers: as immediates the
// compiler encodes the first like the second.
__device__ __forceinline__ uint32_t rest_bf16x2(float x, float y, uint32_t hi) {
  uint32_t first = 0x0000bf80u, second = 0xbf800000u;
  asm("" : "+s"(first));
  asm("" : "+s"(second));
  const bf16x2 h = __builtin_bit_cast(bf16x2, hi);
  return pack_bf16x2(__builtin_amdgcn_fdot2_f32_bf16(h, __builtin_bit_cast(bf16x2, first), x, false),
                     __builtin_amdgcn_fdot2_f32_bf16(h, __builtin_bit_cast(bf16x2, second), y, false));
}

template <>
struct Op<false> {
  typedef uint16_t Elem;
  typedef bf16x8 X;
  struct W {
    bf16x8 hi, lo;
  };
  static __device__ __forceinline__ X narrow(floatx4 a, floatx4 b) {
    return __builtin_bit_cast(
        X, u32x4{pack_bf16x2(a[0], a[1]), pack_bf16x2(a[2], a[3]), pack_bf16x2(b[0], b[1]), pack_bf16x2(b[2], b[3])});
  }
  static __device__ __forceinline__ W wide(floatx4 a, floatx4 b) {
    u32x4 hi, lo;
#pragma unroll
    for (int p = 0; p < 4; ++p) {
      const float x = p < 2 ? a[2 * p] : b[2 * p - 4], y = p < 2 ? a[2 * p + 1] : b[2 * p - 3];
      hi[p] = pack_bf16x2(x, y);
      lo[p] = rest_bf16x2(x, y, hi[p]);
    }
    return W{__builtin_bit_cast(X, hi), __builtin_bit_cast(X, lo)};
  }
  static __device__ __forceinline__ X head(const W& w) { return w.hi; }
  static __device__ __forceinline__ floatx4 mma(X a, X b, floatx4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
  }
  static __device__ __forceinline__ floatx4 mma(X a, const W& b, floatx4 c) {
    return mma(a, b.hi, mma(a, b.lo, c));
  }
  static __device__ __forceinline__ floatx4 mma(const W& a, X b, floatx4 c) {
    return mma(a.hi, b, mma(a.lo, b, c));
  }
  static __device__ __forceinline__ floatx4 mma(const W& a, const W& b, floatx4 c) {
    return mma(a.hi, b.hi, mma(a.hi, b.lo, mma(a.lo, b.hi, c)));
  }
  static __device__ __forceinline__ float value(X x, int e) { return (float)x[e]; }
  static __device__ __forceinline__ float value(const W& w, int e) {
    return (float)w.hi[e] + (float)w.lo[e];
  }
};

template <>
struct Op<true> {
  typedef float Elem;
  typedef floatx8 X;
  struct W {
    floatx8 v;
  };
  static __device__ __forceinline__ X narrow(floatx4 a, floatx4 b) {
    return floatx8{a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]};
  }
  static __device__ __forceinline__ W wide(floatx4 a, floatx4 b) { return W{narrow(a, b)}; }
  static __device__ __forceinline__ X head(const W& w) { return w.v; }
  static __device__ __forceinline__ floatx4 mma(X a, X b, floatx4 c) {
#pragma unroll
    for (int e = 0; e < 8; ++e) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a[e], b[e], c, 0, 0, 0);
    return c;
  }
  static __device__ __forceinline__ floatx4 mma(X a, const W& b, floatx4 c) { return mma(a, b.v, c); }
  static __device__ __forceinline__ floatx4 mma(const W& a, X b, floatx4 c) { return mma(a.v, b, c); }
  static __device__ __forceinline__ floatx4 mma(const W& a, const W& b, floatx4 c) {
    return mma(a.v, b.v, c);
  }
  static __device__ __forceinline__ float value(X x, int e) { return x[e]; }
  static __device__ __forceinline__ float value(const W& w, int e) { return w.v[e]; }
};

typedef __attribute__((address_space(3))) void lds_void;
typedef __attribute__((address_space(3))) shortx4 lds_shortx4;

// ---------------------------------------------------------------------------
// Row tiles in LDS: 16 tokens x 32 channels, each lane's 16 bytes (eight
// consecutive channels 8 lg .. of token li; fp32: four, in two halves of 1 KB)
// in one place, so that an operand of the rows is one read at a lane's own
// offset plus a constant: no address is computed in a loop.  Columns are
// read across lanes' places (ds_read_b64_tr_b16, in which lane i of 16 receives
// element i % 4 of the 8-byte pieces that lanes i / 4 + 4 e address; or four
// words in fp32).  Places are permuted (bf16: place_shift) so that the 16 lanes
// whose 16 bytes are read together meet the 256 bytes of all banks; they are not
// 16 in a row, but quads 0, 3, 5, 6 and 1, 2, 4, 7 of lanes of every 32.
//
// The 1 KB of a copy to LDS are consecutive places, so their order is also what
// a copy reads from memory at a time: with a row's places 16 apart it was 16
// bytes of each of 16 rows, then the next 16, and the reverse scan took 178 us
// (16401 tokens, 16 heads); with four lanes on 64 bytes of a row 167 us.  Where
// there are two tiles of a row, they share 2 KB, eight lanes take 128 bytes of
// a row, a whole cache line (RowTiles::kPairs).
//
// Channels are paired with results by this order: operand element e of lane
// lg, step s, is channel 32 s + 8 lg + e; so a result whose rows are such a
// contraction comes in halves o = 0, 1 whose row 4 lg + r is channel
// 32 s + 8 lg + 4 o + r.
// ---------------------------------------------------------------------------
template <bool F32>
__host__ __device__ constexpr int row_tile_bytes() { return F32 ? 2048 : 1024; }

// 0, 2, 3, 1 of row / 4.
__device__ __forceinline__ int place_shift(int row) { return ((row >> 1 ^ row >> 2) & 2) | row >> 3; }

template <bool F32>
__device__ __forceinline__ int tile_place(int row, int lg) {
  return F32 ? (16 * lg + (row ^ lg)) * 16 : (4 * row + (lg ^ place_shift(row))) * 16;
}
// ... of a pair of tiles (bf16), lg < 8.
__device__ __forceinline__ int pair_unit(int row, int lg) { return lg ^ ((row & 2) << 1 | place_shift(row)); }
__device__ __forceinline__ int pair_place(int row, int lg) { return (8 * row + pair_unit(row, lg)) * 16; }

// 64 rows of 32 BLOCKS channels: where tile (block s, row tile t) is, and what
// a lane's offsets in a block's tiles are changed by (the second of a pair).
template <bool F32, int BLOCKS>
struct RowTiles {
  static constexpr bool kPairs = !F32 && BLOCKS % 2 == 0;
  __device__ static constexpr int tile(int s, int t) {
    return kPairs ? ((s >> 1) * 4 + t) * 2048 : (s * 4 + t) * row_tile_bytes<F32>();
  }
  __device__ static constexpr int odd(int s) { return kPairs ? (s & 1) * 64 : 0; }
};

// Row of place `row` of tile t in twisted order: paired order (below) with the
// two tiles' rows exchanged for row >= 8.  A tile read by columns in that order
// (twisted_cols) takes both halves of its 16-byte places, and so all banks.
__device__ __forceinline__ int twisted_row(int t, int row) {
  return 32 * (t >> 1) + 8 * (row >> 2) + 4 * ((t ^ (row >> 3)) & 1) + (row & 3);
}

// Offsets of a lane: its row operand, and the columns that it reads.
struct TileLane {
  int row, col[4];
};
template <bool F32, bool PAIRS>
__device__ __forceinline__ TileLane tile_lane(int li, int lg) {
  TileLane l;
  l.row = PAIRS ? pair_place(li, lg) : tile_place<F32>(li, lg);
  if constexpr (F32) {
#pragma unroll
    for (int e = 0; e < 4; ++e) l.col[e] = tile_place<true>(4 * lg + e, li >> 2) + (li & 3) * 4;
  } else {
    const int row = 4 * lg + (li >> 2), unit = li & 3;
    l.col[0] = PAIRS ? pair_place(row, unit) : tile_place<false>(row, unit);
    l.col[1] = l.col[2] = l.col[3] = 0;
  }
  return l;
}

// The column offsets of half o of block s, both runtime, from the tiles' begin
// (read with o 0 and odd 0): an address that is one addition to a named array.
// Of a longer chain the compiler does not see which array it is in, and waits
// for all copies into LDS before the read (the reverse scan's map took 100 us
// so, and takes 87: 16401 tokens, 16 heads).
template <bool F32, int BLOCKS>
__device__ __forceinline__ TileLane tile_block(const TileLane& l, int s, int o) {
  typedef RowTiles<F32, BLOCKS> Rows;
  TileLane b = l;
#pragma unroll
  for (int e = 0; e < 4; ++e) b.col[e] = (l.col[e] ^ Rows::odd(s)) + Rows::tile(s, 0) + o * (F32 ? 1024 : 8);
  return b;
}

template <bool F32>
__device__ __forceinline__ typename Op<F32>::X tile_row(const char* tile, int odd, const TileLane& l) {
  if constexpr (F32) {
    const floatx4 a = *reinterpret_cast<const floatx4*>(tile + l.row);
    const floatx4 b = *reinterpret_cast<const floatx4*>(tile + 1024 + l.row);
    return Op<true>::narrow(a, b);
  } else {
    return *reinterpret_cast<const bf16x8*>(tile + (l.row ^ odd));
  }
}

// Channel 8 (li / 4) + 4 o + li % 4 of the tile at tokens 4 lg .. + 3.
__device__ __forceinline__ shortx4 tile_col_bf16(const char* tile, int o, int odd, const TileLane& l) {
  return __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_shortx4*)(tile + 8 * o + (l.col[0] ^ odd)));
}
__device__ __forceinline__ floatx4 tile_col_f32(const char* tile, int o, const TileLane& l) {
  floatx4 v;
#pragma unroll
  for (int e = 0; e < 4; ++e) v[e] = *reinterpret_cast<const float*>(tile + 1024 * o + l.col[e]);
  return v;
}

// The same channel of two tiles (tokens t0 .. and t1 ..) as an operand.
template <bool F32>
__device__ __forceinline__ typename Op<F32>::X tile_cols(const char* t0, const char* t1, int o, int odd,
                                                         const TileLane& l) {
  if constexpr (F32) {
    return Op<true>::narrow(tile_col_f32(t0, o, l), tile_col_f32(t1, o, l));
  } else {
    const shortx4 a = tile_col_bf16(t0, o, odd, l), b = tile_col_bf16(t1, o, odd, l);
    typedef short shortx8 __attribute__((ext_vector_type(8)));
    return __builtin_bit_cast(bf16x8, shortx8{a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]});
  }
}

// ... of one tile as fp32.
template <bool F32>
__device__ __forceinline__ floatx4 tile_values(const char* tile, int o, int odd, const TileLane& l) {
  if constexpr (F32) {
    return tile_col_f32(tile, o, l);
  } else {
    const shortx4 a = tile_col_bf16(tile, o, odd, l);
    floatx4 v;
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = __uint_as_float((uint32_t)(uint16_t)a[e] << 16);
    return v;
  }
}

// Offsets of a lane for columns in twisted order: channel 8 (li / 4) + 4 (o ^
// li / 8) + li % 4 of a tile.
struct TwistedLane {
  int row, col[2][4];
};
template <bool F32>
__device__ __forceinline__ TwistedLane twisted_lane(int li, int lg) {
  TwistedLane l;
  l.row = tile_place<F32>(li, lg);
#pragma unroll
  for (int o = 0; o < 2; ++o)
#pragma unroll
    for (int e = 0; e < 4; ++e)
      l.col[o][e] = F32 ? tile_place<true>(4 * lg + e, li >> 2) + (li & 3) * 4 + 1024 * (o ^ (li >> 3))
                        : tile_place<false>(4 * lg + (li >> 2), li & 3) + 8 * (o ^ ((li >> 1) & 1));
  return l;
}
template <bool F32>
__device__ __forceinline__ typename Op<F32>::X twisted_cols(const char* t0, const char* t1, const int (&col)[4]) {
  if constexpr (F32) {
    floatx4 a, b;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      a[e] = *reinterpret_cast<const float*>(t0 + col[e]);
      b[e] = *reinterpret_cast<const float*>(t1 + col[e]);
    }
    return Op<true>::narrow(a, b);
  } else {
    const shortx4 a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_shortx4*)(t0 + col[0]));
    const shortx4 b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_shortx4*)(t1 + col[0]));
    typedef short shortx8 __attribute__((ext_vector_type(8)));
    return __builtin_bit_cast(bf16x8, shortx8{a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]});
  }
}

// Copies 64 rows of 32 BLOCKS channels, row_bytes apart, into row tiles (as
// RowTiles has them, or TWISTED: no pairs, twisted order) by the first COPIERS
// waves (a power of two).  A row at or past `len` repeats row len - 1, so that
// every address is the sequence's own (what such rows meet is zero: their
// writes, their strengths, their stores).
template <bool F32, int BLOCKS, int COPIERS, bool TWISTED = false>
__device__ __forceinline__ void copy_tiles(__amdgpu_buffer_rsrc_t src, char* tiles, int len, uint32_t row_bytes,
                                           int wave, int lane, uint32_t from = 0) {
  constexpr bool kPairs = !TWISTED && RowTiles<F32, BLOCKS>::kPairs;
  constexpr int kHalves = F32 ? 2 : 1, kRow = row_tile_bytes<F32>();
  constexpr int kTiles = 4 * BLOCKS, kSteps = (kTiles + COPIERS - 1) / COPIERS;
  const int row = F32 ? (lane & 15) ^ (lane >> 4) : lane >> 2, lg = F32 ? lane >> 4 : (lane & 3) ^ place_shift(row);
  const uint32_t chan = (uint32_t)lg * (F32 ? 32u : 16u);
#pragma unroll
  for (int i = 0; i < kSteps; ++i) {
    const int p = wave + i * COPIERS;  // tile p % 4 of block p / 4; or half of a pair
    if (kTiles % COPIERS != 0 && p >= kTiles) break;
    if constexpr (kPairs) {
      const int in = 8 * (p & 1) + (lane >> 3), r = 16 * (p >> 1 & 3) + in;
      const uint32_t at = __umul24((uint32_t)(r < len ? r : len - 1), row_bytes) + pair_unit(in, lane & 7) * 16u;
      __builtin_amdgcn_raw_ptr_buffer_load_lds(src, (lds_void*)(tiles + p * 1024), 16, at, from + (p >> 3) * 128, 0, 0);
    } else {
      const int t = p & 3, r = TWISTED ? twisted_row(t, row) : 16 * t + row;
      const uint32_t at = __umul24((uint32_t)(r < len ? r : len - 1), row_bytes) + chan;
#pragma unroll
      for (int half = 0; half < kHalves; ++half)
        __builtin_amdgcn_raw_ptr_buffer_load_lds(src, (lds_void*)(tiles + p * kRow + half * 1024), 16, at,
                                                 from + (p >> 2) * (F32 ? 128 : 64) + half * 16, 0, 0);
    }
  }
}

// Copies BYTES (a multiple of 1024) of contiguous memory, `from` bytes behind
// src, into LDS as it is.
template <int BYTES, int COPIERS>
__device__ __forceinline__ void copy_flat(__amdgpu_buffer_rsrc_t src, char* to, int wave, int lane,
                                          uint32_t from = 0) {
  constexpr int kPieces = BYTES / 1024, kSteps = (kPieces + COPIERS - 1) / COPIERS;
#pragma unroll
  for (int i = 0; i < kSteps; ++i) {
    const int p = wave + i * COPIERS;
    if (kPieces % COPIERS != 0 && p >= kPieces) break;
    __builtin_amdgcn_raw_ptr_buffer_load_lds(src, (lds_void*)(to + p * 1024), 16, (uint32_t)lane * 16u,
                                             from + p * 1024, 0, 0);
  }
}

// No instruction is moved across (bf16 storage; fp32 operands take twice the
// registers, and there the order is left to the compiler).
template <bool F32>
__device__ __forceinline__ void fence() {
  if constexpr (!F32) __builtin_amdgcn_sched_barrier(0);
}

// Barrier behind which copies into LDS issued before it, by any wave, are
// visible: each wave first waits for its own loads and LDS operations.
// LATER: so many of the wave's memory operations at least were issued after
// the copies (stores of the step between) and need not have ended: they end
// in the order of issue.  Waiting for a step's stores as well cost about a
// microsecond of each step.
template <int LATER = 0>
__device__ __forceinline__ void copy_barrier() {
  __builtin_amdgcn_sched_barrier(0);
  __builtin_amdgcn_s_waitcnt((LATER & 15) | 0x0070 | (LATER >> 4 << 14));  // vmcnt LATER, lgkmcnt 0
  __syncthreads();
}

// ---------------------------------------------------------------------------
// Triangular 64 x 64 matrices as operand tiles: six 16 x 32 tiles each, those
// on or below the diagonal (transposed: on or above).  A tile holds each
// lane's operand contiguously: bf16 1 KB (hi), then, for a wide matrix, the
// lo tiles in a second plane; fp32 two 1 KB halves.
// ---------------------------------------------------------------------------
__host__ __device__ constexpr int tri_tile(int t, int s) { return s == 0 ? t : 2 + t; }
__host__ __device__ constexpr int tri_tile_t(int t, int s) { return s == 1 ? t : 4 + t; }
constexpr int kTriTiles = 6;
constexpr int kWideTri = kTriTiles * 2048;  // bytes of a wide (or fp32) matrix

template <bool F32>
__device__ __forceinline__ typename Op<F32>::X tile_x(const char* m, int tile, int lane) {
  if constexpr (F32) {
    const floatx4 a = *reinterpret_cast<const floatx4*>(m + tile * 2048 + lane * 16);
    const floatx4 b = *reinterpret_cast<const floatx4*>(m + tile * 2048 + 1024 + lane * 16);
    return Op<true>::narrow(a, b);
  } else {
    return *reinterpret_cast<const bf16x8*>(m + tile * 1024 + lane * 16);
  }
}

template <bool F32>
__device__ __forceinline__ typename Op<F32>::W tile_w(const char* m, int tile, int lane) {
  if constexpr (F32) {
    return typename Op<true>::W{tile_x<true>(m, tile, lane)};
  } else {
    return typename Op<false>::W{tile_x<false>(m, tile, lane),
                                 tile_x<false>(m + kTriTiles * 1024, tile, lane)};
  }
}

template <bool F32>
__device__ __forceinline__ void store_tile_x(char* m, int tile, int lane, typename Op<F32>::X x) {
  if constexpr (F32) {
    *reinterpret_cast<floatx4*>(m + tile * 2048 + lane * 16) = floatx4{x[0], x[1], x[2], x[3]};
    *reinterpret_cast<floatx4*>(m + tile * 2048 + 1024 + lane * 16) = floatx4{x[4], x[5], x[6], x[7]};
  } else {
    *reinterpret_cast<bf16x8*>(m + tile * 1024 + lane * 16) = x;
  }
}

template <bool F32>
__device__ __forceinline__ void store_tile_w(char* m, int tile, int lane, const typename Op<F32>::W& w) {
  if constexpr (F32) {
    store_tile_x<true>(m, tile, lane, w.v);
  } else {
    store_tile_x<false>(m, tile, lane, w.hi);
    store_tile_x<false>(m + kTriTiles * 1024, tile, lane, w.lo);
  }
}

// What the preparation writes for a chunk of a value head: T (wide; the beta of
// N = diag(beta) E stays outside it, as a rounded beta would be an error of a
// whole row of N), gam, eta and beta (fp32[64] each), and P (the forward pass:
// one part), or the wide transposes of T and P and G in units of log2 (64 bits)
// (the backward pass).
struct ChunkRecord {
  static constexpr int kT = 0, kVec = kWideTri, kP = kWideTri + 1024, kTt = kP, kPt = kP + kWideTri,
                       kPre = kPt + kWideTri;
  static constexpr int kPBytes[2] = {kTriTiles * 1024, kTriTiles * 2048};  // bf16, fp32
  __host__ __device__ static constexpr int bytes(bool f32, bool backward) {
    return backward ? kPre + 1024 : kP + (f32 ? kTriTiles * 2048 : kTriTiles * 1024);
  }
};

// What the scans keep for the gradient kernel (S and dS, value x key channels;
// E and dv, value channels x tokens) lies as that kernel's row tiles, 32 value
// channels after 32, in bf16 hi and lo planes or one of fp32, so that it copies
// contiguous memory.  Place r of tile t of 32 rows is row 8 (r / 4) + 4 t + r % 4
// (paired order: the order that channels have, above, for rows that are
// contracted with channels), which a scan's lane r has of half t.
// Tile: half t of rows 32 s .., block b of `blocks` of 32 columns.
__device__ __forceinline__ int keep_tile(int s, int t, int b, int blocks) { return (s * blocks + b) * 2 + t; }

// Eight channels of a state's row; place: tile_place(li, lg).
template <bool F32>
__device__ __forceinline__ void keep_state(char* base, int tile, int place, size_t plane_elems,
                                           const typename Op<F32>::W& w) {
  char* to = base + tile * row_tile_bytes<F32>() + place;
  if constexpr (F32) {
    *reinterpret_cast<floatx4*>(to) = floatx4{w.v[0], w.v[1], w.v[2], w.v[3]};
    *reinterpret_cast<floatx4*>(to + 1024) = floatx4{w.v[4], w.v[5], w.v[6], w.v[7]};
  } else {
    *reinterpret_cast<bf16x8*>(to) = w.hi;
    *reinterpret_cast<bf16x8*>(to + plane_elems * 2) = w.lo;
  }
}

// Tokens 16 u + 4 lg .. + 3 of a block of 32, of the row of place li.
template <bool F32>
__device__ __forceinline__ void keep_tokens(char* base, int tile, int u, int li, int lg, size_t plane_elems,
                                            floatx4 x) {
  char* to = base + tile * row_tile_bytes<F32>() + tile_place<F32>(li, 2 * u + (lg >> 1));
  if constexpr (F32) {
    *reinterpret_cast<floatx4*>(to + (lg & 1) * 1024) = x;
  } else {
    const uint32_t h0 = pack_bf16x2(x[0], x[1]), h1 = pack_bf16x2(x[2], x[3]);
    to += (lg & 1) * 8;
    *reinterpret_cast<uint2*>(to) = make_uint2(h0, h1);
    *reinterpret_cast<uint2*>(to + plane_elems * 2) =
        make_uint2(rest_bf16x2(x[0], x[1], h0), rest_bf16x2(x[2], x[3], h1));
  }
}

// Eight values along a row, already wide.
template <bool F32>
__device__ __forceinline__ void store_wide8(char* base, size_t elem, size_t plane_elems,
                                            const typename Op<F32>::W& w) {
  if constexpr (F32) {
    *reinterpret_cast<floatx4*>(base + elem * 4) = floatx4{w.v[0], w.v[1], w.v[2], w.v[3]};
    *reinterpret_cast<floatx4*>(base + elem * 4 + 16) = floatx4{w.v[4], w.v[5], w.v[6], w.v[7]};
  } else {
    *reinterpret_cast<bf16x8*>(base + elem * 2) = w.hi;
    *reinterpret_cast<bf16x8*>(base + (plane_elems + elem) * 2) = w.lo;
  }
}
template <bool F32>
__device__ __forceinline__ typename Op<F32>::W load_wide8(const char* base, size_t elem, size_t plane_elems) {
  if constexpr (F32)
    return typename Op<true>::W{Op<true>::narrow(*reinterpret_cast<const floatx4*>(base + elem * 4),
                                                 *reinterpret_cast<const floatx4*>(base + elem * 4 + 16))};
  else
    return typename Op<false>::W{*reinterpret_cast<const bf16x8*>(base + elem * 2),
                                 *reinterpret_cast<const bf16x8*>(base + (plane_elems + elem) * 2)};
}

// ---------------------------------------------------------------------------
// Sequences, chunks and segments
// ---------------------------------------------------------------------------

// A chunk: first token, tokens (1..64), sequence.  A segment: consecutive
// chunks of one sequence that one workgroup (per head) scans.
struct ChunkInfo {
  int tok, len, seq;  // len 0: there is no such chunk
};
struct SegmentInfo {
  int id, chunk, tok, len, seq;  // first chunk, first token, tokens; len < 0: there is no such segment
  int ends;                  // bit 0: the sequence's first, bit 1: its last
};

struct DeltaArgs {
  const void *q, *k, *v, *dout;
  const float *g, *beta;
  int Hk, Hv, group, d_v;
  // Element strides between tokens and between heads.
  size_t qk_tok, qk_head, v_tok, v_head, gate_tok, gate_head;
  float scale;
  // Sequences: n of length L each (cu null), or by table.
  int n_seqs, L, seg_chunks, max_chunks, max_segs;
  const int4 *chunk_tab, *seg_tab;
  const int *counts, *seg_id;  // chunks, segments (by table); the table's segments' numbers in order
  const float *S_in, *dS_out;    // [n][Hv][d_v][d_k] or null
  float *S_out, *dS_in;
  void *out, *dq, *dk, *dv;
  float *dg, *dbeta;
  // Workspace.
  char* rec;          // [chunk][Hv] ChunkRecord
  float *segJ, *segdJ;  // [segment][Hv] states that maps add; the entering states replace them
  char* segM;           // [segment][Hv] map matrices, wide, by rows and by columns
  char *keepS, *keepE, *keepdS, *keepdv;  // [chunk][Hv] what the gradient kernel reads
};

__device__ __forceinline__ int chunks_of(int len) { return (len + kChunk - 1) / kChunk; }

__device__ __forceinline__ ChunkInfo chunk_info(const DeltaArgs& a, int c) {
  if (a.chunk_tab != nullptr) {
    if (c >= a.counts[0]) return ChunkInfo{0, 0, 0};
    const int4 t = a.chunk_tab[c];
    return ChunkInfo{uniform(t.x), uniform(t.y), uniform(t.z)};
  }
  const int per = chunks_of(a.L);
  const int seq = uniform(c / per), at = c - seq * per;
  if (seq >= a.n_seqs) return ChunkInfo{0, 0, 0};
  const int left = a.L - at * kChunk;
  return ChunkInfo{uniform(seq * a.L + at * kChunk), uniform(left < kChunk ? left : kChunk), seq};
}

// The s-th segment to scan.
__device__ __forceinline__ SegmentInfo segment_info(const DeltaArgs& a, int s) {
  if (a.seg_tab != nullptr) {
    if (s >= a.counts[1]) return SegmentInfo{0, 0, 0, -1, 0, 0};
    const int4 t = a.seg_tab[s];
    const int w = uniform(t.w);
    return SegmentInfo{uniform(a.seg_id[s]), uniform(t.x), uniform(t.y), uniform(t.z), w >> 2, w & 3};
  }
  const int per = chunks_of(a.L);
  const int segs = (per + a.seg_chunks - 1) / a.seg_chunks;
  const int seq = uniform(s / segs), at = s - seq * segs;
  if (seq >= a.n_seqs) return SegmentInfo{0, 0, 0, -1, 0, 0};
  const int from = at * a.seg_chunks * kChunk, left = a.L - from, most = a.seg_chunks * kChunk;
  return SegmentInfo{s, uniform(seq * per + at * a.seg_chunks), uniform(seq * a.L + from),
                     uniform(left < most ? left : most), seq,
                     uniform((at == 0 ? 1 : 0) | (at == segs - 1 ? 2 : 0))};
}

// Log decays below this are taken as this: e^-200 is 0 in fp32, and sums of
// them stay finite (a decay of exactly 0, log decay -inf, among them).
constexpr float kMinLogDecay = -200.f;
// 2^x of the matrix of decays: one instruction, results below 2^-126 are 0.
__device__ __forceinline__ float pow2(double x) { return __builtin_amdgcn_exp2f((float)x); }

// Sum over aligned groups of LANES lanes (4, 8 or 16), in every lane: DPP adds.
template <int LANES>
__device__ __forceinline__ float group_sum(float x) {
  auto add = [](float v, int y) { return v + __int_as_float(y); };
  const int all = 0xf;
  x = add(x, __builtin_amdgcn_update_dpp(0, __float_as_int(x), 0xB1, all, all, false));  // quad_perm 1,0,3,2
  x = add(x, __builtin_amdgcn_update_dpp(0, __float_as_int(x), 0x4E, all, all, false));  // quad_perm 2,3,0,1
  if constexpr (LANES >= 8)
    x = add(x, __builtin_amdgcn_update_dpp(0, __float_as_int(x), 0x141, all, all, false));  // row_half_mirror
  if constexpr (LANES >= 16)
    x = add(x, __builtin_amdgcn_update_dpp(0, __float_as_int(x), 0x140, all, all, false));  // row_mirror
  return x;
}

// Inclusive prefix sums over a wave's 64 lanes of g in units of log2, in 64
// bits: differences of far prefixes keep their decay's accuracy.
__device__ __forceinline__ double decay_prefix(float g, int lane) {
  double x = (double)(g < kMinLogDecay ? kMinLogDecay : g) * 1.4426950408889634;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const double y = __shfl_up(x, d);
    if (lane >= d) x += y;
  }
  return x;
}

// Host-side launchers (arguments validated).
struct DeltaPlan {
  bool split;        // sequences are cut into segments that run side by side
  int seg_chunks;    // chunks of a segment
  int whole;         // a sequence of so many chunks is one segment
  int max_chunks, max_segs;
  size_t tabs, rec, segs, keep, total;  // workspace offsets
};
hipError_t launch_delta_plan(const int* cu, int n_seqs, int T, const DeltaPlan& plan, int* tabs,
                             hipStream_t stream);
hipError_t launch_delta_prepare(bool f32, int d_k, bool backward, const DeltaArgs& a, hipStream_t stream);
// what: 0 the segments' maps, 1 the outputs, 2 the states and writes for the gradient kernel.
hipError_t launch_delta_scan(bool f32, int d_k, int what, const DeltaArgs& a, hipStream_t stream);
hipError_t launch_delta_join(bool f32, int d_k, bool reverse, const DeltaArgs& a, hipStream_t stream);
hipError_t launch_delta_reverse(bool f32, int d_k, bool map, const DeltaArgs& a, hipStream_t stream);
hipError_t launch_delta_grad(bool f32, int d_k, const DeltaArgs& a, hipStream_t stream);

}  // namespace vda
