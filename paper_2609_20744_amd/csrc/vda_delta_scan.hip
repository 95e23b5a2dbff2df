// Token-wise gated delta rule: the forward state scan over chunks
// (vda_delta.h), with the outputs, with what the gradient kernel reads, or as
// the affine maps of segments; and the join of those maps.
//
// One workgroup per segment and value head; a wave owns 16 value columns of
// the state (32 in the maps), transposed (key channels x value columns), in
// registers, and nothing passes between waves: each product leaves its result
// with the rows that the next one contracts,
//     Z = K S^T -> X = V - gam Z -> N = beta T X -> S^T <- gam_63 S^T + K^T (eta N),
// so a step is three dependent products with no exchange through LDS.  The
// matrices that all waves share (k, q and v rows, T, P) come through LDS, the
// next chunk's copied by loads straight to LDS while this one's are used, one
// barrier a chunk.  O^T = S Q^T + N^T P^T takes the same registers as left
// operands, so a lane ends with eight consecutive channels of a token's output.
//
// Two waves a SIMD with 16 columns each, rather than one with 32, hide each
// other's waits (with the rows as operand tiles in LDS and copies that no store
// is waited for with, 40320 tokens of 7 heads went from 455 to 362 us).  What
// bounds it, bf16, 128 x 128: where a workgroup runs alone the chain of a chunk,
// 3.4 us (matrix cores, LDS and vector ALUs are busy a third of it each); with
// one on every compute unit memory, 83 KB a chunk: 90 us for the outputs of
// those 40320 tokens, 4.1 TB/s, and 106 us for what the gradient kernel reads
// (16401 tokens, 16 heads), 5.7 TB/s.  The maps' 5.9 us a chunk are products and
// vector operations, twice those of a scan.  Outputs that went through LDS to
// be stored in whole lines were 2% slower than eight bytes a lane.
//
// The chain of a chunk bounds a scan whose workgroups do not fill the device:
// long sequences of few heads are cut into segments.  A segment's map
// S -> S M + J is scanned first (J from zero; M, d_k x d_k, the same scan of the
// identity with v = 0), the maps are joined in order, and every segment then runs
// from its own entering state.
#include "vda_delta.h"

namespace vda {
namespace {

constexpr int kMap = 0, kOutput = 1, kKeep = 2;

// Waves of a workgroup, and 16-column blocks of a wave.  The map's workgroups
// hold both parts, waves of J, then waves of M, of 32 columns each.
template <int DK, int DV, int MODE>
struct ScanShape {
  static constexpr int kNV = MODE == kMap ? 2 : 1;
  static constexpr int kJ = DV / (16 * kNV), kWaves = MODE == kMap ? kJ + DK / 32 : kJ;
  static constexpr int kCopiers = kWaves >= 8 ? 8 : kWaves >= 4 ? 4 : kWaves >= 2 ? 2 : 1;
};

// 4 x 4 values of four lanes, a column each, transposed: a row each.
__device__ __forceinline__ floatx4 quad_transpose(floatx4 v) {
  const int lane = threadIdx.x;
#pragma unroll
  for (int m = 1; m < 4; m <<= 1)
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      if (e & m) continue;
      const bool odd = lane & m;
      const int send = __float_as_int(odd ? v[e] : v[e | m]);
      const float got = __int_as_float(m == 1 ? __builtin_amdgcn_update_dpp(0, send, 0xB1, 0xf, 0xf, false)
                                              : __builtin_amdgcn_update_dpp(0, send, 0x4E, 0xf, 0xf, false));
      v[e] = odd ? got : v[e];
      v[e | m] = odd ? v[e | m] : got;
    }
  return v;
}

// Where a map's matrix has the element (r, c): 16 x 32 tiles with each lane's
// operand, eight consecutive columns of a row, in one place.
template <int DK>
__device__ __forceinline__ size_t map_elem(int r, int c) {
  return ((size_t)((r >> 4) * (DK / 32) + (c >> 5)) * 64 + (c >> 3 & 3) * 16 + (r & 15)) * 8 + (c & 7);
}

template <bool F32, int DK, int DV, int MODE>
__global__ __launch_bounds__((64 * ScanShape<DK, DV, MODE>::kWaves))
__attribute__((amdgpu_waves_per_eu(1, 2))) void delta_scan_kernel(DeltaArgs a) {
  typedef Op<F32> O;
  typedef typename O::X X;
  typedef typename O::W W;
  typedef ScanShape<DK, DV, MODE> Shape;
  constexpr int NV = Shape::kNV, kCopiers = Shape::kCopiers;
  constexpr int ES = F32 ? 4 : 2, KS = DK / 32;
  constexpr int kTileK = kChunk * DK * ES, kTileV = kChunk * DV * ES;
  // Stage: k rows, the chunk's record (T; gam, eta and beta; outputs: P), v
  // rows, then (outputs) q rows.
  constexpr int kRecord = ChunkRecord::kP + (MODE == kOutput ? ChunkRecord::kPBytes[F32] : 0);
  constexpr int kOffT = kTileK, kOffVec = kOffT + ChunkRecord::kVec, kOffP = kOffT + ChunkRecord::kP,
                kOffV = kOffT + kRecord, kOffQ = kOffV + kTileV, kStage = kOffQ + (MODE == kOutput ? kTileK : 0);
  constexpr int kBufs = 2 * kStage <= kLds ? 2 : 1;  // (two stages of 128 fp32 channels do not fit)
  // Two arrays, each named where it is used: with one indexed by the step the
  // compiler takes any read for one of what is still being copied, and waits.
  __shared__ __align__(16) char buf0[kStage], buf1[kBufs == 2 ? kStage : 16];

  const int h = uniform(blockIdx.x % (unsigned)a.Hv);
  const SegmentInfo si = segment_info(a, uniform(blockIdx.x / (unsigned)a.Hv));
  if (si.len < 0) return;
  const int seg = si.id;
  if (MODE == kMap && (si.ends & 2)) return;  // nothing follows the last segment's map

  const int tid = threadIdx.x, lane = tid & 63, li = lane & 15, lg = lane >> 4;
  const int wave = uniform(tid >> 6);
  // The wave's columns: 32 of the state (NV 2), or one of the halves n0 of 32
  // (four of every eight).
  const bool matrix = MODE == kMap && wave >= Shape::kJ;
  const int vw = matrix ? wave - Shape::kJ : wave;
  const int vb = NV == 2 ? vw : vw >> 1, n0 = NV == 2 ? 0 : vw & 1;
  // Nothing precedes the first segment: its M is not needed.
  const bool active = !(matrix && (si.ends & 1));
  const int chunks = chunks_of(si.len);
  const size_t rec_size = ChunkRecord::bytes(F32, MODE == kKeep || (MODE == kMap && a.dout != nullptr));
  typedef RowTiles<F32, KS> RowsK;
  typedef RowTiles<F32, DV / 32> RowsV;
  const TileLane tl = tile_lane<F32, RowsK::kPairs>(li, lg);
  const TileLane vl = tile_block<F32, DV / 32>(tile_lane<F32, RowsV::kPairs>(li, lg), vb, n0);
  const int col = 32 * vb + 8 * (li >> 2) + 4 * n0 + (li & 3);  // + 4 n: this lane's columns

  // The entering state: S[s][o][n] holds channels 32 s + 8 lg + 4 o + r of column col + 4 n.
  floatx4 S[KS][2][NV];
  constexpr size_t mat = (size_t)DV * DK;
  const float* init = nullptr;
  if (!matrix) {
    if (si.ends & 1)
      init = a.S_in ? a.S_in + ((size_t)si.seq * a.Hv + h) * mat : nullptr;
    else if (MODE != kMap)
      init = a.segJ + ((size_t)seg * a.Hv + h) * mat;
  }
#pragma unroll
  for (int s = 0; s < KS; ++s)
#pragma unroll
    for (int o = 0; o < 2; ++o)
#pragma unroll
      for (int n = 0; n < NV; ++n) {
        const int ch = 32 * s + 8 * lg + 4 * o;
        S[s][o][n] = floatx4{0.f, 0.f, 0.f, 0.f};
        if (matrix) {
#pragma unroll
          for (int e = 0; e < 4; ++e) S[s][o][n][e] = ch + e == col + 4 * n ? 1.f : 0.f;
        } else if (init != nullptr) {
          S[s][o][n] = *reinterpret_cast<const floatx4*>(init + (size_t)(col + 4 * n) * DK + ch);
        }
      }

  const uint32_t k_row = (uint32_t)a.qk_tok * ES, v_row = (uint32_t)a.v_tok * ES;
  // The chunks' rows: each chunk's 64 rows further.
  const char* kp = (const char*)a.k + ((size_t)si.tok * a.qk_tok + (size_t)(h / a.group) * a.qk_head) * ES;
  const char* qp = (const char*)a.q + ((size_t)si.tok * a.qk_tok + (size_t)(h / a.group) * a.qk_head) * ES;
  const char* vp = (const char*)a.v + ((size_t)si.tok * a.v_tok + (size_t)h * a.v_head) * ES;
  const char* rp = a.rec + ((size_t)si.chunk * a.Hv + h) * rec_size;
  auto stage = [&](int c, char* buf) __attribute__((always_inline)) {
    const int len = min(kChunk, si.len - c * kChunk);
    if (Shape::kWaves == kCopiers || wave < kCopiers) {
      copy_tiles<F32, KS, kCopiers>(make_rsrc(kp, 64u * k_row), buf, len, k_row, wave, lane);
      copy_flat<kRecord, kCopiers>(make_rsrc(rp, kRecord), buf + kOffT, wave, lane);
      copy_tiles<F32, DV / 32, kCopiers>(make_rsrc(vp, 64u * v_row), buf + kOffV, len, v_row, wave, lane);
      if constexpr (MODE == kOutput)
        copy_tiles<F32, KS, kCopiers>(make_rsrc(qp, 64u * k_row), buf + kOffQ, len, k_row, wave, lane);
    }
    kp += 64u * k_row, vp += 64u * v_row, rp += rec_size * a.Hv;
    if constexpr (MODE == kOutput) qp += 64u * k_row;
    __builtin_amdgcn_sched_barrier(0);  // the step's stores stay behind the copies (copy_barrier)
  };

  const floatx4 zero = {0.f, 0.f, 0.f, 0.f};
  auto step = [&](int c, const char* buf) __attribute__((always_inline)) {
    if (!active) return;
    const float* gam = reinterpret_cast<const float*>(buf + kOffVec) + 4 * lg;
    const float *eta = gam + 64, *beta = gam + 128;
    const int chunk = si.chunk + c;

    // Operands are read from LDS a group of products ahead; the fences keep
    // the compiler from moving a group's reads down to its first use, where
    // each product would wait for them.
    X kr[2][4], qr[2][4];
    auto rows = [&](int s) {
#pragma unroll
      for (int t = 0; t < 4; ++t) {
        kr[s & 1][t] = tile_row<F32>(buf + RowsK::tile(s, t), RowsK::odd(s), tl);
        if constexpr (MODE == kOutput) qr[s & 1][t] = tile_row<F32>(buf + kOffQ + RowsK::tile(s, t), RowsK::odd(s), tl);
      }
    };
    rows(0);
    fence<F32>();

    // Z = K S^T, and the state's part of O^T = S Q^T.  With 16 columns a wave
    // there are registers for what X takes, read ahead as well.
    floatx4 z[4][NV], o[4][NV], gv[4], bv[4], vv[4][NV];
    W T[4];
    auto values = [&](int half) {
#pragma unroll
      for (int t = 2 * half; t < 2 * half + 2; ++t) {
        gv[t] = *reinterpret_cast<const floatx4*>(gam + 16 * t);
        bv[t] = *reinterpret_cast<const floatx4*>(beta + 16 * t);
#pragma unroll
        for (int n = 0; n < NV; ++n) {
          vv[t][n] = zero;
          if (!matrix) vv[t][n] = tile_values<F32>(buf + kOffV + RowsV::tile(0, t), n, 0, vl);
        }
      }
    };
    auto inverse = [&]() {
#pragma unroll
      for (int t = 0; t < 4; ++t) T[t] = tile_w<F32>(buf + kOffT, tri_tile(t, 0), lane);
    };
    char* ks = a.keepS + ((size_t)chunk * a.Hv + h) * mat * 4;
#pragma unroll
    for (int s = 0; s < KS; ++s) {
      W Sw[NV];
#pragma unroll
      for (int n = 0; n < NV; ++n) {
        Sw[n] = O::wide(S[s][0][n], S[s][1][n]);
        if constexpr (MODE == kKeep)
          keep_state<F32>(ks, keep_tile(vb, n0 + n, s, KS), tile_place<F32>(li, lg), mat, Sw[n]);
      }
      if (s + 1 < KS) rows(s + 1);
      if (NV == 1 && s + 1 == KS) {
        values(0);
        values(1);
        inverse();
      }
      fence<F32>();
#pragma unroll
      for (int t = 0; t < 4; ++t)
#pragma unroll
        for (int n = 0; n < NV; ++n) {
          z[t][n] = O::mma(kr[s & 1][t], Sw[n], s == 0 ? zero : z[t][n]);
          if constexpr (MODE == kOutput) o[t][n] = O::mma(O::head(Sw[n]), qr[s & 1][t], s == 0 ? zero : o[t][n]);
        }
    }

    // X = V - gam Z.
    W Xw[2][NV];
#pragma unroll
    for (int half = 0; half < 2; ++half) {
      if (NV == 2) values(half);
#pragma unroll
      for (int n = 0; n < NV; ++n) {
        floatx4 x[2];
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          const int t = 2 * half + u;
          x[u] = vv[t][n] - gv[t] * z[t][n];
        }
        Xw[half][n] = O::wide(x[0], x[1]);
      }
    }

    // E = T X, which is kept, and N = beta E.
    floatx4 N[4][NV];
    if (NV == 2) inverse();
#pragma unroll
    for (int t = 0; t < 4; ++t)
#pragma unroll
      for (int n = 0; n < NV; ++n) N[t][n] = O::mma(T[t], Xw[0][n], zero);
#pragma unroll
    for (int t = 2; t < 4; ++t) T[t] = tile_w<F32>(buf + kOffT, tri_tile(t, 1), lane);
#pragma unroll
    for (int t = 2; t < 4; ++t)
#pragma unroll
      for (int n = 0; n < NV; ++n) N[t][n] = O::mma(T[t], Xw[1][n], N[t][n]);
    if constexpr (MODE == kKeep) {
      char* ke = a.keepE + ((size_t)chunk * a.Hv + h) * DV * kChunk * 4;
#pragma unroll
      for (int t = 0; t < 4; ++t)
#pragma unroll
        for (int n = 0; n < NV; ++n)
          keep_tokens<F32>(ke, keep_tile(vb, n0 + n, t >> 1, 2), t & 1, li, lg, (size_t)DV * kChunk, N[t][n]);
    }
#pragma unroll
    for (int t = 0; t < 4; ++t)
#pragma unroll
      for (int n = 0; n < NV; ++n) N[t][n] *= bv[t];

    // Columns of K for the update, half u of the channels at a time.
    X kt[KS][2];
    auto columns = [&](int u) {
#pragma unroll
      for (int s = 0; s < KS; ++s)
#pragma unroll
        for (int t = 0; t < 2; ++t)
          kt[s][t] = tile_cols<F32>(buf + RowsK::tile(s, 2 * t), buf + RowsK::tile(s, 2 * t + 1), u, RowsK::odd(s), tl);
    };

    if constexpr (MODE == kOutput) {
      X Nx[2][NV], P[kTriTiles];
      float gq[4];
#pragma unroll
      for (int t = 0; t < 4; ++t) gq[t] = reinterpret_cast<const float*>(buf + kOffVec)[16 * t + li];
#pragma unroll
      for (int i = 0; i < kTriTiles; ++i) P[i] = tile_x<F32>(buf + kOffP, i, lane);
#pragma unroll
      for (int s = 0; s < 2; ++s)
#pragma unroll
        for (int n = 0; n < NV; ++n) Nx[s][n] = O::narrow(N[2 * s][n], N[2 * s + 1][n]);
      columns(0);
      fence<F32>();
      const int tok = si.tok + c * kChunk, len = min(kChunk, si.len - c * kChunk);
      const size_t vo = (size_t)tok * a.v_tok + (size_t)h * a.v_head;
      const __amdgpu_buffer_rsrc_t orsrc =
          make_rsrc((char*)a.out + vo * ES, (uint32_t)(len - 1) * v_row + DV * ES);
#pragma unroll
      for (int t = 0; t < 4; ++t) {
#pragma unroll
        for (int n = 0; n < NV; ++n) {
          o[t][n] = O::mma(Nx[0][n], P[tri_tile(t, 0)], (a.scale * gq[t]) * o[t][n]);
          if (t >= 2) o[t][n] = O::mma(Nx[1][n], P[tri_tile(t, 1)], o[t][n]);
        }
        // Rows behind the chunk's end are out of the buffer's range.
        const uint32_t off = (uint32_t)(16 * t + li) * v_row + (uint32_t)(32 * vb + 8 * lg + 4 * n0) * ES;
        if constexpr (F32) {
#pragma unroll
          for (int n = 0; n < NV; ++n) store_b128(orsrc, off + 16 * n, __builtin_bit_cast(u32x4, o[t][n]));
        } else if constexpr (NV == 2) {
          store_b128(orsrc, off, __builtin_bit_cast(u32x4, O::narrow(o[t][0], o[t][1])));
        } else {
          store_b64(orsrc, off,
                    make_uint2(pack_bf16x2(o[t][0][0], o[t][0][1]), pack_bf16x2(o[t][0][2], o[t][0][3])));
        }
      }
    } else {
      columns(0);
      fence<F32>();
    }

    // S <- gam_63 S + N^T diag(eta) K.
    W Nw[2][NV];
#pragma unroll
    for (int s = 0; s < 2; ++s)
#pragma unroll
      for (int n = 0; n < NV; ++n)
        Nw[s][n] = O::wide(N[2 * s][n] * *reinterpret_cast<const floatx4*>(eta + 32 * s),
                           N[2 * s + 1][n] * *reinterpret_cast<const floatx4*>(eta + 32 * s + 16));
    const float gl = reinterpret_cast<const float*>(buf + kOffVec)[63];
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      if (u == 1) columns(1);
#pragma unroll
      for (int s = 0; s < KS; ++s)
#pragma unroll
        for (int n = 0; n < NV; ++n) S[s][u][n] *= gl;
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int s = 0; s < KS; ++s)
#pragma unroll
          for (int n = 0; n < NV; ++n) S[s][u][n] = O::mma(kt[s][t], Nw[t][n], S[s][u][n]);
    }
  };

  if constexpr (kBufs == 2) {
    if (chunks > 0) stage(0, buf0);
    // Stores of a step, all of them of every wave.
    constexpr int kStores = MODE == kOutput ? 4 : MODE == kKeep ? 2 * KS + (F32 ? 4 : 8) : 0;
    for (int c = 0; c < chunks; c += 2) {
      if (c == 0)
        copy_barrier();
      else
        copy_barrier<kStores>();
      if (c + 1 < chunks) stage(c + 1, buf1);
      step(c, buf0);
      if (c + 1 >= chunks) break;
      copy_barrier<kStores>();
      if (c + 2 < chunks) stage(c + 2, buf0);
      step(c + 1, buf1);
    }
  } else {
    for (int c = 0; c < chunks; ++c) {
      if (c > 0) lds_barrier();  // every wave is done with the chunk before
      stage(c, buf0);
      copy_barrier();
      step(c, buf0);
    }
  }

  if (!active) return;
  const size_t km = (size_t)DK * DK;
#pragma unroll
  for (int s = 0; s < KS; ++s)
#pragma unroll
    for (int n = 0; n < NV; ++n) {
      const int u = col + 4 * n, ch = 32 * s + 8 * lg;
      if (MODE == kMap && matrix) {
        // M by rows and by columns, each as wide operand tiles of the join.
        char* m = a.segM + ((size_t)seg * a.Hv + h) * 2 * km * 4;
        store_wide8<F32>(m, map_elem<DK>(u, ch), km, O::wide(S[s][0][n], S[s][1][n]));
        if (n == 0) {
#pragma unroll
          for (int o = 0; o < 2; ++o)
            store_wide8<F32>(m + km * 4, map_elem<DK>(ch + 4 * o + (li & 3), 32 * vb + 8 * (li >> 2)), km,
                             O::wide(quad_transpose(S[s][o][0]), quad_transpose(S[s][o][NV - 1])));
        }
      } else {
        float* to = nullptr;
        if (MODE == kMap)
          to = a.segJ + ((size_t)seg * a.Hv + h) * mat;
        else if ((si.ends & 2) && a.S_out != nullptr)
          to = a.S_out + ((size_t)si.seq * a.Hv + h) * mat;
        if (to != nullptr) {
          *reinterpret_cast<floatx4*>(to + (size_t)u * DK + ch) = S[s][0][n];
          *reinterpret_cast<floatx4*>(to + (size_t)u * DK + ch + 4) = S[s][1][n];
        }
      }
    }
}

// The join: x <- x M_s + J_s over the segments of a sequence in order (or, in
// reverse, x <- x M_s^T + J_s from the last), the state entering each segment
// written over its J.  The rows of a state are independent of each other: one
// workgroup of four waves per sequence, head and 16 rows; a wave makes d_k / 4
// columns of the product (transposed, the matrix as left operand), which the
// others get through LDS (two waves at d_k 32).  The matrices are read two
// segments ahead, a KB of operands at a time (as rows, 16 bytes of 16 rows at a
// time, a step took 2.1 us; now 1.1 us at d_k 128, of loads and their latency).
template <bool F32, int DK>
__global__ __launch_bounds__(kThreads) void delta_join_kernel(DeltaArgs a, bool reverse) {
  typedef Op<F32> O;
  typedef typename O::W W;
  constexpr int KS = DK / 32, NC = DK / 16, WT = (NC + 3) / 4;
  constexpr int kRow = DK + 4;
  __shared__ __align__(16) float x[2][16 * kRow];
  // Workgroups go round the eight dies: those of one sequence and head, which
  // read the same matrices, to one of them.
  const int blocks = a.d_v / 16;
  const int rb = blockIdx.x / 8 % blocks;
  const int item = uniform(blockIdx.x / (8 * blocks) * 8 + blockIdx.x % 8);
  const int seq = uniform(item / a.Hv), h = item - seq * a.Hv;
  if (seq >= a.n_seqs) return;
  const int tid = threadIdx.x, lane = tid & 63, li = lane & 15, lg = lane >> 4;
  const int wave = uniform(tid >> 6);
  // The sequence's segments.
  int first, count;
  if (a.seg_tab != nullptr) {
    const int* spre = a.counts + 4 + a.n_seqs + 1;
    first = spre[seq], count = spre[seq + 1] - first;
    if (first + count > a.counts[1]) count = a.counts[1] - first;
  } else {
    const int per = chunks_of(a.L);
    count = (per + a.seg_chunks - 1) / a.seg_chunks, first = seq * count;
  }
  if (count < 2) return;
  float* J = reverse ? a.segdJ : a.segJ;
  const size_t mat = (size_t)a.d_v * DK, km = (size_t)DK * DK;
  const int row = rb * 16 + li;
  auto index = [&](int i) { return (size_t)(reverse ? first + count - 1 - i : first + i) * a.Hv + h; };
  // Result columns 16 c + 4 lg .. of this wave, c = wave WT + w; the matrix's
  // operand rows 16 c + li.  Past the last segment its own place is read again
  // (in bounds, and not used).
  W m[2][WT][KS];
  floatx4 y[WT], add[2][WT];
  auto load = [&](int i, int slot) __attribute__((always_inline)) {
    const size_t at = index(i < count ? i : count - 1);
    const char* mi = a.segM + at * 2 * km * 4 + (reverse ? 0 : km * 4);
    const float* Ji = J + at * mat + (size_t)row * DK;
#pragma unroll
    for (int w = 0; w < WT; ++w) {
      const int c = wave * WT + w;
      add[slot][w] = *reinterpret_cast<const floatx4*>(Ji + 16 * c + 4 * lg);
#pragma unroll
      for (int s = 0; s < KS; ++s)
        m[slot][w][s] = load_wide8<F32>(mi, map_elem<DK>(16 * c + li, 32 * s + 8 * lg), km);
    }
  };
  // After segment 0 the state is its own J (scanned from the sequence's state).
#pragma unroll
  for (int w = 0; w < WT; ++w)
    y[w] = *reinterpret_cast<const floatx4*>(J + index(0) * mat + (size_t)row * DK + 16 * (wave * WT + w) + 4 * lg);
  // Segment i; false after the last.
  auto join = [&](int i, int slot) __attribute__((always_inline)) {
    float* buf = x[slot];
    float* Ji = J + index(i) * mat + (size_t)row * DK;
#pragma unroll
    for (int w = 0; w < WT; ++w) {
      const int c = wave * WT + w;
      *reinterpret_cast<floatx4*>(Ji + 16 * c + 4 * lg) = y[w];
      *reinterpret_cast<floatx4*>(buf + li * kRow + 16 * c + 4 * lg) = y[w];
    }
    if (i + 1 == count) return false;
    lds_barrier();
#pragma unroll
    for (int w = 0; w < WT; ++w) y[w] = add[slot][w];
#pragma unroll
    for (int s = 0; s < KS; ++s) {
      const float* xr = buf + li * kRow + 32 * s + 8 * lg;
      const W xo = O::wide(*reinterpret_cast<const floatx4*>(xr), *reinterpret_cast<const floatx4*>(xr + 4));
#pragma unroll
      for (int w = 0; w < WT; ++w) y[w] = O::mma(m[slot][w][s], xo, y[w]);
    }
    load(i + 2, slot);
    return true;
  };
  load(1, 1);
  load(2, 0);
  for (int i = 1;; i += 2)
    if (!join(i, 1) || !join(i + 1, 0)) return;
}

template <bool F32, int DK, int DV>
hipError_t run(int what, const DeltaArgs& a, hipStream_t stream) {
  const unsigned items = (unsigned)a.max_segs * (unsigned)a.Hv;
  if (what == kMap)
    delta_scan_kernel<F32, DK, DV, kMap><<<items, 64 * ScanShape<DK, DV, kMap>::kWaves, 0, stream>>>(a);
  else if (what == kOutput)
    delta_scan_kernel<F32, DK, DV, kOutput><<<items, 64 * ScanShape<DK, DV, kOutput>::kWaves, 0, stream>>>(a);
  else
    delta_scan_kernel<F32, DK, DV, kKeep><<<items, 64 * ScanShape<DK, DV, kKeep>::kWaves, 0, stream>>>(a);
  return hipGetLastError();
}

template <bool F32, int DK>
hipError_t run(int what, const DeltaArgs& a, hipStream_t stream) {
  switch (a.d_v) {
    case 32: return run<F32, DK, 32>(what, a, stream);
    case 64: return run<F32, DK, 64>(what, a, stream);
    default: return run<F32, DK, 128>(what, a, stream);
  }
}

template <bool F32>
hipError_t join(int d_k, bool reverse, const DeltaArgs& a, hipStream_t stream) {
  const unsigned grid = ((unsigned)a.n_seqs * (unsigned)a.Hv + 7) / 8 * 8 * (unsigned)(a.d_v / 16);
  switch (d_k) {
    case 32: delta_join_kernel<F32, 32><<<grid, 128, 0, stream>>>(a, reverse); break;
    case 64: delta_join_kernel<F32, 64><<<grid, kThreads, 0, stream>>>(a, reverse); break;
    default: delta_join_kernel<F32, 128><<<grid, kThreads, 0, stream>>>(a, reverse); break;
  }
  return hipGetLastError();
}

}  // namespace

hipError_t launch_delta_scan(bool f32, int d_k, int what, const DeltaArgs& a, hipStream_t stream) {
  switch (d_k) {
    case 32: return f32 ? run<true, 32>(what, a, stream) : run<false, 32>(what, a, stream);
    case 64: return f32 ? run<true, 64>(what, a, stream) : run<false, 64>(what, a, stream);
    default: return f32 ? run<true, 128>(what, a, stream) : run<false, 128>(what, a, stream);
  }
}

hipError_t launch_delta_join(bool f32, int d_k, bool reverse, const DeltaArgs& a, hipStream_t stream) {
  return f32 ? join<true>(d_k, reverse, a, stream) : join<false>(d_k, reverse, a, stream);
}

}  // namespace vda
