// Token-wise gated delta rule, backward pass: the reverse scan of the state's
// gradient over chunks, and the gradients of a chunk's inputs.
//
// With the forward pass's notation (vda_delta.h), dO the output's gradient,
// dS the gradient of the state behind the chunk:
//     dN = P^T dO + diag(eta) K dS^T,      dv = T^T diag(beta) dN   (of V)
//     dS <- gam_63 dS + scale dO^T diag(gam) Q - dv^T diag(gam) K
//     W_ij = scale D_ij dO_i.N_j (i >= j), X_ij = -D_ij dv_i.N_j (i > j)
//     dQ = scale diag(gam) dO S + W K
//     dK = W^T Q + diag(eta) N dS - diag(gam) dv S + (X + X^T) K
//     dbeta_j = E_j.(dN - L^T dv)_j
//             = sum_{i >= j} P_ij dO_i.E_j - sum_{i > j} L_ij dv_i.E_j + eta_j k_j.(E dS)_j
// The decay of token t scales what passes from before it to it or past it:
// from a token j < t to one i >= t, from the entering state to those, from
// those j to the state behind, and from state to state:
//     dg_t = gam_63 <dS, S> + sum_{i >= t} a_i + sum_{j < t} b_j + sum_{i >= t > j} A_ij,
//     A_ij = P_ij dO_i.N_j - D_ij (k_i.k_j) dv_i.N_j
//     a_i  = gam_i (scale q_i.(dO S)_i - k_i.(dv S)_i),   b_j = eta_j k_j.(N dS)_j
// The gradient kernel's products take E in N's place, and beta where their sums
// end (N_j = beta_j E_j): dbeta_j is then what A and b of token j sum to before
// beta_j, and its own output's share P_jj dO_j.E_j.
// (the sum over all (q_i.dq_i - dv_i.v_i) behind t is the same in exact
// arithmetic and needs no A, but its terms cancel to a fraction of their size:
// with wide operands its error was 2e-5 of dg where this one's is 4e-6).
// dg and dbeta are fp32 outputs: what reaches them runs on wide operands.
#include "vda_delta.h"

namespace vda {
namespace {

// The reverse scan, laid out as the forward scan (vda_delta_scan.hip): a wave
// owns 16 value columns of dS, transposed, in registers.  MAP: only what a
// segment adds to the gradient that enters it (its map's matrix is the
// forward one's transpose).  Bound by memory where its workgroups fill the
// device: 134 us for 16401 tokens of 16 heads, 128 x 128, 5.4 TB/s; the map
// 83 us.
template <bool F32, int DK, int DV, bool MAP>
__global__ __launch_bounds__(4 * DV) __attribute__((amdgpu_waves_per_eu(1, 2)))
void delta_reverse_kernel(DeltaArgs a) {
  typedef Op<F32> O;
  typedef typename O::X X;
  typedef typename O::W W;
  constexpr int ES = F32 ? 4 : 2, KS = DK / 32, kWaves = DV / 16;
  constexpr int kTileK = kChunk * DK * ES;
  constexpr int kOffQ = kTileK, kOffVec = 2 * kTileK, kOffTt = kOffVec + 1024, kOffPt = kOffTt + kWideTri,
                kOffDo = kOffPt + kWideTri, kStage = kOffDo + kChunk * DV * ES;
  constexpr int kBufs = 2 * kStage <= kLds ? 2 : 1;  // (two stages of 128 fp32 channels do not fit)
  static_assert(ChunkRecord::kTt == ChunkRecord::kVec + 1024 && ChunkRecord::kPt == ChunkRecord::kTt + kWideTri,
                "copied together");
  __shared__ __align__(16) char buf0[kStage], buf1[kBufs == 2 ? kStage : 16];

  const int h = uniform(blockIdx.x % (unsigned)a.Hv);
  const SegmentInfo si = segment_info(a, uniform(blockIdx.x / (unsigned)a.Hv));
  if (si.len < 0) return;
  const int seg = si.id;
  if (MAP && (si.ends & 1)) return;  // nothing takes the first segment's

  const int tid = threadIdx.x, lane = tid & 63, li = lane & 15, lg = lane >> 4;
  const int wave = uniform(tid >> 6);
  const int vb = wave >> 1, n0 = wave & 1;
  const int col = 32 * vb + 8 * (li >> 2) + 4 * n0 + (li & 3);  // this lane's column
  const int chunks = chunks_of(si.len);
  constexpr size_t mat = (size_t)DV * DK;
  const size_t rec_size = ChunkRecord::bytes(F32, true);
  typedef RowTiles<F32, KS> RowsK;
  typedef RowTiles<F32, DV / 32> RowsV;
  const TileLane tl = tile_lane<F32, RowsK::kPairs>(li, lg);
  const TileLane vl = tile_block<F32, DV / 32>(tile_lane<F32, RowsV::kPairs>(li, lg), vb, n0);

  const float* init = nullptr;
  if (si.ends & 2)
    init = a.dS_out ? a.dS_out + ((size_t)si.seq * a.Hv + h) * mat : nullptr;
  else if (!MAP)
    init = a.segdJ + ((size_t)seg * a.Hv + h) * mat;
  floatx4 S[KS][2];
#pragma unroll
  for (int s = 0; s < KS; ++s)
#pragma unroll
    for (int o = 0; o < 2; ++o)
      S[s][o] = init != nullptr
                    ? *reinterpret_cast<const floatx4*>(init + (size_t)col * DK + 32 * s + 8 * lg + 4 * o)
                    : floatx4{0.f, 0.f, 0.f, 0.f};

  // The chunks' rows, from the last: each chunk's 64 rows back.
  const uint32_t k_row = (uint32_t)a.qk_tok * ES, v_row = (uint32_t)a.v_tok * ES;
  const size_t last = (size_t)si.tok + (size_t)(chunks - 1) * kChunk;
  const size_t qk = (last * a.qk_tok + (size_t)(h / a.group) * a.qk_head) * ES;
  const char *kp = (const char*)a.k + qk, *qp = (const char*)a.q + qk;
  const char* op = (const char*)a.dout + (last * a.v_tok + (size_t)h * a.v_head) * ES;
  const char* rp = a.rec + ((size_t)(si.chunk + chunks - 1) * a.Hv + h) * rec_size + ChunkRecord::kVec;
  auto stage = [&](int at, char* buf) __attribute__((always_inline)) {
    const int len = min(kChunk, si.len - at * kChunk);
    copy_tiles<F32, KS, kWaves>(make_rsrc(kp, 64u * k_row), buf, len, k_row, wave, lane);
    copy_flat<1024 + 2 * kWideTri, kWaves>(make_rsrc(rp, 1024 + 2 * kWideTri), buf + kOffVec, wave, lane);
    copy_tiles<F32, DV / 32, kWaves>(make_rsrc(op, 64u * v_row), buf + kOffDo, len, v_row, wave, lane);
    copy_tiles<F32, KS, kWaves>(make_rsrc(qp, 64u * k_row), buf + kOffQ, len, k_row, wave, lane);
    kp -= 64u * k_row, qp -= 64u * k_row, op -= 64u * v_row, rp -= rec_size * a.Hv;
    __builtin_amdgcn_sched_barrier(0);  // the step's stores stay behind the copies (copy_barrier)
  };

  const floatx4 zero = {0.f, 0.f, 0.f, 0.f};
  auto step = [&](int at, const char* buf) __attribute__((always_inline)) {
    const float* gam = reinterpret_cast<const float*>(buf + kOffVec) + 4 * lg;
    const float *eta = gam + 64, *beta = gam + 128;
    const int chunk = si.chunk + at, len = si.len - at * kChunk;

    X kr[2][4], dO[2];
    auto rows = [&](int s) {
#pragma unroll
      for (int t = 0; t < 4; ++t) kr[s & 1][t] = tile_row<F32>(buf + RowsK::tile(s, t), RowsK::odd(s), tl);
    };
    rows(0);
    floatx4 ev[4];
#pragma unroll
    for (int t = 0; t < 4; ++t) ev[t] = *reinterpret_cast<const floatx4*>(eta + 16 * t);
#pragma unroll
    for (int t = 0; t < 2; ++t)
      dO[t] = tile_cols<F32>(buf + kOffDo + RowsV::tile(0, 2 * t), buf + kOffDo + RowsV::tile(0, 2 * t + 1), 0, 0, vl);
    fence<F32>();

    // dN = diag(eta) K dS^T + P^T dO.
    floatx4 dN[4];
    W M[4];
    char* ks = a.keepdS + ((size_t)chunk * a.Hv + h) * mat * 4;
#pragma unroll
    for (int s = 0; s < KS; ++s) {
      const W Sw = O::wide(S[s][0], S[s][1]);
      if constexpr (!MAP) keep_state<F32>(ks, keep_tile(vb, n0, s, KS), tile_place<F32>(li, lg), mat, Sw);
      if (s + 1 < KS)
        rows(s + 1);
      else
#pragma unroll
        for (int t = 0; t < 4; ++t) M[t] = tile_w<F32>(buf + kOffPt, tri_tile_t(t, 1), lane);
      fence<F32>();
#pragma unroll
      for (int t = 0; t < 4; ++t) dN[t] = O::mma(kr[s & 1][t], Sw, s == 0 ? zero : dN[t]);
    }
    W M0[2], Tt[4];
    floatx4 bv[4];
#pragma unroll
    for (int t = 0; t < 4; ++t) bv[t] = *reinterpret_cast<const floatx4*>(beta + 16 * t);
#pragma unroll
    for (int t = 0; t < 2; ++t) M0[t] = tile_w<F32>(buf + kOffPt, tri_tile_t(t, 0), lane);
#pragma unroll
    for (int t = 0; t < 4; ++t) dN[t] = O::mma(M[t], dO[1], dN[t] * ev[t]);
#pragma unroll
    for (int t = 0; t < 4; ++t) Tt[t] = tile_w<F32>(buf + kOffTt, tri_tile_t(t, 1), lane);
#pragma unroll
    for (int t = 0; t < 2; ++t) dN[t] = O::mma(M0[t], dO[0], dN[t]);
#pragma unroll
    for (int t = 0; t < 2; ++t) M0[t] = tile_w<F32>(buf + kOffTt, tri_tile_t(t, 0), lane);
    fence<F32>();
    W dNw[2];
#pragma unroll
    for (int s = 0; s < 2; ++s) dNw[s] = O::wide(bv[2 * s] * dN[2 * s], bv[2 * s + 1] * dN[2 * s + 1]);

    // dv = T^T (beta dN).
    floatx4 y[4], gv[4];
#pragma unroll
    for (int t = 0; t < 4; ++t) gv[t] = *reinterpret_cast<const floatx4*>(gam + 16 * t);
    // Columns of Q, then of K, half u of the channels at a time.
    X ct[KS][2];
    auto columns = [&](const char* tiles, int u) {
#pragma unroll
      for (int s = 0; s < KS; ++s)
#pragma unroll
        for (int t = 0; t < 2; ++t)
          ct[s][t] = tile_cols<F32>(tiles + RowsK::tile(s, 2 * t), tiles + RowsK::tile(s, 2 * t + 1), u,
                                    RowsK::odd(s), tl);
    };
    columns(buf + kOffQ, 0);
    fence<F32>();
#pragma unroll
    for (int t = 0; t < 4; ++t) y[t] = O::mma(Tt[t], dNw[1], zero);
#pragma unroll
    for (int t = 0; t < 2; ++t) y[t] = O::mma(M0[t], dNw[0], y[t]);

    // dS <- gam_63 dS + Q^T (scale gam dO) - K^T (gam dv); rows of dO behind
    // the chunk's end are left out here (elsewhere P or T has zeros there).
    W dOw[2];
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      floatx4 o[2];
#pragma unroll
      for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int e = 0; e < 4; ++e)
          o[u][e] = 32 * s + 16 * u + 4 * lg + e < len
                        ? a.scale * gv[2 * s + u][e] * O::value(dO[s], 4 * u + e)
                        : 0.f;
      dOw[s] = O::wide(o[0], o[1]);
    }
    const float gl = reinterpret_cast<const float*>(buf + kOffVec)[63];
    auto update = [&](int u, const W (&w)[2]) {
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int s = 0; s < KS; ++s) S[s][u] = O::mma(ct[s][t], w[t], S[s][u]);
    };
#pragma unroll
    for (int s = 0; s < KS; ++s) S[s][0] *= gl, S[s][1] *= gl;
    update(0, dOw);
    columns(buf + kOffQ, 1);
    update(1, dOw);
    columns(buf, 0);
    W yw[2];
    if constexpr (!MAP) {
      char* kd = a.keepdv + ((size_t)chunk * a.Hv + h) * DV * kChunk * 4;
#pragma unroll
      for (int t = 0; t < 4; ++t)
        keep_tokens<F32>(kd, keep_tile(vb, n0, t >> 1, 2), t & 1, li, lg, (size_t)DV * kChunk, y[t]);
    }
#pragma unroll
    for (int s = 0; s < 2; ++s) yw[s] = O::wide(-gv[2 * s] * y[2 * s], -gv[2 * s + 1] * y[2 * s + 1]);
    update(0, yw);
    columns(buf, 1);
    update(1, yw);
  };

  int at = chunks - 1;
  if constexpr (kBufs == 2) {
    if (at >= 0) stage(at, buf0);
    constexpr int kStores = MAP ? 0 : 2 * KS + (F32 ? 4 : 8);  // of a step
    for (; at >= 0; at -= 2) {
      if (at == chunks - 1)
        copy_barrier();
      else
        copy_barrier<kStores>();
      if (at >= 1) stage(at - 1, buf1);
      step(at, buf0);
      if (at < 1) break;
      copy_barrier<kStores>();
      if (at >= 2) stage(at - 2, buf0);
      step(at - 1, buf1);
    }
  } else {
    for (; at >= 0; --at) {
      if (at < chunks - 1) lds_barrier();  // every wave is done with the chunk before
      stage(at, buf0);
      copy_barrier();
      step(at, buf0);
    }
  }

  float* to = nullptr;
  if constexpr (MAP)
    to = a.segdJ + ((size_t)seg * a.Hv + h) * mat;
  else if ((si.ends & 1) && a.dS_in != nullptr)
    to = a.dS_in + ((size_t)si.seq * a.Hv + h) * mat;
  if (to != nullptr)
#pragma unroll
    for (int s = 0; s < KS; ++s)
#pragma unroll
      for (int o = 0; o < 2; ++o)
        *reinterpret_cast<floatx4*>(to + (size_t)col * DK + 32 * s + 8 * lg + 4 * o) = S[s][o];
}

// Gradients of a chunk's inputs.  One workgroup of eight waves per chunk and
// key head, over the value heads that share it in turn, whose dq and dk it
// sums in registers in a fixed order.  Wave w makes the 16 tokens of tile
// w % 4, transposed (channels x tokens), of every other four channels; of the
// scores between tokens it makes the rows of 32 tokens, and the other wave of
// the tile the others, exchanged at a head's end.  The value channels come in
// steps of 32 (S, dS, E, dv and dO of those channels), the next step's copied
// into LDS while this one's are used; all sums over value channels stay in
// registers between steps, <dS, S> too, as the diagonals of products.
// Chunks start with different steps: their matrices lie a power of two apart,
// and in step they would load the memory's channels one after another.  Tokens
// and key channels are taken in twisted order, value channels in paired order
// (vda_delta.h).
//
// 310 us for 16401 tokens of 16 heads, 128 x 128, bf16: the copies alone take
// 267 us (3.6 TB/s: with 142 KB of LDS one workgroup runs on a compute unit, one
// step's 52 KB on the way); the heads' ends, short chains of reads, sums over
// lanes and barriers, hide least of theirs.
template <bool F32, int DK, int DV>
__global__ __launch_bounds__(512) __attribute__((amdgpu_waves_per_eu(2, 2))) void delta_grad_kernel(DeltaArgs a) {
  typedef Op<F32> O;
  typedef typename O::X X;
  typedef typename O::W W;
  constexpr int ES = F32 ? 4 : 2, KS = DK / 32, kPlanes = F32 ? 1 : 2, kRow = row_tile_bytes<F32>();
  constexpr int kTileK = kChunk * DK * ES, kTileS = 32 * DK * ES, kTileN = 32 * kChunk * ES;
  // Two steps in turn: a head's are then a whole number of turns.
  constexpr int steps = DV / 32, kBufs = F32 || steps == 1 ? 1 : 2;
  constexpr int kOffdS = kPlanes * kTileS, kOffE = 2 * kPlanes * kTileS, kOffdv = kOffE + kPlanes * kTileN,
                kOffO = kOffdv + kPlanes * kTileN, kUsed = kOffO + kTileN;
  // (A head's end exchanges six operands of four tiles there.)
  constexpr int kSwap = 4 * 6 * 64 * (int)sizeof(X), kStage = kUsed > kSwap ? kUsed : kSwap;
  constexpr size_t mat = (size_t)DV * DK, nmat = (size_t)DV * kChunk;
  __shared__ __align__(16) char rowsKQ[2 * kTileK], buf0[kStage], buf1[kBufs == 2 ? kStage : 16];
  __shared__ double pre[kChunk];
  __shared__ __align__(16) float strengths[kChunk];
  __shared__ float suffix[2][kChunk], prefix[2][kChunk], writes[2][kChunk], passed[4][kChunk], states[8];

  const int hk = uniform(blockIdx.x % (unsigned)a.Hk);
  const int chunk = uniform(blockIdx.x / (unsigned)a.Hk);
  const ChunkInfo ci = chunk_info(a, chunk);
  if (ci.len == 0) return;
  const int len = ci.len;
  const int tid = threadIdx.x, lane = tid & 63, li = lane & 15, lg = lane >> 4;
  const int wave = uniform(tid >> 6);
  const int w = wave & 3, part = wave >> 2;  // token tile; the channels' half
  const int j = twisted_row(w, li);          // this lane's token
  const TwistedLane tl = twisted_lane<F32>(li, lg);
  int mine[4], own[4];  // column offsets of this wave's channels, and of its tokens
#pragma unroll
  for (int e = 0; e < 4; ++e)
    mine[e] = part ? tl.col[1][e] : tl.col[0][e], own[e] = w & 1 ? tl.col[1][e] : tl.col[0][e];

  const uint32_t k_row = (uint32_t)a.qk_tok * ES, v_row = (uint32_t)a.v_tok * ES;
  const size_t qk = ((size_t)ci.tok * a.qk_tok + (size_t)hk * a.qk_head) * ES;
  const char* const tileK = rowsKQ;
  const char* const tileQ = rowsKQ + kTileK;
  copy_tiles<F32, KS, 8, true>(make_rsrc((const char*)a.k + qk, 64u * k_row), rowsKQ, len,
                                                     k_row, wave, lane);
  copy_tiles<F32, KS, 8, true>(make_rsrc((const char*)a.q + qk, 64u * k_row), rowsKQ + kTileK,
                                                     len, k_row, wave, lane);

  const size_t first = (size_t)chunk * a.Hv + (size_t)hk * a.group;
  const size_t vo = ((size_t)ci.tok * a.v_tok + (size_t)hk * a.group * a.v_head) * ES;
  const int turned = uniform(chunk + hk);
  auto channels = [&](int n) { return (n + turned) & (steps - 1); };  // step n's value channels, 32 s ..
  // Step n: of head n / steps.  (A head's second plane is an offset.)
  auto stage = [&](int n, char* buf) __attribute__((always_inline)) {
    constexpr uint32_t kMat = mat * ES, kNmat = nmat * ES;
    const int s = channels(n);
    const size_t at = first + n / steps;
    const __amdgpu_buffer_rsrc_t sr = make_rsrc(a.keepS + at * mat * 4, kPlanes * kMat),
                                 dsr = make_rsrc(a.keepdS + at * mat * 4, kPlanes * kMat),
                                 er = make_rsrc(a.keepE + at * nmat * 4, kPlanes * kNmat),
                                 dvr = make_rsrc(a.keepdv + at * nmat * 4, kPlanes * kNmat);
#pragma unroll
    for (int p = 0; p < kPlanes; ++p) {
      const uint32_t so = p * kMat + s * kTileS;
      copy_flat<kTileS, 8>(sr, buf + p * kTileS, wave, lane, so);
      copy_flat<kTileS, 8>(dsr, buf + kOffdS + p * kTileS, wave, lane, so);
    }
    // E and dv: the planes together are a piece for each wave.
    constexpr int kPieces = kTileN / 1024;
    static_assert(kPlanes * kPieces == 8, "a piece a wave");
    const uint32_t no = wave / kPieces * kNmat + s * kTileN + wave % kPieces * 1024;
    copy_flat<1024, 1>(er, buf + kOffE + wave * 1024, 0, lane, no);
    copy_flat<1024, 1>(dvr, buf + kOffdv + wave * 1024, 0, lane, no);
    copy_tiles<F32, 1, 8, true>(
        make_rsrc((const char*)a.dout + vo + (n / steps) * a.v_head * ES, 64u * v_row), buf + kOffO, len, v_row, wave,
        lane, 32 * s * ES);
  };
  // Columns of tile block b of 32 rows of value channels: an exact operand of
  // one plane, or a wide one of all.
  auto col_x = [&](const char* tiles, int b, const int(&col)[4]) {
    return twisted_cols<F32>(tiles + 2 * b * kRow, tiles + (2 * b + 1) * kRow, col);
  };
  auto col_w = [&](const char* tiles, int plane, int b, const int(&col)[4]) {
    if constexpr (F32)
      return W{col_x(tiles, b, col)};
    else
      return W{col_x(tiles, b, col), col_x(tiles + plane, b, col)};
  };
  auto rows = [&](const char* tile) {
    if constexpr (F32)
      return Op<true>::narrow(*reinterpret_cast<const floatx4*>(tile + tl.row),
                              *reinterpret_cast<const floatx4*>(tile + 1024 + tl.row));
    else
      return *reinterpret_cast<const bf16x8*>(tile + tl.row);
  };

  const floatx4 zero = {0.f, 0.f, 0.f, 0.f};
  floatx4 dq[KS], dk[KS];
#pragma unroll
  for (int s = 0; s < KS; ++s) dq[s] = zero, dk[s] = zero;

  // Sums over a head's value channels; the scores' rows are tiles 2 part, 2 part + 1.
  floatx4 Wt[2], Wn[2], Xa[2], Xb[2], Q[KS], Ka[KS], Kb[KS], SS;
  // Of a head: this lane's token's, and (wave 0) token `lane`'s G, beta and g.
  struct Gates {
    float gam, eta, beta, ends, strength, decay;
    double pre;
  };
  auto step = [&](int n, const char* buf) __attribute__((always_inline)) {
    const char *tS = buf, *tdS = buf + kOffdS, *tE = buf + kOffE, *tdv = buf + kOffdv, *tO = buf + kOffO;
    const X Oj = rows(tO + w * kRow);
    const W Ej = col_w(tE, kTileN, w >> 1, own), vj = col_w(tdv, kTileN, w >> 1, own);
    // Products with the states, channels x tokens; operands one block ahead.
    W Sc[2], dSc[2];
    Sc[0] = col_w(tS, kTileS, 0, mine), dSc[0] = col_w(tdS, kTileS, 0, mine);
    X Et[2], Ot[2];
    W vt[2];
#pragma unroll
    for (int c = 0; c < KS; ++c) {
      if (c + 1 < KS) {
        Sc[(c + 1) & 1] = col_w(tS, kTileS, c + 1, mine), dSc[(c + 1) & 1] = col_w(tdS, kTileS, c + 1, mine);
      } else {
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          Et[u] = col_x(tE, part, tl.col[u]);
          vt[u] = col_w(tdv, kTileN, part, tl.col[u]);
          Ot[u] = rows(tO + (2 * part + u) * kRow);
        }
      }
      fence<F32>();
      Q[c] = O::mma(Sc[c & 1], Oj, Q[c]);
      Ka[c] = O::mma(dSc[c & 1], Ej, Ka[c]);
      Kb[c] = O::mma(Sc[c & 1], vj, Kb[c]);
      SS = O::mma(Sc[c & 1], dSc[c & 1], SS);
    }
    // Scores between tokens, columns of this wave (those that the order of
    // tokens rules out are left out at the head's end).
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      Wt[u] = O::mma(Et[u], Oj, Wt[u]);           // dO_j.E_i, for i <= j
      Xb[u] = O::mma(Et[u], O::head(vj), Xb[u]);  // dv_j.E_i
      Wn[u] = O::mma(Ot[u], Ej, Wn[u]);           // dO_i.E_j, for i >= j
      Xa[u] = O::mma(vt[u], Ej, Xa[u]);           // dv_i.E_j
    }
    // dv out: its rounding is its first part.  (Half of the waves store; the
    // others' stores are out of the buffer's range, as rows behind the end are.)
    const __amdgpu_buffer_rsrc_t dvr = make_rsrc((char*)a.dv + vo + (n / steps) * a.v_head * ES,
                                                 (uint32_t)(len - 1) * v_row + (uint32_t)DV * ES);
    const bool stores = part == (n & 1);
    const uint32_t off = stores ? (uint32_t)j * v_row + (uint32_t)(32 * channels(n) + 8 * lg) * ES : kOutOfRange;
    const X out = O::head(vj);
    if constexpr (F32) {
      store_b128(dvr, off, __builtin_bit_cast(u32x4, floatx4{out[0], out[1], out[2], out[3]}));
      store_b128(dvr, stores ? off + 16u : kOutOfRange,
                 __builtin_bit_cast(u32x4, floatx4{out[4], out[5], out[6], out[7]}));
    } else {
      store_b128(dvr, off, __builtin_bit_cast(u32x4, out));
    }
  };

  auto gates = [&](int h) {
    const char* rec = a.rec + ((size_t)chunk * a.Hv + h) * ChunkRecord::bytes(F32, true);
    const float* vec = reinterpret_cast<const float*>(rec + ChunkRecord::kVec);
    Gates g;
    g.gam = vec[j], g.eta = vec[64 + j], g.beta = vec[128 + j], g.ends = vec[63];
    g.strength = vec[128 + lane];
    g.pre = reinterpret_cast<const double*>(rec + ChunkRecord::kPre)[lane];
    g.decay = wave == 0 && lane < len ? a.g[(size_t)(ci.tok + lane) * a.gate_tok + (size_t)h * a.gate_head] : 0.f;
    return g;
  };
  auto clear = [&]() {
#pragma unroll
    for (int u = 0; u < 2; ++u) Wt[u] = Wn[u] = Xa[u] = Xb[u] = zero;
#pragma unroll
    for (int c = 0; c < KS; ++c) Q[c] = Ka[c] = Kb[c] = zero;
    SS = zero;
  };

  // The end of a head; `swap` is LDS that nothing else uses now.
  auto finish = [&](int h, const Gates& g, char* swap) {
    if (wave == 0) pre[lane] = g.pre, strengths[lane] = g.strength;
    // (Opaque: the comparisons below, kept from head to head, would take 100
    // scalar registers, and the kernel 343 us instead of 309, of spilled ones.)
    int jj = j, ll = lane;
    asm volatile("" : "+v"(jj), "+v"(ll));
    lds_barrier();
    // Decays between tokens: columns j of this lane.  What passes from j to
    // i > j (A): its sums over i, for token j (before beta_j), and over j, for
    // tokens i; and what j's write gives its own output.
    const double gj = pre[jj];
    floatx4 Xs[2];
    float below = 0.f, self = 0.f;
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const int t = 2 * part + u;
      floatx4 qk = zero, kk = zero;
#pragma unroll
      for (int s = 0; s < KS; ++s) {
        const X kj = rows(tileK + (4 * s + w) * kRow);
        qk = O::mma(rows(tileQ + (4 * s + t) * kRow), kj, qk);
        kk = O::mma(rows(tileK + (4 * s + t) * kRow), kj, kk);
      }
      floatx4 A = zero;
      // (The four rows of a lane are consecutive tokens.)
      const floatx4 bi = *reinterpret_cast<const floatx4*>(strengths + twisted_row(t, 4 * (ll >> 4)));
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int i = twisted_row(t, 4 * (ll >> 4) + e);
        const double apart = pre[i] - gj;
        const float d = pow2(i >= jj ? apart : -apart);
        const float wn = i >= jj && i < len ? a.scale * d * Wn[u][e] : 0.f, xa = -d * Xa[u][e];
        const float past = i > jj && i < len ? wn * qk[e] + xa * kk[e] : 0.f;
        below += past;
        self += i == jj ? wn * qk[e] : 0.f;
        A[e] = group_sum<16>(g.beta * past);
        Wt[u][e] = i <= jj ? a.scale * d * bi[e] * Wt[u][e] : 0.f;
        Wn[u][e] = g.beta * wn;
        Xs[u][e] = i > jj ? g.beta * xa : i < jj ? -d * bi[e] * Xb[u][e] : 0.f;
      }
      if (li == 0)
#pragma unroll
        for (int e = 0; e < 4; ++e) passed[w][twisted_row(t, 4 * lg + e)] = A[e];
    }
    // The tokens' operands of the two waves of a tile: [tile][tokens 32 b ..][which][lane].
    X Wy[2], Wx[2], Xx[2];
    X* const ex = reinterpret_cast<X*>(swap) + w * 6 * 64 + lane;
    ex[part * 192] = O::narrow(Wt[0], Wt[1]);
    ex[part * 192 + 64] = O::narrow(Wn[0], Wn[1]);
    ex[part * 192 + 128] = O::narrow(Xs[0], Xs[1]);
    lds_barrier();
#pragma unroll
    for (int b = 0; b < 2; ++b) Wy[b] = ex[b * 192], Wx[b] = ex[b * 192 + 64], Xx[b] = ex[b * 192 + 128];
    float in = 0.f, end = 0.f;
    const bool second = part ^ (lg >> 1);  // this lane's half of eight channels
#pragma unroll
    for (int c = 0; c < KS; ++c) {
      floatx4 x = (a.scale * g.gam) * Q[c], y = (g.eta * g.beta) * Ka[c] - g.gam * Kb[c];
      // This lane's four channels of its token's q and k.
      const X qv = rows(tileQ + (4 * c + w) * kRow), kv = rows(tileK + (4 * c + w) * kRow);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float qe = second ? O::value(qv, 4 + e) : O::value(qv, e),
                    ke = second ? O::value(kv, 4 + e) : O::value(kv, e);
        in += qe * x[e] - g.gam * ke * Kb[c][e], end += ke * Ka[c][e];
      }
#pragma unroll
      for (int b = 0; b < 2; ++b) {
        const X kt = twisted_cols<F32>(tileK + (4 * c + 2 * b) * kRow, tileK + (4 * c + 2 * b + 1) * kRow, mine);
        const X qt = twisted_cols<F32>(tileQ + (4 * c + 2 * b) * kRow, tileQ + (4 * c + 2 * b + 1) * kRow, mine);
        x = O::mma(kt, Wy[b], x);
        y = O::mma(qt, Wx[b], y);
        y = O::mma(kt, Xx[b], y);
      }
      dq[c] += x;
      dk[c] += y;
    }
    // The diagonal: this lane's share of <dS, S>.
    float ss = 0.f;
#pragma unroll
    for (int e = 0; e < 4; ++e) ss += (ll & 15) == 4 * (ll >> 4) + e ? SS[e] : 0.f;
    // Sums over the lanes of a token (lg), over the channels' halves, then over the chunk.
    float past = below + g.eta * end;
    in += __shfl_xor(in, 16), in += __shfl_xor(in, 32);
    past += __shfl_xor(past, 16), past += __shfl_xor(past, 32);
    self += __shfl_xor(self, 16), self += __shfl_xor(self, 32);
    ss = group_sum<16>(ss);
    ss += __shfl_xor(ss, 16), ss += __shfl_xor(ss, 32);
    if (lg == 0) {
      suffix[part][j] = j < len ? in : 0.f;
      prefix[part][j] = j < len ? g.beta * past : 0.f;
      writes[part][j] = past + self;
    }
    if (lane == 0) states[wave] = ss;
    lds_barrier();
    if (wave == 0) {
      // Token t = lane: sums of suffix from t on, and of prefix less passed before t.
      const float pass = (prefix[0][lane] + prefix[1][lane]) -
                         ((passed[0][lane] + passed[1][lane]) + (passed[2][lane] + passed[3][lane]));
      float x = suffix[0][lane] + suffix[1][lane], y = pass;
#pragma unroll
      for (int d = 1; d < 64; d <<= 1) {
        const float down = __shfl_down(x, d), up = __shfl_up(y, d);
        if (ll + d < 64) x += down;
        if (ll >= d) y += up;
      }
      x += y - pass + g.ends * (states[0] + states[4]);  // (all waves of a half have the same sum)
      if (lane < len) {
        const size_t at = (size_t)(ci.tok + lane) * a.gate_tok + (size_t)h * a.gate_head;
        // A decay of zero: nothing of the state before reaches the token.
        a.dg[at] = g.decay < kMinLogDecay ? 0.f : x;
        a.dbeta[at] = writes[0][lane] + writes[1][lane];
      }
    }
  };

  // Steps of all heads in turn.
  const int total = a.group * steps;
  Gates g = gates(hk * a.group);
  if constexpr (kBufs == 2) stage(0, buf0);
  for (int h = hk * a.group, n = 0; n < total; ++h) {
    clear();
    for (int s = 0; s < steps; s += kBufs, n += kBufs) {
      if constexpr (kBufs == 2) {
        if (n == 0)
          copy_barrier();
        else
          copy_barrier<1>();  // (dv of the step between)
        stage(n + 1, buf1);
        step(n, buf0);
        copy_barrier<1>();
        if (n + 2 < total) stage(n + 2, buf0);
        step(n + 1, buf1);
      } else {
        if (n > 0) lds_barrier();  // every wave is done with the step before
        stage(n, buf0);
        copy_barrier();
        step(n, buf0);
      }
    }
    const Gates next = n < total ? gates(h + 1) : g;
    lds_barrier();  // every wave is done with the last step
    finish(h, g, kBufs == 2 ? buf1 : buf0);
    g = next;
  }

  const uint32_t k_span = (uint32_t)(len - 1) * k_row + DK * ES;
  const __amdgpu_buffer_rsrc_t dqr = make_rsrc((char*)a.dq + qk, k_span);
  const __amdgpu_buffer_rsrc_t dkr = make_rsrc((char*)a.dk + qk, k_span);
#pragma unroll
  for (int c = 0; c < KS; ++c) {
    const uint32_t off = (uint32_t)j * k_row + (uint32_t)(32 * c + 8 * lg + 4 * (part ^ (lg >> 1))) * ES;
    if constexpr (F32) {
      store_b128(dqr, off, __builtin_bit_cast(u32x4, dq[c]));
      store_b128(dkr, off, __builtin_bit_cast(u32x4, dk[c]));
    } else {
      store_b64(dqr, off, make_uint2(pack_bf16x2(dq[c][0], dq[c][1]), pack_bf16x2(dq[c][2], dq[c][3])));
      store_b64(dkr, off, make_uint2(pack_bf16x2(dk[c][0], dk[c][1]), pack_bf16x2(dk[c][2], dk[c][3])));
    }
  }
}

template <bool F32, int DK, int DV>
hipError_t reverse(bool map, const DeltaArgs& a, hipStream_t stream) {
  const unsigned items = (unsigned)a.max_segs * (unsigned)a.Hv;
  if (map)
    delta_reverse_kernel<F32, DK, DV, true><<<items, 4 * DV, 0, stream>>>(a);
  else
    delta_reverse_kernel<F32, DK, DV, false><<<items, 4 * DV, 0, stream>>>(a);
  return hipGetLastError();
}

template <bool F32, int DK>
hipError_t reverse(bool map, const DeltaArgs& a, hipStream_t stream) {
  switch (a.d_v) {
    case 32: return reverse<F32, DK, 32>(map, a, stream);
    case 64: return reverse<F32, DK, 64>(map, a, stream);
    default: return reverse<F32, DK, 128>(map, a, stream);
  }
}

template <bool F32, int DK>
hipError_t grad(const DeltaArgs& a, hipStream_t stream) {
  const unsigned grid = (unsigned)a.max_chunks * (unsigned)a.Hk;
  switch (a.d_v) {
    case 32: delta_grad_kernel<F32, DK, 32><<<grid, 512, 0, stream>>>(a); break;
    case 64: delta_grad_kernel<F32, DK, 64><<<grid, 512, 0, stream>>>(a); break;
    default: delta_grad_kernel<F32, DK, 128><<<grid, 512, 0, stream>>>(a); break;
  }
  return hipGetLastError();
}

}  // namespace

hipError_t launch_delta_reverse(bool f32, int d_k, bool map, const DeltaArgs& a, hipStream_t stream) {
  switch (d_k) {
    case 32: return f32 ? reverse<true, 32>(map, a, stream) : reverse<false, 32>(map, a, stream);
    case 64: return f32 ? reverse<true, 64>(map, a, stream) : reverse<false, 64>(map, a, stream);
    default: return f32 ? reverse<true, 128>(map, a, stream) : reverse<false, 128>(map, a, stream);
  }
}

hipError_t launch_delta_grad(bool f32, int d_k, const DeltaArgs& a, hipStream_t stream) {
  switch (d_k) {
    case 32: return f32 ? grad<true, 32>(a, stream) : grad<false, 32>(a, stream);
    case 64: return f32 ? grad<true, 64>(a, stream) : grad<false, 64>(a, stream);
    default: return f32 ? grad<true, 128>(a, stream) : grad<false, 128>(a, stream);
  }
}

}  // namespace vda
