// Token-wise gated delta rule, backward pass: the reverse scan of the state's
// gradient over chunks, and the gradients of a chunk's inputs.
//
// With the forward pass's notation (vda_delta.h), dO the output's gradient,
// dS the gradient of the state behind the chunk and dv = diag(beta) y:
//     dN = P^T dO + diag(eta) K dS^T,      dv = diag(beta) T^T dN   (of V)
//     dS <- gam_63 dS + scale dO^T diag(gam) Q - dv^T diag(gam) K
//     W_ij = scale D_ij dO_i.N_j (i >= j), X_ij = -D_ij dv_i.N_j (i > j)
//     dQ = scale diag(gam) dO S + W K
//     dK = W^T Q + diag(eta) N dS - diag(gam) dv S + (X + X^T) K
//     dbeta_i = (N_i / beta_i).(dv_i / beta_i)
// The decay of token t scales what passes from before it to it or past it:
// from a token j < t to one i >= t, from the entering state to those, from
// those j to the state behind, and from state to state:
//     dg_t = gam_63 <dS, S> + sum_{i >= t} a_i + sum_{j < t} b_j + sum_{i >= t > j} A_ij,
//     A_ij = P_ij dO_i.N_j - D_ij (k_i.k_j) dv_i.N_j
//     a_i  = gam_i (scale q_i.(dO S)_i - k_i.(dv S)_i),   b_j = eta_j k_j.(N dS)_j
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
// forward one's transpose).
template <bool F32, int DK, bool MAP>
__global__ __launch_bounds__(512) void delta_reverse_kernel(DeltaArgs a) {
  typedef Op<F32> O;
  typedef typename O::X X;
  typedef typename O::W W;
  constexpr int ES = F32 ? 4 : 2, KS = DK / 32, NC = DK / 16;
  constexpr int kLuK = __builtin_ctz(DK * ES / 16);
  constexpr int kBufs = F32 ? 1 : 2;
  constexpr int kTileK = kChunk * DK * ES;
  constexpr int kOffQ = kTileK, kOffVec = 2 * kTileK, kOffTt = kOffVec + 1024, kOffPt = kOffTt + kWideTri,
                kOffDo = kOffPt + kWideTri, kStage = kOffDo + kChunk * 128 * ES;
  static_assert(ChunkRecord::kTt == ChunkRecord::kVec + 1024 && ChunkRecord::kPt == ChunkRecord::kTt + kWideTri,
                "copied together");
  __shared__ __align__(16) char lds[kBufs * kStage];

  const int DV = a.d_v;
  const int h = uniform(blockIdx.x % (unsigned)a.Hv);
  const int seg = uniform(blockIdx.x / (unsigned)a.Hv);
  const SegmentInfo si = segment_info(a, seg);
  if (si.chunks < 0) return;
  if (MAP && (si.ends & 1)) return;  // nothing takes the first segment's

  const int tid = threadIdx.x, lane = tid & 63, li = lane & 15, lg = lane >> 4;
  const int wave = uniform(tid >> 6), waves = uniform(blockDim.x >> 6);
  const int v0 = wave * 16, col = v0 + li;
  const int luv = __builtin_ctz(DV * ES / 16);
  const size_t mat = (size_t)DV * DK;
  const size_t rec_size = ChunkRecord::bytes(F32, true);

  const float* init = nullptr;
  if (si.ends & 2)
    init = a.dS_out ? a.dS_out + ((size_t)si.seq * a.Hv + h) * mat : nullptr;
  else if (!MAP)
    init = a.segdJ + ((size_t)seg * a.Hv + h) * mat;
  floatx4 S[NC];
#pragma unroll
  for (int c = 0; c < NC; ++c)
    S[c] = init != nullptr ? *reinterpret_cast<const floatx4*>(init + (size_t)col * DK + 16 * c + 4 * lg)
                           : floatx4{0.f, 0.f, 0.f, 0.f};

  const uint32_t k_row = (uint32_t)a.qk_tok * ES, v_row = (uint32_t)a.v_tok * ES;
  auto stage = [&](int step) {
    char* buf = lds + (kBufs == 2 && (step & 1) ? kStage : 0);
    const int chunk = si.chunk + si.chunks - 1 - step;
    const ChunkInfo ci = chunk_info(a, chunk);
    const char* rec = a.rec + ((size_t)chunk * a.Hv + h) * rec_size;
    const size_t qk = (size_t)ci.tok * a.qk_tok + (size_t)(h / a.group) * a.qk_head;
    const size_t vo = (size_t)ci.tok * a.v_tok + (size_t)h * a.v_head;
    const uint32_t k_span = (uint32_t)(ci.len - 1) * k_row + DK * ES;
    copy_rows<F32>(make_rsrc((const char*)a.k + qk * ES, k_span), buf, kLuK, kChunk, ci.len, k_row, wave,
                   waves, lane);
    copy_rows<F32>(make_rsrc((const char*)a.q + qk * ES, k_span), buf + kOffQ, kLuK, kChunk, ci.len, k_row,
                   wave, waves, lane);
    copy_rows<F32>(make_rsrc((const char*)a.dout + vo * ES, (uint32_t)(ci.len - 1) * v_row + DV * ES),
                   buf + kOffDo, luv, kChunk, ci.len, v_row, wave, waves, lane);
    copy_flat(rec + ChunkRecord::kVec, buf + kOffVec, 1024 + 2 * kWideTri, wave, waves, lane);
  };

  if (si.chunks > 0) stage(0);
  for (int step = 0; step < si.chunks; ++step) {
    copy_barrier();
    if (kBufs == 2 && step + 1 < si.chunks) stage(step + 1);
    const char* buf = lds + (kBufs == 2 && (step & 1) ? kStage : 0);
    const float* gam = reinterpret_cast<const float*>(buf + kOffVec);
    const float *eta = gam + 64, *beta = gam + 128;
    const int chunk = si.chunk + si.chunks - 1 - step;
    const int len = chunk_info(a, chunk).len;

    W Sw[KS];
#pragma unroll
    for (int s = 0; s < KS; ++s) Sw[s] = O::wide(S[2 * s], S[2 * s + 1]);
    if constexpr (!MAP) {
      char* ks = a.keepdS + ((size_t)chunk * a.Hv + h) * mat * 4;
#pragma unroll
      for (int c = 0; c < NC; ++c) store_wide4<F32>(ks, (size_t)col * DK + 16 * c + 4 * lg, mat, S[c]);
    }

    // dN = diag(eta) K dS^T + P^T dO.
    X dO[2];
#pragma unroll
    for (int s = 0; s < 2; ++s) dO[s] = col_op<F32>(buf + kOffDo, luv, 32 * s, v0, li, lg);
    floatx4 dN[4];
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      dN[t] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int s = 0; s < KS; ++s) dN[t] = O::mma(row_op<F32>(buf, kLuK, 16 * t + li, s, lg), Sw[s], dN[t]);
      dN[t] *= *reinterpret_cast<const floatx4*>(eta + 16 * t + 4 * lg);
#pragma unroll
      for (int s = t / 2; s < 2; ++s)
        dN[t] = O::mma(tile_w<F32>(buf + kOffPt, tri_tile_t(t, s), lane), dO[s], dN[t]);
    }
    W dNw[2];
#pragma unroll
    for (int s = 0; s < 2; ++s) dNw[s] = O::wide(dN[2 * s], dN[2 * s + 1]);

    // dv = beta T^T dN.
    floatx4 y[4];
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      y[t] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int s = t / 2; s < 2; ++s)
        y[t] = O::mma(tile_w<F32>(buf + kOffTt, tri_tile_t(t, s), lane), dNw[s], y[t]);
      y[t] *= *reinterpret_cast<const floatx4*>(beta + 16 * t + 4 * lg);
    }
    if constexpr (!MAP) {
      char* kd = a.keepdv + ((size_t)chunk * a.Hv + h) * DV * kChunk * 4;
#pragma unroll
      for (int t = 0; t < 4; ++t)
        store_wide4<F32>(kd, (size_t)col * kChunk + 16 * t + 4 * lg, (size_t)DV * kChunk, y[t]);
    }

    // dS <- gam_63 dS + Q^T (scale gam dO) - K^T (gam dv); rows of dO behind
    // the chunk's end are left out here (elsewhere P or T has zeros there).
    W dOw[2], yw[2];
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      floatx4 o[2], g[2];
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        g[u] = *reinterpret_cast<const floatx4*>(gam + 32 * s + 16 * u + 4 * lg);
#pragma unroll
        for (int e = 0; e < 4; ++e)
          o[u][e] = 32 * s + 16 * u + 4 * lg + e < len ? a.scale * g[u][e] * O::value(dO[s], 4 * u + e) : 0.f;
      }
      dOw[s] = O::wide(o[0], o[1]);
      yw[s] = O::wide(-g[0] * y[2 * s], -g[1] * y[2 * s + 1]);
    }
    const float gl = gam[63];
#pragma unroll
    for (int c = 0; c < NC; ++c) {
      S[c] *= gl;
#pragma unroll
      for (int s = 0; s < 2; ++s) {
        S[c] = O::mma(col_op<F32>(buf + kOffQ, kLuK, 32 * s, 16 * c, li, lg), dOw[s], S[c]);
        S[c] = O::mma(col_op<F32>(buf, kLuK, 32 * s, 16 * c, li, lg), yw[s], S[c]);
      }
    }
    if (kBufs == 1 && step + 1 < si.chunks) {
      lds_barrier();
      stage(step + 1);
    }
  }

  float* to = nullptr;
  if constexpr (MAP)
    to = a.segdJ + ((size_t)seg * a.Hv + h) * mat;
  else if ((si.ends & 1) && a.dS_in != nullptr)
    to = a.dS_in + ((size_t)si.seq * a.Hv + h) * mat;
  if (to != nullptr)
#pragma unroll
    for (int c = 0; c < NC; ++c) *reinterpret_cast<floatx4*>(to + (size_t)col * DK + 16 * c + 4 * lg) = S[c];
}

// Gradients of a chunk's inputs.  One workgroup of four waves per chunk and
// key head, over the value heads that share it in turn, whose dq and dk it
// sums in registers in a fixed order; wave w makes the 16 tokens of block w,
// transposed (channels x tokens), so a lane stores consecutive channels.  The
// value channels come in steps of 32 (S, dS, N, dv and dO of those channels),
// the next step's copied into LDS while this one's are used; all sums over
// value channels stay in registers between steps.
template <bool F32, int DK>
__global__ __launch_bounds__(kThreads) void delta_grad_kernel(DeltaArgs a) {
  typedef Op<F32> O;
  typedef typename O::X X;
  typedef typename O::W W;
  constexpr int ES = F32 ? 4 : 2, NC = DK / 16, kPlanes = F32 ? 1 : 2;
  constexpr int kLuK = __builtin_ctz(DK * ES / 16), kLuN = F32 ? 4 : 3, kLuO = F32 ? 3 : 2;
  constexpr int kTileK = kChunk * DK * ES, kTileS = 32 * DK * ES, kTileN = 32 * kChunk * ES;
  constexpr int kBufs = F32 ? 1 : 2;
  constexpr int kOffdS = kPlanes * kTileS, kOffN = 2 * kPlanes * kTileS, kOffdv = kOffN + kPlanes * kTileN,
                kOffO = kOffdv + kPlanes * kTileN, kStage = kOffO + kTileN;
  __shared__ __align__(16) char lds[2 * kTileK + kBufs * kStage];
  __shared__ double pre[kChunk];
  __shared__ float gam[kChunk], eta[kChunk], strengths[kChunk], suffix[kChunk], prefix[kChunk], rows[4][kChunk],
      states[4];

  const int hk = uniform(blockIdx.x % (unsigned)a.Hk);
  const int chunk = uniform(blockIdx.x / (unsigned)a.Hk);
  const ChunkInfo ci = chunk_info(a, chunk);
  if (ci.len == 0) return;
  const int DV = a.d_v, steps = DV / 32, len = ci.len;
  const int tid = threadIdx.x, lane = tid & 63, li = lane & 15, lg = lane >> 4;
  const int wave = uniform(tid >> 6);
  const int j0 = 16 * wave, j = j0 + li;  // this lane's token
  const size_t mat = (size_t)DV * DK, nmat = (size_t)DV * kChunk;

  const uint32_t k_row = (uint32_t)a.qk_tok * ES, v_row = (uint32_t)a.v_tok * ES;
  const size_t qk = (size_t)ci.tok * a.qk_tok + (size_t)hk * a.qk_head;
  const uint32_t k_span = (uint32_t)(len - 1) * k_row + DK * ES;
  const uint32_t v_span = (uint32_t)(len - 1) * v_row + DV * ES;
  const char* const tileK = lds;
  const char* const tileQ = lds + kTileK;
  char* const ring = lds + 2 * kTileK;
  copy_rows<F32>(make_rsrc((const char*)a.k + qk * ES, k_span), lds, kLuK, kChunk, len, k_row, wave, 4, lane);
  copy_rows<F32>(make_rsrc((const char*)a.q + qk * ES, k_span), lds + kTileK, kLuK, kChunk, len, k_row, wave, 4,
                 lane);

  const int total = a.group * steps;
  auto stage = [&](int n) {
    char* buf = ring + (kBufs == 2 && (n & 1) ? kStage : 0);
    const int h = hk * a.group + n / steps, s = n % steps;
    const size_t at = (size_t)chunk * a.Hv + h;
#pragma unroll
    for (int p = 0; p < kPlanes; ++p) {
      const size_t so = at * mat * 4 + ((size_t)p * mat + (size_t)32 * s * DK) * ES;
      const size_t no = at * nmat * 4 + ((size_t)p * nmat + (size_t)32 * s * kChunk) * ES;
      copy_rows<F32>(make_rsrc(a.keepS + so, kTileS), buf + p * kTileS, kLuK, 32, 32, DK * ES, wave, 4, lane);
      copy_rows<F32>(make_rsrc(a.keepdS + so, kTileS), buf + kOffdS + p * kTileS, kLuK, 32, 32, DK * ES, wave, 4,
                     lane);
      copy_rows<F32>(make_rsrc(a.keepN + no, kTileN), buf + kOffN + p * kTileN, kLuN, 32, 32, kChunk * ES, wave, 4,
                     lane);
      copy_rows<F32>(make_rsrc(a.keepdv + no, kTileN), buf + kOffdv + p * kTileN, kLuN, 32, 32, kChunk * ES, wave,
                     4, lane);
    }
    const size_t vo = (size_t)ci.tok * a.v_tok + (size_t)h * a.v_head + 32 * s;
    copy_rows<F32>(make_rsrc((const char*)a.dout + vo * ES, (uint32_t)(len - 1) * v_row + 32 * ES), buf + kOffO,
                   kLuO, kChunk, len, v_row, wave, 4, lane);
  };
  // A wide operand from the planes of a tile.
  auto wide_col = [&](const char* tile, int plane, int lu, int c0) {
    if constexpr (F32)
      return W{col_op<true>(tile, lu, 0, c0, li, lg)};
    else
      return W{col_op<false>(tile, lu, 0, c0, li, lg), col_op<false>(tile + plane, lu, 0, c0, li, lg)};
  };

  const floatx4 zero = {0.f, 0.f, 0.f, 0.f};
  floatx4 dq[NC], dk[NC];
#pragma unroll
  for (int c = 0; c < NC; ++c) dq[c] = zero, dk[c] = zero;
  stage(0);
  for (int hv = 0; hv < a.group; ++hv) {
    const int h = hk * a.group + hv;
    // The head's decays and strengths (the barrier below comes before their use).
    if (hv > 0) lds_barrier();
    if (wave == 0) {
      const size_t at = (size_t)(ci.tok + lane) * a.gate_tok + (size_t)h * a.gate_head;
      const bool real = lane < len;
      const double G = decay_prefix(real ? a.g[at] : 0.f, lane);
      const double last = __shfl(G, 63);
      pre[lane] = G;
      gam[lane] = exp2f((float)G);
      eta[lane] = exp2f((float)(last - G));
      strengths[lane] = real ? strength(a.beta[at]) : 1.f;
    }
    floatx4 Wt[4], Wn[4], Xa[4], Xb[4], Q[NC], Ka[NC], Kb[NC];
#pragma unroll
    for (int t = 0; t < 4; ++t) Wt[t] = Wn[t] = Xa[t] = Xb[t] = zero;
#pragma unroll
    for (int c = 0; c < NC; ++c) Q[c] = Ka[c] = Kb[c] = zero;
    float db = 0.f, ss = 0.f;
    const size_t vo = (size_t)ci.tok * a.v_tok + (size_t)h * a.v_head;
    const __amdgpu_buffer_rsrc_t dvr = make_rsrc((char*)a.dv + vo * ES, v_span);
    for (int s = 0; s < steps; ++s) {
      const int n = hv * steps + s;
      copy_barrier();
      if (kBufs == 2 && n + 1 < total) stage(n + 1);
      const char* buf = ring + (kBufs == 2 && (n & 1) ? kStage : 0);
      const char *tS = buf, *tdS = buf + kOffdS, *tN = buf + kOffN, *tdv = buf + kOffdv, *tO = buf + kOffO;

      // Tokens of this wave.
      const X Oj = row_op<F32>(tO, kLuO, j, 0, lg);
      const W Nj = wide_col(tN, kTileN, kLuN, j0), vj = wide_col(tdv, kTileN, kLuN, j0);
      // dv out, and its product with N.
      {
        const uint32_t off = (uint32_t)j * v_row + (uint32_t)(32 * s + 4 * lg) * ES;
        const float ib = 1.f / strengths[j];
        float x[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          x[e] = O::value(vj, e);
          db += (O::value(Nj, e) * ib) * (x[e] * ib);
        }
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          if constexpr (F32)
            store_b128(dvr, off + 64u * u,
                       __builtin_bit_cast(u32x4, floatx4{x[4 * u], x[4 * u + 1], x[4 * u + 2], x[4 * u + 3]}));
          else
            store_b64(dvr, off + 32u * u,
                      make_uint2(pack_bf16x2(x[4 * u], x[4 * u + 1]), pack_bf16x2(x[4 * u + 2], x[4 * u + 3])));
        }
      }
      // Scores between tokens, columns of this wave.
#pragma unroll
      for (int t = 0; t < 4; ++t) {
        if (t <= wave) {
          const X Nt = col_op<F32>(tN, kLuN, 0, 16 * t, li, lg);
          Wt[t] = O::mma(Nt, Oj, Wt[t]);             // dO_j.N_i, rows i <= j
          Xb[t] = O::mma(Nt, O::head(vj), Xb[t]);    // dv_j.N_i
        }
        if (t >= wave) {
          Wn[t] = O::mma(row_op<F32>(tO, kLuO, 16 * t + li, 0, lg), Nj, Wn[t]);  // dO_i.N_j, rows i >= j
          Xa[t] = O::mma(wide_col(tdv, kTileN, kLuN, 16 * t), Nj, Xa[t]);       // dv_i.N_j
        }
      }
      // Products with the states, channels x tokens.
#pragma unroll
      for (int c = 0; c < NC; ++c) {
        const W Sc = wide_col(tS, kTileS, kLuK, 16 * c), dSc = wide_col(tdS, kTileS, kLuK, 16 * c);
        Q[c] = O::mma(Sc, Oj, Q[c]);
        Ka[c] = O::mma(dSc, Nj, Ka[c]);
        Kb[c] = O::mma(Sc, vj, Kb[c]);
        if ((c & 3) == wave)
#pragma unroll
          for (int e = 0; e < 8; ++e) ss += O::value(Sc, e) * O::value(dSc, e);
      }
      if (kBufs == 1 && n + 1 < total) {
        lds_barrier();
        stage(n + 1);
      }
    }

    // Decays between tokens: columns j of this lane.  What passes from j to
    // i > j (A): its sums over i, for token j, and over j, for tokens i.
    const double gj = pre[j];
    const float gamj = gam[j], etaj = eta[j];
    floatx4 Xs[4];
    float below = 0.f;
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      floatx4 qk = zero, kk = zero;
      if (t >= wave)
#pragma unroll
        for (int s = 0; s < DK / 32; ++s) {
          const X kj = row_op<F32>(tileK, kLuK, j, s, lg);
          qk = O::mma(row_op<F32>(tileQ, kLuK, 16 * t + li, s, lg), kj, qk);
          kk = O::mma(row_op<F32>(tileK, kLuK, 16 * t + li, s, lg), kj, kk);
        }
      floatx4 A = zero;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int i = 16 * t + 4 * lg + e;
        const double gi = pre[i];
        const float down = i >= j ? exp2f((float)(gi - gj)) : 0.f, up = i <= j ? exp2f((float)(gj - gi)) : 0.f;
        Wt[t][e] = i <= j ? a.scale * up * Wt[t][e] : 0.f;
        Wn[t][e] = i >= j && i < len ? a.scale * down * Wn[t][e] : 0.f;
        Xs[t][e] = i > j ? -down * Xa[t][e] : i < j ? -up * Xb[t][e] : 0.f;
        A[e] = i > j && i < len ? Wn[t][e] * qk[e] + Xs[t][e] * kk[e] : 0.f;
        below += A[e];
      }
      // Sums over the 16 columns of this wave.
#pragma unroll
      for (int e = 0; e < 4; ++e) {
#pragma unroll
        for (int m = 1; m < 16; m <<= 1) A[e] += __shfl_xor(A[e], m);
      }
      if (li == 0)
#pragma unroll
        for (int e = 0; e < 4; ++e) rows[wave][16 * t + 4 * lg + e] = A[e];
    }
    float in = 0.f, end = 0.f;
    X Xx[2], Wx[2], Wy[2];
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      Xx[s] = O::narrow(Xs[2 * s], Xs[2 * s + 1]);
      Wx[s] = O::narrow(Wn[2 * s], Wn[2 * s + 1]);
      Wy[s] = O::narrow(Wt[2 * s], Wt[2 * s + 1]);
    }
#pragma unroll
    for (int c = 0; c < NC; ++c) {
      floatx4 x = (a.scale * gamj) * Q[c], y = etaj * Ka[c] - gamj * Kb[c];
      // This lane's four channels of its token's q and k.
      const int sw = swizzle<F32>(j, kLuK);
      floatx4 qv, kv;
      if constexpr (F32) {
        const int at = (j << (kLuK + 4)) + (((4 * c + lg) ^ sw) << 4);
        qv = *reinterpret_cast<const floatx4*>(tileQ + at);
        kv = *reinterpret_cast<const floatx4*>(tileK + at);
      } else {
        const int at = (j << (kLuK + 4)) + (((2 * c + (lg >> 1)) ^ sw) << 4) + (lg & 1) * 8;
        const uint2 q2 = *reinterpret_cast<const uint2*>(tileQ + at), k2 = *reinterpret_cast<const uint2*>(tileK + at);
        qv = floatx4{bf16_lo(q2.x), bf16_hi(q2.x), bf16_lo(q2.y), bf16_hi(q2.y)};
        kv = floatx4{bf16_lo(k2.x), bf16_hi(k2.x), bf16_lo(k2.y), bf16_hi(k2.y)};
      }
#pragma unroll
      for (int e = 0; e < 4; ++e) in += qv[e] * x[e] - gamj * kv[e] * Kb[c][e], end += kv[e] * Ka[c][e];
#pragma unroll
      for (int s = 0; s < 2; ++s) {
        const X kt = col_op<F32>(tileK, kLuK, 32 * s, 16 * c, li, lg);
        const X qt = col_op<F32>(tileQ, kLuK, 32 * s, 16 * c, li, lg);
        x = O::mma(kt, Wy[s], x);
        y = O::mma(qt, Wx[s], y);
        y = O::mma(kt, Xx[s], y);
      }
      dq[c] += x;
      dk[c] += y;
    }
    // Sums over the lanes of a token (lg), then over the chunk.
    float past = below + etaj * end;
    in += __shfl_xor(in, 16), in += __shfl_xor(in, 32);
    past += __shfl_xor(past, 16), past += __shfl_xor(past, 32);
    db += __shfl_xor(db, 16), db += __shfl_xor(db, 32);
#pragma unroll
    for (int m = 1; m < 64; m <<= 1) ss += __shfl_xor(ss, m);
    if (lg == 0) {
      suffix[j] = j < len ? in : 0.f;
      prefix[j] = j < len ? past : 0.f;
      if (j < len) a.dbeta[(size_t)(ci.tok + j) * a.gate_tok + (size_t)h * a.gate_head] = db;
    }
    if (lane == 0) states[wave] = ss;
    lds_barrier();
    if (wave == 0) {
      // Token t = lane: sums of suffix from t on, and of prefix less rows before t.
      const float pass = prefix[lane] - ((rows[0][lane] + rows[1][lane]) + (rows[2][lane] + rows[3][lane]));
      float x = suffix[lane], y = pass;
#pragma unroll
      for (int d = 1; d < 64; d <<= 1) {
        const float down = __shfl_down(x, d), up = __shfl_up(y, d);
        if (lane + d < 64) x += down;
        if (lane >= d) y += up;
      }
      x += y - pass + gam[63] * ((states[0] + states[1]) + (states[2] + states[3]));
      if (lane < len) {
        const size_t at = (size_t)(ci.tok + lane) * a.gate_tok + (size_t)h * a.gate_head;
        // A decay of zero: nothing of the state before reaches the token.
        a.dg[at] = a.g[at] < kMinLogDecay ? 0.f : x;
      }
    }
  }

  const __amdgpu_buffer_rsrc_t dqr = make_rsrc((char*)a.dq + qk * ES, k_span);
  const __amdgpu_buffer_rsrc_t dkr = make_rsrc((char*)a.dk + qk * ES, k_span);
#pragma unroll
  for (int c = 0; c < NC; ++c) {
    const uint32_t off = (uint32_t)j * k_row + (uint32_t)(16 * c + 4 * lg) * ES;
    if constexpr (F32) {
      store_b128(dqr, off, __builtin_bit_cast(u32x4, dq[c]));
      store_b128(dkr, off, __builtin_bit_cast(u32x4, dk[c]));
    } else {
      store_b64(dqr, off, make_uint2(pack_bf16x2(dq[c][0], dq[c][1]), pack_bf16x2(dq[c][2], dq[c][3])));
      store_b64(dkr, off, make_uint2(pack_bf16x2(dk[c][0], dk[c][1]), pack_bf16x2(dk[c][2], dk[c][3])));
    }
  }
}

template <bool F32, int DK>
hipError_t reverse(bool map, const DeltaArgs& a, hipStream_t stream) {
  const unsigned items = (unsigned)a.max_segs * (unsigned)a.Hv, threads = 4u * a.d_v;
  if (map)
    delta_reverse_kernel<F32, DK, true><<<items, threads, 0, stream>>>(a);
  else
    delta_reverse_kernel<F32, DK, false><<<items, threads, 0, stream>>>(a);
  return hipGetLastError();
}

template <bool F32, int DK>
hipError_t grad(const DeltaArgs& a, hipStream_t stream) {
  delta_grad_kernel<F32, DK><<<(unsigned)a.max_chunks * (unsigned)a.Hk, kThreads, 0, stream>>>(a);
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
  if (a.max_chunks == 0) return hipSuccess;
  switch (d_k) {
    case 32: return f32 ? grad<true, 32>(a, stream) : grad<false, 32>(a, stream);
    case 64: return f32 ? grad<true, 64>(a, stream) : grad<false, 64>(a, stream);
    default: return f32 ? grad<true, 128>(a, stream) : grad<false, 128>(a, stream);
  }
}

}  // namespace vda
