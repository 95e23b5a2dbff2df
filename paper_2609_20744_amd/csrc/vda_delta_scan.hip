// Token-wise gated delta rule: the forward state scan over chunks
// (vda_delta.h), with the outputs, with what the gradient kernel reads, or as
// the affine maps of segments; and the join of those maps.
//
// One workgroup per segment and value head; a wave owns 16 NV value columns of
// the state, transposed (key channels x value columns), in registers, and
// nothing passes between waves: each product leaves its result with the rows
// that the next one contracts,
//     Z = K S^T -> X = beta (V - gam Z) -> N = T X -> S^T <- gam_63 S^T + K^T (eta N),
// so a step is three dependent products with no exchange through LDS.  The
// matrices that all waves share (k, q and v rows, T, P) come through LDS, the
// next chunk's copied by loads straight to LDS while this one's are used, one
// barrier a chunk.  O^T = S Q^T + N^T P^T takes the same registers as left
// operands, so a lane ends with consecutive channels of a token's output.
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

// Waves of a workgroup over `cols` state columns.
template <int NV>
constexpr int waves_of(int cols) {
  return (cols + 16 * NV - 1) / (16 * NV);
}

template <bool F32, int DK, int NV, int MODE>
__global__ __launch_bounds__(64 * waves_of<NV>(128)) void delta_scan_kernel(DeltaArgs a) {
  typedef Op<F32> O;
  typedef typename O::X X;
  typedef typename O::W W;
  constexpr int ES = F32 ? 4 : 2, KS = DK / 32, NC = DK / 16;
  constexpr int kLuK = __builtin_ctz(DK * ES / 16);
  constexpr int kBufs = F32 ? 1 : 2;
  constexpr int kTileK = kChunk * DK * ES;
  // Stage: k rows, T, gam and eta, v rows, then (outputs) q rows and P.
  constexpr int kOffT = kTileK, kOffVec = kOffT + kWideTri, kOffV = kOffVec + 1024,
                kOffQ = kOffV + kChunk * 128 * ES, kOffP = kOffQ + kTileK,
                kStage = MODE == kOutput ? kOffP + ChunkRecord::kPBytes[F32] : kOffQ;
  __shared__ __align__(16) char lds[kBufs * kStage];

  const int DV = a.d_v;
  unsigned id = blockIdx.x;
  bool matrix = false;  // this workgroup scans M's rows, not J's
  if constexpr (MODE == kMap) matrix = id & 1, id >>= 1;
  const int h = uniform(id % (unsigned)a.Hv);
  const int seg = uniform(id / (unsigned)a.Hv);
  const SegmentInfo si = segment_info(a, seg);
  if (si.chunks < 0) return;
  // The last segment's map is not needed, nor the first one's matrix.
  if (MODE == kMap && ((si.ends & 2) || (matrix && (si.ends & 1)))) return;

  const int tid = threadIdx.x, lane = tid & 63, li = lane & 15, lg = lane >> 4;
  const int wave = uniform(tid >> 6), waves = uniform(blockDim.x >> 6);
  const int cols = matrix ? DK : DV;
  const int v0 = wave * 16 * NV;
  const bool active = v0 < cols;
  const int luv = __builtin_ctz(DV * ES / 16);
  const size_t rec_size = ChunkRecord::bytes(F32, MODE == kKeep || (MODE == kMap && a.dout != nullptr));

  // The entering state.
  floatx4 S[NC][NV];
  const size_t mat = (size_t)DV * DK;
  const float* init = nullptr;
  if (!matrix) {
    if (si.ends & 1)
      init = a.S_in ? a.S_in + ((size_t)si.seq * a.Hv + h) * mat : nullptr;
    else if (MODE != kMap)
      init = a.segJ + ((size_t)seg * a.Hv + h) * mat;
  }
#pragma unroll
  for (int c = 0; c < NC; ++c)
#pragma unroll
    for (int n = 0; n < NV; ++n) {
      S[c][n] = floatx4{0.f, 0.f, 0.f, 0.f};
      const int col = v0 + 16 * n + li;
      if (matrix) {
#pragma unroll
        for (int e = 0; e < 4; ++e) S[c][n][e] = 16 * c + 4 * lg + e == col ? 1.f : 0.f;
      } else if (init != nullptr && active && v0 + 16 * n < cols) {
        S[c][n] = *reinterpret_cast<const floatx4*>(init + (size_t)col * DK + 16 * c + 4 * lg);
      }
    }

  const uint32_t k_row = (uint32_t)a.qk_tok * ES, v_row = (uint32_t)a.v_tok * ES;
  auto stage = [&](int c) {
    char* buf = lds + (kBufs == 2 && (c & 1) ? kStage : 0);
    const int chunk = si.chunk + c;
    const ChunkInfo ci = chunk_info(a, chunk);
    const char* rec = a.rec + ((size_t)chunk * a.Hv + h) * rec_size;
    const size_t qk = (size_t)ci.tok * a.qk_tok + (size_t)(h / a.group) * a.qk_head;
    const uint32_t k_span = (uint32_t)(ci.len - 1) * k_row + DK * ES;
    copy_rows<F32>(make_rsrc((const char*)a.k + qk * ES, k_span), buf, kLuK, kChunk, ci.len, k_row, wave,
                   waves, lane);
    copy_flat(rec + ChunkRecord::kT, buf + kOffT, kWideTri + 1024, wave, waves, lane);
    if (!matrix) {
      const size_t vo = (size_t)ci.tok * a.v_tok + (size_t)h * a.v_head;
      copy_rows<F32>(make_rsrc((const char*)a.v + vo * ES, (uint32_t)(ci.len - 1) * v_row + DV * ES),
                     buf + kOffV, luv, kChunk, ci.len, v_row, wave, waves, lane);
    }
    if constexpr (MODE == kOutput) {
      copy_rows<F32>(make_rsrc((const char*)a.q + qk * ES, k_span), buf + kOffQ, kLuK, kChunk, ci.len,
                     k_row, wave, waves, lane);
      copy_flat(rec + ChunkRecord::kP, buf + kOffP, ChunkRecord::kPBytes[F32], wave, waves, lane);
    }
  };

  const floatx4 zero = {0.f, 0.f, 0.f, 0.f};
  if (si.chunks > 0) stage(0);
  for (int c = 0; c < si.chunks; ++c) {
    copy_barrier();
    if (kBufs == 2 && c + 1 < si.chunks) stage(c + 1);
    const char* buf = lds + (kBufs == 2 && (c & 1) ? kStage : 0);
    if (active) {
      const float* gam = reinterpret_cast<const float*>(buf + kOffVec);
      const float *eta = gam + 64, *beta = gam + 128;
      const int chunk = si.chunk + c;

      W Sw[KS][NV];
#pragma unroll
      for (int s = 0; s < KS; ++s)
#pragma unroll
        for (int n = 0; n < NV; ++n) Sw[s][n] = O::wide(S[2 * s][n], S[2 * s + 1][n]);

      if constexpr (MODE == kKeep) {
        char* ks = a.keepS + ((size_t)chunk * a.Hv + h) * mat * 4;
#pragma unroll
        for (int cc = 0; cc < NC; ++cc)
#pragma unroll
          for (int n = 0; n < NV; ++n)
            if (v0 + 16 * n < cols)
              store_wide4<F32>(ks, (size_t)(v0 + 16 * n + li) * DK + 16 * cc + 4 * lg, mat, S[cc][n]);
      }

      // Z = K S^T, X = beta (V - gam Z).
      W Xw[2][NV];
#pragma unroll
      for (int s2 = 0; s2 < 2; ++s2) {
        floatx4 z[2][NV];
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          const int t = 2 * s2 + u;
#pragma unroll
          for (int n = 0; n < NV; ++n) z[u][n] = zero;
#pragma unroll
          for (int s = 0; s < KS; ++s) {
            const X kop = row_op<F32>(buf, kLuK, 16 * t + li, s, lg);
#pragma unroll
            for (int n = 0; n < NV; ++n) z[u][n] = O::mma(kop, Sw[s][n], z[u][n]);
          }
          const floatx4 gv = *reinterpret_cast<const floatx4*>(gam + 16 * t + 4 * lg);
          const floatx4 bv = *reinterpret_cast<const floatx4*>(beta + 16 * t + 4 * lg);
#pragma unroll
          for (int n = 0; n < NV; ++n) {
            floatx4 vv = zero;
            if (!matrix && v0 + 16 * n < cols)
              vv = result_rows<F32>(buf + kOffV, luv, 16 * t, v0 + 16 * n, li, lg);
            z[u][n] = bv * (vv - gv * z[u][n]);
          }
        }
#pragma unroll
        for (int n = 0; n < NV; ++n) Xw[s2][n] = O::wide(z[0][n], z[1][n]);
      }

      // N = T X.
      floatx4 N[4][NV];
#pragma unroll
      for (int t = 0; t < 4; ++t)
#pragma unroll
        for (int n = 0; n < NV; ++n) N[t][n] = zero;
#pragma unroll
      for (int t = 0; t < 4; ++t)
#pragma unroll
        for (int s = 0; s <= t / 2; ++s) {
          const W T = tile_w<F32>(buf + kOffT, tri_tile(t, s), lane);
#pragma unroll
          for (int n = 0; n < NV; ++n) N[t][n] = O::mma(T, Xw[s][n], N[t][n]);
        }

      if constexpr (MODE == kKeep) {
        char* kn = a.keepN + ((size_t)chunk * a.Hv + h) * DV * kChunk * 4;
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
          for (int n = 0; n < NV; ++n)
            if (v0 + 16 * n < cols)
              store_wide4<F32>(kn, (size_t)(v0 + 16 * n + li) * kChunk + 16 * t + 4 * lg,
                               (size_t)DV * kChunk, N[t][n]);
      }

      if constexpr (MODE == kOutput) {
        X Nx[2][NV];
#pragma unroll
        for (int s = 0; s < 2; ++s)
#pragma unroll
          for (int n = 0; n < NV; ++n) Nx[s][n] = O::narrow(N[2 * s][n], N[2 * s + 1][n]);
        const ChunkInfo ci = chunk_info(a, chunk);
        const size_t vo = (size_t)ci.tok * a.v_tok + (size_t)h * a.v_head;
        const __amdgpu_buffer_rsrc_t orsrc =
            make_rsrc((char*)a.out + vo * ES, (uint32_t)(ci.len - 1) * v_row + DV * ES);
#pragma unroll
        for (int t = 0; t < 4; ++t) {
          floatx4 o[NV];
#pragma unroll
          for (int n = 0; n < NV; ++n) o[n] = zero;
#pragma unroll
          for (int s = 0; s < KS; ++s) {
            const X qop = row_op<F32>(buf + kOffQ, kLuK, 16 * t + li, s, lg);
#pragma unroll
            for (int n = 0; n < NV; ++n) o[n] = O::mma(O::head(Sw[s][n]), qop, o[n]);
          }
          const float gq = a.scale * gam[16 * t + li];
#pragma unroll
          for (int n = 0; n < NV; ++n) o[n] *= gq;
#pragma unroll
          for (int s = 0; s <= t / 2; ++s) {
            const X P = tile_x<F32>(buf + kOffP, tri_tile(t, s), lane);
#pragma unroll
            for (int n = 0; n < NV; ++n) o[n] = O::mma(Nx[s][n], P, o[n]);
          }
#pragma unroll
          for (int n = 0; n < NV; ++n) {
            if (v0 + 16 * n >= cols) continue;
            const uint32_t off = (uint32_t)(16 * t + li) * v_row + (uint32_t)(v0 + 16 * n + 4 * lg) * ES;
            if constexpr (F32)
              store_b128(orsrc, off, __builtin_bit_cast(u32x4, o[n]));
            else
              store_b64(orsrc, off, make_uint2(pack_bf16x2(o[n][0], o[n][1]), pack_bf16x2(o[n][2], o[n][3])));
          }
        }
      }

      // S <- gam_63 S + N^T diag(eta) K.
      W Nw[2][NV];
#pragma unroll
      for (int s = 0; s < 2; ++s) {
        const floatx4 e0 = *reinterpret_cast<const floatx4*>(eta + 32 * s + 4 * lg);
        const floatx4 e1 = *reinterpret_cast<const floatx4*>(eta + 32 * s + 16 + 4 * lg);
#pragma unroll
        for (int n = 0; n < NV; ++n) Nw[s][n] = O::wide(N[2 * s][n] * e0, N[2 * s + 1][n] * e1);
      }
      const float gl = gam[63];
#pragma unroll
      for (int cc = 0; cc < NC; ++cc) {
#pragma unroll
        for (int n = 0; n < NV; ++n) S[cc][n] *= gl;
#pragma unroll
        for (int s = 0; s < 2; ++s) {
          const X kt = col_op<F32>(buf, kLuK, 32 * s, 16 * cc, li, lg);
#pragma unroll
          for (int n = 0; n < NV; ++n) S[cc][n] = O::mma(kt, Nw[s][n], S[cc][n]);
        }
      }
    }
    if (kBufs == 1 && c + 1 < si.chunks) {
      lds_barrier();
      stage(c + 1);
    }
  }

  if (!active) return;
#pragma unroll
  for (int n = 0; n < NV; ++n) {
    if (v0 + 16 * n >= cols) continue;
    const int col = v0 + 16 * n + li;
#pragma unroll
    for (int c = 0; c < NC; ++c) {
      const size_t at = (size_t)col * DK + 16 * c + 4 * lg;
      if constexpr (MODE == kMap) {
        if (matrix) {
          const size_t base = ((size_t)seg * a.Hv + h) * DK * DK;
          *reinterpret_cast<floatx4*>(a.segM + base + at) = S[c][n];
#pragma unroll
          for (int e = 0; e < 4; ++e) a.segMt[base + (size_t)(16 * c + 4 * lg + e) * DK + col] = S[c][n][e];
        } else {
          *reinterpret_cast<floatx4*>(a.segJ + ((size_t)seg * a.Hv + h) * mat + at) = S[c][n];
        }
      } else if ((si.ends & 2) && a.S_out != nullptr) {
        *reinterpret_cast<floatx4*>(a.S_out + ((size_t)si.seq * a.Hv + h) * mat + at) = S[c][n];
      }
    }
  }
}

// The join: x <- x M_s + J_s over the segments of a sequence in order (or, in
// reverse, x <- x M_s^T + J_s from the last), the state entering each segment
// written over its J.  The recurrence of a state's rows is independent of the
// others': one workgroup of four waves per sequence, head and 16 rows; a wave makes
// d_k / 4 columns of the product (transposed, the matrix as left operand),
// which it passes to the others as operands through LDS.  fp32 matrix cores:
// a step's 16 x d_k x d_k product is small beside the chunks it stands for.
template <int DK>
__global__ __launch_bounds__(kThreads) void delta_join_kernel(DeltaArgs a, bool reverse) {
  typedef Op<true> O;
  constexpr int KS = DK / 32, NC = DK / 16, WT = (NC + 3) / 4;
  constexpr int kRow = DK + 4;
  __shared__ __align__(16) float x[2][16 * kRow];
  const int blocks = a.d_v / 16;
  const int rb = blockIdx.x % blocks;
  const int h = (blockIdx.x / blocks) % a.Hv;
  const int seq = blockIdx.x / (blocks * a.Hv);
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
  const float* M = reverse ? a.segM : a.segMt;
  const size_t mat = (size_t)a.d_v * DK;
  const int row = rb * 16 + li;
  auto index = [&](int i) { return (size_t)(reverse ? first + count - 1 - i : first + i) * a.Hv + h; };

  // After segment 0 the state is its own J (scanned from the sequence's state).
  floatx4 y[WT];
#pragma unroll
  for (int w = 0; w < WT; ++w) {
    const int c = wave * WT + w;
    if (c < NC) y[w] = *reinterpret_cast<const floatx4*>(J + index(0) * mat + (size_t)row * DK + 16 * c + 4 * lg);
  }
  for (int i = 1; i < count; ++i) {
    floatx4 add[WT];
    const bool more = i + 1 < count;
    float* Ji = J + index(i) * mat + (size_t)row * DK;
    float* buf = x[i & 1];
#pragma unroll
    for (int w = 0; w < WT; ++w) {
      const int c = wave * WT + w;
      if (c >= NC) continue;
      if (more) add[w] = *reinterpret_cast<const floatx4*>(Ji + 16 * c + 4 * lg);
      *reinterpret_cast<floatx4*>(Ji + 16 * c + 4 * lg) = y[w];
      *reinterpret_cast<floatx4*>(buf + li * kRow + 16 * c + 4 * lg) = y[w];
    }
    if (!more) return;
    lds_barrier();
    const float* Mi = M + index(i) * DK * DK;
#pragma unroll
    for (int w = 0; w < WT; ++w) {
      const int c = wave * WT + w;
      if (c >= NC) continue;
      y[w] = add[w];
#pragma unroll
      for (int s = 0; s < KS; ++s) {
        const float* xr = buf + li * kRow + 32 * s + 4 * lg;
        const float* mr = Mi + (size_t)(16 * c + li) * DK + 32 * s + 4 * lg;
        const O::X xo = O::narrow(*reinterpret_cast<const floatx4*>(xr), *reinterpret_cast<const floatx4*>(xr + 16));
        const O::X mo = O::narrow(*reinterpret_cast<const floatx4*>(mr), *reinterpret_cast<const floatx4*>(mr + 16));
        y[w] = O::mma(mo, xo, y[w]);
      }
    }
  }
}

template <bool F32, int DK, int NV>
hipError_t run(int what, const DeltaArgs& a, hipStream_t stream) {
  const unsigned items = (unsigned)a.max_segs * (unsigned)a.Hv;
  const int waves = waves_of<NV>(a.d_v);
  if (what == kMap) {
    const int w = waves_of<NV>(a.d_v > DK ? a.d_v : DK);
    delta_scan_kernel<F32, DK, NV, kMap><<<items * 2, 64 * w, 0, stream>>>(a);
  } else if (what == kOutput) {
    delta_scan_kernel<F32, DK, NV, kOutput><<<items, 64 * waves, 0, stream>>>(a);
  } else {
    delta_scan_kernel<F32, DK, NV, kKeep><<<items, 64 * waves, 0, stream>>>(a);
  }
  return hipGetLastError();
}

}  // namespace

hipError_t launch_delta_scan(bool f32, int d_k, int what, const DeltaArgs& a, hipStream_t stream) {
  switch (d_k) {
    case 32: return f32 ? run<true, 32, 1>(what, a, stream) : run<false, 32, 1>(what, a, stream);
    case 64: return f32 ? run<true, 64, 1>(what, a, stream) : run<false, 64, 1>(what, a, stream);
    default: return f32 ? run<true, 128, 1>(what, a, stream) : run<false, 128, 1>(what, a, stream);
  }
}

hipError_t launch_delta_join(int d_k, bool reverse, const DeltaArgs& a, hipStream_t stream) {
  const unsigned grid = (unsigned)a.n_seqs * (unsigned)a.Hv * (unsigned)(a.d_v / 16);
  switch (d_k) {
    case 32: delta_join_kernel<32><<<grid, kThreads, 0, stream>>>(a, reverse); break;
    case 64: delta_join_kernel<64><<<grid, kThreads, 0, stream>>>(a, reverse); break;
    default: delta_join_kernel<128><<<grid, kThreads, 0, stream>>>(a, reverse); break;
  }
  return hipGetLastError();
}

}  // namespace vda
