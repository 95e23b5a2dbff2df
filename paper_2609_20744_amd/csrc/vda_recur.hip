// The channel-wise gated recurrence, its gradients and its recurrent form (vda.h,
// vda_recur_*): h_t = a_t h_{t-1} + u_t for each channel of each sequence.
//
// Sequences are taken in tiles of 128 tokens by 128 channels.  A workgroup has 16
// runs of eight consecutive tokens, a lane eight channels of one run: it makes the
// run's decay A = prod a and what the run adds from zero, H, and the 16 runs are
// joined through LDS.  A tile acts on the state that enters it as h -> A h + H, so
// sequences longer than a tile take three kernels: what every tile does (reduce),
// the states that enter them (carry), the outputs (apply).  The gradient runs the
// other way: with E_t = a_t D_t, D_t = dout_t + E_{t+1}, a tile takes the E that
// enters at its end to A E + G, with the same A and G = sum_t (a_1 .. a_t) dout_t, so one
// reduction makes all three; h is made again from x and the gates, nothing is kept.
// A place behind a sequence's end has a = 1, u = 0 and dout = 0.
//
// Bytes bound it: each pass streams its inputs once.
#include "vda_recur.h"
#include "../../include/vda.h"

namespace vda {
namespace {

template <bool F32>
__device__ __forceinline__ void load8(const void* p, size_t at, float (&x)[8]) {
  if constexpr (F32) {
    const floatx4* f = reinterpret_cast<const floatx4*>((const float*)p + at);
    const floatx4 a = f[0], b = f[1];
#pragma unroll
    for (int e = 0; e < 4; ++e) x[e] = a[e], x[4 + e] = b[e];
  } else {
    const uint4 w = *reinterpret_cast<const uint4*>((const uint16_t*)p + at);
    const uint32_t v[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
    for (int e = 0; e < 4; ++e) x[2 * e] = bf16_lo(v[e]), x[2 * e + 1] = bf16_hi(v[e]);
  }
}
template <bool F32>
__device__ __forceinline__ void store8(void* p, size_t at, const float (&x)[8]) {
  if constexpr (F32) {
    floatx4* f = reinterpret_cast<floatx4*>((float*)p + at);
    f[0] = floatx4{x[0], x[1], x[2], x[3]};
    f[1] = floatx4{x[4], x[5], x[6], x[7]};
  } else {
    *reinterpret_cast<uint4*>((uint16_t*)p + at) = make_uint4(pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3]),
                                                              pack_bf16x2(x[4], x[5]), pack_bf16x2(x[6], x[7]));
  }
}

// A token's gate.  a near 1 is 1 less an exact rest, so that it has its own
// rounding only: a long memory's length is 1 / (1 - a).  b = 1 - a.
template <int GATE>
__device__ __forceinline__ void gate_of(float g, float& a, float& b) {
  if constexpr (GATE == VDA_GATE_LOG) {
    const float e = __builtin_amdgcn_exp2f(g * 1.4426950408889634f);
    const float near = fmaf(g * g, fmaf(g, fmaf(g, fmaf(g, 1.f / 120.f, 1.f / 24.f), 1.f / 6.f), 0.5f), g);
    a = fabsf(g) < 0.0625f ? 1.f + near : e;
    b = 0.f;  // not used
  } else {
    const float z = __builtin_amdgcn_fmed3f(g, -80.f, 80.f);
    const float e = __builtin_amdgcn_exp2f(z * -1.4426950408889634f);
    const float r = __builtin_amdgcn_rcpf(1.f + e);
    b = e * r;
    a = e < 1.f ? 1.f - b : r;
    // fmed3 gives -80 for a NaN.
    if (g != g) a = b = g;
  }
}
template <int GATE>
__device__ __forceinline__ float weight_of(float a, float b) {
  return GATE == VDA_GATE_LOG ? 1.f : GATE == VDA_GATE_LOGIT ? b : __builtin_amdgcn_sqrtf(b * (1.f + a));
}

// A sequence and a tile of it.
struct RecurTile {
  int seq, first, len, tile, last;  // first token and tokens of the sequence; the tile's index and that of its last
};
__device__ __forceinline__ bool tile_of(const RecurArgs& a, int t, RecurTile& r) {
  if (a.cu == nullptr) {
    const int each = (a.L + kRecurTile - 1) / kRecurTile;
    r.seq = uniform(t / each), r.tile = t - r.seq * each;
    r.first = r.seq * a.L, r.len = a.L;
  } else {
    // Sequence i has the places from first_i / tile + i on.
    const int lane = threadIdx.x & 63;
    int before = 0;
    for (int b = 0; b < a.n; b += 64) {
      const int i = b + lane, c = a.cu[i < a.n ? i : 0];
      before += __popcll(__ballot(i < a.n && (c < 0 ? 0 : c > a.T ? a.T : c) / kRecurTile + i <= t));
    }
    r.seq = uniform(before) - 1;
    if (r.seq < 0) return false;
    const int c = uniform(a.cu[r.seq]), d = uniform(a.cu[r.seq + 1]);
    r.first = c < 0 ? 0 : c > a.T ? a.T : c;
    const int end = d < 0 ? 0 : d > a.T ? a.T : d;
    r.len = end > r.first ? end - r.first : 0;
    r.tile = t - (r.first / kRecurTile + r.seq);
    if (r.tile < 0) return false;
  }
  r.last = r.len > 0 ? (r.len - 1) / kRecurTile : 0;
  return r.tile <= r.last;
}

// A lane's run: its channels and where its tokens are.
struct Run {
  bool real;     // the lane has channels
  int chan, run, left;  // tokens of the run that there are
  size_t tok;    // the first one's row
};
__device__ __forceinline__ Run run_of(const RecurArgs& a, const RecurTile& r) {
  Run w;
  w.chan = (blockIdx.y * 16 + (threadIdx.x & 15)) * 8;
  w.real = w.chan < a.C;
  if (!w.real) w.chan = 0;
  w.run = threadIdx.x >> 4;
  const int p = r.tile * kRecurTile + w.run * kRecurRun;
  w.left = r.len - p;
  w.tok = a.reverse ? (size_t)r.first + (r.len - 1 - p) : (size_t)r.first + p;  // read only where left > 0
  return w;
}
// Row of the run's i-th token (of its last one behind its end).
__device__ __forceinline__ size_t row_of(const RecurArgs& a, const Run& w, int i) {
  const int at = i < w.left ? i : w.left - 1;
  return a.reverse ? w.tok - at : w.tok + at;
}

__device__ __forceinline__ void clear(float (&x)[kRecurRun][8]) {
#pragma unroll
  for (int i = 0; i < kRecurRun; ++i)
#pragma unroll
    for (int e = 0; e < 8; ++e) x[i][e] = 0.f;
}

template <bool F32>
__device__ __forceinline__ void load_dout(const RecurArgs& a, const Run& w, float (&y)[kRecurRun][8]) {
  if (w.left <= 0) return clear(y);
#pragma unroll
  for (int i = 0; i < kRecurRun; ++i) load8<F32>(a.dout, row_of(a, w, i) * a.C + w.chan, y[i]);
}

template <bool F32, int GATE>
__device__ __forceinline__ void load_run(const RecurArgs& a, const Run& w, float (&x)[kRecurRun][8], float (&g)[kRecurRun][8]) {
  if (w.left <= 0) {
    clear(x), clear(g);
    return;
  }
#pragma unroll
  for (int i = 0; i < kRecurRun; ++i) {
    const size_t row = row_of(a, w, i);
    load8<F32>(a.x, row * a.xs + w.chan, x[i]);
    load8<F32 || GATE == VDA_GATE_LOG>(a.g, row * a.gs + w.chan, g[i]);
  }
}

// The gates of a run in place: x becomes u, g becomes a.
template <int GATE>
__device__ __forceinline__ void make_run(const Run& w, float (&x)[kRecurRun][8], float (&g)[kRecurRun][8]) {
#pragma unroll
  for (int i = 0; i < kRecurRun; ++i)
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      float al, b;
      gate_of<GATE>(g[i][e], al, b);
      const bool is = i < w.left;
      x[i][e] = is ? weight_of<GATE>(al, b) * x[i][e] : 0.f;
      g[i][e] = is ? al : 1.f;
    }
}

template <bool F32, int GATE, bool BACKWARD>
__global__ __launch_bounds__(kThreads) void recur_reduce_kernel(RecurArgs a) {
  __shared__ __align__(16) float sA[kRecurRuns][kRecurChans], sH[kRecurRuns][kRecurChans];
  __shared__ __align__(16) float sG[BACKWARD ? kRecurRuns : 1][kRecurChans];
  RecurTile r;
  if (!tile_of(a, blockIdx.x, r)) return;
  if (r.len <= kRecurTile) return;  // nothing enters its one tile from another
  const Run w = run_of(a, r);
  float x[kRecurRun][8], g[kRecurRun][8], y[kRecurRun][8];
  load_run<F32, GATE>(a, w, x, g);
  if constexpr (BACKWARD) load_dout<F32>(a, w, y);
  make_run<GATE>(w, x, g);
  const int c = (threadIdx.x & 15) * 8;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    float A = 1.f, H = 0.f, G = 0.f;
#pragma unroll
    for (int i = 0; i < kRecurRun; ++i) {
      H = fmaf(g[i][e], H, x[i][e]);
      A *= g[i][e];
      if constexpr (BACKWARD) G = i < w.left ? fmaf(A, y[i][e], G) : G;
    }
    sA[w.run][c + e] = A, sH[w.run][c + e] = H;
    if constexpr (BACKWARD) sG[w.run][c + e] = G;
  }
  __syncthreads();
  const int at = threadIdx.x, chan = blockIdx.y * kRecurChans + at;
  if (at >= kRecurChans || chan >= a.C) return;
  float A = 1.f, H = 0.f, G = 0.f;
#pragma unroll
  for (int i = 0; i < kRecurRuns; ++i) {
    if constexpr (BACKWARD) G = fmaf(A, sG[i][at], G);
    H = fmaf(sA[i][at], H, sH[i][at]);
    A *= sA[i][at];
  }
  const size_t to = (size_t)blockIdx.x * a.C + chan;
  a.A[to] = A, a.H[to] = H;
  if constexpr (BACKWARD) a.G[to] = G;
}

// What enters each tile of a sequence: a lane has a channel, a wave a range of the
// tiles.  H becomes the state that enters a tile, G the E that enters at its end.
constexpr int kCarryWaves = 16;
template <bool BACKWARD>
__global__ __launch_bounds__(64 * kCarryWaves) void recur_carry_kernel(RecurArgs a) {
  __shared__ float sA[kCarryWaves][64], sH[kCarryWaves][64], sG[kCarryWaves][64];
  const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6);
  const int seq = blockIdx.x;
  int first, len;
  if (a.cu == nullptr) {
    first = 0, len = a.L;
  } else {
    const int c = uniform(a.cu[seq]), d = uniform(a.cu[seq + 1]);
    first = c < 0 ? 0 : c > a.T ? a.T : c;
    const int end = d < 0 ? 0 : d > a.T ? a.T : d;
    len = end > first ? end - first : 0;
  }
  if (len <= kRecurTile) return;
  const int tiles = (len + kRecurTile - 1) / kRecurTile;
  const int place = a.cu == nullptr ? seq * tiles : first / kRecurTile + seq;
  if (place + tiles > a.tiles) return;  // offsets out of order only
  const int per = (tiles + kCarryWaves - 1) / kCarryWaves;
  const int from = wave * per < tiles ? wave * per : tiles, to = from + per < tiles ? from + per : tiles;
  const int chan = blockIdx.y * 64 + lane;
  const bool real = chan < a.C;
  const size_t base = (size_t)place * a.C + (real ? chan : 0);
  float A = 1.f, H = 0.f, G = 0.f;
#pragma unroll 8
  for (int t = from; t < to; ++t) {
    const size_t at = base + (size_t)t * a.C;
    const float ta = a.A[at], th = a.H[at];
    if constexpr (BACKWARD) G = fmaf(A, a.G[at], G);
    H = fmaf(ta, H, th);
    A *= ta;
  }
  sA[wave][lane] = A, sH[wave][lane] = H, sG[wave][lane] = G;
  __syncthreads();
  const size_t st = (size_t)seq * a.C + chan;
  float h = real && a.S_in != nullptr ? a.S_in[st] : 0.f;
  for (int w = 0; w < wave; ++w) h = fmaf(sA[w][lane], h, sH[w][lane]);
  float e = 0.f;
  if constexpr (BACKWARD) {
    e = real && a.dS_out != nullptr ? a.dS_out[st] : 0.f;
    for (int w = kCarryWaves - 1; w > wave; --w) e = fmaf(sA[w][lane], e, sG[w][lane]);
  }
  if (!real) return;
#pragma unroll 8
  for (int t = from; t < to; ++t) {
    const size_t at = base + (size_t)t * a.C;
    const float next = fmaf(a.A[at], h, a.H[at]);
    a.H[at] = h;
    h = next;
  }
  if constexpr (BACKWARD) {
#pragma unroll 8
    for (int t = to - 1; t >= from; --t) {
      const size_t at = base + (size_t)t * a.C;
      const float next = fmaf(a.A[at], e, a.G[at]);
      a.G[at] = e;
      e = next;
    }
  }
}

// Eight values of a [.., C] fp32 array, or zeros.
__device__ __forceinline__ void entering(const float* p, size_t at, bool is, float (&x)[8]) {
#pragma unroll
  for (int e = 0; e < 8; ++e) x[e] = 0.f;
  if (is && p != nullptr) load8<true>(p, at, x);
}

template <bool F32, int GATE>
__global__ __launch_bounds__(kThreads) void recur_apply_kernel(RecurArgs a) {
  __shared__ __align__(16) float sA[kRecurRuns][kRecurChans], sH[kRecurRuns][kRecurChans];
  RecurTile r;
  if (!tile_of(a, blockIdx.x, r)) return;
  const Run w = run_of(a, r);
  const bool carried = a.carried && r.len > kRecurTile;
  float x[kRecurRun][8], g[kRecurRun][8], h[8];
  load_run<F32, GATE>(a, w, x, g);
  entering(carried ? a.H : a.S_in, (carried ? (size_t)blockIdx.x : (size_t)r.seq) * a.C + w.chan, w.real, h);
  make_run<GATE>(w, x, g);
  const int c = (threadIdx.x & 15) * 8;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    float A = 1.f, H = 0.f;
#pragma unroll
    for (int i = 0; i < kRecurRun; ++i) H = fmaf(g[i][e], H, x[i][e]), A *= g[i][e];
    sA[w.run][c + e] = A, sH[w.run][c + e] = H;
  }
  __syncthreads();
  for (int i = 0; i < w.run; ++i)
#pragma unroll
    for (int e = 0; e < 8; ++e) h[e] = fmaf(sA[i][c + e], h[e], sH[i][c + e]);
  if (!w.real) return;
#pragma unroll
  for (int i = 0; i < kRecurRun; ++i) {
#pragma unroll
    for (int e = 0; e < 8; ++e) h[e] = fmaf(g[i][e], h[e], x[i][e]);
    if (i < w.left) store8<F32>(a.out, row_of(a, w, i) * a.C + w.chan, h);
  }
  if (a.S_out != nullptr && r.tile == r.last && w.run == kRecurRuns - 1) store8<true>(a.S_out, (size_t)r.seq * a.C + w.chan, h);
}

template <bool F32, int GATE>
__global__ __launch_bounds__(kThreads) void recur_grad_kernel(RecurArgs a) {
  __shared__ __align__(16) float sA[kRecurRuns][kRecurChans], sH[kRecurRuns][kRecurChans], sG[kRecurRuns][kRecurChans];
  RecurTile r;
  if (!tile_of(a, blockIdx.x, r)) return;
  const Run w = run_of(a, r);
  const bool carried = a.carried && r.len > kRecurTile;
  const size_t at = (carried ? (size_t)blockIdx.x : (size_t)r.seq) * a.C + w.chan;
  float x[kRecurRun][8], g[kRecurRun][8], y[kRecurRun][8], h[8], D[8];
  load_run<F32, GATE>(a, w, x, g);
  load_dout<F32>(a, w, y);
  entering(carried ? a.H : a.S_in, at, w.real, h);
  entering(carried ? a.G : a.dS_out, at, w.real, D);
  const int c = (threadIdx.x & 15) * 8;
  // x stays the input; a and the weight are made again where they are used.
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    float A = 1.f, H = 0.f, G = 0.f;
#pragma unroll
    for (int i = 0; i < kRecurRun; ++i) {
      if (i >= w.left) {
        x[i][e] = 0.f, g[i][e] = GATE == VDA_GATE_LOG ? 0.f : INFINITY, y[i][e] = 0.f;
      }
      float al, b;
      gate_of<GATE>(g[i][e], al, b);
      if (i >= w.left) al = 1.f;
      H = fmaf(al, H, weight_of<GATE>(al, b) * x[i][e]);
      A *= al;
      G = fmaf(A, y[i][e], G);
    }
    sA[w.run][c + e] = A, sH[w.run][c + e] = H, sG[w.run][c + e] = G;
  }
  __syncthreads();
  for (int i = 0; i < w.run; ++i)
#pragma unroll
    for (int e = 0; e < 8; ++e) h[e] = fmaf(sA[i][c + e], h[e], sH[i][c + e]);
  for (int i = kRecurRuns - 1; i > w.run; --i)
#pragma unroll
    for (int e = 0; e < 8; ++e) D[e] = fmaf(sA[i][c + e], D[e], sG[i][c + e]);
  if (!w.real) return;
  // Forward over the states, then back: y becomes dx, and x the gate's gradient.
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    float before[kRecurRun], s = h[e], E = D[e];
#pragma unroll
    for (int i = 0; i < kRecurRun; ++i) {
      float al, b;
      gate_of<GATE>(g[i][e], al, b);
      before[i] = s;
      s = fmaf(al, s, weight_of<GATE>(al, b) * x[i][e]);
    }
#pragma unroll
    for (int i = kRecurRun - 1; i >= 0; --i) {
      float al, b;
      gate_of<GATE>(g[i][e], al, b);
      if (i >= w.left) al = 1.f;
      const float wt = weight_of<GATE>(al, b), d = y[i][e] + E;
      if constexpr (GATE == VDA_GATE_LOG)
        x[i][e] = d * al * before[i];
      else if constexpr (GATE == VDA_GATE_LOGIT)
        x[i][e] = d * al * b * (before[i] - x[i][e]);
      else
        x[i][e] = d * (al * b * before[i] - al * al * __builtin_amdgcn_sqrtf(b * __builtin_amdgcn_rcpf(1.f + al)) * x[i][e]);
      y[i][e] = d * wt;
      E = al * d;
    }
    D[e] = E;
  }
#pragma unroll
  for (int i = 0; i < kRecurRun; ++i)
    if (i < w.left) {
      const size_t row = row_of(a, w, i);
      store8<F32>(a.dx, row * a.dxs + w.chan, y[i]);
      store8<F32 || GATE == VDA_GATE_LOG>(a.dg, row * a.dgs + w.chan, x[i]);
    }
  if (a.dS_in != nullptr && r.tile == 0 && w.run == 0) store8<true>(a.dS_in, (size_t)r.seq * a.C + w.chan, D);
}

__device__ __forceinline__ floatx4 load4(const float* p) { return *reinterpret_cast<const floatx4*>(p); }
__device__ __forceinline__ floatx4 load4(const uint16_t* p) {
  const uint2 w = *reinterpret_cast<const uint2*>(p);
  return floatx4{bf16_lo(w.x), bf16_hi(w.x), bf16_lo(w.y), bf16_hi(w.y)};
}

// A lane has four channels of a sequence.
template <bool F32, int GATE>
__global__ __launch_bounds__(kThreads) void recur_step_kernel(RecurStepArgs a) {
  const unsigned per = (unsigned)a.C / 4;
  const size_t id = (size_t)blockIdx.x * kThreads + threadIdx.x;
  const size_t i = id / per;
  const int chan = (int)(id - i * per) * 4;
  if (i >= (size_t)a.n) return;
  const int slot = a.slots != nullptr ? a.slots[i] : (int)i;
  if (slot < 0 || slot >= a.n_slots) return;  // a row of padding
  float* S = a.state + (size_t)slot * a.C + chan;
  floatx4 h = load4(S);
  for (int t = 0; t < a.tokens; ++t) {
    const size_t at = (i * a.tokens + t) * a.C + chan;
    floatx4 x, g;
    if constexpr (F32)
      x = load4((const float*)a.x + at);
    else
      x = load4((const uint16_t*)a.x + at);
    if constexpr (F32 || GATE == VDA_GATE_LOG)
      g = load4((const float*)a.g + at);
    else
      g = load4((const uint16_t*)a.g + at);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      float al, b;
      gate_of<GATE>(g[e], al, b);
      h[e] = fmaf(al, h[e], weight_of<GATE>(al, b) * x[e]);
    }
    if constexpr (F32)
      *reinterpret_cast<floatx4*>((float*)a.out + at) = h;
    else
      *reinterpret_cast<uint2*>((uint16_t*)a.out + at) = make_uint2(pack_bf16x2(h[0], h[1]), pack_bf16x2(h[2], h[3]));
  }
  *reinterpret_cast<floatx4*>(S) = h;
}

dim3 grid_of(const RecurArgs& a) { return dim3(a.tiles, (a.C + kRecurChans - 1) / kRecurChans); }

template <bool F32, int GATE>
hipError_t reduce(bool backward, const RecurArgs& a, hipStream_t stream) {
  backward ? recur_reduce_kernel<F32, GATE, true><<<grid_of(a), kThreads, 0, stream>>>(a)
           : recur_reduce_kernel<F32, GATE, false><<<grid_of(a), kThreads, 0, stream>>>(a);
  return hipGetLastError();
}
template <bool F32, int GATE>
hipError_t apply(bool backward, const RecurArgs& a, hipStream_t stream) {
  backward ? recur_grad_kernel<F32, GATE><<<grid_of(a), kThreads, 0, stream>>>(a)
           : recur_apply_kernel<F32, GATE><<<grid_of(a), kThreads, 0, stream>>>(a);
  return hipGetLastError();
}
template <bool F32, int GATE>
hipError_t step(const RecurStepArgs& a, hipStream_t stream) {
  const unsigned grid = (unsigned)(((size_t)a.n * (a.C / 4) + kThreads - 1) / kThreads);
  recur_step_kernel<F32, GATE><<<grid, kThreads, 0, stream>>>(a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_recur_reduce(bool f32, bool backward, const RecurArgs& a, hipStream_t stream) {
  switch (a.gate) {
    case VDA_GATE_LOG: return f32 ? reduce<true, VDA_GATE_LOG>(backward, a, stream) : reduce<false, VDA_GATE_LOG>(backward, a, stream);
    case VDA_GATE_LOGIT:
      return f32 ? reduce<true, VDA_GATE_LOGIT>(backward, a, stream) : reduce<false, VDA_GATE_LOGIT>(backward, a, stream);
    default: return f32 ? reduce<true, VDA_GATE_NORM>(backward, a, stream) : reduce<false, VDA_GATE_NORM>(backward, a, stream);
  }
}

hipError_t launch_recur_apply(bool f32, bool backward, const RecurArgs& a, hipStream_t stream) {
  switch (a.gate) {
    case VDA_GATE_LOG: return f32 ? apply<true, VDA_GATE_LOG>(backward, a, stream) : apply<false, VDA_GATE_LOG>(backward, a, stream);
    case VDA_GATE_LOGIT:
      return f32 ? apply<true, VDA_GATE_LOGIT>(backward, a, stream) : apply<false, VDA_GATE_LOGIT>(backward, a, stream);
    default: return f32 ? apply<true, VDA_GATE_NORM>(backward, a, stream) : apply<false, VDA_GATE_NORM>(backward, a, stream);
  }
}

hipError_t launch_recur_carry(bool backward, const RecurArgs& a, hipStream_t stream) {
  const dim3 grid(a.n, (a.C + 63) / 64);
  backward ? recur_carry_kernel<true><<<grid, 64 * kCarryWaves, 0, stream>>>(a)
           : recur_carry_kernel<false><<<grid, 64 * kCarryWaves, 0, stream>>>(a);
  return hipGetLastError();
}

hipError_t launch_recur_step(bool f32, const RecurStepArgs& a, hipStream_t stream) {
  switch (a.gate) {
    case VDA_GATE_LOG: return f32 ? step<true, VDA_GATE_LOG>(a, stream) : step<false, VDA_GATE_LOG>(a, stream);
    case VDA_GATE_LOGIT: return f32 ? step<true, VDA_GATE_LOGIT>(a, stream) : step<false, VDA_GATE_LOGIT>(a, stream);
    default: return f32 ? step<true, VDA_GATE_NORM>(a, stream) : step<false, VDA_GATE_NORM>(a, stream);
  }
}

}  // namespace vda
