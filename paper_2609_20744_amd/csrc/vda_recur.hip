// The channel-wise gated recurrence, its gradients and its recurrent form (vda.h,
// vda_recur_*): h_t = a_t h_{t-1} + u_t for each channel of each sequence.
//
// A stretch of tokens acts on the state that enters it as h -> A h + H, A = prod a.  A
// workgroup has 128 channels, eight to a lane, and 16 runs of consecutive tokens side by
// side: each run makes its A and H from zero in registers, and the 16 are joined
// through LDS.
//
// Forward: sequences are cut into segments, as many as fill the device.  One kernel
// makes the segments' A and H, the other composes those before its own segment,
// and goes through it in tiles, the next tile's loads on the way.  A
// sequence of one segment takes the second kernel alone.
//
// The gradient runs the other way: with E_t = a_t D_t, D_t = dout_t + E_{t+1}, a tile takes the
// E that enters at its end to A E + G, with the same A and G = sum_t (a_1 .. a_t) dout_t, so
// one reduction makes all three; h is made again from x and the gates, nothing is kept.
// Three kernels: what every tile does, what enters it from both sides, the gradients.
// A place behind a sequence's end has a = 1, u = 0 and dout = 0.
//
// Bytes bound it: each pass streams its inputs once.
#include <type_traits>

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

// A token's decay a, and b = 1 - a with its own rounding only (log: not made).
template <int GATE>
__device__ __forceinline__ void gate_of(float g, float& a, float& b) {
  if constexpr (GATE == VDA_GATE_LOG) {
    a = __builtin_amdgcn_exp2f(g * 1.4426950408889634f), b = 0.f;
  } else {
    // Below -80 a is 0 beside any state; e stays finite there.
    const float e = __builtin_amdgcn_exp2f(fmaxf(g, -80.f) * -1.4426950408889634f);
    a = __builtin_amdgcn_rcpf(1.f + e), b = e * a;
  }
}
// The state h behind a token, or a stretch of tokens, of decay a that adds u.  A decay of 0 forgets h,
// whatever it is: 0 times an infinity or NaN would keep it.
__device__ __forceinline__ float after(float a, float h, float u) { return a == 0.f ? u : fmaf(a, h, u); }
// ... of one token: a sigmoid is never 0.
template <int GATE>
__device__ __forceinline__ float after(float a, float h, float u) {
  return GATE == VDA_GATE_LOG ? after(a, h, u) : fmaf(a, h, u);
}
// What x is multiplied by.
template <int GATE>
__device__ __forceinline__ float weight_of(float a, float b) {
  return GATE == VDA_GATE_LOG ? 1.f : GATE == VDA_GATE_LOGIT ? b : __builtin_amdgcn_sqrtf(b * (1.f + a));
}

// A sequence and a part of it, of `per` tokens (a tile, a segment).
struct RecurTile {
  int seq, first, len, tile, last;  // first token and tokens of the sequence; the part's index and that of its last
};
__device__ __forceinline__ bool tile_of(const RecurArgs& a, int t, int per, RecurTile& r) {
  if (a.cu == nullptr) {
    const int each = (a.L + per - 1) / per;
    r.seq = uniform(t / each), r.tile = t - r.seq * each;
    r.first = r.seq * a.L, r.len = a.L;
  } else {
    // Sequence i has the places from first_i / per + i on.
    const int lane = threadIdx.x & 63;
    int before = 0;
    for (int b = 0; b < a.n; b += 64) {
      const int i = b + lane, c = a.cu[i < a.n ? i : 0];
      before += __popcll(__ballot(i < a.n && (c < 0 ? 0 : c > a.T ? a.T : c) / per + i <= t));
    }
    r.seq = uniform(before) - 1;
    if (r.seq < 0) return false;
    const int c = uniform(a.cu[r.seq]), d = uniform(a.cu[r.seq + 1]);
    r.first = c < 0 ? 0 : c > a.T ? a.T : c;
    const int end = d < 0 ? 0 : d > a.T ? a.T : d;
    r.len = end > r.first ? end - r.first : 0;
    r.tile = t - (r.first / per + r.seq);
    if (r.tile < 0) return false;
  }
  r.last = r.len > 0 ? (r.len - 1) / per : 0;
  return r.tile <= r.last;
}

// A workgroup's part and channels: all channels of a part after each other, so that
// workgroups that run together read and write whole rows.
__device__ __forceinline__ void place_of(const RecurArgs& a, int& place, int& slab) {
  const unsigned slabs = (unsigned)(a.C + kRecurChans - 1) / kRecurChans;
  place = uniform(blockIdx.x / slabs), slab = uniform(blockIdx.x - place * slabs);
}

// A lane's channels and run.
struct Lane {
  bool real;  // there are such channels
  int chan, run;
};
__device__ __forceinline__ Lane lane_of(const RecurArgs& a, int slab) {
  Lane w;
  w.chan = (slab * 16 + (threadIdx.x & 15)) * 8;
  w.real = w.chan < a.C;
  if (!w.real) w.chan = 0;
  w.run = threadIdx.x >> 4;
  return w;
}

// The row of place p of a sequence, in the order of the recurrence; the last one's behind its end.
__device__ __forceinline__ size_t row_at(const RecurArgs& a, const RecurTile& r, int p) {
  p = p < r.len ? p : r.len - 1;
  return (size_t)(a.reverse ? r.first + r.len - 1 - p : r.first + p);
}

// Eight channels of N tokens as they are in memory.
template <bool F32, int N>
struct Raw {
  static constexpr int kWords = F32 ? 8 : 4;
  uint32_t w[N][kWords];
  __device__ __forceinline__ void load(const void* p, size_t at, int i) {
    const uint4* from = reinterpret_cast<const uint4*>((const char*)p + at * (F32 ? 4 : 2));
#pragma unroll
    for (int j = 0; j < kWords / 4; ++j) {
      const uint4 v = from[j];
      w[i][4 * j] = v.x, w[i][4 * j + 1] = v.y, w[i][4 * j + 2] = v.z, w[i][4 * j + 3] = v.w;
    }
  }
  __device__ __forceinline__ float value(int i, int e) const {
    if constexpr (F32)
      return __uint_as_float(w[i][e]);
    else
      return e & 1 ? bf16_hi(w[i][e / 2]) : bf16_lo(w[i][e / 2]);
  }
};

// A run of N tokens from place p of the sequence (none read where it is empty).
template <bool F32, int GATE, int N>
struct Tokens {
  static constexpr bool kGate32 = F32 || GATE == VDA_GATE_LOG;
  Raw<F32, N> x;
  Raw<kGate32, N> g;
  __device__ __forceinline__ void load(const RecurArgs& a, const RecurTile& r, const Lane& w, int p) {
    if (r.len == 0) return;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const size_t row = row_at(a, r, p + i);
      x.load(a.x, row * a.xs + w.chan, i);
      g.load(a.g, row * a.gs + w.chan, i);
    }
  }
  // a and u of token i, channel e; `is`: whether there is such a token.
  __device__ __forceinline__ void step(int i, int e, bool is, float& al, float& u) const {
    float b;
    gate_of<GATE>(g.value(i, e), al, b);
    u = weight_of<GATE>(al, b) * x.value(i, e);
    if (!is) al = 1.f, u = 0.f;
  }
};

// What the runs of a tile do, through LDS: [run][A or H][channel].
typedef float RunTable[kRecurRuns][2][kRecurChans];
__device__ __forceinline__ void put_run(RunTable& t, int run, const float (&A)[8], const float (&H)[8]) {
  const int c = (threadIdx.x & 15) * 8;
#pragma unroll
  for (int e = 0; e < 8; e += 4) {
    *reinterpret_cast<floatx4*>(&t[run][0][c + e]) = floatx4{A[e], A[e + 1], A[e + 2], A[e + 3]};
    *reinterpret_cast<floatx4*>(&t[run][1][c + e]) = floatx4{H[e], H[e + 1], H[e + 2], H[e + 3]};
  }
}
// What enters each run, given what enters the first: the state (h -> A h + H), a thread a
// channel, which keeps it from tile to tile.
typedef float RunStates[kRecurRuns][kRecurChans];
__device__ __forceinline__ float scan_runs(const RunTable& t, RunStates& to, float h, int c) {
  float A[kRecurRuns], H[kRecurRuns];
#pragma unroll
  for (int i = 0; i < kRecurRuns; ++i) A[i] = t[i][0][c], H[i] = t[i][1][c];
#pragma unroll
  for (int i = 0; i < kRecurRuns; ++i) {
    to[i][c] = h;
    h = after(A[i], h, H[i]);
  }
  return h;
}
__device__ __forceinline__ void get_states(const RunStates& t, int run, float (&h)[8]) {
  const int c = (threadIdx.x & 15) * 8;
#pragma unroll
  for (int e = 0; e < 8; e += 4) {
    const floatx4 x = *reinterpret_cast<const floatx4*>(&t[run][c + e]);
#pragma unroll
    for (int u = 0; u < 4; ++u) h[e + u] = x[u];
  }
}

// What a segment does: a run has an equal share of its tokens, kBatch at a time.  40320 tokens of
// 896 channels, log decays in fp32: 50 us, 217 MB at 4.3 TB/s.
template <bool F32, int GATE>
__global__ __launch_bounds__(kThreads) void recur_segment_kernel(RecurArgs a) {
  constexpr int N = F32 || GATE == VDA_GATE_LOG ? 4 : 8;
  __shared__ __align__(16) RunTable table;
  RecurTile r;
  int place, slab;
  place_of(a, place, slab);
  if (!tile_of(a, place, a.seg, r)) return;
  if (r.tile == r.last) return;  // nothing comes behind it
  const Lane w = lane_of(a, slab);
  const int share = a.seg / kRecurRuns, p0 = r.tile * a.seg + w.run * share;
  float A[8], H[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) A[e] = 1.f, H[e] = 0.f;
  Tokens<F32, GATE, N> now, next;
  now.load(a, r, w, p0);
  for (int i0 = 0; i0 < share; i0 += N) {
    if (i0 + N < share) next.load(a, r, w, p0 + i0 + N);
#pragma unroll
    for (int i = 0; i < N; ++i)
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        float al, u;
        now.step(i, e, true, al, u);  // only the last segment has an end
        H[e] = fmaf(al, H[e], u);
        A[e] *= al;
      }
    now = next;
  }
  put_run(table, w.run, A, H);
  lds_barrier();
  const int at = threadIdx.x, chan = slab * kRecurChans + at;
  if (at >= kRecurChans || chan >= a.C) return;
  float X = 1.f, Y = 0.f;
#pragma unroll
  for (int i = 0; i < kRecurRuns; ++i) {
    Y = fmaf(table[i][0][at], Y, table[i][1][at]);
    X *= table[i][0][at];
  }
  const size_t to = (size_t)place * a.C + chan;
  a.A[to] = X, a.H[to] = Y;
}

// The outputs: what enters the segment from all before it, then tile after tile.  As above 49 us,
// 289 MB at 5.9 TB/s, some of it from the last-level cache.
template <bool F32, int GATE>
__global__ __launch_bounds__(kThreads) void recur_apply_kernel(RecurArgs a) {
  constexpr int N = 4, kTile = kRecurRuns * N;
  __shared__ __align__(16) RunTable table;
  __shared__ __align__(16) RunStates states;
  RecurTile r;
  int place, slab;
  place_of(a, place, slab);
  if (!tile_of(a, place, a.seg, r)) return;
  const Lane w = lane_of(a, slab);
  const int begin = r.tile * a.seg, end = r.tile == r.last ? r.len : begin + a.seg;
  Tokens<F32, GATE, N> now, next;
  now.load(a, r, w, begin + w.run * N);
  // The thread's channel, whose state it carries.
  const int c = threadIdx.x, chan = slab * kRecurChans + c;
  const bool carries = c < kRecurChans, real = carries && chan < a.C;
  float h = 0.f;
  if (real && a.S_in != nullptr) h = a.S_in[(size_t)r.seq * a.C + chan];
  if (r.tile > 0) {
    // The segments before this one, an equal share of them by each run.
    const int share = (r.tile + kRecurRuns - 1) / kRecurRuns;
    const int from = w.run * share, to = from + share < r.tile ? from + share : r.tile;
    const size_t base = ((size_t)place - r.tile) * a.C + w.chan;
    float A[8], H[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) A[e] = 1.f, H[e] = 0.f;
#pragma unroll 4
    for (int j = from; j < to; ++j) {
      float x[8], y[8];
      load8<true>(a.A, base + (size_t)j * a.C, x);
      load8<true>(a.H, base + (size_t)j * a.C, y);
#pragma unroll
      for (int e = 0; e < 8; ++e) H[e] = fmaf(x[e], H[e], y[e]), A[e] *= x[e];
    }
    put_run(table, w.run, A, H);
    lds_barrier();
    if (carries) h = scan_runs(table, states, h, c);
    lds_barrier();
  }
  auto tile = [&](int p0, auto full) {
    const int p = p0 + w.run * N;
    float al[N][8], u[N][8], A[8], H[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) A[e] = 1.f, H[e] = 0.f;
#pragma unroll
    for (int i = 0; i < N; ++i)
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        now.step(i, e, full || p + i < end, al[i][e], u[i][e]);
        H[e] = fmaf(al[i][e], H[e], u[i][e]);
        A[e] *= al[i][e];
      }
    put_run(table, w.run, A, H);
    lds_barrier();
    if (carries) h = scan_runs(table, states, h, c);
    lds_barrier();
    get_states(states, w.run, H);
    if (w.real) {
#pragma unroll
      for (int i = 0; i < N; ++i) {
#pragma unroll
        for (int e = 0; e < 8; ++e) H[e] = after<GATE>(al[i][e], H[e], u[i][e]);
        if (full || p + i < end) store8<F32>(a.out, row_at(a, r, p + i) * a.C + w.chan, H);
      }
    }
  };
  int p0 = begin;
  for (; p0 + kTile < end; p0 += kTile) {
    next.load(a, r, w, p0 + kTile + w.run * N);
    tile(p0, std::true_type());
    now = next;
  }
  tile(p0, std::false_type());
  if (a.S_out != nullptr && r.tile == r.last && real) a.S_out[(size_t)r.seq * a.C + chan] = h;
}

// What every tile of 64 tokens does, in both directions.  9 sequences of 16401 tokens, 2048 channels:
// 48 us, 202 MB at 4.2 TB/s.
template <bool F32, int GATE>
__global__ __launch_bounds__(kThreads) void recur_reduce_kernel(RecurArgs a) {
  __shared__ __align__(16) RunTable table;
  __shared__ __align__(16) float sG[kRecurRuns][kRecurChans];
  RecurTile r;
  int place, slab;
  place_of(a, place, slab);
  if (!tile_of(a, place, kRecurTile, r)) return;
  if (r.len <= kRecurTile) return;  // nothing enters its one tile from another
  const Lane w = lane_of(a, slab);
  const int p = r.tile * kRecurTile + w.run * kRecurRun;
  Tokens<F32, GATE, kRecurRun> t;
  Raw<F32, kRecurRun> y;
  t.load(a, r, w, p);
#pragma unroll
  for (int i = 0; i < kRecurRun; ++i) y.load(a.dout, row_at(a, r, p + i) * a.C + w.chan, i);
  float A[8], H[8], G[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    A[e] = 1.f, H[e] = 0.f, G[e] = 0.f;
#pragma unroll
    for (int i = 0; i < kRecurRun; ++i) {
      float al, u;
      t.step(i, e, p + i < r.len, al, u);
      H[e] = fmaf(al, H[e], u);
      A[e] *= al;
      G[e] = p + i < r.len ? fmaf(A[e], y.value(i, e), G[e]) : G[e];
    }
  }
  put_run(table, w.run, A, H);
  const int c = (threadIdx.x & 15) * 8;
#pragma unroll
  for (int e = 0; e < 8; e += 4) *reinterpret_cast<floatx4*>(&sG[w.run][c + e]) = floatx4{G[e], G[e + 1], G[e + 2], G[e + 3]};
  lds_barrier();
  const int at = threadIdx.x, chan = slab * kRecurChans + at;
  if (at >= kRecurChans || chan >= a.C) return;
  float X = 1.f, Y = 0.f, Z = 0.f;
#pragma unroll
  for (int i = 0; i < kRecurRuns; ++i) {
    Z = fmaf(X, sG[i][at], Z);
    Y = fmaf(table[i][0][at], Y, table[i][1][at]);
    X *= table[i][0][at];
  }
  const size_t to = (size_t)place * a.C + chan;
  a.A[to] = X, a.H[to] = Y, a.G[to] = Z;
}

// What enters each tile of a sequence: a lane has a channel, a wave a range of the
// tiles.  H becomes the state that enters a tile, G the E that enters at its end.  As above 8 us
// (with a tile's values kept in registers for the second way 12 us).
constexpr int kCarryWaves = 16;
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
    G = fmaf(A, a.G[at], G);
    H = fmaf(ta, H, th);
    A *= ta;
  }
  sA[wave][lane] = A, sH[wave][lane] = H, sG[wave][lane] = G;
  lds_barrier();
  const size_t st = (size_t)seq * a.C + chan;
  float h = real && a.S_in != nullptr ? a.S_in[st] : 0.f;
  for (int w = 0; w < wave; ++w) h = after(sA[w][lane], h, sH[w][lane]);
  float e = real && a.dS_out != nullptr ? a.dS_out[st] : 0.f;
  for (int w = kCarryWaves - 1; w > wave; --w) e = fmaf(sA[w][lane], e, sG[w][lane]);
  if (!real) return;
#pragma unroll 8
  for (int t = from; t < to; ++t) {
    const size_t at = base + (size_t)t * a.C;
    const float next = after(a.A[at], h, a.H[at]);
    a.H[at] = h;
    h = next;
  }
#pragma unroll 8
  for (int t = to - 1; t >= from; --t) {
    const size_t at = base + (size_t)t * a.C;
    const float next = fmaf(a.A[at], e, a.G[at]);
    a.G[at] = e;
    e = next;
  }
}

// The gradients of a tile: its states and E again from what enters it.  As above 63 us, 336 MB at
// 5.3 TB/s; runs of 4 tokens, as with 8 the registers spilled.
template <bool F32, int GATE>
__global__ __launch_bounds__(kThreads) void recur_grad_kernel(RecurArgs a) {
  constexpr int N = kRecurRun;
  constexpr bool kGate32 = F32 || GATE == VDA_GATE_LOG;
  __shared__ __align__(16) RunTable table;
  __shared__ __align__(16) RunStates sG, states, grads;
  RecurTile r;
  int place, slab;
  place_of(a, place, slab);
  if (!tile_of(a, place, kRecurTile, r)) return;
  const Lane w = lane_of(a, slab);
  const int p = r.tile * kRecurTile + w.run * N;
  Tokens<F32, GATE, N> t;
  Raw<F32, N> y;
  t.load(a, r, w, p);
  if (r.len > 0)
#pragma unroll
    for (int i = 0; i < N; ++i) y.load(a.dout, row_at(a, r, p + i) * a.C + w.chan, i);
  // A thread has the state of a channel, or the gradient that comes to it from behind.
  const int c = threadIdx.x % kRecurChans, chan = slab * kRecurChans + c;
  const bool back = threadIdx.x >= kRecurChans, real = chan < a.C;
  const bool carried = a.carried && r.len > kRecurTile;
  const float* from = carried ? (back ? a.G : a.H) : back ? a.dS_out : a.S_in;
  float z = 0.f;
  if (real && from != nullptr) z = from[(carried ? (size_t)place : (size_t)r.seq) * a.C + chan];

  float al[N][8], b[N][8], A[8], H[8], G[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    A[e] = 1.f, H[e] = 0.f, G[e] = 0.f;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      gate_of<GATE>(t.g.value(i, e), al[i][e], b[i][e]);
      float u = weight_of<GATE>(al[i][e], b[i][e]) * t.x.value(i, e), d = y.value(i, e);
      if (p + i >= r.len) al[i][e] = 1.f, u = d = 0.f;
      H[e] = fmaf(al[i][e], H[e], u);
      A[e] *= al[i][e];
      G[e] = fmaf(A[e], d, G[e]);
    }
  }
  put_run(table, w.run, A, H);
#pragma unroll
  for (int e = 0; e < 8; e += 4)
    *reinterpret_cast<floatx4*>(&sG[w.run][(threadIdx.x & 15) * 8 + e]) = floatx4{G[e], G[e + 1], G[e + 2], G[e + 3]};
  lds_barrier();
  if (!back) {
    scan_runs(table, states, z, c);
  } else {
#pragma unroll
    for (int i = kRecurRuns - 1; i >= 0; --i) {
      grads[i][c] = z;
      z = fmaf(table[i][0][c], z, sG[i][c]);
    }
    if (a.dS_in != nullptr && r.tile == 0 && real) a.dS_in[(size_t)r.seq * a.C + chan] = z;
  }
  lds_barrier();
  if (!w.real) return;
  get_states(states, w.run, H);
  get_states(grads, w.run, G);
  // Over the states, then back.
  float dx[N][8], dg[N][8];
#pragma unroll
  for (int i = 0; i < N; ++i)
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      dg[i][e] = H[e];  // the state before the token
      dx[i][e] = weight_of<GATE>(al[i][e], b[i][e]);
      H[e] = after<GATE>(al[i][e], H[e], dx[i][e] * t.x.value(i, e));
    }
#pragma unroll
  for (int i = N - 1; i >= 0; --i)
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const bool is = p + i < r.len;
      const float x = t.x.value(i, e), d = (is ? y.value(i, e) : 0.f) + G[e], ai = al[i][e];
      if constexpr (GATE == VDA_GATE_LOG)
        dg[i][e] = ai == 0.f ? 0.f : dg[i][e] * (d * ai);
      else if constexpr (GATE == VDA_GATE_LOGIT)
        dg[i][e] = d * ai * b[i][e] * (dg[i][e] - x);
      else
        dg[i][e] = d * (ai * b[i][e] * dg[i][e] -
                        ai * ai * __builtin_amdgcn_sqrtf(b[i][e] * __builtin_amdgcn_rcpf(1.f + ai)) * x);
      dx[i][e] *= d;
      G[e] = ai * d;
    }
#pragma unroll
  for (int i = 0; i < N; ++i)
    if (p + i < r.len) {
      const size_t row = row_at(a, r, p + i);
      store8<F32>(a.dx, row * a.dxs + w.chan, dx[i]);
      store8<kGate32>(a.dg, row * a.dgs + w.chan, dg[i]);
    }
}

__device__ __forceinline__ floatx4 load4(const float* p) { return *reinterpret_cast<const floatx4*>(p); }
__device__ __forceinline__ floatx4 load4(const uint16_t* p) {
  const uint2 w = *reinterpret_cast<const uint2*>(p);
  return floatx4{bf16_lo(w.x), bf16_hi(w.x), bf16_lo(w.y), bf16_hi(w.y)};
}

// A lane has four channels of a sequence.  192 sequences of 2048 channels: 3 us, a launch's latency.
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
      h[e] = after<GATE>(al, h[e], weight_of<GATE>(al, b) * x[e]);
    }
    if constexpr (F32)
      *reinterpret_cast<floatx4*>((float*)a.out + at) = h;
    else
      *reinterpret_cast<uint2*>((uint16_t*)a.out + at) = make_uint2(pack_bf16x2(h[0], h[1]), pack_bf16x2(h[2], h[3]));
  }
  *reinterpret_cast<floatx4*>(S) = h;
}

unsigned grid_of(const RecurArgs& a) { return (unsigned)a.tiles * (unsigned)((a.C + kRecurChans - 1) / kRecurChans); }

template <bool F32, int GATE>
hipError_t forward(const RecurArgs& a, hipStream_t stream) {
  if (a.carried) recur_segment_kernel<F32, GATE><<<grid_of(a), kThreads, 0, stream>>>(a);
  recur_apply_kernel<F32, GATE><<<grid_of(a), kThreads, 0, stream>>>(a);
  return hipGetLastError();
}
template <bool F32, int GATE>
hipError_t backward(const RecurArgs& a, hipStream_t stream) {
  if (a.carried) {
    recur_reduce_kernel<F32, GATE><<<grid_of(a), kThreads, 0, stream>>>(a);
    recur_carry_kernel<<<dim3(a.n, (a.C + 63) / 64), 64 * kCarryWaves, 0, stream>>>(a);
  }
  recur_grad_kernel<F32, GATE><<<grid_of(a), kThreads, 0, stream>>>(a);
  return hipGetLastError();
}
template <bool F32, int GATE>
hipError_t step(const RecurStepArgs& a, hipStream_t stream) {
  const unsigned grid = (unsigned)(((size_t)a.n * (a.C / 4) + kThreads - 1) / kThreads);
  recur_step_kernel<F32, GATE><<<grid, kThreads, 0, stream>>>(a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_recur(bool f32, bool back, const RecurArgs& a, hipStream_t stream) {
  switch (a.gate) {
    case VDA_GATE_LOG:
      return f32 ? (back ? backward<true, VDA_GATE_LOG>(a, stream) : forward<true, VDA_GATE_LOG>(a, stream))
                 : (back ? backward<false, VDA_GATE_LOG>(a, stream) : forward<false, VDA_GATE_LOG>(a, stream));
    case VDA_GATE_LOGIT:
      return f32 ? (back ? backward<true, VDA_GATE_LOGIT>(a, stream) : forward<true, VDA_GATE_LOGIT>(a, stream))
                 : (back ? backward<false, VDA_GATE_LOGIT>(a, stream) : forward<false, VDA_GATE_LOGIT>(a, stream));
    default:
      return f32 ? (back ? backward<true, VDA_GATE_NORM>(a, stream) : forward<true, VDA_GATE_NORM>(a, stream))
                 : (back ? backward<false, VDA_GATE_NORM>(a, stream) : forward<false, VDA_GATE_NORM>(a, stream));
  }
}

hipError_t launch_recur_step(bool f32, const RecurStepArgs& a, hipStream_t stream) {
  switch (a.gate) {
    case VDA_GATE_LOG: return f32 ? step<true, VDA_GATE_LOG>(a, stream) : step<false, VDA_GATE_LOG>(a, stream);
    case VDA_GATE_LOGIT: return f32 ? step<true, VDA_GATE_LOGIT>(a, stream) : step<false, VDA_GATE_LOGIT>(a, stream);
    default: return f32 ? step<true, VDA_GATE_NORM>(a, stream) : step<false, VDA_GATE_NORM>(a, stream);
  }
}

}  // namespace vda
