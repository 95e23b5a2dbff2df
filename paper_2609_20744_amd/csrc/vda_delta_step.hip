// Token-wise gated delta rule, recurrent form: a few tokens of each sequence
// of a batch against the state pool, in place (vda.h, vda_delta_step).
//
// The call reads and writes each state once, 8 d_v d_k bytes, beside which
// everything else is small, so it is bound by HBM for a full batch and by latency
// for one sequence.  The rows of a state are independent but for k and q: a
// group of d_k / 4 lanes (at most 16) holds a row, a wave ROWS rows, all
// loaded before the first is used, and the rows stay in registers over the
// call's tokens.  Both products with the state take it before the update,
//     u = S k, w = S q:  e = v - a u,  S <- a S + beta e k,  o = scale (a w + beta e (k.q)),
// so their sums over a row's lanes (DPP adds within 16 lanes) run together.
// fp32 throughout.  192 sequences of 32 heads, 128 x 128: 163 us, 4.98 TB/s (a
// large copy: 4.96; rows of padding cost nothing: 180 of 192, 153 us); one
// sequence of 16 heads: 4.5 us.
#include "vda_delta.h"
#include "vda_delta_step.h"

namespace vda {
namespace {

__device__ __forceinline__ floatx4 load4(const float* p) { return *reinterpret_cast<const floatx4*>(p); }
__device__ __forceinline__ floatx4 load4(const uint16_t* p) {
  const uint2 w = *reinterpret_cast<const uint2*>(p);
  return floatx4{bf16_lo(w.x), bf16_hi(w.x), bf16_lo(w.y), bf16_hi(w.y)};
}
__device__ __forceinline__ float load1(const float* p) { return *p; }
__device__ __forceinline__ float load1(const uint16_t* p) { return __uint_as_float((uint32_t)*p << 16); }
__device__ __forceinline__ void store1(float* p, float x) { *p = x; }
__device__ __forceinline__ void store1(uint16_t* p, float x) { *p = __builtin_bit_cast(uint16_t, (__bf16)x); }

// PASSES: rows of a wave = PASSES * 64 / LANES.
template <bool F32, int DK, int PASSES>
__global__ __launch_bounds__(kThreads) void delta_step_kernel(StepArgs a) {
  typedef typename Op<F32>::Elem E;
  constexpr int LANES = DK / 4 < 16 ? DK / 4 : 16, VEC = DK / 4 / LANES;
  constexpr int kRows = PASSES * 64 / LANES;  // of a wave
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = uniform(tid >> 6);
  const int per = (a.d_v + 4 * kRows - 1) / (4 * kRows);  // workgroups of a head
  const int rb = blockIdx.x % (unsigned)per;
  const unsigned nh = blockIdx.x / (unsigned)per;
  const int h = uniform(nh % (unsigned)a.Hv), n = uniform(nh / (unsigned)a.Hv);
  const int slot = a.slots != nullptr ? uniform(a.slots[n]) : n;
  // Padding rows, and slots that the pool does not have.
  if (slot < 0 || slot >= a.n_slots) return;
  const int at = lane % LANES, row0 = (rb * 4 + wave) * kRows + lane / LANES;
  if ((rb * 4 + wave) * kRows >= a.d_v) return;
  float* S = a.state + ((size_t)slot * a.Hv + h) * a.d_v * DK;

  floatx4 s[PASSES][VEC];
#pragma unroll
  for (int p = 0; p < PASSES; ++p) {
    const int row = row0 + p * (64 / LANES);
#pragma unroll
    for (int c = 0; c < VEC; ++c)
      s[p][c] = row < a.d_v ? load4(S + (size_t)row * DK + 4 * (c * LANES + at)) : floatx4{0.f, 0.f, 0.f, 0.f};
  }
  for (int t = 0; t < a.tokens; ++t) {
    const size_t tok = (size_t)n * a.tokens + t;
    const size_t qk = (tok * a.Hk + h / a.group) * DK, vo = (tok * a.Hv + h) * a.d_v;
    floatx4 k[VEC], q[VEC];
    float kq = 0.f;
#pragma unroll
    for (int c = 0; c < VEC; ++c) {
      k[c] = load4((const E*)a.k + qk + 4 * (c * LANES + at));
      q[c] = load4((const E*)a.q + qk + 4 * (c * LANES + at));
    }
    float v[PASSES];
#pragma unroll
    for (int p = 0; p < PASSES; ++p) {
      const int row = row0 + p * (64 / LANES);
      v[p] = row < a.d_v ? load1((const E*)a.v + vo + row) : 0.f;
    }
    const float decay = expf(a.g[tok * a.Hv + h]), beta = a.beta[tok * a.Hv + h];
#pragma unroll
    for (int c = 0; c < VEC; ++c)
#pragma unroll
      for (int e = 0; e < 4; ++e) kq += k[c][e] * q[c][e];
    kq = group_sum<LANES>(kq);
#pragma unroll
    for (int p = 0; p < PASSES; ++p) {
      float u = 0.f, w = 0.f;
#pragma unroll
      for (int c = 0; c < VEC; ++c)
#pragma unroll
        for (int e = 0; e < 4; ++e) u += s[p][c][e] * k[c][e], w += s[p][c][e] * q[c][e];
      u = group_sum<LANES>(u), w = group_sum<LANES>(w);
      const float write = beta * (v[p] - decay * u);
#pragma unroll
      for (int c = 0; c < VEC; ++c) s[p][c] = decay * s[p][c] + write * k[c];
      const int row = row0 + p * (64 / LANES);
      if (at == 0 && row < a.d_v) store1((E*)a.out + vo + row, a.scale * (decay * w + write * kq));
    }
  }
#pragma unroll
  for (int p = 0; p < PASSES; ++p) {
    const int row = row0 + p * (64 / LANES);
    if (row < a.d_v)
#pragma unroll
      for (int c = 0; c < VEC; ++c) *reinterpret_cast<floatx4*>(S + (size_t)row * DK + 4 * (c * LANES + at)) = s[p][c];
  }
}

template <bool F32, int DK>
hipError_t run(const StepArgs& a, hipStream_t stream) {
  constexpr int LANES = DK / 4 < 16 ? DK / 4 : 16, PASSES = 4, rows = 4 * PASSES * 64 / LANES;
  const unsigned grid = (unsigned)a.n * (unsigned)a.Hv * (unsigned)((a.d_v + rows - 1) / rows);
  delta_step_kernel<F32, DK, PASSES><<<grid, kThreads, 0, stream>>>(a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_delta_step(bool f32, int d_k, const StepArgs& a, hipStream_t stream) {
  switch (d_k) {
    case 32: return f32 ? run<true, 32>(a, stream) : run<false, 32>(a, stream);
    case 64: return f32 ? run<true, 64>(a, stream) : run<false, 64>(a, stream);
    default: return f32 ? run<true, 128>(a, stream) : run<false, 128>(a, stream);
  }
}

}  // namespace vda
