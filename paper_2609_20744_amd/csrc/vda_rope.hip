// Rotary positions over time, height and width, and their gradient (vda.h,
// vda_rope).  Pair p of a head's channels is turned by the angle
// position * inv_freq[p], the position being the token's on the pair's axis;
// with the L2 map each token of each head is divided by sqrt(sum x^2 + eps)
// first.
//
// Everything is read and written once, so HBM bounds it.  The angles are the
// work: they are taken in 64 bits (a position of 2^20 times a frequency of 1
// leaves 4 bits of a fp32 angle's fraction), as turns, whose integer part falls away
// before the fp32 sine and cosine.  All heads of a token share them: a
// workgroup makes those of a few tokens once, in LDS, and then streams the
// tokens' rows, a lane taking eight pairs (two vectors of eight channels) of one
// head at a time.  138240 tokens of 16 heads of 128 channels, bf16, with the L2
// map: 211 us, 5.4 TB/s (a large copy: 4.96); the gradient of 32760 tokens of 24
// heads 119 us, 5.1 TB/s.
#include "vda_delta.h"
#include "vda_rope.h"

namespace vda {
namespace {

constexpr int kTokens = 4;    // of a workgroup
constexpr int kMaxPairs = 64; // d / 2

template <bool F32>
struct Vec8 {
  float x[8];
  __device__ __forceinline__ void load(const void* p, size_t at) {
    if constexpr (F32) {
      const float* f = (const float*)p + at;
      const floatx4 a = *reinterpret_cast<const floatx4*>(f), b = *reinterpret_cast<const floatx4*>(f + 4);
#pragma unroll
      for (int e = 0; e < 4; ++e) x[e] = a[e], x[4 + e] = b[e];
    } else {
      const uint4 w = *reinterpret_cast<const uint4*>((const uint16_t*)p + at);
      const uint32_t v[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
      for (int e = 0; e < 4; ++e) x[2 * e] = bf16_lo(v[e]), x[2 * e + 1] = bf16_hi(v[e]);
    }
  }
  __device__ __forceinline__ void store(void* p, size_t at) const {
    if constexpr (F32) {
      float* f = (float*)p + at;
      *reinterpret_cast<floatx4*>(f) = floatx4{x[0], x[1], x[2], x[3]};
      *reinterpret_cast<floatx4*>(f + 4) = floatx4{x[4], x[5], x[6], x[7]};
    } else {
      *reinterpret_cast<uint4*>((uint16_t*)p + at) =
          make_uint4(pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3]), pack_bf16x2(x[4], x[5]),
                     pack_bf16x2(x[6], x[7]));
    }
  }
};

// Sum over aligned groups of `lanes` lanes (2, 4 or 8), in every lane.
__device__ __forceinline__ float row_sum(float x, int lanes) {
  for (int m = 1; m < lanes; m <<= 1) x += __shfl_xor(x, m);
  return x;
}

template <bool F32, bool BACKWARD>
__global__ __launch_bounds__(kThreads) void rope_kernel(RopeArgs a) {
  __shared__ __align__(16) float2 turn[kTokens][kMaxPairs];  // cos, sin
  const int R = a.pairs[0] + a.pairs[1] + a.pairs[2];
  const size_t tokens = (size_t)a.B * a.L;
  const size_t tok0 = (size_t)blockIdx.x * kTokens;
  const int here = tokens - tok0 < kTokens ? (int)(tokens - tok0) : kTokens;
  for (int i = threadIdx.x; i < here * R; i += kThreads) {
    const int t = i / R, p = i - t * R;
    const int axis = p < a.pairs[0] ? 0 : p < a.pairs[0] + a.pairs[1] ? 1 : 2;
    int pos;
    if (a.positions != nullptr) {
      pos = a.positions[(tok0 + t) * 3 + axis];
    } else {
      const int n = (int)((tok0 + t) % (unsigned)a.L);
      const int col = n % a.grid_w, y = n / a.grid_w;
      pos = axis == 2 ? col : axis == 1 ? y % a.grid_h : a.frame_offset + y / a.grid_h;
    }
    double turns = (double)pos * (double)a.inv_freq[p] * 0.15915494309189535;
    turns -= rint(turns);
    float s, c;
    sincospif(2.f * (float)turns, &s, &c);
    turn[t][p] = make_float2(c, BACKWARD ? -s : s);
  }
  __syncthreads();

  const int lanes = a.d / 16;  // of one head of one token
  const int items = here * a.H * lanes;
  for (int i = threadIdx.x; i < items; i += kThreads) {
    const int slot = i % lanes, th = i / lanes;
    const int t = th / a.H, h = th - t * a.H;
    // The lane's two vectors of eight channels.
    const bool rot = 8 * slot < R;
    const int c0 = !rot || a.interleaved ? 16 * slot : 8 * slot;
    const int c1 = !rot || a.interleaved ? 16 * slot + 8 : R + 8 * slot;
    const size_t tok = tok0 + t;
    const size_t b = tok / (unsigned)a.L, n = tok - b * a.L;
    const size_t row_x = tok * a.x_stride + (size_t)h * a.d;
    const size_t row_y = a.heads ? ((b * a.H + h) * a.L + n) * a.d : (tok * a.H + h) * a.d;
    Vec8<F32> u, v;
    if constexpr (BACKWARD) {
      u.load(a.dout, row_y + c0), v.load(a.dout, row_y + c1);
    } else {
      u.load(a.x, row_x + c0), v.load(a.x, row_x + c1);
      if (a.l2) {
        float ss = 0.f;
#pragma unroll
        for (int e = 0; e < 8; ++e) ss += u.x[e] * u.x[e] + v.x[e] * v.x[e];
        const float r = 1.f / sqrtf(row_sum(ss, lanes) + kL2Eps);
#pragma unroll
        for (int e = 0; e < 8; ++e) u.x[e] *= r, v.x[e] *= r;
      }
    }
    if (rot) {
      if (a.interleaved) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float2 p = turn[t][8 * slot + e], q = turn[t][8 * slot + 4 + e];
          const float x0 = u.x[2 * e], x1 = u.x[2 * e + 1], y0 = v.x[2 * e], y1 = v.x[2 * e + 1];
          u.x[2 * e] = x0 * p.x - x1 * p.y, u.x[2 * e + 1] = x0 * p.y + x1 * p.x;
          v.x[2 * e] = y0 * q.x - y1 * q.y, v.x[2 * e + 1] = y0 * q.y + y1 * q.x;
        }
      } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const float2 p = turn[t][8 * slot + e];
          const float x0 = u.x[e], x1 = v.x[e];
          u.x[e] = x0 * p.x - x1 * p.y, v.x[e] = x0 * p.y + x1 * p.x;
        }
      }
    }
    if constexpr (BACKWARD) {
      if (a.l2) {
        // dx = (dy - xh (xh . dy)) / n, xh = x / n.
        Vec8<F32> x, z;
        x.load(a.x, row_x + c0), z.load(a.x, row_x + c1);
        float ss = 0.f, sd = 0.f;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          ss += x.x[e] * x.x[e] + z.x[e] * z.x[e];
          sd += x.x[e] * u.x[e] + z.x[e] * v.x[e];
        }
        const float r = 1.f / sqrtf(row_sum(ss, lanes) + kL2Eps);
        const float m = row_sum(sd, lanes) * r * r;
#pragma unroll
        for (int e = 0; e < 8; ++e) u.x[e] = r * (u.x[e] - m * x.x[e]), v.x[e] = r * (v.x[e] - m * z.x[e]);
      }
      const size_t row = tok * a.out_stride + (size_t)h * a.d;
      u.store(a.out, row + c0), v.store(a.out, row + c1);
    } else {
      u.store(a.out, row_y + c0), v.store(a.out, row_y + c1);
    }
  }
}

}  // namespace

hipError_t launch_rope(bool f32, bool backward, const RopeArgs& a, hipStream_t stream) {
  const unsigned grid = (unsigned)(((size_t)a.B * a.L + kTokens - 1) / kTokens);
  if (backward)
    f32 ? rope_kernel<true, true><<<grid, kThreads, 0, stream>>>(a)
        : rope_kernel<false, true><<<grid, kThreads, 0, stream>>>(a);
  else
    f32 ? rope_kernel<true, false><<<grid, kThreads, 0, stream>>>(a)
        : rope_kernel<false, false><<<grid, kThreads, 0, stream>>>(a);
  return hipGetLastError();
}

}  // namespace vda
