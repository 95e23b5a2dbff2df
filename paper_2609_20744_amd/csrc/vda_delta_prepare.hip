// Token-wise gated delta rule: the sequences' tables, and what each chunk's
// products need that does not depend on the state (vda_delta.h): the
// triangular inverse T and the decayed scores P, as operand tiles, and the
// decays gam and eta.
//
// One workgroup of four waves per chunk and value head.  The scores k.k and
// q.k come from the matrix cores, the rows copied to LDS as operand tiles (with
// operands loaded straight from memory, 16 bytes of 16 rows at a time, the
// kernel took 68 us where it now takes 46: 16411 tokens, 16 heads, 128 x 128;
// backward, 16401 tokens, 102 and 54 us); wave w makes row block w.  The
// decays multiply the fp32 results.  I + L diag(beta) is unit lower triangular
// and is inverted in fp32, in LDS: its four 16 x 16 diagonal blocks by
// forward substitution (a lane per column; a series of powers would be all
// products, but its terms grow with repeated keys before they cancel), then
// the blocks below by products with the blocks already inverted,
// T21 = -T22 M21 T11, first in pairs of 16, then of 32, on the fp32 matrix
// cores.
#include "vda_delta.h"

namespace vda {
namespace {

constexpr int kLd = 68;  // floats per row of the matrix in LDS

__device__ __forceinline__ floatx4 mfma_f32(floatx4 a, floatx4 b, floatx4 c) {
#pragma unroll
  for (int e = 0; e < 4; ++e) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a[e], b[e], c, 0, 0, 0);
  return c;
}

// Operand of 16 rows of a [64][kLd] matrix: row r0 + li, columns c0 + 4 lg ..
__device__ __forceinline__ floatx4 mat_row(const float* m, int r0, int c0, int li, int lg) {
  return *reinterpret_cast<const floatx4*>(m + (r0 + li) * kLd + c0 + 4 * lg);
}
// Column c0 + li, rows r0 + 4 lg ..
__device__ __forceinline__ floatx4 mat_col(const float* m, int r0, int c0, int li, int lg) {
  floatx4 v;
#pragma unroll
  for (int e = 0; e < 4; ++e) v[e] = m[(r0 + 4 * lg + e) * kLd + c0 + li];
  return v;
}

// Inverse of the unit lower triangular I + M in place; M's strict lower part
// is in m, the rest is not read.  Leaves the 16 x 16 blocks on and below the
// diagonal (zeros above within the diagonal blocks).  256 threads.
__device__ __forceinline__ void invert_unit_lower(float* m, int wave, int li, int lg) {
  {
    const int r0 = 16 * wave;
    float x[16];
#pragma unroll
    for (int b = 0; b < 4; ++b) {
      floatx4 row[4][4];
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int c = 0; c <= b; ++c)
          row[i][c] = *reinterpret_cast<const floatx4*>(m + (r0 + 4 * b + i) * kLd + r0 + 4 * c);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        float v = li == 4 * b + i ? 1.f : 0.f;
#pragma unroll
        for (int l = 0; l < 4 * b + i; ++l) v -= row[i][l >> 2][l & 3] * x[l];
        x[4 * b + i] = v;
      }
      // Four rows at a time (the next rows are read after these are used): all
      // at once would take 120 registers.
      asm volatile("" : "+v"(x[4 * b + 3]) : : "memory");
    }
    // Every lane of the wave has read the block before it is overwritten: the
    // values above are used.
    __builtin_amdgcn_wave_barrier();
#pragma unroll
    for (int i = 0; i < 16; ++i)
      if ((i >> 2) == lg) m[(r0 + i) * kLd + r0 + li] = x[i];
  }
  lds_barrier();
  if (wave < 2) {
    const int r0 = 32 * wave + 16, c0 = 32 * wave;
    const floatx4 zero = {0.f, 0.f, 0.f, 0.f};
    const floatx4 y = mfma_f32(mat_row(m, r0, c0, li, lg), mat_col(m, c0, c0, li, lg), zero);
    const floatx4 t = mfma_f32(mat_row(m, r0, r0, li, lg), y, zero);
#pragma unroll
    for (int e = 0; e < 4; ++e) m[(r0 + 4 * lg + e) * kLd + c0 + li] = -t[e];
  }
  lds_barrier();
  const int c = wave & 1, rr = wave >> 1;
  floatx4 y[2] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
#pragma unroll
  for (int t = 0; t < 2; ++t)
#pragma unroll
    for (int b = 0; b < 2; ++b)
      if (b >= c) y[t] = mfma_f32(mat_row(m, 32 + 16 * t, 16 * b, li, lg), mat_col(m, 16 * b, 16 * c, li, lg), y[t]);
  floatx4 t = mfma_f32(mat_row(m, 32 + 16 * rr, 32, li, lg), y[0], floatx4{0.f, 0.f, 0.f, 0.f});
  if (rr == 1) t = mfma_f32(mat_row(m, 48, 48, li, lg), y[1], t);
  lds_barrier();  // every wave has read M21
#pragma unroll
  for (int e = 0; e < 4; ++e) m[(32 + 16 * rr + 4 * lg + e) * kLd + 16 * c + li] = -t[e];
  lds_barrier();
}

// x where `keep`, else 0.  The mask is opaque to the compiler, which otherwise
// jumps around the score's exponential: a score is cheaper than a jump.
__device__ __forceinline__ float keep_if(bool keep, float x) {
  uint32_t mask = keep ? 0xffffffffu : 0u;
  asm("" : "+v"(mask));
  return __uint_as_float(__float_as_uint(x) & mask);
}

// The prefixes of four tokens in a row.
struct Prefix4 {
  double x[4];
};
__device__ __forceinline__ Prefix4 prefix4(const double* pre) {
  typedef double double2v __attribute__((ext_vector_type(2)));
  const double2v a = *reinterpret_cast<const double2v*>(pre), b = *reinterpret_cast<const double2v*>(pre + 2);
  return {{a[0], a[1], b[0], b[1]}};
}

template <bool F32, int DK, bool BACKWARD>
__global__ __launch_bounds__(kThreads)
void delta_prepare_kernel(DeltaArgs a) {
  typedef Op<F32> O;
  typedef typename O::X X;
  constexpr int KS = DK / 32, ES = F32 ? 4 : 2, kTileK = kChunk * DK * ES;
  typedef RowTiles<F32, KS> Rows;
  // The matrix takes the place of q's rows, which makes four workgroups a compute unit.
  constexpr int kMatrix = kChunk * kLd * (int)sizeof(float);
  __shared__ __align__(16) char rowsK[kTileK], rowsQ[kTileK > kMatrix ? kTileK : kMatrix];
  float* const m = reinterpret_cast<float*>(rowsQ);
  __shared__ __align__(16) double pre[kChunk];
  __shared__ __align__(16) float strengths[kChunk];
  const int h = blockIdx.x % (unsigned)a.Hv;
  const int chunk = blockIdx.x / (unsigned)a.Hv;
  const ChunkInfo ci = chunk_info(a, chunk);
  if (ci.len == 0) return;
  const int tid = threadIdx.x, lane = tid & 63, li = lane & 15, lg = lane >> 4;
  const int wave = uniform(tid >> 6);
  char* rec = a.rec + ((size_t)chunk * a.Hv + h) * ChunkRecord::bytes(F32, BACKWARD);

  // The gates first: the decays are summed while the rows are on their way.
  float decay = 0.f, beta = 0.f;
  if (wave == 0 && lane < ci.len) {
    const size_t at = (size_t)(ci.tok + lane) * a.gate_tok + (size_t)h * a.gate_head;
    decay = a.g[at], beta = a.beta[at];
  }
  // The rows.  Those behind the chunk's end repeat its last: of T they reach
  // nothing (such tokens have no strength), of P rows that only the backward
  // pass reads, which are cleared there.
  const size_t qk = ((size_t)ci.tok * a.qk_tok + (size_t)(h / a.group) * a.qk_head) * ES;
  const uint32_t row_bytes = (uint32_t)a.qk_tok * ES;
  copy_tiles<F32, KS, 4>(make_rsrc((const char*)a.k + qk, 64u * row_bytes), rowsK, ci.len, row_bytes, wave, lane);
  copy_tiles<F32, KS, 4>(make_rsrc((const char*)a.q + qk, 64u * row_bytes), rowsQ, ci.len, row_bytes, wave, lane);
  const TileLane tl = tile_lane<F32, Rows::kPairs>(li, lg);
  auto row = [&](const char* rows, int t, int s) __attribute__((always_inline)) {
    return tile_row<F32>(rows + Rows::tile(s, t), Rows::odd(s), tl);
  };
  if (wave == 0) {
    const double G = decay_prefix(decay, lane);
    pre[lane] = G;
    strengths[lane] = beta;
    const double last = __shfl(G, 63);
    float* vec = reinterpret_cast<float*>(rec + ChunkRecord::kVec);
    vec[lane] = pow2(G);
    vec[64 + lane] = pow2(last - G);
    vec[128 + lane] = strengths[lane];
    if constexpr (BACKWARD) reinterpret_cast<double*>(rec + ChunkRecord::kPre)[lane] = G;
  }
  copy_barrier();

  const int r0 = 16 * wave;
  const Prefix4 gi = prefix4(pre + r0 + 4 * lg);

  // The operands of this wave's rows: of k, and in the forward pass of q.
  X kw[KS], qw[KS];
#pragma unroll
  for (int s = 0; s < KS; ++s) {
    kw[s] = row(rowsK, wave, s);
    if (!BACKWARD) qw[s] = row(rowsQ, wave, s);
  }
  // P, row block `wave`, as operand tiles: the product's rows are the columns j of P.
  if constexpr (!BACKWARD) {
    const double gq = pre[r0 + li];
    const int i = r0 + li;
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      if (32 * s > r0 + 15) continue;
      floatx4 p[2];
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        const int t = 2 * s + u;
        p[u] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int c = 0; c < KS; ++c) p[u] = O::mma(row(rowsK, t, c), qw[c], p[u]);
        const Prefix4 gj = prefix4(pre + 16 * t + 4 * lg);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int j = 16 * t + 4 * lg + e;
          p[u][e] = keep_if(i >= j, a.scale * pow2(gq - gj.x[e]) * p[u][e]);
        }
      }
      store_tile_x<F32>(rec + ChunkRecord::kP, tri_tile(wave, s), lane, O::narrow(p[0], p[1]));
    }
  } else {
    // P transposed, row block j of `wave`: the product's rows are the rows i of P.
    const int j = r0 + li;
    const double gj = pre[j];
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      if (32 * s + 31 < r0) continue;
      floatx4 p[2];
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        const int t = 2 * s + u;
        p[u] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int c = 0; c < KS; ++c) p[u] = O::mma(row(rowsQ, t, c), kw[c], p[u]);
        const Prefix4 gi = prefix4(pre + 16 * t + 4 * lg);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int i = 16 * t + 4 * lg + e;
          p[u][e] = keep_if(i >= j && i < ci.len, a.scale * pow2(gi.x[e] - gj) * p[u][e]);
        }
      }
      store_tile_w<F32>(rec + ChunkRecord::kPt, tri_tile_t(wave, s), lane, O::wide(p[0], p[1]));
    }
  }
  lds_barrier();  // every wave is done with q

  // M = L diag(beta), rows of this wave.
#pragma unroll
  for (int t = 0; t < 4; ++t) {
    if (t > wave) continue;
    floatx4 acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int s = 0; s < KS; ++s) acc = O::mma(kw[s], row(rowsK, t, s), acc);
    const int j = 16 * t + li;
    const double gj = pre[j];
    const float bj = strengths[j];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int i = r0 + 4 * lg + e;
      m[i * kLd + j] = keep_if(i > j, bj * pow2(gi.x[e] - gj) * acc[e]);
    }
  }
  lds_barrier();
  invert_unit_lower(m, wave, li, lg);

  // T, row block `wave`.
#pragma unroll
  for (int s = 0; s < 2; ++s) {
    if (32 * s > r0 + 15) continue;
    floatx4 x[2];
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const int t = 2 * s + u;
      x[u] = floatx4{0.f, 0.f, 0.f, 0.f};
      if (t <= wave) x[u] = mat_row(m, r0, 16 * t, li, lg);
    }
    store_tile_w<F32>(rec + ChunkRecord::kT, tri_tile(wave, s), lane, O::wide(x[0], x[1]));
  }
  if constexpr (BACKWARD) {
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      if (32 * s + 31 < r0) continue;
      floatx4 x[2];
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        const int t = 2 * s + u;
        x[u] = floatx4{0.f, 0.f, 0.f, 0.f};
        if (t >= wave) x[u] = mat_col(m, 16 * t, r0, li, lg);
      }
      store_tile_w<F32>(rec + ChunkRecord::kTt, tri_tile_t(wave, s), lane, O::wide(x[0], x[1]));
    }
  }
}

// Tables of the chunks and segments of sequences [cu[i], cu[i + 1]): tabs
// holds counts[2] (and padding to 4), prefix sums of chunks and segments
// [n + 1] each, then the int4 tables and the segments' numbers.  Offsets are
// clamped to [0, T] and the tables to their sizes, and sums stop at kMost,
// above any table's size, so that no malformed list can address anything else.
//
// Segments are listed the longest first, by classes of 1/32 of the greatest
// length (in any order within one: each is scanned by itself): the device then
// ends with short ones.  9 uneven sequences of 16401 tokens with 16 heads,
// backward: 910 us in the sequences' order, 887 us in this one.
constexpr int kPlanThreads = 1024, kMost = 0x3fffffff, kClasses = 32;

__global__ __launch_bounds__(kPlanThreads) void delta_plan_kernel(const int* cu, int n, int T, int seg_chunks,
                                                                 int whole, int max_chunks, int max_segs,
                                                                 int* tabs) {
  __shared__ int pre[2][kPlanThreads], ends[2][kPlanThreads / 64], at_class[kClasses];
  int* counts = tabs;
  int* cpre = tabs + 4;
  int* spre = cpre + n + 1;
  int4* chunk_tab = reinterpret_cast<int4*>(tabs + (4 + 2 * (n + 1) + 3) / 4 * 4);
  int4* seg_tab = chunk_tab + max_chunks;
  int* seg_id = reinterpret_cast<int*>(seg_tab + max_segs);
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const bool small = n <= kPlanThreads;  // the prefixes are in LDS as well
  auto clamp = [&](int x) { return x < 0 ? 0 : x > T ? T : x; };
  auto add = [](int x, int y) { return x + y < kMost ? x + y : kMost; };
  if (tid < kClasses) at_class[tid] = 0;
  int base[2] = {0, 0};
  for (int at = 0; at < n; at += kPlanThreads) {
    const int i = at + tid;
    int x[2] = {0, 0};  // chunks, segments
    if (i < n) {
      const int len = clamp(cu[i + 1]) - clamp(cu[i]);
      x[0] = len > 0 ? chunks_of(len) : 0;
      x[1] = x[0] > whole ? (x[0] + seg_chunks - 1) / seg_chunks : 1;
    }
#pragma unroll
    for (int w = 0; w < 2; ++w) {
#pragma unroll
      for (int d = 1; d < 64; d <<= 1) {
        const int y = __shfl_up(x[w], d);
        if (lane >= d) x[w] = add(x[w], y);
      }
      if (lane == 63) ends[w][wave] = x[w];
    }
    __syncthreads();
#pragma unroll
    for (int w = 0; w < 2; ++w) {
      int before = base[w];
      for (int v = 0; v < kPlanThreads / 64; ++v) {
        const int y = ends[w][v];
        if (v < wave) before = add(before, y);
        base[w] = add(base[w], y);
      }
      const int mine = __shfl_up(x[w], 1);
      before = add(before, lane ? mine : 0);
      if (i < n) (w ? spre : cpre)[i] = before;
      if (small) pre[w][tid] = before;
    }
    __syncthreads();
  }
  const int nc = base[0] < max_chunks ? base[0] : max_chunks, ns = base[1] < max_segs ? base[1] : max_segs;
  if (tid == 0) {
    cpre[n] = base[0], spre[n] = base[1];
    counts[0] = nc, counts[1] = ns;
  }
  __threadfence_block();
  __syncthreads();
  auto prefix = [&](int w, int i) { return i == n ? base[w] : small ? pre[w][i] : (w ? spre : cpre)[i]; };
  // The sequence that entry x belongs to: the last whose prefix is <= x.
  auto find = [&](int w, int x) {
    int lo = 0, hi = n - 1;
    while (lo < hi) {
      const int mid = (lo + hi + 1) >> 1;
      if (prefix(w, mid) <= x) lo = mid; else hi = mid - 1;
    }
    return lo;
  };
  for (int c = tid; c < nc; c += kPlanThreads) {
    const int seq = find(0, c);
    const int b = clamp(cu[seq]), len = clamp(cu[seq + 1]) - b, at = (c - prefix(0, seq)) * kChunk;
    chunk_tab[c] = make_int4(b + at, len - at < kChunk ? len - at : kChunk, seq, 0);
  }
  auto segment = [&](int s) {
    const int seq = find(1, s);
    const int at = s - prefix(1, seq), first = prefix(0, seq) + at * seg_chunks, from = at * seg_chunks * kChunk;
    const int b = clamp(cu[seq]);
    int len = clamp(cu[seq + 1]) - b - from;
    if (prefix(1, seq + 1) - prefix(1, seq) > 1 && len > seg_chunks * kChunk) len = seg_chunks * kChunk;
    const int room = nc > first ? nc - first : 0;  // offsets that decrease: the table of chunks ends
    if (len > room * kChunk) len = room * kChunk;
    const bool last = s + 1 >= prefix(1, seq + 1);
    return make_int4(first, b + from, len > 0 ? len : 0, seq << 2 | (at == 0 ? 1 : 0) | (last ? 2 : 0));
  };
  auto cls = [&](int len) {
    const int c = chunks_of(len);
    return kClasses - 1 - (c < whole ? c : whole) * kClasses / (whole + 1);
  };
  int4 mine = make_int4(0, 0, 0, 0);
  if (tid < ns) mine = segment(tid);
  for (int s = tid; s < ns; s += kPlanThreads) atomicAdd(&at_class[cls(s == tid ? mine.z : segment(s).z)], 1);
  __syncthreads();
  if (wave == 0) {
    int x = lane < kClasses ? at_class[lane] : 0;
    const int count = x;
    for (int d = 1; d < kClasses; d <<= 1) {
      const int y = __shfl_up(x, d);
      if (lane >= d) x += y;
    }
    if (lane < kClasses) at_class[lane] = x - count;
  }
  __syncthreads();
  for (int s = tid; s < ns; s += kPlanThreads) {
    const int4 e = s == tid ? mine : segment(s);
    const int to = atomicAdd(&at_class[cls(e.z)], 1);
    seg_tab[to] = e, seg_id[to] = s;
  }
}

template <bool F32, int DK>
hipError_t run(bool backward, const DeltaArgs& a, hipStream_t stream) {
  const unsigned grid = (unsigned)a.max_chunks * (unsigned)a.Hv;
  if (backward)
    delta_prepare_kernel<F32, DK, true><<<grid, kThreads, 0, stream>>>(a);
  else
    delta_prepare_kernel<F32, DK, false><<<grid, kThreads, 0, stream>>>(a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_delta_plan(const int* cu, int n_seqs, int T, const DeltaPlan& plan, int* tabs,
                             hipStream_t stream) {
  delta_plan_kernel<<<1, kPlanThreads, 0, stream>>>(cu, n_seqs, T, plan.seg_chunks, plan.whole, plan.max_chunks,
                                                    plan.max_segs, tabs);
  return hipGetLastError();
}

hipError_t launch_delta_prepare(bool f32, int d_k, bool backward, const DeltaArgs& a, hipStream_t stream) {
  switch (d_k) {
    case 32: return f32 ? run<true, 32>(backward, a, stream) : run<false, 32>(backward, a, stream);
    case 64: return f32 ? run<true, 64>(backward, a, stream) : run<false, 64>(backward, a, stream);
    default: return f32 ? run<true, 128>(backward, a, stream) : run<false, 128>(backward, a, stream);
  }
}

}  // namespace vda
