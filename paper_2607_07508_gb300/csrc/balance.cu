// Load-balance loss of a mixture of experts, with per-expert counts and gradients.
//
// Scores of token t: s_te = softmax(x_t)_e, or sigmoid(x_te) / sum_j sigmoid(x_tj). Over
// the n counted rows of a segment (the batch, or one packed trajectory), with k experts
// chosen per token:
//   c_e = how often e was chosen, P_e = sum_t s_te
//   loss = E / (k n^2) sum_e c_e P_e                (1 when both are even)
// and the mean of it over the segments that have a counted row. c is not
// differentiated, so with w_e = g E c_e / (k n^2 segments):
//   d x_te = s_te (w_e - sum_j s_tj w_j)            (sigmoid: times 1 - sigmoid(x_te))
//
// Rows are cut into chunks of equal size whatever the trajectories. A chunk writes one
// partial for each segment that it meets, at slot chunk + segment (along the batch
// either number grows, so the slots differ), and a segment's partials are added in the
// order of its chunks: no atomics on floating-point sums, the same bits every time.
#include <cuda_bf16.h>
#include <math.h>
#include <stdint.h>

#include "balance.cuh"
#include "sao_common.cuh"
#include "sao_internal.h"

namespace sao {
namespace {

constexpr int kThreads = 256, kWarps = kThreads / 32;
constexpr int kSlices = kThreads / 32;  // slices of a segment's partials that a CTA of the reduction adds side by side

struct BalanceArgs {
  const void *x;
  const int32_t *ids;
  const uint8_t *mask;   // or null
  const int32_t *cu;     // or null: one segment
  int B;
  int64_t N;
  int E, k;
  int chunk;             // rows per chunk
  int chunks;
  unsigned int *err;
};

template <class T>
__device__ __forceinline__ float to_float(T v) {
  return float(v);
}
__device__ __forceinline__ float to_float(__nv_bfloat16 v) { return __bfloat162float(v); }
template <class T>
__device__ __forceinline__ T from_float(float v) {
  return T(v);
}
template <>
__device__ __forceinline__ __nv_bfloat16 from_float<__nv_bfloat16>(float v) {
  return __float2bfloat16_rn(v);
}

// Segment b's first row and the row after its last, inside [0, N] whatever cu holds.
__device__ __forceinline__ int64_t seg_at(const BalanceArgs &a, int b) {
  if (a.cu == nullptr) return b == 0 ? 0 : a.N;
  const int64_t v = ld(a.cu + b);
  return v < 0 ? 0 : v > a.N ? a.N : v;
}
// The segment that holds row r: the last one that starts at or before it.
__device__ __forceinline__ int seg_of(const BalanceArgs &a, int64_t r) {
  int lo = 0, hi = a.B - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (seg_at(a, mid) <= r)
      lo = mid;
    else
      hi = mid - 1;
  }
  return lo;
}
__device__ __forceinline__ float warp_max(float v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, o));
  return v;
}
__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}

// A row of -inf alone has no probabilities.
__device__ __forceinline__ float inverse(float sum) { return sum == 0.f ? 0.f : 1.f / sum; }
// A row's scores up to a factor, which the normalisation takes out: exp(x - max), or
// sigmoid(x), divided by exp(max) where max is below 0 (e^x / (1 + e^x) would vanish with it).
template <bool kSigmoid>
__device__ __forceinline__ float shift(float max) {
  if (max == -INFINITY) return 0.f;
  return kSigmoid ? fminf(max, 0.f) : max;
}
template <bool kSigmoid>
__device__ __forceinline__ float score(float x, float m) {
  if constexpr (!kSigmoid) return expf(x - m);
  return x > 0.f ? 1.f / (1.f + expf(-x)) : expf(x - m) / (1.f + expf(x));
}

// Runs f(segment, first row, row after the last) for the segments of chunk c (all threads).
template <class F>
__device__ __forceinline__ void for_segments(const BalanceArgs &a, int c, F f) {
  int64_t r = int64_t(c) * a.chunk;
  const int64_t end = r + a.chunk < a.N ? r + a.chunk : a.N;
  for (int b = seg_of(a, r); b < a.B && r < end; ++b) {
    int64_t e = seg_at(a, b + 1);
    e = e < end ? e : end;
    if (e <= r) continue;
    f(b, r, e);
    r = e;
  }
}

// A warp per row; each warp adds its rows' scores in its own shared-memory columns.
template <class T, bool kSigmoid>
__global__ void __launch_bounds__(kThreads)
    balance_partial_kernel(const BalanceArgs a, float *psum, int *pcount, int *prows, unsigned int *ticket) {
  extern __shared__ float sums[];  // [kWarps][E], then the counts [E]
  __shared__ int n_rows[kWarps];
  grid_wait();
  if (blockIdx.x == 0 && threadIdx.x == 0) *ticket = 0;
  int *counts = reinterpret_cast<int *>(sums + kWarps * a.E);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  float *mine = sums + warp * a.E;
  const T *x = static_cast<const T *>(a.x);
  for_segments(a, blockIdx.x, [&](int b, int64_t r0, int64_t r1) {
    for (int e = threadIdx.x; e < a.E; e += kThreads) counts[e] = 0;
    for (int e = lane; e < a.E; e += 32) mine[e] = 0.f;
    __syncthreads();
    int n = 0;
    for (int64_t r = r0 + warp; r < r1; r += kWarps) {
      if (a.mask && a.mask[r] == 0) continue;
      ++n;
      const T *row = x + r * a.E;
      float m = -INFINITY;
      for (int e = lane; e < a.E; e += 32) m = fmaxf(m, to_float(ld(row + e)));
      m = shift<kSigmoid>(warp_max(m));
      float s = 0.f;
      for (int e = lane; e < a.E; e += 32) {
        const float v = to_float(ld(row + e));
        s += score<kSigmoid>(v, m);
      }
      s = inverse(warp_sum(s));
      for (int e = lane; e < a.E; e += 32) {
        const float v = to_float(ld(row + e));
        mine[e] += s * score<kSigmoid>(v, m);
      }
      for (int j = lane; j < a.k; j += 32) {
        const int id = ld(a.ids + r * a.k + j);
        if (id >= 0 && id < a.E)
          atomicAdd(counts + id, 1);
        else if (id >= a.E)
          raise_device_error(a.err, SAO_DEVERR_EXPERT_ID);
      }
    }
    if (lane == 0) n_rows[warp] = n;
    __syncthreads();
    const int64_t slot = int64_t(blockIdx.x) + b;
    for (int e = threadIdx.x; e < a.E; e += kThreads) {
      float v = 0.f;
      for (int w = 0; w < kWarps; ++w) v += sums[w * a.E + e];
      psum[slot * a.E + e] = v;
      pcount[slot * a.E + e] = counts[e];
    }
    if (threadIdx.x == 0) {
      int t = 0;
      for (int w = 0; w < kWarps; ++w) t += n_rows[w];
      prows[slot] = t;
    }
    __syncthreads();
  });
}

// CTA (b, 32 columns): adds the segment's partials, kSlices of them side by side; the
// last CTA adds the products of all of them.
__global__ void __launch_bounds__(kThreads)
    balance_reduce_kernel(const BalanceArgs a, const float *psum, const int *pcount, const int *prows, float *loss,
                          int64_t *counts, float *prob_sums, int64_t *rows, double *terms, unsigned int *ticket) {
  __shared__ float sh_sum[kSlices][32];
  __shared__ long long sh_count[kSlices][32];
  __shared__ long long sh_rows[kSlices];
  __shared__ double sh_term[kThreads];
  __shared__ int sh_used[kThreads];
  __shared__ bool last;
  grid_wait();
  const int cols = (a.E + 31) / 32;
  const int b = blockIdx.x / cols, g = blockIdx.x % cols;
  const int slice = threadIdx.x >> 5, lane = threadIdx.x & 31, e = g * 32 + lane;
  const int64_t r0 = seg_at(a, b), r1 = seg_at(a, b + 1);
  float s = 0.f;
  long long n = 0, nr = 0;
  if (r1 > r0) {
    const int c1 = int((r1 - 1) / a.chunk);
    for (int c = int(r0 / a.chunk) + slice; c <= c1; c += kSlices) {
      const int64_t slot = int64_t(c) + b;
      if (e < a.E) {
        s += ld(psum + slot * a.E + e);
        n += ld(pcount + slot * a.E + e);
      }
      nr += ld(prows + slot);
    }
  }
  sh_sum[slice][lane] = s;
  sh_count[slice][lane] = n;
  if (lane == 0) sh_rows[slice] = nr;
  __syncthreads();
  if (slice == 0) {
    s = 0.f;
    n = nr = 0;
    for (int k = 0; k < kSlices; ++k) {
      s += sh_sum[k][lane];
      n += sh_count[k][lane];
      nr += sh_rows[k];
    }
    double term = 0.0;
    if (e < a.E) {
      prob_sums[int64_t(b) * a.E + e] = s;
      counts[int64_t(b) * a.E + e] = n;
      term = nr > 0 ? double(s) * double(n) * (double(a.E) / (double(a.k) * double(nr) * double(nr))) : 0.0;
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) term += __shfl_xor_sync(0xffffffffu, term, o);
    if (lane == 0) {
      terms[blockIdx.x] = term;
      if (g == 0) rows[b] = nr;
      // checked mode: cu_seqlens runs from 0 to N and never falls
      if (a.cu && g == 0) {
        const int64_t u = ld(a.cu + b), v = ld(a.cu + b + 1);
        if (u > v || (b == 0 && u != 0) || (b == a.B - 1 && v != a.N)) raise_device_error(a.err, SAO_DEVERR_CU_SEQLENS);
      }
      __threadfence();
      last = atomicAdd(ticket, 1u) == gridDim.x - 1;
    }
  }
  __syncthreads();
  if (!last) return;
  __threadfence();
  double t = 0.0;
  int used = 0;
  for (int64_t i = threadIdx.x; i < gridDim.x; i += kThreads) t += __ldcg(terms + i);
  for (int i = threadIdx.x; i < a.B; i += kThreads) used += __ldcg(rows + i) > 0;
  sh_term[threadIdx.x] = t;
  sh_used[threadIdx.x] = used;
  __syncthreads();
  for (int o = kThreads / 2; o > 0; o >>= 1) {
    if (threadIdx.x < o) {
      sh_term[threadIdx.x] += sh_term[threadIdx.x + o];
      sh_used[threadIdx.x] += sh_used[threadIdx.x + o];
    }
    __syncthreads();
  }
  if (threadIdx.x == 0) loss[0] = sh_used[0] ? float(sh_term[0] / double(sh_used[0])) : 0.f;
}

template <class T, bool kSigmoid>
__global__ void __launch_bounds__(kThreads)
    balance_grad_kernel(const BalanceArgs a, const int64_t *counts, const int64_t *rows, const float *grad_loss,
                        T *dx) {
  extern __shared__ float w[];  // [E]
  __shared__ int sh_used[kWarps];
  grid_wait();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  int used = 0;
  for (int i = threadIdx.x; i < a.B; i += kThreads) used += ld(rows + i) > 0;
  used = __reduce_add_sync(0xffffffffu, used);
  if (lane == 0) sh_used[warp] = used;
  __syncthreads();
  used = 0;
  for (int i = 0; i < kWarps; ++i) used += sh_used[i];
  const T *x = static_cast<const T *>(a.x);
  const float g = ld(grad_loss);
  for_segments(a, blockIdx.x, [&](int b, int64_t r0, int64_t r1) {
    const float n = float(ld(rows + b));
    const float f = n > 0.f ? g * float(a.E) / (float(a.k) * n * n * float(used)) : 0.f;
    for (int e = threadIdx.x; e < a.E; e += kThreads) w[e] = f * float(ld(counts + int64_t(b) * a.E + e));
    __syncthreads();
    for (int64_t r = r0 + warp; r < r1; r += kWarps) {
      T *out = dx + r * a.E;
      if (a.mask && a.mask[r] == 0) {
        for (int e = lane; e < a.E; e += 32) out[e] = from_float<T>(0.f);
        continue;
      }
      const T *row = x + r * a.E;
      float m = -INFINITY;
      for (int e = lane; e < a.E; e += 32) m = fmaxf(m, to_float(ld(row + e)));
      m = shift<kSigmoid>(warp_max(m));
      float s = 0.f, d = 0.f;
      for (int e = lane; e < a.E; e += 32) {
        const float v = to_float(ld(row + e));
        const float q = score<kSigmoid>(v, m);
        s += q;
        d += q * w[e];
      }
      s = inverse(warp_sum(s));
      d = warp_sum(d) * s;
      for (int e = lane; e < a.E; e += 32) {
        const float v = to_float(ld(row + e));
        const float q = score<kSigmoid>(v, m);
        const float slope = kSigmoid ? q * s / (1.f + expf(v)) : q * s;
        out[e] = from_float<T>(slope * (w[e] - d));
      }
    }
    __syncthreads();
  });
}

int chunk_rows(int64_t N) {
  int64_t c = (N + 303) / 304;  // two CTAs per SM
  return int(c < 32 ? 32 : c);
}
BalanceArgs make_args(const void *x, const int32_t *ids, const uint8_t *mask, const int32_t *cu, int32_t B, int64_t N,
                      int32_t E, int32_t k, unsigned int *err) {
  BalanceArgs a{x, ids, mask, cu, cu ? B : 1, N, E, k, chunk_rows(N), 0, err};
  a.chunks = int((N + a.chunk - 1) / a.chunk);
  return a;
}

struct Scratch {
  float *psum;
  int *pcount, *prows;
  double *terms;
  unsigned int *ticket;
};
Scratch take(Carver &c, int64_t N, int32_t E, int32_t B) {
  const int64_t chunk = chunk_rows(N);
  const size_t slots = size_t((N + chunk - 1) / chunk) + size_t(B);
  Scratch s;
  s.psum = c.take<float>(slots * size_t(E));
  s.pcount = c.take<int>(slots * size_t(E));
  s.prows = c.take<int>(slots);
  s.terms = c.take<double>(size_t(B) * size_t((E + 31) / 32));
  s.ticket = c.take<unsigned int>(1);
  return s;
}

}  // namespace

size_t balance_ws_bytes(int64_t N, int32_t E, int32_t B) {
  Carver c(nullptr, ~size_t(0));
  take(c, N, E, B);
  return c.off;
}

sao_status balance_fwd_launch(const void *x, sao_dtype dt, const int32_t *ids, const uint8_t *mask, const int32_t *cu,
                              int32_t B, int64_t N, int32_t E, int32_t k, int score, float *loss, int64_t *counts,
                              float *prob_sums, int64_t *rows, unsigned int *err, void *ws, size_t ws_bytes,
                              cudaStream_t s) {
  const BalanceArgs a = make_args(x, ids, mask, cu, B, N, E, k, err);
  Carver c(ws, ws_bytes);
  const Scratch w = take(c, N, E, a.B);
  if (!c.ok()) return fail(SAO_ERR_WORKSPACE, "workspace too small for the balance loss");
  auto kern = dt == SAO_BF16
                  ? (score == SAO_SCORE_SIGMOID ? balance_partial_kernel<__nv_bfloat16, true>
                                                : balance_partial_kernel<__nv_bfloat16, false>)
                  : (score == SAO_SCORE_SIGMOID ? balance_partial_kernel<float, true> : balance_partial_kernel<float, false>);
  int slot = launch_begin("balance_partial", s);
  pdl(kern, unsigned(a.chunks), kThreads, size_t(E) * (kWarps + 1) * sizeof(float), s)(a, w.psum, w.pcount, w.prows,
                                                                                      w.ticket);
  SAO_TRY(launch_end(slot, s));
  slot = launch_begin("balance_reduce", s);
  pdl(balance_reduce_kernel, unsigned(a.B) * unsigned((E + 31) / 32), kThreads, 0, s)(
      a, w.psum, w.pcount, w.prows, loss, counts, prob_sums, rows, w.terms, w.ticket);
  return launch_end(slot, s);
}

sao_status balance_bwd_launch(const void *x, sao_dtype dt, const uint8_t *mask, const int32_t *cu, int32_t B, int64_t N,
                              int32_t E, int32_t k, int score, const int64_t *counts, const int64_t *rows,
                              const float *grad_loss, void *dx, unsigned int *err, cudaStream_t s) {
  const BalanceArgs a = make_args(x, nullptr, mask, cu, B, N, E, k, err);
  int slot = launch_begin("balance_grad", s);
  const size_t smem = size_t(E) * sizeof(float);
  if (dt == SAO_BF16)
    pdl(score == SAO_SCORE_SIGMOID ? balance_grad_kernel<__nv_bfloat16, true> : balance_grad_kernel<__nv_bfloat16, false>,
        unsigned(a.chunks), kThreads, smem, s)(a, counts, rows, grad_loss, static_cast<__nv_bfloat16 *>(dx));
  else
    pdl(score == SAO_SCORE_SIGMOID ? balance_grad_kernel<float, true> : balance_grad_kernel<float, false>,
        unsigned(a.chunks), kThreads, smem, s)(a, counts, rows, grad_loss, static_cast<float *>(dx));
  return launch_end(slot, s);
}

}  // namespace sao
