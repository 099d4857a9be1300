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

#include <type_traits>

#include "balance.cuh"
#include "sao_common.cuh"
#include "sao_internal.h"
#include "tc_ptx.cuh"

namespace sao {
namespace {

constexpr int kThreads = 256, kWarps = kThreads / 32;
constexpr float kLog2e = 1.4426950408889634f;

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

// How a row lies over `lanes` (a power of two) consecutive lanes, kC columns each: kVec
// columns (16 bytes, or one) per load, lane l holding loads l, l + lanes, ... Columns
// past E, and all of a row that is not counted, read as -inf: they have no score.
template <class T, int kVec, int kC>
struct Row {
  static constexpr int kLoads = kC / kVec;
  static constexpr int kWords = kVec == 1 ? kLoads : kLoads * 4;
  uint32_t raw[kWords];
  __device__ __forceinline__ void load(const T *row, int E, int l, int lanes, bool live) {
#pragma unroll
    for (int v = 0; v < kLoads; ++v) {
      const int c = (l + v * lanes) * kVec;
      if constexpr (kVec == 1) {
        constexpr uint32_t none = sizeof(T) == 2 ? 0xff80u : 0xff800000u;  // -inf
        raw[v] = none;
        if (live && c < E) {
          if constexpr (sizeof(T) == 2)
            raw[v] = ld(reinterpret_cast<const uint16_t *>(row) + c);
          else
            raw[v] = ld(reinterpret_cast<const uint32_t *>(row) + c);
        }
      } else {
        constexpr uint32_t none = sizeof(T) == 2 ? 0xff80ff80u : 0xff800000u;
        uint4 x = make_uint4(none, none, none, none);
        if (live && c < E) x = ld(reinterpret_cast<const uint4 *>(row + c));
        raw[4 * v] = x.x;
        raw[4 * v + 1] = x.y;
        raw[4 * v + 2] = x.z;
        raw[4 * v + 3] = x.w;
      }
    }
  }
  __device__ __forceinline__ float at(int j) const {
    if constexpr (sizeof(T) == 4) return __uint_as_float(raw[j]);
    if constexpr (kVec == 1) return __uint_as_float(raw[j] << 16);
    return __uint_as_float(j & 1 ? raw[j / 2] & 0xffff0000u : raw[j / 2] << 16);
  }
  static __device__ __forceinline__ int column(int j, int l, int lanes) {
    return (l + j / kVec * lanes) * kVec + j % kVec;
  }
  static __device__ __forceinline__ void store(T *row, const float (&v)[kC], int E, int l, int lanes) {
#pragma unroll
    for (int k = 0; k < kLoads; ++k) {
      const int c = (l + k * lanes) * kVec;
      if (c >= E) continue;
      if constexpr (kVec == 1) {
        if constexpr (sizeof(T) == 2)
          row[c] = __float2bfloat16_rn(v[k]);
        else
          row[c] = v[k];
      } else if constexpr (sizeof(T) == 4) {
        *reinterpret_cast<float4 *>(row + c) = make_float4(v[4 * k], v[4 * k + 1], v[4 * k + 2], v[4 * k + 3]);
      } else {
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const __nv_bfloat162 b = __floats2bfloat162_rn(v[8 * k + 2 * i], v[8 * k + 2 * i + 1]);
          w[i] = *reinterpret_cast<const uint32_t *>(&b);
        }
        *reinterpret_cast<uint4 *>(row + c) = make_uint4(w[0], w[1], w[2], w[3]);
      }
    }
  }
};

__device__ __forceinline__ float lanes_max(float v, int lanes) {
  for (int o = 1; o < lanes; o <<= 1) v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, o));
  return v;
}
__device__ __forceinline__ float lanes_sum(float v, int lanes) {
  for (int o = 1; o < lanes; o <<= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}

// A row's scores q, up to a factor that the normalisation takes out, and 1 / their sum
// (0 for a row of -inf alone, which has no probabilities). Softmax: e^(x - max). Sigmoid:
// e^-m sigmoid(x) = 1 / (e^m + e^(m - x)) with m = min(max, 0): sigmoid(x) itself, but
// for rows far below 0, whose sigmoids vanish. em: e^m. (The difference is taken before
// it is scaled, so an exponent is off by 2^-24 of itself.)
template <bool kSigmoid, class R, int kC>
__device__ __forceinline__ float row_scores(const R &x, float (&q)[kC], int lanes, float &em) {
  float m4[4];
#pragma unroll
  for (int j = 0; j < kC; ++j) m4[j & 3] = j < 4 ? x.at(j) : fmaxf(m4[j & 3], x.at(j));
  float m = lanes_max(fmaxf(fmaxf(m4[0], m4[1]), fmaxf(m4[2], m4[3])), lanes);
  if (m == -INFINITY) m = 0.f;
  if constexpr (kSigmoid) {
    m = fminf(m, 0.f);
    em = tc::ex2_approx(m * kLog2e);
  }
  // two columns per fp32 operation
  const tc::f32x2 neg = tc::pack_f32x2(-m, -m), scale = tc::pack_f32x2(kSigmoid ? -kLog2e : kLog2e, kSigmoid ? -kLog2e : kLog2e);
  tc::f32x2 s2[2] = {0, 0};
#pragma unroll
  for (int j = 0; j < kC; j += 2) {
    float t0, t1;
    tc::unpack_f32x2(tc::mul_f32x2(tc::add_f32x2(tc::pack_f32x2(x.at(j), x.at(j + 1)), neg), scale), t0, t1);
    q[j] = tc::ex2_approx(t0);
    q[j + 1] = tc::ex2_approx(t1);
    if constexpr (kSigmoid) {
      q[j] = __fdividef(1.f, em + q[j]);
      q[j + 1] = __fdividef(1.f, em + q[j + 1]);
    }
    s2[j / 2 & 1] = tc::add_f32x2(s2[j / 2 & 1], tc::pack_f32x2(q[j], q[j + 1]));
  }
  float s, s1;
  tc::unpack_f32x2(tc::add_f32x2(s2[0], s2[1]), s, s1);
  s = lanes_sum(s + s1, lanes);
  return s == 0.f ? 0.f : 1.f / s;
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

// CTAs that an SM holds: as many registers as a lane's columns, the next row's and their sums take.
template <class T, int kC>
constexpr int kCtas = kC <= 8 ? 4 : (kC <= 16 || (kC <= 24 && sizeof(T) == 2)) ? 3 : 2;

// Each group of `lanes` lanes takes a row at a time, the next one's logits in flight,
// and keeps the sums of its columns in registers. One pass over the logits: bound by
// reading them.
template <class T, int kVec, int kC, bool kSigmoid>
__global__ void __launch_bounds__(kThreads, kCtas<T, kC>)
    balance_partial_kernel(const BalanceArgs a, int lanes, float *psum, int *pcount, int *prows, unsigned int *ticket) {
  extern __shared__ float sums[];  // [kWarps][E], then the counts [E]
  __shared__ int n_rows[kWarps];
  grid_wait();
  if (blockIdx.x == 0 && threadIdx.x == 0) *ticket = 0;
  int *counts = reinterpret_cast<int *>(sums + kWarps * a.E);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int groups = 32 / lanes, l = lane & (lanes - 1), step = kWarps * groups;
  const T *x = static_cast<const T *>(a.x);
  for_segments(a, blockIdx.x, [&](int b, int64_t r0, int64_t r1) {
    for (int e = threadIdx.x; e < a.E; e += kThreads) counts[e] = 0;
    __syncthreads();
    float acc[kC];
#pragma unroll
    for (int j = 0; j < kC; ++j) acc[j] = 0.f;
    int n = 0;
    auto counted = [&](int64_t r) { return r < r1 && (a.mask == nullptr || ld(a.mask + r) != 0); };
    int64_t r = r0 + warp * groups + lane / lanes;
    Row<T, kVec, kC> next;
    bool next_on = counted(r);
    next.load(x + r * a.E, a.E, l, lanes, next_on);
    bool after_on = counted(r + step);
    auto first_id = [&](int64_t row, bool on) { return on && l < a.k ? ld(a.ids + row * a.k + l) : -1; };
    auto count = [&](int id) {
      if (id >= 0 && id < a.E)
        atomicAdd(counts + id, 1);
      else if (id >= a.E)
        raise_device_error(a.err, SAO_DEVERR_EXPERT_ID);
    };
    int next_id = first_id(r, next_on);
    for (int64_t base = r0 + warp * groups; base < r1; base += step, r += step) {  // the warp's lanes stay together
      const Row<T, kVec, kC> row = next;
      const bool on = next_on;
      const int id = next_id;
      next_on = after_on;
      next.load(x + (r + step) * a.E, a.E, l, lanes, next_on);
      next_id = first_id(r + step, next_on);
      after_on = counted(r + 2 * step);
      if (!__any_sync(0xffffffffu, on)) continue;  // spans of masked rows
      if (on) {
        if (l == 0) ++n;
        count(id);
        for (int j = l + lanes; j < a.k; j += lanes) count(ld(a.ids + r * a.k + j));
      }
      float q[kC], em;
      const float inv = row_scores<kSigmoid>(row, q, lanes, em);
      const tc::f32x2 inv2 = tc::pack_f32x2(inv, inv);
#pragma unroll
      for (int j = 0; j < kC; j += 2)
        tc::unpack_f32x2(tc::fma_f32x2(tc::pack_f32x2(q[j], q[j + 1]), inv2, tc::pack_f32x2(acc[j], acc[j + 1])), acc[j],
                         acc[j + 1]);
    }
    for (int o = lanes; o < 32; o <<= 1) {  // the warp's groups
#pragma unroll
      for (int j = 0; j < kC; ++j) acc[j] += __shfl_xor_sync(0xffffffffu, acc[j], o);
    }
    if (lane < lanes) {
#pragma unroll
      for (int j = 0; j < kC; ++j) {
        const int c = Row<T, kVec, kC>::column(j, l, lanes);
        if (c < a.E) sums[warp * a.E + c] = acc[j];
      }
    }
    n = __reduce_add_sync(0xffffffffu, n);
    if (lane == 0) n_rows[warp] = n;
    __syncthreads();
    const int64_t slot = int64_t(blockIdx.x) + b;
    for (int e = threadIdx.x; e < a.E; e += kThreads) {
      float v = 0.f;
#pragma unroll
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

// CTA (b, 32 columns): adds the segment's partials, kSlices warps side by side;
// the last CTA adds the products of all of them.
template <int kSlices>
__global__ void __launch_bounds__(32 * kSlices)
    balance_reduce_kernel(const BalanceArgs a, const float *psum, const int *pcount, const int *prows, float *loss,
                          int64_t *counts, float *prob_sums, int64_t *rows, double *terms, unsigned int *ticket) {
  __shared__ float sh_sum[kSlices][32];
  __shared__ long long sh_count[kSlices][32];
  __shared__ long long sh_rows[kSlices];
  __shared__ double sh_term[kSlices];
  __shared__ int sh_used[kSlices];
  __shared__ bool last;
  grid_wait();
  const int cols = (a.E + 31) / 32;
  const int b = blockIdx.x / cols, g = blockIdx.x % cols;
  const int slice = threadIdx.x >> 5, lane = threadIdx.x & 31, e = g * 32 + lane;
  const int64_t r0 = seg_at(a, b), r1 = seg_at(a, b + 1);
  float s = 0.f;
  long long n = 0, nr = 0;
  if (r1 > r0) {
    const int c0 = int(r0 / a.chunk), c1 = int((r1 - 1) / a.chunk);
#pragma unroll 4
    for (int c = c0 + slice; c <= c1; c += kSlices) {
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
  for (int64_t i = threadIdx.x; i < gridDim.x; i += 32 * kSlices) t += __ldcg(terms + i);
  for (int i = threadIdx.x; i < a.B; i += 32 * kSlices) used += __ldcg(rows + i) > 0;
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) t += __shfl_xor_sync(0xffffffffu, t, o);
  used = __reduce_add_sync(0xffffffffu, used);
  if (lane == 0) {
    sh_term[slice] = t;
    sh_used[slice] = used;
  }
  __syncthreads();
  if (threadIdx.x == 0) {
    t = 0.0;
    used = 0;
    for (int k = 0; k < kSlices; ++k) {
      t += sh_term[k];
      used += sh_used[k];
    }
    loss[0] = used ? float(t / double(used)) : 0.f;
  }
}

// A group of `lanes` lanes per row, as in the forward; the segment's weights of its columns
// stay in registers until the segment ends. One pass: bound by reading the logits and
// writing their gradient.
template <class T, int kVec, int kC, bool kSigmoid>
__global__ void __launch_bounds__(kThreads, kCtas<T, kC>)
    balance_grad_kernel(const BalanceArgs a, int lanes, const int64_t *counts, const int64_t *rows,
                        const float *grad_loss, T *dx) {
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
  const int groups = 32 / lanes, l = lane & (lanes - 1), step = kWarps * groups;
  const int64_t r0 = int64_t(blockIdx.x) * a.chunk, r1 = r0 + a.chunk < a.N ? r0 + a.chunk : a.N;
  auto counted = [&](int64_t r) { return r < r1 && (a.mask == nullptr || ld(a.mask + r) != 0); };
  int64_t r = r0 + warp * groups + lane / lanes;
  Row<T, kVec, kC> next;
  bool next_on = counted(r);
  next.load(x + r * a.E, a.E, l, lanes, next_on);
  bool after_on = counted(r + step);
  int b = -1;
  int64_t seg_end = -1;  // of segment b: the weights are those of another one from there on
  float w[kC];
#pragma unroll
  for (int j = 0; j < kC; ++j) w[j] = 0.f;
  for (int64_t base = r0 + warp * groups; base < r1; base += step, r += step) {
    const Row<T, kVec, kC> row = next;
    const bool on = next_on;
    next_on = after_on;
    next.load(x + (r + step) * a.E, a.E, l, lanes, next_on);
    after_on = counted(r + 2 * step);
    if (on && r >= seg_end) {
      b = seg_of(a, r);
      seg_end = b + 1 < a.B ? seg_at(a, b + 1) : a.N;
      if (seg_end <= r) seg_end = r + 1;  // (cu_seqlens that do not rise)
      const float n = float(ld(rows + b));
      const float f = n > 0.f ? g * float(a.E) / (float(a.k) * n * n * float(used)) : 0.f;
#pragma unroll
      for (int j = 0; j < kC; ++j) {
        const int c = Row<T, kVec, kC>::column(j, l, lanes);
        w[j] = c < a.E ? f * float(ld(counts + int64_t(b) * a.E + c)) : 0.f;
      }
    }
    __syncwarp();
    float q[kC], em = 0.f;
    if (__any_sync(0xffffffffu, on)) {
      const float inv = row_scores<kSigmoid>(row, q, lanes, em);
      float d = 0.f;
#pragma unroll
      for (int j = 0; j < kC; ++j) d = fmaf(q[j], w[j], d);
      d = lanes_sum(d, lanes) * inv;
#pragma unroll
      for (int j = 0; j < kC; ++j) {
        const float s = kSigmoid ? q[j] * inv * fmaf(-em, q[j], 1.f) : q[j] * inv;
        q[j] = s * (w[j] - d);
      }
    } else {  // spans of masked rows
#pragma unroll
      for (int j = 0; j < kC; ++j) q[j] = 0.f;
    }
    if (r < r1) Row<T, kVec, kC>::store(dx + r * a.E, q, a.E, l, lanes);
  }
}

// The layout of a row of E: kC columns a lane and the lanes that take it.
struct Layout {
  int columns, lanes;
  bool vec;
};
// Vector loads where every row starts on 16 bytes. Of the layouts the one with the
// least work: a lane's columns at about 7 instructions each, the exchanges between
// lanes and 24 more, times the lanes (160 bf16 logits: 8 lanes x 24 columns, not
// 16 x 16, of which 96 would be idle).
Layout layout(const void *x, const void *dx, sao_dtype dt, int E) {
  const int size = dt == SAO_BF16 ? 2 : 4, per = 16 / size;
  Layout best{0, 0, E % per == 0 && aligned16(x) && aligned16(dx)};
  int least = 0;
  for (int c = 8; c <= 32; c += 8) {
    const int vec = best.vec ? per : 1, loads = c / vec, units = E / vec;
    int lanes = 1, log = 0;
    while (lanes * loads < units) {
      lanes <<= 1;
      ++log;
    }
    if (lanes > 32) continue;
    const int cost = lanes * (7 * c + 4 * log + 24);
    if (best.columns == 0 || (c < 32 && cost < least)) {  // 32 columns: where no other fits
      best.columns = c;
      best.lanes = lanes;
      least = cost;
    }
  }
  return best;
}

// f(type, loads, columns, score) with the layout's values as types.
template <int kValue>
using Int = std::integral_constant<int, kValue>;
template <class T, class F>
void with_layout(const Layout &l, int score, F f) {
  auto columns = [&](auto vec, auto sig) {
    switch (l.columns) {
      case 8: return f(T{}, vec, Int<8>{}, sig);
      case 16: return f(T{}, vec, Int<16>{}, sig);
      case 24: return f(T{}, vec, Int<24>{}, sig);
      default: return f(T{}, vec, Int<32>{}, sig);
    }
  };
  auto loads = [&](auto sig) { l.vec ? columns(Int<int(16 / sizeof(T))>{}, sig) : columns(Int<1>{}, sig); };
  score == SAO_SCORE_SIGMOID ? loads(std::true_type{}) : loads(std::false_type{});
}

// Rows per CTA: three CTAs on each of 152 SMs, at least one row for every lane group of
// the CTA's with the fewest lanes. From N and E alone: the sums' order, and so their
// bits, are those of any device and alignment.
int chunk_rows(int64_t N, int E) {
  const int64_t c = (N + 455) / 456, least = E <= 16 ? 256 : 32;
  return int(c < least ? least : c);
}
BalanceArgs make_args(const void *x, const int32_t *ids, const uint8_t *mask, const int32_t *cu, int32_t B, int64_t N,
                      int32_t E, int32_t k, unsigned int *err) {
  BalanceArgs a{x, ids, mask, cu, cu ? B : 1, N, E, k, chunk_rows(N, E), 0, err};
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
  const int64_t chunk = chunk_rows(N, E);
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
  const Layout lay = layout(x, x, dt, E);
  int slot = launch_begin("balance_partial", s);
  auto partial = [&](auto t, auto vec, auto columns, auto sig) {
    pdl(balance_partial_kernel<decltype(t), vec.value, columns.value, sig.value>, unsigned(a.chunks), kThreads,
        size_t(E) * (kWarps + 1) * sizeof(float), s)(a, lay.lanes, w.psum, w.pcount, w.prows, w.ticket);
  };
  dt == SAO_BF16 ? with_layout<__nv_bfloat16>(lay, score, partial) : with_layout<float>(lay, score, partial);
  SAO_TRY(launch_end(slot, s));
  // a batch's partials, hundreds in few CTAs: 32 warps to each; many trajectories: 8
  const unsigned grid = unsigned(a.B) * unsigned((E + 31) / 32);
  slot = launch_begin("balance_reduce", s);
  auto reduce = grid <= 152 ? balance_reduce_kernel<32> : balance_reduce_kernel<8>;
  pdl(reduce, grid, grid <= 152 ? 1024 : 256, 0, s)(a, w.psum, w.pcount, w.prows, loss, counts, prob_sums, rows,
                                                    w.terms, w.ticket);
  return launch_end(slot, s);
}

sao_status balance_bwd_launch(const void *x, sao_dtype dt, const uint8_t *mask, const int32_t *cu, int32_t B, int64_t N,
                              int32_t E, int32_t k, int score, const int64_t *counts, const int64_t *rows,
                              const float *grad_loss, void *dx, unsigned int *err, cudaStream_t s) {
  const BalanceArgs a = make_args(x, nullptr, mask, cu, B, N, E, k, err);
  const Layout lay = layout(x, dx, dt, E);
  int slot = launch_begin("balance_grad", s);
  auto grad = [&](auto t, auto vec, auto columns, auto sig) {
    using T = decltype(t);
    pdl(balance_grad_kernel<T, vec.value, columns.value, sig.value>, unsigned(a.chunks), kThreads, 0, s)(
        a, lay.lanes, counts, rows, grad_loss, static_cast<T *>(dx));
  };
  dt == SAO_BF16 ? with_layout<__nv_bfloat16>(lay, score, grad) : with_layout<float>(lay, score, grad);
  return launch_end(slot, s);
}

}  // namespace sao
