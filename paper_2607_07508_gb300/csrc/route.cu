// Routing to experts: each token's k experts and their weights, and the gradient of the logits.
//
//   s_e = softmax(x)_e or sigmoid(x_e),  key_e = s_e + bias_e,  the k largest keys of the groups that stay
//   w_j = scale s_j, over the sum of the chosen s where weights are renormalised
//
// A warp takes a row; a lane holds consecutive experts of one group, so that the lowest index of equal keys is
// the lowest lane's, and a group's best two come from the few lanes that share it. Softmax and sigmoid keep the
// logits' order: without a bias experts are picked by their logits, which is exact, and renormalised weights need
// the chosen logits alone. Keys with a bias (and sums of two keys) are formed in fp32 first; a row in which two of
// them are nearer to one another than their errors, and not the same logit and bias, is chosen again in fp64.
#include <cuda_bf16.h>
#include <math.h>
#include <stdint.h>

#include <type_traits>

#include "route.cuh"
#include "sao_common.cuh"
#include "sao_internal.h"

namespace sao {
namespace {

constexpr int kWarps = 8;  // rows of a CTA at a time
constexpr unsigned kAll = 0xffffffffu;

// Where a lane's experts lie: `per` of them from `first` on, `count` of them there.
struct Lanes {
  int share;  // lanes to a group (a power of two)
  int per;    // experts to a lane
  int size;   // experts to a group
  int groups;
};
__device__ __forceinline__ int first_of(const Lanes &l, int lane) {
  return lane / l.share * l.size + lane % l.share * l.per;
}
__device__ __forceinline__ int count_of(const Lanes &l, int lane) {
  if (lane / l.share >= l.groups) return 0;
  const int left = l.size - lane % l.share * l.per;
  return left < l.per ? (left > 0 ? left : 0) : l.per;
}

__device__ __forceinline__ float value(const float *p) { return ld(p); }
__device__ __forceinline__ float value(const __nv_bfloat16 *p) {
  return __uint_as_float(uint32_t(ld(reinterpret_cast<const uint16_t *>(p))) << 16);
}

// fp32 values in the order of unsigned integers.
__device__ __forceinline__ uint32_t ordered(float v) {
  const uint32_t u = __float_as_uint(v);
  return u ^ (uint32_t(int32_t(u) >> 31) | 0x80000000u);
}
__device__ __forceinline__ float unordered(uint32_t u) {
  return __uint_as_float(u & 0x80000000u ? u ^ 0x80000000u : ~u);
}
__device__ __forceinline__ float warp_max(float v) { return unordered(__reduce_max_sync(kAll, ordered(v))); }
__device__ __forceinline__ double warp_max(double v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v = fmax(v, __shfl_xor_sync(kAll, v, o));
  return v;
}
template <class F>
__device__ __forceinline__ F warp_sum(F v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(kAll, v, o);
  return v;
}

__device__ __forceinline__ float exp_of(float v) { return expf(v); }
__device__ __forceinline__ double exp_of(double v) { return exp(v); }
template <class F>
__device__ __forceinline__ F sigmoid(F x) {
  const F e = exp_of(-fabs(x));  // never past the range, and small scores keep their digits
  return (x < F(0) ? e : F(1)) / (F(1) + e);
}

template <class F>
__device__ __forceinline__ void merge_two(F &a1, F &a2, F b1, F b2) {
  a2 = fmax(fmin(a1, b1), fmax(a2, b2));
  a1 = fmax(a1, b1);
}

// The choice of one row from its logits x (-inf: none there, or never chosen). Lane j gets choice j, -1 if there
// is none. F: float, or double where fp32 cannot tell (*near).
template <class F, int kPer>
__device__ __forceinline__ int choose(const RouteArgs &a, const Lanes &l, const float (&x)[kPer], float top,
                                      bool *near) {
  constexpr bool k32 = std::is_same<F, float>::value;
  const int lane = threadIdx.x & 31, e0 = first_of(l, lane), n = count_of(l, lane);
  const F none = -INFINITY;
  const bool soft = a.score == SAO_SCORE_SOFTMAX, biased = a.bias != nullptr;
  F key[kPer];
  F inverse = 1, most = 1;  // most: no score is larger
  if (soft && biased) {
    F sum = 0;
#pragma unroll
    for (int i = 0; i < kPer; ++i) sum += exp_of(F(x[i]) - F(top));
    inverse = most = F(1) / warp_sum(sum);
  }
#pragma unroll
  for (int i = 0; i < kPer; ++i) {
    key[i] = F(x[i]);
    if (biased && i < n && x[i] > -INFINITY) {
      const float b = ld(a.bias + e0 + i);
      const F s = soft ? exp_of(F(x[i]) - F(top)) * inverse : sigmoid(F(x[i]));
      key[i] = b > -INFINITY ? s + F(b) + F(0) : none;
    }
  }
  *near = false;
  // fp32: a score is off by at most 2^-19 of the row's largest one (exponential, difference from the largest logit,
  // sum of up to 1024, quotient), a key by another 2^-24 of itself; twice that for a difference
  const auto tell = [&](F v) { return F(0x1p-18) * most + F(0x1p-22) * fabs(v); };

  if (l.groups > 1) {
    F b1 = none, b2 = none;
#pragma unroll
    for (int i = 0; i < kPer; ++i) merge_two(b1, b2, key[i], none);
    for (int o = 1; o < l.share; o <<= 1) {
      const F c1 = __shfl_xor_sync(kAll, b1, o), c2 = __shfl_xor_sync(kAll, b2, o);
      merge_two(b1, b2, c1, c2);
    }
    const bool exact = !biased && !a.two;
    F v = b1;
    if (a.two) {
      if (!biased) {  // the scores of the two largest logits (softmax: times their common sum)
        const F s1 = soft ? exp_of(b1 - F(top)) : sigmoid(b1), s2 = soft ? exp_of(b2 - F(top)) : sigmoid(b2);
        v = b1 > none ? s1 + s2 : none;
      } else if (b2 > none) {
        v = b1 + b2;
      }
    }
    const int mine = lane / l.share;
    int rank = 0;
    for (int g = 0; g < l.groups; ++g) {
      const F other = __shfl_sync(kAll, v, g * l.share);
      rank += other > v || (other == v && g < mine);
    }
    const bool real = mine < l.groups, stays = real && rank < a.kept;
    if (k32 && !exact) {
      const int last = __ffs(__ballot_sync(kAll, real && rank == a.kept - 1)) - 1;
      const F vl = __shfl_sync(kAll, v, last), l1 = __shfl_sync(kAll, b1, last), l2 = __shfl_sync(kAll, b2, last);
      const bool close = real && !(fabs(v - vl) > 2 * tell(vl)) && v > none;
      const bool same = !biased && b1 == l1 && b2 == l2;
      *near = __any_sync(kAll, close && !stays) && __any_sync(kAll, close && !same);
    }
    if (!stays) {
#pragma unroll
      for (int i = 0; i < kPer; ++i) key[i] = none;
    }
  }

  int id = -1;
  F before = 0;
  float x_before = 0.f, b_before = 0.f;
  const bool compare = k32 && biased;
  for (int j = 0; j < a.k + (compare ? 1 : 0); ++j) {
    F best = key[0];
#pragma unroll
    for (int i = 1; i < kPer; ++i) best = fmax(best, key[i]);
    const F m = warp_max(best);
    if (!(m > none)) break;
    const unsigned from = __ballot_sync(kAll, best == m);
    const int win = __ffs(from) - 1;
    int at = 0;
    float xv = 0.f;
    bool found = false;
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      const bool hit = !found && lane == win && key[i] == m;
      if (hit) at = i, xv = x[i], key[i] = none;
      found |= hit;
    }
    const int e = __shfl_sync(kAll, e0 + at, win);
    if (lane == j && j < a.k) id = e;
    if (compare) {
      xv = __shfl_sync(kAll, xv, win);
      const float b = ld(a.bias + e);
      if (j > 0 && !(before - m > 2 * tell(before)) && !(xv == x_before && b == b_before)) *near = true;
      before = m, x_before = xv, b_before = b;
    }
  }
  return id;
}

template <class T, int kPer>
__device__ __forceinline__ void load_row(const T *row, const Lanes &l, float (&x)[kPer]) {
  const int lane = threadIdx.x & 31, e0 = first_of(l, lane), n = count_of(l, lane);
#pragma unroll
  for (int i = 0; i < kPer; ++i) x[i] = i < n ? value(row + e0 + i) + 0.f : -INFINITY;  // -0 and 0 are one key
}

// The choice in fp64, the row read again: few rows come here, and none of their registers are held for it.
template <class T, int kPer>
__device__ __noinline__ int choose_again(const RouteArgs *a, const Lanes *l, const T *row, float top) {
  float x[kPer];
  load_row<T, kPer>(row, *l, x);
  bool near;
  return choose<double, kPer>(*a, *l, x, top, &near);
}

template <class T, int kPer>
__global__ void __launch_bounds__(kWarps * 32) route_fwd_kernel(const __grid_constant__ RouteArgs a,
                                                                const __grid_constant__ Lanes l) {
  grid_wait();
  const int lane = threadIdx.x & 31;
  const bool soft = a.score == SAO_SCORE_SOFTMAX;
  for (int64_t row = int64_t(blockIdx.x) * kWarps + threadIdx.x / 32; row < a.N; row += int64_t(gridDim.x) * kWarps) {
    int32_t *ids = a.ids + row * a.k;
    float *weights = a.weights + row * a.k;
    if (a.mask && ld(a.mask + row) == 0) {
      if (lane < a.k) {
        if (!a.replay) ids[lane] = -1;
        weights[lane] = 0.f;
      }
      continue;
    }
    const T *from = static_cast<const T *>(a.x) + row * a.E;
    float x[kPer];
    load_row<T, kPer>(from, l, x);
    bool bad = false;
    float top = -INFINITY;
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      bad |= !(x[i] < INFINITY) && (soft || x[i] != x[i]);
      top = fmaxf(top, x[i]);
    }
    top = warp_max(top);
    bad = __any_sync(kAll, bad);
    if (bad && lane == 0) raise_device_error(a.err, SAO_DEVERR_LOGITS);
    int id = -1;
    const bool scores = !bad && top > -INFINITY;
    if (a.replay) {
      if (lane < a.k) id = ld(ids + lane);
      if (id >= a.E) raise_device_error(a.err, SAO_DEVERR_EXPERT_ID);
      if (id >= a.E || !scores) id = -1;
    } else {
      if (scores) {
        bool near;
        id = choose<float, kPer>(a, l, x, top, &near);
        if (__any_sync(kAll, near)) id = choose_again<T, kPer>(&a, &l, from, top);
      }
      if (lane < a.k) ids[lane] = id;
    }
    float w = 0.f;
    const float chosen = id >= 0 ? value(from + id) : -INFINITY;
    if (a.renorm) {
      // sigmoid(x) = exp(min(x, 0)) / (1 + exp(-|x|)): relative to the largest, no sum vanishes
      const float low = soft ? chosen : fminf(chosen, 0.f), m = warp_max(low);
      if (m > -INFINITY) {
        float s = expf(low - m);
        if (!soft) s /= 1.f + expf(-fabsf(chosen));
        w = s / warp_sum(s);
      }
    } else if (!soft) {
      w = sigmoid(chosen);
    } else {
      float sum = 0.f;
#pragma unroll
      for (int i = 0; i < kPer; ++i) sum += scores ? expf(x[i] - top) : 0.f;
      sum = warp_sum(sum);
      if (scores) w = expf(chosen - top) / sum;
    }
    if (lane < a.k) weights[lane] = a.scale * w;
  }
}

template <class T, int kPer>
__global__ void __launch_bounds__(kWarps * 32) route_bwd_kernel(const __grid_constant__ RouteBwdArgs a, int per) {
  grid_wait();
  const int lane = threadIdx.x & 31;
  const Lanes l{32, per, a.E, 1};
  const int e0 = first_of(l, lane), n = count_of(l, lane);
  const bool soft = a.score == SAO_SCORE_SOFTMAX, dense = soft && !a.renorm;
  for (int64_t row = int64_t(blockIdx.x) * kWarps + threadIdx.x / 32; row < a.N; row += int64_t(gridDim.x) * kWarps) {
    const T *x = static_cast<const T *>(a.x) + row * a.E;
    T *dx = static_cast<T *>(a.dx) + row * a.E;
    const bool on = a.scale != 0.f && (a.mask == nullptr || ld(a.mask + row) != 0);
    int id = -1;
    float w = 0.f, g = 0.f;
    if (on && lane < a.k) {
      id = ld(a.ids + row * a.k + lane);
      if (id >= a.E) raise_device_error(a.err, SAO_DEVERR_EXPERT_ID), id = -1;
      if (id >= 0) w = ld(a.weights + row * a.k + lane), g = ld(a.grad + row * a.k + lane);
    }
    const float c = warp_sum(g * w);
    float d = 0.f;  // of choice j in lane j
    if (dense)
      d = a.scale * g;
    else if (w != 0.f) {
      d = a.renorm ? w * (g - c / a.scale) : w * g;
      if (!soft) d *= sigmoid(-value(x + id));
    }
    float v[kPer];
#pragma unroll
    for (int i = 0; i < kPer; ++i) v[i] = 0.f;
    for (int j = 0; j < a.k; ++j) {
      const int at = __shfl_sync(kAll, id, j) - e0;
      const float dj = __shfl_sync(kAll, d, j);
#pragma unroll
      for (int i = 0; i < kPer; ++i)
        if (at == i) v[i] += dj;
    }
    if (dense) {
      float p[kPer], sum = 0.f, top = -INFINITY;
      const bool any = __any_sync(kAll, id >= 0);
      if (any) load_row<T, kPer>(x, l, p);
#pragma unroll
      for (int i = 0; i < kPer; ++i) {
        if (!any) p[i] = 0.f;
        top = fmaxf(top, p[i]);
      }
      top = warp_max(top);
#pragma unroll
      for (int i = 0; i < kPer; ++i) sum += p[i] = expf(p[i] - top);
      const float inverse = 1.f / warp_sum(sum);
      const bool scores = any && top > -INFINITY && inverse > 0.f;  // a NaN, +inf: the sum is NaN
#pragma unroll
      for (int i = 0; i < kPer; ++i) v[i] = scores ? p[i] * inverse * (v[i] - c) : 0.f;
    }
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      if (i >= n) continue;
      if (a.accumulate) v[i] += value(dx + e0 + i);
      if constexpr (sizeof(T) == 2)
        dx[e0 + i] = __float2bfloat16_rn(v[i]);
      else
        dx[e0 + i] = v[i];
    }
  }
}

template <class F>
sao_status by_count(int per, F f) {
  if (per <= 1) return f(std::integral_constant<int, 1>());
  if (per <= 2) return f(std::integral_constant<int, 2>());
  if (per <= 4) return f(std::integral_constant<int, 4>());
  if (per <= 5) return f(std::integral_constant<int, 5>());
  if (per <= 8) return f(std::integral_constant<int, 8>());
  if (per <= 16) return f(std::integral_constant<int, 16>());
  if (per <= 32) return f(std::integral_constant<int, 32>());
  return f(std::integral_constant<int, 64>());  // 17 to 31 groups, a lane each: up to 60 experts
}

template <class F>
sao_status by_type(sao_dtype dt, F f) {
  return dt == SAO_BF16 ? f(__nv_bfloat16()) : f(float());
}

sao_status grid_of(int64_t N, unsigned *grid) {
  DeviceInfo di;
  SAO_TRY(device_info(&di));
  const int64_t most = int64_t(di.sm_count) * 16, g = (N + kWarps - 1) / kWarps;
  *grid = unsigned(g < most ? g : most);
  return SAO_OK;
}

}  // namespace

sao_status route_fwd_launch(const RouteArgs &args, sao_dtype dt, cudaStream_t s) {
  RouteArgs a = args;
  if (a.groups == a.kept || a.replay) a.groups = a.kept = 1;
  Lanes l{32, 0, a.E / a.groups, a.groups};
  while (l.share * a.groups > 32) l.share /= 2;
  l.per = (l.size + l.share - 1) / l.share;
  unsigned grid;
  SAO_TRY(grid_of(a.N, &grid));
  const int slot = launch_begin("route_fwd", s);
  SAO_TRY(by_type(dt, [&](auto t) {
    return by_count(l.per, [&](auto per) {
      pdl(route_fwd_kernel<decltype(t), decltype(per)::value>, grid, kWarps * 32, 0, s)(a, l);
      return SAO_OK;
    });
  }));
  return launch_end(slot, s);
}

sao_status route_bwd_launch(const RouteBwdArgs &a, sao_dtype dt, cudaStream_t s) {
  const int per = (a.E + 31) / 32;
  unsigned grid;
  SAO_TRY(grid_of(a.N, &grid));
  const int slot = launch_begin("route_bwd", s);
  SAO_TRY(by_type(dt, [&](auto t) {
    return by_count(per, [&](auto count) {
      pdl(route_bwd_kernel<decltype(t), decltype(count)::value>, grid, kWarps * 32, 0, s)(a, per);
      return SAO_OK;
    });
  }));
  return launch_end(slot, s);
}

}  // namespace sao
