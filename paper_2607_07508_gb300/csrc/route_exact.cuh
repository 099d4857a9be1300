// What the forms of the choice share: where experts lie in a warp, keys as integers, and a row's choice in fp64.
#pragma once

#include "route_common.cuh"

namespace sao {
namespace route {

// Where a lane's experts lie: consecutive ones of one group, `per` of them or fewer.
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

// Values in the order of unsigned integers.
__device__ __forceinline__ uint32_t ordered(float v) {
  const uint32_t u = __float_as_uint(v);
  return u ^ (uint32_t(int32_t(u) >> 31) | 0x80000000u);
}
__device__ __forceinline__ float unordered(uint32_t u) {
  return __uint_as_float(u & 0x80000000u ? u ^ 0x80000000u : ~u);
}
__device__ __forceinline__ uint64_t ordered(double v) {
  const uint64_t u = uint64_t(__double_as_longlong(v));
  return u ^ (uint64_t(int64_t(u) >> 63) | 0x8000000000000000ull);
}
__device__ __forceinline__ float warp_max(float v) { return unordered(__reduce_max_sync(kAll, ordered(v))); }
__device__ __forceinline__ uint64_t warp_max(uint64_t v) {
  const uint32_t high = __reduce_max_sync(kAll, uint32_t(v >> 32));
  const uint32_t low = __reduce_max_sync(kAll, uint32_t(v >> 32) == high ? uint32_t(v) : 0u);
  return uint64_t(high) << 32 | low;
}

template <class F>
__device__ __forceinline__ void merge_two(F &a1, F &a2, F b1, F b2) {
  a2 = fmax(fmin(a1, b1), fmax(a2, b2));
  a1 = fmax(a1, b1);
}

// The choice of one row in fp64 (without a bias: by its logits, and sums of scores in fp64). Lane j gets choice
// j, -1 if there is none. Few rows come here; keys are compared as integers, as the fp64 units are few.
struct Exactly {
  const float *bias;
  int k, kept;
  bool soft, two;
};
template <class T, int kPer, bool kBiased>
__device__ __noinline__ int choose_exactly(Exactly a, Lanes l, const T *row) {
  const int lane = threadIdx.x & 31, e0 = first_of(l, lane), n = count_of(l, lane);
  const bool soft = a.soft;
  constexpr int kUnroll = kPer <= 16 ? kPer : 1;  // (else in local memory, which costs the kernel no registers)
  float top = -INFINITY;
#pragma unroll 1
  for (int i = 0; i < n; ++i) top = fmaxf(top, value(row + e0 + i));
  top = warp_max(top);
  double inverse = 1.0;
  if (kBiased && soft) {
    double sum = 0.0;
#pragma unroll 1
    for (int i = 0; i < n; ++i) sum += exp(double(value(row + e0 + i)) - double(top));
    inverse = 1.0 / warp_sum(sum);
  }
  uint64_t key[kPer];  // 0: none
  const auto key_at = [&](int i) {
    const float x = value(row + e0 + i) + 0.f, b = kBiased ? ld(a.bias + e0 + i) : 0.f;  // -0 and 0 are one key
    if (!(x > -INFINITY && b > -INFINITY)) return uint64_t(0);
    double k = double(x);
    if (kBiased) k = (soft ? exp(double(x) - double(top)) * inverse : sigmoid(double(x))) + double(b) + 0.0;
    return ordered(k);
  };
#pragma unroll kUnroll
  for (int i = 0; i < kPer; ++i) key[i] = 0;
#pragma unroll 1
  for (int j = 0; j < n; ++j) {  // (one exponential's code and registers)
    const uint64_t k = key_at(j);
#pragma unroll kUnroll
    for (int i = 0; i < kPer; ++i)
      if (i == j) key[i] = k;
  }
  bool stays = true;
  if (l.groups > 1) {
    uint64_t b1 = 0, b2 = 0;
#pragma unroll kUnroll
    for (int i = 0; i < kPer; ++i) {
      b2 = max(b2, min(b1, key[i]));
      b1 = max(b1, key[i]);
    }
    for (int o = 1; o < l.share; o <<= 1) {
      const uint64_t c1 = __shfl_xor_sync(kAll, b1, o), c2 = __shfl_xor_sync(kAll, b2, o);
      b2 = max(min(b1, c1), max(b2, c2));
      b1 = max(b1, c1);
    }
    uint64_t v = b1;
    if (a.two && b1 != 0) {
      const auto plain = [&](uint64_t u) {  // its score, or key with the bias
        const double k = __longlong_as_double(int64_t(u & 0x8000000000000000ull ? u ^ 0x8000000000000000ull : ~u));
        return u == 0 ? 0.0 : kBiased ? k : soft ? exp(k - double(top)) : sigmoid(k);
      };
      v = ordered(plain(b1) + plain(b2) + 0.0);
    }
    const int mine = lane / l.share;
    int rank = 0;
    for (int g = 0; g < l.groups; ++g) {
      const uint64_t other = __shfl_sync(kAll, v, g * l.share);
      rank += other > v || (other == v && g < mine);
    }
    stays = mine < l.groups && rank < a.kept;
  }
  int id = -1;
  for (int j = 0; j < a.k; ++j) {
    uint64_t best = 0;
    int at = -1;
#pragma unroll kUnroll
    for (int i = 0; i < kPer; ++i)
      if (stays && key[i] > best) best = key[i], at = i;
    const uint64_t m = warp_max(best);
    if (m == 0) break;
    const int win = __ffs(__ballot_sync(kAll, best == m)) - 1;
#pragma unroll kUnroll
    for (int i = 0; i < kPer; ++i)
      if (lane == win && i == at) key[i] = 0;
    const int e = __shfl_sync(kAll, e0 + at, win);
    if (lane == j) id = e;
  }
  return id;
}

// exp and sigmoid for keys alone. With |x| 2^-23.4 for the product's rounding and 2^-22.5 for the exponential's
// error (of itself), a sigmoid is off by s (1 - s) of those, its sum's 2^-24 and the reciprocal's 2^-23: less
// than 2^-21.
__device__ __forceinline__ float exp_fast(float x) {
  float e;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e) : "f"(x * 1.4426950408889634f));
  return e;
}
__device__ __forceinline__ float sigmoid_fast(float x) {
  float r;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(1.f + exp_fast(-x)));
  return r;
}
// How near two keys may be for their order in fp32 to be doubted, but for rounding with their own size: twice a score's
// error. Under softmax that has the sum's, 2^-18 of the row's largest score.
constexpr float kDoubtSigmoid = 0x1p-20f, kDoubtSoftmax = 0x1p-17f;

}  // namespace route

// route_lists.cu: whether its form takes the call, of which `groups` is 1 where all stay.
bool route_lists_take(const RouteArgs &a, int sms);
sao_status route_lists_launch(const RouteArgs &a, const route::Lanes &l32, sao_dtype dt, int sms, cudaStream_t s);

}  // namespace sao
