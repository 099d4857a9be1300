// Routing to experts, the form for many tokens: eight lanes take a row, each an eighth of its experts, and keep the
// largest eight keys of those in a sorted list; three exchanges merge the lists.
//
// What bounds it is the number of instructions: a list costs 9 of them a key (a block of eight is sorted by a
// network of 19 exchanges and merged with eight maxima and 12 exchanges), where picking one expert after another
// from a warp's 32 lanes costs 11 to 20 a pick and lane, and nothing is summed or compared over a whole warp.
//
// Keys are packed in 32 bits, the expert's index (inverted: the lower of equal keys is the larger) below
//   a bf16 logit, which leaves room for it;
//   an fp32 logit without its lowest bits;
//   a sigmoid with a bias as a fraction, in units of 2^-23 of the range that biases and scores span.
// Where the bits above the index do not decide, rows are ranked again: picks among themselves by their logits or
// by keys in fp64, a lane each, and rows whose last pick is in doubt as a whole (choose_exactly).
#include "route_exact.cuh"

namespace sao {
namespace {

using namespace route;

constexpr int kShare = 8;   // lanes to a row
constexpr int kList = 8;    // keys to a list, and experts to a token at most
constexpr int kRows = 32 / kShare;
constexpr int kListWarps = 4;

__device__ __forceinline__ void exchange(uint32_t &a, uint32_t &b) {  // a >= b behind it
  const uint32_t high = max(a, b), low = min(a, b);
  a = high, b = low;
}
// Eight keys in falling order: odd-even merge sort.
__device__ __forceinline__ void sort8(uint32_t (&v)[8]) {
  exchange(v[0], v[1]), exchange(v[2], v[3]), exchange(v[4], v[5]), exchange(v[6], v[7]);
  exchange(v[0], v[2]), exchange(v[1], v[3]), exchange(v[4], v[6]), exchange(v[5], v[7]);
  exchange(v[1], v[2]), exchange(v[5], v[6]);
  exchange(v[0], v[4]), exchange(v[1], v[5]), exchange(v[2], v[6]), exchange(v[3], v[7]);
  exchange(v[2], v[4]), exchange(v[3], v[5]);
  exchange(v[1], v[2]), exchange(v[3], v[4]), exchange(v[5], v[6]);
}
// The largest eight of two lists, in falling order; `rest` becomes the largest of those left out, of which it was one.
template <bool kRest>
__device__ __forceinline__ void merge8(uint32_t (&v)[8], const uint32_t (&w)[8], uint32_t &rest) {
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    if (kRest) rest = max(rest, min(v[i], w[7 - i]));
    v[i] = max(v[i], w[7 - i]);  // falling, then rising: bitonic
  }
#pragma unroll
  for (int o = 4; o > 0; o >>= 1)
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if ((i & o) == 0) exchange(v[i], v[i + o]);
}

struct ListPlan {
  int per;        // experts to a lane
  int blocks;     // of eight
  int unit;       // bytes of a load: 16, 8, or those of a logit
  uint32_t mask;  // the bits of a packed fp32 logit that hold the expert
};
constexpr uint32_t kFractionMask = 511u;  // of a fraction: its 23 bits fill the others
constexpr float kFractionLeast = 1.f + 0x1p-10f;

// Eight logits from p on, `n` of them there (others: -inf).
template <class T>
__device__ __forceinline__ void load8(const T *p, int n, int unit, float (&x)[8]) {
  constexpr int kSize = int(sizeof(T));
  const auto put = [&](int at, uint32_t w) {
    if constexpr (kSize == 4)
      x[at] = __uint_as_float(w);
    else
      x[at] = __uint_as_float(w << 16), x[at + 1] = __uint_as_float(w & 0xffff0000u);
  };
  if (unit == 16 && n >= 8) {
#pragma unroll
    for (int i = 0; i < 8; i += 16 / kSize) {
      const uint4 v = ld(reinterpret_cast<const uint4 *>(p + i));
      put(i, v.x), put(i + 4 / kSize, v.y), put(i + 8 / kSize, v.z), put(i + 12 / kSize, v.w);
    }
  } else if (unit >= 8) {
#pragma unroll
    for (int i = 0; i < 8; i += 8 / kSize) {
      if (i + 8 / kSize <= n) {
        const uint2 v = ld(reinterpret_cast<const uint2 *>(p + i));
        put(i, v.x), put(i + 4 / kSize, v.y);
      } else {
#pragma unroll
        for (int j = 0; j < 8 / kSize; ++j) x[i + j] = i + j < n ? value(p + i + j) : -INFINITY;
      }
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = i < n ? value(p + i) : -INFINITY;
  }
}

// Over the kShare lanes of a row.
__device__ __forceinline__ bool row_any(bool v) {
  return (__ballot_sync(kAll, v) >> (threadIdx.x & 24u) & 0xffu) != 0u;
}

// kBiased: sigmoid scores with a bias. kRest: the largest key left out is kept, which the check of the last pick needs
// where the picks fill the list. l: eight lanes to a row; l32: all of a warp's, for choose_exactly.
template <class T, bool kBiased, bool kRest>
__global__ void __launch_bounds__(kListWarps * 32)
    route_lists_kernel(const __grid_constant__ RouteArgs a, const __grid_constant__ Lanes l,
                       const __grid_constant__ Lanes l32, ListPlan plan) {
  grid_wait();
  constexpr bool kExact = !kBiased && sizeof(T) == 2;
  __shared__ float offset[kBiased ? 512 : 1];
  __shared__ float range[3][kListWarps];
  const int lane = threadIdx.x & 31, warp = threadIdx.x / 32, s = lane & (kShare - 1), base = lane & ~(kShare - 1);
  const bool soft = a.score == SAO_SCORE_SOFTMAX;
  float least = 0.f, units = 1.f;
  bool all_exactly = false;
  if (kBiased) {
    float low = INFINITY, high = -INFINITY, most = -INFINITY;
    for (int e = threadIdx.x; e < a.E; e += kListWarps * 32) {
      const float b = ld(a.bias + e);
      most = fmaxf(most, b);
      if (fabsf(b) < INFINITY) low = fminf(low, b), high = fmaxf(high, b);
    }
    low = -warp_max(-low), high = warp_max(high), most = warp_max(most);
    if (lane == 0) range[0][warp] = low, range[1][warp] = high, range[2][warp] = most;
    __syncthreads();
    for (int w = 0; w < kListWarps; ++w)
      low = fminf(low, range[0][w]), high = fmaxf(high, range[1][w]), most = fmaxf(most, range[2][w]);
    if (high < low) low = high = 0.f;
    least = low;
    // a key is (s + b - least) units + 1 + 2^-10: in [1, 2), with room for its errors
    units = (1.f - 0x1p-9f) / (1.f + (high - low));
    all_exactly = most == INFINITY || !(units >= 0x1p-20f);  // biases that leave no digits to scores
    for (int e = threadIdx.x; e < a.E; e += kListWarps * 32) {
      const float b = ld(a.bias + e);
      offset[e] = fabsf(b) < INFINITY ? fmaf(b - low, units, kFractionLeast) : -INFINITY;
    }
    __syncthreads();
  }
  const uint32_t mask = kExact ? 0xffffu : kBiased ? kFractionMask : plan.mask;
  const uint32_t none = kExact ? 0x007fffffu : kBiased ? kFractionMask : 0x007fffffu | mask;
  // two fractions are off by 2^-20 units (the scores) and 3 2^-23 (offset, difference from the least bias, sum)
  const uint32_t apart = kBiased ? uint32_t(8.f * units) + 4u : 0u;
  const int e0 = s / l.share * l.size + s % l.share * plan.per;
  int n = l.size - s % l.share * plan.per;
  n = n < plan.per ? (n > 0 ? n : 0) : plan.per;
  const auto packed = [&](float x, int e, bool there) {
    if (kBiased) {
      const float f = fmaf(sigmoid_fast(x), units, there ? offset[e] : -INFINITY);
      return f >= 1.f && x > -INFINITY ? __float_as_uint(f) << 9 | (kFractionMask - e) : 0u;
    }
    return (ordered(x + 0.f) & ~mask) | ((mask - e) & mask);  // -0 and 0 are one key; -inf comes to `none` or less
  };
  const int64_t step = int64_t(gridDim.x) * kListWarps * kRows;
  for (int64_t row0 = (int64_t(blockIdx.x) * kListWarps + warp) * kRows; row0 < a.N; row0 += step) {
    const int64_t row = row0 + lane / kShare;
    const bool real = row < a.N;
    const bool on = real && (a.mask == nullptr || ld(a.mask + (real ? row : 0)) != 0);
    if (!__any_sync(kAll, on)) {
      if (real && s < a.k) a.ids[row * a.k + s] = -1, a.weights[row * a.k + s] = 0.f;
      continue;
    }
    const T *logits = static_cast<const T *>(a.x) + (real ? row : a.N - 1) * a.E, *from = logits + e0;
    uint32_t v[8], rest = 0u;
    float probe = 0.f;
#pragma unroll 1
    for (int block = 0; block < plan.blocks; ++block) {
      const int here = on ? n - block * 8 : 0;
      float x[8];
      load8(from + block * 8, here, plan.unit, x);
      uint32_t w[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        probe = fmaf(i < here ? x[i] : 0.f, 0.f, probe);
        w[i] = packed(x[i], e0 + block * 8 + i, i < here);
      }
      sort8(w);
      if (block == 0) {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = w[i];
      } else {
        merge8<kRest>(v, w, rest);
      }
    }
    bool scores = on;
    if (__any_sync(kAll, probe != 0.f)) {  // an infinity or a NaN
      bool bad = false;
      for (int i = 0; i < (on ? n : 0); ++i) {
        const float x = value(from + i);
        bad |= !(x < INFINITY) && (soft || x != x);
      }
      bad = row_any(bad);
      if (bad && s == 0) raise_device_error(a.err, SAO_DEVERR_LOGITS);
      scores = on && !bad;
    }
    const auto join = [&](int o) {
      uint32_t w[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) w[i] = __shfl_xor_sync(kAll, v[i], o);
      if (kRest) rest = max(rest, __shfl_xor_sync(kAll, rest, o));
      merge8<kRest>(v, w, rest);
    };
    for (int o = 1; o < l.share; o <<= 1) join(o);
    float top = 0.f;  // a reference for exponentials: the row's largest logit, but for the bits that its key has lost
    if (!kBiased && soft && (!a.renorm || a.two)) {
      uint32_t first = v[0];
      for (int o = l.share; o < kShare; o <<= 1) first = max(first, __shfl_xor_sync(kAll, first, o));
      if (first > none) top = value(logits + (mask - (first & mask)));
    }
    bool again = all_exactly, stays = true;  // again: choose_exactly
    if (l.groups > 1) {
      const bool one = v[0] > none, both = v[1] > none;
      float worth = -INFINITY;
      if (kBiased) {
        const auto key = [&](uint32_t p) {
          return (__uint_as_float(0x3f800000u | p >> 9) - kFractionLeast) / units + least;
        };
        if (one) worth = key(v[0]) + (a.two && both ? key(v[1]) : 0.f);
      } else if (a.two) {
        // scores of the two best logits (softmax: times their common sum)
        const float x0 = one ? value(logits + (mask - (v[0] & mask))) : 0.f;
        const float x1 = both ? value(logits + (mask - (v[1] & mask))) : -INFINITY;
        if (one) worth = soft ? exp_fast(x0 - top) + exp_fast(x1 - top) : sigmoid_fast(x0) + sigmoid_fast(x1);
      } else if (one) {
        worth = unordered(v[0] & ~mask);
      }
      int rank = 0;
      for (int o = l.share; o < kShare; o += l.share) {
        const float other = __shfl_xor_sync(kAll, worth, o);
        rank += other > worth || (other == worth && (s ^ o) < s);
      }
      stays = rank < a.kept;
      float lowest = stays ? worth : INFINITY, highest = stays ? -INFINITY : worth;
      for (int o = l.share; o < kShare; o <<= 1) {
        lowest = fminf(lowest, __shfl_xor_sync(kAll, lowest, o));
        highest = fmaxf(highest, __shfl_xor_sync(kAll, highest, o));
      }
      if (!kExact || a.two) {
        // of two sums of two: of scores, or of keys, with the rounding of those
        const float error = kBiased ? 0x1p-18f + 0x1p-20f / units + 0x1p-21f * (fabsf(lowest) + fabsf(highest))
                            : a.two ? 0x1p-18f
                                    : 0.f;
        const bool doubt = highest > -INFINITY && !(lowest - highest > error);
        if (__any_sync(kAll, doubt)) {
          // groups about the border of the same logits and biases are equal, and in their order
          const int id0 = one ? int(mask - (v[0] & mask)) : -1, id1 = a.two && both ? int(mask - (v[1] & mask)) : -1;
          const float x0 = id0 >= 0 ? value(logits + id0) : 0.f, x1 = id1 >= 0 ? value(logits + id1) : -INFINITY;
          const float b0 = kBiased && id0 >= 0 ? ld(a.bias + id0) : 0.f;
          const float b1 = kBiased && id1 >= 0 ? ld(a.bias + id1) : 0.f;
          const bool border = fabsf(worth - lowest) <= 2.f * error || fabsf(worth - highest) <= 2.f * error;
          const int at = base + __ffs(__ballot_sync(kAll, rank == a.kept - 1) >> base & 0xffu) - 1;
          // (every lane shuffles: none of this behind an &&)
          const float its_x0 = __shfl_sync(kAll, x0, at), its_x1 = __shfl_sync(kAll, x1, at);
          const float its_b0 = __shfl_sync(kAll, b0, at), its_b1 = __shfl_sync(kAll, b1, at);
          const bool same = x0 == its_x0 && x1 == its_x1 && b0 == its_b0 && b1 == its_b1;
          again |= row_any(doubt && border && !same);
        }
      }
      if (!stays) {
        rest = 0u;
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = 0u;
      }
    }
    for (int o = l.share; o < kShare; o <<= 1) join(o);

    // lane s has choice s; after: the key behind it
    uint32_t pick = 0u, last = 0u, next = rest;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      if (s == i) pick = v[i];
      if (i == a.k - 1) last = v[i];
      if (i == a.k) next = v[i];
    }
    int id = scores && s < a.k && pick > none ? int(mask - (pick & mask)) : -1;
    float chosen = id >= 0 ? value(logits + id) : -INFINITY;
    if (!kExact) {
      const auto near = [&](uint32_t p, uint32_t q) {
        return p > none && q > none && (kBiased ? (p >> 9) - (q >> 9) <= apart : ((p ^ q) & ~mask) == 0u);
      };
      const float bias = kBiased && id >= 0 ? ld(a.bias + id) : 0.f;
      // picks among one another
      const uint32_t after = __shfl_down_sync(kAll, pick, 1);
      const float x_after = __shfl_down_sync(kAll, chosen, 1), b_after = __shfl_down_sync(kAll, bias, 1);
      const bool swap = id >= 0 && s < a.k - 1 && near(pick, after) && !(chosen == x_after && bias == b_after);
      if (__any_sync(kAll, swap)) {
        double key = -INFINITY;
        if (id >= 0) key = kBiased ? sigmoid(double(chosen)) + double(bias) : double(chosen);
        int rank = 0;
        for (int o = 1; o < kShare; ++o) {
          const double other = __shfl_xor_sync(kAll, key, o);
          const int its = __shfl_xor_sync(kAll, id, o);
          rank += other > key || (other == key && (id < 0 ? (s ^ o) < s : its >= 0 && its < id));
        }
        int source = lane;
        for (int i = 0; i < kShare; ++i)
          if (__shfl_sync(kAll, rank, base + i) == s) source = base + i;
        id = __shfl_sync(kAll, id, source);
        chosen = __shfl_sync(kAll, chosen, source);
      }
      // the last one and what was left out: in doubt unless all keys about it are of one logit and bias
      const bool border = scores && near(last, next);
      if (__any_sync(kAll, border)) {
        const int at = int(mask - (last & mask));
        const float x_last = border ? value(logits + at) : 0.f, b_last = kBiased && border ? ld(a.bias + at) : 0.f;
        bool mixed = false;
        for (int i = 0; i < (border && stays ? n : 0); ++i) {
          const float x = value(from + i);
          const uint32_t p = packed(x, e0 + i, true);
          const bool about = p > none && (p > last ? near(p, last) : near(last, p));
          mixed |= about && !(x == x_last && (!kBiased || ld(a.bias + e0 + i) == b_last));
        }
        again |= row_any(mixed);
      }
    }
    unsigned todo = __ballot_sync(kAll, again && scores);
    while (todo != 0u) {
      const int r = (__ffs(todo) - 1) / kShare;
      const T *its_row = static_cast<const T *>(a.x) + (row0 + r) * a.E;
      const int found = choose_exactly<T, 16, kBiased>({a.bias, a.k, a.kept, soft, a.two != 0}, l32, its_row);
      const int its = __shfl_sync(kAll, found, s);
      if (lane / kShare == r) {
        id = s < a.k ? its : -1;
        chosen = id >= 0 ? value(logits + id) : -INFINITY;
      }
      todo &= ~(0xffu << (r * kShare));
    }
    float w = 0.f;
    if (a.renorm) {
      // sigmoid(x) = exp(min(x, 0)) / (1 + exp(-|x|)): relative to the largest, no sum vanishes
      const float lower = soft ? chosen : fminf(chosen, 0.f), m = share_max(lower, 0, kShare, true);
      float t = m > -INFINITY ? expf(lower - m) : 0.f;
      if (!soft) t /= 1.f + expf(-fabsf(chosen));
      const float sum = share_sum(t, 0, kShare, true);
      if (sum > 0.f) w = t / sum;
    } else if (!soft) {
      w = sigmoid(chosen);
    } else {
      float sum = 0.f;
#pragma unroll 4
      for (int i = 0; i < (scores ? n : 0); ++i) sum += expf(value(from + i) - top);
      sum = share_sum(sum, 0, kShare, true);
      if (id >= 0) w = expf(chosen - top) / sum;
    }
    if (real && s < a.k) {
      a.ids[row * a.k + s] = id;
      a.weights[row * a.k + s] = id >= 0 ? a.scale * w : 0.f;
    }
  }
}

}  // namespace

bool route_lists_take(const RouteArgs &a, int sms) {
  if (a.replay || a.k > kList || a.E < 16 || a.E > 512 || a.groups > kShare || (a.groups & (a.groups - 1)) != 0)
    return false;
  return !(a.bias && a.score == SAO_SCORE_SOFTMAX) && a.N >= int64_t(sms) * kRows * kListWarps;
}

sao_status route_lists_launch(const RouteArgs &a, const Lanes &l32, sao_dtype dt, int sms, cudaStream_t s) {
  const Lanes l{kShare / a.groups, 0, a.E / a.groups, a.groups};
  const int size = dt == SAO_BF16 ? 2 : 4;
  ListPlan p{};
  p.per = (l.size + l.share - 1) / l.share;
  p.blocks = (p.per + 7) / 8;
  while (p.mask < unsigned(a.E) - 1u) p.mask = 2 * p.mask + 1u;
  p.unit = 16;  // where rows, groups and lanes start on it
  while (p.unit >= 8 && (reinterpret_cast<uintptr_t>(a.x) % p.unit != 0 || a.E * size % p.unit != 0 ||
                         l.size * size % p.unit != 0 || (l.share > 1 && p.per * size % p.unit != 0)))
    p.unit /= 2;
  const int64_t grid = least((a.N + kRows * kListWarps - 1) / (kRows * kListWarps), int64_t(sms) * 16);
  const int slot = launch_begin("route_lists", s);
  const auto launch = [&](auto kernel) { pdl(kernel, unsigned(grid), kListWarps * 32, 0, s)(a, l, l32, p); };
  const bool rest = a.k == kList;
  if (a.bias && dt == SAO_BF16) {
    using T = __nv_bfloat16;
    rest ? launch(route_lists_kernel<T, true, true>) : launch(route_lists_kernel<T, true, false>);
  } else if (a.bias) {
    rest ? launch(route_lists_kernel<float, true, true>) : launch(route_lists_kernel<float, true, false>);
  } else if (dt == SAO_BF16) {
    launch(route_lists_kernel<__nv_bfloat16, false, false>);
  } else {
    rest ? launch(route_lists_kernel<float, false, true>) : launch(route_lists_kernel<float, false, false>);
  }
  return launch_end(slot, s);
}

}  // namespace sao
