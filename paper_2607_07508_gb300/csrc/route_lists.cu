// Routing to experts, the forms for many tokens: eight lanes take a row, each an eighth of its experts, and keep the
// largest eight keys of those in a sorted list; three exchanges merge the lists. Or a thread takes a row (below).
//
// A list costs 9 minima and maxima a key (a block of eight is sorted by a network of 19 exchanges and merged with eight maxima
// and 12 exchanges), where picking one expert after another from a warp's 32 lanes costs 11 to 20 instructions a pick and
// lane, and nothing is summed or compared over a whole warp. 8 of 65,536 x 128 fp32 19 to 22 us (205 instructions a row; by
// warps 23 us, 300), of 65,536 x 256 bf16 in groups with a bias 38 (410; 57, 675), of 2^20 x 160 bf16 in groups 282 (258;
// 419, 357): 335 MB of logits at 1.2 TB/s. The last is bound by the units of minima and maxima, 85 % busy. The others
// are not at a unit's limit: 72 % busy for 128 fp32 experts and 48 % with groups and a bias, with 56 to 62 % of the issue
// slots used, and a warp waits for its loads first. A block of logits is asked for and used at once, and 72 to 80
// registers leave 27 to 37 % of the warps to hide that.
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

// Eight logits from p on as they lie in memory, `n` of them there (others: -inf).
template <class T>
struct Block {
  static constexpr int kSize = int(sizeof(T)), kWords = 2 * kSize;
  uint32_t w[kWords];
  __device__ __forceinline__ void load(const T *p, int n, int unit) {
    if (unit == 16 && n >= 8) {
#pragma unroll
      for (int i = 0; i < kWords; i += 4) {
        const uint4 v = ld(reinterpret_cast<const uint4 *>(p) + i / 4);
        w[i] = v.x, w[i + 1] = v.y, w[i + 2] = v.z, w[i + 3] = v.w;
      }
    } else if (unit >= 8 && (n >= 8 || n * kSize % 8 == 0)) {
      constexpr uint32_t kNone = kSize == 4 ? 0xff800000u : 0xff80ff80u;
#pragma unroll
      for (int i = 0; i < kWords; i += 2) {
        uint2 v = make_uint2(kNone, kNone);
        if ((i + 2) * 4 <= n * kSize) v = ld(reinterpret_cast<const uint2 *>(p) + i / 2);
        w[i] = v.x, w[i + 1] = v.y;
      }
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        if constexpr (kSize == 4) {
          w[i] = i < n ? ld(reinterpret_cast<const uint32_t *>(p) + i) : 0xff800000u;
        } else {
          const uint32_t u = i < n ? ld(reinterpret_cast<const uint16_t *>(p) + i) : 0xff80u;
          w[i / 2] = i & 1 ? w[i / 2] | u << 16 : u;
        }
      }
    }
  }
  __device__ __forceinline__ float at(int i) const {
    if constexpr (kSize == 4) return __uint_as_float(w[i]);
    return __uint_as_float(i & 1 ? w[i / 2] & 0xffff0000u : w[i / 2] << 16);
  }
};

// The packed keys of a block of bf16 logits, the first of which has index `low` (the next ones lower): two at a time.
__device__ __forceinline__ void pack(const Block<__nv_bfloat16> &x, uint32_t low, uint32_t, uint32_t (&p)[8]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const __nv_bfloat162 zero = __floats2bfloat162_rn(0.f, 0.f);
    const __nv_bfloat162 sum = __hadd2(*reinterpret_cast<const __nv_bfloat162 *>(&x.w[i]), zero);  // (-0: 0)
    uint32_t u = *reinterpret_cast<const uint32_t *>(&sum);
    u ^= (u >> 15 & 0x00010001u) * 0x7fffu + 0x80008000u;  // both halves in the order of integers
    p[2 * i] = u * 0x10000u + (low - 2 * i);
    p[2 * i + 1] = (u & 0xffff0000u) + (low - 2 * i - 1);
  }
}
__device__ __forceinline__ void pack(const Block<float> &x, uint32_t low, uint32_t mask, uint32_t (&p)[8]) {
#pragma unroll
  for (int i = 0; i < 8; ++i) p[i] = (ordered(x.at(i) + 0.f) & ~mask) + (low - i);
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
    for (int e = threadIdx.x; e < 512; e += kListWarps * 32) {
      const float b = e < a.E ? ld(a.bias + e) : -INFINITY;
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
  const auto packed = [&](float x, int e) {  // as the blocks below, one expert
    if (kBiased) {
      const float f = fmaf(sigmoid_fast(x), units, offset[e]);
      return f >= 1.f && x > -INFINITY ? __float_as_uint(f) << 9 | (kFractionMask - e) : 0u;
    }
    return (ordered(x + 0.f) & ~mask) | (mask - e);  // -0 and 0 are one key; -inf comes to `none` or less
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
    bool odd = false;  // perhaps an infinity or a NaN
#pragma unroll 1
    for (int block = 0; block < plan.blocks; ++block) {
      const int here = on ? n - block * 8 : 0, e = e0 + block * 8;
      Block<T> x;
      x.load(from + block * 8, here, plan.unit);
      uint32_t w[8];
      if constexpr (kBiased) {
        float probe = 0.f;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          probe = fmaf(x.at(i), 0.f, probe);
          // (1: an expert that is out, as is one of a NaN)
          const float f = fmaxf(fmaf(sigmoid_fast(x.at(i)), units, offset[e + i]), 1.f);
          w[i] = __float_as_uint(f) * 512u + (kFractionMask - e - i);
        }
        if (probe != 0.f) {  // (places past the last expert are -inf too)
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            if (!(x.at(i) > -INFINITY)) w[i] = 0u;
            odd |= i < here && !(fabsf(x.at(i)) < INFINITY);
          }
        }
        sort8(w);
      } else {
        pack(x, mask - e, mask, w);
        sort8(w);
        if (here >= 8) {
          odd |= w[0] >= (0xff800000u & ~mask) || w[7] <= none;
        } else {
#pragma unroll
          for (int i = 0; i < 8; ++i) odd |= i < here && !(fabsf(x.at(i)) < INFINITY);
        }
      }
      if (block == 0) {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = w[i];
      } else {
        merge8<kRest>(v, w, rest);
      }
    }
    bool scores = on;
    if (__any_sync(kAll, on && odd)) {
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
    // whether two keys, the first of them not the smaller one, may be in another order than their exact values
    const auto near = [&](uint32_t p, uint32_t q) {
      if (kExact) return false;
      return p > none && q > none && (kBiased ? (p >> 9) - (q >> 9) <= apart : ((p ^ q) & ~mask) == 0u);
    };
    float top = 0.f;  // the row's largest logit, for exponentials
    if (!kBiased && soft && (!a.renorm || a.two)) {
      uint32_t first = v[0];
      for (int o = l.share; o < kShare; o <<= 1) first = max(first, __shfl_xor_sync(kAll, first, o));
      if (first > none) top = value(logits + (mask - (first & mask)));
      if constexpr (!kExact) {
        // Of logits that share the leading bits of the first one's key another may be the largest, and of large ones by more
        // than an exponential has room for.
        const bool blurred = row_any(near(first, v[1]) || (v[0] != first && near(first, v[0])));
        if (__any_sync(kAll, blurred)) {
          for (int i = 0; i < (blurred ? n : 0); ++i) top = fmaxf(top, value(from + i));
          for (int o = 1; o < kShare; o <<= 1) top = fmaxf(top, __shfl_xor_sync(kAll, top, o));
        }
      }
    }
    const auto exactly = [&](float x, float b) { return kBiased ? sigmoid(double(x)) + double(b) : double(x); };
    bool again = all_exactly, stays = true;  // again: choose_exactly
    if (l.groups > 1) {
      const bool one = v[0] > none, both = v[1] > none;
      float worth = -INFINITY, x0 = 0.f, x1 = -INFINITY;  // the best two logits, where they are looked at
      if (kBiased) {
        const auto key = [&](uint32_t p) {
          return (__uint_as_float(0x3f800000u | p >> 9) - kFractionLeast) / units + least;
        };
        if (one) worth = key(v[0]) + (a.two && both ? key(v[1]) : 0.f);
      } else if (a.two) {
        // scores of the two best logits (softmax: times their common sum)
        if (one) x0 = value(logits + (mask - (v[0] & mask)));
        if (both) x1 = value(logits + (mask - (v[1] & mask)));
        if constexpr (!kExact) {
          // An fp32 key has lost up to nine bits of its logit, 2^-14 of it: of those that share the second one's leading
          // bits the list has the first, not the largest. The group's logits themselves tell.
          const bool blurred = both && near(v[1], v[2]);
          if (__any_sync(kAll, blurred)) {
            float b1 = -INFINITY, b2 = -INFINITY;
            for (int i = 0; i < (blurred ? n : 0); ++i) {
              const float x = value(from + i);
              b2 = fmaxf(b2, fminf(b1, x));
              b1 = fmaxf(b1, x);
            }
            for (int o = 1; o < l.share; o <<= 1) {
              const float c1 = __shfl_xor_sync(kAll, b1, o), c2 = __shfl_xor_sync(kAll, b2, o);
              merge_two(b1, b2, c1, c2);
            }
            if (blurred) x0 = b1, x1 = b2;
          }
        }
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
        if (__any_sync(kAll, doubt)) {  // ranked again by fp64
          const bool plain = !kBiased && a.two;  // x0 and x1 are there, and certain
          const int id0 = one ? int(mask - (v[0] & mask)) : -1, id1 = a.two && both ? int(mask - (v[1] & mask)) : -1;
          if (!plain) {
            x0 = id0 >= 0 ? value(logits + id0) : 0.f;
            x1 = id1 >= 0 ? value(logits + id1) : 0.f;
          }
          const float b0 = kBiased && id0 >= 0 ? ld(a.bias + id0) : 0.f;
          const float b1 = kBiased && id1 >= 0 ? ld(a.bias + id1) : 0.f;
          const auto term = [&](float x, float b) {
            if (kBiased || !a.two) return exactly(x, b);
            return soft ? exp(double(x) - double(top)) : sigmoid(double(x));
          };
          const double fine = one ? term(x0, b0) + (id1 >= 0 ? term(x1, b1) : 0.0) : -INFINITY;
          const bool border = fabsf(worth - lowest) <= 2.f * error || fabsf(worth - highest) <= 2.f * error;
          // uncertain: keys about the last of those, unless they are of one logit and bias
          const uint32_t least_of = a.two ? v[1] : v[0];
          const float x_of = a.two ? x1 : x0, b_of = a.two ? b1 : b0;
          const bool unsure = !plain && doubt && border && near(least_of, a.two ? v[2] : v[1]);
          if (__any_sync(kAll, unsure)) {
            int mixed = 0;
            for (int i = 0; i < (unsure ? n : 0); ++i) {
              const float x = value(from + i);
              const uint32_t p = packed(x, e0 + i);
              if (!(p > none && (p > least_of ? near(p, least_of) : near(least_of, p)))) continue;
              mixed |= !(x == x_of && (!kBiased || ld(a.bias + e0 + i) == b_of));
            }
            again |= row_any(mixed != 0);
          }
          rank = 0;
          for (int o = l.share; o < kShare; o += l.share) {
            const double other = __shfl_xor_sync(kAll, fine, o);
            rank += other > fine || (other == fine && (s ^ o) < s);
          }
          if (doubt) stays = rank < a.kept;
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
      const float bias = kBiased && id >= 0 ? ld(a.bias + id) : 0.f;
      // picks among one another
      const uint32_t after = __shfl_down_sync(kAll, pick, 1);
      const float x_after = __shfl_down_sync(kAll, chosen, 1), b_after = __shfl_down_sync(kAll, bias, 1);
      const bool swap = id >= 0 && s < a.k - 1 && near(pick, after) && !(chosen == x_after && bias == b_after);
      // the last one and what was left out: nothing to do if all keys about it are of one logit and bias
      const bool border = scores && near(last, next);
      bool compare = false;  // the one key left out that is about the last one may have to be a pick
      if (__any_sync(kAll, border)) {
        const int at = int(mask - (last & mask));
        const float x_last = border ? value(logits + at) : 0.f, b_last = kBiased && border ? ld(a.bias + at) : 0.f;
        bool mixed = false;
        int left = 0;
        for (int i = 0; i < (border && stays ? n : 0); ++i) {
          const float x = value(from + i);
          const uint32_t p = packed(x, e0 + i);
          if (!(p > none && (p > last ? near(p, last) : near(last, p)))) continue;
          left += p < last;
          mixed |= !(x == x_last && (!kBiased || ld(a.bias + e0 + i) == b_last));
        }
        for (int o = 1; o < kShare; o <<= 1) left += __shfl_xor_sync(kAll, left, o);
        mixed = row_any(mixed);
        compare = mixed && left == 1;
        again |= mixed && left != 1;
      }
      if (__any_sync(kAll, swap || compare)) {
        double key = id >= 0 ? exactly(chosen, bias) : -INFINITY;
        const auto rank_of = [&] {
          int rank = 0;
          for (int o = 1; o < kShare; ++o) {
            const double other = __shfl_xor_sync(kAll, key, o);
            const int its = __shfl_xor_sync(kAll, id, o);
            rank += other > key || (other == key && (id < 0 ? (s ^ o) < s : its >= 0 && its < id));
          }
          return rank;
        };
        int rank = rank_of();
        if (__any_sync(kAll, compare)) {
          const int its = compare ? int(mask - (next & mask)) : 0;
          const float x = compare ? value(logits + its) : 0.f, b = kBiased && compare ? ld(a.bias + its) : 0.f;
          const double k = exactly(x, b);
          if (compare && rank == a.k - 1 && (k > key || (k == key && its < id))) id = its, chosen = x, key = k;
          rank = rank_of();
        }
        int source = lane;
        for (int i = 0; i < kShare; ++i) {
          const int its = __shfl_sync(kAll, rank, base + i);
          if (its == s) source = base + i;
        }
        id = __shfl_sync(kAll, id, source);
        chosen = __shfl_sync(kAll, chosen, source);
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
      const float sum = share_sum(sum_of_exponentials<4>(from, scores ? n : 0, top), 0, kShare, true);
      if (id >= 0) w = expf(chosen - top) / sum;
    }
    if (real && s < a.k) {
      a.ids[row * a.k + s] = id;
      a.weights[row * a.k + s] = id >= 0 ? a.scale * w : 0.f;
    }
  }
}

// The same with a thread to a row, nothing to merge or to sum with another lane: up to 32 experts in registers (kBlocks
// of eight), or, kBlocks 0, one group and no softmax with a bias, any number of blocks one after another. Choices
// and weights go through shared memory, so that a warp's 32 rows are stored together.
// 395,545 x 15 bf16 with a softmax and a bias 23 us, 65,536 x 8 fp32 5 (a warp to a row 105 and 15).
template <class T, int kBlocks, bool kBiased>
__global__ void __launch_bounds__(kListWarps * 32)
    route_rows_kernel(const __grid_constant__ RouteArgs a, const __grid_constant__ Lanes l32, ListPlan plan) {
  grid_wait();
  constexpr bool kExact = !kBiased && sizeof(T) == 2, kLong = kBlocks == 0;
  constexpr int kPlaces = kLong ? 512 : 8 * kBlocks;  // biases
  __shared__ float all_offsets[kBiased ? (kLong ? 1 : kListWarps) * kPlaces : 1];
  __shared__ int all_ids[kListWarps][32 * kList];
  __shared__ float all_weights[kListWarps][32 * kList];
  const int lane = threadIdx.x & 31, warp = threadIdx.x / 32;
  int *its_ids = all_ids[warp];
  float *its_weights = all_weights[warp], *offset = all_offsets + (kLong ? 0 : warp * kPlaces);
  __shared__ uint32_t all_worths[kLong ? 1 : kListWarps * 32 * 32];  // of each group, by lanes
  uint32_t *worths = all_worths + (kLong ? 0 : warp * 32 * 32) + lane;
  const bool soft = a.score == SAO_SCORE_SOFTMAX, sums = soft && (kBiased || !a.renorm);
  float units = 1.f, least = 0.f;
  bool all_exactly = false;
  if (kBiased) {  // keys as fractions, as above
    float low = INFINITY, high = -INFINITY, most = -INFINITY;
    for (int e = lane; e < a.E; e += 32) {
      const float b = ld(a.bias + e);
      most = fmaxf(most, b);
      if (fabsf(b) < INFINITY) low = fminf(low, b), high = fmaxf(high, b);
    }
    low = -warp_max(-low), high = warp_max(high), most = warp_max(most);
    if (high < low) low = high = 0.f;
    least = low;
    units = (1.f - 0x1p-9f) / (1.f + (high - low));
    all_exactly = most == INFINITY || !(units >= 0x1p-20f);
    for (int e = kLong ? int(threadIdx.x) : lane; e < kPlaces; e += kLong ? kListWarps * 32 : 32) {
      const float b = e < a.E ? ld(a.bias + e) : -INFINITY;
      offset[e] = fabsf(b) < INFINITY ? fmaf(b - low, units, kFractionLeast) : -INFINITY;
    }
    __syncthreads();
  }
  const uint32_t mask = kExact ? 0xffffu : kBiased ? kFractionMask : plan.mask;
  const uint32_t none = kExact ? 0x007fffffu : kBiased ? kFractionMask : 0x007fffffu | mask;
  const int64_t step = int64_t(gridDim.x) * kListWarps * 32;
  for (int64_t row0 = (int64_t(blockIdx.x) * kListWarps + warp) * 32; row0 < a.N; row0 += step) {
    const int rows = int(a.N - row0 < 32 ? a.N - row0 : 32);
    const bool on = lane < rows && (a.mask == nullptr || ld(a.mask + row0 + lane) != 0);
    const T *logits = static_cast<const T *>(a.x) + (row0 + (lane < rows ? lane : 0)) * a.E;
    bool bad = false;
    float top = -INFINITY, total = 1.f, inverse = 1.f;
    uint32_t v[8], rest = 0u;
    const auto fraction = [&](float x, float s, int e) {  // of score s; 1: out
      return x > -INFINITY ? fmaxf(fmaf(s, units, offset[e]), 1.f) : 1.f;
    };
    const auto key = [&](float x, float s, int e) {
      return __float_as_uint(fraction(x, s, e)) * 512u + (kFractionMask - e);
    };
    bool again = all_exactly;
    const auto take = [&](uint32_t(&w)[8], bool first) {
      sort8(w);
      if (first) {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = w[i];
      } else {
        merge8<!kExact>(v, w, rest);
      }
    };
    const auto look = [&](float x) {
      bad |= !(x < INFINITY) && (soft || x != x);
      top = fmaxf(top, x);
    };
    if constexpr (kLong) {
      Block<T> x, ahead;
      ahead.load(logits, on ? a.E : 0, plan.unit);
#pragma unroll 1
      for (int b = 0; b < plan.blocks; ++b) {
        x = ahead;
        if (b + 1 < plan.blocks) ahead.load(logits + 8 * b + 8, on ? a.E - 8 * b - 8 : 0, plan.unit);
#pragma unroll
        for (int i = 0; i < 8; ++i) look(x.at(i));
        if (a.replay) continue;
        uint32_t w[8];
        if constexpr (kBiased) {
#pragma unroll
          for (int i = 0; i < 8; ++i) w[i] = key(x.at(i), sigmoid_fast(x.at(i)), 8 * b + i);
        } else {
          pack(x, mask - 8 * b, mask, w);
        }
        take(w, b == 0);
      }
      if (sums && on) {
        total = sum_of_exponentials<8>(logits, a.E, top);
        inverse = 1.f / total;
      }
    } else {
      Block<T> x[kBlocks];
#pragma unroll
      for (int b = 0; b < kBlocks; ++b) x[b].load(logits + 8 * b, on ? a.E - 8 * b : 0, plan.unit);
#pragma unroll
      for (int b = 0; b < kBlocks; ++b)
#pragma unroll
        for (int i = 0; i < 8; ++i) look(x[b].at(i));
      float e[kBlocks][8];
      if (sums) {
        total = 0.f;
#pragma unroll
        for (int b = 0; b < kBlocks; ++b)
#pragma unroll
          for (int i = 0; i < 8; ++i) {  // (where weights have this sum's error it is that of expf)
            const float d = x[b].at(i) - top;
            total += e[b][i] = a.renorm ? exp_fast(d) : expf(d);
          }
        inverse = 1.f / total;
      }
      float f[kBiased ? kBlocks : 1][8];
      if (kBiased) {
#pragma unroll
        for (int b = 0; b < kBlocks; ++b)
#pragma unroll
          for (int i = 0; i < 8; ++i)
            f[b][i] = fraction(x[b].at(i), soft ? e[b][i] * inverse : sigmoid_fast(x[b].at(i)), 8 * b + i);
      }
      unsigned stay = kAll;  // groups
      if (a.groups > 1 && !a.replay) {
        const int size = a.E / a.groups;
        const float out = kBiased ? 1.f : -INFINITY;
        float b1 = out, b2 = out;
        int group = 0, inside = 0;
#pragma unroll
        for (int b = 0; b < kBlocks; ++b)
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            if (group == a.groups) continue;
            const float v = kBiased ? f[kBiased ? b : 0][i] : x[b].at(i) + 0.f;
            b2 = fmaxf(b2, fminf(b1, v));
            b1 = fmaxf(b1, v);
            if (++inside < size) continue;
            float worth = b1;
            if (a.two) {
              if (kBiased)
                worth = (b1 - kFractionLeast) / units + least +
                        (b2 > out ? (b2 - kFractionLeast) / units + least : 0.f);
              else
                worth = soft ? exp_fast(b1 - top) + exp_fast(b2 - top) : sigmoid_fast(b1) + sigmoid_fast(b2);
            }
            worths[32 * group] = b1 > out ? (ordered(worth) & ~31u) | (31u - group) : 0u;
            b1 = b2 = out, inside = 0, ++group;
          }
        uint32_t last = ~0u;
        for (int c = 0; c < a.kept; ++c) {
          uint32_t best = 0u;
          for (int g = 0; g < a.groups; ++g) {
            const uint32_t u = worths[32 * g];
            best = max(best, u < last ? u : 0u);
          }
          last = best;
        }
        uint32_t after = 0u;
        stay = 0u;
        for (int g = 0; g < a.groups; ++g) {
          const uint32_t u = worths[32 * g];
          stay |= u >= last ? 1u << g : 0u;
          after = max(after, u < last ? u : 0u);
        }
        if (after != 0u && (!kExact || a.two)) {
          const float p = unordered(last & ~31u), q = unordered(after & ~31u), reach = fabsf(p) + fabsf(q);
          float error = 0x1p-18f * reach;  // of the five bits
          if (kBiased && !a.two)
            error += 0x1p-16f * (soft ? inverse : 0x1p-3f) * units + 0x1p-20f;
          else if (a.two)
            error += 0x1p-18f + 0x1p-20f / units + 0x1p-21f * reach + (kBiased && soft ? 0x1p-15f * inverse : 0.f);
          again |= !(p - q > error);
        }
      }
      int group = 0, inside = 0;
      const int size = a.groups > 1 ? a.E / a.groups : 64;
#pragma unroll
      for (int b = 0; b < kBlocks; ++b) {
        uint32_t w[8];
        if constexpr (kBiased) {
#pragma unroll
          for (int i = 0; i < 8; ++i) w[i] = __float_as_uint(f[b][i]) * 512u + (kFractionMask - 8 * b - i);
        } else {
          pack(x[b], mask - 8 * b, mask, w);
        }
        if (a.groups > 1) {
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            if (!(stay >> group & 1u)) w[i] = 0u;
            if (++inside == size) inside = 0, group = group < 31 ? group + 1 : 31;
          }
        }
        take(w, b == 0);
      }
    }
    if (bad) raise_device_error(a.err, SAO_DEVERR_LOGITS);
    const bool scores = on && !bad && top > -INFINITY;
    // two fractions are off by twice a score's error (of a softmax 2^-18 of its largest, which `inverse` is) and 3 2^-23
    const uint32_t apart = !kBiased ? 0u : uint32_t((soft ? 64.f * inverse : 8.f) * units) + 5u;
    const auto near = [&](uint32_t p, uint32_t q) {  // p >= q
      return p > none && q > none && (kBiased ? (p >> 9) - (q >> 9) <= apart : ((p ^ q) & ~mask) == 0u);
    };
    bool border = false;
    if (a.replay) {
      for (int t = lane; t < rows * a.k; t += 32) {
        int id = ld(a.ids + row0 * a.k + t);
        if (id >= a.E) {  // (an error where the row takes part)
          if (a.mask == nullptr || ld(a.mask + row0 + t / a.k) != 0) raise_device_error(a.err, SAO_DEVERR_EXPERT_ID);
          id = -1;
        }
        its_ids[t] = id;
      }
      again = false;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      if (i >= a.k || a.replay) continue;
      const int id = scores && v[i] > none ? int(mask - (v[i] & mask)) : -1;
      its_ids[lane * a.k + i] = id;
      const uint32_t q = i < 7 ? v[i < 7 ? i + 1 : 7] : rest;
      if (!kExact && id >= 0 && near(v[i], q)) {
        // those of one logit and bias are equal, but about the last choice a third one may be as near
        const int next = int(mask - (q & mask));
        bool same = value(logits + id) == value(logits + next);
        if (kBiased) same = same && ld(a.bias + id) == ld(a.bias + next);
        again |= !same;
        border |= i == a.k - 1;
      }
    }
    if (!kExact && border && !again) {
      uint32_t last = 0u;
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (i == a.k - 1) last = v[i];
      const int at = int(mask - (last & mask));
      const float x_last = value(logits + at), b_last = kBiased ? ld(a.bias + at) : 0.f;
      for (int e = 0; e < a.E; ++e) {
        const float x = value(logits + e);
        uint32_t p;
        if constexpr (kBiased)
          p = key(x, soft ? exp_fast(x - top) * inverse : sigmoid_fast(x), e);
        else
          p = (ordered(x + 0.f) & ~mask) + (mask - e);
        if (p > last ? near(p, last) : near(last, p))
          again |= !(x == x_last && (!kBiased || ld(a.bias + e) == b_last));
      }
    }
    __syncwarp();
    unsigned todo = __ballot_sync(kAll, again && scores);
    while (todo != 0u) {
      const int r = __ffs(todo) - 1;
      todo &= todo - 1u;
      const T *its_row = static_cast<const T *>(a.x) + (row0 + r) * a.E;
      const int found =
          choose_exactly<T, kLong ? 16 : 2, kBiased>({a.bias, a.k, a.kept, soft, a.two != 0}, l32, its_row);
      if (lane < a.k) its_ids[r * a.k + lane] = found;
      __syncwarp();
    }
    float c[8], m = -INFINITY, sum = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int id = i < a.k && scores ? its_ids[lane * a.k + i] : -1;
      c[i] = id >= 0 ? value(logits + id) : -INFINITY;
      m = fmaxf(m, soft ? c[i] : fminf(c[i], 0.f));
    }
    if (a.renorm) {
      // sigmoid(x) = exp(min(x, 0)) / (1 + exp(-|x|)): relative to the largest, no sum vanishes
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        float t = m > -INFINITY ? expf((soft ? c[i] : fminf(c[i], 0.f)) - m) : 0.f;
        if (!soft) t /= 1.f + expf(-fabsf(c[i]));
        sum += c[i] = t;
      }
      const float f = sum > 0.f ? 1.f / sum : 0.f;
#pragma unroll
      for (int i = 0; i < 8; ++i) c[i] *= f;
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i)
        c[i] = !soft ? sigmoid(c[i]) : c[i] > -INFINITY ? expf(c[i] - top) * inverse : 0.f;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (i < a.k) its_weights[lane * a.k + i] = scores && its_ids[lane * a.k + i] >= 0 ? a.scale * c[i] : 0.f;
    __syncwarp();
    for (int t = lane; t < rows * a.k; t += 32) {
      if (!a.replay) a.ids[row0 * a.k + t] = its_ids[t];
      a.weights[row0 * a.k + t] = its_weights[t];
    }
    __syncwarp();
  }
}

}  // namespace

// A thread to a row: up to 32 experts from 32 rows for each SM on; more of them take a thread long, and pay where there are
// threads enough (and by eight lanes: 65,536 x 40 bf16 9 us and 13, 400,000 x 64 fp32 48 and 77, x 128 75 and 99, 65,536 x
// 128 both 22, 20,000 x 128 16 and 12; 400,000 x 256 bf16 with a bias 144 and 179, without 107 and 104).
bool route_rows_take(const RouteArgs &a, int sms) {
  if (a.k > kList) return false;
  if (a.E <= 32) return a.N >= int64_t(sms) * 32;
  if (a.groups != 1) return false;
  if (a.bias && a.score == SAO_SCORE_SOFTMAX) return false;
  return (a.E <= 64 && a.N >= int64_t(sms) * 256) || (a.E <= (a.bias ? 256 : 128) && a.N >= int64_t(sms) * 1024);
}

bool route_lists_take(const RouteArgs &a, int sms) {
  if (route_rows_take(a, sms)) return true;
  if (a.replay || a.k > kList || a.E < 16 || a.E > 512 || a.groups > kShare || (a.groups & (a.groups - 1)) != 0)
    return false;
  return !(a.bias && a.score == SAO_SCORE_SOFTMAX) && a.N >= int64_t(sms) * kRows * kListWarps;
}

sao_status route_rows_launch(const RouteArgs &a, const Lanes &l32, sao_dtype dt, int sms, cudaStream_t s) {
  const int size = dt == SAO_BF16 ? 2 : 4;
  ListPlan p{a.E, (a.E + 7) / 8, 16, 7u};
  while (p.mask + 1u < 8u * (p.blocks == 3 ? 4 : p.blocks)) p.mask = 2 * p.mask + 1u;
  while (p.unit >= 8 && (reinterpret_cast<uintptr_t>(a.x) % p.unit != 0 || a.E * size % p.unit != 0)) p.unit /= 2;
  const int64_t tiles = (a.N + 32 * kListWarps - 1) / (32 * kListWarps), most = int64_t(sms) * 128;
  const int slot = launch_begin("route_rows", s);
  SAO_TRY(by_type(dt, [&](auto t) {
    using T = decltype(t);
    const auto launch = [&](auto biased, auto plain) {
      pdl(a.bias ? biased : plain, unsigned(least(tiles, most)), kListWarps * 32, 0, s)(a, l32, p);
      return SAO_OK;
    };
    if (p.blocks == 1) return launch(route_rows_kernel<T, 1, true>, route_rows_kernel<T, 1, false>);
    if (p.blocks == 2) return launch(route_rows_kernel<T, 2, true>, route_rows_kernel<T, 2, false>);
    if (p.blocks <= 4) return launch(route_rows_kernel<T, 4, true>, route_rows_kernel<T, 4, false>);
    return launch(route_rows_kernel<T, 0, true>, route_rows_kernel<T, 0, false>);
  }));
  return launch_end(slot, s);
}

sao_status route_lists_launch(const RouteArgs &a, const Lanes &l32, sao_dtype dt, int sms, cudaStream_t s) {
  if (route_rows_take(a, sms)) return route_rows_launch(a, l32, dt, sms, s);
  const Lanes l{kShare / a.groups, 0, a.E / a.groups, a.groups};
  const int size = dt == SAO_BF16 ? 2 : 4;
  ListPlan p{};
  p.per = (l.size + l.share - 1) / l.share;
  p.blocks = (p.per + 7) / 8;
  // (the last lane's blocks may reach past the last expert: 511 at most)
  const int e_most = (kShare - 1) / l.share * l.size + (kShare - 1) % l.share * p.per + p.blocks * 8 - 1;
  while (p.mask < unsigned(e_most)) p.mask = 2 * p.mask + 1u;
  p.unit = 16;  // where rows, groups and lanes start on it
  while (p.unit >= 8 && (reinterpret_cast<uintptr_t>(a.x) % p.unit != 0 || a.E * size % p.unit != 0 ||
                         l.size * size % p.unit != 0 || (l.share > 1 && p.per * size % p.unit != 0)))
    p.unit /= 2;
  // as many CTAs as there is work for, or, with a bias to set up, few that take equal shares
  const int64_t tiles = (a.N + kRows * kListWarps - 1) / (kRows * kListWarps);
  const int64_t most = int64_t(sms) * (a.bias ? 6 : 128), turns = (tiles + most - 1) / most;
  const int64_t grid = (tiles + turns - 1) / turns;
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
