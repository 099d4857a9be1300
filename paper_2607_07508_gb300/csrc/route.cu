// Routing to experts: each token's k experts and their weights.
//
//   s_e = softmax(x)_e or sigmoid(x_e),  key_e = s_e + bias_e,  the k largest keys of the groups that stay
//   w_j = scale s_j, over the sum of the chosen s where weights are renormalised
//
// Softmax and sigmoid keep the logits' order: without a bias experts are picked by their logits, which is exact, and
// renormalised weights need the chosen logits alone. Keys with a bias (and sums of two keys) are formed in fp32; where
// two of them are nearer to one another than their errors, and not of the same logit and bias, fp64 decides.
//
// This form takes what route_lists.cu does not: few tokens, more than eight experts a token or 512 in all, and, among more
// than 32 experts, softmax with a bias, groups that are no power of two, and replayed choices (which a thread to a row
// takes among up to 64 experts from 256 tokens for each SM on, among up to 128 from 1,024). A warp to a row keeps latency
// low: 7 x 256 in groups 7.2 us with nothing in the caches. With many rows its instructions count, 11 to 20 a pick and
// lane: 65,536 x 256 with 10 experts a token take 32 us in bf16 and 38 in fp32, 6 and 4 times their bytes at the rate of
// HBM, with 70 % of the issue slots used at 34 % of the warps; a warp waits first for the instruction before, its picks
// being a chain of reductions.
#include "route_exact.cuh"

namespace sao {
namespace {

using namespace route;

// A lane's logits of one row as they lie in memory: vectors of up to 16 bytes where they are aligned to those (kWide).
template <class T, int kPer>
struct Logits {
  static constexpr bool kCanWide = kPer >= 2 && (kPer & (kPer - 1)) == 0;
  uint32_t w[kPer];
  __device__ __forceinline__ void load(const T *p, int n, bool full, bool wide) {
    if constexpr (kCanWide) {
      constexpr int kWords = kPer * int(sizeof(T)) / 4;
      if (wide) {
        if constexpr (kWords == 1) {
          w[0] = ld(reinterpret_cast<const uint32_t *>(p));
        } else if constexpr (kWords == 2) {
          const uint2 v = ld(reinterpret_cast<const uint2 *>(p));
          w[0] = v.x, w[1] = v.y;
        } else {
#pragma unroll
          for (int i = 0; i < kWords; i += 4) {
            const uint4 v = ld(reinterpret_cast<const uint4 *>(p) + i / 4);
            w[i] = v.x, w[i + 1] = v.y, w[i + 2] = v.z, w[i + 3] = v.w;
          }
        }
        return;
      }
    }
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      w[i] = 0u;
      if (full || i < n) {
        if constexpr (sizeof(T) == 2)
          w[i] = ld(reinterpret_cast<const uint16_t *>(p) + i);
        else
          w[i] = ld(reinterpret_cast<const uint32_t *>(p) + i);
      }
    }
  }
  __device__ __forceinline__ void get(float (&x)[kPer], bool wide) const {
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      if constexpr (sizeof(T) == 4) {
        x[i] = __uint_as_float(w[i]);
      } else {
        if (kCanWide && wide)
          x[i] = __uint_as_float(i & 1 ? w[i / 2] & 0xffff0000u : w[i / 2] << 16);
        else
          x[i] = __uint_as_float(w[i] << 16);
      }
    }
  }
};

// How a call's rows are taken.
struct Plan {
  int batch;      // consecutive rows of a warp at a time: their choices fill its lanes
  uint32_t mask;  // the bits of a packed key that hold the expert
  int wide;       // rows are aligned for vectors
};

// A warp takes `batch` rows, one after another up to the choices, which come to lie in lane r k + j; their weights
// are then computed and written for all of them at once.
//
// Keys are packed: bits in the order of integers, the lowest of them replaced by the expert's index (inverted:
// the lower of equal ones is the larger), so that a pick is one integer maximum over the warp and gives key and
// index, and the next one is the largest below it: p - m, as unsigned numbers, is larger for each p < m than for
// any other. A bf16 logit has room for the index. Other keys are packed by their distance d from the row's
// largest, whose leading bits say most where it counts: those of the picks are small. Neighbours that differ in
// the replaced bits alone, or by less than their errors, are looked at again (choose_exactly) unless they are of
// one logit and bias.
//
// kFull: 32 kPer experts, no lane with fewer than another.
template <class T, int kPer, bool kFull, bool kBiased>
__global__ void __launch_bounds__(kWarps * 32, kPer <= 4 ? 5 : kPer <= 8 ? 3 : 1)
    route_fwd_kernel(const __grid_constant__ RouteArgs a, const __grid_constant__ Lanes l, Plan plan) {
  grid_wait();
  constexpr bool kExact = !kBiased && sizeof(T) == 2;
  const int lane = threadIdx.x & 31;
  const int e0 = kFull ? lane * kPer : first_of(l, lane), n = kFull ? kPer : count_of(l, lane);
  const bool soft = a.score == SAO_SCORE_SOFTMAX, wide = kFull && plan.wide;
  const bool sums = soft && (kBiased || !a.renorm), need_top = sums || (soft && a.two && l.groups > 1);
  const uint32_t mask = kExact ? 0xffffu : plan.mask, low = mask - uint32_t(e0);
  const auto index = [&](int i) { return kFull ? low - i : (low - i) & mask; };
  // no packed key of an expert that can be chosen is below it (-inf, or a distance of inf)
  const uint32_t none = (kExact ? 0x007fffffu : 0x00ffffffu) | mask;
  const int mine = lane / a.k, j = lane - mine * a.k, first = mine * a.k;
  const bool even = (a.k & (a.k - 1)) == 0;
  float b[kPer];
  if (kBiased) {
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      b[i] = -INFINITY;
      if (kFull || i < n) b[i] = fmaxf(ld(a.bias + e0 + i), -INFINITY);  // (a NaN is out as well)
    }
  }
  const int64_t step = int64_t(gridDim.x) * kWarps * plan.batch;
  for (int64_t row0 = (int64_t(blockIdx.x) * kWarps + threadIdx.x / 32) * plan.batch; row0 < a.N; row0 += step) {
    const int rows = int(a.N - row0 < plan.batch ? a.N - row0 : plan.batch);
    unsigned on = rows == 32 ? kAll : (1u << rows) - 1u;
    if (a.mask) on &= __ballot_sync(kAll, lane < rows && ld(a.mask + row0 + (lane < rows ? lane : 0)) != 0);
    unsigned good = 0u;             // rows with scores
    unsigned doubt = 0u;            // rows whose groups are in doubt, or whose keys have no distances
    uint32_t pick = 0u, next = 0u;  // this lane's choice; the key after the row's last one
    float peak = 0.f, total = 1.f;  // of this lane's row, where they are needed: largest logit, sum of exponentials
    const T *from = static_cast<const T *>(a.x) + row0 * a.E + e0;
    Logits<T, kPer> ahead;
    ahead.load(from, n, kFull, wide);
    for (int r = 0; r < rows; ++r) {
      float x[kPer];
      ahead.get(x, wide);
      from += a.E;
      if (r + 1 < rows) ahead.load(from, n, kFull, wide);
      if (!(on >> r & 1u)) continue;
      float probe = 0.f;
#pragma unroll
      for (int i = 0; i < kPer; ++i) probe = fmaf(x[i], 0.f, probe);
      bool out = false;  // some logit is -inf
      if (__any_sync(kAll, probe != 0.f)) {  // a NaN or an infinity
        bool bad = false;
#pragma unroll
        for (int i = 0; i < kPer; ++i) bad |= !(x[i] < INFINITY) && (soft || x[i] != x[i]);
        if (__any_sync(kAll, bad)) {
          if (lane == 0) raise_device_error(a.err, SAO_DEVERR_LOGITS);
          continue;
        }
        out = true;
      }
      if (!kFull) {
#pragma unroll
        for (int i = 0; i < kPer; ++i) x[i] = i < n ? x[i] : -INFINITY;
      }
      float top = 0.f, inverse = 1.f;
      if (need_top || out) {
        top = x[0];
#pragma unroll
        for (int i = 1; i < kPer; ++i) top = fmaxf(top, x[i]);
        top = warp_max(top);
        if (!(top > -INFINITY)) continue;
      }
      good |= 1u << r;
      float key[kPer];
      if (sums) {
        constexpr int kParts = kPer > 32 ? 2 : 1;  // chains of 32 additions at most
        float part[kParts] = {};
        if (a.renorm) {
#pragma unroll
          for (int i = 0; i < kPer; ++i) part[i % kParts] += key[i] = exp_fast(x[i] - top);
        } else {  // the weights have this sum's error
#pragma unroll
          for (int i = 0; i < kPer; ++i) part[i % kParts] += key[i] = expf(x[i] - top);
        }
        float sum = part[0];
        if (kParts > 1) sum += part[kParts - 1];
        sum = warp_sum(sum);
        inverse = 1.f / sum;
        if (mine == r) peak = top, total = sum;
      }
      if (a.replay) continue;
      if (kBiased) {
        if (soft) {
#pragma unroll
          for (int i = 0; i < kPer; ++i) key[i] = fmaf(key[i], inverse, b[i]);
        } else {
#pragma unroll
          for (int i = 0; i < kPer; ++i) key[i] = sigmoid_fast(x[i]) + b[i];
        }
        if (out) {
#pragma unroll
          for (int i = 0; i < kPer; ++i) key[i] = x[i] > -INFINITY ? key[i] : -INFINITY;
        }
      } else {
#pragma unroll
        for (int i = 0; i < kPer; ++i) key[i] = x[i] + 0.f;  // -0 and 0 are one key
      }
      float b1 = -INFINITY;
      if (l.groups > 1) {
        float b2 = -INFINITY;
        if (a.two) {
#pragma unroll
          for (int i = 0; i < kPer; ++i) {
            b2 = fmaxf(b2, fminf(b1, key[i]));
            b1 = fmaxf(b1, key[i]);
          }
          for (int o = 1; o < l.share; o <<= 1) {
            const float c1 = __shfl_xor_sync(kAll, b1, o), c2 = __shfl_xor_sync(kAll, b2, o);
            merge_two(b1, b2, c1, c2);
          }
        } else {
#pragma unroll
          for (int i = 0; i < kPer; ++i) b1 = fmaxf(b1, key[i]);
          for (int o = 1; o < l.share; o <<= 1) b1 = fmaxf(b1, __shfl_xor_sync(kAll, b1, o));
        }
        float v = b1;
        if (a.two && b1 > -INFINITY) {
          if (kBiased)
            v = b2 > -INFINITY ? b1 + b2 : b1;
          else
            v = soft ? exp_fast(b1 - top) + exp_fast(b2 - top) : sigmoid_fast(b1) + sigmoid_fast(b2);
        }
        // picked like experts, the group in the last five bits
        const int group = lane / l.share;
        const uint32_t u = v > -INFINITY && group < l.groups ? (ordered(v) & ~31u) | (31u - group) : 0u;
        uint32_t last = __reduce_max_sync(kAll, u);
        for (int i = 1; i < a.kept; ++i) last = __reduce_max_sync(kAll, u < last ? u : 0u);
        if (!kExact || a.two) {
          const uint32_t after = __reduce_max_sync(kAll, u < last ? u : 0u);
          if (after != 0u) {
            const float p = unordered(last & ~31u), q = unordered(after & ~31u), size = fabsf(p) + fabsf(q);
            float error = 0x1p-18f * size;  // of the five bits
            if (kBiased || a.two)
              error += 2.f * (soft ? kDoubtSoftmax * (kBiased ? inverse : 1.f) : kDoubtSigmoid) + 0x1p-22f * size;
            if (!(p - q > error)) doubt |= 1u << r;
          }
        }
        if (u < last) {
          b1 = -INFINITY;
#pragma unroll
          for (int i = 0; i < kPer; ++i) key[i] = -INFINITY;
        }
      }
      uint32_t p[kPer];
      if (kExact) {
#pragma unroll
        for (int i = 0; i < kPer; ++i) p[i] = (ordered(key[i]) & ~mask) | index(i);
      } else {
        if (l.groups == 1) {
#pragma unroll
          for (int i = 0; i < kPer; ++i) b1 = fmaxf(b1, key[i]);
        }
        const float largest = warp_max(b1);
        if (!(fabsf(largest) < INFINITY)) {  // no expert, or one whose distances from the others say nothing
          doubt |= 1u << r;
          continue;
        }
#pragma unroll
        for (int i = 0; i < kPer; ++i) p[i] = (~(__float_as_uint(largest - key[i]) << 1) & ~mask) | index(i);
      }
      uint32_t m = 0u;
      const auto below = [&] {  // the largest packed key below m
        uint32_t best = p[0] - m;
#pragma unroll
        for (int i = 1; i < kPer; ++i) best = max(best, p[i] - m);
        return m + __reduce_max_sync(kAll, best);
      };
      const int its = lane - r * a.k;
#pragma unroll 4
      for (int c = 0; c < a.k; ++c) {
        m = below();
        if (its == c) pick = m;
      }
      if (!kExact) {
        const uint32_t found = below();
        if (mine == r && found < m) next = found;  // (not where all experts are picked)
      }
    }

    // the choices of all rows
    const bool there = lane < rows * a.k;
    const int64_t row = row0 + (there ? mine : 0);
    from = static_cast<const T *>(a.x) + row * a.E;
    int id = -1;
    const bool scores = there && (good >> mine & 1u);
    if (a.replay) {
      if (there && (on >> mine & 1u)) id = ld(a.ids + row0 * a.k + lane);
      if (id >= a.E) raise_device_error(a.err, SAO_DEVERR_EXPERT_ID);
      if (id >= a.E || !scores) id = -1;
    } else if (scores && pick > none) {
      id = int(mask - (pick & mask));
    }
    float chosen = id >= 0 ? value(from + id) : -INFINITY;
    if (!a.replay && (!kExact || doubt != 0u)) {
      // (a row that ran out of experts may only have run out of distances below inf)
      bool near = scores && ((doubt >> mine & 1u) || (!kExact && id < 0));
      float b_pick = 0.f;
      float window = -1.f;  // the last choice and the key behind it are of one logit and bias: how far about to look
      if (!kExact) {
        uint32_t after = __shfl_down_sync(kAll, pick, 1);
        float x_after = __shfl_down_sync(kAll, chosen, 1);
        if (j == a.k - 1) {
          after = next;
          x_after = after > none && id >= 0 ? value(from + int(mask - (after & mask))) : 0.f;
        }
        if (id >= 0 && after > none) {
          const float d = __uint_as_float((~pick & ~mask) >> 1), d_after = __uint_as_float((~after & ~mask) >> 1);
          float error = 0x1p-23f * float(mask + 2u) * d_after;
          bool apart = (pick & ~mask) > (after & ~mask), same = chosen == x_after;
          if (kBiased) {
            b_pick = ld(a.bias + id);
            const float b_after = ld(a.bias + int(mask - (after & mask)));
            error += (soft ? kDoubtSoftmax / total : kDoubtSigmoid) + 0x1p-23f * (2.f + fabsf(b_pick) + fabsf(b_after));
            apart = d_after - d > error;
            same &= b_pick == b_after;
          }
          near |= !apart && !same;
          if (j == a.k - 1 && !apart && same) window = 2.f * error;
        }
      }
      unsigned again = __ballot_sync(kAll, near);
      // equal ones go by their index, unless some other key is as near to them
      unsigned equal = __ballot_sync(kAll, window >= 0.f);
      while (equal != 0u) {
        const int at = __ffs(equal) - 1;
        equal &= equal - 1u;
        const float x_last = __shfl_sync(kAll, chosen, at), b_last = __shfl_sync(kAll, b_pick, at);
        const float reach = __shfl_sync(kAll, window, at), its_peak = __shfl_sync(kAll, peak, at);
        const float its_total = __shfl_sync(kAll, total, at);
        const auto key_of = [&](float x, float b) {
          return !kBiased ? x : (soft ? exp_fast(x - its_peak) / its_total : sigmoid_fast(x)) + b;
        };
        const T *its_row = static_cast<const T *>(a.x) + (row0 + at / a.k) * a.E;
        const float last = key_of(x_last, b_last);
        bool other = false;
        for (int e = lane; e < a.E; e += 32) {
          const float x = value(its_row + e), b = kBiased ? ld(a.bias + e) : 0.f;
          other |= fabsf(key_of(x, b) - last) <= reach && !(x == x_last && b == b_last);
        }
        if (__any_sync(kAll, other)) again |= 1u << at;
      }
      while (again != 0u) {
        const int r = (__ffs(again) - 1) / a.k;
        const T *its_row = static_cast<const T *>(a.x) + (row0 + r) * a.E;
        const int found = choose_exactly<T, kPer, kBiased>({a.bias, a.k, a.kept, soft, a.two != 0}, l, its_row);
        const int its = __shfl_sync(kAll, found, j);
        if (there && mine == r) {
          id = its;
          chosen = id >= 0 ? value(from + id) : -INFINITY;
        }
        again &= ~__ballot_sync(kAll, mine == r);
      }
    }
    float w = 0.f;
    if (a.renorm) {
      // sigmoid(x) = exp(min(x, 0)) / (1 + exp(-|x|)): relative to the largest, no sum vanishes
      const float lower = soft ? chosen : fminf(chosen, 0.f), m = share_max(lower, first, a.k, even);
      float s = m > -INFINITY ? expf(lower - m) : 0.f;
      if (!soft) s /= 1.f + expf(-fabsf(chosen));
      const float sum = share_sum(s, first, a.k, even);
      if (sum > 0.f) w = s / sum;
    } else if (!soft) {
      w = sigmoid(chosen);
    } else if (id >= 0) {
      w = expf(chosen - peak) / total;
    }
    if (there) {
      if (!a.replay) a.ids[row0 * a.k + lane] = id;
      a.weights[row0 * a.k + lane] = id >= 0 ? a.scale * w : 0.f;
    }
  }
}

// f(the least count of a table that is `per` or more, whether the experts are 32 of it)
template <class F>
sao_status by_count(int E, int per, F f) {
  const auto full = [&](auto count) { return f(count, std::integral_constant<bool, true>()); };
  const auto part = [&](auto count) { return f(count, std::integral_constant<bool, false>()); };
  using std::integral_constant;
  if (E == 32 * per) {
    if (per == 1) return full(integral_constant<int, 1>());
    if (per == 2) return full(integral_constant<int, 2>());
    if (per == 4) return full(integral_constant<int, 4>());
    if (per == 5) return full(integral_constant<int, 5>());
    if (per == 8) return full(integral_constant<int, 8>());
    if (per == 16) return full(integral_constant<int, 16>());
  }
  if (per <= 1) return part(integral_constant<int, 1>());
  if (per <= 2) return part(integral_constant<int, 2>());
  if (per <= 4) return part(integral_constant<int, 4>());
  if (per <= 6) return part(integral_constant<int, 6>());
  if (per <= 8) return part(integral_constant<int, 8>());
  if (per <= 12) return part(integral_constant<int, 12>());
  if (per <= 16) return part(integral_constant<int, 16>());
  if (per <= 32) return part(integral_constant<int, 32>());
  return part(integral_constant<int, 64>());  // groups of few lanes: 3 of 341 experts (43 a lane), 9 of 113 (57), 17 of 60
}

}  // namespace

sao_status route_fwd_launch(const RouteArgs &args, sao_dtype dt, cudaStream_t s) {
  DeviceInfo di;
  SAO_TRY(device_info(&di));
  RouteArgs a = args;
  if (a.groups == a.kept || a.replay) a.groups = a.kept = 1;
  if (a.replay) a.bias = nullptr;
  Lanes l{32, 0, a.E / a.groups, a.groups};
  while (l.share * a.groups > 32) l.share /= 2;
  l.per = (l.size + l.share - 1) / l.share;
  if (route_lists_take(a, di.sm_count)) return route_lists_launch(a, l, dt, di.sm_count, s);
  // as many rows to a warp as its lanes have room for, while there are rows for every warp
  const int64_t spread = a.N / (int64_t(di.sm_count) * 4 * kWarps);
  Plan p{int(least(32 / a.k, spread < 1 ? 1 : spread)), 0u, 0};
  while (p.mask < unsigned(a.E) - 1u) p.mask = 2 * p.mask + 1u;
  const int bytes = l.per * (dt == SAO_BF16 ? 2 : 4);
  p.wide = reinterpret_cast<uintptr_t>(a.x) % unsigned(bytes < 16 ? bytes : 16) == 0;
  const int64_t grid = least((a.N + kWarps * p.batch - 1) / (kWarps * p.batch), int64_t(di.sm_count) * 128);
  const int slot = launch_begin("route_fwd", s);
  SAO_TRY(by_type(dt, [&](auto t) {
    return by_count(a.E, l.per, [&](auto per, auto full) {
      using T = decltype(t);
      constexpr int kPer = decltype(per)::value;
      constexpr bool kFull = decltype(full)::value;
      const auto kernel = a.bias ? route_fwd_kernel<T, kPer, kFull, true> : route_fwd_kernel<T, kPer, kFull, false>;
      pdl(kernel, unsigned(grid), kWarps * 32, 0, s)(a, l, p);
      return SAO_OK;
    });
  }));
  return launch_end(slot, s);
}

}  // namespace sao
