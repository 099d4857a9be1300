// Routing to experts: the gradient of the router's logits.
//
//   renormalised  d x_j = w_j (g_j - c / scale), sigmoid times 1 - s_j;  else softmax d x_e = s_e (scale g_e - c),
//   sigmoid d x_j = w_j g_j (1 - s_j);  c = sum_j g_j w_j
//
// It writes every logit's gradient, most of them 0 (renormalised weights, and sigmoid scores, depend on the chosen
// logits alone): 2^20 x 160 bf16 91 us, 4.8 TB/s, 1.4 times the bytes at the rate of HBM; 65,536 x 128 fp32 8 to 10 us
// (34 MB written). A warp waits first for its tile in shared memory and for its choices' ids, weights and gradients: 623,932
// rows of 6 of 16 experts, of little but choices, take 41 us for 65 MB. The gradient of every logit of a softmax takes 21 us
// for 98,301 x 63 bf16, with 52 % of the issue slots used at 30 % of the warps, which wait for shared memory first.
#include "bulk.cuh"
#include "route_common.cuh"

namespace sao {
namespace {

using namespace route;

__device__ __forceinline__ void put(float *p, float v) { *p = v; }
__device__ __forceinline__ void put(__nv_bfloat16 *p, float v) { *p = __float2bfloat16_rn(v); }
__device__ __forceinline__ float at_smem(const float *p) { return *p; }
__device__ __forceinline__ float at_smem(const __nv_bfloat16 *p) { return __bfloat162float(*p); }

constexpr int kTileBytes = 4 << 10;  // of a warp's rows, but for eight rows that are more
constexpr int kSmem = 48 << 10;

struct BwdPlan {
  int rows;   // of a warp's tile: a multiple of 8, so that tiles start on 16 bytes
  int bytes;  // of a warp's shared memory
  int share;  // kDense: lanes to a row
  int wide;   // dx (and x) on 16 bytes
};

// A warp writes the gradient of `rows` rows at a time, made up in shared memory and sent off in one bulk copy
// (the rows lie one after another): zeros with the chosen experts' gradients put between them, or, kDense, the
// softmax gradient of every logit. Lane r k + j has choice j of row r, 32 / k rows at a time; an id that a row
// has twice is found with match_any and written once, by its first lane. kEach (kDense): a lane's logits of a
// row, at most.
template <class T, bool kDense, int kEach>
__global__ void __launch_bounds__(128) route_bwd_kernel(const __grid_constant__ RouteBwdArgs a, BwdPlan plan) {
  grid_wait();
  extern __shared__ __align__(128) unsigned char shared[];
  const int lane = threadIdx.x & 31, warps = blockDim.x / 32, warp = threadIdx.x / 32;
  T *tile = reinterpret_cast<T *>(shared + size_t(warp) * plan.bytes);
  // kDense, behind the tile: each row's c, largest logit and inverse sum, the choices' gradients and ids
  float *row_c = reinterpret_cast<float *>(tile + size_t(plan.rows) * a.E), *peak = row_c + plan.rows;
  float *inverse = peak + plan.rows, *chosen_d = inverse + plan.rows;
  int *chosen_id = reinterpret_cast<int *>(chosen_d + plan.rows * a.k);
  const bool soft = a.score == SAO_SCORE_SOFTMAX;
  const int at_once = 32 / a.k, mine = lane / a.k, first = mine * a.k;
  const bool even = (a.k & (a.k - 1)) == 0;
  const int64_t step = int64_t(gridDim.x) * warps * plan.rows;
  for (int64_t row0 = (int64_t(blockIdx.x) * warps + warp) * plan.rows; row0 < a.N; row0 += step) {
    const int rows = int(a.N - row0 < plan.rows ? a.N - row0 : plan.rows), count = rows * a.E;
    T *dx = static_cast<T *>(a.dx) + row0 * a.E;
    const T *x = static_cast<const T *>(a.x) + row0 * a.E;
    const bool live = lane < rows && a.scale != 0.f && (a.mask == nullptr || ld(a.mask + row0 + lane) != 0);
    const unsigned on = __ballot_sync(kAll, live);
    constexpr int kPer16 = 16 / int(sizeof(T));
    const int vectors = plan.wide ? count / kPer16 : 0;
    if (lane == 0) tc::bulk_wait_group_read<0>();  // the tile before is on its way
    __syncwarp();
    if (kDense) {
      for (int i = lane; i < vectors; i += 32)
        reinterpret_cast<uint4 *>(tile)[i] = ld(reinterpret_cast<const uint4 *>(x) + i);
      for (int i = vectors * kPer16 + lane; i < count; i += 32) tile[i] = ld(x + i);
    } else if (!a.accumulate) {
      const int words = (count * int(sizeof(T)) + 15) / 16;
      for (int i = lane; i < words; i += 32) reinterpret_cast<uint4 *>(tile)[i] = make_uint4(0u, 0u, 0u, 0u);
    }
    __syncwarp();
    // a choice's id, weight and gradient, those of the next rows loaded while these are worked on
    const auto fetch = [&](int r0, int &id, float &w, float &g) {
      const int64_t flat = (row0 + r0) * a.k + lane;
      id = -1, w = g = 0.f;
      if (mine < at_once && r0 + mine < rows && (on >> (r0 + mine) & 1u))
        id = ld(a.ids + flat), w = ld(a.weights + flat), g = ld(a.grad + flat);
    };
    int next_id;
    float next_w, next_g;
    fetch(0, next_id, next_w, next_g);
    for (int r0 = 0; r0 < rows; r0 += at_once) {
      const int r = r0 + mine;
      const bool real = mine < at_once && r < rows;
      int id = next_id;
      float w = next_w, g = next_g;
      if (r0 + at_once < rows) fetch(r0 + at_once, next_id, next_w, next_g);
      if (id >= a.E) raise_device_error(a.err, SAO_DEVERR_EXPERT_ID), id = -1;
      if (id < 0) w = g = 0.f;
      const float c = share_sum(g * w, first, a.k, even);
      float d = 0.f;
      if (kDense) {
        d = a.scale * g;
      } else if (w != 0.f) {
        d = a.renorm ? w * (g - c / a.scale) : w * g;
        if (!soft) d *= sigmoid(-value(x + int64_t(r) * a.E + id));
      }
      const unsigned same = __match_any_sync(kAll, id >= 0 ? r << 10 | id : -1 - lane);
      if (__any_sync(kAll, (same & (same - 1u)) != 0u)) {
        float sum = 0.f;
        for (int i = 0; i < a.k; ++i) {
          const float other = __shfl_sync(kAll, d, first + i);
          if (same >> ((first + i) & 31) & 1u) sum += other;
        }
        if (id >= 0) d = sum;
      }
      const bool writes = id >= 0 && __ffs(same) - 1 == lane;
      if (kDense) {
        if (real) {
          if (lane == first) row_c[r] = c;
          chosen_d[r0 * a.k + lane] = d;
          chosen_id[r0 * a.k + lane] = writes ? id : -1;
        }
      } else if (writes) {
        if (a.accumulate) {
          T *p = dx + int64_t(r) * a.E + id;
          put(p, value(p) + d);
        } else {
          put(tile + r * a.E + id, d);
        }
      }
    }
    if (!kDense && a.accumulate) continue;
    __syncwarp();
    if (kDense) {
      const int s = lane & (plan.share - 1), by = 32 / plan.share;
      for (int r0 = 0; r0 < rows; r0 += by) {
        const int r = r0 + lane / plan.share;
        const bool real = r < rows;
        T *row = tile + (real ? r : 0) * a.E;
        float top = -INFINITY, v[kEach], sum = 0.f;
#pragma unroll
        for (int i = 0; i < kEach; ++i) {
          const int e = s + i * plan.share;
          v[i] = e < a.E ? at_smem(row + e) : -INFINITY;
          top = fmaxf(top, v[i]);
        }
        for (int o = plan.share / 2; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(kAll, top, o));
#pragma unroll
        for (int i = 0; i < kEach; ++i) sum += v[i] = expf(v[i] - top);
        for (int o = plan.share / 2; o > 0; o >>= 1) sum += __shfl_xor_sync(kAll, sum, o);
        if (real) {
          // masked, or no scores (a NaN, +inf, -inf throughout: the sum is NaN): gradients of 0
          const float f = sum > 0.f && (on >> r & 1u) ? 1.f / sum : 0.f, c = -row_c[r] * f;
          if (s == 0) peak[r] = top, inverse[r] = f;
#pragma unroll
          for (int i = 0; i < kEach; ++i) {
            const int e = s + i * plan.share;
            if (e >= a.E) continue;
            const float before = a.accumulate ? value(dx + r * a.E + e) : 0.f;
            put(row + e, f > 0.f ? fmaf(v[i], c, before) : before);
          }
        }
      }
      __syncwarp();
      for (int r0 = 0; r0 < rows; r0 += at_once) {
        const int r = r0 + mine, i = r0 * a.k + lane;
        if (mine >= at_once || r >= rows) continue;
        const int id = chosen_id[i], at = r * a.E + id;
        if (id < 0 || !(inverse[r] > 0.f)) continue;
        const float before = a.accumulate ? value(dx + at) : 0.f;
        put(tile + at, fmaf(expf(value(x + at) - peak[r]) * inverse[r], chosen_d[i] - row_c[r], before));
      }
      __syncwarp();
    }
    if (vectors > 0) {
      tc::fence_proxy_async_smem();
      __syncwarp();
      if (lane == 0) {
        bulk::store(dx, tile, uint32_t(vectors) * 16u);
        tc::bulk_commit_group();
      }
    }
    for (int i = vectors * kPer16 + lane; i < count; i += 32) dx[i] = tile[i];
  }
  if (lane == 0) tc::bulk_wait_group<0>();
}

}  // namespace

sao_status route_bwd_launch(const RouteBwdArgs &a, sao_dtype dt, cudaStream_t s) {
  DeviceInfo di;
  SAO_TRY(device_info(&di));
  const int size = dt == SAO_BF16 ? 2 : 4;
  const bool dense = a.score == SAO_SCORE_SOFTMAX && !a.renorm;
  BwdPlan p{32, 0, 1, aligned16(a.x) && aligned16(a.dx)};
  while (p.rows > 8 && (p.rows * a.E * size > kTileBytes || a.N < int64_t(di.sm_count) * 4 * p.rows)) p.rows /= 2;
  while (p.share < 32 && p.share * 8 < a.E) p.share *= 2;
  p.bytes = p.rows * a.E * size + (dense ? p.rows * (12 + 8 * a.k) : 0);
  p.bytes = (p.bytes + 127) / 128 * 128;
  const int warps = int(least(4, kSmem / p.bytes));
  const int64_t grid = least((a.N + p.rows * warps - 1) / (p.rows * warps), int64_t(di.sm_count) * 128);
  const int slot = launch_begin("route_bwd", s);
  SAO_TRY(by_type(dt, [&](auto t) {
    using T = decltype(t);
    const auto launch = [&](auto kernel) {
      pdl(kernel, unsigned(grid), unsigned(warps * 32), size_t(warps) * p.bytes, s)(a, p);
      return SAO_OK;
    };
    if (!dense) return launch(route_bwd_kernel<T, false, 1>);
    if (a.E <= 8 * 32) return launch(route_bwd_kernel<T, true, 8>);
    return launch(route_bwd_kernel<T, true, 32>);
  }));
  return launch_end(slot, s);
}

}  // namespace sao
