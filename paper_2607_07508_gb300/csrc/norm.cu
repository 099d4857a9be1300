// Root-mean-square norm of a residual stream, with its gradients.
//
//   r    = x + residual, rounded to the arrays' type and stored (sum); x itself without one
//   rstd = (mean_c r_c^2 + eps)^-1/2,      y_c = r_c rstd w_c
// and in 8 bits y8 = e4m3(y / scale), a scale for each row, 128 columns or 32 columns. Backward,
// with a = w dy and the gradient ds that reaches the stream past the norm:
//   dx_c = ds_c + rstd (a_c - r_c rstd mean_j(a_j r_j rstd)),    dw_c = sum_t dy_tc r_tc rstd_t
//
// Bound by HBM: every array goes by once. A row lies in the registers of the warps that take it, kVec columns (16
// bytes, or one column) to a load, so that nothing is read twice; a warp's columns lie together, so that a block of 32 or
// 128 of them never leaves a warp. The norm is that of the stored stream, as the backward sees it. Sums are fp32 over at
// most 64 columns a lane, then by halves; dw's over the rows of a CTA, then over the CTAs in their order.
//
// 65,536 x 2,048 bf16: forward 157 us (1.07 GB, 6.8 TB/s), backward 166 (6.5 TB/s) and 2 for dw's sum. 16,384 x 6,144
// with 32-column scales 115 us (0.71 GB, 6.2 TB/s): instructions next, 25 a column.
// 20,000 x 6,144 fp32 282 and 338 us (7.0 and 5.8 TB/s). Rows that are no whole vectors, and short ones: norm_tiles.cu.
#include <cuda_bf16.h>
#include <cuda_fp8.h>
#include <float.h>
#include <math.h>
#include <stdint.h>

#include <type_traits>

#include "norm.cuh"
#include "sao_common.cuh"
#include "sao_internal.h"

namespace sao {
namespace {

using namespace norm;

constexpr int kThreads = 256;   // of a CTA, or one row's where they are more
constexpr int kMaxThreads = 512;
constexpr int kMaxWarps = kMaxThreads / 32;

// kVec columns of a row as they lie in memory.
template <class T, int kVec>
struct Pack {
  static constexpr int kWords = kVec == 1 ? 1 : kVec * int(sizeof(T)) / 4;
  uint32_t w[kWords];
  __device__ __forceinline__ void load(const T *p) {
    if constexpr (kVec == 1) {
      if constexpr (sizeof(T) == 2)
        w[0] = ld(reinterpret_cast<const uint16_t *>(p));
      else
        w[0] = ld(reinterpret_cast<const uint32_t *>(p));
    } else {
      const uint4 v = ld(reinterpret_cast<const uint4 *>(p));
      w[0] = v.x, w[1] = v.y, w[2] = v.z, w[3] = v.w;
    }
  }
  __device__ __forceinline__ void store(T *p) const {
    if constexpr (kVec == 1) {
      if constexpr (sizeof(T) == 2)
        *reinterpret_cast<uint16_t *>(p) = uint16_t(w[0]);
      else
        *reinterpret_cast<uint32_t *>(p) = w[0];
    } else {
      *reinterpret_cast<uint4 *>(p) = make_uint4(w[0], w[1], w[2], w[3]);
    }
  }
  __device__ __forceinline__ void zero() {
#pragma unroll
    for (int i = 0; i < kWords; ++i) w[i] = 0u;
  }
  __device__ __forceinline__ float at(int j) const {
    if constexpr (sizeof(T) == 4) return __uint_as_float(w[j]);
    if constexpr (kVec == 1) return __uint_as_float(w[0] << 16);
    return __uint_as_float(j & 1 ? w[j / 2] & 0xffff0000u : w[j / 2] << 16);
  }
  __device__ __forceinline__ void set(const float (&v)[kVec]) {
    if constexpr (sizeof(T) == 4) {
#pragma unroll
      for (int j = 0; j < kVec; ++j) w[j] = __float_as_uint(v[j]);
    } else if constexpr (kVec == 1) {
      w[0] = __bfloat16_as_ushort(__float2bfloat16_rn(v[0]));
    } else {
#pragma unroll
      for (int j = 0; j < kVec / 2; ++j) {
        const __nv_bfloat162 b = __floats2bfloat162_rn(v[2 * j], v[2 * j + 1]);
        w[j] = *reinterpret_cast<const uint32_t *>(&b);
      }
    }
  }
};

// kVec weights from column c on.
template <class WT, int kVec>
__device__ __forceinline__ void weights(const void *weight, int c, float (&w)[kVec]) {
  if constexpr (kVec == 1) {
    Pack<WT, 1> p;
    p.load(static_cast<const WT *>(weight) + c);
    w[0] = p.at(0);
  } else if constexpr (sizeof(WT) == 4) {
#pragma unroll
    for (int j = 0; j < kVec; j += 4) {
      const float4 v = ld(reinterpret_cast<const float4 *>(static_cast<const float *>(weight) + c + j));
      w[j] = v.x, w[j + 1] = v.y, w[j + 2] = v.z, w[j + 3] = v.w;
    }
  } else {
#pragma unroll
    for (int j = 0; j < kVec; j += 4) {
      const uint2 v = ld(reinterpret_cast<const uint2 *>(static_cast<const __nv_bfloat16 *>(weight) + c + j));
      w[j] = __uint_as_float(v.x << 16), w[j + 1] = __uint_as_float(v.x & 0xffff0000u);
      w[j + 2] = __uint_as_float(v.y << 16), w[j + 3] = __uint_as_float(v.y & 0xffff0000u);
    }
  }
}

// The warps of a CTA that share a row: `warps` of them, this thread's one being `warp`.
struct Team {
  int warps, warp, team;
  uint32_t turn = 0;
  float *slots;  // [2][kMaxWarps] of the CTA
  __device__ __forceinline__ Team(int warps_, float *s) : warps(warps_), slots(s) {
    const int w = threadIdx.x / 32;
    team = w / warps;
    warp = w - team * warps;
  }
  // Over the row. Two sets of slots: those of the reduction before may still be read.
  template <class Op>
  __device__ __forceinline__ float all(float v, Op op) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v = op(v, __shfl_xor_sync(0xffffffffu, v, o));
    if (warps == 1) return v;
    float *mine = slots + (turn++ & 1u) * kMaxWarps + team * warps;
    if ((threadIdx.x & 31) == 0) mine[warp] = v;
    asm volatile("bar.sync %0, %1;" ::"r"(team + 1), "r"(warps * 32) : "memory");
    v = mine[0];
    for (int i = 1; i < warps; ++i) v = op(v, mine[i]);
    return v;
  }
  __device__ __forceinline__ float sum(float v) {
    return all(v, [](float a, float b) { return a + b; });
  }
  __device__ __forceinline__ float max(float v) {
    return all(v, [](float a, float b) { return max_nan(a, b); });
  }
};

// kTiny: eps is below kSmall. (As a condition of one kernel this cost every call registers, 16,384 x 6,144 in 8 bits 121
// us to 138. Calls with an eps of 0 take up to a tenth longer than others: 65,536 x 2,048 bf16 178 us and 161.)
template <class T, class WT, int kVec, int kLoads, bool kTiny>
__global__ void __launch_bounds__(kMaxThreads, kVec < 8 && kVec * kLoads == 32 ? 1 : 2)
    norm_fwd_kernel(NormFwd a, int warps) {
  grid_wait();
  __shared__ float slots[2 * kMaxWarps];
  Team team(warps, slots);
  const int lane = threadIdx.x & 31, teams = blockDim.x / (32 * warps);
  const int c0 = (team.warp * kLoads * 32 + lane) * kVec;  // column of load 0; load i: 32 kVec further on
  const auto column = [&](int i) { return c0 + i * 32 * kVec; };
  const float mean = 1.f / float(a.h);
  for (int64_t row = int64_t(blockIdx.x) * teams + team.team; row < a.N; row += int64_t(gridDim.x) * teams) {
    const int64_t at = row * a.h;
    Pack<T, kVec> r[kLoads];
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      r[i].zero();
      if (column(i) < a.h) r[i].load(static_cast<const T *>(a.x) + at + column(i));
    }
    if (a.residual) {
      Pack<T, kVec> q[kLoads];
#pragma unroll
      for (int i = 0; i < kLoads; ++i) {
        q[i].zero();
        if (column(i) < a.h) q[i].load(static_cast<const T *>(a.residual) + at + column(i));
      }
#pragma unroll
      for (int i = 0; i < kLoads; ++i) {
        float v[kVec];
#pragma unroll
        for (int j = 0; j < kVec; ++j) v[j] = r[i].at(j) + q[i].at(j);
        r[i].set(v);
        if (column(i) < a.h) r[i].store(static_cast<T *>(a.sum) + at + column(i));
      }
    }
    float s[2] = {0.f, 0.f};
#pragma unroll
    for (int i = 0; i < kLoads; ++i)
#pragma unroll
      for (int j = 0; j < kVec; ++j) s[j & 1] = fmaf(r[i].at(j), r[i].at(j), s[j & 1]);
    const float square = fmaf(team.sum(s[0] + s[1]), mean, a.eps);
    float rstd = 1.f / sqrtf(square);
    if (kTiny && square < kSmall) {  // (all of the row's threads)
      s[0] = s[1] = 0.f;
#pragma unroll
      for (int i = 0; i < kLoads; ++i)
#pragma unroll
        for (int j = 0; j < kVec; ++j) {
          const float v = r[i].at(j) * kUp;
          s[j & 1] = fmaf(v, v, s[j & 1]);
        }
      rstd = 1.f / sqrtf(fmaf(team.sum(s[0] + s[1]), mean, a.eps * kUp * kUp)) * kUp;
    }
    if (a.rstd && team.warp == 0 && lane == 0) a.rstd[row] = rstd;
    float y[kLoads][kVec];
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
#pragma unroll
      for (int j = 0; j < kVec; ++j) y[i][j] = 0.f;
      if (column(i) >= a.h) continue;
      float w[kVec];
      weights<WT, kVec>(a.weight, column(i), w);
#pragma unroll
      for (int j = 0; j < kVec; ++j) y[i][j] = r[i].at(j) * rstd * w[j];
      if (a.y) {
        Pack<T, kVec> p;
        p.set(y[i]);
        p.store(static_cast<T *>(a.y) + at + column(i));
      }
    }
    if (!a.y8) continue;
    const auto amax_of = [&](int i) {
      float m = 0.f;
#pragma unroll
      for (int j = 0; j < kVec; ++j) m = max_nan(m, fabsf(y[i][j]));
      return m;
    };
    const auto put = [&](int i, float inverse) {
      if (column(i) >= a.h) return;
      uint8_t *p = a.y8 + at + column(i);
      if constexpr (kVec == 1) {
        *p = __nv_cvt_float_to_fp8(y[i][0] * inverse, __NV_SATFINITE, __NV_E4M3);
      } else {
        uint16_t q[kVec / 2];
#pragma unroll
        for (int j = 0; j < kVec / 2; ++j)
          q[j] = __nv_cvt_float2_to_fp8x2(make_float2(y[i][2 * j] * inverse, y[i][2 * j + 1] * inverse), __NV_SATFINITE,
                                          __NV_E4M3);
        const uint32_t low = q[0] | uint32_t(q[1]) << 16;
        if constexpr (kVec == 8)
          *reinterpret_cast<uint2 *>(p) = make_uint2(low, q[2] | uint32_t(q[3]) << 16);
        else
          *reinterpret_cast<uint32_t *>(p) = low;
      }
    };
    float inverse;
    if (a.scaling == SAO_SCALE_ROW) {
      float m = 0.f;
#pragma unroll
      for (int i = 0; i < kLoads; ++i) m = max_nan(m, amax_of(i));
      const float scale = scale_of(team.max(m), &inverse);
      if (team.warp == 0 && lane == 0) static_cast<float *>(a.scales)[row] = scale;
#pragma unroll
      for (int i = 0; i < kLoads; ++i) put(i, inverse);
      continue;
    }
    const auto by_blocks = [&](auto size) {
      constexpr int kSize = decltype(size)::value;
      constexpr bool kMx = kSize == 32;
      const int blocks = (a.h + kSize - 1) / kSize;
      // loads that a block spans (single columns: 4 of 32), and lanes of a load that share one
      constexpr int kStep = kVec == 1 ? 4 : 1, kLanes = kSize / kVec < 32 ? kSize / kVec : 32;
#pragma unroll
      for (int i = 0; i < kLoads; i += kStep) {
        float m[kStep];
#pragma unroll
        for (int k = 0; k < kStep; ++k) {
          m[k] = amax_of(i + k);
#pragma unroll
          for (int o = 1; o < kLanes; o <<= 1) m[k] = max_nan(m[k], __shfl_xor_sync(0xffffffffu, m[k], o));
        }
        if (kStep > 1 && !kMx) {
          float all = m[0];
#pragma unroll
          for (int k = 1; k < kStep; ++k) all = max_nan(all, m[k]);
#pragma unroll
          for (int k = 0; k < kStep; ++k) m[k] = all;
        }
#pragma unroll
        for (int k = 0; k < kStep; ++k) {
          const int c = column(i + k);
          const bool first = c < a.h && (c & (kSize - 1)) == 0;
          if (kMx) {
            const uint32_t b = power_of(m[k], &inverse);
            if (first) static_cast<uint8_t *>(a.scales)[row * blocks + c / kSize] = uint8_t(b);
          } else {
            const float scale = scale_of(m[k], &inverse);
            if (first) static_cast<float *>(a.scales)[row * blocks + c / kSize] = scale;
          }
          put(i + k, inverse);
        }
      }
    };
    if (a.scaling == SAO_SCALE_MX32)
      by_blocks(std::integral_constant<int, 32>());
    else
      by_blocks(std::integral_constant<int, 128>());
  }
}

// A CTA's sums for dw go to row blockIdx.x of `partial`.
template <class T, class WT, int kVec, int kLoads>
__global__ void __launch_bounds__(kMaxThreads) norm_bwd_kernel(NormBwd a, int warps, float *partial) {
  grid_wait();
  __shared__ float slots[2 * kMaxWarps];
  extern __shared__ float sums[];  // a place for each of a lane's columns, with more than one team
  Team team(warps, slots);
  const int lane = threadIdx.x & 31, teams = blockDim.x / (32 * warps);
  const int c0 = (team.warp * kLoads * 32 + lane) * kVec;
  const auto column = [&](int i) { return c0 + i * 32 * kVec; };
  const float mean = 1.f / float(a.h);
  float dw[kLoads * kVec];
#pragma unroll
  for (int i = 0; i < kLoads * kVec; ++i) dw[i] = 0.f;
  for (int64_t row = int64_t(blockIdx.x) * teams + team.team; row < a.N; row += int64_t(gridDim.x) * teams) {
    const int64_t at = row * a.h;
    Pack<T, kVec> r[kLoads], d[kLoads], g[kLoads];
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      r[i].zero(), d[i].zero(), g[i].zero();
      if (column(i) < a.h) {
        r[i].load(static_cast<const T *>(a.x) + at + column(i));
        d[i].load(static_cast<const T *>(a.dy) + at + column(i));
        if (a.dsum) g[i].load(static_cast<const T *>(a.dsum) + at + column(i));
      }
    }
    const float rstd = ld(a.rstd + row);
    float s[2] = {0.f, 0.f};
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      if (column(i) < a.h) {
        float w[kVec];
        weights<WT, kVec>(a.weight, column(i), w);
#pragma unroll
        for (int j = 0; j < kVec; ++j) {
          const float t = d[i].at(j) * (r[i].at(j) * rstd);
          dw[i * kVec + j] += t;
          s[j & 1] = fmaf(t, w[j], s[j & 1]);
        }
      }
    }
    const float c = team.sum(s[0] + s[1]) * mean * rstd;  // times r rstd, below
#pragma unroll
    for (int i = 0; i < kLoads; ++i)
      if (column(i) < a.h) {
        float w[kVec], v[kVec];
        weights<WT, kVec>(a.weight, column(i), w);
#pragma unroll
        for (int j = 0; j < kVec; ++j)
          v[j] = g[i].at(j) + rstd * fmaf(-c, r[i].at(j), d[i].at(j) * w[j]);
        Pack<T, kVec> p;
        p.set(v);
        p.store(static_cast<T *>(a.dx) + at + column(i));
      }
  }
  if (partial == nullptr) return;
  // The teams' sums in their order, a thread's where no other's banks are (by columns this took 10 us of a call).
  const int width = 32 * warps, place = team.warp * 32 + lane;
  for (int t = 0; t < teams; ++t) {
    if (t > 0) __syncthreads();
    if (t != team.team) continue;
#pragma unroll
    for (int i = 0; i < kLoads * kVec; ++i) {
      if (t > 0) dw[i] += sums[i * width + place];
      if (t < teams - 1) sums[i * width + place] = dw[i];
    }
  }
  if (team.team != teams - 1) return;
  float *out = partial + int64_t(blockIdx.x) * a.h;
#pragma unroll
  for (int i = 0; i < kLoads; ++i) {
    if (column(i) >= a.h) continue;
    if constexpr (kVec == 1) {
      out[column(i)] = dw[i];
    } else {
#pragma unroll
      for (int j = 0; j < kVec; j += 4)
        *reinterpret_cast<float4 *>(out + column(i) + j) =
            make_float4(dw[i * kVec + j], dw[i * kVec + j + 1], dw[i * kVec + j + 2], dw[i * kVec + j + 3]);
    }
  }
}

// dw = (dw +) the partials' sums: 32 columns to a CTA, its warps side by side in the partials.
constexpr int kSumWarps = 32;
__global__ void __launch_bounds__(32 * kSumWarps) norm_dw_kernel(const float *partial, int parts, int h, float *dw,
                                                                 int accumulate) {
  grid_wait();
  __shared__ float warp_sum[kSumWarps][32];
  const int lane = threadIdx.x & 31, warp = threadIdx.x / 32, c = blockIdx.x * 32 + lane;
  float s = 0.f;
  constexpr int kBatch = 10;  // parts in flight: all of a warp's where there are two CTAs to an SM
  for (int p0 = warp; c < h && p0 < parts; p0 += kSumWarps * kBatch) {
    float v[kBatch];
#pragma unroll
    for (int i = 0; i < kBatch; ++i) {
      const int p = p0 + i * kSumWarps;
      v[i] = p < parts ? ld(partial + int64_t(p) * h + c) : 0.f;
    }
#pragma unroll
    for (int i = 0; i < kBatch; ++i) s += v[i];
  }
  warp_sum[warp][lane] = s;
  __syncthreads();
  if (warp != 0 || c >= h) return;
  for (int w = 1; w < kSumWarps; ++w) s += warp_sum[w][lane];
  dw[c] = accumulate ? dw[c] + s : s;
}

sao_status sum_parts(const NormBwd &a, const float *partial, int parts, cudaStream_t s) {
  const int slot = launch_begin("norm_dw", s);
  pdl(norm_dw_kernel, unsigned((a.h + 31) / 32), 32 * kSumWarps, 0, s)(partial, parts, a.h, a.dweight, a.accumulate);
  return launch_end(slot, s);
}

constexpr int kBwdCtas = 2 * 160, kTileCtas = 6 * 160;  // partials of dw, at most

// Loads a lane (each a power of two) and warps a row: f(integral constants) for the least of
// kFew, 2 kFew .. kMost that leaves at most `wish` warps to a row.
struct Shape {
  int loads, warps;
};
Shape shape_of(int h, int vec, int few, int most, int wish) {
  Shape p{few, 0};
  for (;; p.loads *= 2) {
    p.warps = (h + 32 * vec * p.loads - 1) / (32 * vec * p.loads);
    if (p.warps <= wish || p.loads == most) return p;
  }
}

template <class F>
void by_loads(int loads, F f) {
  switch (loads) {
    case 1: f(std::integral_constant<int, 1>()); break;
    case 2: f(std::integral_constant<int, 2>()); break;
    case 4: f(std::integral_constant<int, 4>()); break;
    case 8: f(std::integral_constant<int, 8>()); break;
    case 16: f(std::integral_constant<int, 16>()); break;
    default: f(std::integral_constant<int, 32>()); break;
  }
}

int teams_of(int warps) { return warps < kThreads / 32 ? kThreads / 32 / warps : 1; }

template <class T, class WT, int kVec>
sao_status fwd(const NormFwd &a, int sms, cudaStream_t s) {
  // few rows: few loads a lane, for latency. Many: 16 columns a lane up to 8 warps to a row, else 32, which keeps 64
  // registers and half an SM's warps (65,536 x 2,048 161 us with 16, 168 with 32; 16,384 x 6,144 in 8 bits 166 and 153)
  constexpr int kFewLoads = kVec == 1 ? 4 : 1, kMostLoads = 32 / kVec;
  const Shape p = a.N <= 4 * sms ? shape_of(a.h, kVec, kFewLoads, kMostLoads, kThreads / 32)
                             : shape_of(a.h, kVec, kVec == 1 ? 8 : 16 / kVec, kMostLoads, kThreads / 32);
  const int teams = teams_of(p.warps);
  int64_t grid = (a.N + teams - 1) / teams;
  grid = grid < 64 * int64_t(sms) ? grid : 64 * int64_t(sms);
  const int slot = launch_begin("norm_fwd", s);
  by_loads(p.loads, [&](auto loads) {
    constexpr int kLoads = decltype(loads)::value;
    if constexpr (kLoads >= kFewLoads && kLoads <= kMostLoads) {
      const auto kernel =
          a.eps < kSmall ? norm_fwd_kernel<T, WT, kVec, kLoads, true> : norm_fwd_kernel<T, WT, kVec, kLoads, false>;
      pdl(kernel, unsigned(grid), unsigned(teams * p.warps * 32), 0, s)(a, p.warps);
    }
  });
  return launch_end(slot, s);
}

template <class T, class WT, int kVec>
sao_status bwd(const NormBwd &a, int sms, float *partial, cudaStream_t s) {
  constexpr int kFewLoads = kVec == 1 ? 8 : kVec == 4 ? 4 : 1, kMostLoads = 32 / kVec;
  // many rows: 32 bf16 columns a lane, fewer fp32 or single ones, for registers
  const int wish = a.N <= 4 * sms ? kThreads / 32 : kVec < 8 ? kMaxWarps : 1;
  const Shape p = shape_of(a.h, kVec, kFewLoads, kMostLoads, wish);
  const int teams = teams_of(p.warps);
  int64_t grid = (a.N + teams - 1) / teams;
  // (few single columns: few registers, and few loads in flight without the warps)
  const bool light = kVec == 1 && p.loads <= 8;
  const int most = light ? (6 * sms < kTileCtas ? 6 * sms : kTileCtas) : 2 * sms < kBwdCtas ? 2 * sms : kBwdCtas;
  grid = grid < most ? grid : most;
  const int slot = launch_begin("norm_bwd", s);
  by_loads(p.loads, [&](auto loads) {
    if constexpr (decltype(loads)::value >= kFewLoads && decltype(loads)::value <= kMostLoads)
      pdl(norm_bwd_kernel<T, WT, kVec, decltype(loads)::value>, unsigned(grid), unsigned(teams * p.warps * 32),
          teams > 1 ? size_t(p.loads) * kVec * 32 * p.warps * sizeof(float) : 0, s)(
          a, p.warps, a.dweight ? partial : nullptr);
  });
  SAO_TRY(launch_end(slot, s));
  return a.dweight ? sum_parts(a, partial, int(grid), s) : SAO_OK;
}

// f(type of the arrays, of the weight, columns of a load)
template <class F>
sao_status by_types(sao_dtype dt, sao_dtype w_dt, bool wide, F f) {
  using Wide16 = std::integral_constant<int, 8>;
  using Wide32 = std::integral_constant<int, 4>;
  using One = std::integral_constant<int, 1>;
  if (dt == SAO_BF16) {
    if (w_dt == SAO_BF16)
      return wide ? f(__nv_bfloat16(), __nv_bfloat16(), Wide16()) : f(__nv_bfloat16(), __nv_bfloat16(), One());
    return wide ? f(__nv_bfloat16(), float(), Wide16()) : f(__nv_bfloat16(), float(), One());
  }
  if (w_dt == SAO_BF16) return wide ? f(float(), __nv_bfloat16(), Wide32()) : f(float(), __nv_bfloat16(), One());
  return wide ? f(float(), float(), Wide32()) : f(float(), float(), One());
}

// Whether rows go by tiles: short ones, which leave most of a warp idle, and in the forward those that are no
// whole vectors, but for fp32 ones of up to 1,024 columns. (Forward by tiles and else: 300,000 x 20 bf16 21 and 93
// us, 400,003 x 64 76 and 113, x 128 142 and 118; 4,099 x 515 9 and 13.5, in fp32 16 and 14, 20,001 x 4,099 190
// and 256, in fp32 270 and 322. Backward: 300,000 x 20 31 and 111, 400,003 x 64 130 and 161, x 77 192 and 171; it
// reads its tiles three times.)
bool fwd_by_tiles(int h, sao_dtype dt, bool wide, bool to8) {
  return h <= kShortRow || (!wide && (to8 || dt == SAO_BF16 || h > 1024));
}

}  // namespace

size_t norm_ws_bytes(int64_t N, int32_t h) {
  const int64_t parts = N < kTileCtas ? N : kTileCtas;
  return round256(size_t(parts) * size_t(h) * sizeof(float));
}

sao_status norm_fwd_launch(const NormFwd &a, sao_dtype dt, sao_dtype w_dt, cudaStream_t s) {
  DeviceInfo di;
  SAO_TRY(device_info(&di));
  const bool wide = a.h % (dt == SAO_BF16 ? 8 : 4) == 0 && aligned16(a.x) && aligned16(a.residual) &&
                    aligned16(a.sum) && aligned16(a.y) && aligned16(a.weight) && aligned16(a.y8);
  const bool tiles = aligned16(a.x) && aligned16(a.residual) && aligned16(a.sum) && aligned16(a.y) && aligned16(a.y8);
  if (tiles && fwd_by_tiles(a.h, dt, wide, a.y8 != nullptr)) return norm_fwd_tiles_launch(a, dt, w_dt, s);
  return by_types(dt, w_dt, wide, [&](auto t, auto w, auto vec) {
    return fwd<decltype(t), decltype(w), decltype(vec)::value>(a, di.sm_count, s);
  });
}

sao_status norm_bwd_launch(const NormBwd &a, sao_dtype dt, sao_dtype w_dt, void *ws, size_t ws_bytes, cudaStream_t s) {
  DeviceInfo di;
  SAO_TRY(device_info(&di));
  Carver c(ws, ws_bytes);
  float *partial = c.take<float>(size_t(a.N < kTileCtas ? a.N : kTileCtas) * size_t(a.h));
  if (a.dweight && !c.ok()) return fail(SAO_ERR_WORKSPACE, "workspace of the norm's backward too small");
  const bool wide = a.h % (dt == SAO_BF16 ? 8 : 4) == 0 && aligned16(a.x) && aligned16(a.dy) && aligned16(a.dsum) &&
                    aligned16(a.dx) && aligned16(a.weight);
  if (aligned16(a.x) && aligned16(a.dy) && aligned16(a.dsum) && aligned16(a.dx) && a.h <= kShortRow) {
    int parts;
    const int most = 6 * di.sm_count < kTileCtas ? 6 * di.sm_count : kTileCtas;
    SAO_TRY(norm_bwd_tiles_launch(a, dt, w_dt, partial, int(a.N < most ? a.N : most), &parts, s));
    return a.dweight ? sum_parts(a, partial, parts, s) : SAO_OK;
  }
  return by_types(dt, w_dt, wide, [&](auto t, auto w, auto vec) {
    return bwd<decltype(t), decltype(w), decltype(vec)::value>(a, di.sm_count, partial, s);
  });
}

}  // namespace sao
