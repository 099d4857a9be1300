// Root-mean-square norm of rows that are no whole number of 16-byte vectors, or short: by tiles of rows in shared
// memory.
//
// Rows lie one after another, so a tile of them is one run of memory, whatever their length: it is loaded and stored by
// vectors (but for its first and last few elements), every lane busy, and only shared memory is read column by column,
// by a part of a warp, a warp or several to a row. That takes two passes of the forward and three of the backward over
// shared memory, and no load is in flight while a CTA computes: 300,000 x 20 bf16 20 and 31 us (48 MB each, 2.4 and
// 1.5 TB/s; a warp to a row 93 and 111), forward of 20,001 x 4,099 190 to 202 us (0.66 GB, 3.3 to 3.5 TB/s; single columns
// from memory 256, vectors that the rows' ends cut 191). Which calls come here: fwd_by_tiles in norm.cu.
#include <cuda_bf16.h>
#include <cuda_fp8.h>
#include <math.h>
#include <stdint.h>

#include <initializer_list>

#include "norm.cuh"
#include "per_device.h"
#include "sao_common.cuh"

namespace sao {
namespace {

using namespace norm;

constexpr int kThreads = 256, kWarps = kThreads / 32;
static_assert(kShortRow < kThreads, "the backward's sums");
constexpr unsigned kAll = 0xffffffffu;

__device__ __forceinline__ float get(const float *p) { return *p; }
__device__ __forceinline__ float get(const __nv_bfloat16 *p) { return __bfloat162float(*p); }
__device__ __forceinline__ void put(float *p, float v) { *p = v; }
__device__ __forceinline__ void put(__nv_bfloat16 *p, float v) { *p = __float2bfloat16_rn(v); }
__device__ __forceinline__ float column_weight(const void *w, bool bf16, int c) {
  if (bf16) return __uint_as_float(uint32_t(ld(static_cast<const uint16_t *>(w) + c)) << 16);
  return ld(static_cast<const float *>(w) + c);
}

// How a tile's rows are shared out: `lanes` of a warp to a row (a power of two), or `warps` of the CTA where those are
// more than one.
struct TilePlan {
  int rows, lanes, warps;
  int bytes;  // of a tile, with room for what its alignment leaves in front and behind
};

// The elements [from, from + count) of an array and a tile that holds them: the tile's first vector is the one of
// memory that holds element `from`, so that vectors of both lie on 16 bytes. f(at, vector) with the tile's
// vectors, one(i) with single elements of the tile.
template <class T, class Vector, class One>
__device__ __forceinline__ void flat(int64_t from, int count, Vector vector, One one) {
  constexpr int kVec = 16 / int(sizeof(T)), kBatch = 4;
  const int lead = int(from % kVec), end = lead + count, first = (lead + kVec - 1) / kVec, last = end / kVec;
  for (int v = first + threadIdx.x; v < last; v += kThreads * kBatch) vector(v, last);
  if (last < first) {  // (within one vector)
    if (int(threadIdx.x) < count) one(lead + threadIdx.x);
    return;
  }
  const int head = first * kVec - lead, tail = end - last * kVec;
  if (int(threadIdx.x) < head) one(lead + threadIdx.x);
  if (int(threadIdx.x) >= 32 && int(threadIdx.x) - 32 < tail) one(last * kVec + threadIdx.x - 32);
}

template <class T>
__device__ __forceinline__ void load_tile(T *tile, const T *array, int64_t from, int count) {
  constexpr int kVec = 16 / int(sizeof(T)), kBatch = 4;
  const T *base = array + (from - from % kVec);
  flat<T>(
      from, count,
      [&](int v, int last) {
        uint4 w[kBatch];
#pragma unroll
        for (int i = 0; i < kBatch; ++i)
          if (v + i * kThreads < last) w[i] = ld(reinterpret_cast<const uint4 *>(base) + v + i * kThreads);
#pragma unroll
        for (int i = 0; i < kBatch; ++i)
          if (v + i * kThreads < last) reinterpret_cast<uint4 *>(tile)[v + i * kThreads] = w[i];
      },
      [&](int i) { tile[i] = ld(base + i); });
}

template <class T>
__device__ __forceinline__ void store_tile(const T *tile, T *array, int64_t from, int count) {
  constexpr int kVec = 16 / int(sizeof(T)), kBatch = 4;
  T *base = array + (from - from % kVec);
  flat<T>(
      from, count,
      [&](int v, int last) {
#pragma unroll
        for (int i = 0; i < kBatch; ++i)
          if (v + i * kThreads < last)
            reinterpret_cast<uint4 *>(base)[v + i * kThreads] = reinterpret_cast<const uint4 *>(tile)[v + i * kThreads];
      },
      [&](int i) { base[i] = tile[i]; });
}

// tile = array + other, rounded, and stored to `sum`.
template <class T>
__device__ __forceinline__ void load_sum(T *tile, const T *array, const T *other, T *sum, int64_t from, int count) {
  constexpr int kVec = 16 / int(sizeof(T)), kBatch = 4;
  const int64_t start = from - from % kVec;
  const T *a = array + start, *b = other + start;
  T *out = sum + start;
  flat<T>(
      from, count,
      [&](int v, int last) {
        uint4 p[kBatch], q[kBatch];
#pragma unroll
        for (int i = 0; i < kBatch; ++i)
          if (v + i * kThreads < last) {
            p[i] = ld(reinterpret_cast<const uint4 *>(a) + v + i * kThreads);
            q[i] = ld(reinterpret_cast<const uint4 *>(b) + v + i * kThreads);
          }
#pragma unroll
        for (int i = 0; i < kBatch; ++i) {
          if (v + i * kThreads >= last) continue;
          const uint32_t x[4] = {p[i].x, p[i].y, p[i].z, p[i].w}, y[4] = {q[i].x, q[i].y, q[i].z, q[i].w};
          uint32_t r[4];
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            if constexpr (sizeof(T) == 4) {
              r[j] = __float_as_uint(__uint_as_float(x[j]) + __uint_as_float(y[j]));
            } else {
              const __nv_bfloat162 s =
                  __floats2bfloat162_rn(__uint_as_float(x[j] << 16) + __uint_as_float(y[j] << 16),
                                        __uint_as_float(x[j] & 0xffff0000u) + __uint_as_float(y[j] & 0xffff0000u));
              r[j] = *reinterpret_cast<const uint32_t *>(&s);
            }
          }
          const uint4 w = make_uint4(r[0], r[1], r[2], r[3]);
          reinterpret_cast<uint4 *>(tile)[v + i * kThreads] = w;
          reinterpret_cast<uint4 *>(out)[v + i * kThreads] = w;
        }
      },
      [&](int i) {
        put(tile + i, get(a + i) + get(b + i));
        out[i] = tile[i];
      });
}

// The threads of a row: this one's row of the tile, its first column and their step.
struct Share {
  int row, rows_at_once, column, step, lanes, warps;
  float *slots;  // [2][kWarps]
  uint32_t turn = 0;
  __device__ __forceinline__ Share(const TilePlan &p, float *s) : lanes(p.lanes), warps(p.warps), slots(s) {
    const int warp = threadIdx.x / 32, lane = threadIdx.x & 31;
    row = warps > 1 ? warp / warps : warp * (32 / lanes) + lane / lanes;
    rows_at_once = warps > 1 ? kWarps / warps : kWarps * (32 / lanes);
    column = warps > 1 ? warp % warps * 32 + lane : lane & (lanes - 1);
    step = warps > 1 ? warps * 32 : lanes;
  }
  // Over the row, in all of its threads. All threads of the CTA call it (those without a row too).
  template <class Op>
  __device__ __forceinline__ float all(float v, Op op) {
    for (int o = lanes / 2; o > 0; o >>= 1) v = op(v, __shfl_xor_sync(kAll, v, o));
    if (warps == 1) return v;
    float *mine = slots + (turn++ & 1u) * kWarps;
    const int warp = threadIdx.x / 32, first = warp / warps * warps;
    if ((threadIdx.x & 31) == 0) mine[warp] = v;
    __syncthreads();
    v = mine[first];
    for (int i = 1; i < warps; ++i) v = op(v, mine[first + i]);
    return v;
  }
  __device__ __forceinline__ float sum(float v) {
    return all(v, [](float a, float b) { return a + b; });
  }
  __device__ __forceinline__ float max(float v) {
    return all(v, [](float a, float b) { return max_nan(a, b); });
  }
};

__device__ __forceinline__ uint8_t to8(float v) { return __nv_cvt_float_to_fp8(v, __NV_SATFINITE, __NV_E4M3); }

// A row in 8 bits to `out`, from its columns' values: blocks of kSize columns (0: the row) by a part of a warp or, of a
// row of several warps, one of them each. All threads of the CTA call it; those without a row write nothing.
template <int kSize, class Value>
__device__ __forceinline__ void quantise(Share &share, const NormFwd &a, int64_t row, bool real, uint8_t *out,
                                         Value value) {
  float inverse;
  if constexpr (kSize == 0) {
    float m = 0.f;
    for (int c = share.column; c < (real ? a.h : 0); c += share.step) m = max_nan(m, fabsf(value(c)));
    const float scale = scale_of(share.max(m), &inverse);
    if (real && share.column == 0) static_cast<float *>(a.scales)[row] = scale;
    for (int c = share.column; c < (real ? a.h : 0); c += share.step) out[c] = to8(value(c) * inverse);
  } else {
    const int lane = share.warps > 1 ? threadIdx.x & 31 : share.column, blocks = (a.h + kSize - 1) / kSize;
    const int first = share.warps > 1 ? threadIdx.x / 32 % share.warps : 0;
    const auto scale = [&](int b, float m, bool writes) {
      if (kSize == 32) {
        const uint32_t power = power_of(m, &inverse);
        if (writes) static_cast<uint8_t *>(a.scales)[row * blocks + b] = uint8_t(power);
      } else {
        const float f = scale_of(m, &inverse);
        if (writes) static_cast<float *>(a.scales)[row * blocks + b] = f;
      }
    };
    if (share.lanes == 32) {  // a warp's 128 columns at a time: four blocks of 32, or one, with their values in registers
      constexpr int kBlocks = 128 / kSize;
      for (int b0 = first * kBlocks; b0 < blocks; b0 += share.warps * kBlocks) {
        float v[4];
        uint32_t m[kBlocks] = {};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int c = b0 * kSize + i * 32 + lane;
          v[i] = real && c < a.h ? value(c) : 0.f;
          uint32_t &its = m[i * kBlocks / 4];
          its = max(its, __float_as_uint(v[i]) & 0x7fffffffu);  // (a NaN is the largest)
        }
#pragma unroll
        for (int i = 0; i < kBlocks; ++i) m[i] = __reduce_max_sync(kAll, m[i]);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int c = b0 * kSize + i * 32 + lane, b = b0 + i * kBlocks / 4;
          if (i % (4 / kBlocks) == 0) scale(b, __uint_as_float(m[i * kBlocks / 4]), real && lane == 0 && b < blocks);
          if (real && c < a.h) out[c] = to8(v[i] * inverse);
        }
      }
      return;
    }
    for (int b = 0; b < blocks; ++b) {
      const int end = !real ? 0 : (b + 1) * kSize < a.h ? (b + 1) * kSize : a.h;
      float m = 0.f;
#pragma unroll 4
      for (int c = b * kSize + lane; c < end; c += share.lanes) m = max_nan(m, fabsf(value(c)));
      for (int o = share.lanes / 2; o > 0; o >>= 1) m = max_nan(m, __shfl_xor_sync(kAll, m, o));
      scale(b, m, real && lane == 0);
#pragma unroll 4
      for (int c = b * kSize + lane; c < end; c += share.lanes) out[c] = to8(value(c) * inverse);
    }
  }
}

// Squares of a row: kLong, in two chains, of rows longer than 32 columns a thread (for all rows this took up to 4 % of a
// call); kTiny, with an eps below kSmall too.
enum Squares { kPlain, kLong, kTiny };

// Shared memory: the tile of the stream, then that of the 8-bit rows if there are any.
template <class T, Squares kSquares>
__global__ void __launch_bounds__(kThreads, 4) norm_fwd_tiles(const __grid_constant__ NormFwd a, bool w_bf16,
                                                           TilePlan plan) {
  grid_wait();
  extern __shared__ __align__(16) unsigned char shared[];
  __shared__ float slots[2 * kWarps];
  T *tile = reinterpret_cast<T *>(shared);
  uint8_t *tile8 = shared + plan.bytes;
  constexpr int kVec = 16 / int(sizeof(T));
  Share share(plan, slots);
  const float mean = 1.f / float(a.h);
  const int64_t tiles = (a.N + plan.rows - 1) / plan.rows;
  for (int64_t t = blockIdx.x; t < tiles; t += gridDim.x) {
    const int64_t row0 = t * plan.rows, from = row0 * a.h;
    const int rows = int(a.N - row0 < plan.rows ? a.N - row0 : plan.rows), count = rows * a.h;
    const T *x = static_cast<const T *>(a.x);
    if (a.residual)
      load_sum<T>(tile, x, static_cast<const T *>(a.residual), static_cast<T *>(a.sum), from, count);
    else
      load_tile<T>(tile, x, from, count);
    __syncthreads();
    T *first = tile + from % kVec;
    for (int r0 = 0; r0 < rows; r0 += share.rows_at_once) {
      const int r = r0 + share.row;
      const bool real = r < rows;
      T *row = first + (real ? r : 0) * a.h;
      const int end = real ? a.h : 0;
      const auto squares = [&](int c, int to, float by) {
        float s = 0.f;
#pragma unroll 4
        for (; c < to; c += share.step) {
          const float v = kSquares == kTiny ? get(row + c) * by : get(row + c);
          s = fmaf(v, v, s);
        }
        return s;
      };
      const auto all_squares = [&](float by) {
        if (kSquares == kPlain) return squares(share.column, end, by);
        const int half = 32 * share.step;
        return squares(share.column, end < half ? end : half, by) + squares(share.column + half, end, by);
      };
      const float square = fmaf(share.sum(all_squares(1.f)), mean, a.eps);
      float rstd = 1.f / sqrtf(square);
      if (kSquares == kTiny) {
        const bool small = real && square < kSmall;
        if (share.warps > 1 ? __syncthreads_or(small) : __any_sync(kAll, small)) {
          const float s = share.sum(all_squares(kUp));
          if (small) rstd = 1.f / sqrtf(fmaf(s, mean, a.eps * kUp * kUp)) * kUp;
        }
      }
      if (real && a.rstd && share.column == 0) a.rstd[row0 + r] = rstd;
      const auto value = [&](int c) { return get(row + c) * rstd * column_weight(a.weight, w_bf16, c); };
      if (a.y8) {
        uint8_t *out = tile8 + from % 16 + (real ? r : 0) * a.h;
        if (a.scaling == SAO_SCALE_ROW)
          quantise<0>(share, a, row0 + r, real, out, value);
        else if (a.scaling == SAO_SCALE_BLOCK128)
          quantise<128>(share, a, row0 + r, real, out, value);
        else
          quantise<32>(share, a, row0 + r, real, out, value);
        // y takes the place of the stream, which other threads of the row have read
        if (a.y) share.warps > 1 ? __syncthreads() : __syncwarp();
      }
      if (!real || !a.y) continue;
#pragma unroll 4
      for (int c = share.column; c < a.h; c += share.step) put(row + c, value(c));
    }
    __syncthreads();
    if (a.y) store_tile<T>(tile, static_cast<T *>(a.y), from, count);
    if (a.y8) store_tile<uint8_t>(tile8, a.y8, from, count);
    __syncthreads();
  }
}

// Rows shorter than kThreads. A CTA's sums for dw go to row blockIdx.x of `partial`. Shared memory: the tiles of the
// stream and of dy, then kThreads / h sums of each column for dw, then each row's rstd and factor of the stream.
template <class T>
__global__ void __launch_bounds__(kThreads, 4) norm_bwd_tiles(const __grid_constant__ NormBwd a, bool w_bf16,
                                                           TilePlan plan, float *partial) {
  grid_wait();
  extern __shared__ __align__(16) unsigned char shared[];
  __shared__ float slots[2 * kWarps];
  constexpr int kVec = 16 / int(sizeof(T));
  T *stream = reinterpret_cast<T *>(shared), *grad = reinterpret_cast<T *>(shared + plan.bytes);
  float *sums = reinterpret_cast<float *>(shared + 2 * plan.bytes);
  const int parts = kThreads / a.h;
  float *row_rstd = sums + kThreads, *row_c = row_rstd + plan.rows;
  Share share(plan, slots);
  const float mean = 1.f / float(a.h);
  for (int i = threadIdx.x; i < parts * a.h; i += kThreads) sums[i] = 0.f;
  for (int64_t row0 = int64_t(blockIdx.x) * plan.rows; row0 < a.N; row0 += int64_t(gridDim.x) * plan.rows) {
    const int64_t from = row0 * a.h;
    const int rows = int(a.N - row0 < plan.rows ? a.N - row0 : plan.rows), count = rows * a.h;
    load_tile<T>(stream, static_cast<const T *>(a.x), from, count);
    load_tile<T>(grad, static_cast<const T *>(a.dy), from, count);
    for (int r = threadIdx.x; r < rows; r += kThreads) row_rstd[r] = ld(a.rstd + row0 + r);
    __syncthreads();
    const T *x = stream + from % kVec;
    T *d = grad + from % kVec;
    for (int r0 = 0; r0 < rows; r0 += share.rows_at_once) {
      const int r = r0 + share.row;
      const bool real = r < rows;
      const int at = (real ? r : 0) * a.h;
      const float rstd = row_rstd[real ? r : 0];
      float s = 0.f;
#pragma unroll 4
      for (int c = share.column; c < (real ? a.h : 0); c += share.step)
        s = fmaf(get(d + at + c) * column_weight(a.weight, w_bf16, c), get(x + at + c) * rstd, s);
      s = share.sum(s);
      if (real && share.column == 0) row_c[r] = s * mean * rstd;  // times the stream and rstd, below
    }
    __syncthreads();
    if (partial != nullptr) {  // each thread its part of a column's rows
      const int part = threadIdx.x / a.h, c = threadIdx.x - part * a.h;
      if (part < parts) {
        float s = 0.f;
        for (int r = part; r < rows; r += parts)
          s = fmaf(get(d + r * a.h + c), get(x + r * a.h + c) * row_rstd[r], s);
        sums[threadIdx.x] += s;
      }
      __syncthreads();
    }
    const T *past = a.dsum ? static_cast<const T *>(a.dsum) + from : nullptr;
    for (int r0 = 0; r0 < rows; r0 += share.rows_at_once) {
      const int r = r0 + share.row;
      if (r >= rows) continue;
      const float rstd = row_rstd[r], f = row_c[r];
#pragma unroll 4
      for (int c = share.column; c < a.h; c += share.step) {
        const int at = r * a.h + c;
        const float v = rstd * fmaf(-f, get(x + at), get(d + at) * column_weight(a.weight, w_bf16, c));
        put(d + at, past ? v + get(past + at) : v);
      }
    }
    __syncthreads();
    store_tile<T>(grad, static_cast<T *>(a.dx), from, count);
    __syncthreads();
  }
  if (partial == nullptr) return;
  __syncthreads();
  for (int c = threadIdx.x; c < a.h; c += kThreads) {
    float s = sums[c];
    for (int p = 1; p < parts; ++p) s += sums[p * a.h + c];
    partial[int64_t(blockIdx.x) * a.h + c] = s;
  }
}

// Rows of a tile and how they are shared out. A tile has about 16 KB, or less to have two for each SM; from eight rows
// on a warp or less takes one.
TilePlan plan_of(int64_t N, int h, int size, int sms) {
  TilePlan p{1, 32, kWarps, 0};
  while (p.rows < 512 && 2 * p.rows * h * size <= (16 << 10) && 2 * p.rows * int64_t(sms) < N) p.rows *= 2;
  p.warps = p.rows >= kWarps ? 1 : kWarps / p.rows;
  while (p.lanes > 4 && p.lanes * 4 > h && p.rows >= kWarps * (64 / p.lanes)) p.lanes /= 2;
  p.bytes = (p.rows * h * size + 2 * 16 + 15) / 16 * 16;
  return p;
}

// Shared memory beyond 48 KB is asked for once on each device.
template <class T>
sao_status allow(int device, size_t most) {
  static PerDevice<cudaError_t> forward, backward;
  SAO_CUDA_TRY(forward.get(device, [&] {
    for (const auto kernel : {norm_fwd_tiles<T, kPlain>, norm_fwd_tiles<T, kLong>, norm_fwd_tiles<T, kTiny>}) {
      const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, int(most));
      if (e != cudaSuccess) return e;
    }
    return cudaSuccess;
  }));
  SAO_CUDA_TRY(backward.get(device, [&] {
    return cudaFuncSetAttribute(norm_bwd_tiles<T>, cudaFuncAttributeMaxDynamicSharedMemorySize, int(most));
  }));
  return SAO_OK;
}
constexpr size_t kMostShared = 200 << 10;

int ctas_of(size_t bytes, int most) {
  const int fit = int((220u << 10) / (bytes + 2048));
  return fit < 1 ? 1 : fit < most ? fit : most;
}

template <class T>
sao_status fwd(const NormFwd &a, bool w_bf16, const DeviceInfo &di, cudaStream_t s) {
  SAO_TRY(allow<T>(di.device, kMostShared));
  const TilePlan p = plan_of(a.N, a.h, sizeof(T), di.sm_count);
  const size_t bytes = p.bytes + (a.y8 ? size_t(p.rows) * a.h + 32 : 0);
  const int64_t tiles = (a.N + p.rows - 1) / p.rows, most = int64_t(di.sm_count) * 4 * ctas_of(bytes, 6);
  const int slot = launch_begin("norm_fwd", s);
  const auto kernel = a.eps < kSmall          ? norm_fwd_tiles<T, kTiny>
                      : a.h > 32 * kThreads ? norm_fwd_tiles<T, kLong>
                                            : norm_fwd_tiles<T, kPlain>;
  pdl(kernel, unsigned(tiles < most ? tiles : most), kThreads, bytes, s)(a, w_bf16, p);
  return launch_end(slot, s);
}

template <class T>
sao_status bwd(const NormBwd &a, bool w_bf16, const DeviceInfo &di, float *partial, int most, int *parts,
               cudaStream_t s) {
  SAO_TRY(allow<T>(di.device, kMostShared));
  const TilePlan p = plan_of(a.N, a.h, sizeof(T), di.sm_count);
  const size_t bytes = 2 * size_t(p.bytes) + sizeof(float) * (size_t(kThreads) + 2 * p.rows);
  const int64_t tiles = (a.N + p.rows - 1) / p.rows;
  *parts = int(tiles < most ? tiles : most);
  const int slot = launch_begin("norm_bwd", s);
  pdl(norm_bwd_tiles<T>, unsigned(*parts), kThreads, bytes, s)(a, w_bf16, p, a.dweight ? partial : nullptr);
  return launch_end(slot, s);
}

}  // namespace

sao_status norm_fwd_tiles_launch(const NormFwd &a, sao_dtype dt, sao_dtype w_dt, cudaStream_t s) {
  DeviceInfo di;
  SAO_TRY(device_info(&di));
  const bool w = w_dt == SAO_BF16;
  return dt == SAO_BF16 ? fwd<__nv_bfloat16>(a, w, di, s) : fwd<float>(a, w, di, s);
}
sao_status norm_bwd_tiles_launch(const NormBwd &a, sao_dtype dt, sao_dtype w_dt, float *partial, int most, int *parts,
                                 cudaStream_t s) {
  DeviceInfo di;
  SAO_TRY(device_info(&di));
  const bool w = w_dt == SAO_BF16;
  return dt == SAO_BF16 ? bwd<__nv_bfloat16>(a, w, di, partial, most, parts, s)
                        : bwd<float>(a, w, di, partial, most, parts, s);
}

}  // namespace sao
